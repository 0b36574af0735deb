"""The operators on a caller-owned paged cache against the float64 definitions of oracle/paged.py.

Tolerances.  u = 2^-24 (half a step of float32).  A score scale q.k is a sum of head_dim products: its error is at most
es = (head_dim + 2) u S with S = scale sum_d |q_d k_d|; the exponential (base 2, of a product with log2 e) adds
2^-21 + 2 u S relative, so a weight is off by at most ew = es + 2 u S + 2^-21, and its normalisation by the same again
plus the n u of a sum of n terms.  An output element sums n products weight * value: with A = sum_j w_j |v_j| it is off
by at most A (2 ew + 3 n u).  16-bit storage also rounds the unnormalised weights (half a step: 2^-8 relative, so
2^-8 A) and the output (2^-8 |o|).
"""
import numpy as np
import pytest
import torch

import paper_2601_19404_b200 as rpo
from oracle import paged
from gpu_util import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def contexts():
    made = {n: rpo.Context(rpo.shape_preset("tiny", dtype=1 if n == "bf16" else 0), kv_pool_blocks=8, max_groups=1, max_seqs=1,
                           max_chunk_tokens=16, max_positions=32) for n in DTYPES}
    yield made
    for c in made.values():
        c.close()


class Case:
    """Random chunk and cache; everything no row may depend on is NaN (behind the last token, unused blocks)."""

    def __init__(self, dtype, hq, hkv, dh, new, lens, seed=0, spread=1.5, extra_rows=0, window=0, sinks=0, bad=float("nan")):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.hq, self.hkv, self.dh, self.window, self.sinks = DTYPES[dtype], hq, hkv, dh, window, sinks
        self.new, self.lens, self.scale = list(new), list(lens), dh ** -0.5
        self.off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        rows = int(self.off[-1]) + extra_rows
        qkv = torch.randn(rows, hq + 2 * hkv, dh, generator=g)
        qkv[:, :hq] *= spread
        self.qkv = qkv.to(self.dtype).to(DEV)                            # fused projection: q, k, v are strided views
        self.q, self.k_new, self.v_new = self.qkv[:, :hq], self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:]
        pages = [-(-n // 16) for n in lens]
        width = max(pages + [1]) + 2
        n_blocks = sum(pages) + 3
        order = torch.randperm(n_blocks, generator=g).tolist()
        table = np.full((len(lens), width), -1, dtype=np.int32)
        k = torch.full((hkv, n_blocks, 16, dh), bad)
        v = torch.full((hkv, n_blocks, 16, dh), bad)
        for s, n in enumerate(lens):
            for p in range(pages[s]):
                b = table[s, p] = order.pop()
                live = min(16, n - 16 * p)
                k[:, b, :live] = torch.randn(hkv, live, dh, generator=g)
                v[:, b, :live] = torch.randn(hkv, live, dh, generator=g)
        self.table = table
        self.k, self.v = k.to(self.dtype).to(DEV), v.to(self.dtype).to(DEV)
        self.kv = rpo.PagedKV(self.k, self.v, torch.from_numpy(table).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV))
        self.d_off = torch.from_numpy(self.off).to(DEV)
        self.max_chunk = max(max(new), 1)

    def hide_pages(self):
        """Table entries and contents of pages that the window hides from every row are taken away."""
        for s, (n, c) in enumerate(zip(self.lens, self.new)):
            seen = paged.visible(c, n, self.window, self.sinks).any(0) if c else np.zeros(n, dtype=bool)
            for p in range(-(-n // 16)):
                if not seen[16 * p:16 * p + 16].any():
                    self.k[:, self.table[s, p]] = float("nan")
                    self.v[:, self.table[s, p]] = float("nan")
                    self.kv.d_block_table[s, p] = -1

    def np(self, t):
        return t.detach().float().cpu().numpy().astype(np.float64)

    def attend(self, ctx, append=False, lse=True):
        out = torch.full(self.q.shape, 7.0, dtype=self.dtype, device=DEV)
        d_lse = torch.full(self.q.shape[:2], 7.0, device=DEV) if lse else None
        ctx.chunk_attention(self.q, self.kv, self.d_off, self.max_chunk, out, d_lse, d_k_new=self.k_new if append else None,
                            d_v_new=self.v_new if append else None, window=self.window, sinks=self.sinks)
        torch.cuda.synchronize()
        return out, d_lse

    def attend_into(self, ctx, out):
        ctx.chunk_attention(self.q, self.kv, self.d_off, self.max_chunk, out, window=self.window, sinks=self.sinks)

    def errors(self):
        """Per row and head: (relative error of a weight, error of the log-sum, sum of |w v|) by the header's bounds."""
        q, k, v = self.np(self.q), np.nan_to_num(self.np(self.k)), np.nan_to_num(self.np(self.v))
        rows = q.shape[0]
        ew, el = np.zeros((rows, self.hq)), np.zeros((rows, self.hq))
        a = np.zeros((rows, self.hq, self.dh))
        rep = self.hq // self.hkv
        for s, n in enumerate(self.lens):
            lo, hi = self.off[s], self.off[s + 1]
            kk, vv = paged.token_rows(k, self.table[s], n), paged.token_rows(v, self.table[s], n)
            for h in range(self.hq):
                big = (self.scale * np.abs(q[lo:hi, h]) @ np.abs(kk[h // rep]).T).max(1, initial=0.0)
                ew[lo:hi, h] = (self.dh + 4) * U * big + 2.0 ** -21
                el[lo:hi, h] = ew[lo:hi, h] + n * U + 2.0 ** -22 * (big + 10)
                w, _ = paged._weights(q[lo:hi, h], kk[h // rep], self.scale, self.window, self.sinks)
                a[lo:hi, h] = w @ np.abs(vv[h // rep])
        return ew, el, a

    def check(self, out, lse):
        k, v = np.nan_to_num(self.np(self.k)), np.nan_to_num(self.np(self.v))
        want, want_lse = paged.chunk_attention(self.np(self.q), k, v, self.table, self.lens, self.off, self.scale, self.window, self.sinks)
        ew, el, a = self.errors()
        n, half = int(self.off[-1]), torch.finfo(self.dtype).eps / 2
        tol = a * (2 * ew + 3 * max(self.lens + [1]) * U)[..., None] + half * np.abs(want)
        if self.dtype == torch.bfloat16:
            tol += 2.0 ** -8 * a
        got = self.np(out)
        assert np.all(np.isfinite(got[:n]))
        assert np.all(np.abs(got[:n] - want[:n]) <= tol[:n] + 1e-30), np.max(np.abs(got[:n] - want[:n]) - tol[:n])
        assert np.all(got[n:] == 7.0)                                    # rows behind the last sequence
        if lse is not None:
            g = self.np(lse)
            empty = np.isneginf(want_lse[:n])
            assert np.array_equal(np.isneginf(g[:n]), empty)
            assert np.all(np.abs(g[:n][~empty] - want_lse[:n][~empty]) <= el[:n][~empty]) and np.all(g[n:] == 7.0)


# (new tokens, tokens in the cache): single tokens, chunks, empty sequences, chunks longer than their cache, ends of pages and tiles
STEPS = ([1, 1, 0, 1, 1, 1, 1], [1, 16, 40, 17, 0, 128, 333])
CHUNKS = ([1, 5, 0, 40, 16, 3, 129], [300, 5, 9, 35, 16, 129, 260])
LONG = ([300, 1], [700, 1030])
HEADS = [(4, 2, 64), (12, 2, 128), (7, 1, 64), (3, 3, 128), (28, 4, 128), (64, 1, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("rows", [STEPS, CHUNKS, LONG], ids=["steps", "chunks", "long"])
@pytest.mark.parametrize("mask", [(0, 0), (1, 0), (70, 0), (33, 5), (128, 200)])
def test_attention(contexts, dtype, heads, rows, mask):
    if rows is LONG and heads not in HEADS[:2] + HEADS[4:5]:
        pytest.skip("long chunks on three head layouts")
    c = Case(dtype, *heads, *rows, seed=sum(heads), extra_rows=2, window=mask[0], sinks=mask[1])
    c.check(*c.attend(contexts[dtype]))
    assert contexts[dtype].device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [STEPS, CHUNKS], ids=["steps", "chunks"])
def test_attention_does_not_use_hidden_pages(contexts, dtype, rows):
    c = Case(dtype, 12, 2, 128, *rows, seed=3, window=20, sinks=3)
    c.hide_pages()
    c.check(*c.attend(contexts[dtype]))
    assert contexts[dtype].device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [STEPS, CHUNKS], ids=["steps", "chunks"])
def test_attention_appends_the_chunk(contexts, dtype, rows):
    c = Case(dtype, 8, 4, 64, *rows, seed=5, extra_rows=1)
    k, v = c.np(c.k), c.np(c.v)
    for cache, new in ((k, c.k_new), (v, c.v_new)):
        paged.append(cache, c.np(new), c.table, c.lens, c.off)
    out, lse = c.attend(contexts[dtype], append=True)
    assert np.array_equal(c.np(c.k), k, equal_nan=True) and np.array_equal(c.np(c.v), v, equal_nan=True)
    c.check(out, lse)
    again, _ = c.attend(contexts[dtype], append=True, lse=False)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_on_one_long_sequence_and_on_many_short_ones(contexts, dtype):
    for rows in (([1], [20011]), ([2], [5003]), ([1] * 300, list(range(300))), ([40], [9000])):
        c = Case(dtype, 12, 2, 128, *rows, seed=8)
        out, lse = c.attend(contexts[dtype])
        c.check(out, lse)
        again, lse2 = c.attend(contexts[dtype])
        assert torch.equal(out, again) and torch.equal(lse, lse2)          # whatever the order in which the parts finish


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_with_single_keys_that_decide(contexts, dtype):
    """Scores spread over hundreds: the running maximum moves many times, late and by much."""
    for rows in (STEPS, CHUNKS, ([200], [2000])):
        c = Case(dtype, 4, 2, 64, *rows, seed=9, spread=60.0)
        c.check(*c.attend(contexts[dtype]))


def test_attention_on_another_stream_and_in_a_graph():
    s = torch.cuda.Stream()
    with rpo.Context(rpo.shape_preset("tiny", dtype=1), kv_pool_blocks=8, max_groups=1, max_seqs=1, max_chunk_tokens=16, max_positions=32,
                     stream=s) as ctx:
        for rows in (([1] * 5, [100, 3000, 20, 17, 1]), ([50, 1], [300, 200])):
            c = Case("bf16", 12, 2, 128, *rows, seed=4)
            torch.cuda.synchronize()
            out = torch.zeros(c.q.shape, dtype=c.dtype, device=DEV)
            lse = torch.zeros(c.q.shape[:2], device=DEV)
            mass = torch.zeros(len(c.lens), 2, 3001, device=DEV)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                ctx.chunk_attention(c.q, c.kv, c.d_off, c.max_chunk, out, lse, d_k_new=c.k_new, d_v_new=c.v_new)
                ctx.attention_mass(c.q, c.kv, c.d_off, c.max_chunk, lse, mass)
            torch.cuda.synchronize()
            paged_k = c.np(c.k)
            paged.append(paged_k, c.np(c.k_new), c.table, c.lens, c.off)
            for _ in range(2):
                with torch.cuda.stream(s):
                    graph.replay()
                torch.cuda.synchronize()
                assert np.array_equal(c.np(c.k), paged_k, equal_nan=True)
                c.check(out, lse)
                assert abs(mass.double().sum().item() - sum(c.new) * 12) < 1e-3 * sum(c.new) * 12
            # a longer cache of the same tables: the replay follows the lengths on the device
            c.kv.d_lens.copy_(torch.tensor([max(1, n - 1) for n in c.lens], dtype=torch.int32))
            c.lens = [max(1, n - 1) for n in c.lens]
            with torch.cuda.stream(s):
                graph.replay()
            torch.cuda.synchronize()
            c.check(out, lse)
            del graph
        assert ctx.device_status() == 0


FIRST_CALL = """
import torch, paper_2601_19404_b200 as rpo
s = torch.cuda.Stream()
for dt, code in ((torch.bfloat16, 1), (torch.float32, 0)):
    ctx = rpo.Context(rpo.shape_preset("tiny", dtype=code), kv_pool_blocks=8, max_groups=1, max_seqs=1, max_chunk_tokens=16, max_positions=32, stream=s)
    for n in (1, 90):
        k = torch.randn(2, 40, 16, 64, device="cuda").to(dt); v = torch.randn_like(k)
        lens = torch.full((2,), 300, dtype=torch.int32, device="cuda")
        kv = rpo.PagedKV(k, v, torch.arange(38, dtype=torch.int32, device="cuda").reshape(2, 19), lens)
        q = torch.randn(2 * n, 4, 64, device="cuda").to(dt); off = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
        out = torch.zeros_like(q); lse = torch.zeros(2 * n, 4, device="cuda"); mass = torch.zeros(2, 2, 304, device="cuda")
        pos = torch.arange(304, dtype=torch.int32, device="cuda").expand(2, 2, 304).contiguous()
        src = torch.zeros(2, 2, 64, dtype=torch.int32, device="cuda"); n_out = torch.zeros(2, dtype=torch.int32, device="cuda")
        m_out, p_out = torch.zeros(2, 2, 64, device="cuda"), torch.zeros(2, 2, 64, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ctx.chunk_attention(q, kv, off, n, out, lse)
            ctx.attention_mass(q, kv, off, n, lse, mass)
            ctx.evict_cache(kv, mass, pos, 64, n_out, src, m_out, p_out)
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.synchronize()
        assert abs(mass.double().sum().item() - 8 * n) < 1e-3 * n and n_out.tolist() == [64, 64]
        assert ctx.device_status() == 0
        del g
    ctx.close()
print("captured")
"""


def test_a_process_may_capture_its_first_calls():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("rows", [STEPS, CHUNKS, LONG], ids=["steps", "chunks", "long"])
@pytest.mark.parametrize("mask", [(0, 0), (33, 5), (128, 200)])
def test_mass(contexts, dtype, heads, rows, mask):
    if rows is LONG and heads not in HEADS[:2] + HEADS[4:5]:
        pytest.skip("long chunks on three head layouts")
    c = Case(dtype, *heads, *rows, seed=sum(heads) + 1, extra_rows=2, window=mask[0], sinks=mask[1])
    q, k = c.np(c.q), np.nan_to_num(c.np(c.k))
    slots = max(c.lens) + 5
    want = paged.attention_mass(q, k, c.table, c.lens, c.off, c.scale, slots, *mask)
    lse = np.zeros(q.shape[:2])
    lse[:] = paged.chunk_attention(q, k, k, c.table, c.lens, c.off, c.scale, *mask)[1]
    ew, _, _ = c.errors()
    d_lse = torch.from_numpy(lse.astype(np.float32)).to(DEV)
    start = torch.rand(len(c.lens), c.hkv, slots, generator=torch.Generator().manual_seed(1)).to(DEV)
    base = c.np(start)
    live = np.broadcast_to(np.arange(slots)[None, None] < np.array(c.lens)[:, None, None], base.shape)
    for given in (start, None):
        out = torch.full_like(start, 9.0)
        contexts[dtype].attention_mass(c.q, c.kv, c.d_off, c.max_chunk, d_lse, out, d_mass_in=given, window=mask[0], sinks=mask[1])
        torch.cuda.synchronize()
        got, full = c.np(out), want + (base if given is not None else 0.0)
        # every weight is off by ew and by the rounding of its lse; the sum of R of them, and the start, by their roundings
        n = max(c.new) * (c.hq // c.hkv)
        finite = lse[np.isfinite(lse)]
        rel = ew.max() + U * (np.abs(finite).max() if finite.size else 0.0) + 2.0 ** -20 + (n + 2) * U
        assert np.all(np.abs(got - full)[live] <= (rel * full + 1e-35)[live])
        assert np.all(got[~live] == 9.0)
    accumulated = start.clone()
    contexts[dtype].attention_mass(c.q, c.kv, c.d_off, c.max_chunk, d_lse, accumulated, d_mass_in=accumulated, window=mask[0], sinks=mask[1])
    torch.cuda.synchronize()
    got = c.np(accumulated)
    assert np.array_equal(got[~live], base[~live]) and np.all(np.abs(got - want - base)[live] <= (rel * (want + base) + 1e-35)[live])
    assert contexts[dtype].device_status() == 0


@pytest.mark.parametrize("heads,new,lens", [((8, 8, 64), [590, 60, 300, 1, 412], [640, 900, 300, 77, 5000]), ((64, 1, 128), [300], [2100]),
                                            ((12, 2, 128), [700, 233, 0, 5], [1500, 4000, 10, 2600])], ids=["narrow", "wide", "mixed"])
def test_calls_of_many_steps_repeat_bit_for_bit(contexts, heads, new, lens):
    """Hundreds of steps per CTA, again and again: hand-overs between the kernels' roles that only hold by luck would show as
    different bits, wrong sums or an expired wait."""
    ctx = contexts["bf16"]
    c = Case("bf16", *heads, new, lens, seed=21)
    first_out, lse = c.attend(ctx)
    first = None
    for _ in range(25):
        mass = torch.zeros(len(lens), heads[1], max(lens), device=DEV)
        ctx.attention_mass(c.q, c.kv, c.d_off, c.max_chunk, lse, mass)
        out, _ = c.attend(ctx, lse=False)
        assert torch.equal(out, first_out)
        if first is None:
            first = mass
        assert torch.equal(mass, first)
    assert ctx.device_status() == 0
    per_head = np.array(new) * (heads[0] // heads[1])
    assert np.allclose(first.double().sum(2).cpu().numpy(), per_head[:, None], rtol=1e-4)


EVICT = [([40, 9, 0, 33, 34, 100], 33, 2, 5, 41), ([1000, 1025, 1024, 31], 1024, 4, 200, 1030), ([5000, 2], 64, 3, 10, 5000), ([17, 40], 1, 0, 1, 64),
         ([200, 300], 16, 8, 8, 301), ([70000], 8191, 16, 500, 70001),
         ([1700, 300, 5] * 20, 600, 4, 60, 1701), ([3000] * 9 + [100] * 21, 1000, 2, 30, 3001), ([9000, 16000, 70] * 20, 41, 4, 20, 16001),
         ([20000] * 3 + [50] * 20, 3000, 8, 900, 20001)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("case", EVICT, ids=lambda c: f"{len(c[0])}x{max(c[0])}to{c[1]}")
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(contexts, dtype, dh, case, in_place):
    lens, budget, sinks, recent, slots = case
    hkv = 1 if max(lens) > 5000 or len(lens) > 10 else 3
    rng = np.random.default_rng(budget)
    c = Case(dtype, hkv, hkv, dh, [0] * len(lens), lens, seed=1, bad=0.5)
    mass = (np.round(rng.exponential(size=(len(lens), hkv, slots)) * 8) / 8).astype(np.float32)       # many ties
    mass[rng.random(mass.shape) < 0.02] = np.nan
    mass[rng.random(mass.shape) < 0.02] = -0.0
    mass[rng.random(mass.shape) < 0.01] = np.inf
    mass[rng.random(mass.shape) < 0.01] = -3.0
    pos = np.stack([np.stack([rng.permutation(slots) for _ in range(hkv)]) for _ in lens]).astype(np.int32)
    if budget % 2 == 0:
        pos[:] = np.arange(slots)
    d_mass, d_pos = torch.from_numpy(mass).to(DEV), torch.from_numpy(pos).to(DEV)
    lens_out = c.kv.d_lens if in_place else torch.full((len(lens),), -5, dtype=torch.int32, device=DEV)
    src = torch.full((len(lens), hkv, budget), -9, dtype=torch.int32, device=DEV)
    if in_place and budget <= slots:
        mass_out, pos_out = d_mass, d_pos
    else:
        mass_out = torch.full((len(lens), hkv, budget + 3), 7.0, device=DEV)
        pos_out = torch.full((len(lens), hkv, budget + 3), -7, dtype=torch.int32, device=DEV)
    k0, v0 = c.np(c.k), c.np(c.v)
    contexts[dtype].evict_cache(c.kv, d_mass, d_pos, budget, lens_out, src, mass_out, pos_out, sinks=sinks, recent=recent)
    torch.cuda.synchronize()
    k1, v1, got_src = c.np(c.k), c.np(c.v), src.cpu().numpy()
    got_mass, got_pos = mass_out.cpu().numpy(), pos_out.cpu().numpy()
    want_k, want_v = k0.copy(), v0.copy()
    assert lens_out.tolist() == [min(n, budget) for n in lens]
    for s, n in enumerate(lens):
        for h in range(hkv):
            want = paged.evict(mass[s, h, :n], pos[s, h, :n], budget, sinks, recent) if n else []
            m = len(want)
            assert got_src[s, h, :m].tolist() == want and np.all(got_src[s, h, m:] == -1)
            assert np.array_equal(got_mass[s, h, :m], mass[s, h, want], equal_nan=True) and np.array_equal(got_pos[s, h, :m], pos[s, h, want])
            if mass_out is d_mass:
                assert np.array_equal(got_mass[s, h, m:], mass[s, h, m:], equal_nan=True)
            else:
                assert np.all(got_mass[s, h, m:] == 7.0) and np.all(got_pos[s, h, m:] == -7)
            for i, f in enumerate(want):
                if f != i:
                    to, frm = (c.table[s, i // 16], i % 16), (c.table[s, f // 16], f % 16)
                    want_k[h][to], want_v[h][to] = k0[h][frm], v0[h][frm]
    assert np.array_equal(k1, want_k) and np.array_equal(v1, want_v)
    assert contexts[dtype].device_status() == (8 if max(lens) > slots else 0)            # tokens without a weight: clamped and reported


def test_evict_with_more_protected_slots_than_budget(contexts):
    """Positions that repeat protect more slots than sinks + recent: the heaviest of them stay."""
    c = Case("fp32", 1, 1, 64, [0], [50], seed=2, bad=0.0)
    mass = torch.arange(50, dtype=torch.float32).reshape(1, 1, 50).to(DEV)
    pos = torch.zeros(1, 1, 50, dtype=torch.int32, device=DEV)
    src = torch.zeros(1, 1, 8, dtype=torch.int32, device=DEV)
    out, pout, lens = torch.zeros(1, 1, 8, device=DEV), torch.zeros(1, 1, 8, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    contexts["fp32"].evict_cache(c.kv, mass, pos, 8, lens, src, out, pout, sinks=1, recent=0)
    torch.cuda.synchronize()
    assert src[0, 0].tolist() == list(range(42, 50)) and lens.item() == 8


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_bounded_rollout_of_chunks(contexts, dtype):
    """Append and attend, gather the weights, evict, go on: several chunks, against a simulation that keeps per-head lists."""
    ctx, dt = contexts[dtype], DTYPES[dtype]
    n, hq, hkv, dh, budget, width, sinks, recent = 3, 4, 2, 64, 48, 160, 2, 8
    g = torch.Generator().manual_seed(6)
    pages = width // 16
    table = torch.randperm(n * pages, generator=g).reshape(n, pages).to(torch.int32)
    k = torch.full((hkv, n * pages, 16, dh), float("nan"), dtype=dt, device=DEV)
    v = k.clone()
    lens = torch.zeros(n, dtype=torch.int32, device=DEV)
    kv = rpo.PagedKV(k, v, table.to(DEV), lens)
    mass, pos = torch.zeros(n, hkv, width, device=DEV), torch.zeros(n, hkv, width, dtype=torch.int32, device=DEV)
    src = torch.zeros(n, hkv, budget, dtype=torch.int32, device=DEV)
    ref = [[[] for _ in range(hkv)] for _ in range(n)]             # (position, key, value) per slot
    done = [0] * n
    for new in ([70, 1, 33], [1, 1, 1], [9, 100, 0], [1, 1, 1], [1, 1, 1], [30, 2, 17]):
        off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        rows = int(off[-1])
        x = torch.randn(rows, hq + 2 * hkv, dh, generator=g).to(dt)
        xf = x.double().numpy()
        before = lens.tolist()
        lens += torch.tensor(new, dtype=torch.int32, device=DEV)
        for s in range(n):
            for h in range(hkv):
                pos[s, h, before[s]:before[s] + new[s]] = torch.arange(done[s], done[s] + new[s], dtype=torch.int32)
                mass[s, h, before[s]:before[s] + new[s]] = 0.0
                ref[s][h] += [(done[s] + i, xf[off[s] + i, hq + h], xf[off[s] + i, hq + hkv + h]) for i in range(new[s])]
            done[s] += new[s]
        d = x.to(DEV)
        out, lse = torch.zeros(rows, hq, dh, dtype=dt, device=DEV), torch.zeros(rows, hq, device=DEV)
        d_off = torch.from_numpy(off).to(DEV)
        ctx.chunk_attention(d[:, :hq], kv, d_off, max(new), out, lse, d_k_new=d[:, hq:hq + hkv], d_v_new=d[:, hq + hkv:])
        ctx.attention_mass(d[:, :hq], kv, d_off, max(new), lse, mass, d_mass_in=mass)
        torch.cuda.synchronize()
        got, got_mass, at = out.double().cpu().numpy(), mass.cpu().numpy(), pos.cpu().numpy()
        for s in range(n):
            for h in range(hkv):
                kk, vv = np.array([r[1] for r in ref[s][h]]), np.array([r[2] for r in ref[s][h]])
                for j in range(2 * h, 2 * h + 2):
                    w, _ = paged._weights(xf[off[s]:off[s + 1], j], kk, dh ** -0.5, 0, 0)
                    a = w @ np.abs(vv)
                    half = torch.finfo(dt).eps / 2
                    # scores stay below 30 here, so a weight is off by less than 70 u 30 + 2^-21 (see the header)
                    tol = a * (2e-4 + (2.0 ** -8 if dt == torch.bfloat16 else 0)) + half * np.abs(w @ vv)
                    assert np.all(np.abs(got[off[s]:off[s + 1], j] - w @ vv) <= tol)
                assert at[s, h, :len(ref[s][h])].tolist() == [r[0] for r in ref[s][h]]
        ctx.evict_cache(kv, mass, pos, budget, lens, src, mass, pos, sinks=sinks, recent=recent)
        torch.cuda.synchronize()
        for s in range(n):
            for h in range(hkv):
                m = len(ref[s][h])
                order = paged.evict(got_mass[s, h, :m], at[s, h, :m], budget, sinks, recent)       # the library's own weights decide
                assert src[s, h, :len(order)].tolist() == order
                ref[s][h] = [ref[s][h][i] for i in order]
        assert lens.tolist() == [min(b + c, budget) for b, c in zip(before, new)]
    assert ctx.device_status() == 0


def test_bad_lengths_offsets_and_pages_are_reported_not_followed(contexts):
    """Bits 2 and 3 of the status word; neighbours of the bad sequence keep their results."""
    for dtype in DTYPES:
        ctx = contexts[dtype]
        for rows in (([1, 1, 1], [50, 60, 40]), ([20, 30, 10], [50, 60, 40])):
            for what in ("block", "length", "offset", "chunk"):
                c = Case(dtype, 4, 2, 64, *rows, seed=12, bad=0.0)
                good, good_lse = c.attend(ctx)
                assert ctx.device_status() == 0
                max_chunk, k = c.max_chunk, c.k.clone()
                if what == "block":
                    c.kv.d_block_table[1, 1] = c.k.shape[1] + 1000
                    c.kv.d_block_table[1, 2] = -77
                elif what == "length":
                    c.kv.d_lens[1] = 1 << 30
                elif what == "offset":
                    c.d_off[3] = 1 << 29
                else:
                    c.max_chunk -= 1
                    if c.max_chunk == 0:
                        continue
                out, lse = c.attend(ctx, append=what == "block")
                mass = torch.zeros(3, 2, 70, device=DEV)
                ctx.attention_mass(c.q, c.kv, c.d_off, c.max_chunk, good_lse, mass)
                word = ctx.device_status()
                assert word & (4 if what in ("block", "length") else 8), (what, word)
                if what != "chunk":
                    assert torch.equal(out[:rows[0][0]], good[:rows[0][0]]) or what == "block"
                if what == "block":
                    # the newest 32 of 50, 60 and 40 tokens stay: sequence 1 moves rows of both bad blocks
                    mass = torch.arange(70.0, device=DEV).expand(3, 2, 70).contiguous()
                    src = torch.zeros(3, 2, 32, dtype=torch.int32, device=DEV)
                    pos = torch.arange(70, dtype=torch.int32, device=DEV).expand(3, 2, 70).contiguous()
                    ctx.evict_cache(c.kv, mass, pos, 32, torch.zeros(3, dtype=torch.int32, device=DEV), src, torch.zeros(3, 2, 32, device=DEV),
                                    torch.zeros(3, 2, 32, dtype=torch.int32, device=DEV))
                    assert ctx.device_status() & 4
                c.max_chunk = max_chunk
        c = Case(dtype, 2, 2, 64, [1], [30], seed=1)
        c.attend(ctx)
        assert ctx.device_status() == 0                                   # nothing of it lingers


def test_refusals(contexts):
    ctx = contexts["bf16"]
    c = Case("bf16", 4, 2, 64, [3, 1], [20, 30], seed=1)
    out, lse = torch.zeros(4, 4, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(4, 4, device=DEV)

    def code(f, *a, **kw):
        with pytest.raises(rpo.RpoError) as e:
            f(*a, **kw)
        return e.value.code

    att = ctx.chunk_attention
    assert code(att, c.q, c.kv, c.d_off, 0, out) == -1 and code(att, c.q, c.kv, c.d_off, 3, out, scale=0.0) == -1
    assert code(att, c.q, c.kv, c.d_off, 3, out, scale=float("nan")) == -1 and code(att, c.q, c.kv, c.d_off, 3, out, window=-1) == -1
    assert code(att, c.q, c.kv, c.d_off, 3, out, sinks=-1) == -1
    q3 = torch.zeros(4, 3, 64, dtype=torch.bfloat16, device=DEV)
    assert code(att, q3, c.kv, c.d_off, 3, q3.clone()) == -2               # 3 query heads on 2 KV heads
    q130 = torch.zeros(4, 130, 64, dtype=torch.bfloat16, device=DEV)
    assert code(att, q130, c.kv, c.d_off, 3, q130.clone()) == -2           # 65 query heads per KV head
    shifted = torch.zeros(4 * 4 * 64 + 8, dtype=torch.bfloat16, device=DEV)[1:1 + 4 * 4 * 64].view(4, 4, 64)
    assert code(att, shifted, c.kv, c.d_off, 3, out) == -1                 # not 16-byte aligned
    assert code(att, c.q, c.kv, c.d_off, 3, shifted) == -1
    wide = torch.zeros(4, 4 * 64 + 4, dtype=torch.bfloat16, device=DEV)[:, :256].unflatten(1, (4, 64))
    assert code(att, wide, c.kv, c.d_off, 3, out) == -1                    # rows not 16-byte aligned
    mass, pos = torch.zeros(2, 2, 40, device=DEV), torch.zeros(2, 2, 40, dtype=torch.int32, device=DEV)
    src, lens = torch.zeros(2, 2, 8, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    ev = ctx.evict_cache
    assert code(ev, c.kv, mass, pos, 8, lens, src, mass[..., :8].contiguous(), pos[..., :8].contiguous(), sinks=5, recent=4) == -1
    assert code(ev, c.kv, mass, pos, 8, lens, src, mass[..., :4].contiguous(), pos[..., :4].contiguous()) == -1
    assert code(ev, c.kv, mass, pos, 8, lens, src, mass, pos, sinks=-1) == -1
    dh32 = torch.zeros(2, 4, 16, 32, dtype=torch.bfloat16, device=DEV)
    kv32 = rpo.PagedKV(dh32, dh32.clone(), c.kv.d_block_table, c.kv.d_lens)
    q32 = torch.zeros(4, 4, 32, dtype=torch.bfloat16, device=DEV)
    assert code(att, q32, kv32, c.d_off, 3, q32.clone()) == -2
    assert code(ctx.attention_mass, q32, kv32, c.d_off, 3, lse, mass) == -2
    # no rows at all: nothing to attend, every weight stays
    none, zero = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    att(none, c.kv, zero, 3, none.clone(), lse[:0])
    start, got = torch.rand(2, 2, 40, device=DEV), torch.full((2, 2, 40), 5.0, device=DEV)
    ctx.attention_mass(none, c.kv, zero, 3, lse[:0], got, d_mass_in=start)
    torch.cuda.synchronize()
    assert torch.equal(got[0, :, :20], start[0, :, :20]) and torch.equal(got[1, :, :30], start[1, :, :30])
    assert torch.all(got[0, :, 20:] == 5.0) and torch.all(got[1, :, 30:] == 5.0)
    assert ctx.device_status() == 0


def test_windows_and_sinks_beyond_every_position(contexts):
    """Far beyond the cache they change nothing."""
    for rows in (STEPS, CHUNKS):
        c = Case("bf16", 4, 2, 64, *rows, seed=14)
        _, lse = c.attend(contexts["bf16"])
        for c.window, c.sinks in ((2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 31 - 1)):
            c.check(*c.attend(contexts["bf16"]))
            mass, same = torch.zeros(7, 2, 400, device=DEV), torch.zeros(7, 2, 400, device=DEV)
            contexts["bf16"].attention_mass(c.q, c.kv, c.d_off, c.max_chunk, lse, mass, window=c.window, sinks=c.sinks)
            contexts["bf16"].attention_mass(c.q, c.kv, c.d_off, c.max_chunk, lse, same)
            # (the same weights, added up in the same tiles)
            assert torch.allclose(mass, same, rtol=1e-5, atol=1e-30)
    assert contexts["bf16"].device_status() == 0


def test_two_contexts_at_once():
    """Contexts own their workspaces: calls on two of them may overlap on the GPU."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ctx = [rpo.Context(rpo.shape_preset("tiny", dtype=1), kv_pool_blocks=8, max_groups=1, max_seqs=1, max_chunk_tokens=16, max_positions=32, stream=s)
           for s in streams]
    cases = [Case("bf16", 12, 2, 128, [200, 3], [3000, 900], seed=31), Case("bf16", 12, 2, 128, [150, 90], [1000, 4000], seed=32)]
    want = [c.attend(ctx[0])[0] for c in cases]
    out = [[torch.zeros_like(w) for _ in range(10)] for w in want]
    torch.cuda.synchronize()
    for i in range(10):
        for k in (0, 1):
            cases[k].attend_into(ctx[k], out[k][i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[k]) for k in (0, 1) for o in out[k])
    for x in ctx:
        assert x.device_status() == 0
        x.close()
