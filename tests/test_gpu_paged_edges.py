"""The operators on a caller-owned paged cache at the edges of what the header allows; tolerances as derived in
test_gpu_paged_ops.py."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2601_19404_b200 as rpo
from gpu_util import DEV
from oracle import paged
from test_gpu_paged_ops import CHUNKS, LONG, STEPS, U, Case, contexts  # noqa: F401

pytestmark = pytest.mark.gpu


def check_mass(ctx, c, slots, in_place=False):
    """attention_mass of a Case against the definition, on log-sums of the definition; entries behind a sequence stay."""
    q, k = c.np(c.q), np.nan_to_num(c.np(c.k))
    mask = (c.window, c.sinks)
    want = paged.attention_mass(q, k, c.table, c.lens, c.off, c.scale, slots, *mask)
    lse = paged.chunk_attention(q, k, k, c.table, c.lens, c.off, c.scale, *mask)[1]
    ew, _, _ = c.errors()
    start = torch.rand(len(c.lens), c.hkv, slots, generator=torch.Generator().manual_seed(1)).to(DEV)
    base = c.np(start)
    live = np.broadcast_to(np.arange(slots)[None, None] < np.array(c.lens)[:, None, None], base.shape)
    out = start.clone() if in_place else torch.full_like(start, 9.0)
    ctx.attention_mass(c.q, c.kv, c.d_off, c.max_chunk, torch.from_numpy(lse.astype(np.float32)).to(DEV), out,
                       d_mass_in=out if in_place else start, window=c.window, sinks=c.sinks)
    torch.cuda.synchronize()
    got, full = c.np(out), want + base
    n = max(c.new) * (c.hq // c.hkv)
    finite = lse[np.isfinite(lse)]
    rel = ew.max() + U * (np.abs(finite).max() if finite.size else 0.0) + 2.0 ** -20 + (n + 2) * U
    assert np.all(np.abs(got - full)[live] <= (rel * full + 1e-35)[live])
    assert np.array_equal(got[~live], base[~live] if in_place else np.full_like(got[~live], 9.0))
    assert ctx.device_status() == 0


@pytest.mark.parametrize("new,sinks", [([1] * 64, 3), ([2] * 32 + [0] * 32, 70), ([0] * 40 + [9] * 24, 0)], ids=["steps", "sinks", "empty"])
def test_32_bit_mass_goes_from_unseen_to_seen_keys(contexts, new, sinks):  # noqa: F811
    """More tiles of keys than CTAs per (sequence, KV head): a CTA takes tiles that no row sees (between sinks and window, or
    of a sequence without rows) before tiles that some row sees, in the same shared memory."""
    c = Case("fp32", 8, 8, 64, new, [1200 + 13 * (s % 7) for s in range(64)], seed=41, window=150, sinks=sinks)
    c.hide_pages()
    check_mass(contexts["fp32"], c, 1300)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 100], ids=["step", "chunk"])
def test_large_values_behind_growing_scores(contexts, dtype, new):  # noqa: F811
    """Values of 1e33 whose scores are 22 higher than those of the first keys, and than each other's 64 keys on: the sums stay
    within what weights of about 1 give."""
    c = Case(dtype, 4, 2, 64, [new, new], [1100, 801], seed=43)
    c.q.mul_(0.02)
    c.q[..., 0] = 8.0                                                     # a score is about the key's first element
    c.v.mul_(1e33)
    for s, n in enumerate(c.lens):
        at = torch.arange(n, device=DEV)
        page = torch.from_numpy(c.table[s]).to(DEV).long()[at // 16]
        c.k[:, page, at % 16, 0] = torch.where(at < 300, 0.0, torch.where(at < 700, 22.0, 22.0 + (at - 700) // 64)).to(c.dtype)
    c.check(*c.attend(contexts[dtype]))
    assert contexts[dtype].device_status() == 0


FIRST_CALLS = """
import threading, torch, paper_2601_19404_b200 as rpo
N = 4
streams = [torch.cuda.Stream() for _ in range(N)]
ctx = [rpo.Context(rpo.shape_preset("tiny", dtype=1), kv_pool_blocks=8, max_groups=1, max_seqs=1, max_chunk_tokens=16, max_positions=32, stream=s)
       for s in streams]
work = []
for i in range(N):
    k = torch.randn(2, 40, 16, 128, device="cuda").bfloat16()
    lens = torch.full((2,), 300, dtype=torch.int32, device="cuda")
    kv = rpo.PagedKV(k, torch.randn_like(k), torch.arange(38, dtype=torch.int32, device="cuda").reshape(2, 19), lens)
    for n in (1, 6, 90):                                       # a kernel of its own for each
        q = torch.randn(2 * n, 8, 128, device="cuda").bfloat16(); off = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
        work.append((i, n, q, kv, off, torch.zeros_like(q), torch.zeros(2 * n, 8, device="cuda"), torch.zeros(2, 2, 304, device="cuda")))
torch.cuda.synchronize()
gate, failed = threading.Barrier(N), []
def run(i):
    try:
        for j, n, q, kv, off, out, lse, mass in work:
            if j == i:
                gate.wait()
                ctx[i].chunk_attention(q, kv, off, n, out, lse)
                gate.wait()
                ctx[i].attention_mass(q, kv, off, n, lse, mass)
    except Exception as e:
        failed.append(repr(e)); gate.abort()
threads = [threading.Thread(target=run, args=(i,)) for i in range(N)]
[t.start() for t in threads]; [t.join() for t in threads]
torch.cuda.synchronize()
assert not failed, failed
for j, n, q, kv, off, out, lse, mass in work:
    assert abs(mass.double().sum().item() - 16 * n) < 1e-3 * n, (j, n)
assert all(c.device_status() == 0 for c in ctx)
print("all done")
"""


def test_first_calls_from_several_threads():
    """Contexts of several host threads, whose first launches of every kernel in the process come at once."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "all done" in r.stdout, r.stdout + r.stderr[-2000:]


@pytest.mark.parametrize("rows", [1 << 18, (1 << 18) + 64])
def test_the_largest_number_of_rows(contexts, rows):  # noqa: F811
    """2^18 rows of 4096 sequences fit, in 32 bits with 64 query heads on a KV head too, where every row is an item; more
    rows do not, and nothing is written.  Under a window of one token a row's output is its own value."""
    n, hq, dh = 4096, 64, 64
    new = [64] * n
    new[0] += rows - (1 << 18)
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
    k = torch.zeros(1, n * 8, 16, dh, device=DEV)
    kv = rpo.PagedKV(k, torch.zeros_like(k), torch.arange(n * 8, dtype=torch.int32, device=DEV).reshape(n, 8), torch.tensor(new, dtype=torch.int32, device=DEV))
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    q = torch.randn(rows, hq, dh, generator=g, device=DEV)
    k_new, v_new = torch.randn(rows, 1, dh, generator=g, device=DEV), torch.randn(rows, 1, dh, generator=g, device=DEV)
    out, ctx = torch.full_like(q, 7.0), contexts["fp32"]
    call = lambda: ctx.chunk_attention(q, kv, off, max(new), out, d_k_new=k_new, d_v_new=v_new, window=1)  # noqa: E731
    if rows > 1 << 18:
        with pytest.raises(rpo.RpoError) as e:
            call()
        assert e.value.code == -7
    else:
        call()
    torch.cuda.synchronize()
    assert bool((out == (7.0 if rows > 1 << 18 else v_new)).all()) and ctx.device_status() == 0


FEW = [((28, 4, 128), [4, 1, 0, 3, 4, 4, 2, 4], [300, 16, 40, 2, 17, 128, 18, 5003]), ((8, 1, 64), [3, 4, 0, 4, 1, 2], [50, 4, 9, 33, 0, 700]),
       ((4, 2, 64), [16, 9, 13, 2, 16], [200, 9, 7, 65, 1000]), ((12, 2, 128), [5, 5, 1, 4], [36, 3, 17, 260]), ((32, 1, 64), [1, 1, 0, 1], [77, 16, 3, 1030])]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("few", FEW, ids=lambda f: "x".join(map(str, f[0])))
@pytest.mark.parametrize("mask", [(0, 0), (1, 0), (3, 0), (70, 0), (33, 5), (20, 40)])
def test_a_few_tokens_per_step(contexts, dtype, few, mask):  # noqa: F811
    """17 to 32 rows per sequence and KV head: chunks over two pages, longer than their cache, written to it by the same call."""
    heads, new, lens = few
    c = Case(dtype, *heads, new, lens, seed=heads[0], extra_rows=2, window=mask[0], sinks=mask[1])
    k, v = c.np(c.k), c.np(c.v)
    for cache, fresh in ((k, c.k_new), (v, c.v_new)):
        paged.append(cache, c.np(fresh), c.table, c.lens, c.off)
    out, lse = c.attend(contexts[dtype], append=True)
    assert np.array_equal(c.np(c.k), k, equal_nan=True) and np.array_equal(c.np(c.v), v, equal_nan=True)
    c.check(out, lse)
    again, lse2 = c.attend(contexts[dtype])
    assert torch.equal(out, again) and torch.equal(lse, lse2)              # the same values, read from the cache now
    c.hide_pages()
    c.check(*c.attend(contexts[dtype]))
    check_mass(contexts[dtype], c, max(lens) + 3)
    check_mass(contexts[dtype], c, max(lens) + 3, in_place=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads", [(12, 2, 128), (3, 3, 64)])
@pytest.mark.parametrize("rows", [STEPS, CHUNKS, LONG], ids=["steps", "chunks", "long"])
@pytest.mark.parametrize("mask", [(20, 3), (100, 0)])
def test_mass_does_not_use_hidden_pages(contexts, dtype, heads, rows, mask):  # noqa: F811
    c = Case(dtype, *heads, *rows, seed=3, window=mask[0], sinks=mask[1])
    c.hide_pages()
    for in_place in (False, True):
        check_mass(contexts[dtype], c, max(c.lens) + 5, in_place)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [[1] * 6, [3, 1, 4, 0, 2, 4], [40, 1, 129, 9, 0, 33]], ids=["steps", "few", "chunks"])
def test_sequences_that_share_blocks(contexts, dtype, new):  # noqa: F811
    """Continuations of one prefix: the prefix' whole pages are the same blocks, what is written lies behind them."""
    lens = [160 + n + 7 * s for s, n in enumerate(new)]
    c = Case(dtype, 12, 2, 128, new, lens, seed=51)
    c.table[1:, :10] = c.table[0, :10]
    c.kv.d_block_table.copy_(torch.from_numpy(c.table))
    out, lse = c.attend(contexts[dtype], append=True)
    c.check(out, lse)
    check_mass(contexts[dtype], c, max(lens))


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("fp32", 64)])
def test_a_pool_beyond_32_bit_offsets(contexts, dtype, dh):  # noqa: F811
    """Blocks whose elements lie behind 2^31 of their KV head (and behind 2^32 bytes)."""
    for new, lens in (([1, 1, 0], [100, 2000, 30]), ([4, 2, 3], [100, 500, 30]), ([90, 1, 33], [500, 100, 200])):
        c = Case(dtype, 4, 2, dh, new, lens, seed=61)
        used, blocks = c.k.shape[1], (1 << 31) // (16 * dh) + 64
        pools = []
        for cache in (c.k, c.v):
            pool = torch.empty(2, blocks, 16, dh, dtype=c.dtype, device=DEV)
            pool[:, blocks - used:] = cache
            pools.append(pool)
        table = np.where(c.table >= 0, c.table + blocks - used, c.table)
        small, c.kv = c.kv, rpo.PagedKV(*pools, torch.from_numpy(table.astype(np.int32)).to(DEV), c.kv.d_lens)
        out, lse = c.attend(contexts[dtype], append=True)
        c.k, c.v = pools[0][:, blocks - used:], pools[1][:, blocks - used:]
        c.check(out, lse)
        check_mass(contexts[dtype], c, max(lens))
        # the same eviction in the large pool and in a small one
        small = rpo.PagedKV(c.k.contiguous(), c.v.contiguous(), small.d_block_table, small.d_lens)
        mass = torch.rand(len(lens), 2, max(lens), generator=torch.Generator().manual_seed(2)).to(DEV)
        pos = torch.arange(max(lens), dtype=torch.int32, device=DEV).expand(len(lens), 2, max(lens)).contiguous()
        for kv in (c.kv, small):
            src, out = torch.zeros(len(lens), 2, 40, dtype=torch.int32, device=DEV), torch.zeros(len(lens), 2, 40, device=DEV)
            contexts[dtype].evict_cache(kv, mass, pos, 40, torch.zeros_like(c.kv.d_lens), src, out, torch.zeros_like(src), recent=3)
        torch.cuda.synchronize()
        for a, b in ((c.k, small.d_k), (c.v, small.d_v)):
            assert torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float()))
        assert contexts[dtype].device_status() == 0
        del c, small, pools, pool
        torch.cuda.empty_cache()


def evict_src(mass, pos, budget, sinks, recent):
    """oracle.paged.evict for long caches: the slot each kept slot's row comes from."""
    n = len(mass)
    if n <= budget:
        return np.arange(n)
    safe, nan = (pos < sinks) | (pos > int(pos.max()) - recent), np.isnan(mass)
    kept = np.sort(np.lexsort((np.arange(n), np.where(nan, 0.0, -mass), nan, ~safe))[:budget])
    src = np.arange(budget)
    holes = np.ones(budget, dtype=bool)
    holes[kept[kept < budget]] = False
    src[holes] = kept[kept >= budget]
    return src


def test_the_long_reference_is_the_oracle():
    rng = np.random.default_rng(3)
    for n, budget, sinks, recent in ((40, 17, 2, 5), (9, 9, 0, 0), (300, 20, 8, 12), (64, 63, 0, 0)):
        mass = np.round(rng.exponential(size=n) * 4) / 4
        mass[rng.random(n) < 0.1] = np.nan
        pos = rng.permutation(n) if n % 2 else np.zeros(n, dtype=int)
        assert evict_src(mass, pos, budget, sinks, recent).tolist() == paged.evict(mass, pos, budget, sinks, recent)


# (lengths, budget, sinks, recent, slots of the arrays): counts of caches and slots at which the CTAs of a cache, their threads and
# the slots in registers change; the longest arrays, with as many moved slots as there can be
EVICT = [([4000, 70, 2500] * 27, 900, 4, 60, 4001), ([8192, 8191, 30] * 16, 2000, 0, 0, 8192), ([2049, 5000] * 10, 2048, 3, 9, 6001),
         ([9000, 10, 16384] * 27, 41, 4, 20, 16384), ([12000, 300] * 20, 5000, 16, 100, 12001), ([131072, 9], 60000, 4, 100, 131072),
         ([131073, 500], 65536, 4, 1000, 131073), ([200001], 1, 0, 1, 262147), ([1 << 19], 1 << 18, 16, 5000, 1 << 19),
         ([(1 << 19) - 3, 1 << 19], (1 << 19) - 4, 0, 0, 1 << 19)]


@pytest.mark.parametrize("case", EVICT, ids=lambda c: f"{len(c[0])}x{max(c[0])}to{c[1]}")
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_over_the_range_of_sizes(contexts, case, in_place):  # noqa: F811
    lens, budget, sinks, recent, slots = case
    rng = np.random.default_rng(slots)
    n, shape = len(lens), (len(lens), 1, slots)
    pages = [-(-x // 16) for x in lens]
    table = np.full((n, max(pages) + 1), -1, dtype=np.int32)
    order, at = rng.permutation(sum(pages)).astype(np.int32), 0
    for s, p in enumerate(pages):
        table[s, :p], at = order[at:at + p], at + p
    g = torch.Generator(device=DEV)
    g.manual_seed(slots)
    k = torch.randn(1, sum(pages), 16, 64, generator=g, device=DEV).bfloat16()
    v = torch.randn(1, sum(pages), 16, 64, generator=g, device=DEV).bfloat16()
    d_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    kv = rpo.PagedKV(k, v, torch.from_numpy(table).to(DEV), d_lens)
    mass = (np.round(rng.exponential(size=shape) * 8) / 8).astype(np.float32)                         # many ties
    mass[rng.random(shape) < 0.02] = np.nan
    mass[rng.random(shape) < 0.02] = -0.0
    mass[rng.random(shape) < 0.01] = np.inf
    # the heavy ones lie at the end: every hole below the budget is filled from behind it
    mass[:, :, slots // 2:] += 100.0
    pos = np.stack([rng.permutation(slots) for _ in lens])[:, None].astype(np.int32)
    if len(lens) % 2:
        pos[:] = np.arange(slots)
    d_mass, d_pos = torch.from_numpy(mass).to(DEV), torch.from_numpy(pos).to(DEV)
    k0, v0 = k.clone(), v.clone()
    src = torch.full((n, 1, budget), -9, dtype=torch.int32, device=DEV)
    lens_out = d_lens if in_place else torch.full_like(d_lens, -5)
    mass_out = d_mass if in_place else torch.full((n, 1, budget + 3), 7.0, device=DEV)
    pos_out = d_pos if in_place else torch.full((n, 1, budget + 3), -7, dtype=torch.int32, device=DEV)
    contexts["bf16"].evict_cache(kv, d_mass, d_pos, budget, lens_out, src, mass_out, pos_out, sinks=sinks, recent=recent)
    torch.cuda.synchronize()
    got_src, got_mass, got_pos = src.cpu().numpy(), mass_out.cpu().numpy(), pos_out.cpu().numpy()
    assert lens_out.tolist() == [min(x, budget) for x in lens]
    want_k, want_v = k0.clone().view(-1, 64), v0.clone().view(-1, 64)
    for s, x in enumerate(lens):
        want = evict_src(mass[s, 0, :x], pos[s, 0, :x], budget, sinks, recent)
        m = len(want)
        assert np.array_equal(got_src[s, 0, :m], want) and np.all(got_src[s, 0, m:] == -1)
        assert np.array_equal(got_mass[s, 0, :m], mass[s, 0, want], equal_nan=True) and np.array_equal(got_pos[s, 0, :m], pos[s, 0, want])
        assert np.array_equal(got_mass[s, 0, m:], mass[s, 0, m:], equal_nan=True) if in_place else np.all(got_mass[s, 0, m:] == 7.0)
        assert np.array_equal(got_pos[s, 0, m:], pos[s, 0, m:]) if in_place else np.all(got_pos[s, 0, m:] == -7)
        to = np.nonzero(want != np.arange(m))[0]
        row = lambda i: torch.from_numpy(table[s, i // 16].astype(np.int64) * 16 + i % 16).to(DEV)  # noqa: E731
        want_k[row(to)], want_v[row(to)] = k0.view(-1, 64)[row(want[to])], v0.view(-1, 64)[row(want[to])]
    assert torch.equal(k.view(-1, 64), want_k) and torch.equal(v.view(-1, 64), want_v)
    assert contexts["bf16"].device_status() == 0


def test_evict_refuses_longer_arrays(contexts):  # noqa: F811
    kv = rpo.PagedKV(torch.zeros(1, 2, 16, 64, device=DEV), torch.zeros(1, 2, 16, 64, device=DEV), torch.zeros(1, 2, dtype=torch.int32, device=DEV),
                     torch.full((1,), 20, dtype=torch.int32, device=DEV))
    mass, pos = torch.zeros(1, 1, (1 << 19) + 1, device=DEV), torch.zeros(1, 1, (1 << 19) + 1, dtype=torch.int32, device=DEV)
    src, n = torch.zeros(1, 1, 8, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    with pytest.raises(rpo.RpoError) as e:
        contexts["fp32"].evict_cache(kv, mass, pos, 8, n, src, mass, pos)
    assert e.value.code == -7


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [([1, 1, 1], [50, 60, 40]), ([4, 3, 2], [50, 60, 40]), ([20, 30, 10], [50, 60, 40])], ids=["steps", "few", "chunks"])
@pytest.mark.parametrize("what", ["block", "length", "negative length", "offset", "backward offsets", "chunk"])
def test_a_bad_sequence_is_reported_and_leaves_its_neighbours_alone(contexts, dtype, rows, what):  # noqa: F811
    ctx = contexts[dtype]
    c = Case(dtype, 8, 2, 64, *rows, seed=12, bad=0.0)
    good, good_lse = c.attend(ctx, append=True)
    slots = 128                                                            # more than the table can name: nothing is cut there
    start = torch.rand(3, 2, slots, device=DEV)
    good_mass = start.clone()
    ctx.attention_mass(c.q, c.kv, c.d_off, c.max_chunk, good_lse, good_mass, d_mass_in=good_mass)
    assert ctx.device_status() == 0
    k0 = c.k.clone()
    if what == "block":
        c.kv.d_block_table[1, 1] = c.k.shape[1] + 1000
        c.kv.d_block_table[1, 2] = -77
    elif what == "length":
        c.kv.d_lens[1] = 1 << 30
    elif what == "negative length":
        c.kv.d_lens[1] = -3
    elif what == "offset":
        c.d_off[3] = 1 << 29
    elif what == "backward offsets":
        c.d_off[1:3] = torch.tensor([rows[0][0] + 1, rows[0][0]], dtype=torch.int32)
    elif c.max_chunk == 1:
        return
    else:
        c.max_chunk = max(rows[0]) - 1
    bit = 4 if what == "block" else 8
    out, lse = c.attend(ctx, append=what not in ("length", "backward offsets"))
    assert ctx.device_status() & bit
    mass = start.clone()
    ctx.attention_mass(c.q, c.kv, c.d_off, c.max_chunk, good_lse, mass, d_mass_in=mass)
    assert ctx.device_status() & bit
    torch.cuda.synchronize()
    # the neighbours.  Where the lengths stay, so does the division of the work: bit for bit.  Elsewhere pieces may end at
    # other pages, and both results lie within the tolerances of the definition
    want, want_lse = paged.chunk_attention(c.np(c.q), c.np(k0), np.nan_to_num(c.np(c.v)), c.table, c.lens, c.off, c.scale)
    ew, el, a = c.errors()
    tol = a * (2 * ew + 3 * max(c.lens) * U)[..., None] + torch.finfo(c.dtype).eps / 2 * np.abs(want) + (2.0 ** -8 * a if dtype == "bf16" else 0)
    for s in (0, 2):
        if (what, s) in (("backward offsets", 0), ("backward offsets", 2)) or (what == "chunk" and rows[0][s] > c.max_chunk):
            continue                                                       # its own rows are others now
        r = slice(c.off[s], c.off[s + 1])
        if what in ("block", "offset"):
            assert torch.equal(out[r], good[r]) and torch.equal(lse[r], good_lse[r]) and torch.equal(mass[s], good_mass[s])
        assert np.all(np.abs(c.np(out)[r] - want[r]) <= tol[r]) and np.all(np.abs(c.np(lse)[r] - want_lse[r]) <= el[r])
        m, n = c.np(mass)[s], c.lens[s]
        # both sums are off by the weights' errors and their own roundings
        terms = rows[0][s] * 4
        rel = ew.max() + U * np.abs(want_lse).max() + 2.0 ** -20 + (terms + 2) * U
        assert np.all(np.abs(m - c.np(good_mass)[s])[:, :n] <= 2 * rel * m[:, :n]) and np.array_equal(m[:, n:], c.np(start)[s][:, n:])
    # nothing of the other sequences' keys was written
    for s in (0, 2):
        mine = torch.from_numpy(c.table[s, :-(-c.lens[s] // 16)].astype(np.int64)).to(DEV)
        if what not in ("chunk",):
            assert torch.equal(c.k[:, mine], k0[:, mine])


def test_layers_that_share_their_lengths(contexts):  # noqa: F811
    """Every layer evicts from the same lengths; the last call writes them in place."""
    lens, budget, n = torch.tensor([50, 20, 33], dtype=torch.int32, device=DEV), 24, 3
    table = torch.arange(12, dtype=torch.int32, device=DEV).reshape(3, 4)
    pos = torch.arange(64, dtype=torch.int32, device=DEV).expand(n, 2, 64).contiguous()
    scratch = torch.zeros_like(lens)
    for layer in range(3):
        k = torch.randn(2, 12, 16, 64, generator=torch.Generator().manual_seed(layer)).bfloat16().to(DEV)
        kv = rpo.PagedKV(k, k.clone(), table, lens)
        mass = torch.rand(n, 2, 64, generator=torch.Generator().manual_seed(layer)).to(DEV)
        src, out = torch.zeros(n, 2, budget, dtype=torch.int32, device=DEV), torch.zeros(n, 2, budget, device=DEV)
        contexts["bf16"].evict_cache(kv, mass, pos, budget, lens if layer == 2 else scratch, src, out, torch.zeros_like(src), sinks=2, recent=4)
        torch.cuda.synchronize()
        for s, m in enumerate((50, 20, 33)):
            for h in range(2):
                want = paged.evict(mass[s, h, :m].tolist(), list(range(m)), budget, 2, 4)
                assert src[s, h, :len(want)].tolist() == want
    assert lens.tolist() == [24, 20, 24] and contexts["bf16"].device_status() == 0


def test_long_runs_of_single_tokens_before_chunks(contexts):  # noqa: F811
    """A call of chunks and single tokens: of the two halves of a row tile only the first works on single tokens, for about a
    millisecond here.  The second one's wait meanwhile does not count against the limit of device-side waits."""
    ctx, (hq, hkv, dh), keys = contexts["bf16"], (28, 4, 128), 40000
    new = ([1] * 25 + [100]) * 4
    g = torch.Generator(device=DEV)
    g.manual_seed(71)
    k, v = (torch.randn(hkv, keys // 16, 16, dh, generator=g, device=DEV).bfloat16() for _ in range(2))
    table = torch.randperm(keys // 16, generator=g, device=DEV).to(torch.int32).expand(len(new), -1).contiguous()     # one cache for all
    kv = rpo.PagedKV(k, v, table, torch.full((len(new),), keys, dtype=torch.int32, device=DEV))
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
    q = torch.randn(sum(new), hq, dh, generator=g, device=DEV).bfloat16()
    got = []
    for limit in (0, 500000):                                              # the default; about 0.3 ms
        ctx.set_option("wait_limit_cycles", limit)
        try:
            out, lse = torch.zeros_like(q), torch.zeros(len(q), hq, device=DEV)
            ctx.chunk_attention(q, kv, off, 100, out, lse)
            mass = torch.zeros(len(new), hkv, keys, device=DEV)
            ctx.attention_mass(q, kv, off, 100, lse, mass)
            assert ctx.device_status() == 0
            got.append((out, lse, mass))
        finally:
            ctx.set_option("wait_limit_cycles", 0)
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("longest", [2, 64], ids=["steps", "chunks"])
def test_a_captured_call_follows_offsets_and_lengths(dtype, longest):
    """One graph, replayed for other chunks: rows before the first sequence and behind the last are left alone."""
    s = torch.cuda.Stream()
    with rpo.Context(rpo.shape_preset("tiny", dtype=1 if dtype == "bf16" else 0), kv_pool_blocks=8, max_groups=1, max_seqs=1, max_chunk_tokens=16,
                     max_positions=32, stream=s) as ctx:
        c = Case(dtype, 8, 2, 64, [longest] * 4, [300, 90, 1000, 64], seed=81, extra_rows=5, window=200, sinks=2)
        out, lse = torch.zeros_like(c.q), torch.zeros(c.q.shape[:2], device=DEV)
        mass = torch.zeros(4, 2, 1000, device=DEV)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ctx.chunk_attention(c.q, c.kv, c.d_off, longest, out, lse, window=200, sinks=2)
            ctx.attention_mass(c.q, c.kv, c.d_off, longest, lse, mass, window=200, sinks=2)
        full = list(c.lens)
        for first, new, less in ((0, [longest] * 4, 0), (3, [1, 0, longest, 2], 17), (5, [0, 0, 0, 0], 5), (1, [2, longest, 0, 1], 60)):
            c.new, c.lens = new, [n - less for n in full]
            c.off = (first + np.concatenate([[0], np.cumsum(new)])).astype(np.int32)
            c.d_off.copy_(torch.from_numpy(c.off))
            c.kv.d_lens.copy_(torch.tensor(c.lens, dtype=torch.int32))
            out.fill_(7.0)
            lse.fill_(7.0)
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                graph.replay()
            torch.cuda.synchronize()
            assert bool((out[:first] == 7.0).all()) and bool((lse[:first] == 7.0).all())
            n = int(c.off[-1])
            want, want_lse = paged.chunk_attention(c.np(c.q), np.nan_to_num(c.np(c.k)), np.nan_to_num(c.np(c.v)), c.table, c.lens, c.off, c.scale, 200, 2)
            ew, el, a = c.errors()
            tol = a * (2 * ew + 3 * max(c.lens) * U)[..., None] + torch.finfo(c.dtype).eps / 2 * np.abs(want) + (2.0 ** -8 * a if dtype == "bf16" else 0)
            assert np.all(np.abs(c.np(out) - want)[first:n] <= tol[first:n] + 1e-30) and np.all(c.np(out)[n:] == 7.0)
            g, want_lse, empty = c.np(lse), want_lse[first:n], np.isneginf(want_lse[first:n])          # rows before their first token
            assert np.array_equal(np.isneginf(g[first:n]), empty) and np.all(g[n:] == 7.0)
            assert np.all(np.abs(g[first:n][~empty] - want_lse[~empty]) <= el[first:n][~empty])
            total = c.np(mass)
            for i in range(4):
                assert np.allclose(total[i, :, :c.lens[i]].sum(1), min(new[i], c.lens[i]) * 4, rtol=1e-4, atol=1e-30)
        assert ctx.device_status() == 0
        del graph
