"""Drafted tokens and shared pages on a caller-owned cache against oracle/drafts.py.

Tolerances of the attention are those of test_gpu_paged_ops.py (u = 2^-24): with S = scale sum_d |q_d k_d| a score is off by at
most (head_dim + 2) u S, the exponential of it adds 2^-21 + 2 u S, a sum of n terms n u: an output by A (2 ew + 3 n u), A = sum_j
w_j |v_j|, with 16-bit storage 2^-8 A (weights) and half a step of the output more.  Log-probabilities are z - z_max - log(sum):
the float32 z and its division are each off by u |z|, the sum of V positive terms (at most V / 4096 in a row per thread, the
rest in trees) by (V / 4096 + 64) u relative.  Paths, tokens, tables, counts, stacks and moved rows are exact.
"""
import numpy as np
import pytest
import torch

import paper_2601_19404_b200 as rpo
from oracle import drafts, paged, philox
from gpu_util import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def make_context(dtype, stream=None):
    return rpo.Context(rpo.shape_preset("tiny", dtype=1 if dtype == "bf16" else 0), kv_pool_blocks=8, max_groups=1, max_seqs=1, max_chunk_tokens=16,
                       max_positions=32, stream=stream)


@pytest.fixture(scope="module")
def contexts():
    made = {n: make_context(n) for n in DTYPES}
    yield made
    for c in made.values():
        c.close()


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


# ---- trees ---------------------------------------------------------------------------------------------------------
def random_tree(n, rng, holes=0.0):
    p = [-1] + [int(rng.integers(-1, i)) if rng.random() < 0.5 else i - 1 - int(rng.integers(0, min(i, 3))) for i in range(1, n)] if n else []
    return [-2 if rng.random() < holes else x for x in p]


class Tree:
    """Random trees and cache; whatever no row may depend on is NaN (behind the last slot, unused blocks, slots without a node)."""

    def __init__(self, dtype, hq, hkv, dh, nodes, past, seed=0, spread=1.5, extra_rows=0, window=0, sinks=0, holes=0.0, parents=None):
        rng, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        self.dtype, self.hq, self.hkv, self.dh, self.window, self.sinks = DTYPES[dtype], hq, hkv, dh, window, sinks
        self.lens, self.scale = [a + b for a, b in zip(nodes, past)], dh ** -0.5
        self.off = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
        rows = int(self.off[-1]) + extra_rows
        trees = parents or [random_tree(n, rng, holes) for n in nodes]
        self.parents = np.array([p for t in trees for p in t] + [-1] * extra_rows, dtype=np.int32)
        qkv = torch.randn(rows, hq + 2 * hkv, dh, generator=g)
        qkv[:, :hq] *= spread
        self.qkv = qkv.to(self.dtype).to(DEV)
        self.q, self.k_new, self.v_new = self.qkv[:, :hq], self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:]
        pages = [-(-n // 16) for n in self.lens]
        n_blocks = sum(pages) + 3
        order = torch.randperm(n_blocks, generator=g).tolist()
        self.table = np.full((len(nodes), max(pages + [1]) + 2), -1, dtype=np.int32)
        k, v = (torch.full((hkv, n_blocks, 16, dh), float("nan")) for _ in range(2))
        for s, n in enumerate(self.lens):
            for p in range(pages[s]):
                b = self.table[s, p] = order.pop()
                live = min(16, n - 16 * p)
                k[:, b, :live], v[:, b, :live] = torch.randn(hkv, live, dh, generator=g), torch.randn(hkv, live, dh, generator=g)
            for i, chain in enumerate(drafts.chains(trees[s])):
                if chain is None:
                    j = past[s] + i
                    k[:, self.table[s, j // 16], j % 16] = v[:, self.table[s, j // 16], j % 16] = float("nan")
        self.k, self.v = k.to(self.dtype).to(DEV), v.to(self.dtype).to(DEV)
        self.kv = rpo.PagedKV(self.k, self.v, i32(self.table), i32(self.lens))
        self.d_off, self.d_parents, self.max_nodes = i32(self.off), i32(self.parents), max(max(nodes), 1)

    def attend(self, ctx, append=False, lse=True):
        out = torch.full(self.q.shape, 7.0, dtype=self.dtype, device=DEV)
        d_lse = torch.full(self.q.shape[:2], 7.0, device=DEV) if lse else None
        ctx.tree_attention(self.q, self.kv, self.d_off, self.d_parents, self.max_nodes, out, d_lse, d_k_new=self.k_new if append else None,
                           d_v_new=self.v_new if append else None, window=self.window, sinks=self.sinks)
        torch.cuda.synchronize()
        return out, d_lse

    def check(self, out, lse):
        q, k, v = f64(self.q), np.nan_to_num(f64(self.k)), np.nan_to_num(f64(self.v))
        want, want_lse = drafts.tree_attention(q, k, v, self.table, self.lens, self.off, self.parents, self.scale, self.window, self.sinks)
        n, rep = int(self.off[-1]), self.hq // self.hkv
        tol, el = np.zeros(want.shape), np.zeros(want_lse.shape)
        for s, keys in enumerate(self.lens):
            a, b = self.off[s], self.off[s + 1]
            kk, vv = paged.token_rows(k, self.table[s], keys), paged.token_rows(v, self.table[s], keys)
            seen = drafts.visible(self.parents[a:b], keys, self.window, self.sinks)
            for h in range(self.hq):
                big = (self.scale * np.abs(q[a:b, h]) @ np.abs(kk[h // rep]).T).max(1, initial=0.0)
                ew = (self.dh + 4) * U * big + 2.0 ** -21
                total = drafts.weights(q[a:b, h], kk[h // rep], seen, self.scale)[0] @ np.abs(vv[h // rep])
                tol[a:b, h] = total * (2 * ew + 3 * keys * U + (2.0 ** -8 if self.dtype == torch.bfloat16 else 0))[:, None]
                el[a:b, h] = ew + keys * U + 2.0 ** -22 * (big + 10)
        tol += torch.finfo(self.dtype).eps / 2 * np.abs(want)
        got = f64(out)
        assert np.all(np.isfinite(got[:n]))
        assert np.all(np.abs(got[:n] - want[:n]) <= tol[:n] + 1e-30), np.max(np.abs(got[:n] - want[:n]) - tol[:n])
        assert np.all(got[n:] == 7.0)
        if lse is not None:
            g, empty = f64(lse), np.isneginf(want_lse[:n])
            assert np.array_equal(np.isneginf(g[:n]), empty)
            assert np.all(np.abs(g[:n][~empty] - want_lse[:n][~empty]) <= el[:n][~empty]) and np.all(g[n:] == 7.0)


HEADS = [(4, 2, 64), (12, 2, 128), (7, 1, 64), (3, 3, 128), (28, 4, 128), (64, 1, 128)]
# (nodes, cached tokens)
SIZES = {"small": ([2, 1, 0, 2, 1, 2], [0, 15, 9, 33, 128, 300]),
         "mixed": ([16, 1, 0, 40, 5, 17, 33], [300, 7, 9, 0, 16, 111, 223]),
         "large": ([256, 60, 129], [70, 1030, 0])}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("mask", [(0, 0), (1, 0), (5, 0), (33, 5), (128, 200)])
@pytest.mark.parametrize("holes", [0.0, 0.3])
def test_tree_attention(contexts, dtype, heads, size, mask, holes):
    if size == "large" and heads not in HEADS[:2] + HEADS[4:5]:
        pytest.skip("large trees on three head layouts")
    c = Tree(dtype, *heads, *SIZES[size], seed=sum(heads), extra_rows=2, window=mask[0], sinks=mask[1], holes=holes)
    c.check(*c.attend(contexts[dtype]))
    assert contexts[dtype].device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES)
def test_tree_attention_appends_its_nodes(contexts, dtype, size):
    c = Tree(dtype, 8, 4, 64, *SIZES[size], seed=5, extra_rows=1, holes=0.2)
    k, v = f64(c.k), f64(c.v)
    for cache, new in ((k, c.k_new), (v, c.v_new)):
        drafts.append(cache, f64(new), c.table, c.lens, c.off, c.parents)
    out, lse = c.attend(contexts[dtype], append=True)
    assert np.array_equal(f64(c.k), k, equal_nan=True) and np.array_equal(f64(c.v), v, equal_nan=True)
    c.check(out, lse)
    again, _ = c.attend(contexts[dtype], append=True, lse=False)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sizes", [([4], [20011]), ([60, 60], [9000, 5003]), ([3] * 200, list(range(200))), ([100], [7])])
def test_tree_attention_on_long_sequences_and_many_short_ones(contexts, dtype, sizes):
    c = Tree(dtype, 12, 2, 128, *sizes, seed=8)
    out, lse = c.attend(contexts[dtype])
    c.check(out, lse)
    again, lse2 = c.attend(contexts[dtype])
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_tree_attention_with_single_keys_that_decide(contexts, dtype):
    for size in SIZES.values():
        c = Tree(dtype, 4, 2, 64, *size, seed=9, spread=60.0, holes=0.1)
        c.check(*c.attend(contexts[dtype]))


@pytest.mark.parametrize("hq,hkv,dh", [(14, 2, 128), (8, 2, 64), (64, 1, 128)])
@pytest.mark.parametrize("seed", range(4))
def test_tree_attention_of_large_and_small_trees_side_by_side(contexts, hq, hkv, dh, seed):
    """Work lists whose items cost different amounts, cut anywhere."""
    rng = np.random.default_rng(seed)
    nodes, past = rng.integers(1, 120, 5), rng.integers(0, (100, 1000, 3000, 6000)[seed], 5)
    t = Tree("bf16", hq, hkv, dh, nodes.tolist(), past.tolist(), seed=seed, window=0 if seed % 2 else 500, sinks=0 if seed % 2 else 9)
    t.check(*t.attend(contexts["bf16"], append=True))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [5, 60])
def test_a_chain_is_a_chunk(contexts, dtype, n):
    c = Tree(dtype, 12, 2, 128, [n, n], [100, 333], seed=2, parents=[list(range(-1, n - 1))] * 2, window=40, sinks=3)
    out, lse = c.attend(contexts[dtype])
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    contexts[dtype].chunk_attention(c.q, c.kv, c.d_off, n, out2, lse2, window=40, sinks=3)
    assert np.max(np.abs(f64(out) - f64(out2))) <= 2 ** -6 * np.max(np.abs(f64(out2))) and torch.allclose(lse, lse2, atol=1e-4)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_trees_without_any_node_and_bad_parents(contexts, dtype):
    ctx = contexts[dtype]
    for rows in (3, 40):
        c = Tree(dtype, 12, 2, 128, [rows, rows], [50, 50], seed=3, parents=[[-2] * rows, list(range(-1, rows - 1))])
        c.k[:, i32(c.table[0, :3]).long()] = float("nan")                # a sequence that nobody looks at
        c.v[:, i32(c.table[0, :3]).long()] = float("nan")
        c.check(*c.attend(ctx))
        assert ctx.device_status() == 0
        c.parents[rows + 1:rows + 3] = [1, 9]                            # itself; one behind it
        c.d_parents.copy_(i32(c.parents))
        got, lse = c.attend(ctx)
        assert ctx.device_status() == 8
        assert torch.isfinite(got.float()).all() and torch.isneginf(lse[rows + 1:]).all() and (got[rows + 1:] == 0).all() and torch.isfinite(lse[rows]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads", [(2, 2, 64), (3, 3, 128), (8, 4, 64), (4, 2, 128), (6, 2, 64), (16, 4, 128), (5, 1, 128)])
@pytest.mark.parametrize("mask", [(0, 0), (2, 0), (7, 40), (64, 3)])
@pytest.mark.parametrize("append", [False, True])
def test_trees_of_at_most_sixteen_packed_rows(contexts, dtype, heads, mask, append):
    """Nodes x query heads of a KV head within one tile of sixteen rows: chains, stars, siblings at every level, holes in the middle, random ones."""
    most = 16 // (heads[0] // heads[1])
    shapes = [list(range(-1, most - 1)), [-1] + [0] * (most - 1), [(i - 1) // 2 if i else -1 for i in range(most)], [-1] * most,
              [-2 if i == most // 2 else i - 1 for i in range(most)], [-1, 0, 0, 1, 1, 2, 2, 3, -2, 5, 8, 4, 11, 12, -1, 14][:most],
              [-2] + [max(i - 2, -1) for i in range(1, most)], [-1]]
    trees = shapes + [random_tree(most - k % 2, np.random.default_rng(k), 0.15 * (k % 3)) for k in range(8)] + [[]]
    past = [0, 1, 15, 16, 17, 31, 100, 0, 300, 2000, 7, 33, 48, 250, 640, 5, 9]
    c = Tree(dtype, *heads, [len(t) for t in trees], past, seed=sum(heads) + mask[0], extra_rows=1, window=mask[0], sinks=mask[1], parents=trees)
    k, v = f64(c.k), f64(c.v)
    if append:
        for cache, new in ((k, c.k_new), (v, c.v_new)):
            drafts.append(cache, f64(new), c.table, c.lens, c.off, c.parents)
    out, lse = c.attend(contexts[dtype], append=append)
    assert np.array_equal(f64(c.k), k, equal_nan=True) and np.array_equal(f64(c.v), v, equal_nan=True)
    c.check(out, lse)
    assert contexts[dtype].device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,dh", [(4, 2, 64), (12, 2, 128)])
@pytest.mark.parametrize("mask", [(0, 0), (3, 0), (4, 9)])
@pytest.mark.parametrize("append", [False, True])
def test_trees_longer_than_their_sequences(contexts, dtype, hq, hkv, dh, mask, append):
    """Fewer tokens than nodes: nodes whose slots would be negative are none, the others see one another; bit 3."""
    for nodes, lens in (([6, 8, 5, 3, 7], [5, 1, 0, 3, 4]), ([40, 20, 33, 90], [39, 3, 0, 50])):
        c = Tree(dtype, hq, hkv, dh, nodes, [0] * len(nodes), seed=dh, extra_rows=1, window=mask[0], sinks=mask[1],
                 parents=[[-1 if i % 7 == 0 or i == 4 else i - 1 - (i % 3 == 2) for i in range(n)] for n in nodes])
        k, v = c.k.clone(), c.v.clone()
        for s, n in enumerate(lens):                                     # (also what lies behind the sequences' new ends)
            for j in range(n, c.lens[s]):
                k[:, c.table[s, j // 16], j % 16] = v[:, c.table[s, j // 16], j % 16] = float("nan")
        c.k.copy_(k), c.v.copy_(v)
        c.lens = lens
        c.kv.d_lens.copy_(i32(lens))
        if append:
            k, v = f64(c.k), f64(c.v)
            for cache, new in ((k, c.k_new), (v, c.v_new)):
                drafts.append(cache, f64(new), c.table, c.lens, c.off, c.parents)
        out, lse = c.attend(contexts[dtype], append=append)
        assert contexts[dtype].device_status() == 8
        if append:
            assert np.array_equal(f64(c.k), k, equal_nan=True) and np.array_equal(f64(c.v), v, equal_nan=True)
        c.check(out, lse)


def test_tree_attention_refusals(contexts):
    c, ctx = Tree("bf16", 4, 2, 64, [3], [20]), contexts["bf16"]
    out = torch.empty_like(c.q.contiguous())
    for change in (dict(max_nodes=257), dict(max_nodes=0), dict(scale=0.0), dict(window=-1)):
        args = dict(d_q=c.q, kv=c.kv, d_q_offsets=c.d_off, d_parents=c.d_parents, max_nodes=3, d_out=out)
        with pytest.raises(rpo.RpoError):
            ctx.tree_attention(**{**args, **change})


# ---- verification --------------------------------------------------------------------------------------------------
class Drafts:
    def __init__(self, vocab, trees, seed=0, given=True, spread=3.0, temperature=1.0, top_p=1.0, greedy=False, eos_id=-1, max_path=None, pad=0):
        rng = np.random.default_rng(seed)
        self.cfg = dict(temperature=temperature, top_p=top_p, greedy=greedy, eos_id=eos_id)
        self.off = np.concatenate([[0], np.cumsum([len(t) for t in trees])]).astype(np.int32)
        rows = int(self.off[-1])
        self.parents = np.array([p for t in trees for p in t], dtype=np.int32)
        self.logits = (rng.standard_normal((rows, vocab + pad)) * spread).astype(np.float32)[:, :vocab]
        near = self.logits / np.float32(temperature) + (rng.standard_normal((rows, vocab)) * 0.7).astype(np.float32)
        q = np.exp((near - near.max(1, keepdims=True)).astype(np.float64))
        self.probs = (q / q.sum(1, keepdims=True)).astype(np.float32) if given else None
        self.tokens = rng.integers(0, vocab, rows).astype(np.int32)
        for s, t in enumerate(trees):
            for i, p in enumerate(t):
                if p >= 0:
                    at = self.off[s] + p
                    self.tokens[self.off[s] + i] = rng.choice(vocab, p=q[at] / q[at].sum()) if given else np.argsort(-near[at], kind="stable")[i % 3 % vocab]
        self.uniform = (rng.integers(0, 2 ** 24, rows) / 2 ** 24).astype(np.float32)
        self.trees, self.pad, self.max_path = trees, pad, max_path or max(len(t) for t in trees + [[0]])

    def device(self, x):
        if x is None:
            return None
        if not self.pad:
            return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
        wide = torch.full((x.shape[0], x.shape[1] + self.pad), float("nan"), device=DEV)
        wide[:, :x.shape[1]] = torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
        return wide[:, :x.shape[1]]

    def run(self, ctx, logprobs=True):
        n = len(self.trees)
        path, n_path, nxt = (torch.full(s, 77, dtype=torch.int32, device=DEV) for s in ((n, self.max_path), (n,), (n,)))
        logp = torch.full((n, self.max_path), 7.0, device=DEV) if logprobs else None
        sampler = rpo.Sampler(self.cfg["temperature"], self.cfg["top_p"], self.cfg["greedy"], self.cfg["eos_id"])
        ctx.verify_drafts(self.device(self.logits), i32(self.tokens), i32(self.parents), i32(self.off), torch.from_numpy(self.uniform).to(DEV), sampler, path,
                          n_path, nxt, d_logprobs_out=logp, d_draft_probs=self.device(self.probs))
        torch.cuda.synchronize()
        return path, n_path, nxt, logp

    def check(self, path, n_path, nxt, logp):
        for s in range(len(self.trees)):
            a, b = self.off[s], self.off[s + 1]
            want, token, lp = drafts.verify(self.logits[a:b], self.tokens[a:b], self.parents[a:b], self.uniform[a:b], self.max_path,
                                            probs=None if self.probs is None else self.probs[a:b], **self.cfg)
            assert path[s].tolist() == want + [-1] * (self.max_path - len(want)), s
            assert int(n_path[s]) == len(want) and int(nxt[s]) == token, s
            if logp is not None:
                got, lp = f64(logp[s]), np.array(lp + [0.0] * (self.max_path - len(lp)))
                empty = np.isneginf(lp)
                big = np.nan_to_num(np.abs(self.logits[a:b]), posinf=0.0).max(initial=1.0) / self.cfg["temperature"]
                tol = 6 * U * big + (self.logits.shape[1] / 4096 + 64) * U + 4 * U * np.abs(np.where(empty, 0, lp))
                assert np.array_equal(np.isneginf(got), empty) and np.all(np.abs(got[~empty] - lp[~empty]) <= tol[~empty] if len(lp) else True)


CHAINS = [list(range(-1, n - 1)) for n in (5, 1, 9, 2)] + [[]]
TREES = [[-1, 0, 0, 0, 1, 1, 2, 4, 4], [-1], [], [-1, 0, 0, 0, 0, 0], [-1, 0, 1, 1, 2, 2, 3, 3, 4, 4, -1, 10, -2, 12]]


@pytest.mark.parametrize("vocab", [1, 2, 37, 1000, 4099, 32000])
@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("top_p", [1.0, 0.9, 0.3, 0.0])
@pytest.mark.parametrize("trees", [CHAINS, TREES], ids=["chains", "trees"])
def test_verification(contexts, vocab, given, top_p, trees):
    for seed, (temperature, spread) in enumerate([(1.0, 3.0), (0.7, 1.0), (1.5, 9.0), (1.0, 0.0)]):
        c = Drafts(vocab, trees, seed=seed, given=given, top_p=top_p, temperature=temperature, spread=spread)
        c.check(*c.run(contexts["bf16"]))
    assert contexts["bf16"].device_status() == 0


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("vocab", [151936, 152063, 262143])
def test_verification_with_large_vocabularies(contexts, given, vocab):
    for top_p, spread in ((0.95, 4.0), (1.0, 3.0), (0.999, 0.01)):
        c = Drafts(vocab, [CHAINS[0], TREES[0]], seed=3, given=given, top_p=top_p, spread=spread)
        c.check(*c.run(contexts["fp32"]))
        again = c.run(contexts["fp32"])
        assert all(torch.equal(x, y) for x, y in zip(again, c.run(contexts["fp32"])))


def test_verification_of_many_sequences(contexts):
    trees = [TREES[i % 5] if i % 2 else CHAINS[i % 5] for i in range(300)]
    for given in (True, False):
        c = Drafts(503, trees, seed=11, given=given, top_p=0.95)
        c.check(*c.run(contexts["bf16"]))


@pytest.mark.parametrize("n", [6, 200])
def test_verification_whose_clusters_start_apart(n):
    """CTAs of a cluster speak to one another once all have started: clusters of sixteen and of eight, some without rows, begin whenever another
    call's leave room for them."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    made = [make_context("bf16", s) for s in streams]
    cases = [Drafts(20011, [(TREES + CHAINS)[(i + k) % 10] for i in range(n)], seed=20 + k, top_p=0.9) for k in range(2)]
    inputs, outs = [], []
    for c in cases:
        inputs.append(([c.device(c.logits), i32(c.tokens), i32(c.parents), i32(c.off), torch.from_numpy(c.uniform).to(DEV), rpo.Sampler(top_p=0.9)], c.device(c.probs)))
        outs.append([[torch.full(s, 77, dtype=torch.int32, device=DEV) for s in ((n, c.max_path), (n,), (n,))] + [torch.full((n, c.max_path), 7.0, device=DEV)]
                     for _ in range(12)])
    torch.cuda.synchronize()
    for i in range(12):
        for ctx, (args, probs), out in zip(made, inputs, outs):
            ctx.verify_drafts(*args, *out[i], d_draft_probs=probs)
    torch.cuda.synchronize()
    for ctx, c, out in zip(made, cases, outs):
        c.check(*out[0])
        assert all(torch.equal(x, y) for again in out[1:] for x, y in zip(again, out[0])) and ctx.device_status() == 0
        ctx.close()


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("top_p", [1.0, 0.9])
def test_verification_of_many_nodes(contexts, given, top_p):
    """Sequences of more than 128 rows: random trees, a root whose children, equal tokens among them, lie on both sides of row 128 (and are
    all refused before some row), and accepted chains that cross it."""
    ctx = contexts["bf16"]
    trees = [random_tree(n, np.random.default_rng(n)) for n in (129, 128, 256, 300)] + [[-1] + [0] * 255, [-1] + [0] * 128, list(range(-1, 199)), [-1, 0] * 100]
    for seed in range(3):
        c = Drafts(97, trees, seed=40 + seed, given=given, top_p=top_p, spread=1.0)
        c.check(*c.run(ctx))
        for first in (100, 128, 129, 200):                               # refused with the largest number, as a rule, before that row
            for s in (4, 5):
                a, b = int(c.off[s]), int(c.off[s + 1])
                c.uniform[a + 1:min(a + first, b)] = 1.0 - 2.0 ** -24
                c.uniform[a + first:b] = 0.0
            c.check(*c.run(ctx))
        for u0 in (0.0, 0.6, 1.0 - 2.0 ** -24):                          # all refused: what is drawn then
            c.uniform[:] = 1.0 - 2.0 ** -24
            c.uniform[c.off[:-1]] = u0
            c.check(*c.run(ctx))
        c.cfg["greedy"] = True
        best = c.logits.argmax(1)
        for s in range(len(trees)):                                      # the target's own choice, but for one node behind row 128
            for i, p in enumerate(trees[s]):
                if p >= 0 and i != 150 + 10 * seed:
                    c.tokens[c.off[s] + i] = best[c.off[s] + p]
        got = c.run(ctx)
        c.check(*got)
        assert int(got[1][6]) == 150 + 10 * seed
        c.cfg["eos_id"] = int(c.tokens[c.off[6] + 140])
        c.check(*c.run(ctx))
    assert ctx.device_status() == 0


def test_verification_on_padded_rows_short_paths_and_without_logprobs(contexts):
    for pad in (1, 4):
        c = Drafts(1003, TREES, seed=4, pad=pad, top_p=0.9, max_path=2)
        c.check(*c.run(contexts["bf16"]))
        c.check(*c.run(contexts["bf16"], logprobs=False))
    c = Drafts(64, [CHAINS[2]], seed=4, max_path=1)
    c.check(*c.run(contexts["bf16"]))


def test_verification_greedy_and_end_of_sequence(contexts):
    for given in (True, False):
        for seed in range(4):
            c = Drafts(50, CHAINS + TREES, seed=seed, given=given, greedy=True, spread=1.0)
            best = c.logits.argmax(1)
            for s, t in enumerate(c.trees):                              # some drafts are the target's own choice
                for i, p in enumerate(t):
                    if p >= 0 and (i + seed) % 3:
                        c.tokens[c.off[s] + i] = best[c.off[s] + p]
            c.check(*c.run(contexts["bf16"]))
            c.cfg["eos_id"] = int(c.tokens[2])
            c.check(*c.run(contexts["bf16"]))
            c.cfg["greedy"] = False
            c.check(*c.run(contexts["bf16"]))


def test_verification_at_the_borders(contexts):
    """u at its ends and out of range, equal distributions, q of zeros, no numbers and infinities, equal tokens, no tokens left."""
    ctx = contexts["bf16"]
    for u in (0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, float("nan")):
        for given in (True, False):
            c = Drafts(300, TREES, seed=5, given=given, top_p=0.9)
            c.uniform[:] = u
            keep = c.uniform.copy()
            c.uniform[:] = min(max(np.nan_to_num(np.float32(u), nan=0.0), 0.0), 1.0)
            want = c
            got = c.run(ctx)
            want.check(*got)
            c.uniform = keep
            assert all(torch.equal(x, y) for x, y in zip(got, c.run(ctx)))
    c = Drafts(300, TREES, seed=6)
    z = c.logits.astype(np.float64)
    p = np.exp(z - z.max(1, keepdims=True))
    c.probs = (p / p.sum(1, keepdims=True)).astype(np.float32)
    c.uniform[:] = 1.0 - 2.0 ** -24
    c.check(*c.run(ctx))
    c.probs *= np.float32(1.5)                                           # sums above one: nothing is left after a refusal
    c.check(*c.run(ctx))
    c.probs[:] = 0
    c.check(*c.run(ctx))
    c.probs[:] = np.float32("nan")
    c.check(*c.run(ctx))
    c.probs[:] = np.float32("inf")
    c.check(*c.run(ctx))
    c = Drafts(300, [[-1] + [0] * 7], seed=7, given=False)
    c.tokens[1:] = [5, 9, 5, 5, 9, 1, 5]
    for u in (0.999, 0.5, 0.01):
        c.uniform[:] = u
        c.check(*c.run(ctx))
    assert ctx.device_status() == 0
    for value in (-np.inf, np.nan, np.inf):
        c = Drafts(300, TREES, seed=8, top_p=0.9)
        c.logits[::2] = value
        c.logits[1::2, 7:] = value
        c.check(*c.run(ctx))
    c = Drafts(40, TREES, seed=9, given=False)
    c.tokens[1:4] = [-1, 40, 2 ** 31 - 1]
    c.check(*c.run(ctx))
    assert ctx.device_status() == 2
    c = Drafts(40, TREES, seed=9)
    c.off[2] = 10 ** 6
    c.run(ctx)
    assert ctx.device_status() & 8


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("top_p", [1.0, 0.9, 0.3])
@pytest.mark.parametrize("vocab", [40, 5003])
def test_verification_of_tokens_outside_the_vocabulary(contexts, given, top_p, vocab):
    """A negative token is no draft: what is left for others stays as it is.  One beyond the vocabulary is refused as any that the target excludes."""
    wide = [[-1, 0, 0, 0, 0, 0, 0, 1, 2, 3, 4, 5, 6]] * 12
    for bad in ([-1], [vocab], [-2 ** 31, 2 ** 31 - 1], [-1, vocab + 7, -5]):
        for seed in range(4):
            c = Drafts(vocab, wide + TREES, seed=30 + seed, given=given, top_p=top_p, greedy=seed == 3)
            rng = np.random.default_rng(seed)
            for i in range(int(c.off[-1])):
                if c.parents[i] >= 0 and rng.random() < (0.3, 0.6, 1.0, 0.5)[seed]:
                    c.tokens[i] = bad[int(rng.integers(len(bad)))]
            c.check(*c.run(contexts["bf16"]))
            assert contexts["bf16"].device_status() in ((0, 2) if seed < 2 else (2,))


def test_verification_without_drafts_is_the_sampler(contexts):
    """One row per sequence: rpo_sample_rows with the same random numbers gives the same tokens and log-probabilities."""
    ctx, n, vocab = contexts["fp32"], 40, 5003
    logits = torch.randn(n, vocab, device=DEV, generator=torch.Generator(DEV).manual_seed(1)) * 3
    u = np.array([philox.sampler_u24(3, s, 11) for s in range(n)])
    for top_p in (1.0, 0.9):
        sampler = rpo.Sampler(0.8, top_p, seed=3)
        tok, lp = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n, device=DEV)
        ctx.sample_rows(logits, sampler, torch.arange(n, dtype=torch.int64, device=DEV), 11, tok, lp)
        path, n_path, nxt, logp = torch.zeros(n, 3, dtype=torch.int32, device=DEV), torch.zeros_like(tok), torch.zeros_like(tok), torch.zeros(n, 3, device=DEV)
        ctx.verify_drafts(logits, torch.zeros_like(tok), torch.full_like(tok, -1), torch.arange(n + 1, dtype=torch.int32, device=DEV),
                          torch.tensor(u / 2.0 ** 24, dtype=torch.float32, device=DEV), sampler, path, n_path, nxt, logp)
        assert torch.equal(nxt, tok) and torch.allclose(logp[:, 0], lp, atol=2e-5)


# ---- pages ---------------------------------------------------------------------------------------------------------
class Cache:
    """A pool of several layers, and its twin in plain Python."""

    def __init__(self, dtype, layers, hkv, dh, n_blocks, n_seqs, width, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.kv = torch.randn(layers, 2, hkv, n_blocks, 16, dh, generator=g).to(DTYPES[dtype]).to(DEV)
        self.pool = rpo.PagePool.empty(n_blocks, n_seqs, width, DEV)
        self.pool.d_free.copy_(torch.randperm(n_blocks, generator=g).to(torch.int32))
        self.lens = torch.zeros(n_seqs, dtype=torch.int32, device=DEV)
        self.layers = rpo.PagedLayers([rpo.PagedKV(self.kv[i, 0], self.kv[i, 1], self.pool.d_block_table, self.lens) for i in range(layers)])
        self.twin = drafts.Pages(self.pool.d_refs.tolist(), self.pool.d_free.tolist(), n_blocks, self.pool.d_block_table.tolist(), [0] * n_seqs)
        self.content = f64(self.kv)

    def same(self):
        torch.cuda.synchronize()
        p, t = self.pool, self.twin
        assert p.d_held.tolist() == t.held and p.d_block_table.tolist() == t.table and p.d_refs.tolist() == t.refs
        assert int(p.d_n_free) == t.n_free and p.d_free.tolist() == t.free
        t.copy(self.content)
        assert np.array_equal(f64(self.kv), self.content)


@pytest.mark.parametrize("dtype,layers,hkv,dh", [("bf16", 3, 2, 128), ("fp32", 2, 3, 64), ("bf16", 1, 1, 64), ("fp32", 1, 2, 128)])
def test_pages_over_many_calls(contexts, dtype, layers, hkv, dh):
    """Forks, growth, cuts and releases at random, some beyond what the pool has: everything as in the plain twin, after every call."""
    ctx, rng = contexts[dtype], np.random.default_rng(layers)
    n, width, blocks = 9, 7, 45
    c = Cache(dtype, layers, hkv, dh, blocks, n, width)
    lens, short, left_out = [0] * n, 0, 0
    for step in range(120):
        if rng.random() < 0.6:
            target = [int(rng.integers(0, width * 16 + 1)) if rng.random() < 0.4 else x for x in lens]
            ctx.reserve_pages(c.pool, c.layers, i32(lens), i32(target))
            held = list(c.twin.held)
            c.twin.reserve(lens, target)
            short += c.twin.short
            assert ctx.device_status() == (16 if c.twin.short else 0)
            lens = [min(t, c.twin.held[s] * 16) if c.twin.held[s] != held[s] or t <= held[s] * 16 else x for s, (t, x) in enumerate(zip(target, lens))]
        else:
            k = int(rng.integers(1, 6))
            src, dst = rng.integers(0, n, k), rng.integers(0, n, k)
            cut = [int(rng.integers(0, lens[s] + 1)) for s in src]
            c.lens.copy_(i32(lens))
            ctx.fork_pages(c.pool, c.layers, i32(src), i32(dst), i32(cut), c.lens)
            left = c.twin.fork(src, dst, cut, lens)
            left_out += len(left)
            assert ctx.device_status() == (8 if left else 0) + (16 if c.twin.short else 0)
            assert c.lens.tolist() == lens
        c.same()
    assert short and left_out


def test_pages_of_many_sequences(contexts):
    """Clusters of several CTAs: hundreds of forks of long sequences, shared pages dropped by many at once."""
    ctx, rng = contexts["bf16"], np.random.default_rng(0)
    n, width, blocks = 700, 90, 9000
    c = Cache("bf16", 1, 1, 64, blocks, n, width)
    lens = [1400 - 13 * (s % 7) if s < 20 else 0 for s in range(n)]
    ctx.reserve_pages(c.pool, c.layers, i32([0] * n), i32(lens))
    c.twin.reserve([0] * n, lens)
    c.same()
    src, dst = rng.integers(0, 20, n - 20), 20 + rng.permutation(n - 20)
    for _ in range(2):
        cut = [int(rng.integers(0, lens[s] + 1)) for s in src]
        ctx.fork_pages(c.pool, c.layers, i32(src), i32(dst), i32(cut))
        assert not c.twin.fork(src, dst, cut, lens)
        c.same()
    target = [x if s % 3 else 0 for s, x in enumerate(lens)]
    lens = [max(0, x - int(rng.integers(0, 40))) for x in lens]           # copies where tokens are cut off
    ctx.reserve_pages(c.pool, c.layers, i32(lens), i32(target))
    c.twin.reserve(lens, target)
    c.same()
    assert c.twin.copies
    ctx.reserve_pages(c.pool, c.layers, i32(lens), i32([0] * n))
    c.twin.reserve(lens, [0] * n)
    c.same()
    assert int(c.pool.d_n_free) == blocks and ctx.device_status() == 0


@pytest.mark.parametrize("n,width,second,slot", [(2, 1000, 1, 990), (300, 40, 256, 0), (300, 40, 299, 39), (700, 1100, 512, 1000)])
def test_a_shared_page_is_pushed_where_it_was_first_given_up(contexts, n, width, second, slot):
    """Two sequences hold one page and give it up in one call, the second of them long after the first."""
    ctx = contexts["bf16"]
    c = Cache("bf16", 1, 1, 64, 2 * width + n, n, width)
    lens = [0] * n
    lens[0] = lens[second] = width * 16
    ctx.reserve_pages(c.pool, c.layers, i32([0] * n), i32(lens))
    c.twin.reserve([0] * n, lens)
    c.same()
    # the second's page in `slot` goes back to the stack by hand, the first's page 0 takes its place
    t = c.twin
    page, lost = t.table[0][0], t.table[second][slot]
    t.table[second][slot] = page
    t.refs[page], t.refs[lost], t.free[t.n_free] = 2, 0, lost
    t.n_free += 1
    c.pool.d_block_table.copy_(i32(t.table))
    c.pool.d_refs.copy_(i32(t.refs))
    c.pool.d_free.copy_(i32(t.free))
    c.pool.d_n_free.fill_(t.n_free)
    c.same()
    ctx.reserve_pages(c.pool, c.layers, i32(lens), i32([0] * n))
    t.reserve(lens, [0] * n)
    c.same()
    assert ctx.device_status() == 0


def test_pages_of_one_long_sequence(contexts):
    ctx = contexts["bf16"]
    c = Cache("bf16", 1, 1, 64, 14000, 3, 6300)
    for lens, target in (([0, 0, 0], [100003, 0, 0]), ([100003, 0, 0], [100003, 0, 0]), ([100003, 99999, 0], [50001, 0, 0])):
        if lens[1]:
            ctx.fork_pages(c.pool, c.layers, i32([0]), i32([1]), i32([99999]))
            c.twin.fork([0], [1], [99999])
            c.same()
            target[1] = 99999 + 64
        ctx.reserve_pages(c.pool, c.layers, i32(lens), i32(target))
        c.twin.reserve(lens, target)
        c.same()


def test_bad_arguments_of_page_calls(contexts):
    ctx, n = contexts["bf16"], 4
    c = Cache("bf16", 1, 1, 64, 30, n, 5)
    ctx.reserve_pages(c.pool, c.layers, i32([0] * n), i32([40, 80, 0, 0]))
    c.twin.reserve([0] * n, [40, 80, 0, 0])
    c.same()
    assert ctx.device_status() == 0
    src, dst, cut = [0, -1, 4, 0, 1, 0, 1, 0], [2, 2, 2, 2, 2, -1, 4, 3], [10, 5, 5, 5, 5, 5, 5, 49]
    ctx.fork_pages(c.pool, c.layers, i32(src), i32(dst), i32(cut))
    assert c.twin.fork(src, dst, cut) == [1, 2, 3, 4, 5, 6, 7]
    c.same()
    assert ctx.device_status() == 8
    ctx.reserve_pages(c.pool, c.layers, i32([999, -5, 10, 0]), i32([90, 20, -7, 10 ** 6]))
    c.twin.reserve([999, -5, 10, 0], [90, 20, -7, 10 ** 6])
    c.same()
    assert ctx.device_status() == 8
    # entries of the table, the stack or the counts that name no page: reported, never followed
    for entry in (-1, 30, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 3):
        c = Cache("bf16", 1, 1, 64, 30, n, 5)
        ctx.reserve_pages(c.pool, c.layers, i32([0] * n), i32([40, 80, 0, 0]))
        c.pool.d_block_table[0, 1] = entry
        c.pool.d_free[int(c.pool.d_n_free) - 2] = entry
        ctx.fork_pages(c.pool, c.layers, i32([0, 0, 1]), i32([2, 3, 0]), i32([20, 33, 3]))
        ctx.reserve_pages(c.pool, c.layers, i32([20, 30, 20, 30]), i32([60, 10, 60, 0]))
        ctx.reserve_pages(c.pool, c.layers, i32([20, 10, 20, 0]), i32([0, 0, 0, 0]))
        assert ctx.device_status() & 4
    for held, free in ((-3, 30), (99, -1), (2, 10 ** 6)):
        c = Cache("bf16", 1, 1, 64, 30, n, 5)
        ctx.reserve_pages(c.pool, c.layers, i32([0] * n), i32([40, 80, 0, 0]))
        c.pool.d_held[0], c.pool.d_n_free[0] = held, free
        ctx.fork_pages(c.pool, c.layers, i32([0, 1]), i32([2, 3]), i32([20, 33]))
        ctx.reserve_pages(c.pool, c.layers, i32([20, 30, 20, 30]), i32([60, 80, 60, 80]))
        assert ctx.device_status() & 8


def test_lengths_beyond_what_is_held(contexts):
    """Bit 3 where tokens that would stay are not there; not for a length that the target cuts to what is held."""
    ctx = contexts["bf16"]
    for held, lens, target, bit in ((16, 40, 40, 8), (16, 40, 17, 8), (16, 17, 80, 8), (16, 40, 16, 0), (16, 40, 5, 0), (16, 40, 0, 0), (0, 40, 0, 0), (0, 1, 1, 8), (16, 16, 80, 0),
                                    (80, 81, 0, 8), (80, -1, 0, 8), (80, 80, 81, 8), (80, 80, -1, 8)):
        c = Cache("bf16", 1, 1, 64, 20, 3, 5)
        ctx.reserve_pages(c.pool, c.layers, i32([0] * 3), i32([20, held, 33]))
        c.twin.reserve([0] * 3, [20, held, 33])
        assert ctx.device_status() == 0
        ctx.reserve_pages(c.pool, c.layers, i32([20, lens, 33]), i32([40, target, 20]))
        c.twin.reserve([20, lens, 33], [40, target, 20])
        c.same()
        assert ctx.device_status() == bit, (held, lens, target)


@pytest.mark.parametrize("entry", [-1, 30, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 3])
def test_a_bad_entry_concerns_its_sequence_alone(contexts, entry):
    """One number of a table, or of the stack, that names no page: what all others hold, and where pages go, is as without it."""
    ctx, n = contexts["bf16"], 4

    def made():
        c = Cache("bf16", 1, 1, 64, 30, n, 5)
        lens = [40, 80, 0, 20]
        ctx.reserve_pages(c.pool, c.layers, i32([0] * n), i32(lens))
        c.twin.reserve([0] * n, lens)
        c.same()
        return c

    calls = [("fork", [1, 1], [2, 0], [33, 20]), ("fork", [1], [0], [64]), ("reserve", [40, 80, 0, 20], [0, 20, 50, 40]), ("reserve", [5, 80, 0, 20], [40, 81 - 1, 16, 0])]
    for what, *args in calls:
        run = lambda c: (ctx.fork_pages if what == "fork" else ctx.reserve_pages)(c.pool, c.layers, *[i32(x) for x in args])
        twin = lambda c: getattr(c.twin, what)(*args)
        # the second page of sequence 0
        c = made()
        lost = c.twin.table[0][1]
        c.pool.d_block_table[0, 1] = entry
        run(c), twin(c)
        given_up = c.twin.table[0][1] != lost or c.twin.held[0] < 2
        assert ctx.device_status() == (4 if given_up or what == "reserve" else 0), what
        assert c.pool.d_held.tolist() == c.twin.held and c.pool.d_block_table.tolist()[1:] == c.twin.table[1:]
        refs, free = list(c.twin.refs), c.twin.free[:c.twin.n_free]
        if c.twin.refs[lost] == 0:                                       # nobody can say any more that it was held
            refs[lost] = 1
            free.remove(lost)
        assert c.pool.d_refs.tolist() == refs and c.pool.d_free.tolist()[:int(c.pool.d_n_free)] == free
        # the second page that a call takes
        c = made()
        lost = c.twin.free[c.twin.n_free - 2]
        c.pool.d_free[c.twin.n_free - 2] = entry
        run(c), twin(c)
        taken = c.twin.refs[lost] > 0
        assert ctx.device_status() == (4 if taken else 0)
        got, want = c.pool.d_block_table.tolist(), c.twin.table
        for s in range(n):
            for j in range(5):
                assert got[s][j] == (-1 if want[s][j] == lost and j < c.twin.held[s] else want[s][j]), (what, s, j)
        refs = list(c.twin.refs)
        refs[lost] = 0
        assert c.pool.d_held.tolist() == c.twin.held and c.pool.d_refs.tolist() == refs and int(c.pool.d_n_free) == c.twin.n_free
        if taken:
            assert c.pool.d_free.tolist()[:c.twin.n_free] == c.twin.free[:c.twin.n_free]


@pytest.mark.parametrize("dtype,layers,hkv,dh", [("bf16", 3, 2, 128), ("fp32", 2, 3, 64), ("bf16", 1, 1, 64), ("fp32", 1, 2, 128)])
def test_commit(contexts, dtype, layers, hkv, dh):
    ctx, rng = contexts[dtype], np.random.default_rng(dh)
    nodes, past = [7, 0, 1, 60, 9, 5, 33, 20, 6, 4], [30, 5, 15, 100, 0, 16, 3, 7, 2, 1]
    n = len(nodes)
    lens = [a + b for a, b in zip(nodes, past)]
    c = Cache(dtype, layers, hkv, dh, sum(-(-x // 16) for x in lens) + 4, n, 12)
    ctx.reserve_pages(c.pool, c.layers, i32([0] * n), i32(lens))
    c.twin.reserve([0] * n, lens)
    off = np.concatenate([[0], np.cumsum(nodes)])
    path = np.full((n, 40), -1, dtype=np.int32)
    n_path = np.zeros(n, dtype=np.int32)
    for s in range(n):
        keep = sorted(rng.choice(nodes[s], min(nodes[s], int(rng.integers(1, 40)), 40), replace=False)) if nodes[s] else []
        path[s, :len(keep)], n_path[s] = keep, len(keep)
    path[7, :4], n_path[7] = [3, 4, 4, 9], 4                               # left alone: not ascending, outside, too many
    path[8, :2], n_path[8] = [2, 6], 2
    n_path[9] = 41
    for in_place in (False, True):
        c.lens.copy_(i32(lens))
        before = f64(c.kv)
        want = drafts.commit(before, c.twin.table, lens, off, path, n_path)
        out = c.lens if in_place else torch.full((n,), -9, dtype=torch.int32, device=DEV)
        ctx.commit_path(c.layers, i32(off), i32(path), i32(n_path), out)
        assert ctx.device_status() == 8
        assert out.tolist() == want and np.array_equal(f64(c.kv), before)
        assert want[7:] == lens[7:]


@pytest.mark.parametrize("dtype,layers,hkv,dh", [("fp32", 2, 1, 128), ("bf16", 3, 2, 128), ("fp32", 1, 2, 64), ("bf16", 2, 1, 64)])
def test_commit_of_long_paths(contexts, dtype, layers, hkv, dh):
    """Paths of many batches of rows (64 to 256, by type and head size; places are looked up 256 at a time): nearly every row moves by a few slots,
    onto rows that others come from."""
    ctx, rng = contexts[dtype], np.random.default_rng(dh)
    nodes, past = [300, 400, 129, 700, 65, 257, 0], [5, 37, 100, 1, 16, 0, 9]
    n = len(nodes)
    lens = [a + b for a, b in zip(nodes, past)]
    off = np.concatenate([[0], np.cumsum(nodes)])
    for drops in (1, 5, 60):
        c = Cache(dtype, layers, hkv, dh, sum(-(-x // 16) for x in lens) + 4, n, 48, seed=drops)
        ctx.reserve_pages(c.pool, c.layers, i32([0] * n), i32(lens))
        c.twin.reserve([0] * n, lens)
        path, n_path = np.full((n, 700), -1, dtype=np.int32), np.zeros(n, dtype=np.int32)
        for s in range(n):
            lost = {0} | set(rng.integers(0, max(nodes[s], 1), drops).tolist()) if drops != 5 else set(rng.integers(0, max(nodes[s], 1), drops).tolist())
            keep = [i for i in range(nodes[s]) if i not in lost]
            path[s, :len(keep)], n_path[s] = keep, len(keep)
        c.lens.copy_(i32(lens))
        before = f64(c.kv)
        want = drafts.commit(before, c.twin.table, lens, off, path, n_path)
        ctx.commit_path(c.layers, i32(off), i32(path), i32(n_path), c.lens)
        assert c.lens.tolist() == want and np.array_equal(f64(c.kv), before) and ctx.device_status() == 0


def test_commit_with_bad_tables(contexts):
    ctx = contexts["bf16"]
    c = Cache("bf16", 2, 1, 64, 10, 2, 3)
    c.pool.d_block_table.copy_(i32([[0, 99, 2], [3, -1, 4]]))
    c.lens.copy_(i32([40, 60]))
    ctx.commit_path(c.layers, i32([0, 20, 30]), i32([[5, 19], [0, 9]]), i32([2, 2]), c.lens)
    assert ctx.device_status() == 4 + 8 and c.lens.tolist()[0] == 22


def test_refusals_of_calls_on_layers(contexts):
    ctx = contexts["bf16"]
    c = Cache("bf16", 2, 1, 64, 10, 2, 3)
    other = Cache("bf16", 1, 1, 64, 10, 2, 3)
    with pytest.raises(ValueError):
        rpo.PagedLayers([c.layers.layers[0], other.layers.layers[0]])
    with pytest.raises(ValueError):
        ctx.reserve_pages(other.pool, c.layers, c.lens, c.lens)
    with pytest.raises(ValueError):
        contexts["fp32"].reserve_pages(c.pool, c.layers, c.lens, c.lens)
    many = rpo.PagedLayers([c.layers.layers[0]] * 129)
    with pytest.raises(rpo.RpoError) as e:
        ctx.reserve_pages(c.pool, many, c.lens, c.lens)
    assert e.value.code == -7


# ---- together ------------------------------------------------------------------------------------------------------
def test_a_rollout_with_drafted_tokens():
    """Samples of two questions from cut prefixes, trees of drafted tokens, one attention layer as the model: fork, then step by step
    reserve, tree attention, verification, commit.  Greedy, so every emitted token must be the one that plain decoding (chunks of
    one token on a cache of its own) gives; once step by step, once as a captured graph that is replayed."""
    vocab, hq, hkv, dh, samples, steps, nodes = 211, 4, 2, 64, 3, 6, 7
    g = torch.Generator().manual_seed(3)
    embed = torch.randn(vocab, (hq + 2 * hkv) * dh, generator=g).to(DEV)
    head = (torch.randn(vocab, hq * dh, generator=g) * 2).to(DEV)
    place = torch.randn(400, (hq + 2 * hkv) * dh, generator=g).to(DEV) * 0.5
    prompts = [torch.randint(0, vocab, (n,), generator=g).tolist() for n in (37, 90)]
    cuts = [[37, 30, 16], [90, 71, 64]]

    def project(tokens, positions):
        return (embed[tokens] + place[positions]).reshape(len(tokens), hq + 2 * hkv, dh)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream), make_context("fp32", stream) as ctx:
        def plain(tokens, n_new):
            """Greedy continuation, one token at a time."""
            c = Cache("fp32", 1, hkv, dh, 30, 1, 20)
            got, feed = [], list(tokens)
            for _ in range(n_new):
                ctx.reserve_pages(c.pool, c.layers, c.lens, c.lens + len(feed))
                qkv = project(torch.tensor(feed, device=DEV), torch.arange(int(c.lens), int(c.lens) + len(feed), device=DEV))
                c.lens += len(feed)
                out = torch.empty(len(feed), hq, dh, device=DEV)
                ctx.chunk_attention(qkv[:, :hq], c.layers.layers[0], i32([0, len(feed)]), len(feed), out, d_k_new=qkv[:, hq:hq + hkv], d_v_new=qkv[:, hq + hkv:])
                got.append(int((out[-1].reshape(-1) @ head.T).argmax()))
                feed = [got[-1]]
            return got

        n = 2 + 2 * samples
        c = Cache("fp32", 1, hkv, dh, 120, n, 16)
        lens0 = [len(p) - 1 for p in prompts] + [0] * (n - 2)                # the last token of a prompt is fed as a root
        ctx.reserve_pages(c.pool, c.layers, c.lens, i32(lens0))
        for s, p in enumerate(prompts):
            qkv = project(torch.tensor(p[:-1], device=DEV), torch.arange(len(p) - 1, device=DEV))
            one = torch.zeros(n, dtype=torch.int32, device=DEV)
            one[s] = len(p) - 1
            off = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
            off[s + 1:] = len(p) - 1
            c.lens.copy_(one)
            out = torch.empty(len(p) - 1, hq, dh, device=DEV)
            ctx.chunk_attention(qkv[:, :hq], c.layers.layers[0], off, len(p), out, d_k_new=qkv[:, hq:hq + hkv], d_v_new=qkv[:, hq + hkv:])
        c.lens.copy_(i32(lens0))
        src, dst, cut = [0] * samples + [1] * samples, list(range(2, n)), [x - 1 for row in cuts for x in row]
        ctx.fork_pages(c.pool, c.layers, i32(src), i32(dst), i32(cut), c.lens)
        ctx.reserve_pages(c.pool, c.layers, c.lens, c.lens * (torch.arange(n, device=DEV) >= 2).to(torch.int32))      # the questions themselves leave
        c.lens[:2] = 0
        roots = [prompts[i // samples][cut[i]] for i in range(2 * samples)]
        want = [plain(prompts[i // samples][:cut[i] + 1], steps * 5 + 6) for i in range(2 * samples)]

        rows = 2 * samples * nodes
        parents = i32([-1, 0, 0, 1, 1, 3, 5] * (2 * samples))
        off = i32([0, 0, 0] + [nodes * (i + 1) for i in range(2 * samples)])
        depth = torch.tensor([0, 1, 1, 2, 2, 3, 4] * (2 * samples), device=DEV)
        tokens, uniform = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.rand(rows, device=DEV)
        out, path = torch.empty(rows, hq, dh, device=DEV), torch.zeros(n, 5, dtype=torch.int32, device=DEV)
        n_path, nxt, logp = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n, 5, device=DEV)
        seq_of = torch.arange(2 * samples, device=DEV).repeat_interleave(nodes) + 2
        grows = (torch.arange(n, device=DEV) >= 2).to(torch.int32) * nodes

        def step():
            room = c.lens + grows
            ctx.reserve_pages(c.pool, c.layers, c.lens, room)
            qkv = project(tokens.long(), c.lens.long()[seq_of] + depth)
            c.lens.copy_(room)
            ctx.tree_attention(qkv[:, :hq], c.layers.layers[0], off, parents, nodes, out, d_k_new=qkv[:, hq:hq + hkv], d_v_new=qkv[:, hq + hkv:])
            logits = out.reshape(rows, -1) @ head.T
            ctx.verify_drafts(logits, tokens, parents, off, uniform, rpo.Sampler(greedy=True), path, n_path, nxt, d_logprobs_out=logp)
            ctx.commit_path(c.layers, off, path, n_path, c.lens)

        def drafts_for(i, done, rng):
            """Root and drafts: the true continuation at some nodes, something else at others."""
            ahead = [([roots[i]] + want[i])[done + d] for d in range(5)]
            got = [ahead[0]] + [0] * 6
            for node, d in ((1, 1), (2, 1), (3, 2), (4, 2), (5, 3), (6, 4)):
                got[node] = ahead[d] if rng.random() < 0.6 else int(rng.integers(vocab))
            return got

        rng, got = np.random.default_rng(0), [[] for _ in range(2 * samples)]
        graph = None
        for k in range(steps):
            tokens.copy_(i32([t for i in range(2 * samples) for t in drafts_for(i, len(got[i]), rng)]))
            feed = tokens.view(-1, nodes).tolist()
            if k < 2:
                step()
            else:
                if graph is None:
                    torch.cuda.synchronize()
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph, stream=stream):
                        step()
                graph.replay()
            torch.cuda.synchronize()
            for i in range(2 * samples):
                p = path[i + 2, :int(n_path[i + 2])].tolist()
                got[i] += [feed[i][j] for j in p[1:]] + [int(nxt[i + 2])]
        assert ctx.device_status() == 0
        for i in range(2 * samples):
            m = min(len(got[i]), len(want[i]))
            assert got[i][:m] == want[i][:m] and len(got[i]) >= steps
        assert max(len(x) for x in got) > steps                              # some drafts were accepted
        held = c.pool.d_held.tolist()
        counts = np.bincount([p for s, row in enumerate(c.pool.d_block_table.tolist()) for p in row[:held[s]]], minlength=120)
        assert c.pool.d_refs.tolist() == counts.tolist() and int(c.pool.d_n_free) == int((counts == 0).sum())
        del graph


# ---- beside one another, and far into memory -----------------------------------------------------------------------
def test_two_contexts_on_two_streams_at_once():
    """Workspaces belong to a context: calls of two contexts that overlap give what they give alone."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    made = [make_context("bf16", s) for s in streams]
    cases = [Tree("bf16", 12, 2, 128, [40, 60], [3000, 900], seed=k) for k in range(2)]
    checks = [Drafts(5003, TREES, seed=k, top_p=0.9) for k in range(2)]
    alone = [(c.attend(x), d.run(x)) for x, c, d in zip(made, cases, checks)]
    outs = [[(torch.zeros_like(a[0][0]), torch.zeros_like(a[0][1])) for _ in range(10)] for a in alone]
    torch.cuda.synchronize()
    for i in range(10):
        for x, c, o in zip(made, cases, outs):
            x.tree_attention(c.q, c.kv, c.d_off, c.d_parents, c.max_nodes, *o[i])
    torch.cuda.synchronize()
    for a, o in zip(alone, outs):
        assert all(torch.equal(y, a[0][0]) and torch.equal(z, a[0][1]) for y, z in o)
    for x, d, a in zip(made, checks, alone):
        assert all(torch.equal(y, z) for y, z in zip(d.run(x), a[1]))
        assert x.device_status() == 0
        x.close()


@pytest.mark.parametrize("n", [2, 30])
def test_a_captured_step_follows_parents_lengths_and_numbers(n):
    """Attention and verification replayed from a graph with other trees, lengths, tokens and random numbers in the same buffers."""
    s = torch.cuda.Stream()
    with make_context("bf16", s) as ctx:
        first, second = (Tree("bf16", 12, 2, 128, [n, n, n], past, seed=k, holes=0.2 * k) for k, past in ((0, [200, 3, 50]), (1, [90, 77, 0])))
        stride = first.kv.d_block_table.shape[1]
        c = Drafts(997, [t for t in ([list(range(-1, n - 1))] * 3)], seed=1, top_p=0.9)
        d = Drafts(997, [random_tree(n, np.random.default_rng(k)) for k in range(3)], seed=2, top_p=0.9, max_path=c.max_path)
        out, lse = torch.zeros_like(first.q.contiguous()), torch.zeros(first.q.shape[:2], device=DEV)
        buf = [torch.from_numpy(np.array(x)).to(DEV) for x in (c.logits, c.probs, c.tokens, c.parents, c.uniform)]
        off = i32(c.off)
        path, n_path, nxt = (torch.zeros(x, dtype=torch.int32, device=DEV) for x in ((3, c.max_path), (3,), (3,)))
        logp = torch.zeros(3, c.max_path, device=DEV)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ctx.tree_attention(first.q, first.kv, first.d_off, first.d_parents, n, out, lse)
            ctx.verify_drafts(buf[0], buf[2], buf[3], off, buf[4], rpo.Sampler(1.0, 0.9), path, n_path, nxt, logp, d_draft_probs=buf[1])
        torch.cuda.synchronize()
        for tree, drafted in ((first, c), (second, d), (first, c)):
            if tree is second:                                            # into the buffers that were captured
                keep = first.k.clone(), first.v.clone(), first.q.clone()
                blocks = min(first.k.shape[1], second.k.shape[1])
                used = second.table[second.table >= 0]
                assert used.max() < blocks or second.k.shape[1] <= first.k.shape[1]
                first.k[:, :blocks], first.v[:, :blocks] = second.k[:, :blocks], second.v[:, :blocks]
                first.q.copy_(second.q)
            elif tree is first and drafted is c and "keep" in dir():
                first.k.copy_(keep[0]); first.v.copy_(keep[1]); first.q.copy_(keep[2])
            width = min(stride, tree.table.shape[1])
            first.kv.d_block_table.fill_(-1)
            first.kv.d_block_table[:, :width] = i32(tree.table[:, :width])
            first.kv.d_lens.copy_(i32(tree.lens))
            first.d_parents.copy_(i32(tree.parents))
            for b, x in zip(buf, (drafted.logits, drafted.probs, drafted.tokens, drafted.parents, drafted.uniform)):
                b.copy_(torch.from_numpy(np.array(x)))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            tree.check(out, lse)
            drafted.check(path, n_path, nxt, logp)
        assert ctx.device_status() == 0
        del graph


def test_pools_beyond_32_bit_offsets(contexts):
    """The last pages of a pool of more than 2^32 bytes: attention, copies and moves."""
    ctx, hkv, blocks, dh = contexts["bf16"], 4, (1 << 18) + 40, 128
    k, v = (torch.zeros(hkv, blocks, 16, dh, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pool = rpo.PagePool.empty(blocks, 2, 8, DEV)
    pool.d_free.copy_(torch.arange(blocks, dtype=torch.int32, device=DEV))          # the last pages on top
    lens = torch.zeros(2, dtype=torch.int32, device=DEV)
    kv = rpo.PagedKV(k, v, pool.d_block_table, lens)
    layers = rpo.PagedLayers([kv])
    ctx.reserve_pages(pool, layers, lens, i32([60, 0]))
    g = torch.Generator(DEV).manual_seed(0)
    new = torch.randn(60, 8 + 2 * hkv, dh, device=DEV, generator=g).to(torch.bfloat16)
    q, kn, vn = new[:, :8], new[:, 8:8 + hkv], new[:, 8 + hkv:]
    lens.copy_(i32([60, 0]))
    out = torch.zeros(60, 8, dh, dtype=torch.bfloat16, device=DEV)
    parents = i32(range(-1, 59))
    ctx.tree_attention(q, kv, i32([0, 60, 60]), parents, 60, out, d_k_new=kn, d_v_new=vn)
    ctx.fork_pages(pool, layers, i32([0]), i32([1]), i32([55]), lens)
    ctx.commit_path(layers, i32([0, 4, 4]), i32([[0, 3], [0, 0]]), i32([2, 0]), lens)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0 and lens.tolist() == [58, 55]
    table = pool.d_block_table.tolist()
    assert min(table[0][:4] + table[1][3:4]) > (1 << 18) and table[0][:3] == table[1][:3] and table[0][3] != table[1][3]
    for cache, want in ((k, kn), (v, vn)):
        assert torch.equal(cache[:, table[0][3], :8], want[48:56].transpose(0, 1)) and torch.equal(cache[:, table[0][3], 8], want[56]) and torch.equal(cache[:, table[0][3], 9], want[59])
        assert torch.equal(cache[:, table[1][3], :7], want[48:55].transpose(0, 1)) and not cache[:, table[1][3], 7:].any()
    z = torch.einsum("rhd,khd->hrk", q[:, ::2].double(), kn.double()) * dh ** -0.5
    w = torch.softmax(z.masked_fill(~torch.tril(torch.ones(60, 60, dtype=torch.bool, device=DEV)), -float("inf")), -1)
    want = torch.einsum("hrk,khd->rhd", w, vn.double())
    scale = torch.einsum("hrk,khd->rhd", w, vn.double().abs())
    assert torch.all((out[:, ::2].double() - want).abs() <= scale * (2.0 ** -8 + 2.0 ** -18) + 2.0 ** -8 * want.abs())
