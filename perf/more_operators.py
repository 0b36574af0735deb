"""Measured cases of the operators that rollouts with drafted tokens and shared prefixes run on a caller-owned paged cache.

  tree     attention of a tree of drafted tokens per sequence: every node sees the cached tokens and its own ancestors; the
           nodes' K and V are written to their pages
  verify   the drafted tokens against the target's distribution with given random numbers: the accepted path, the token
           drawn behind it and the log-probabilities of both
  commit   the accepted nodes' K and V, of all layers, move to the front of the tree's slots
  fork     sequences become the first tokens of others: whole pages are shared, the last one is copied
  reserve  sequences take the pages that their next tokens need, or give back what they hold

`run` computes them in plain torch operations, or with the library's calls where `own` is set.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
# (query heads, KV heads, head dim): the decoder shapes of the workloads, and generic ones
_HEADS = [(12, 2, 128), (28, 4, 128), (4, 2, 64), (8, 8, 64), (8, 1, 128), (32, 8, 128)]


def _tree(name, dtype, heads, n_seqs, nodes, past_lo, past_hi, window=0, sinks=0, padded=False):
    return {"name": name, "op": "tree", "dtype": dtype, "hq": heads[0], "hkv": heads[1], "dh": heads[2], "n_seqs": n_seqs, "nodes": nodes,
            "branch": 3, "past_lo": past_lo, "past_hi": past_hi, "window": window, "sinks": sinks, "padded": padded}


def _verify(name, n_seqs, nodes, branch, vocab, temperature, top_p, drafts):
    return {"name": name, "op": "verify", "n_seqs": n_seqs, "nodes": nodes, "branch": branch, "vocab": vocab, "temperature": temperature,
            "top_p": top_p, "drafts": drafts}


def _pages(name, op, layers, heads, n_seqs, len_lo, len_hi, **more):
    return {"name": name, "op": op, "dtype": "bf16", "layers": layers, "hkv": heads[1], "dh": heads[2], "n_seqs": n_seqs, "len_lo": len_lo,
            "len_hi": len_hi, **more}


def listed():
    return [
        # eight drafted tokens for each of a few short sequences: what the call costs when there is little to read
        _tree("tree_small", "bf16", (12, 2, 128), 4, 8, 100, 300),
        # trees of sixteen drafted tokens for a batch over long ragged prefixes (the 7B-class shape)
        _tree("tree_batch", "bf16", (28, 4, 128), 64, 16, 1024, 6144),
        # large trees on two long sequences: many rows for every key, few sequences to share the work over
        _tree("tree_long", "bf16", (28, 4, 128), 2, 48, 40000, 60001),
        # 32-bit trees under a window with first tokens that stay visible, padded to one size, nothing divisible by anything
        _tree("tree_window", "fp32", (4, 2, 64), 3, 33, 0, 1500, window=500, sinks=3, padded=True),
        # eight tokens of a draft model for every sequence of a batch, its probabilities given, sampled as the rollouts are
        _verify("verify_chain", 128, 9, 1, 152064, 1.0, 0.95, True),
        # a few trees of tokens that were looked up or ranked, not drawn
        _verify("verify_tree", 4, 24, 3, 151936, 0.7, 1.0, False),
        # eight samples of one question continue its cached path from where it was cut (1.5B-class shape, all layers)
        _pages("fork_few", "fork", 28, (12, 2, 128), 1, 500, 1500, samples=8),
        # the same for a batch of questions (7B-class shape, all layers)
        _pages("fork_groups", "fork", 28, (28, 4, 128), 16, 1024, 3000, samples=8),
        # accepted tokens of a few small trees
        _pages("commit_few", "commit", 28, (12, 2, 128), 4, 100, 300, nodes=8),
        # accepted tokens of a batch of trees (7B-class shape, all layers)
        _pages("commit_batch", "commit", 28, (28, 4, 128), 64, 500, 1500, nodes=16),
        # room for the next sixteen tokens of every sequence of a batch, given back afterwards
        _pages("reserve_step", "reserve", 28, (12, 2, 128), 128, 100, 700, grow=16, empty=False),
        # a batch begins and ends: all pages of long sequences taken and given back
        _pages("reserve_batch", "reserve", 1, (28, 4, 128), 256, 1024, 6144, grow=256, empty=True),
    ]


_MOST_PAIRS = 28 * 48 * 2 * 60001           # (query row, key) pairs of the largest listed tree call
_MOST_ROWS = 64 * 4 * 6144 * 128            # cache elements of K of the largest listed cache
_MOST_VOCAB = 128 * 9 * 152064              # logits of the largest listed verification
_MOST_POOL = 28 * 4 * 128 * PAGE * 3200     # elements of K of the largest listed pool of all layers


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "verify", "verify", "fork", "commit", "reserve"])
    if op == "tree":
        dtype, heads = rng.choice(["bf16", "bf16", "bf16", "fp32"]), rng.choice(_HEADS)
        hq, hkv, dh = heads
        nodes, hi = _log(rng, 1, 256), rng.choice([_log(rng, 1, 200), _log(rng, 200, 20000), _log(rng, 200, 20000)])
        lo = rng.choice([hi, hi // 4, 0])
        pairs = _MOST_PAIRS // (8 if dtype == "fp32" else 1)
        n_seqs = max(1, min(_log(rng, 1, 128), pairs // (hq * nodes * (hi + nodes)), _MOST_ROWS // (hkv * (hi + nodes) * dh)))
        window = rng.choice([0, 0, _log(rng, 1, 4096)])
        case = _tree("", dtype, heads, n_seqs, nodes, lo, hi, window, rng.randint(0, 40) if window else 0, rng.random() < 0.4)
        case["branch"] = rng.randint(1, 6)
    elif op == "verify":
        nodes, vocab, branch = _log(rng, 1, 64), _log(rng, 1000, 152064), rng.randint(1, 4)
        levels = nodes if branch == 1 else min(nodes, 12)
        n_seqs = max(1, min(_log(rng, 1, 128), _MOST_VOCAB // (vocab * levels), _MOST_VOCAB // (vocab * nodes)))
        case = _verify("", n_seqs, nodes, branch, vocab, rng.choice([1.0, 0.7, 1.3]), rng.choice([1.0, 0.95, 0.9, 0.5]), rng.random() < 0.5)
    else:
        heads, layers = rng.choice(_HEADS), rng.choice([1, 4, 28])
        hi = _log(rng, 20, 6000)
        per_token = layers * heads[1] * heads[2]
        n_seqs = max(1, min(_log(rng, 1, 256), _MOST_POOL // (per_token * (hi + 300))))
        more = ({"samples": rng.randint(1, 16)} if op == "fork" else {"nodes": _log(rng, 1, 64)} if op == "commit"
                else {"grow": _log(rng, 1, 256), "empty": rng.random() < 0.3})
        if op == "fork":
            n_seqs = max(1, min(n_seqs // 2, _MOST_POOL // (per_token * (hi + 32 * more["samples"] + PAGE))))
        case = _pages("", op, layers, heads, n_seqs, rng.choice([hi, hi // 4 + 1]), hi, **more)
    return {k: v for k, v in case.items() if k != "name"}


def _rng(case):
    return np.random.RandomState((case["n_seqs"] * 7919 + case.get("nodes", 5) * 31 + case.get("len_hi", case.get("past_hi", case.get("vocab", 0)))) % (1 << 31))


def _between(rng, lo, hi, n):
    x = rng.randint(lo, hi + 1, n)
    x[rng.randint(n)] = hi
    return x


def _trees(case, rng):
    """Parents of every sequence's nodes (-1: the last cached token), each before its children; at most `branch` children."""
    got = []
    for _ in range(case["n_seqs"]):
        n = case["nodes"]
        kids, parent = np.zeros(n, dtype=int), np.full(n, -1)
        for i in range(1, n):
            open_ = np.flatnonzero(kids[:i] < case["branch"])
            parent[i] = open_[-1] if case["branch"] == 1 else open_[int(len(open_) * rng.rand() ** 2)]
            kids[parent[i]] += 1
        got.append(parent)
    return got


def _depths(parent):
    d = np.zeros(len(parent), dtype=int)
    for i in range(1, len(parent)):
        d[i] = d[parent[i]] + 1 if parent[i] >= 0 else 0
    return d


_contexts = {}


def _context(dtype):
    """The library context of a storage type: a program keeps one for all its calls."""
    import paper_2601_19404_b200 as rpo
    if dtype not in _contexts:
        shape = rpo.shape_preset("tiny", dtype=1 if dtype == "bf16" else 0)
        _contexts[dtype] = rpo.Context(shape, kv_pool_blocks=16, max_groups=1, max_seqs=1, max_chunk_tokens=32, max_positions=64)
    return _contexts[dtype]


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _offsets(counts):
    return _i32(np.concatenate([[0], np.cumsum(counts)]))


def _table(pages, stride, order):
    """Block table of sequences with `pages` pages each, taken from `order` in turn; -1 behind them."""
    first = torch.from_numpy(np.concatenate([[0], np.cumsum(pages)[:-1]])).cuda()
    slot = torch.arange(stride, device="cuda")
    inside = slot[None, :] < torch.from_numpy(pages).cuda()[:, None]
    return torch.where(inside, order[(first[:, None] + slot[None, :]).clamp(max=len(order) - 1)], -1).to(torch.int32).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = _rng(case)
    return {"tree": _prepare_tree, "verify": _prepare_verify}.get(case["op"], _prepare_pages)(case, g, rng)


def _prepare_tree(case, g, rng):
    dt, hq, hkv, dh, n, c = _DTYPES[case["dtype"]], case["hq"], case["hkv"], case["dh"], case["n_seqs"], case["nodes"]
    past = _between(rng, case["past_lo"], case["past_hi"], n)
    parents = np.stack(_trees(case, rng))
    if case["padded"]:                     # some trees are smaller than the size that all are padded to
        live = _between(rng, 1, c, n)
        parents[np.arange(c)[None, :] >= live[:, None]] = -2
    lens = past + c
    pages = -(-lens // PAGE)
    n_blocks = int(pages.sum()) + 5
    order = torch.randperm(n_blocks, generator=g, device="cuda", dtype=torch.int32)
    k, v = (torch.randn(hkv, n_blocks, PAGE, dh, generator=g, device="cuda").to(dt) for _ in range(2))
    # queries, keys and values of the drafted tokens as one fused projection leaves them
    qkv = torch.randn(n * c, hq + 2 * hkv, dh, generator=g, device="cuda")
    qkv[:, :hq] *= 1.5
    qkv = qkv.to(dt)
    st = {"case": case, "k": k, "v": v, "table": _table(pages, int(pages.max()) + 3, order), "lens": _i32(lens), "offsets": _offsets(np.full(n, c)),
          "parents": _i32(parents.reshape(-1)), "q": qkv[:, :hq], "k_new": qkv[:, hq:hq + hkv], "v_new": qkv[:, hq + hkv:]}
    if own:
        import paper_2601_19404_b200 as rpo
        st["ctx"], st["kv"] = _context(case["dtype"]), rpo.PagedKV(k, v, st["table"], st["lens"])
    return st


def _prepare_verify(case, g, rng):
    n, c, vocab = case["n_seqs"], case["nodes"], case["vocab"]
    parents = np.stack(_trees(case, rng))
    levels = max(int(_depths(p).max()) for p in parents) + 1
    rank = np.zeros((n, c), dtype=np.int64)             # of a node among its parent's children
    for s in range(n):
        seen = {}
        for i in range(1, c):
            rank[s, i] = seen.get(parents[s, i], 0)
            seen[parents[s, i]] = rank[s, i] + 1
    # logits of a trained model are peaked, some rows more than others; the draft model's are near them
    logits = torch.randn(n * c, vocab, generator=g, device="cuda")
    logits *= torch.empty(n * c, 1, device="cuda").uniform_(2.5, 5.0, generator=g)
    draft = torch.randn(n * c, vocab, generator=g, device="cuda").mul_(0.8).add_(logits)
    at = torch.from_numpy((np.arange(n)[:, None] * c + np.maximum(parents, 0)).reshape(-1)).cuda()
    tokens = torch.randint(0, vocab, (n * c,), generator=g, device="cuda")
    inner = torch.from_numpy((parents >= 0).reshape(-1)).cuda()
    st = {"case": case, "logits": logits, "offsets": _offsets(np.full(n, c)), "parents": _i32(parents.reshape(-1)),
          "uniform": torch.rand(n * c, generator=g, device="cuda"), "levels": levels}
    if case["drafts"]:                                  # children drawn from the draft model's distribution
        probs = draft.div_(case["temperature"])
        probs.sub_(probs.amax(1, keepdim=True)).exp_()
        probs.div_(probs.sum(1, keepdim=True))
        drawn = torch.stack([(probs[a] / torch.empty(vocab, device="cuda").exponential_(1.0, generator=g)).argmax() for a in at.tolist()])
        tokens = torch.where(inner, drawn, tokens)
        st["probs"] = probs
    else:                                               # children ranked by the draft model
        best = draft.topk(case["branch"], 1)[1]
        tokens = torch.where(inner, best[at, torch.from_numpy(rank.reshape(-1)).cuda()], tokens)
        st["probs"] = None
    st["tokens"] = tokens.to(torch.int32)
    st["path"], st["logprobs"] = torch.zeros(n, levels, dtype=torch.int32, device="cuda"), torch.zeros(n, levels, device="cuda")
    st["n_path"], st["next"] = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
    if own:
        import paper_2601_19404_b200 as rpo
        st["ctx"], st["sampler"] = _context("bf16"), rpo.Sampler(case["temperature"], case["top_p"])
    return st


def _lengths(case, rng):
    lens = _between(rng, case["len_lo"], case["len_hi"], case["n_seqs"])
    # reserve: every second sequence is a copy of the one before it, all of its pages shared
    return np.repeat(lens[::2], 2)[:len(lens)] if case["op"] == "reserve" else lens


def _prepare_pages(case, g, rng):
    op, n, layers, hkv, dh, dt = case["op"], case["n_seqs"], case["layers"], case["hkv"], case["dh"], _DTYPES[case["dtype"]]
    lens = _lengths(case, rng)
    room = lens + (case["nodes"] if op == "commit" else case["grow"] if op == "reserve" else 0)
    held = -(-room // PAGE) if op == "commit" else 0 * lens if op == "reserve" and case["empty"] else -(-lens // PAGE)
    copies = n * case["samples"] if op == "fork" else 0
    n_blocks = int(np.maximum(held, -(-room // PAGE)).sum()) + 2 * copies + n + 5
    order = torch.randperm(n_blocks, generator=g, device="cuda", dtype=torch.int32)
    own_pages = held * (np.arange(n) % 2 == 0) if op == "reserve" else held
    used, stride = int(own_pages.sum()), int(-(-room.max() // PAGE)) + 3
    table = _table(np.concatenate([own_pages, np.zeros(copies, dtype=held.dtype)]), stride, order)
    if op == "reserve":
        table[1::2] = table[:-1:2][:n // 2]
    refs = torch.zeros(n_blocks, dtype=torch.int32, device="cuda")
    refs.index_add_(0, table[table >= 0].long(), torch.ones_like(table[table >= 0]))
    st = {"case": case, "kv": torch.randn(layers, 2, hkv, n_blocks, PAGE, dh, generator=g, device="cuda", dtype=dt), "table": table, "refs": refs,
          "held": _i32(np.concatenate([held, np.zeros(copies)])), "free": torch.cat([order[used:], order[:used]]).contiguous(), "n_free": _i32([n_blocks - used]),
          "lens": _i32(np.concatenate([lens, np.zeros(copies)]))}
    if op == "fork":
        # every sample continues its question's path from where that was cut
        st["src"] = _i32(np.repeat(np.arange(n), case["samples"]))
        st["dst"] = _i32(n + rng.permutation(copies))
        cut = torch.rand(n, generator=g, device="cuda") * 0.3
        st["cut"] = (st["lens"][:n] * (1 - cut)).to(torch.int32)[st["src"].long()].clamp(min=1).contiguous()
    elif op == "commit":
        c = case["nodes"]
        st["lens"] = _i32(room)
        st["offsets"], st["lens_out"] = _offsets(np.full(n, c)), torch.zeros(n, dtype=torch.int32, device="cuda")
        keep = torch.rand(n, c, generator=g, device="cuda") < 0.3          # accepted nodes: the root, and some of the others
        keep[:, 0] = True
        st["n_path"] = keep.sum(1).to(torch.int32)
        i = torch.arange(c, device="cuda")
        st["path"] = torch.sort(torch.where(keep, i, c), 1)[0]
        st["path"] = torch.where(st["path"] < c, st["path"], -1).to(torch.int32).contiguous()
    else:
        st["room"], st["back"] = _i32(room), _i32(0 * lens if case["empty"] else lens)
        if case["empty"]:
            st["lens"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    if own:
        import paper_2601_19404_b200 as rpo
        st["ctx"] = _context(case["dtype"])
        st["layers"] = rpo.PagedLayers([rpo.PagedKV(st["kv"][i, 0], st["kv"][i, 1], table, st["lens"]) for i in range(layers)])
        st["pool"] = rpo.PagePool(st["refs"], st["free"], st["n_free"], table, st["held"])
    return st


# ------------------------------------------------------------------------------------------------------------
# plain forms
# ------------------------------------------------------------------------------------------------------------
def _gather(cache, table):
    """[n_seqs, KV heads, tokens, head dim] in 32 bits of a paged cache."""
    rows = cache[:, table.clamp(min=0).long()].float()
    return rows.permute(1, 0, 2, 3, 4).reshape(table.shape[0], cache.shape[0], -1, cache.shape[3])


def _ancestors(parents):
    """[n_seqs, nodes, nodes]: is the second node the first one or one of its ancestors; which nodes there are."""
    n, c = parents.shape
    own_ = torch.eye(c, device=parents.device)
    step = torch.zeros(n, c, c, device=parents.device).scatter_(2, parents.clamp(min=0).long()[..., None], (parents >= 0).float()[..., None])
    reach = own_ + step
    for _ in range(max(1, (c - 1).bit_length())):
        reach = (torch.matmul(reach, reach) > 0).float()
    lost = torch.matmul(reach, (parents < -1).float()[..., None])[..., 0] > 0
    return (reach > 0) & ~lost[..., None], ~lost


def _tree_plain(st):
    case = st["case"]
    n, c, hq, hkv, dh, k, v = case["n_seqs"], case["nodes"], case["hq"], case["hkv"], case["dh"], st["k"], st["v"]
    rep = hq // hkv
    reach, exists = _ancestors(st["parents"].view(n, c))
    past = (st["lens"] - c).long()
    slot = past[:, None] + torch.arange(c, device=k.device)
    at = (st["table"].gather(1, slot // PAGE).long() * PAGE + slot % PAGE)[exists]
    for cache, new in ((k, st["k_new"]), (v, st["v_new"])):
        cache.view(hkv, -1, dh)[:, at] = new[exists.view(-1)].transpose(0, 1)
    keys, values = _gather(k, st["table"]), _gather(v, st["table"])
    # positions of the cached tokens and of the nodes' slots
    depth = reach.sum(-1) - 1
    key = torch.arange(keys.shape[2], device=k.device)
    node = key[None, :] - past[:, None]
    inside = (node >= 0) & (node < c)
    at_node = node.clamp(0, c - 1)
    pos = torch.where(inside, past[:, None] + depth.gather(1, at_node), key[None, :])
    here = past[:, None] + depth
    seen = torch.where(inside[:, None], reach.gather(2, at_node[:, None].expand(-1, c, -1)), node[:, None] < 0) & exists[..., None]
    if case["window"]:
        seen &= (pos[:, None] > here[..., None] - case["window"]) | (pos[:, None] < case["sinks"])
    q = st["q"].float().reshape(n, c, hkv, rep, dh).permute(0, 2, 3, 1, 4).reshape(n, hkv, rep * c, dh)
    s = torch.matmul(q, keys.transpose(2, 3)).reshape(n, hkv, rep, c, -1)
    s *= 1.0 / math.sqrt(dh)
    s.masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    e = torch.exp(s.sub_(top))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.reshape(n, hkv, rep * c, -1), values).reshape(n, hkv, rep, c, dh)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (torch.log(total) + top)[..., 0]
    return o.permute(0, 3, 1, 2, 4).reshape(n * c, hq, dh).to(st["q"].dtype), lse.permute(0, 3, 1, 2).reshape(n * c, hq).contiguous()


_LN2_HI = 0.693145751953125
_EXP = [1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0]


def _exp(x):
    """exp of 32-bit numbers <= 0 as the sampler defines it: additions and products, each rounded; 0 below -24."""
    dead = x < -24.0
    x = torch.where(dead, torch.zeros_like(x), x)
    n = torch.round(x * np.float32(math.log2(math.e)).item())
    r = x - n * _LN2_HI
    r = r - n * np.float32(math.log(2.0) - _LN2_HI).item()
    p = torch.full_like(r, np.float32(_EXP[0]).item())
    for coefficient in _EXP[1:]:
        p = p * r
        p = p + np.float32(coefficient).item()
    scale = ((n.to(torch.int32) + 127) << 23).view(torch.float32)
    return torch.where(dead, torch.zeros_like(p), p * scale)


def _share(mass, u24):
    """(mass * u24) >> 24 of whole numbers below 2^48 and 2^24."""
    return (mass >> 24) * u24 + (((mass & 0xFFFFFF) * u24) >> 24)


def _verify_plain(st):
    case, logits, probs, levels = st["case"], st["logits"], st["probs"], st["levels"]
    n, c, dev = case["n_seqs"], case["nodes"], logits.device
    parents, tokens = st["parents"].view(n, c).long(), st["tokens"].view(n, c).long()
    u24 = (st["uniform"].view(n, c) * 16777216.0).long().clamp(0, (1 << 24) - 1)
    first, who, temperature = torch.arange(n, device=dev) * c, torch.arange(n, device=dev), torch.full((1,), case["temperature"], device=dev)
    share = int(math.floor(np.float32(case["top_p"]) * np.float32(2.0 ** 24)))
    path, logp = torch.full((n, levels), -1, dtype=torch.int32, device=dev), torch.zeros(n, levels, device=dev)
    n_path, nxt = torch.zeros(n, dtype=torch.int32, device=dev), torch.full((n,), -1, dtype=torch.int32, device=dev)
    cur, live = torch.zeros(n, dtype=torch.long, device=dev), torch.ones(n, dtype=torch.bool, device=dev)
    for level in range(levels):
        path[:, level] = torch.where(live, cur, -1).to(torch.int32)
        n_path += live.to(torch.int32)
        # the sampler's weights of the node's row: whole numbers, those outside the nucleus 0
        z = logits[first + cur] / temperature
        z -= z.amax(1, keepdim=True)
        e = _exp(z)
        a = (e * 1073741824.0).long()
        if share < 1 << 24:
            down = torch.sort(a, 1, descending=True)[0]
            run_ = down.cumsum(1)
            k = (run_ >= _share(run_[:, -1], share)[:, None]).to(torch.int8).argmax(1)
            a = torch.where(a >= down.gather(1, k[:, None]), a, 0)
        mass = a.sum(1)
        # the node's children in order
        kid = (parents == cur[:, None]) & (level + 1 < levels)
        taken = torch.full((n,), -1, dtype=torch.long, device=dev)
        for _ in range(case["branch"]):
            at = kid.to(torch.int8).argmax(1)
            is_, token = kid.any(1) & (taken < 0), tokens[who, at][:, None]
            kid[who, at] = False
            if probs is None:
                d = torch.zeros_like(a).scatter_(1, token, mass[:, None])
            else:
                d = (probs[first + cur].double() * mass[:, None].double()).long()
            accept = is_ & (_share(d.gather(1, token)[:, 0], u24[who, at]) < a.gather(1, token)[:, 0])
            taken = torch.where(accept, at, taken)
            less = (a - d).clamp_(min=0)
            left = less.sum(1)
            refuse = is_ & ~accept & (left > 0)
            a, mass = torch.where(refuse[:, None], less, a), torch.where(refuse, left, mass)
        # without an accepted child: a token drawn from what is left
        r = _share(mass, u24[:, 0])
        drawn = (a.cumsum(1) > r[:, None]).to(torch.int8).argmax(1)
        ends = live & (taken < 0)
        nxt = torch.where(ends, drawn.to(torch.int32), nxt)
        emitted = torch.where(ends, drawn, tokens[who, taken.clamp(min=0)])
        logp[:, level] = torch.where(live, z.gather(1, emitted[:, None])[:, 0] - torch.log(e.sum(1)), 0.0)
        live, cur = live & (taken >= 0), taken.clamp(min=0)
    return {"path": path, "n_path": n_path, "next": nxt, "logprobs": logp}


def _release(st, dropped, pages):
    """One reference less for every page of `pages` where `dropped` says so; pages without any go on the stack in order."""
    refs, flat, drop = st["refs"], pages.clamp(min=0).long().reshape(-1), dropped.reshape(-1)
    refs -= torch.zeros_like(refs).index_add_(0, flat, drop.to(torch.int32))
    order = torch.arange(len(flat), device=flat.device)
    earliest = torch.full((len(refs),), len(flat), device=flat.device).scatter_reduce_(0, flat, torch.where(drop, order, len(flat)), "amin")
    goes = drop & (refs[flat] == 0) & (earliest[flat] == order)
    to = torch.where(goes, st["n_free"].long() + goes.long().cumsum(0) - 1, len(refs))
    st["free"].copy_(torch.cat([st["free"], st["free"][:1]]).scatter_(0, to, flat.to(torch.int32))[:len(refs)])
    st["n_free"] += goes.sum().to(torch.int32)


def _copy_rows(st, do, frm, to, rows):
    """The first `rows` tokens of pages frm to pages to, of all layers, where `do`."""
    i, t = torch.nonzero(do[:, None] & (torch.arange(PAGE, device=do.device) < rows[:, None]), as_tuple=True)
    st["kv"][:, :, :, to[i].long(), t] = st["kv"][:, :, :, frm[i].long(), t]


def _fork_plain(st):
    """dst[i] becomes the first cut[i] tokens of src[i].  (The cases' forks are all within the pool.)"""
    table, held, refs, src, dst, cut = st["table"], st["held"], st["refs"], st["src"].long(), st["dst"].long(), st["cut"].long()
    whole, rest = cut // PAGE, cut % PAGE
    needs = rest > 0
    slot = torch.arange(table.shape[1], device=table.device)
    shared = slot < whole[:, None]
    old, dropped = table[dst].clone(), slot < held[dst][:, None]
    from_ = table[src]
    refs += torch.zeros_like(refs).index_add_(0, from_.clamp(min=0).long().reshape(-1), shared.reshape(-1).to(torch.int32))
    taken = needs.long().cumsum(0)
    page = st["free"][(st["n_free"].long() - taken).clamp(min=0)]
    refs += torch.zeros_like(refs).index_add_(0, page.long(), needs.to(torch.int32))
    last = from_.gather(1, whole[:, None])[:, 0]
    now = torch.where(shared, from_, torch.where((slot == whole[:, None]) & needs[:, None], page[:, None], old))
    table[dst] = now
    held[dst] = (whole + needs).to(torch.int32)
    st["lens"][dst] = cut.to(torch.int32)
    st["n_free"] -= taken[-1].to(torch.int32)
    _copy_rows(st, needs, last, page, rest)
    _release(st, dropped, old)


def _reserve_plain(st, target):
    """Pages for `target` tokens; those behind the first lens tokens are the sequence's own.  (The pool has enough.)"""
    table, held, refs, lens = st["table"], st["held"].long(), st["refs"], torch.minimum(st["lens"], target).long()
    want = (target.long() + PAGE - 1) // PAGE
    slot = torch.arange(table.shape[1], device=table.device)
    has = slot < held[:, None]
    others = has & (refs[table.clamp(min=0).long()] > 1)
    fresh = (slot < want[:, None]) & (~has | (others & (slot >= (lens // PAGE)[:, None])))
    dropped = has & ((slot >= want[:, None]) | fresh)
    nth = fresh.reshape(-1).long().cumsum(0)
    page = st["free"][(st["n_free"].long() - nth).clamp(min=0)].view(table.shape)
    old = table.clone()
    refs += torch.zeros_like(refs).index_add_(0, page.reshape(-1).long(), fresh.reshape(-1).to(torch.int32))
    table.copy_(torch.where(fresh, page, table))
    st["held"].copy_(want)
    st["n_free"] -= nth[-1].to(torch.int32)
    at = (lens // PAGE).clamp(max=table.shape[1] - 1)[:, None]
    _copy_rows(st, (dropped & fresh).gather(1, at)[:, 0], old.gather(1, at)[:, 0], page.gather(1, at)[:, 0], lens % PAGE)
    _release(st, dropped, old)


def _commit_plain(st):
    past = (st["lens"] - (st["offsets"][1:] - st["offsets"][:-1])).long()
    i, t = torch.nonzero(st["path"] >= 0, as_tuple=True)
    row = lambda slot: (st["table"][i, slot // PAGE].long(), slot % PAGE)  # noqa: E731
    (b0, r0), (b1, r1) = row(past[i] + st["path"][i, t]), row(past[i] + t)
    st["kv"][:, :, :, b1, r1] = st["kv"][:, :, :, b0, r0]
    st["lens_out"].copy_(past + st["n_path"])


def run(st):
    case = st["case"]
    if case["op"] == "tree":
        if own:
            out, lse = torch.empty(st["q"].shape, dtype=st["q"].dtype, device="cuda"), torch.empty(st["q"].shape[:2], device="cuda")
            st["ctx"].tree_attention(st["q"], st["kv"], st["offsets"], st["parents"], case["nodes"], out, d_lse_out=lse, d_k_new=st["k_new"],
                                     d_v_new=st["v_new"], window=case["window"], sinks=case["sinks"])
        else:
            out, lse = _tree_plain(st)
        return {"out": out, "lse": lse, "k": st["k"], "v": st["v"]}
    if case["op"] == "verify":
        if not own:
            return _verify_plain(st)
        st["ctx"].verify_drafts(st["logits"], st["tokens"], st["parents"], st["offsets"], st["uniform"], st["sampler"], st["path"], st["n_path"],
                                st["next"], d_logprobs_out=st["logprobs"], d_draft_probs=st["probs"])
        return {name: st[name] for name in ("path", "n_path", "next", "logprobs")}
    if case["op"] == "commit":
        if own:
            st["ctx"].commit_path(st["layers"], st["offsets"], st["path"], st["n_path"], st["lens_out"])
        else:
            _commit_plain(st)
        return {"lens": st["lens_out"], "kv": st["kv"]}
    if case["op"] == "fork":
        if own:
            st["ctx"].fork_pages(st["pool"], st["layers"], st["src"], st["dst"], st["cut"], st["lens"])
        else:
            _fork_plain(st)
    elif own:
        st["ctx"].reserve_pages(st["pool"], st["layers"], st["lens"], st["room"])
        st["ctx"].reserve_pages(st["pool"], st["layers"], st["lens"], st["back"])
    else:
        _reserve_plain(st, st["room"])
        _reserve_plain(st, st["back"])
    return {name: st[name] for name in ("table", "held", "refs", "free", "n_free", "lens", "kv")}


_TAKEN = 0.6                                # about the share of drafted tokens that the cases' target accepts


def work(case):
    """Bytes and operations of one pass: every visible cache row, query, result, logit row of the path and moved row once."""
    rng, n, e = _rng(case), case["n_seqs"], 4 if case.get("dtype") == "fp32" else 2
    if case["op"] == "tree":
        hq, hkv, dh, c = case["hq"], case["hkv"], case["dh"], case["nodes"]
        past = _between(rng, case["past_lo"], case["past_hi"], n)
        if case["window"]:
            past = np.minimum(past, case["window"] + case["sinks"])
        depth = sum(float(_depths(p).sum()) + c for p in _trees(case, rng))
        pairs = hq * (float(past.sum()) * c + depth)
        return {"bytes": float(hkv * (past + 2 * c).sum()) * 2 * dh * e + n * c * hq * (2 * dh * e + 4), "flops": 4 * pairs * dh}
    if case["op"] == "verify":
        levels = min(max(int(_depths(p).max()) for p in _trees(case, rng)) + 1, 12)
        rows = n * sum(_TAKEN ** i for i in range(levels))
        return {"bytes": 4.0 * case["vocab"] * (rows + (n if case["drafts"] and case["nodes"] > 1 else 0)), "flops": 30.0 * rows * case["vocab"]}
    lens = _lengths(case, rng)
    row = case["layers"] * 2 * case["hkv"] * case["dh"] * e
    if case["op"] == "commit":
        return {"bytes": 2.0 * row * n * 0.3 * (case["nodes"] - 1) + 8 * n * case["nodes"], "flops": float(n * case["nodes"])}
    if case["op"] == "fork":
        copies = n * case["samples"]
        return {"bytes": copies * (2.0 * row * (PAGE - 1) / 2 + 12) + 12 * case["samples"] * float((0.85 * lens / PAGE).sum()), "flops": float(copies)}
    pages = float((-(-(lens + case["grow"]) // PAGE) - (0 if case["empty"] else -(-lens // PAGE))).sum())
    return {"bytes": 2 * (12.0 * pages + 16 * n), "flops": pages}


# ------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, one sequence at a time
# ------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] in ("fork", "commit", "reserve"):
        return None                         # whole numbers and copies
    return {"tree": _exact_tree, "verify": _exact_verify}[case["op"]](case, prepare(case, seed))


def _exact_tree(case, st):
    hkv, rep, dh, c = case["hkv"], case["hq"] // case["hkv"], case["dh"], case["nodes"]
    parents, lens = st["parents"].view(-1, c).tolist(), st["lens"].tolist()
    k, v = st["k"].double(), st["v"].double()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for i in range(case["n_seqs"]):
        past, sees, place = lens[i] - c, [], []
        for node, parent in enumerate(parents[i]):
            above = None if parent < -1 else [] if parent < 0 else sees[parent]
            sees.append(None if above is None else above + [node])
            place.append(-1 if sees[-1] is None else past + len(sees[-1]) - 1)
        seen = np.zeros((c, lens[i]), dtype=bool)
        for node in range(c):
            if sees[node] is not None:
                where = np.arange(lens[i])
                where[past:] = place
                visible = np.zeros(lens[i], dtype=bool)
                visible[:past] = True
                visible[[past + a for a in sees[node]]] = True
                if case["window"]:
                    visible &= (where > place[node] - case["window"]) | (where < case["sinks"])
                seen[node] = visible
        seen = torch.from_numpy(seen).cuda()
        pages = st["table"][i, :-(-lens[i] // PAGE)].long()
        for node in range(c):
            if sees[node] is not None:
                b, r = pages[(past + node) // PAGE], (past + node) % PAGE
                k[:, b, r], v[:, b, r] = st["k_new"][i * c + node].double(), st["v_new"][i * c + node].double()
        at = [node for node in range(c) if sees[node] is not None]
        rows = torch.tensor([i * c + node for node in at], device="cuda")
        for h in range(hkv):
            kk, vv = (x[h, pages].reshape(-1, dh)[:lens[i]] for x in (k, v))
            for j in range(h * rep, (h + 1) * rep):
                z = (st["q"][rows, j].double() @ kk.T / math.sqrt(dh)).masked_fill(~seen[at], -math.inf)
                out[rows, j] = torch.softmax(z, -1) @ torch.where(seen[at].any(0)[:, None], vv, 0.0)
                lse[rows, j] = torch.logsumexp(z, -1)
    return {"out": out, "lse": lse, "k": k, "v": v}


def _exact_weights(x, top_p):
    """Whole weights of one row of 32-bit z - max z, in numpy."""
    f = np.float32
    live = x >= f(-24)
    y = np.where(live, x, f(0))
    n = np.rint(y * f(math.log2(math.e)))
    r = (y - n * f(_LN2_HI)) - n * f(math.log(2.0) - _LN2_HI)
    p = f(_EXP[0])
    for coefficient in _EXP[1:]:
        p = p * r + f(coefficient)
    w = np.where(live, np.ldexp(p, n.astype(np.int32)), f(0)) * f(2.0 ** 30)
    w = w.astype(np.int64)
    want = (int(w.sum()) * int(math.floor(f(top_p) * f(2.0 ** 24)))) >> 24
    values = np.sort(w)[::-1]
    least = values[int(np.searchsorted(np.cumsum(values), want))]
    return np.where(w >= least, w, 0)


def _exact_verify(case, st):
    n, c, levels = case["n_seqs"], case["nodes"], st["levels"]
    parents, tokens, uniform = st["parents"].view(n, c).tolist(), st["tokens"].view(n, c).tolist(), st["uniform"].view(n, c).cpu().numpy().astype(np.float64)
    logp = np.zeros((n, levels))
    for s in range(n):
        node, level = 0, 0
        while True:
            x = st["logits"][s * c + node]
            z = (x.cpu().numpy() / np.float32(case["temperature"])).astype(np.float32)
            a = _exact_weights(z - z.max(), case["top_p"])
            q = None if st["probs"] is None else st["probs"][s * c + node].cpu().numpy().astype(np.float64)
            found, token = -1, -1
            for kid in [j for j in range(c) if parents[s][j] == node] if level + 1 < levels else []:
                token, mass = tokens[s][kid], int(a.sum())
                d = np.where(np.arange(len(a)) == token, mass, 0) if q is None else np.floor(q * float(mass)).astype(np.int64)
                if (int(d[token]) * int(uniform[s, kid] * 2 ** 24)) >> 24 < int(a[token]):
                    found = kid
                    break
                if np.maximum(a - d, 0).any():
                    a = np.maximum(a - d, 0)
            if found < 0:
                token = int(np.searchsorted(np.cumsum(a), (int(a.sum()) * int(uniform[s, 0] * 2 ** 24)) >> 24, side="right"))
            z = x.double() / case["temperature"]
            logp[s, level] = float(z[token] - torch.logsumexp(z, 0))
            if found < 0:
                break
            node, level = found, level + 1
    return {"path": None, "n_path": None, "next": None, "logprobs": torch.from_numpy(logp)}
