"""Measured cases of the operators on a caller-owned paged KV cache.

Three operators that a rollout with a bounded cache runs one after the other:

  attention  a chunk of new tokens per sequence (one token in a decode step) is written to its pages and attends to
             the cache: causal, optionally with a sliding window and first tokens ("sinks") that stay visible
  mass       the attention weight that every cached key receives from the chunk, added to a running total
  evict      each sequence and KV head keeps `budget` keys: sinks, the most recent ones, then the heaviest; the rows
             that stay but lie behind the budget move into the holes in front of it

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


def _attn(name, dtype, heads, n_seqs, chunk, past_lo, past_hi, window=0, sinks=0, ragged=False):
    return {"name": name, "op": "attention", "dtype": dtype, "hq": heads[0], "hkv": heads[1], "dh": heads[2], "n_seqs": n_seqs,
            "chunk": chunk, "past_lo": past_lo, "past_hi": past_hi, "window": window, "sinks": sinks, "ragged": ragged}


def _mass(name, dtype, heads, n_seqs, chunk, past_lo, past_hi, window=0, sinks=0, ragged=False):
    return {**_attn(name, dtype, heads, n_seqs, chunk, past_lo, past_hi, window, sinks, ragged), "op": "mass"}


def _evict(name, dtype, heads, n_seqs, len_lo, len_hi, budget, recent, sinks):
    return {"name": name, "op": "evict", "dtype": dtype, "hq": heads[0], "hkv": heads[1], "dh": heads[2], "n_seqs": n_seqs,
            "past_lo": len_lo, "past_hi": len_hi, "budget": budget, "recent": recent, "sinks": sinks}


def listed():
    return [
        # one decode step of a few short sequences: what the call costs when there is next to nothing to read
        _attn("step_small", "bf16", (12, 2, 128), 4, 1, 100, 300),
        # one decode step of a full batch over long ragged prefixes (the 7B-class shape)
        _attn("step_ragged", "bf16", (28, 4, 128), 128, 1, 1024, 6144),
        # one decode step of ONE long sequence: little to share the work over
        _attn("step_long", "bf16", (12, 2, 128), 1, 1, 100003, 100003),
        # one decode step of long generations under a window with sinks
        _attn("step_window", "bf16", (28, 4, 128), 256, 1, 2048, 4352, window=1024, sinks=4),
        # tool outputs or user turns of odd lengths appended to cached responses
        _attn("turn_ragged", "bf16", (12, 2, 128), 16, 233, 1000, 5000, ragged=True),
        # a long prompt chunk over a cached prefix: the largest call
        _attn("chunk_long", "bf16", (28, 4, 128), 4, 2048, 4096, 4096),
        # a prompt chunk under a window with sinks, 64-wide heads, nothing divisible by anything
        _attn("chunk_window", "fp32", (4, 2, 64), 3, 777, 0, 1500, window=500, sinks=3, ragged=True),
        # the weights of a decode step, gathered for a later eviction
        _mass("mass_step", "bf16", (28, 4, 128), 128, 1, 1024, 6144),
        # the weights of a whole prompt chunk
        _mass("mass_chunk", "bf16", (12, 2, 128), 8, 1024, 1000, 4096, ragged=True),
        # one token over budget: the eviction that follows every decode step
        _evict("evict_step", "bf16", (28, 4, 128), 128, 1025, 1025, 1024, 256, 4),
        # ragged caches cut down once after the prefix has been read
        _evict("evict_prefix", "bf16", (28, 4, 128), 64, 1024, 6144, 1024, 128, 4),
        # one long 32-bit cache
        _evict("evict_long", "fp32", (4, 2, 64), 2, 65001, 65001, 8191, 1000, 16),
    ]


_MOST_PAIRS = 4 * 28 * 2048 * 6144          # (query row, key) pairs of the largest listed call
_MOST_ROWS = 128 * 4 * 6144 * 128           # cache elements of K of the largest listed cache


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "mass", "evict"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    heads = rng.choice(_HEADS)
    hq, hkv, dh = heads
    if op == "evict":
        budget = _log(rng, 16, 8192)
        hi = budget + _log(rng, 1, 32768)
        lo = rng.choice([hi, max(1, hi // 5), 1])
        n_seqs = max(1, min(_log(rng, 1, 256), _MOST_ROWS // (hkv * hi * dh)))
        sinks = rng.randint(0, min(16, budget))
        return {k: v for k, v in _evict("", dtype, heads, n_seqs, lo, hi, budget, rng.randint(0, (budget - sinks) // 2), sinks).items() if k != "name"}
    chunk = 1 if rng.random() < 0.4 else _log(rng, 2, 2048)
    hi = rng.choice([0, _log(rng, 1, 200), _log(rng, 200, 20000), _log(rng, 200, 20000)])
    lo = rng.choice([hi, hi // 4, 0])
    pairs = _MOST_PAIRS // (8 if dtype == "fp32" else 1)
    n_seqs = max(1, min(_log(rng, 1, 256), pairs // (hq * chunk * (hi + chunk)), _MOST_ROWS // (hkv * (hi + chunk) * dh)))
    while n_seqs * hq * chunk * (hi + chunk) > pairs:
        chunk = max(1, chunk // 2)
    window = rng.choice([0, 0, _log(rng, 1, 4096)])
    sinks = rng.randint(0, 40) if window else 0
    case = _attn("", dtype, heads, n_seqs, chunk, lo, hi, window, sinks, rng.random() < 0.6)
    case["op"] = op
    return {k: v for k, v in case.items() if k != "name"}


def _lengths(case):
    """(past tokens, new tokens) of every sequence, the same for every seed; for an eviction the new tokens are 0."""
    n = case["n_seqs"]
    rng = np.random.RandomState(n * 7919 + case["past_hi"])
    past = rng.randint(case["past_lo"], case["past_hi"] + 1, n)
    past[rng.randint(n)] = case["past_hi"]
    if case["op"] == "evict":
        return past, np.zeros(n, dtype=past.dtype)
    new = np.full(n, case["chunk"])
    if case["ragged"]:
        new = rng.randint(1, case["chunk"] + 1, n)
        new[rng.randint(n)] = case["chunk"]
    return past, new


_contexts = {}


def _context(dtype):
    """The library context of a storage type: a program keeps one for all its calls."""
    import paper_2601_19404_b200 as rpo
    if dtype not in _contexts:
        shape = rpo.shape_preset("tiny", dtype=1 if dtype == "bf16" else 0)
        _contexts[dtype] = rpo.Context(shape, kv_pool_blocks=16, max_groups=1, max_seqs=1, max_chunk_tokens=32, max_positions=64)
    return _contexts[dtype]


def prepare(case, seed):
    dt, hq, hkv, dh, n = _DTYPES[case["dtype"]], case["hq"], case["hkv"], case["dh"], case["n_seqs"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    past, new = _lengths(case)
    lens = past + new
    pages = -(-lens // PAGE)
    stride = int(pages.max()) + 3
    n_blocks = int(pages.sum()) + 5
    # pages lie anywhere in the pool; what is behind a sequence's last page in its table is not set
    order = torch.randperm(n_blocks, generator=g, device="cuda", dtype=torch.int32)
    first = torch.from_numpy(np.concatenate([[0], np.cumsum(pages)[:-1]])).cuda()
    slot = torch.arange(stride, device="cuda")
    inside = slot[None, :] < torch.from_numpy(pages).cuda()[:, None]
    table = torch.where(inside, order[(first[:, None] + slot[None, :]).clamp(max=n_blocks - 1)], -1).to(torch.int32).contiguous()
    k = torch.randn(hkv, n_blocks, PAGE, dh, generator=g, device="cuda", dtype=torch.float32).to(dt)
    v = torch.randn(hkv, n_blocks, PAGE, dh, generator=g, device="cuda", dtype=torch.float32).to(dt)
    st = {"case": case, "k": k, "v": v, "table": table, "lens": torch.from_numpy(lens.astype(np.int32)).cuda()}
    if case["op"] == "evict":
        width = int(lens.max()) + 7
        # accumulated weights: most keys got little, a few got much; several are equal
        st["mass"] = torch.round(torch.empty(n, hkv, width, device="cuda").exponential_(1.0, generator=g) ** 2 * 64) / 64
        st["pos"] = torch.arange(width, device="cuda", dtype=torch.int32).expand(n, hkv, width).contiguous()
        st["out_lens"] = torch.zeros(n, dtype=torch.int32, device="cuda")
        st["src"] = torch.zeros(n, hkv, case["budget"], dtype=torch.int32, device="cuda")
        st["mass_out"] = torch.zeros(n, hkv, case["budget"], device="cuda")
        st["pos_out"] = torch.zeros(n, hkv, case["budget"], dtype=torch.int32, device="cuda")
    else:
        rows = int(new.sum())
        off = np.zeros(n + 1, dtype=np.int32)
        off[1:] = np.cumsum(new)
        st["offsets"] = torch.from_numpy(off).cuda()
        st["chunk"] = int(new.max())
        # queries, keys and values of the new tokens as one fused projection leaves them
        qkv = torch.randn(rows, hq + 2 * hkv, dh, generator=g, device="cuda", dtype=torch.float32)
        qkv[:, :hq] *= 1.5
        qkv = qkv.to(dt)
        st["q"], st["k_new"], st["v_new"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        if case["op"] == "mass":
            width = int(lens.max()) + 7
            st["lse"] = _attend(st)[1]
            st["mass"] = torch.rand(n, hkv, width, generator=g, device="cuda")
            st["mass_out"] = torch.zeros(n, hkv, width, device="cuda")
    if own:
        import paper_2601_19404_b200 as rpo
        st["ctx"] = _context(case["dtype"])
        st["kv"] = rpo.PagedKV(k, v, table, st["lens"])
    return st


# ------------------------------------------------------------------------------------------------------------
# plain forms
# ------------------------------------------------------------------------------------------------------------
def _gather(cache, table):
    """[n_seqs, KV heads, tokens, head dim] in 32 bits of a paged cache."""
    hkv, _, page, dh = cache.shape
    rows = cache[:, table.clamp(min=0).long()].float()                       # [hkv, n, pages, page, dh]
    return rows.permute(1, 0, 2, 3, 4).reshape(table.shape[0], hkv, -1, dh)


def _padded(st):
    """Row numbers of the new tokens padded to [n_seqs, longest chunk], which of them exist, and their positions."""
    off, lens = st["offsets"].long(), st["lens"].long()
    new = off[1:] - off[:-1]
    t = torch.arange(st["chunk"], device=off.device)
    exists = t[None, :] < new[:, None]
    return (off[:-1, None] + t[None, :]).clamp(max=max(st["q"].shape[0] - 1, 0)), exists, lens[:, None] - new[:, None] + t[None, :]


def _visible(case, positions, n_keys):
    """[n_seqs, chunk, keys]: causal, inside the window or one of the first tokens."""
    key = torch.arange(n_keys, device=positions.device)
    seen = key <= positions[..., None]
    if case["window"]:
        seen &= (key > positions[..., None] - case["window"]) | (key < case["sinks"])
    return seen


def _scores(st, keys):
    """Scaled products [n_seqs, KV heads, heads of a group, chunk, keys], -inf where a key is not seen."""
    case = st["case"]
    hkv, rep, dh = case["hkv"], case["hq"] // case["hkv"], case["dh"]
    row, exists, pos = _padded(st)
    q = st["q"].float()[row].reshape(row.shape[0], row.shape[1], hkv, rep, dh).permute(0, 2, 3, 1, 4)
    n, c = row.shape
    s = torch.matmul(q.reshape(n, hkv, rep * c, dh), keys.transpose(2, 3)).reshape(n, hkv, rep, c, -1)
    s *= 1.0 / math.sqrt(dh)
    seen = _visible(case, pos, keys.shape[2]) & exists[..., None]
    return s.masked_fill_(~seen[:, None, None], -math.inf), row, exists


def _attend(st):
    case = st["case"]
    hkv, hq, dh = case["hkv"], case["hq"], case["dh"]
    s, row, exists = _scores(st, _gather(st["k"], st["table"]))
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    e = torch.exp(s.sub_(top))
    total = e.sum(-1, keepdim=True)
    n, c = row.shape
    o = torch.matmul(e.reshape(n, hkv, -1, e.shape[-1]), _gather(st["v"], st["table"])).reshape(n, hkv, hq // hkv, c, dh)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (torch.log(total) + top)[..., 0]                                    # [n, hkv, rep, chunk]
    out = torch.empty(st["q"].shape[0], hq, dh, dtype=st["q"].dtype, device=s.device)
    lse_out = torch.empty(st["q"].shape[0], hq, device=s.device)
    at = row[exists]
    out[at] = o.permute(0, 3, 1, 2, 4).reshape(n, c, hq, dh)[exists].to(out.dtype)
    lse_out[at] = lse.permute(0, 3, 1, 2).reshape(n, c, hq)[exists]
    return out, lse_out


def _append(st):
    """The chunk's keys and values into their pages."""
    row, exists, pos = _padded(st)
    pos, row = torch.where(exists, pos, 0), row[exists]
    slot = (st["table"].gather(1, pos // PAGE).long() * PAGE + pos % PAGE)[exists]
    for cache, new in ((st["k"], st["k_new"]), (st["v"], st["v_new"])):
        cache.view(cache.shape[0], -1, cache.shape[3])[:, slot] = new[row].transpose(0, 1)


def _weights(st):
    s, row, exists = _scores(st, _gather(st["k"], st["table"]))
    n, c = row.shape
    hkv, hq = st["case"]["hkv"], st["case"]["hq"]
    lse = st["lse"][row].reshape(n, c, hkv, hq // hkv).permute(0, 2, 3, 1)[..., None]
    got = torch.exp(s.sub_(torch.where(torch.isinf(lse), torch.zeros_like(lse), lse))).sum((2, 3))       # [n, hkv, keys]
    width = st["mass"].shape[2]
    key = torch.arange(width, device=got.device)
    got = torch.nn.functional.pad(got, (0, max(0, width - got.shape[2])))[..., :width]
    return torch.where(key < st["lens"][:, None, None], st["mass"] + got, st["mass_out"])


def _evicted(st):
    case, mass, pos, lens = st["case"], st["mass"], st["pos"], st["lens"].long()
    budget, dev = case["budget"], st["mass"].device
    n, hkv, width = mass.shape
    slot = torch.arange(width, device=dev).expand(n, hkv, width)
    live = slot < lens[:, None, None]
    newest = torch.where(live, pos, -1).amax(-1, keepdim=True)
    safe = (pos < case["sinks"]) | (pos > newest - case["recent"])
    # order of the 32-bit weights as whole numbers (a weight that is no number counts least), protected keys first
    bits = (mass + 0.0).view(torch.int32).long()
    rank = torch.where(bits < 0, -1 - (bits & 0x7FFFFFFF), bits)
    rank = torch.where(torch.isnan(mass), -(1 << 32), rank) + safe.long() * (1 << 40)
    rank = torch.where(live, rank, -(1 << 50))
    chosen = torch.sort(rank, dim=-1, descending=True, stable=True)[1][..., :min(budget, width)]
    kept = torch.zeros_like(live).scatter_(2, chosen, True) & live
    n_kept = lens.clamp(max=budget)[:, None, None]
    hole, mover = ~kept & (slot < n_kept), kept & (slot >= budget)
    # the i-th mover goes into the i-th hole
    nth = torch.zeros(n, hkv, width + 1, dtype=torch.long, device=dev)
    nth.scatter_(2, torch.where(mover, mover.long().cumsum(-1) - 1, width), slot)
    src = torch.where(hole, nth.gather(2, (hole.long().cumsum(-1) - 1).clamp(min=0)), slot)
    src = torch.nn.functional.pad(src, (0, max(0, budget - width)))[..., :budget]
    fits = torch.arange(budget, device=dev) < n_kept
    st["out_lens"].copy_(n_kept[:, 0, 0])
    st["src"].copy_(torch.where(fits, src, -1))
    at = torch.where(fits, src, 0)
    st["mass_out"].copy_(torch.where(fits, mass.gather(2, at), st["mass_out"]))
    st["pos_out"].copy_(torch.where(fits, pos.gather(2, at), st["pos_out"]))
    # rows that moved
    i, h, to = torch.nonzero(fits & (src != torch.arange(budget, device=dev)), as_tuple=True)
    frm = src[i, h, to]
    row = lambda s: st["table"][i, s // PAGE].long() * PAGE + s % PAGE  # noqa: E731
    at_from, at_to = row(frm), row(to)
    for cache in (st["k"], st["v"]):
        flat = cache.view(hkv, -1, cache.shape[3])
        flat[h, at_to] = flat[h, at_from]


def run(st):
    case = st["case"]
    scale = 1.0 / math.sqrt(case["dh"])
    if case["op"] == "attention":
        if own:
            out = torch.empty(st["q"].shape, dtype=st["q"].dtype, device="cuda")
            lse = torch.empty(st["q"].shape[:2], device="cuda")
            st["ctx"].chunk_attention(st["q"], st["kv"], st["offsets"], st["chunk"], out, d_lse_out=lse, d_k_new=st["k_new"], d_v_new=st["v_new"],
                                      scale=scale, window=case["window"], sinks=case["sinks"])
        else:
            _append(st)
            out, lse = _attend(st)
        return {"out": out, "lse": lse, "k": st["k"], "v": st["v"]}
    if case["op"] == "mass":
        if own:
            st["ctx"].attention_mass(st["q"], st["kv"], st["offsets"], st["chunk"], st["lse"], st["mass_out"], d_mass_in=st["mass"],
                                     scale=scale, window=case["window"], sinks=case["sinks"])
        else:
            st["mass_out"] = _weights(st)
        return {"mass": st["mass_out"]}
    if own:
        st["ctx"].evict_cache(st["kv"], st["mass"], st["pos"], case["budget"], st["out_lens"], st["src"], st["mass_out"], st["pos_out"],
                              sinks=case["sinks"], recent=case["recent"])
    else:
        _evicted(st)
    return {name: st[name] for name in ("out_lens", "src", "mass_out", "pos_out", "k", "v")}


def work(case):
    """Bytes and operations of one pass: every visible cache row, query, result and weight once."""
    e, hq, hkv, dh = (2 if case["dtype"] == "bf16" else 4), case["hq"], case["hkv"], case["dh"]
    past, new = _lengths(case)
    if case["op"] == "evict":
        kept = np.minimum(past, case["budget"])
        # at random about kept * (past - kept) / past of the kept rows lie behind the budget; each is read and written
        moved = kept * (past - kept) / np.maximum(past, 1)
        return {"bytes": float(hkv * (past * 8 + kept * 12 + moved * 4 * dh * e).sum()), "flops": float(hkv * past.sum())}
    keys, seen = past + new, past + (new + 1) / 2
    if case["window"]:
        reach = case["window"] + case["sinks"]
        keys, seen = np.minimum(keys, new + reach), np.minimum(seen, reach)
    rows, pairs = float(hq * new.sum()), float(hq * (new * seen).sum())
    if case["op"] == "mass":
        return {"bytes": float(hkv * keys.sum()) * (dh * e + 8) + rows * (dh * e + 4), "flops": 2 * pairs * dh}
    return {"bytes": float(hkv * (keys + new).sum()) * 2 * dh * e + rows * (2 * dh * e + 4), "flops": 4 * pairs * dh}


# ------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, one sequence and KV head at a time
# ------------------------------------------------------------------------------------------------------------
def _token_rows(cache, pages, n):
    return cache[pages.long()].reshape(-1, cache.shape[-1])[:n].double()


def exact(case, seed):
    if case["op"] == "evict":
        return None                       # whole numbers and copies
    st = prepare(case, seed)
    hkv, rep, dh = case["hkv"], case["hq"] // case["hkv"], case["dh"]
    off, lens = st["offsets"].tolist(), st["lens"].tolist()
    k, v = st["k"].clone(), st["v"].clone()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(st["q"].shape[:2], dtype=torch.float64, device="cuda")
    mass = st["mass_out"].double() if case["op"] == "mass" else None
    for i in range(case["n_seqs"]):
        a, b, n = off[i], off[i + 1], lens[i]
        pages = st["table"][i, :-(-n // PAGE)]
        at = torch.arange(n - (b - a), n, device="cuda")
        seen = torch.arange(n, device="cuda")[None, :] <= at[:, None]
        if case["window"]:
            seen &= (torch.arange(n, device="cuda")[None, :] > at[:, None] - case["window"]) | (torch.arange(n, device="cuda")[None, :] < case["sinks"])
        for h in range(hkv):
            if case["op"] == "attention":
                k[h, pages[at // PAGE].long(), at % PAGE] = st["k_new"][a:b, h]
                v[h, pages[at // PAGE].long(), at % PAGE] = st["v_new"][a:b, h]
            kk, vv = _token_rows(k[h], pages, n), _token_rows(v[h], pages, n)
            for j in range(h * rep, (h + 1) * rep):
                z = (st["q"][a:b, j].double() @ kk.T / math.sqrt(dh)).masked_fill(~seen, -math.inf)
                if case["op"] == "mass":
                    if j == h * rep:
                        mass[i, h, :n] = st["mass"][i, h, :n].double()
                    mass[i, h, :n] += torch.softmax(z, -1).sum(0)
                else:
                    out[a:b, j] = torch.softmax(z, -1) @ vv
                    lse[a:b, j] = torch.logsumexp(z, -1)
    return {"mass": mass} if case["op"] == "mass" else {"out": out, "lse": lse, "k": k.double(), "v": v.double()}
