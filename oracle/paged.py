"""Operators on a paged KV cache, by definition, in float64 numpy.

A cache is K, V [kv_head][block][16][head_dim], a block table [sequence][blocks] and a length per sequence.  Row i of a
chunk of n new tokens sits at position p = len - n + i and sees the keys j <= p of its sequence; with a window only
those with j > p - window or j < sinks.
"""
import numpy as np

PAGE = 16


def token_rows(cache, table_row, n):
    """[kv_head][n][head_dim] rows of a sequence's first n tokens."""
    pages = np.asarray(table_row[:-(-n // PAGE)], dtype=np.int64)
    return np.asarray(cache)[:, pages].reshape(cache.shape[0], -1, cache.shape[3])[:, :n].astype(np.float64)


def append(cache, new, table, lens, offsets):
    """The chunks' rows new [rows][kv_head][head_dim] in their pages (in place); rows at negative positions are dropped."""
    for s, n in enumerate(lens):
        a, b = offsets[s], offsets[s + 1]
        for r in range(a, b):
            p = n - b + r
            if p >= 0:
                cache[:, table[s][p // PAGE], p % PAGE] = new[r]


def visible(n_rows, n_keys, window, sinks):
    """[row][key] of a chunk of n_rows tokens at the end of n_keys."""
    p = np.arange(n_keys - n_rows, n_keys)[:, None]
    j = np.arange(n_keys)[None, :]
    seen = j <= p
    if window > 0:
        seen &= (j > p - window) | (j < sinks)
    return seen


def _weights(q, k, scale, window, sinks):
    """(w [row][key], lse [row]) of one head; rows that see nothing have weights 0 and lse -inf."""
    z = np.where(visible(q.shape[0], k.shape[0], window, sinks), scale * (q @ k.T), -np.inf)
    top = np.max(z, axis=1, initial=-np.inf, keepdims=True)
    top = np.where(np.isinf(top), 0.0, top)
    e = np.exp(z - top)
    total = e.sum(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        return np.where(total > 0, e / total, 0.0), (np.log(total) + top)[:, 0]


def chunk_attention(q, k, v, table, lens, offsets, scale, window=0, sinks=0):
    """(out [rows][q_head][head_dim], lse [rows][q_head]); rows of no sequence are 0 / 0."""
    rows, hq, dh = q.shape
    rep = hq // k.shape[0]
    out, lse = np.zeros((rows, hq, dh)), np.zeros((rows, hq))
    for s, n in enumerate(lens):
        a, b = offsets[s], offsets[s + 1]
        kk, vv = token_rows(k, table[s], n), token_rows(v, table[s], n)
        for h in range(hq):
            w, lse[a:b, h] = _weights(q[a:b, h].astype(np.float64), kk[h // rep], scale, window, sinks)
            out[a:b, h] = w @ vv[h // rep]
    return out, lse


def attention_mass(q, k, table, lens, offsets, scale, n_slots, window=0, sinks=0):
    """[sequence][kv_head][n_slots] weight every key received; 0 behind a sequence's end."""
    hq, hkv = q.shape[1], k.shape[0]
    mass = np.zeros((len(lens), hkv, n_slots))
    for s, n in enumerate(lens):
        a, b = offsets[s], offsets[s + 1]
        kk = token_rows(k, table[s], n)
        for h in range(hq):
            g = h // (hq // hkv)
            mass[s, g, :n] += _weights(q[a:b, h].astype(np.float64), kk[g], scale, window, sinks)[0].sum(0)
    return mass


def evict_order(mass, positions, sinks, recent):
    """Slots in the order in which they stay: protected first, then heavier, then lower; NaN counts least."""
    newest = max(int(p) for p in positions)
    safe = [int(p) < sinks or int(p) > newest - recent for p in positions]

    def key(i):
        m = float(mass[i])
        return (not safe[i], m != m, -m if m == m else 0.0, i)

    return sorted(range(len(mass)), key=key)


def evict(mass, positions, budget, sinks=0, recent=0):
    """For one sequence and KV head (arrays of its len slots): src, the slot that each of the first min(len, budget) slots
    is filled from."""
    n = len(mass)
    if n <= budget:
        return list(range(n))
    kept = sorted(evict_order(mass, positions, sinks, recent)[:budget])
    src = list(range(budget))
    holes = [i for i in range(budget) if i not in set(kept)]
    for hole, mover in zip(holes, [i for i in kept if i >= budget]):
        src[hole] = mover
    return src
