"""Drafted tokens and shared pages on a caller-owned cache, by definition, in plain numpy and Python integers.

Trees: node i of a sequence's n nodes lies in slot len - n + i, its parent is a node before it, or -1 (the last cached
token); -2, or a chain of parents that ends in one: no node, nor is there one where the slot would be negative.  Verification: the sampler's integer weights.  Pages: reference
counts and a stack of free pages; which page goes where is decided by the order of forks or sequences alone.
"""
import numpy as np

from . import paged, sampler

PAGE = paged.PAGE


# ---- trees ---------------------------------------------------------------------------------------------------------
def chains(parents, first=0):
    """Every node's ancestors from itself up (None: no node, as before the first-th)."""
    got = []
    for i, p in enumerate(parents):
        up = None if p < -1 or p >= i or i < first else [] if p == -1 else got[p]
        got.append(None if up is None else [i] + up)
    return got


def visible(parents, n_keys, window=0, sinks=0):
    """[node][key] of a tree in the last slots of n_keys."""
    past = n_keys - len(parents)
    up = chains(parents, -past)
    seen = np.zeros((len(parents), n_keys), dtype=bool)
    for i, chain in enumerate(up):
        if chain is None:
            continue
        p = past + len(chain) - 1
        for j in range(past):
            seen[i, j] = window <= 0 or j > p - window or j < sinks
        for steps, a in enumerate(chain):
            at = p - steps
            seen[i, past + a] = window <= 0 or at > p - window or at < sinks
    return seen


def weights(q, k, seen, scale):
    """(w [row][key], lse [row]) of one head; rows that see nothing: 0 and -inf."""
    z = np.where(seen, scale * (q @ k.T), -np.inf)
    top = np.max(z, axis=1, initial=-np.inf, keepdims=True)
    top = np.where(np.isinf(top), 0.0, top)
    e = np.exp(z - top)
    total = e.sum(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        return np.where(total > 0, e / total, 0.0), (np.log(total) + top)[:, 0]


def tree_attention(q, k, v, table, lens, offsets, parents, scale, window=0, sinks=0):
    rows, hq, dh = q.shape
    rep = hq // k.shape[0]
    out, lse = np.zeros((rows, hq, dh)), np.zeros((rows, hq))
    for s, n in enumerate(lens):
        a, b = offsets[s], offsets[s + 1]
        seen = visible(parents[a:b], n, window, sinks)
        kk, vv = paged.token_rows(k, table[s], n), paged.token_rows(v, table[s], n)
        for h in range(hq):
            w, lse[a:b, h] = weights(q[a:b, h].astype(np.float64), kk[h // rep], seen, scale)
            out[a:b, h] = w @ np.where(seen.any(0)[:, None], vv[h // rep], 0.0)
    return out, lse


def append(cache, new, table, lens, offsets, parents):
    """The nodes' rows into their slots (in place)."""
    for s, n in enumerate(lens):
        a, b = offsets[s], offsets[s + 1]
        for i, chain in enumerate(chains(parents[a:b], b - a - n)):
            if chain is not None:
                p = n - (b - a) + i
                cache[:, table[s][p // PAGE], p % PAGE] = new[a + i]


# ---- verification --------------------------------------------------------------------------------------------------
def kept_weights(row, temperature, top_p, greedy):
    """Integer weights of a row inside its nucleus; all zero where every token is excluded."""
    x = np.where(np.asarray(row) < np.inf, np.asarray(row, dtype=np.float32), np.float32(-np.inf))
    if not np.any(x > -np.inf):
        return np.zeros(len(x), dtype=np.int64)
    if greedy:
        return (np.arange(len(x)) == int(np.argmax(x))).astype(np.int64)
    w = sampler.quantised_weights(x, temperature)
    tau, _ = sampler.nucleus_threshold(w, top_p)
    return np.where(w >= tau, w, 0).astype(np.int64)


def u24(u):
    return min(max(int(np.float64(u) * 2 ** 24), 0), 2 ** 24 - 1)


def first_above(a, r):
    return int(np.argmax(np.cumsum(a) > r))


def verify(logits, tokens, parents, uniform, max_path, temperature=1.0, top_p=1.0, greedy=False, eos_id=-1, probs=None):
    """(path, next token or -1, log-probabilities) of one sequence's nodes (row i: node i)."""
    path, logp, node = [], [], 0
    vocab = logits.shape[1]
    while len(tokens):
        path.append(node)
        if eos_id >= 0 and tokens[node] == eos_id:
            return path, -1, logp + [0.0]
        a = kept_weights(logits[node], temperature, top_p, greedy)
        accepted = -1
        for child in [j for j in range(node + 1, len(tokens)) if parents[j] == node] if len(path) < max_path else []:
            x, mass = int(tokens[child]), int(a.sum())
            if x < 0:                                    # no draft in this place
                continue
            if probs is None:
                d = np.where(np.arange(vocab) == x, mass, 0)
            else:
                q = np.where(probs[node] > 0, probs[node], 0).astype(np.float64)
                d = np.minimum(np.floor(q * float(mass)), 4.0e18).astype(np.int64)
            # (a token beyond the target's vocabulary, of a draft model with a larger one, has no weight)
            if x < vocab and (int(d[x]) * u24(uniform[child])) >> 24 < int(a[x]):
                accepted = child
                break
            if np.maximum(a - d, 0).any():
                a = np.maximum(a - d, 0)
        mass = int(a.sum())
        if accepted < 0 and mass == 0:
            return path, -1, logp + [-np.inf]
        token = int(tokens[accepted]) if accepted >= 0 else first_above(a, (mass * u24(uniform[0])) >> 24)
        x = np.where(logits[node] < np.inf, logits[node], -np.inf)
        logp.append(sampler.token_logprob(x, temperature, token))
        if accepted < 0:
            return path, token, logp
        node = accepted
    return path, -1, logp


# ---- pages ---------------------------------------------------------------------------------------------------------
class Pages:
    """Tables, counts and the stack of free pages; `copies` lists what the last call copied: (from, to, rows)."""

    def __init__(self, refs, free, n_free, table, held):
        self.refs, self.free, self.n_free = [int(x) for x in refs], [int(x) for x in free], int(n_free)
        self.table, self.held = [[int(x) for x in row] for row in table], [int(x) for x in held]
        self.copies, self.short = [], False

    def _begin(self):
        self.copies, self.short, self._start, self._taken, self._wanted, self._gone = [], False, self.n_free, 0, 0, []

    def _served(self, need):
        """In order, as long as the pages that were free at the start last."""
        self._wanted += need
        if need and self._wanted > self._start:
            self.short = True
            return False
        return True

    def _take(self):
        self._taken += 1
        return self.free[self._start - self._taken]

    def _end(self):
        for page in self._gone:
            self.refs[page] -= 1
        self.n_free = self._start - self._taken
        for page in dict.fromkeys(self._gone):
            if self.refs[page] == 0:
                self.free[self.n_free] = page
                self.n_free += 1

    def fork(self, src, dst, lens, lens_out=None):
        self._begin()
        n = len(self.table)
        first = {}
        for i, d in enumerate(dst):
            first.setdefault(int(d), i)
        left_out = []
        for i, (s, d, length) in enumerate(zip(src, dst, lens)):
            s, d, length = int(s), int(d), int(length)
            if not (0 <= s < n and 0 <= d < n and first[d] == i and s not in first and 0 <= length <= self.held[s] * PAGE):
                left_out.append(i)
                continue
            whole, rest = divmod(length, PAGE)
            if not self._served(1 if rest else 0):
                continue
            pages = self.table[s][:whole]
            for page in pages:
                self.refs[page] += 1
            if rest:
                page = self._take()
                self.refs[page] = 1
                self.copies.append((self.table[s][whole], page, rest))
                pages = pages + [page]
            self._gone += self.table[d][:self.held[d]]
            self.table[d][:len(pages)] = pages
            self.held[d] = len(pages)
            if lens_out is not None:
                lens_out[d] = length
        self._end()
        return left_out

    def reserve(self, lens, target):
        self._begin()
        refs = list(self.refs)
        plans = []
        for s, (length, goal) in enumerate(zip(lens, target)):
            most = len(self.table[s]) * PAGE
            goal = min(max(int(goal), 0), most)
            length = min(min(max(int(length), 0), most), goal, self.held[s] * PAGE)
            want, row, held = -(-goal // PAGE), self.table[s], self.held[s]
            fresh = [j for j in range(want) if j >= held or (j >= length // PAGE and refs[row[j]] > 1)]
            if self._served(len(fresh)):
                plans.append((s, length, want, fresh))
        for s, length, want, fresh in plans:
            row, held = self.table[s], self.held[s]
            self._gone += [row[j] for j in range(held) if j >= want or j in set(fresh)]
            for j in fresh:
                page = self._take()
                self.refs[page] = 1
                if j < held and j == length // PAGE and length % PAGE:
                    self.copies.append((row[j], page, length % PAGE))
                row[j] = page
            self.held[s] = want
        self._end()

    def copy(self, cache):
        """What the last call copies, in a cache [..., block, 16, head_dim] (in place)."""
        for a, b, rows in self.copies:
            cache[..., b, :rows, :] = cache[..., a, :rows, :]


def commit(cache, table, lens, offsets, path, n_path):
    """Accepted rows to the front (in place, cache [..., block, 16, head_dim]); the new lengths."""
    out = list(lens)
    for s, n in enumerate(lens):
        nodes, k = offsets[s + 1] - offsets[s], int(n_path[s])
        p = [int(x) for x in path[s][:max(k, 0)]]
        if not (0 <= k <= len(path[s]) and k <= nodes <= n and all(x >= i for i, x in enumerate(p)) and p == sorted(set(p)) and (not p or p[-1] < nodes)):
            continue
        past = n - nodes
        for i, x in enumerate(p):
            a, b = past + x, past + i
            cache[..., table[s][b // PAGE], b % PAGE, :] = cache[..., table[s][a // PAGE], a % PAGE, :]
        out[s] = past + k
    return out
