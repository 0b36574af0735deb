"""Pins of oracle/drafts.py: chains are chunks, emitted tokens are distributed as sampled ones, pages stay accounted for."""
import numpy as np
import pytest

from oracle import drafts, paged, sampler


def test_a_chain_is_a_chunk():
    for n, keys, window, sinks in ((1, 1, 0, 0), (5, 9, 0, 0), (7, 40, 3, 2), (4, 4, 2, 0), (6, 30, 12, 20)):
        assert np.array_equal(drafts.visible([i - 1 for i in range(n)], keys, window, sinks), paged.visible(n, keys, window, sinks))


def test_a_path_of_a_tree_is_a_chunk_of_its_own():
    parents = [-1, 0, 0, 1, 2, 3, 5, -1, 7]
    rng = np.random.default_rng(0)
    keys, values, q = rng.standard_normal((20 + 9, 8)), rng.standard_normal((20 + 9, 8)), rng.standard_normal((9, 8))
    for window, sinks in ((0, 0), (4, 0), (4, 2), (23, 22)):
        seen = drafts.visible(parents, 29, window, sinks)
        w, lse = drafts.weights(q, keys, seen, 0.3)
        for node, chain in enumerate(drafts.chains(parents)):
            at = list(range(20)) + [20 + a for a in reversed(chain)]
            want, want_lse = paged._weights(q[[a for a in reversed(chain)]], keys[at], 0.3, window, sinks)
            assert np.allclose(w[node] @ values, want[-1] @ values[at], atol=1e-12) and np.isclose(lse[node], want_lse[-1])


def test_rows_without_a_node():
    parents = [-1, -2, 1, 0, 7, 4, -3]
    assert drafts.chains(parents) == [[0], None, None, [3, 0], None, None, None]
    assert not drafts.visible(parents, 10)[[1, 2, 4, 5, 6]].any() and not drafts.visible(parents, 10)[:, 3 + 1].any()


def test_verification_without_drafts_is_the_sampler():
    rng = np.random.default_rng(1)
    for _ in range(50):
        row = (rng.standard_normal((1, 40)) * 3).astype(np.float32)
        u = np.float32(rng.integers(0, 2 ** 24) / 2 ** 24)
        path, token, logp = drafts.verify(row, [3], [-1], [u], 4, 0.8, 0.9)
        assert path == [0] and token == sampler.sample_token(row[0], 0.8, 0.9, int(u * 2 ** 24))
        assert np.isclose(logp[0], sampler.token_logprob(row[0], 0.8, token))


@pytest.mark.parametrize("given", [True, False])
def test_emitted_tokens_are_distributed_as_sampled_ones(given):
    """The first emitted token of a root with two drafted children, 20 000 times: every frequency within five standard deviations."""
    rng = np.random.default_rng(2)
    vocab, n = 6, 20000
    logits = np.zeros((3, vocab), dtype=np.float32)
    logits[0] = [1.0, 0.3, -0.5, 2.0, 0.0, -3.0]
    q = np.exp(np.array([0.2, 1.5, 0.0, 0.1, -1.0, 0.0]))
    q = (q / q.sum()).astype(np.float32)
    w = drafts.kept_weights(logits[0], 1.0, 0.95, False)
    p, counts = w / w.sum(), np.zeros(vocab)
    assert p[5] == 0
    for _ in range(n):
        kids = rng.choice(vocab, 2, p=q / q.sum()) if given else [1, 3]
        probs = np.stack([q, q, q]) if given else None
        path, token, _ = drafts.verify(logits, [0, kids[0], kids[1]], [-1, 0, 0], rng.random(3), 3, 1.0, 0.95, probs=probs)
        counts[token if len(path) == 1 else kids[path[1] - 1]] += 1
    assert np.all(np.abs(counts / n - p) <= 5 * np.sqrt(p * (1 - p) / n))


STEPS = 2 ** 24
ROOT, LEVEL2 = [1.0, 0.3, -0.5, 2.0], [[0.0, 1.0, 2.0, -1.0], [2.0, 0.0, 0.1, 0.2], [0.5, 0.5, 3.0, 0.4], [-1.0, 0.0, 1.0, 1.5]]


def first_u(holds):
    """How many of the numbers u24 = 0, 1, ... come before the first for which `holds` (once true, true for all behind)."""
    lo, hi = 0, STEPS
    while lo < hi:
        mid = (lo + hi) // 2
        lo, hi = (lo, mid) if holds(mid / STEPS) else (mid + 1, hi)
    return lo


def emitted(walk, tokens, vocab):
    """Distribution of the token that walk(u, u0) emits behind its last accepted node, or at the accepted child: child by child and with
    the last number u0, in exact counts of the numbers that lead there.  walk(u, u0) -> (accepted child or -1, next token)."""
    p, left, refused = np.zeros(vocab), 1.0, {}
    for c, x in tokens.items():
        n = first_u(lambda u: walk({**refused, c: u}, 0.0)[0] != c)
        p[x if n else 0] += left * n / STEPS
        left *= 1 - n / STEPS
        refused[c] = 1 - 1 / STEPS
        if n == STEPS:
            return p
    at = [0] + [first_u(lambda u0: walk(refused, u0)[1] >= t) for t in range(1, vocab)] + [STEPS]
    return p + left * np.diff(at) / STEPS


@pytest.mark.parametrize("top_p", [1.0, 0.9])
@pytest.mark.parametrize("kind", ["drawn", "given", "larger", "padded"])
def test_all_draws_together_are_the_sampler(kind, top_p):
    """Every draw of two children of the root and of one child of each, every random number, at both levels.

    drawn    children drawn from q independently             larger   from a q of five tokens, of which the target has four
    given    other children, without probabilities           padded   drawn, with a row without a draft (-1) before and between
    Drafted probabilities are sums of powers of two that add up to one, so the draws' weights are exact.  An acceptance is then off by at most
    2^-24 + 2^-29 (numbers u24, whole weights of a mass above 2^30), an entry of the last draw by twice that: below 8 x 2^-24 in all."""
    vocab = 4
    q = {"larger": [0.25, 0.25, 0.125, 0.125, 0.25]}.get(kind, [0.5, 0.25, 0.125, 0.125])
    place = {"padded": [2, 4]}.get(kind, [1, 2])                           # rows of the root's children
    parents = [-1, 0, 0, 0, 0, 2, 4] if kind == "padded" else [-1, 0, 0, 1, 2]
    below = [5, 6] if kind == "padded" else [3, 4]
    pairs = [(x, y, q[x] * q[y]) for x in range(len(q)) for y in range(len(q))] if kind != "given" else [(1, 2, 1.0), (3, 0, 1.0), (0, 3, 1.0), (1, 1, 1.0)]

    def verify(tokens, u, u0, max_path=3):
        logits = np.zeros((len(parents), vocab), dtype=np.float32)
        logits[0] = ROOT
        for row in place:
            if 0 <= tokens[row] < vocab:
                logits[row] = LEVEL2[tokens[row]]
        probs = None if kind == "given" else np.tile(np.array(q[:vocab], dtype=np.float32), (len(parents), 1))
        uniform = np.zeros(len(parents))
        uniform[0] = u0
        for row, x in u.items():
            uniform[row] = x
        return drafts.verify(logits, tokens, parents, uniform, max_path, 1.0, top_p, probs=probs)

    def share(row):
        w = drafts.kept_weights(np.array(row, dtype=np.float32), 1.0, top_p, False)
        return w / w.sum()

    got = [np.zeros(vocab) for _ in range(len(pairs) if kind == "given" else 1)]
    for i, (x, y, weight) in enumerate(pairs):
        tokens = [0] * len(parents)
        tokens[place[0]], tokens[place[1]] = x, y
        for row in ([1, 3] if kind == "padded" else []):
            tokens[row] = -1
        behind = lambda u, u0: (lambda path, token, _: (path[1] if len(path) > 1 else -1, token))(*verify(tokens, u, u0, 2))
        got[i % len(got)] += weight * emitted(behind, {row: tokens[row] for row in place}, vocab)
    for p in got:
        assert np.all(np.abs(p - share(ROOT)) <= 8 / STEPS)
    # behind an accepted child
    for first in (0, 1) if kind != "given" else ():
        for x in range(vocab):
            if share(ROOT)[x] == 0:
                continue
            got = np.zeros(vocab)
            for y, weight in enumerate(q):
                tokens = [0] * len(parents)
                for row in ([1, 3] if kind == "padded" else []):
                    tokens[row] = -1
                tokens[place[first]], tokens[below[first]] = x, y
                tokens[place[1 - first]] = -1                              # (only the other one can be accepted)
                behind = lambda u, u0: (lambda path, token, _: (path[2] if len(path) > 2 else -1, token))(*verify(tokens, u, u0))
                got += weight * emitted(behind, {below[first]: y}, vocab)
            assert np.all(np.abs(got - share(LEVEL2[x])) <= 8 / STEPS)


def test_greedy_eos_and_rows_that_exclude_everything():
    logits = np.full((3, 4), -np.inf, dtype=np.float32)
    logits[0] = [0, 5, 5, 1]
    assert drafts.verify(logits, [0, 2, 1], [-1, 0, 0], [0.9] * 3, 3, greedy=True)[:2] == ([0, 2], -1)
    assert drafts.verify(logits, [0, 2, 1], [-1, 0, 0], [0.9] * 3, 3, greedy=True, eos_id=1)[1:] == (-1, [drafts.sampler.token_logprob(logits[0], 1.0, 1), 0.0])
    assert drafts.verify(logits, [0, 2, 1], [-1, 0, 0], [0.9] * 3, 1, greedy=True)[:2] == ([0], 1)
    assert drafts.verify(logits, [7], [-1], [0.5], 3, greedy=True, eos_id=7) == ([0], -1, [0.0])
    logits[0, 1] = np.nan
    logits[0, 3] = np.inf
    assert drafts.verify(logits[:1], [0], [-1], [0.9], 3, greedy=True)[1] == 2
    assert drafts.verify(logits[1:2], [0], [-1], [0.9], 3)[1:] == (-1, [-np.inf])


def accounted(pages, n_blocks):
    held = [p for row, n in zip(pages.table, pages.held) for p in row[:n]]
    counts = [held.count(p) for p in range(n_blocks)]
    assert pages.refs == counts
    assert sorted(pages.free[:pages.n_free]) == [p for p in range(n_blocks) if counts[p] == 0]


def test_pages_stay_accounted_for():
    rng = np.random.default_rng(3)
    n, blocks, width = 7, 40, 9
    pages = drafts.Pages([0] * blocks, list(range(blocks)), blocks, -np.ones((n, width), dtype=int), [0] * n)
    lens, content, short = [0] * n, np.full((blocks, 16, 1), -1), 0
    text = [[] for _ in range(n)]
    for step in range(400):
        if rng.random() < 0.6:
            target = [int(rng.integers(0, width * 16 + 1)) if rng.random() < 0.4 else x for x in lens]
            before = list(pages.held)
            pages.reserve(lens, target)
            pages.copy(content)
            for s in range(n):
                room = pages.held[s] * 16
                text[s] = text[s][:min(lens[s], target[s])] if pages.held[s] * 16 >= target[s] or before[s] != pages.held[s] else text[s]
                goal = min(target[s], room)
                for j in range(len(text[s]), goal):
                    if pages.refs[pages.table[s][j // 16]] == 1:
                        text[s].append(int(rng.integers(1000)))
                        content[pages.table[s][j // 16], j % 16] = text[s][-1]
                    else:
                        break
                lens[s] = len(text[s])
        else:
            src, dst = int(rng.integers(n)), rng.permutation(n)[:3]
            cut = [int(rng.integers(0, lens[src] + 1)) for _ in dst]
            old = list(lens)
            left = pages.fork([src] * 3, dst, cut, lens)
            pages.copy(content)
            assert left == ([0, 1, 2] if src in dst else [])
            for d, c in zip(dst, cut):
                if lens[d] != old[d] or (not left and pages.held[d] == -(-c // 16) and lens[d] == c):
                    text[d] = text[src][:c]
        short += pages.short
        accounted(pages, blocks)
        for s in range(n):
            assert [int(content[pages.table[s][j // 16], j % 16, 0]) for j in range(lens[s])] == text[s][:lens[s]]
    assert 0 < short < 400


def test_commit():
    cache = np.arange(3 * 16).reshape(3, 16, 1).copy()
    lens = drafts.commit(cache, [[2, 0], [1, 1]], [20, 9], [0, 7, 10], [[0, 2, 5], [1, 1, -1]], [3, 2])
    assert lens == [16, 9]                                                         # the second path is not ascending
    want = np.arange(3 * 16).reshape(3, 16, 1)
    assert cache[2, 13:, 0].tolist() == [want[2, 13, 0], want[2, 15, 0], want[0, 2, 0]]
