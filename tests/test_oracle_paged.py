"""Pins of the float64 definitions in oracle/paged.py: closed forms, invariants, brute force."""
import numpy as np
import pytest

from oracle import paged


def _cache(rng, hkv, lens, dh, extra=2):
    pages = [-(-n // 16) for n in lens]
    n_blocks = sum(pages) + extra
    order = rng.permutation(n_blocks)
    table = np.full((len(lens), max(pages + [1])), -1)
    at = 0
    for s, p in enumerate(pages):
        table[s, :p] = order[at:at + p]
        at += p
    return rng.normal(size=(hkv, n_blocks, 16, dh)), rng.normal(size=(hkv, n_blocks, 16, dh)), table


def test_equal_keys_give_the_mean_of_the_visible_values():
    rng = np.random.default_rng(0)
    k, v, table = _cache(rng, 1, [40], 4)
    k[:] = 1.0
    q = rng.normal(size=(5, 2, 4))
    out, lse = paged.chunk_attention(q, k, v, table, [40], [0, 5], 0.5)
    vv = paged.token_rows(v, table[0], 40)[0]
    for i in range(5):
        n = 36 + i
        assert np.allclose(out[i, 0], vv[:n].mean(0)) and np.allclose(lse[i, 1], 0.5 * q[i, 1].sum() + np.log(n))
    out, _ = paged.chunk_attention(q, k, v, table, [40], [0, 5], 0.5, window=3, sinks=2)
    assert np.allclose(out[4, 0], vv[[0, 1, 37, 38, 39]].mean(0))


def test_scalar_brute_force_and_mass():
    rng = np.random.default_rng(1)
    lens, off = [33, 7, 16], [0, 4, 4, 9]
    k, v, table = _cache(rng, 2, lens, 3)
    q = rng.normal(size=(9, 4, 3))
    for window, sinks in ((0, 0), (5, 0), (6, 2)):
        out, lse = paged.chunk_attention(q, k, v, table, lens, off, 0.7, window, sinks)
        mass = paged.attention_mass(q, k, table, lens, off, 0.7, 40, window, sinks)
        want = np.zeros_like(mass)
        for s in range(3):
            for r in range(off[s], off[s + 1]):
                p = lens[s] - off[s + 1] + r
                for h in range(4):
                    z = {}
                    for j in range(p + 1):
                        if window == 0 or j > p - window or j < sinks:
                            z[j] = 0.7 * sum(q[r, h, d] * k[h // 2, table[s, j // 16], j % 16, d] for d in range(3))
                    tot = sum(np.exp(x) for x in z.values())
                    o = sum(np.exp(x) / tot * v[h // 2, table[s, j // 16], j % 16] for j, x in z.items())
                    assert np.allclose(out[r, h], o) and np.isclose(lse[r, h], np.log(tot))
                    for j, x in z.items():
                        want[s, h // 2, j] += np.exp(x) / tot
        assert np.allclose(mass, want)
        # every (row, head) hands out exactly 1
        assert np.isclose(mass.sum(), 9 * 4)


def test_rows_without_keys_and_append():
    rng = np.random.default_rng(2)
    k, v, table = _cache(rng, 1, [2], 4)
    q = rng.normal(size=(4, 1, 4))                       # four rows, two tokens: two rows sit before the first token
    out, lse = paged.chunk_attention(q, k, v, table, [2], [0, 4], 1.0)
    assert np.all(out[:2] == 0) and np.all(np.isneginf(lse[:2])) and np.all(np.isfinite(lse[2:]))
    new = rng.normal(size=(4, 1, 4))
    paged.append(k, new, table, [2], [0, 4])
    assert np.array_equal(k[0, table[0, 0], :2], new[2:, 0])


def test_chunks_equal_token_by_token():
    rng = np.random.default_rng(3)
    k, v, table = _cache(rng, 2, [50], 4)
    q = rng.normal(size=(20, 4, 4))
    whole, _ = paged.chunk_attention(q, k, v, table, [50], [0, 20], 0.5, 9, 3)
    for i in range(20):
        one, _ = paged.chunk_attention(q[i:i + 1], k, v, table, [31 + i], [0, 1], 0.5, 9, 3)
        assert np.allclose(one[0], whole[i])


@pytest.mark.parametrize("n,budget,sinks,recent", [(20, 8, 2, 3), (9, 8, 0, 0), (8, 8, 1, 1), (30, 1, 0, 1), (12, 6, 3, 3)])
def test_evict_keeps_the_best_and_moves_little(n, budget, sinks, recent):
    rng = np.random.default_rng(n + budget)
    mass = np.round(rng.exponential(size=n) * 4) / 4                   # ties
    pos = rng.permutation(n)
    src = paged.evict(mass, pos, budget, sinks, recent)
    assert len(set(src)) == len(src) == min(n, budget)
    kept = set(src)
    for i in range(n):
        if pos[i] < sinks or pos[i] > n - 1 - recent:
            assert i in kept
    free = [i for i in range(n) if not (pos[i] < sinks or pos[i] > n - 1 - recent)]
    for i in free:
        for j in free:
            if i in kept and j not in kept:
                assert mass[i] > mass[j] or (mass[i] == mass[j] and i < j)
    moved = [s for i, s in enumerate(src) if s != i]
    assert moved == sorted(moved) and all(s >= budget for s in moved)


def test_evict_counts_nan_least():
    mass = np.array([np.nan, 0.0, -np.inf, np.nan, 5.0])
    assert paged.evict_order(mass, range(5), 0, 0) == [4, 1, 2, 0, 3]
    assert paged.evict(mass, range(5), 2) == [4, 1]
