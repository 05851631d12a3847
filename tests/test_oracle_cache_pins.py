"""Pins of the cache oracle: the format against bit arithmetic, pages against their invariants, attention against a dense
softmax, commits against a second attention."""
import numpy as np
import pytest

from oracle import cache


def test_scale_bytes_are_e4m3():
    torch = pytest.importorskip("torch")
    want = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(cache.SCALES, want)


def test_nearest_scale_takes_the_even_one_of_two_as_near():
    for b in range(126):
        mid = (cache.SCALES[b] + cache.SCALES[b + 1]) / 2
        assert cache.nearest_scale(mid) == (b if b % 2 == 0 else b + 1)
        assert cache.nearest_scale(np.nextafter(mid, 0)) == b and cache.nearest_scale(np.nextafter(mid, 1e9)) == b + 1
    assert cache.nearest_scale(1e9) == 126 and cache.nearest_scale(0.0) == 0


@pytest.mark.parametrize("Dh", [64, 128])
def test_a_blocks_bytes_are_used_once(Dh):
    used = sorted(b for t in range(16) for part in cache.token_bytes(Dh, t) for b in part)
    assert used == list(range(18 * Dh))


@pytest.mark.parametrize("exp", [0, -3, 5])
def test_round_trip_is_within_half_a_step(exp):
    rng = np.random.default_rng(1)
    k, v = rng.normal(size=(5, 2, 64)) * 2.0 ** exp, rng.normal(size=(5, 2, 64)) * 2.0 ** exp
    pool = np.zeros((2, 2, 1, 18 * 64), np.uint8)
    kv, vv = cache.append(pool, 16, [3, 17, 31, -1, 0], k, v, exp, exp)
    for i, s in ((0, 3), (1, 17), (2, 31), (4, 0)):
        for h in range(2):
            got = cache.read(pool, 16, s, h, 64, exp, exp)
            assert np.array_equal(got[0], kv[i, h]) and np.array_equal(got[1], vv[i, h])
            for x, y in ((k[i, h], got[0]), (v[i, h], got[1])):
                for g in range(0, 64, 16):
                    step = cache.SCALES[cache.nearest_scale(np.abs(x[g:g + 16]).max() * 2.0 ** -exp / 7)] * 2.0 ** exp
                    assert np.abs(x[g:g + 16] - y[g:g + 16]).max() <= step / 2 * (1 + 1e-12)   # (scales here are normal: 7 steps reach the largest but for 1/16 of it)
    assert not kv[3].any()


def test_a_row_that_is_not_finite_is_nan_in_its_head_only():
    k = np.ones((1, 2, 64)); v = np.ones((1, 2, 64)); v[0, 1, 5] = np.inf
    pool = np.zeros((1, 2, 1, 18 * 64), np.uint8)
    kv, vv = cache.append(pool, 16, [4], k, v)
    assert np.isnan(kv[0, 1]).all() and np.isnan(vv[0, 1]).all() and np.isfinite(kv[0, 0]).all()
    assert np.isnan(cache.read(pool, 16, 4, 1, 64)[0]).all()


def test_reserve_keeps_pages_apart_and_gives_them_back():
    rng = np.random.default_rng(2)
    B, ps, pages, R = 5, 16, 40, 9
    table, held = np.full((B, 20), -1), [0] * B
    free, count = list(rng.permutation(pages)), pages
    seq = [0] * B
    for rnd in range(12):
        rows = [int(rng.integers(1, R + 1)) for _ in range(B)]
        before = [s if not (rnd == 7 and b == 2) else -1 for b, s in enumerate(seq)]
        table, held, free, count, slots, status = cache.reserve(ps, pages, before, rows, held, free, count, table, R)
        pages_held = [int(p) for b in range(B) for p in table[b, :held[b]]]
        assert len(set(pages_held)) == len(pages_held) and sorted(pages_held + [int(p) for p in free[:count]]) == list(range(pages))
        used = slots[slots >= 0]
        assert len(set(used.tolist())) == used.size
        for b in range(B):
            assert (slots[b] >= 0).sum() == (rows[b] if before[b] >= 0 and status[b] == 0 else 0)
            if before[b] < 0:
                seq[b] = 0
            elif status[b] == 0:
                seq[b] += rows[b]
    assert held[2] < max(held)


def test_attention_of_a_chain_is_causal_softmax():
    rng = np.random.default_rng(3)
    Dh, L, rows = 64, 21, 3
    pool = np.zeros((2, 1, 1, 18 * Dh), np.uint8)
    slots = [16 + i for i in range(16)] + [i for i in range(8)]
    k, v = rng.normal(size=(24, 1, Dh)), rng.normal(size=(24, 1, Dh))
    kv, vv = cache.append(pool, 16, slots, k, v)
    q = rng.normal(size=(rows, 2, Dh))
    out, lse = cache.attention(pool, 16, [1, 0], L, rows, q, None, 0.125)
    for i in range(rows):
        x = 0.125 * kv[:L + i + 1, 0] @ q[i, 1]
        w = np.exp(x) / np.exp(x).sum()
        assert np.allclose(out[i, 1], w @ vv[:L + i + 1, 0]) and np.allclose(lse[i, 1], np.log(np.exp(x).sum()))


def test_commit_makes_a_path_the_prefix():
    """The last row of an accepted path sees the same tokens before the commit, by its mask, and after it, as the prefix."""
    rng = np.random.default_rng(4)
    Dh, L, parent = 64, 13, [-1, -1, 0, 1, 3, 2]
    n = len(parent)
    words = []
    for i, p in enumerate(parent):
        words.append([(words[p][0] if p >= 0 else 0) | 1 << i])
    pool = np.zeros((1, 3, 1, 1, 18 * Dh), np.uint8)
    row = [2, 0, 1]
    slots = [row[p // 16] * 16 + p % 16 for p in range(L + 1 + n)]
    cache.append(pool[0], 16, slots, rng.normal(size=(len(slots), 1, Dh)), rng.normal(size=(len(slots), 1, Dh)))
    q = rng.normal(size=(1 + n, 1, Dh))
    path = [1, 3, 4]
    before, _ = cache.attention(pool[0], 16, row, L, 1 + n, q, words, 0.1)
    new = cache.commit(pool, 16, row, L, len(path), path, n)
    assert new == L + 4
    after, _ = cache.attention(pool[0], 16, row, new - 1, 1, q[[1 + path[-1]]], None, 0.1)   # (its own row is the last token)
    assert np.allclose(before[1 + path[-1]], after[0])
