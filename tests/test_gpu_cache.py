"""GPU parity of the 4-bit cache calls against their oracle (oracle/cache.py): pages and slots, the write, the commit exactly;
the attention within tolerances that count its roundings.

Tolerances of the attention.  Scores: q is exact in the kernels (bf16 in fp16 after a power of two, fp32 as two fp16 parts to
2^-22), keys are exact, sums of Dh products are held in fp32; with S = scale * max sum |q_d k_d| a score is off by at most
e = S * (2^-22 + 16 * 2^-23) (16: steps of accumulation, each of at most one unit in the last place), in fp32 and bf16 alike.
Weights: exp2 to 2^-22, then rounded to fp16 (half a step: 2^-11; fp32: two parts, 2^-22), and the sum of weights likewise:
a weight's relative error is at most w = 2 e + 2^-21 + 2^-11 (bf16) or 2 e + 2^-20 (fp32).  So |error| <= w * sum p |v| +
accumulation of O in fp32 (L / 16 steps of 2^-23 of at most sum p |v|) + half a step of the result's type; sum p |v| <= max |v|.
lse: e + 2^-21 + L / 16 steps of 2^-24 of the sum + half a step of fp32."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2609_22098_b200 import binding, synth
from paper_2609_22098_b200.binding import CacheLayout, TreeSpark, TreeSparkError

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def context(Nmax=16, B=8, D=4, dtype=BF16):
    return TreeSpark(V=1024, D=D, r=8, K=4, Nmax=Nmax, max_batch=B, dtype=dtype)


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def random_table(rng, lens, ps, cols, n_pages):
    """A table whose pages lie anywhere in the pool; unused entries -1."""
    order = rng.permutation(n_pages)
    table, at = np.full((len(lens), cols), -1, np.int64), 0
    for b, n in enumerate(lens):
        need = -(-n // ps)
        table[b, :need] = order[at:at + need]
        at += need
    return table


def slot_of(table, b, pos, ps):
    return int(table[b, pos // ps]) * ps + pos % ps


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype,Hkv,Dh,ps,rows,ld,exps", [
    (BF16, 2, 128, 16, 37, "tight", (0, 0)), (BF16, 3, 64, 48, 21, "wide", (0, 0)), (F32, 1, 128, 32, 19, "wide", (-4, 3)),
    (F32, 2, 64, 16, 1, "tight", (2, -2)), (BF16, 8, 128, 128, 9, "wide", (1, 0)), (F32, 5, 64, 80, 33, "tight", (0, 0)), (BF16, 1, 64, 16, 16, "wide", (30, -30))])
def test_append_writes_the_oracles_bytes(dtype, Hkv, Dh, ps, rows, ld, exps):
    rng = np.random.default_rng(rows)
    pages = -(-2 * rows // ps) + 2
    ts, lay = context(dtype=dtype), CacheLayout(Hkv, Hkv, Dh, ps, pages, 4, dtype, *exps)
    wide = 2 if ld == "wide" else 1
    x = torch.tensor(rng.normal(size=(rows, wide, 2, Hkv, Dh)), device="cuda").to(dtype)
    x[:, :, 0] *= 2.0 ** exps[0]
    x[:, :, 1] *= 2.0 ** exps[1]
    x[::5, 0, 0, 0, :16] = 0          # a group of zeros
    x[1::5, 0, 0, 0, 16:32] *= 1e-3   # scales among the subnormals
    x[2::5, 0, 1, 0, :16] *= 300.0    # scales that saturate
    x[3::7, 0, 0, 0, 3] = float("nan")
    x[4::7, 0, 1, Hkv - 1, 7] = float("inf")
    # values half-way between codes and scales half-way between two
    x[0, 0, 0, 0, 32:48] = torch.tensor([7, 0.5, 1.5, -2.5, 3.5, -0.5, 6.5, -6.5, 4.5, 5.5, 2.5, -3.5, 0, 1, -1, 0.25], device="cuda").to(dtype) * 2.0 ** exps[0]
    x[0, 0, 1, 0, 32] = 7 * 1.0625 * 2.0 ** exps[1]
    k, v = (x[:, 0, 0], x[:, 0, 1]) if wide == 2 else (x[:, 0, 0].contiguous(), x[:, 0, 1].contiguous())
    slots = rng.permutation(pages * ps)[:rows]
    slots[2::9] = -1
    if rows > 8:
        slots[7] = pages * ps          # outside the pool
    start = rng.integers(0, 256, (pages, Hkv, ps // 16, 18 * Dh), dtype=np.uint8)
    pool = torch.from_numpy(start.copy()).cuda()
    k_val, v_val = (torch.full((rows, Hkv, Dh), -7.0, dtype=dtype, device="cuda") for _ in range(2))
    ts.cache_append(lay, k, v, i32(slots), pool, k_val, v_val)
    kv, vv = oc.append(start, ps, slots, k.double().cpu().numpy(), v.double().cpu().numpy(), *exps)
    assert np.array_equal(pool.cpu().numpy(), start)
    held = (slots >= 0) & (slots < pages * ps)
    for got, want in ((k_val, kv), (v_val, vv)):
        got = got.double().cpu().numpy()
        assert np.array_equal(got[held], want[held], equal_nan=True) and (got[~held] == -7.0).all()
    again = torch.from_numpy(start.copy()).cuda()
    ts.cache_append(lay, k, v, i32(slots), again)     # without values; the same bytes again
    assert torch.equal(again, pool)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_rounds_codes_to_the_nearest_even(dtype):
    """Values at every border between two codes and a last place to either side, for all scales."""
    Dh, ps = 64, 16
    scales = [float(x) for x in torch.arange(1, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).float()]
    near = []
    for s in scales:
        t = torch.tensor([7 * s] + [(c + 0.5) * s for c in range(-8, 7)], dtype=torch.float64).to(dtype)   # (borders of bf16 values are rounded: they are near one then)
        up, down = (torch.nextafter(t, torch.full_like(t, d)) for d in (float("inf"), float("-inf")))
        up[0] = down[0] = t[0]
        near += [t, up, down, -t]
    x = torch.stack(near).reshape(-1, 1, Dh)
    rows = x.shape[0]
    ts, lay = context(dtype=dtype), CacheLayout(1, 1, Dh, ps, -(-rows // ps), 4, dtype)
    start = np.zeros(lay.pool_shape(), np.uint8)
    pool = torch.from_numpy(start.copy()).cuda()
    k_val, v_val = (torch.zeros(rows, 1, Dh, dtype=dtype, device="cuda") for _ in range(2))
    ts.cache_append(lay, x.cuda(), x.flip(0).contiguous().cuda(), i32(range(rows)), pool, k_val, v_val)
    kv, vv = oc.append(start, ps, list(range(rows)), x.double().numpy(), x.flip(0).double().numpy(), 0, 0)
    assert np.array_equal(pool.cpu().numpy(), start)
    assert np.array_equal(k_val.double().cpu().numpy(), kv) and np.array_equal(v_val.double().cpu().numpy(), vv)


def test_append_beyond_32_bit_offsets():
    Dh, ps = 128, 16
    pages = (5 << 30) // (18 * Dh)
    ts, lay = context(), CacheLayout(1, 1, Dh, ps, pages, 4, BF16)
    pool = torch.zeros(lay.pool_shape(), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(3)
    k, v = (torch.tensor(rng.normal(size=(3, 1, Dh)), device="cuda").to(BF16) for _ in range(2))
    slots = [pages * ps - 1, (4 << 30) // (18 * Dh) * ps + 5, 0]
    ts.cache_append(lay, k, v, i32(slots), pool)
    for i, s in enumerate(slots):
        small = np.zeros((1, 1, 1, 18 * Dh), np.uint8)
        oc.append(small, ps, [s % ps], k[i:i + 1].double().cpu().numpy(), v[i:i + 1].double().cpu().numpy())
        assert np.array_equal(pool[s // ps].cpu().numpy(), small[0])
    assert torch.nonzero(pool.flatten(1).amax(1)).flatten().tolist() == sorted(s // ps for s in slots)
    # and read there by the attention and the commit
    q = torch.tensor(rng.normal(size=(1, 1, 1, Dh)), device="cuda").to(BF16)
    kk, vv = (torch.tensor(rng.normal(size=(2, 1, Dh)), device="cuda").to(BF16) for _ in range(2))
    last = pages - 1
    ts.cache_append(lay, kk, vv, i32([last * ps, last * ps + 1]), pool)
    table = i32([[last, -1, -1, -1]])
    lse = torch.zeros(1, 1, 1, device="cuda")
    out = ts.tree_attention(lay, q, pool, table, i32([1]), lse=lse)
    small = np.zeros((1, 1, 1, 18 * Dh), np.uint8)
    oc.append(small, ps, [0, 1], kk.double().cpu().numpy(), vv.double().cpu().numpy())
    want, wl = oc.attention(small, ps, [0], 1, 1, q[0].double().cpu().numpy(), None, Dh ** -0.5)
    assert np.abs(out[0].double().cpu().numpy() - want).max() < 2 ** -7 * np.abs(want).max() and abs(float(lse) - float(wl.item())) < 1e-4
    before = pool[last].clone()
    ts.cache_commit(lay, pool, table, i32([0]), i32([1]), torch.tensor([[3, 0, 0, 0]], dtype=torch.int32, device="cuda"))
    now = before.cpu().numpy()[None, None]
    oc.commit(now, ps, [0], 0, 1, [3], 16)
    assert np.array_equal(pool[last].cpu().numpy(), now[0, 0])


# ------------------------------------------------------------------------------------------------ reserve
def check_reserve(ts, lay, seq, n_nodes, held, free, count, table, in_place):
    B, R = len(seq), 1 if n_nodes is None else ts.Nmax + 1
    rows = [1] * B if n_nodes is None else [min(max(n, 0), ts.Nmax) + 1 for n in n_nodes]
    w = oc.reserve(lay.page_size, lay.n_pages, seq, rows, held, free, count, table, R)
    g = dict(seq=i32(seq), held=i32(held), free=i32(free), count=i32([count]), table=i32(table))
    out = None if in_place else dict(held=torch.full((B,), -9, dtype=torch.int32, device="cuda"), free_count=i32([-9]),
                                     slot_map=torch.full((B, R), -9, dtype=torch.int32, device="cuda"), status=i32([-9] * B))
    o = ts.cache_reserve(lay, g["seq"], g["held"], g["free"], g["count"], g["table"], n_nodes=None if n_nodes is None else i32(n_nodes), out=out)
    assert o["status"].tolist() == w[5]
    assert np.array_equal(g["table"].cpu().numpy(), w[0]) and o["held"].tolist() == w[1] and int(o["free_count"]) == w[3]
    assert g["free"].tolist()[:w[3]] == [int(p) for p in w[2][:w[3]]]
    assert np.array_equal(o["slot_map"].cpu().numpy(), w[4])
    if in_place:
        assert o["held"] is g["held"]
    else:
        assert g["held"].tolist() == list(held) and int(g["count"]) == count
    return w


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,cols,pages,ps,Nmax,seed", [(1, 4, 3, 16, 5, 0), (2, 4000, 5000, 16, 4, 7), (3, 30000, 40000, 16, 4, 8), (7, 40, 150, 16, 64, 1), (33, 9, 200, 48, 16, 2), (600, 300, 60000, 16, 16, 3), (700, 3, 900, 32, 1, 4),
                                                        (8, 20, 60, 16, 200, 5), (1500, 100, 4000, 16, 8, 6)])
def test_reserve_matches_the_oracle(B, cols, pages, ps, Nmax, seed, in_place):
    """Rounds with finished, refused, idle and growing requests, on the one-cluster form and (above 64 requests or 65,536 entries) on
    many CTAs."""
    rng = np.random.default_rng(seed)
    ts, lay = context(Nmax, B), CacheLayout(4, 2, 64, ps, pages, cols)
    free, count, table, held = rng.permutation(pages), pages, np.full((B, cols), -1, np.int64), [0] * B
    for rnd in range(5):
        seq = rng.integers(0, max(1, int(1.1 * min(cols * ps, 2 * pages * ps / B))), B)
        seq[rng.random(B) < 0.2] = -1
        if rnd == 3:
            seq[:] = -1
        n_nodes = None if rnd == 4 else rng.integers(-2, Nmax + 3, B)
        table, held, free, count, _, status = check_reserve(ts, lay, seq, n_nodes, held, free, count, table, in_place)
        if rnd == 3:
            assert count == pages and sorted(int(p) for p in free) == list(range(pages))


def test_reserve_of_an_empty_list_and_entries_that_are_no_pages():
    ts, lay = context(4, 4), CacheLayout(4, 2, 64, 16, 8, 4)
    check_reserve(ts, lay, [0, 3, 20, -1], [0, 1, 2, 3], [0, 1, 1, 0], list(range(8)), 0, np.array([[-1] * 4, [2, -1, -1, -1], [3, -1, -1, -1], [-1] * 4]), True)
    check_reserve(ts, lay, [0, 3, 20, 70], [0, 1, 2, 3], [0, 1, 1, 0], list(range(8)), 8, np.array([[-1] * 4, [99, -1, -1, -1], [3, -1, -1, -1], [-1] * 4]), False)


# ------------------------------------------------------------------------------------------------ attention
def tree_masks(rng, B, N, n_nodes, chance=0.7):
    """Ancestor bitmasks (canonical order) with bits behind the last node set at random: those do not count."""
    words = (N + 63) // 64
    mask = rng.integers(0, 2 ** 63, (B, N, words), dtype=np.int64).astype(np.uint64)
    for b in range(B):
        p = -1
        for i in range(n_nodes[b]):
            p = min(i - 1, p + int(rng.random() < chance)) if i else -1
            row = mask[b, p].copy() if p >= 0 else np.zeros(words, np.uint64)
            for w in range(words):
                keep = max(0, min(64, n_nodes[b] - 64 * w))
                low = np.uint64((1 << keep) - 1)
                row[w] = (row[w] & low) | (mask[b, i, w] & ~low)
            row[i // 64] |= np.uint64(1 << (i % 64))
            mask[b, i] = row
    return mask


def tolerance(dtype, S, vmax, L):
    e = S * (2.0 ** -22 + 16 * 2.0 ** -23)
    w = 2 * e + (2.0 ** -21 + 2.0 ** -11 if dtype == BF16 else 2.0 ** -20)
    steps = L / 16 + 16
    return w * vmax + steps * 2.0 ** -23 * vmax, 2.0 ** -8 if dtype == BF16 else 2.0 ** -24, e + 2.0 ** -21 + steps * 2.0 ** -24


def check_attention(ts, dtype, Hq, Hkv, Dh, ps, lens, n_nodes, mode, seed, exps=(0, 0), wide=False, scale=None, poison=None, lift=1.0, junk=255):
    """One call against the oracle.  mode: "one" (no n_nodes), "chain" (no mask), "tree".  poison: rows of request 0 that hold a NaN."""
    rng = np.random.default_rng(seed)
    B, N = len(lens), ts.Nmax
    R = 1 if mode == "one" else N + 1
    rows = [1] * B if mode == "one" else [min(max(n, 0), N) + 1 for n in n_nodes]
    total = [max(0, n) + r for n, r in zip(lens, rows)]
    cols = max(-(-n // ps) for n in total) + 2
    pages = sum(-(-n // ps) for n in total) + 3
    lay = CacheLayout(Hq, Hkv, Dh, ps, pages, cols, dtype, *exps)
    table = random_table(rng, total, ps, cols, pages)
    pool = np.full((pages, Hkv, ps // 16, 18 * Dh), junk, np.uint8)       # NaN scales wherever nothing has been written
    gpool = torch.from_numpy(pool.copy()).cuda()
    S = vmax = 0.0
    scale = Dh ** -0.5 if scale is None else scale
    q = (torch.tensor(rng.normal(size=(B, R, Hq * (2 if wide else 1), Dh)), device="cuda") * 1.5 * lift).to(dtype)[:, :, :Hq]
    for b in range(B):
        k = torch.tensor(rng.normal(size=(total[b], Hkv, Dh)) * 2.0 ** exps[0] / lift).to(dtype)
        v = torch.tensor(rng.normal(size=(total[b], Hkv, Dh)) * 2.0 ** exps[1]).to(dtype)
        if b == 0 and poison:
            for r in poison:
                (k if r % 2 else v)[max(0, lens[0]) + r, 0, r % Dh] = float("nan")
        slots = [slot_of(table, b, p, ps) for p in range(total[b])]
        kv, vv = oc.append(pool, ps, slots, k.double().numpy(), v.double().numpy(), *exps)
        ts.cache_append(lay, k.cuda(), v.cuda(), i32(slots), gpool)
        G = Hq // Hkv
        qa = q[b, :rows[b]].double().abs().cpu().numpy().reshape(rows[b], Hkv, G, Dh)
        S = max(S, abs(scale) * float(np.einsum("rhgd,thd->rhgt", qa, np.nan_to_num(np.abs(kv))).max()))
        vmax = max(vmax, float(np.nanmax(np.abs(vv))))
    mask = tree_masks(rng, B, N, [r - 1 for r in rows]) if mode == "tree" else None
    out = torch.full((B, R, Hq * (2 if wide else 1), Dh), -3.0, dtype=dtype, device="cuda")[:, :, :Hq]
    lse = torch.full((B, R, Hq), -5.0, device="cuda")
    ts.tree_attention(lay, q, gpool, i32(table), i32(lens), n_nodes=None if mode == "one" else i32(n_nodes),
                      mask=None if mask is None else torch.from_numpy(mask.view(np.int64)).cuda(), scale=scale, out=out, lse=lse)
    tol, half, tol_lse = tolerance(dtype, S, vmax, max(total))
    og, lg = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in range(B):
        if lens[b] < 0:
            assert (og[b] == -3.0).all() and (lg[b] == -5.0).all()
            continue
        want, wl = oc.attention(pool, ps, table[b], lens[b], rows[b], q[b].double().cpu().numpy(), None if mask is None else mask[b], scale, *exps)
        assert (og[b, rows[b]:] == -3.0).all() and (lg[b, rows[b]:] == -5.0).all(), b
        o, l = og[b, :rows[b]], lg[b, :rows[b]]
        assert np.array_equal(np.isnan(o), np.isnan(want)) and np.array_equal(np.isnan(l), np.isnan(wl)), b
        fine = ~np.isnan(want)
        err = np.abs(o - want)[fine] - half * np.abs(want[fine])
        assert not fine.any() or err.max() <= tol, (b, float(err.max()), tol)
        fine = np.isfinite(wl)
        assert np.array_equal(l[~fine & ~np.isnan(wl)], wl[~fine & ~np.isnan(wl)])
        assert not fine.any() or (np.abs(l - wl)[fine] - 2.0 ** -23 * np.abs(wl[fine])).max() <= tol_lse, b
    return out, lse


SHAPES = [  # dtype, Hq, Hkv, Dh, page size
    (BF16, 4, 1, 128, 16), (BF16, 8, 8, 64, 32), (BF16, 6, 2, 128, 48), (BF16, 16, 1, 64, 16), (BF16, 10, 2, 128, 64), (F32, 4, 2, 128, 16), (F32, 3, 3, 64, 80), (F32, 12, 1, 64, 16)]


@pytest.mark.parametrize("dtype,Hq,Hkv,Dh,ps", SHAPES)
def test_single_tokens(dtype, Hq, Hkv, Dh, ps):
    check_attention(context(dtype=dtype), dtype, Hq, Hkv, Dh, ps, [0, 1, 15, 16, 17, 150, -1, 63], None, "one", 11)


@pytest.mark.parametrize("dtype,Hq,Hkv,Dh,ps", SHAPES)
def test_trees_and_chains(dtype, Hq, Hkv, Dh, ps):
    ts = context(Nmax=21, dtype=dtype)
    check_attention(ts, dtype, Hq, Hkv, Dh, ps, [0, 7, 33, 100, -1, 16], [5, 21, 0, 13, 4, 30], "tree", 12)
    check_attention(ts, dtype, Hq, Hkv, Dh, ps, [0, 31, 80, 16], [21, -2, 9, 15], "chain", 13, wide=True)


@pytest.mark.parametrize("dtype,Hq,Hkv,Dh,N,n", [(BF16, 4, 1, 128, 256, 256), (BF16, 2, 2, 64, 130, 129), (F32, 2, 1, 64, 100, 65), (BF16, 24, 1, 128, 64, 64)])
def test_trees_of_many_words(dtype, Hq, Hkv, Dh, N, n):
    check_attention(context(Nmax=N, dtype=dtype), dtype, Hq, Hkv, Dh, 16, [40, 3], [n, n // 2], "tree", 14)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_nan_in_the_cache_reaches_the_rows_that_see_it_and_no_other(dtype):
    ts = context(Nmax=21, dtype=dtype)
    check_attention(ts, dtype, 4, 2, 128, 16, [20, 30], [21, 8], "tree", 15, poison=[5, 8, 17])
    check_attention(ts, dtype, 4, 2, 64, 32, [0, 30], [12, 8], "chain", 16, poison=[3, 9])
    check_attention(ts, dtype, 4, 2, 64, 32, [9, 30], [12, 8], "tree", 17, poison=[0])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("exps,scale,lift", [((5, -4), 0.002, 1.0), ((-20, 25), 100.0, 1.0), ((0, 0), -0.09, 1.0), ((0, 0), 0.0, 1.0), ((0, 0), 0.09, 2.0 ** 8), ((0, 0), 2.0 ** -60, 2.0 ** 60)])
def test_exponents_and_scales(dtype, exps, scale, lift):
    """Powers of two of the cache, scales of any sign, queries far from unit size (2^60 with a scale that takes it back)."""
    ts = context(Nmax=9, dtype=dtype)
    if lift > 2.0 ** 20:   # keys as usual, the product of query and scale as usual
        check_attention(ts, dtype, 4, 2, 128, 16, [40, 5], [9, 3], "tree", 18, exps=(-30, 0), scale=scale * 2.0 ** 30 * 0.09, lift=1.0)
    check_attention(ts, dtype, 4, 2, 128, 16, [40, 5], [9, 3], "tree", 18, exps=exps, scale=scale * 0.09 if lift > 2.0 ** 20 else scale, lift=lift if lift < 2.0 ** 20 else 1.0)


def test_queries_that_are_not_finite_spoil_their_rows_only():
    ts = context(Nmax=5)
    lay = CacheLayout(2, 1, 64, 16, 8, 4)
    rng = np.random.default_rng(0)
    pool = torch.zeros(lay.pool_shape(), dtype=torch.uint8, device="cuda")
    kv = torch.tensor(rng.normal(size=(2, 26, 1, 64)), device="cuda").to(BF16)
    table = i32([[3, 5, -1, -1]])
    ts.cache_append(lay, kv[0], kv[1], i32([3 * 16 + i for i in range(16)] + [5 * 16 + i for i in range(10)]), pool)
    q = torch.tensor(rng.normal(size=(1, 6, 2, 64)), device="cuda").to(BF16)
    args = dict(n_nodes=i32([5]))
    good = ts.tree_attention(lay, q, pool, table, i32([20]), **args)
    bad = q.clone()
    bad[0, 2, 1, 9] = float("inf")
    bad[0, 4, 0, 0] = float("nan")
    got = ts.tree_attention(lay, bad, pool, table, i32([20]), **args)
    hit = torch.zeros(1, 6, 2, dtype=torch.bool, device="cuda")
    hit[0, 2, 1] = hit[0, 4, 0] = True
    assert torch.equal(got[~hit], good[~hit]) and torch.isnan(got[hit]).all()


def test_absent_pages_and_empty_rows():
    """Entries outside the pool are absent tokens; a row that sees nothing is 0 with lse -inf."""
    ts = context(Nmax=5)
    lay = CacheLayout(4, 2, 128, 16, 8, 3)
    rng = np.random.default_rng(1)
    pool = np.full((8, 2, 1, 18 * 128), 255, np.uint8)
    kv = rng.normal(size=(2, 16, 2, 128))
    kv = torch.tensor(kv).to(BF16).double().numpy()
    oc.append(pool, 16, [2 * 16 + i for i in range(16)], kv[0], kv[1])
    q = torch.tensor(rng.normal(size=(5, 6, 4, 128)), device="cuda").to(BF16)
    table = np.array([[-1, 2, -1], [-1, -1, -1], [2, 8, 1 << 30], [2, -5, -1], [2, -1, -1]])
    seq = [20, 3, 16, 40, 300]                  # the last has fewer table columns than tokens
    n = [5, 5, 5, 2, 5]
    out, lse = torch.full((5, 6, 4, 128), -3.0, dtype=BF16, device="cuda"), torch.full((5, 6, 4), -5.0, device="cuda")
    ts.tree_attention(lay, q, torch.from_numpy(pool).cuda(), i32(table), i32(seq), n_nodes=i32(n), out=out, lse=lse)
    for b in range(5):
        want, wl = oc.attention(pool, 16, table[b], seq[b], n[b] + 1, q[b].double().cpu().numpy(), None, 128 ** -0.5)
        o, l = out[b, :n[b] + 1].double().cpu().numpy(), lse[b, :n[b] + 1].double().cpu().numpy()
        assert np.array_equal(np.isneginf(l), np.isneginf(wl)) and np.abs(o - want).max() <= 2.0 ** -8 * np.abs(want).max() + 4 * 2.0 ** -11
        assert (o[np.isneginf(wl)] == 0).all() and np.abs(l[np.isfinite(wl)] - wl[np.isfinite(wl)]).max(initial=0) < 1e-4
        assert b != 1 or np.isneginf(wl).all()


# ---- long contexts and large batches: the same formula in float64 on the device
def decode64(pool, slots, Dh):
    """K, V [tokens][Hkv][Dh] of slots, float64."""
    ps = pool.shape[2] * 16
    at = torch.tensor([np.concatenate(oc.token_bytes(Dh, t)) for t in range(16)], device="cuda")
    rows = pool[slots // ps, :, slots % ps // 16]                             # [tokens][Hkv][18 Dh]
    rows = torch.gather(rows, 2, at[slots % 16][:, None].expand(-1, pool.shape[1], -1))
    sc = torch.tensor(np.append(oc.SCALES, np.nan), device="cuda")
    out = []
    for c0, s0 in ((0, Dh), (Dh // 2, Dh + Dh // 16)):
        b = rows[..., c0:c0 + Dh // 2].unflatten(-1, (-1, 4)).long()
        nib = torch.stack([(b[..., (e // 2 + 4 * (e % 2)) // 2] >> (4 * ((e // 2 + 4 * (e % 2)) % 2))) & 15 for e in range(8)], -1).flatten(-2)
        out.append((nib - 8).double() * sc[rows[..., s0:s0 + Dh // 16].long()].repeat_interleave(16, -1))
    return out


def random_pool(rng_seed, shape):
    """Codes of all values and scales between 2^-3 and 2^-1."""
    g = torch.Generator(device="cuda").manual_seed(rng_seed)
    pool = torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)
    Dh = shape[-1] // 18
    pool[..., 16 * Dh:] = torch.randint(32, 48, (*shape[:-1], 2 * Dh), generator=g, device="cuda", dtype=torch.uint8)
    return pool


@pytest.mark.parametrize("dtype,Hq,Hkv,Dh,ps,lens,N,n_nodes", [
    (BF16, 4, 1, 128, 16, [70001], 7, None), (BF16, 8, 1, 64, 64, [33000, 5], 7, [7, 3]), (F32, 2, 1, 128, 32, [40000], 7, [5]), (BF16, 32, 8, 128, 16, [4000, 17, 901, 2500], 64, [64, 30, 7, 12]),
    (BF16, 40, 4, 128, 128, [3000, 5000], 40, [40, 17]), (BF16, 8, 2, 64, 16, list(range(0, 640, 2)), 7, [b % 8 for b in range(320)]), (BF16, 16, 1, 128, 16, [1000] * 50, 7, None),
    (F32, 8, 4, 64, 16, [700] * 20, 7, [3] * 20), (F32, 8, 2, 64, 64, [33000, 5], 7, [7, 3]), (BF16, 64, 2, 128, 16, [9000, 2000], 256, [256, 100])])
def test_long_contexts_and_large_batches(dtype, Hq, Hkv, Dh, ps, lens, N, n_nodes):
    B = len(lens)
    ts = context(Nmax=N, B=B, dtype=dtype)
    rng = np.random.default_rng(len(lens))
    rows = [1 + (n_nodes[b] if n_nodes else 0) for b in range(B)]
    total = [n + r for n, r in zip(lens, rows)]
    cols, pages = max(-(-n // ps) for n in total) + 1, sum(-(-n // ps) for n in total) + 2
    lay = CacheLayout(Hq, Hkv, Dh, ps, pages, cols, dtype)
    table = random_table(rng, total, ps, cols, pages)
    pool = random_pool(5, lay.pool_shape())
    R = 1 if n_nodes is None else N + 1
    q = torch.randn(B, R, Hq, Dh, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(dtype)
    mask = tree_masks(rng, B, N, [r - 1 for r in rows]) if n_nodes else None
    out, lse = torch.zeros_like(q), torch.zeros(B, R, Hq, device="cuda")
    gt, gm = i32(table), None if mask is None else torch.from_numpy(mask.view(np.int64)).cuda()
    args = (lay, q, pool, gt, i32(lens))
    kw = dict(n_nodes=None if n_nodes is None else i32(n_nodes), mask=gm)
    ts.tree_attention(*args, **kw, out=out, lse=lse)
    again, lse2 = torch.zeros_like(q), torch.zeros_like(lse)
    ts.tree_attention(*args, **kw, out=again, lse=lse2, ws=torch.full_like(ts.attention_workspace(lay, B), 255))
    assert torch.equal(out, again) and torch.equal(lse, lse2)      # nothing depends on timing or on the workspace's contents
    for b in list(range(B))[:: max(1, B // 12)]:
        pos = torch.arange(total[b], device="cuda")
        K, V = decode64(pool, gt[b].long()[pos // ps] * ps + pos % ps, Dh)
        see = np.array([[t < lens[b] or oc.sees(None if mask is None else mask[b], i, t - lens[b]) for t in range(lens[b], total[b])] for i in range(rows[b])])
        see = torch.cat([torch.ones(rows[b], lens[b], dtype=torch.bool), torch.from_numpy(see)], 1).cuda()
        qb = q[b, :rows[b]].double().unflatten(1, (Hkv, Hq // Hkv))
        x = torch.einsum("rhgd,thd->rhgt", qb, K) * Dh ** -0.5
        x = x.masked_fill(~see[:, None, None], float("-inf"))
        z = torch.logsumexp(x, -1)
        want = torch.einsum("rhgt,thd->rhgd", torch.exp(x - z[..., None]), V).flatten(1, 2)
        S = float((Dh ** -0.5) * torch.einsum("rhgd,hd->rhg", qb.abs(), K.abs().amax(0)).max())
        tol, half, tol_lse = tolerance(dtype, S, float(V.abs().max()), total[b])
        err = (out[b, :rows[b]].double() - want).abs() - half * want.abs()
        assert float(err.max()) <= tol, (b, float(err.max()), tol)
        assert float((lse[b, :rows[b]].double() - z.flatten(1)).abs().max()) <= tol_lse + 2.0 ** -23 * float(z.abs().max())


# ------------------------------------------------------------------------------------------------ commit
@pytest.mark.parametrize("B,layers,Hkv,Dh,ps,D,N,in_place", [(1, 1, 1, 128, 16, 4, 16, True), (5, 3, 2, 64, 16, 16, 40, False), (9, 37, 8, 128, 32, 8, 64, True), (3, 2, 3, 64, 80, 1, 1, False), (2, 70, 8, 64, 16, 4, 16, True)])
def test_commit_moves_the_oracles_bytes(B, layers, Hkv, Dh, ps, D, N, in_place):
    """Paths with nodes in place, nodes that lie in other targets, the longest and the empty path, and nodes that are none."""
    rng = np.random.default_rng(B)
    ts = context(N, B, D)
    seq = [int(x) for x in rng.integers(0, 90, B)]
    if B > 2:
        seq[2] = -1
    total = [max(0, s) + N + 1 for s in seq]
    cols, pages = max(-(-n // ps) for n in total), sum(-(-n // ps) for n in total) + 1
    lay = CacheLayout(2 * Hkv, Hkv, Dh, ps, pages, cols)
    table = random_table(rng, total, ps, cols, pages)
    pool = rng.integers(0, 256, (layers, *lay.pool_shape()), dtype=np.uint8)
    acc_len = rng.integers(0, min(D, N) + 1, B)
    acc_len[0] = min(D, N)
    node = np.zeros((B, D), np.int64)
    for b in range(B):
        node[b, :acc_len[b]] = np.sort(rng.permutation(N)[:acc_len[b]])
    if B > 3:
        acc_len[3], node[3, 0] = max(1, acc_len[3]), N       # no such node
        acc_len[4], node[4, :3] = 3, [2, 1, 0]               # any order: sources are read before targets are written
        table[4, -1] = -1
    g, seq_g = torch.from_numpy(pool.copy()).cuda(), i32(seq)
    new = ts.cache_commit(lay, g if layers > 1 else g[0], i32(table), seq_g, i32(acc_len), i32(node), None if in_place else torch.zeros(B, dtype=torch.int32, device="cuda"))
    want = [oc.commit(pool, ps, table[b], seq[b], int(acc_len[b]), node[b], N) for b in range(B)]
    assert new.tolist() == want and (new is seq_g) == in_place and (in_place or seq_g.tolist() == seq)
    assert np.array_equal(g.cpu().numpy(), pool)


# ------------------------------------------------------------------------------------------------ together
def round_inputs(wl, B, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    A = (torch.randn(wl.V, wl.r, generator=g, device="cuda") * 0.2).to(BF16)
    W = (torch.randn(wl.r, wl.V, generator=g, device="cuda") * 0.5).to(BF16)
    U = (torch.randn(B, wl.D, wl.V, generator=g, device="cuda") * 3).to(BF16)
    U.scatter_add_(2, torch.randint(0, wl.V, (B, wl.D, 1), generator=g, device="cuda"), torch.full((B, wl.D, 1), 8.0, device="cuda", dtype=BF16))
    return U, A, W


@pytest.mark.parametrize("graph", [False, True])
def test_rounds_of_a_batch_with_trees_cache_and_verification(graph):
    """Rounds as a program would run them: trees, pages, per layer append and attention over the trees' own masks, verification,
    commit.  One request ends and another starts in its place.  With `graph` a round is captured once and replayed, on
    a stream of its own."""
    import dataclasses
    wl = dataclasses.replace(synth.WORKLOADS["serve32"], V=4096, D=5, K=4, Nmax=20, r=16)
    B, layers, Hq, Hkv, Dh, ps = 6, 2, 8, 2, 64, 16
    ts = TreeSpark(wl.V, wl.D, wl.r, wl.K, wl.Nmax, B)
    R = wl.Nmax + 1
    lay = CacheLayout(Hq, Hkv, Dh, ps, 6 * 6, 8)
    cache = ts.alloc_cache(lay, layers, B)
    ws = ts.attention_workspace(lay, B)
    tree, verdict = ts.alloc_tree(B), ts.alloc_verdict(B)
    U, A, W = round_inputs(wl, B, 1)
    anchor, theta = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), 0.02, device="cuda")
    Z = torch.zeros(B * R, wl.V, dtype=BF16, device="cuda")
    zoff = torch.arange(B + 1, dtype=torch.int64, device="cuda") * R
    kv = torch.zeros(layers, 2, B, R, Hkv, Dh, dtype=BF16, device="cuda")
    q = torch.zeros(layers, B, R, Hq, Dh, dtype=BF16, device="cuda")
    out = torch.zeros_like(q)
    slots = torch.empty(B, R, dtype=torch.int32, device="cuda")
    res = dict(held=cache["held"], free_count=cache["free_count"], slot_map=slots, status=torch.empty(B, dtype=torch.int32, device="cuda"))
    shadow = np.zeros(cache["pool"].shape, np.uint8)
    seq_before = torch.empty_like(cache["seq_len"])

    def one_round():
        ts.expand_tree(U, A, W, anchor, theta, 1.0, 17, out=tree)
        seq_before.copy_(cache["seq_len"])
        ts.cache_reserve(lay, cache["seq_len"], cache["held"], cache["free_pages"], cache["free_count"], cache["block_table"], n_nodes=tree["n_nodes"], out=res)
        for l in range(layers):
            ts.cache_append(lay, kv[l, 0], kv[l, 1], slots, cache["pool"][l])
            ts.tree_attention(lay, q[l], cache["pool"][l], cache["block_table"], cache["seq_len"], n_nodes=tree["n_nodes"], mask=tree["mask"], out=out[l], ws=ws)
        ts.verify_tree(U, A, W, Z, zoff, anchor, tree, 1.0, 17, out=verdict)
        ts.cache_commit(lay, cache["pool"], cache["block_table"], cache["seq_len"], verdict["acc_len"], verdict["acc_node"])

    g = torch.Generator(device="cuda").manual_seed(9)
    stream = torch.cuda.Stream()
    replay = None
    grew = 0
    for rnd in range(5):
        with torch.cuda.stream(stream):
            anchor.copy_(torch.randint(0, wl.V, (B,), generator=g, device="cuda", dtype=torch.int32))
            for t in (kv, q, Z):
                t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
            # the target agrees with the drafter: paths of some length are accepted
            Z.view(B, R, wl.V)[:, :, :] += 2 * U.mean(1, keepdim=True)
            if rnd == 3:   # request 1 ends and starts anew
                ts.cache_reserve(lay, torch.where(torch.arange(B, device="cuda") == 1, -1, cache["seq_len"]).to(torch.int32), cache["held"], cache["free_pages"],
                                 cache["free_count"], cache["block_table"])
                cache["seq_len"][1] = 0
            if graph and replay is None:
                keep = {k: v.clone() for k, v in cache.items()}
                one_round()                                   # (what a first call looks up is looked up)
                torch.cuda.current_stream().synchronize()
                replay = torch.cuda.CUDAGraph()
                with torch.cuda.graph(replay, stream=stream):
                    one_round()
                for k, v in cache.items():
                    v.copy_(keep[k])
            replay.replay() if graph else one_round()
        stream.synchronize()
        assert res["status"].tolist() == [0] * B
        n, seq, table = tree["n_nodes"].tolist(), seq_before.tolist(), cache["block_table"].cpu().numpy()
        assert max(n) > 2
        mask = tree["mask"].cpu().numpy().view(np.uint64)
        for l in range(layers):
            oc.append(shadow[l], ps, slots.flatten().tolist(), kv[l, 0].flatten(0, 1).double().cpu().numpy(), kv[l, 1].flatten(0, 1).double().cpu().numpy())
            for b in range(B):
                want, _ = oc.attention(shadow[l], ps, table[b], seq[b], n[b] + 1, q[l, b].double().cpu().numpy(), mask[b], Dh ** -0.5)
                assert np.abs(out[l, b, :n[b] + 1].double().cpu().numpy() - want).max() <= 2.0 ** -8 * np.abs(want).max() + 2.0 ** -10 * 4
        al, an = verdict["acc_len"].tolist(), verdict["acc_node"].tolist()
        new = [oc.commit(shadow, ps, table[b], seq[b], al[b], an[b], wl.Nmax) for b in range(B)]
        assert cache["seq_len"].tolist() == new
        held_pages = [int(p) for b in range(B) for p in table[b] if p >= 0]
        assert len(set(held_pages)) == len(held_pages) == int(cache["held"].sum()) and len(held_pages) + int(cache["free_count"]) == lay.n_pages
        got = cache["pool"].cpu().numpy()
        for b in range(B):
            for p in range(new[b]):
                at = np.concatenate(oc.token_bytes(Dh, p % 16))
                assert np.array_equal(got[:, table[b, p // ps], :, p % ps // 16][..., at], shadow[:, table[b, p // ps], :, p % ps // 16][..., at])
        grew += sum(al)
    assert grew > 0


def test_calls_on_two_streams_with_workspaces_of_their_own():
    ts = context(Nmax=7, B=16)
    lay = CacheLayout(8, 2, 128, 16, 2000, 130)
    pool = random_pool(1, lay.pool_shape())
    table = torch.randint(0, 2000, (16, 130), device="cuda", dtype=torch.int32)
    qs = [torch.randn(16, 8, 8, 128, device="cuda").to(BF16) for _ in range(2)]
    lens = [torch.randint(0, 2000, (16,), device="cuda", dtype=torch.int32) for _ in range(2)]
    n = torch.full((16,), 7, dtype=torch.int32, device="cuda")
    want = [ts.tree_attention(lay, qs[i], pool, table, lens[i], n_nodes=n) for i in range(2)]
    ws = [ts.attention_workspace(lay, 16) for _ in range(2)]
    outs = [torch.zeros_like(qs[0]) for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                ts.tree_attention(lay, qs[i], pool, table, lens[i], n_nodes=n, out=outs[i], ws=ws[i])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


@pytest.mark.parametrize("dtype,N,Hq", [(BF16, 2, 2), (F32, 7, 4), (BF16, 21, 4)])
def test_a_wait_that_runs_out_gives_nan_and_returns(dtype, N, Hq):
    """Copies that the tensor-core kernel waits for and that never count as arrived: it gives up after a few thousand polls and its rows
    are NaN (units of one CTA and cut ones); the context is usable afterwards, and shortened waits alone change nothing.  The
    kernels for few rows have no such waits."""
    ts = context(Nmax=N, B=4, dtype=dtype)
    lay = CacheLayout(Hq, 2, 128, 16, 300, 200, dtype)
    pool = random_pool(2, lay.pool_shape())
    table = i32(np.random.default_rng(0).permutation(300)[:200][None].repeat(2, 0))
    q = torch.randn(2, N + 1, Hq, 128, device="cuda").to(dtype)
    args, n = (lay, q, pool, table, i32([2500, 40])), i32([N, 0])
    good = ts.tree_attention(*args, n_nodes=n)
    ts.set_test_mode(binding.TEST_SHORT_WAITS | binding.TEST_LOST_ARRIVAL)
    lse = torch.zeros(2, N + 1, Hq, device="cuda")
    lost = ts.tree_attention(*args, n_nodes=n, lse=lse)
    if dtype == BF16 and (N + 1) * Hq // 2 > 16:
        assert torch.isnan(lost[0]).all() and torch.isnan(lost[1, 0]).all() and not lost[1, 1:].any()
        assert torch.isnan(lse[0]).all() and torch.isnan(lse[1, 0]).all()
    else:
        assert torch.equal(lost, good)
    ts.set_test_mode(binding.TEST_SHORT_WAITS)
    assert torch.equal(ts.tree_attention(*args, n_nodes=n), good)
    ts.set_test_mode(0)
    assert torch.equal(ts.tree_attention(*args, n_nodes=n), good)


def test_refusals_of_the_binding():
    ts, lay = context(Nmax=4, B=4), CacheLayout(4, 2, 64, 16, 8, 4)
    pool = torch.zeros(lay.pool_shape(), dtype=torch.uint8, device="cuda")
    k = torch.zeros(2, 2, 64, dtype=BF16, device="cuda")
    sl, seq, table = i32([0, 1]), i32([0, 0]), i32([[0] * 4] * 2)
    q = torch.zeros(2, 4, 64, dtype=BF16, device="cuda")
    for call in (lambda: ts.cache_append(lay, k.float(), k, sl, pool), lambda: ts.cache_append(lay, k, k[:1], sl, pool), lambda: ts.cache_append(lay, k, k, sl.long(), pool),
                 lambda: ts.cache_append(lay, k, k, sl, pool[:4]), lambda: ts.cache_append(lay, k, k, sl, pool, k_val=k[:1]), lambda: ts.cache_append(lay, k.transpose(0, 1), k, sl, pool),
                 lambda: ts.cache_append(lay, k.cpu(), k, sl, pool), lambda: ts.tree_attention(lay, q, pool, table, seq, n_nodes=seq), lambda: ts.tree_attention(lay, q, pool, table[:, :2], seq),
                 lambda: ts.tree_attention(lay, q, pool, table, seq, scale=float("nan")), lambda: ts.tree_attention(lay, q, pool, table, seq, ws=pool.flatten()[:64]),
                 lambda: ts.tree_attention(lay, q, pool, table, seq, lse=torch.zeros(3, device="cuda")),
                 lambda: ts.tree_attention(lay, q, pool, table, seq, mask=torch.zeros(2, 4, 1, dtype=torch.int64, device="cuda")),
                 lambda: ts.cache_commit(lay, pool, table, seq, seq, i32([[0] * 3] * 2)), lambda: ts.cache_reserve(lay, seq, i32([0]), i32(range(8)), i32([8]), table),
                 lambda: ts.cache_append(CacheLayout(4, 2, 96, 16, 8, 4), k, k, sl, pool), lambda: CacheLayout(4, 2, 64, 16, 8, 4, torch.float16)):
        with pytest.raises(TreeSparkError):
            call()
