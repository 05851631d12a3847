"""GPU tests of the attention over the 4-bit cache that see single tokens: rows whose weight lies on one token, placed at the borders of
steps, pages and the pieces that the work is cut into; pages missing inside long contexts; the forms that the other files
reach with few rows only.

Tolerance, per row and channel, with A = sum p |v| in 64 bits (not max |v|), S = scale * max_j sum_d |q_d k_jd| of the row:
  scores: e = S * (2^-22 + 16 * 2^-23) (queries exact or in two parts, sixteen accumulations of Dh products at most), in the
    numerator and in the sum: 2 e;
  weights: exp2 to 2^-21, its argument (below 32 in magnitude wherever a weight counts) to 2^-24 of itself: 2^-19, and half a step of
    fp16, 2^-11 (fp32: two parts, 2^-22); where a weight is among fp16's subnormals, below 2^-14 with the row's largest at
    2^7 or more, it is off by 2^-25 at most: 2^-32 of the sum for each token (fp32: the largest at 2^15, two parts: 2^-40);
  accumulation: each product of sixteen tokens off by 2^-23 of what is summed, along the tokens of one piece; pieces, and changes of
    reference (one for every eight powers of two, counted as 32), by 2^-24 each;
  the result's type: half a step of the result.
lse: e + 2^-19 + 2^-24 for each fp32 addition of a thread, one for every four tokens of a piece at most, of pieces, and 96
  more within a CTA + a step of fp32 of its own value."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2609_22098_b200.binding import CacheLayout
from test_gpu_cache import BF16, F32, check_attention, context, decode64, i32, random_pool, random_table, tree_masks

pytestmark = pytest.mark.gpu


def line(dtype, Dh, G, Hkv, lens, rows, R):
    """How a call's work is cut: steps of TOK tokens behind a lead for each unit, equal pieces.  Returns the pieces' borders as
    (request, head, token), the longest piece in tokens and how many pieces there are."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    if dtype == BF16 and R * G > 16:
        QT, TOK, lead, grid, least = 256, 128, 4, sms, 1
    else:
        two = R * G > 8 and not (dtype == F32 and Dh == 128)
        QT, TOK, lead, grid, least = 16 if two else 8, 48, 8, sms * (2 if two or dtype == F32 else 3), 4
    units = [(b, h, -(-(lens[b] + rows[b]) // TOK)) for b in range(len(lens)) if lens[b] >= 0 for h in range(Hkv) for _ in range(-(-rows[b] * G // QT))]
    begins = np.cumsum([0] + [n + lead for _, _, n in units])
    total = int(begins[-1])
    active = min(grid, max(1, total // least))
    borders = []
    for c in range(1, active):
        x = total * c // active
        u = int(np.searchsorted(begins, x, side="right")) - 1
        borders.append((units[u][0], units[u][1], max(0, x - int(begins[u]) - lead) * TOK))
    return borders, (-(-total // active)) * TOK, active


def dense(pool, table_row, ps, seq, rows, q, see, scale):
    """out, lse, A, S and the weights of rows q [rows][Hq][Dh] in float64; see [rows][rows] of the round's own rows."""
    Hkv, Dh, dev = pool.shape[1], q.shape[-1], q.device
    pos = torch.arange(min(seq + rows, len(table_row) * ps), device=dev)
    page = table_row[pos // ps].long()
    pos = pos[(page >= 0) & (page < pool.shape[0])]
    Hq = q.shape[1]
    if pos.numel() == 0:
        z = torch.zeros(rows, Hq, Dh, dtype=torch.float64, device=dev)
        return z, torch.full((rows, Hq), -float("inf"), dtype=torch.float64, device=dev), z, z[..., 0], None, pos
    K, V = decode64(pool, table_row[pos // ps].long() * ps + pos % ps, Dh)
    vis = torch.ones(rows, pos.numel(), dtype=torch.bool, device=dev)
    own = pos >= seq
    vis[:, own] = see.to(dev)[:, (pos[own] - seq)]
    qd = q.double().unflatten(1, (Hkv, Hq // Hkv))
    x = (scale * torch.einsum("rhgd,thd->rhgt", qd, K)).masked_fill(~vis[:, None, None], -float("inf"))
    z = torch.logsumexp(x, -1)
    p = torch.exp(x - z[..., None]).masked_fill(~vis[:, None, None], 0.0)   # (a row that sees nothing: 0)
    S = scale * torch.einsum("rhgd,hd->rhg", qd.abs(), K.abs().amax(0))
    out, A = torch.einsum("rhgt,thd->rhgd", p, V), torch.einsum("rhgt,thd->rhgd", p, V.abs())
    return out.flatten(1, 2), z.flatten(1), A.flatten(1, 2), S.flatten(1), p.flatten(1, 2), pos


def close(dtype, out, lse, ref, tokens, piece, pieces, vmax):
    want, z, A, S = ref[:4]
    e = (S * (2.0 ** -22 + 16 * 2.0 ** -23))[..., None]
    w = 2 * e + 2.0 ** -21 + 2.0 ** -19 + (2.0 ** -11 if dtype == BF16 else 2.0 ** -22)
    small = tokens * (2.0 ** -32 if dtype == BF16 else 2.0 ** -40) * vmax
    acc = piece / 16 * 2.0 ** -23 + (pieces + 32) * 2.0 ** -24
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    over = (out.double() - want).abs() - ((w + acc) * A + small + half * want.abs())
    assert float(over.max()) <= 0, float(over.max())
    none = torch.isneginf(z)
    assert torch.equal(torch.isneginf(lse), none) and not out[none].any()
    off = (lse.double() - z).abs() - (e[..., 0] + 2.0 ** -19 + (piece / 4 + pieces + 96) * 2.0 ** -24 + 2.0 ** -23 * z.abs())
    assert none.all() or float(off[~none].max()) <= 0, float(off[~none].max())


def chain(rows):
    return torch.ones(rows, rows, dtype=torch.bool).tril()


@pytest.mark.parametrize("dtype,Hq,Hkv,Dh,ps,lens,N", [
    (BF16, 8, 2, 128, 16, [70001], None), (BF16, 16, 1, 64, 64, [33007, 900], None), (BF16, 2, 1, 128, 128, [9000], 7), (F32, 8, 2, 128, 32, [40001], None), (F32, 8, 1, 64, 16, [33000, 5000], 1),
    (BF16, 40, 1, 128, 16, [70001], None), (BF16, 24, 1, 64, 64, [33007, 5000, 1], 4), (BF16, 32, 1, 128, 128, [40003], 7), (BF16, 64, 2, 64, 16, [9000, 20001], 7)])
def test_rows_that_look_for_one_token(dtype, Hq, Hkv, Dh, ps, lens, N):
    """Queries along one token's key, with a score of sixty, which no other comes near (keys of equal scales): the result is that token's value.  The tokens are those to
    both sides of each border between pieces, of some pages, the first and the last, and others at random."""
    rng = np.random.default_rng(sum(lens))
    B, R, G = len(lens), 1 if N is None else N + 1, Hq // Hkv
    ts = context(Nmax=N or 1, B=B, dtype=dtype)
    rows = [R] * B
    total = [n + R for n in lens]
    cols, pages = max(-(-n // ps) for n in total) + 1, sum(-(-n // ps) for n in total) + 2
    lay = CacheLayout(Hq, Hkv, Dh, ps, pages, cols, dtype)
    table = random_table(rng, total, ps, cols, pages)
    pool, gt = random_pool(7, lay.pool_shape()), i32(table)
    pool[..., 16 * Dh:17 * Dh] = 40
    borders, piece, pieces = line(dtype, Dh, G, Hkv, lens, rows, R)
    look = {(b, h): [0, lens[b]] + [p * ps + d for p in rng.integers(1, max(2, lens[b] // ps), 4) for d in (-1, 0)] for b in range(B) for h in range(Hkv)}
    for b, h, t in borders:
        look[b, h] += [t - 1, t, t + 1]
    look = {k: [int(t) for t in v if 0 <= t <= lens[k[0]]] for k, v in look.items()}   # (the anchor's own row is the last that all rows see)
    calls = max(-(-len(v) // (R * G)) for v in look.values())
    keys = [decode64(pool, gt[b].long()[(pos := torch.arange(total[b], device="cuda")) // ps] * ps + pos % ps, Dh) for b in range(B)]
    ws = ts.attention_workspace(lay, B)
    scale = Dh ** -0.5
    for call in range(calls):
        q = torch.zeros(B, R, Hq, Dh, dtype=dtype, device="cuda")
        at = torch.zeros(B, R, Hq, dtype=torch.long)
        for b in range(B):
            for h in range(Hkv):
                mine = look[b, h][call * R * G:(call + 1) * R * G]
                mine = np.array(mine + list(rng.integers(0, lens[b] + 1, R * G - len(mine)))).reshape(R, G)
                k = keys[b][0][torch.from_numpy(mine).cuda(), h]
                q[b, :, h * G:(h + 1) * G] = (k * (60 / scale / (k * k).sum(-1, keepdim=True))).to(dtype)
                at[b, :, h * G:(h + 1) * G] = torch.from_numpy(mine)
        out, lse = torch.zeros_like(q), torch.zeros(B, R, Hq, device="cuda")
        ts.tree_attention(lay, q, pool, gt, i32(lens), n_nodes=None if N is None else i32([N] * B), out=out, lse=lse, ws=ws)
        for b in range(B):
            ref = dense(pool, gt[b], ps, lens[b], R, q[b], chain(R), scale)
            if lens[b] > 100:   # (what the test is for)
                assert float(torch.gather(ref[4], 2, at[b].cuda()[..., None]).min()) > 0.9
            close(dtype, out[b], lse[b], ref, total[b], piece, pieces, float(keys[b][1].abs().max()))


@pytest.mark.parametrize("dtype,Hq,Hkv,Dh,ps,lens,N,n_nodes,mode", [
    (BF16, 4, 1, 128, 16, [70001], 7, None, None), (F32, 2, 1, 128, 32, [40000], 7, [5], "tree"), (BF16, 32, 8, 128, 16, [4000, 17, 901, 2500], 64, [64, 30, 7, 12], "tree"),
    (BF16, 64, 2, 128, 16, [9000, 2000], 256, [256, 100], "tree"), (F32, 8, 2, 64, 64, [33000, 5], 7, [7, 3], "tree"),
    (BF16, 1, 1, 64, 16, [700, 0, 300], 256, [256, 255, 130], "chain"), (BF16, 8, 2, 128, 32, [1000, 90], 256, [256, 200], "chain"), (BF16, 6, 2, 64, 16, [3000], 128, [128], "chain"),
    (F32, 4, 1, 64, 16, [500, 0], 256, [256, 256], "chain")])
def test_long_contexts_to_their_own_tolerance(dtype, Hq, Hkv, Dh, ps, lens, N, n_nodes, mode):
    """Spread weights over long contexts, trees, and chains (chunks of prompts) of up to 257 rows over several steps and words."""
    rng = np.random.default_rng(len(lens))
    B = len(lens)
    ts = context(Nmax=N, B=B, dtype=dtype)
    R, rows = 1 if n_nodes is None else N + 1, [1 + (n_nodes[b] if n_nodes else 0) for b in range(B)]
    total = [n + r for n, r in zip(lens, rows)]
    cols, pages = max(-(-n // ps) for n in total) + 1, sum(-(-n // ps) for n in total) + 2
    lay = CacheLayout(Hq, Hkv, Dh, ps, pages, cols, dtype)
    table, pool = i32(random_table(rng, total, ps, cols, pages)), random_pool(11, lay.pool_shape())
    q = torch.randn(B, R, Hq, Dh, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).to(dtype)
    mask = tree_masks(rng, B, N, [r - 1 for r in rows]) if mode == "tree" else None
    out, lse = torch.zeros_like(q), torch.zeros(B, R, Hq, device="cuda")
    ts.tree_attention(lay, q, pool, table, i32(lens), n_nodes=None if n_nodes is None else i32(n_nodes), mask=None if mask is None else torch.from_numpy(mask.view(np.int64)).cuda(), out=out, lse=lse)
    _, piece, pieces = line(dtype, Dh, Hq // Hkv, Hkv, lens, rows, R)
    for b in range(B):
        see = chain(rows[b]) if mask is None else torch.tensor([[oc.sees(mask[b], i, t) for t in range(rows[b])] for i in range(rows[b])])
        ref = dense(pool, table[b], ps, lens[b], rows[b], q[b, :rows[b]], see, Dh ** -0.5)
        close(dtype, out[b, :rows[b]], lse[b, :rows[b]], ref, total[b], piece, pieces, 14.0)   # (|v| <= 8 * 1.75)


@pytest.mark.parametrize("dtype,Hq,Hkv,Dh,ps,N,n", [
    (BF16, 6, 2, 128, 16, 1, 1), (F32, 4, 2, 64, 16, 5, 4), (BF16, 4, 1, 128, 16, 21, 20), (BF16, 8, 2, 64, 48, 30, 17), (BF16, 8, 1, 64, 16, 30, 30), (BF16, 16, 2, 128, 64, 20, 20), (BF16, 20, 1, 128, 16, 20, 20)])
@pytest.mark.parametrize("mode", ["tree", "chain"])
def test_pages_missing_inside_contexts(dtype, Hq, Hkv, Dh, ps, N, n, mode):
    """Tables with holes: single pages, whole runs over several steps, all of a prefix, all of a request, a table shorter than the context;
    on both kernels, one and two tiles, contexts of one step and cut ones."""
    rng = np.random.default_rng(N)
    lens = [20000, 9001, 400, 2500, 30, 50, 3000]
    B, ts = len(lens), None
    ts = context(Nmax=N, B=B, dtype=dtype)
    total = [x + n + 1 for x in lens]
    cols, pages = max(-(-x // ps) for x in total), sum(-(-x // ps) for x in total) + 2
    table = random_table(rng, total, ps, cols, pages)
    cut = 2000 // ps
    lay = CacheLayout(Hq, Hkv, Dh, ps, pages, cols, dtype)
    table[0][rng.random(cols) < 0.3] = -1
    table[0, 5000 // ps:9000 // ps] = pages            # no block for many steps
    table[1, :lens[1] // ps] = -3                      # only the rows of the round, the first of them perhaps not
    table[2, ::2] = 1 << 30
    table[3, :] = -1                                   # nothing at all
    table[4, 0] = -1
    table[5, 50 // ps:] = -1                           # rows of the round only partly there
    table[6, cut:] = -1
    pool = random_pool(13, lay.pool_shape())
    q = torch.randn(B, N + 1, Hq, Dh, device="cuda", generator=torch.Generator(device="cuda").manual_seed(6)).to(dtype)
    mask = tree_masks(rng, B, N, [n] * B) if mode == "tree" else None
    out, lse = torch.full_like(q, -3.0), torch.full((B, N + 1, Hq), -5.0, device="cuda")
    gt = i32(table)
    ts.tree_attention(lay, q, pool, gt, i32(lens), n_nodes=i32([n] * B), mask=None if mask is None else torch.from_numpy(mask.view(np.int64)).cuda(), out=out, lse=lse)
    assert (out[:, n + 1:] == -3.0).all() and (lse[:, n + 1:] == -5.0).all()
    assert not out[3, :n + 1].any() and torch.isneginf(lse[3, :n + 1]).all()
    _, piece, pieces = line(dtype, Dh, Hq // Hkv, Hkv, lens, [n + 1] * B, N + 1)
    for b in range(B):
        see = chain(n + 1) if mask is None else torch.tensor([[oc.sees(mask[b], i, t) for t in range(n + 1)] for i in range(n + 1)])
        ref = dense(pool, gt[b], ps, lens[b], n + 1, q[b, :n + 1], see, Dh ** -0.5)
        close(dtype, out[b, :n + 1], lse[b, :n + 1], ref, total[b], piece, pieces, 14.0)
    # a table with fewer columns than the contexts have pages
    short = CacheLayout(Hq, Hkv, Dh, ps, pages, cut, dtype)
    o2, l2, t2 = torch.full_like(q, -3.0), torch.full_like(lse, -5.0), gt[:, :cut].contiguous()
    ts.tree_attention(short, q, pool, t2, i32(lens), n_nodes=i32([n] * B), mask=None if mask is None else torch.from_numpy(mask.view(np.int64)).cuda(), out=o2, lse=l2)
    for b in range(B):
        see = chain(n + 1) if mask is None else torch.tensor([[oc.sees(mask[b], i, t) for t in range(n + 1)] for i in range(n + 1)])
        ref = dense(pool, t2[b], ps, lens[b], n + 1, q[b, :n + 1], see, Dh ** -0.5)
        close(dtype, o2[b, :n + 1], l2[b, :n + 1], ref, total[b], piece, pieces, 14.0)


@pytest.mark.parametrize("dtype,Hq,Hkv,N,B", [(BF16, 2, 2, None, 4096), (BF16, 20, 1, None, 3001), (BF16, 6, 1, 3, 1500), (F32, 6, 3, 2, 2050)])
def test_thousands_of_requests(dtype, Hq, Hkv, N, B):
    """More requests than a CTA has threads, a third of them idle (and whole runs of them), contexts of no token to a few steps; all of
    them idle in the end."""
    rng = np.random.default_rng(B)
    R, Dh, ps = 1 if N is None else N + 1, 64, 16
    ts = context(Nmax=N or 1, B=B, dtype=dtype)
    lens = rng.integers(0, 300, B) * (rng.random(B) < 0.5)
    lens[rng.random(B) < 0.3] = -1
    lens[B // 3:B // 2] = -1
    lens[-1], lens[0] = 290, -1
    total = [max(0, x + R) if x >= 0 else 0 for x in lens]
    cols, pages = 1 + max(-(-x // ps) for x in total), sum(-(-x // ps) for x in total) + 2
    lay = CacheLayout(Hq, Hkv, Dh, ps, pages, cols, dtype)
    table, pool = i32(random_table(rng, total, ps, cols, pages)), random_pool(17, lay.pool_shape())
    q = torch.randn(B, R, Hq, Dh, device="cuda", generator=torch.Generator(device="cuda").manual_seed(8)).to(dtype)
    out, lse = torch.full_like(q, -3.0), torch.full((B, R, Hq), -5.0, device="cuda")
    args = dict(n_nodes=None if N is None else i32([N] * B), out=out, lse=lse)
    ts.tree_attention(lay, q, pool, table, i32(lens), **args)
    idle = torch.from_numpy(lens < 0).cuda()
    assert (out[idle] == -3.0).all() and (lse[idle] == -5.0).all()
    _, piece, pieces = line(dtype, Dh, Hq // Hkv, Hkv, [int(x) for x in lens], [R] * B, R)
    for b in [b for b in list(range(0, B, B // 50)) + [B - 1] if lens[b] >= 0]:
        ref = dense(pool, table[b], ps, int(lens[b]), R, q[b], chain(R), Dh ** -0.5)
        close(dtype, out[b], lse[b], ref, total[b], piece, pieces, 14.0)
    before = out.clone()
    ts.tree_attention(lay, q, pool, table, i32([-1] * B), **args)
    assert torch.equal(out, before)


@pytest.mark.parametrize("Hq,Dh,N", [(4, 128, 20), (32, 64, 5), (12, 128, 20)])
def test_queries_that_are_not_finite_on_the_tensor_cores(Hq, Dh, N):
    """One tile and two, a context cut into pieces and one of a step: the rows of the bad queries are NaN, the others what they were."""
    ts = context(Nmax=N, B=2)
    lay = CacheLayout(Hq, 1, Dh, 16, 400, 350)
    pool = random_pool(3, lay.pool_shape())
    table = i32(np.random.default_rng(1).permutation(400)[:350][None].repeat(2, 0))
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(2, N + 1, Hq, Dh, device="cuda", generator=g).to(BF16)
    args = dict(n_nodes=i32([N, N]))
    good = ts.tree_attention(lay, q, pool, table, i32([5000, 20]), **args)
    bad, hit = q.clone(), torch.zeros(2, N + 1, Hq, dtype=torch.bool, device="cuda")
    for b, i, h, d, x in ((0, 0, 0, 3, float("inf")), (0, N, Hq - 1, Dh - 1, float("nan")), (1, 2, 1, 0, -float("inf")), (1, N // 2, 2, 40, float("nan"))):
        bad[b, i, h, d] = x
        hit[b, i, h] = True
    lse = torch.zeros(2, N + 1, Hq, device="cuda")
    got = ts.tree_attention(lay, bad, pool, table, i32([5000, 20]), lse=lse, **args)
    assert torch.isfinite(good).all() and torch.equal(got[~hit], good[~hit])
    assert torch.isnan(got[hit]).all() and torch.isnan(lse[hit]).all() and torch.isfinite(lse[~hit]).all()


def test_nan_in_the_cache_with_few_rows():
    """The bf16 kernel for up to 16 rows a kv head (one tile of eight and two): trees, chains, single tokens."""
    ts = context(Nmax=6)
    check_attention(ts, BF16, 2, 2, 128, 16, [20, 30], [6, 3], "tree", 15, poison=[2, 5])
    check_attention(ts, BF16, 4, 2, 64, 32, [0, 90], [6, 4], "chain", 16, poison=[3])
    check_attention(ts, BF16, 4, 2, 64, 32, [9, 30], [6, 2], "tree", 17, poison=[0])
    check_attention(ts, BF16, 8, 1, 128, 16, [33, 200], None, "one", 18, poison=[0])
