"""GPU tests of the 4-bit cache calls where they meet: requests that are refused pages and served later, against the cache's oracle
(oracle/cache.py)."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2609_22098_b200 import binding, synth
from paper_2609_22098_b200.binding import CacheLayout, TreeSpark
from test_gpu_cache import BF16, F32, check_reserve, context, i32, random_pool, random_table, round_inputs

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ reserve
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,cols,pages,seed", [(1, 4, 8, 0), (6, 70, 300, 1), (64, 300, 9000, 2), (3, 30000, 50000, 3), (300, 90, 20000, 4), (4096, 5, 9000, 5)])
def test_pages_given_back_are_pages(B, cols, pages, seed, in_place):
    """Tables with entries that are no pages (negative, the pool's end, far beyond) at any place: released, they are dropped, and the
    list holds each page once.  One cluster and many CTAs."""
    rng = np.random.default_rng(seed)
    ts, lay = context(4, B), CacheLayout(4, 2, 64, 16, pages, cols)
    held = rng.integers(0, cols + 1, B)
    held = np.minimum(held, pages // B)
    order, at = rng.permutation(pages), 0
    table = np.full((B, cols), -1, np.int64)
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    free, count = np.zeros(pages, np.int64), pages - at
    free[:count] = order[at:]
    own = np.arange(cols)[None] < held[:, None]
    junk = own & (rng.random((B, cols)) < 0.2)
    junk[0, :held[0]] |= seed == 0      # one request without a single page
    table[junk] = rng.choice([-1, -7, pages, pages + 1, 1 << 30], int(junk.sum()))
    seq = np.where(rng.random(B) < 0.6, -1, rng.integers(0, 16 * cols - 8, B))
    seq[0] = -1
    w = check_reserve(ts, lay, seq, rng.integers(0, 5, B), held.tolist(), free, count, table, in_place)
    left = [int(p) for p in w[2][:w[3]]]
    assert len(set(left)) == len(left) and all(0 <= p < pages for p in left)
    check_reserve(ts, lay, [0] * B, None, w[1], w[2], w[3], w[0], in_place)
    all_back = check_reserve(ts, lay, [-1] * B, None, w[1], w[2], w[3], w[0], in_place)
    assert all_back[3] == pages - int(junk.sum())


@pytest.mark.parametrize("B", [6, 80])
def test_a_request_beyond_the_table_is_refused_alone(B):
    """On the one-cluster form and on many CTAs, by the six requests of the oracle's own test (idle ones behind them)."""
    ts, lay = context(20, B), CacheLayout(4, 2, 64, 16, 10, 3)
    table = np.full((B, 3), -1, np.int64)
    table[5, 0] = 9
    idle = B - 6
    w = check_reserve(ts, lay, [3, 40, 20, 30, 0, 3] + [-1] * idle, [3, 8, 3, 17, 1, 3] + [0] * idle, [0, 0, 0, 0, 0, 1] + [0] * idle, [0, 1, 2, 3, 4, 0, 0, 0, 0, 0], 5, table, True)
    assert w[5][:6] == [0, -6, 0, -6, -6, 0] and w[1][:6] == [1, 0, 2, 0, 0, 1]


@pytest.mark.parametrize("shape", [(0,), (4, 0), (0, 5)])
def test_append_of_no_rows(shape):
    ts, lay = context(), CacheLayout(2, 2, 64, 16, 3, 3)
    pool = torch.full(lay.pool_shape(), 77, dtype=torch.uint8, device="cuda")
    k = torch.zeros(*shape, 2, 64, dtype=BF16, device="cuda")
    ts.cache_append(lay, k, k, torch.zeros(shape, dtype=torch.int32, device="cuda"), pool, k_val=torch.empty_like(k))
    assert (pool == 77).all()


# ------------------------------------------------------------------------------------------------ attention
@pytest.mark.parametrize("dtype,Hq,Dh", [(BF16, 1, 64), (BF16, 16, 128), (BF16, 32, 64), (BF16, 40, 128), (F32, 3, 64), (F32, 2, 128)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_queries_with_infinities_give_nan_whatever_their_scores(dtype, Hq, Dh, sign):
    """One or more visible tokens whose keys have one sign: a query of zeros and one infinity scores +inf or -inf on all of them,
    and with both the softmax has no value.  A row that sees nothing stays 0."""
    ts, lay = context(dtype=dtype, Nmax=4), CacheLayout(Hq, 1, Dh, 16, 40, 33, dtype)
    pool = torch.zeros(lay.pool_shape(), dtype=torch.uint8, device="cuda")
    k = torch.ones(33 * 16, 1, Dh, dtype=dtype, device="cuda")
    ts.cache_append(lay, k, k, i32(range(33 * 16)), pool)
    q = torch.zeros(3, Hq, Dh, dtype=dtype, device="cuda")
    q[:, ::2, 5] = sign * float("inf")
    q[:, 1::2] = 1.0
    table = np.stack([np.arange(33), np.arange(33), np.full(33, -1)])
    lse = torch.full((3, Hq), -5.0, device="cuda")
    out = ts.tree_attention(lay, q, pool, i32(table), i32([0, 520, 7]), lse=lse)
    assert torch.isnan(out[:2, ::2]).all() and torch.isnan(lse[:2, ::2]).all()
    assert torch.isfinite(out[:2, 1::2]).all() and torch.isfinite(lse[:2, 1::2]).all()
    assert not out[2].any() and torch.isneginf(lse[2]).all()


@pytest.mark.parametrize("Dh,N,Hq", [(128, 1, 32), (64, 1, 24), (128, 4, 48), (64, 7, 32)])
def test_a_wait_that_runs_out_behind_issued_products(Dh, N, Hq):
    """The tensor-core kernel gives up in the fifth of some ten steps a CTA, with products of the steps before issued: it waits for them
    and for its copies, its rows are NaN, and the same call without lost bytes gives what it gave before."""
    ts = context(Nmax=N, B=1)
    n = 10 * 128 * torch.cuda.get_device_properties(0).multi_processor_count
    pages = n // 64 + 1
    lay = CacheLayout(Hq, 1, Dh, 64, pages, pages)
    pool = random_pool(2, lay.pool_shape())
    table = i32(np.random.default_rng(0).permutation(pages)[None])
    q = torch.randn(1, N + 1, Hq, Dh, device="cuda").to(BF16)
    args, kw = (lay, q, pool, table, i32([n])), dict(n_nodes=i32([N]))
    good = ts.tree_attention(*args, **kw)
    ts.set_test_mode(binding.TEST_SHORT_WAITS | binding.TEST_LOST_ARRIVAL)
    lse = torch.zeros(1, N + 1, Hq, device="cuda")
    lost = ts.tree_attention(*args, **kw, lse=lse)
    assert torch.isnan(lost).all() and torch.isnan(lse).all()
    ts.set_test_mode(0)
    assert torch.isfinite(good).all() and torch.equal(ts.tree_attention(*args, **kw), good)


# ------------------------------------------------------------------------------------------------ commit
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,layers,Hkv,Dh", [(7, 2, 2, 64), (3, 40, 8, 128)])
def test_commit_leaves_refused_requests_as_they_are(B, layers, Hkv, Dh, in_place):
    rng = np.random.default_rng(B)
    ts = context(20, B, 4)
    seq = [int(x) for x in rng.integers(0, 60, B)]
    seq[-1] = -1
    total = [max(0, s) + 21 for s in seq]
    cols, pages = max(-(-n // 16) for n in total), sum(-(-n // 16) for n in total) + 1
    lay = CacheLayout(Hkv, Hkv, Dh, 16, pages, cols)
    table = random_table(rng, total, 16, cols, pages)
    pool = rng.integers(0, 256, (layers, *lay.pool_shape()), dtype=np.uint8)
    status = [-6 if b % 2 else 0 for b in range(B)]
    acc_len = rng.integers(1, 5, B)
    node = np.sort(np.stack([rng.permutation(20)[:4] for _ in range(B)]), 1)
    g, seq_g = torch.from_numpy(pool.copy()).cuda(), i32(seq)
    new = ts.cache_commit(lay, g, i32(table), seq_g, i32(acc_len), i32(node), None if in_place else torch.full((B,), -9, dtype=torch.int32, device="cuda"), status=i32(status))
    want = [seq[b] if status[b] else oc.commit(pool, 16, table[b], seq[b], int(acc_len[b]), node[b], 20) for b in range(B)]
    assert new.tolist() == want and (in_place or seq_g.tolist() == seq)
    assert np.array_equal(g.cpu().numpy(), pool)


@pytest.mark.parametrize("graph", [False, True])
def test_a_request_that_is_refused_pages_is_served_in_a_later_round(graph):
    """Rounds (expand, reserve, append, attention, verify, commit) with a pool that is too small: refused requests keep their length
    though their last page has room, and after other requests have ended they go on as if the rounds between had not been.  What was
    never written is NaN.  (Four requests hold a page each from the first round on; with sixteen tokens each would need two, which are
    two more than there are.)"""
    wl = dataclasses.replace(synth.WORKLOADS["serve32"], V=4096, D=5, K=4, Nmax=20, r=16)
    B, layers, Hq, Hkv, Dh, ps = 4, 2, 4, 2, 64, 16
    ts = TreeSpark(wl.V, wl.D, wl.r, wl.K, wl.Nmax, B)
    R = wl.Nmax + 1
    lay = CacheLayout(Hq, Hkv, Dh, ps, 6, 6)
    cache = ts.alloc_cache(lay, layers, B)
    cache["pool"].fill_(255)
    ws = ts.attention_workspace(lay, B)
    tree, verdict = ts.alloc_tree(B), ts.alloc_verdict(B)
    U, A, W = round_inputs(wl, B, 1)
    anchor, theta = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), 0.02, device="cuda")
    Z = torch.zeros(B * R, wl.V, dtype=BF16, device="cuda")
    zoff = torch.arange(B + 1, dtype=torch.int64, device="cuda") * R
    kv = torch.zeros(layers, 2, B, R, Hkv, Dh, dtype=BF16, device="cuda")
    q = torch.zeros(layers, B, R, Hq, Dh, dtype=BF16, device="cuda")
    out = torch.zeros_like(q)
    res = dict(held=cache["held"], free_count=cache["free_count"], slot_map=torch.empty(B, R, dtype=torch.int32, device="cuda"),
               status=torch.empty(B, dtype=torch.int32, device="cuda"))

    def one_round():
        ts.expand_tree(U, A, W, anchor, theta, 1.0, 17, out=tree)
        ts.cache_reserve(lay, cache["seq_len"], cache["held"], cache["free_pages"], cache["free_count"], cache["block_table"], n_nodes=tree["n_nodes"], out=res)
        for l in range(layers):
            ts.cache_append(lay, kv[l, 0], kv[l, 1], res["slot_map"], cache["pool"][l])
            ts.tree_attention(lay, q[l], cache["pool"][l], cache["block_table"], cache["seq_len"], n_nodes=tree["n_nodes"], mask=tree["mask"], out=out[l], ws=ws)
        ts.verify_tree(U, A, W, Z, zoff, anchor, tree, 1.0, 17, out=verdict)
        ts.cache_commit(lay, cache["pool"], cache["block_table"], cache["seq_len"], verdict["acc_len"], verdict["acc_node"], status=res["status"])

    g = torch.Generator(device="cuda").manual_seed(9)
    stream, replay = torch.cuda.Stream(), None
    # the oracle's own account of the cache
    seq, held, free, count, table = [0] * B, [0] * B, list(range(lay.n_pages - 1, -1, -1)), lay.n_pages, np.full((B, lay.max_pages), -1, np.int64)
    shadow = np.full(cache["pool"].shape, 255, np.uint8)
    refused_before, served_later, with_room = set(), 0, 0
    for rnd in range(24):
        with torch.cuda.stream(stream):
            anchor.copy_(torch.randint(0, wl.V, (B,), generator=g, device="cuda", dtype=torch.int32))
            for t in (kv, q, Z):
                t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
            Z.view(B, R, wl.V)[:, :, :] += 2 * U.mean(1, keepdim=True)
            if rnd in (12, 18):   # request 0, later 1, ends
                ends = 0 if rnd == 12 else 1
                gone = [-1 if b == ends else s for b, s in enumerate(seq)]
                ts.cache_reserve(lay, i32(gone), cache["held"], cache["free_pages"], cache["free_count"], cache["block_table"])
                table, held, free, count, _, _ = oc.reserve(ps, lay.n_pages, gone, [1] * B, held, free, count, table, 1)
                cache["seq_len"][ends] = -1
                seq[ends] = -1
            if graph and replay is None:
                keep = {k: v.clone() for k, v in cache.items()}
                one_round()
                torch.cuda.current_stream().synchronize()
                replay = torch.cuda.CUDAGraph()
                with torch.cuda.graph(replay, stream=stream):
                    one_round()
                for k, v in cache.items():
                    v.copy_(keep[k])
            replay.replay() if graph else one_round()
        stream.synchronize()
        n = tree["n_nodes"].tolist()
        table, held, free, count, slots, status = oc.reserve(ps, lay.n_pages, seq, [x + 1 for x in n], held, free, count, table, R)
        assert res["status"].tolist() == status and np.array_equal(res["slot_map"].cpu().numpy(), slots)
        assert np.array_equal(cache["block_table"].cpu().numpy(), table)
        mask = tree["mask"].cpu().numpy().view(np.uint64)
        al, an = verdict["acc_len"].tolist(), verdict["acc_node"].tolist()
        for l in range(layers):
            oc.append(shadow[l], ps, slots.flatten().tolist(), kv[l, 0].flatten(0, 1).double().cpu().numpy(), kv[l, 1].flatten(0, 1).double().cpu().numpy())
        for b in range(B):
            if seq[b] < 0:
                continue
            if status[b]:
                with_room += held[b] * ps > seq[b]
                refused_before.add(b)
                continue
            served_later += b in refused_before
            for l in range(layers):
                # (bf16 results to half a step; 4: the largest value, 2^-10: twice a weight's rounding)
                want, _ = oc.attention(shadow[l], ps, table[b], seq[b], n[b] + 1, q[l, b].double().cpu().numpy(), mask[b], Dh ** -0.5)
                assert np.isfinite(want).all()
                assert np.abs(out[l, b, :n[b] + 1].double().cpu().numpy() - want).max() <= 2.0 ** -8 * np.abs(want).max() + 2.0 ** -10 * 4, (rnd, b)
            seq[b] = oc.commit(shadow, ps, table[b], seq[b], al[b], an[b], wl.Nmax)
        assert cache["seq_len"].tolist() == seq, rnd
    assert with_room > 0 and served_later > 0, (with_room, served_later, seq, held)
