"""Cases of the cache operators: the page tables of a batch, the cache in 4 bits, the attention of draft trees over it, and the
commit of an accepted path.

A round of a program that keeps its keys and values in such a cache is: ``cache_reserve`` (pages and slots for the rows of this
round), per layer ``cache_append`` and ``tree_attention``, and after the verification ``cache_commit``.

Layout of the cache (one layer): [n_pages][Hkv][page_size / 16][18 * Dh] bytes.  The 18 * Dh bytes of 16 tokens of one head are
K codes [16][Dh / 2], V codes [2][Dh / 16][8][8], K scales [16][Dh / 16], V scales [2][Dh / 16][8].  A code c in 0..15 stands for
(c - 8) * scale * 2 ** exp with one e4m3 scale per 16 elements; eight elements share a 32-bit word, element 2j in nibble j and
element 2j + 1 in nibble j + 4.
"""
import functools
import math

import numpy as np
import torch

own = False

DEV = "cuda"
NO_PAGE = -1
REFUSED = -6          # status of a request for which no pages are left


# ---------------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the tables of one round: 32 running requests, trees of up to 64 nodes, most pages held already
        dict(name="reserve_round", op="reserve", B=32, Nmax=64, n_lo=8, n_hi=64, ps=16, len_lo=300, len_hi=8000, fresh=False),
        # many requests that start at once from stored prefixes: whole tables
        dict(name="reserve_start", op="reserve", B=500, Nmax=16, n_lo=0, n_hi=16, ps=16, len_lo=40, len_hi=30000, fresh=True),
        # one token of each of 32 requests
        dict(name="append_tokens", op="append", B=32, Nmax=0, n_lo=0, n_hi=0, Hkv=8, Dh=128, ps=32, dtype="bf16", values=False),
        # the rows of 32 trees
        dict(name="append_trees", op="append", B=32, Nmax=64, n_lo=8, n_hi=64, Hkv=8, Dh=128, ps=16, dtype="bf16", values=True),
        # prompt chunks in fp32
        dict(name="append_chunks_f32", op="append", B=64, Nmax=256, n_lo=101, n_hi=256, Hkv=4, Dh=64, ps=64, dtype="f32", values=True),
        # a single request, single token, short context: latency
        dict(name="attn_one", op="attn", B=1, Nmax=0, n_lo=0, n_hi=0, Hq=32, Hkv=8, Dh=128, ps=16, len_lo=517, len_hi=517, dtype="bf16", tree=False),
        # single tokens of a batch with ragged lengths
        dict(name="attn_batch", op="attn", B=64, Nmax=0, n_lo=0, n_hi=0, Hq=32, Hkv=8, Dh=128, ps=16, len_lo=1001, len_hi=16000, dtype="bf16", tree=False),
        # chains of eight rows behind two very long contexts, in fp32
        dict(name="attn_long_f32", op="attn", B=2, Nmax=7, n_lo=7, n_hi=7, Hq=8, Hkv=2, Dh=64, ps=64, len_lo=65000, len_hi=131000, dtype="f32", tree=False),
        # the trees of 32 requests (8 to 30 nodes: what a calibrated stop price gives)
        dict(name="attn_trees", op="attn", B=32, Nmax=64, n_lo=8, n_hi=30, Hq=32, Hkv=8, Dh=128, ps=16, len_lo=501, len_hi=6000, dtype="bf16", tree=True),
        # crowded trees behind long contexts
        dict(name="attn_wide", op="attn", B=8, Nmax=256, n_lo=120, n_hi=256, Hq=32, Hkv=4, Dh=128, ps=64, len_lo=2000, len_hi=16001, dtype="bf16", tree=True),
        # accepted paths of one request and of a batch, all layers at once
        dict(name="commit_one", op="commit", B=1, Nmax=64, n_lo=40, n_hi=40, D=8, layers=36, Hkv=8, Dh=128, ps=16, len_lo=77, len_hi=77),
        dict(name="commit_batch", op="commit", B=32, Nmax=64, n_lo=8, n_hi=64, D=8, layers=12, Hkv=8, Dh=128, ps=16, len_lo=30, len_hi=400),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["reserve", "append", "append", "attn", "attn", "attn", "attn", "commit"])
    ps = rng.choice([16, 16, 32, 64, 80, 128])
    Nmax = rng.choice([0, rng.randint(1, 64), rng.randint(1, 256)])
    n_hi = rng.randint(0, Nmax)
    n_lo = rng.randint(0, n_hi)
    if op == "reserve":
        B = _log_int(rng, 1, 500)
        hi = _log_int(rng, 1, 30000)
        return dict(op=op, B=B, Nmax=min(Nmax, 64), n_lo=min(n_lo, 64), n_hi=min(n_hi, 64), ps=ps, len_lo=rng.randint(0, hi), len_hi=hi, fresh=rng.random() < 0.5)
    Hkv, Dh = rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "append":
        return dict(op=op, B=_log_int(rng, 1, 64), Nmax=Nmax, n_lo=n_lo, n_hi=n_hi, Hkv=Hkv, Dh=Dh, ps=ps, dtype=dtype, values=rng.random() < 0.7)
    if op == "commit":
        Nmax = max(Nmax, 4)
        D = rng.randint(1, min(16, Nmax))
        return dict(op=op, B=_log_int(rng, 1, 32), Nmax=Nmax, n_lo=D, n_hi=Nmax, D=D, layers=rng.randint(1, 12), Hkv=Hkv, Dh=Dh, ps=ps, len_lo=0, len_hi=_log_int(rng, 1, 400))
    g = rng.choice([1, 2, 3, 4, 5, 8, 16])
    B = _log_int(rng, 1, 64)
    # the largest listed batch has 131,000 tokens a head and a request of it, 550,000 in all; crowded trees have less
    room = 400000 // (B * (1 + Nmax * g // 64))
    hi = max(1, min(131000, _log_int(rng, 1, max(2, room))))
    if dtype == "f32":
        hi = max(1, min(hi, 4000000 // (B * (1 + n_hi) * g)))
    return dict(op=op, B=B, Nmax=Nmax, n_lo=n_lo, n_hi=n_hi, Hq=Hkv * g, Hkv=Hkv, Dh=Dh, ps=ps, len_lo=rng.randint(0, hi), len_hi=hi, dtype=dtype, tree=rng.random() < 0.6)


def _spread(lo, hi, B):
    """B whole numbers from lo to hi, evenly spread."""
    return [lo + (hi - lo) * i // max(1, B - 1) for i in range(B)] if B > 1 else [hi]


def _lens(case):
    return _spread(case["len_lo"], case["len_hi"], case["B"])


def _rows(case):
    """Rows of each request (the anchor and its nodes), spread the other way round than the lengths are."""
    return [1 + n for n in reversed(_spread(case["n_lo"], case["n_hi"], case["B"]))]


def _es(case):
    return 2 if case["dtype"] == "bf16" else 4


def work(case):
    B, R = case["B"], case["Nmax"] + 1
    if case["op"] == "reserve":
        held = 0 if case["fresh"] else None
        new = 0
        for n, r in zip(_lens(case), _rows(case)):
            have = held if held is not None else -(-n // case["ps"])
            new += max(0, -(-(n + r) // case["ps"]) - have)
        return dict(bytes=8 * new + 4 * B * R + 4 * B * 5, flops=0)
    if case["op"] == "append":
        el = 2 * sum(_rows(case)) * case["Hkv"] * case["Dh"]
        return dict(bytes=el * (_es(case) + 0.5625 + (_es(case) if case["values"] else 0)) + 4 * B * R, flops=4 * el)
    if case["op"] == "commit":
        moved = sum(_paths(case)[0].tolist())
        return dict(bytes=moved * 2 * case["layers"] * case["Hkv"] * case["Dh"] * 1.125 + 4 * B * (3 + case["D"]), flops=0)
    toks = sum(n + r for n, r in zip(_lens(case), _rows(case)))
    pairs = sum((n + 1) * r for n, r in zip(_lens(case), _rows(case)))
    q = sum(_rows(case)) * case["Hq"] * case["Dh"]
    return dict(bytes=toks * case["Hkv"] * case["Dh"] * 1.125 + 2 * q * _es(case) + 4 * sum(_rows(case)) * case["Hq"], flops=4 * pairs * case["Hq"] * case["Dh"])


# ---------------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _pages(case, lens, rows, spare, g):
    """A pool of pages in random order: table and pages held for `lens` + `rows` tokens of each request, and the free list."""
    ps = case["ps"]
    need = [-(-(n + r) // ps) for n, r in zip(lens, rows)]
    total = sum(need) + spare
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lens), max(need) + 3), NO_PAGE, dtype=torch.int32, device=DEV)
    at = torch.arange(table.shape[1], device=DEV)
    need_t = torch.tensor(need, device=DEV)
    off = torch.cumsum(need_t, 0) - need_t
    inside = at[None] < need_t[:, None]
    table[inside] = order[(off[:, None] + at[None])[inside]]
    return table, total


def _slots(table, lens, rows, R, ps):
    i = torch.arange(R, device=DEV)
    pos = torch.tensor(lens, device=DEV)[:, None] + i[None]
    page = torch.gather(table, 1, (pos // ps).clamp(max=table.shape[1] - 1))
    slot = page * ps + pos % ps
    return torch.where(i[None] < torch.tensor(rows, device=DEV)[:, None], slot, NO_PAGE).to(torch.int32)


def _kv(shape, g):
    """Keys or values: unit variance, a few channels that stand out, and rows of differing size."""
    x = torch.randn(shape, generator=g, device=DEV)
    x *= 1 + 3 * (torch.rand(shape[-1], generator=g, device=DEV) < 0.04)
    return x


def _filled_pool(case, pages, g):
    """A layer's cache with the codes of random keys and values, made page by page as they come."""
    Hkv, Dh, nb = case["Hkv"], case["Dh"], case["ps"] // 16
    pool = torch.empty(pages, Hkv, nb, 18 * Dh, dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 25) // (Hkv * case["ps"] * Dh))
    for p in range(0, pages, step):
        part = pool[p:p + step]
        shape = (part.shape[0], Hkv, nb, 16, Dh)
        (kc, ks), (vc, vs) = _encode(_kv(shape, g)), _encode(_kv(shape, g))
        part[..., :8 * Dh] = kc.flatten(-2)
        part[..., 8 * Dh:16 * Dh] = vc.unflatten(-1, (Dh // 16, 8)).unflatten(-3, (2, 8)).transpose(-3, -2).flatten(-4)
        part[..., 16 * Dh:17 * Dh] = ks.flatten(-2)
        part[..., 17 * Dh:] = vs.unflatten(-2, (2, 8)).transpose(-2, -1).flatten(-3)
    return pool


def _trees(case, rows, seed):
    """Ancestor bitmasks of random trees in canonical order: node i's parent is about f * i, which grows with i."""
    B, N = case["B"], case["Nmax"]
    words = (N + 63) // 64
    rng = np.random.default_rng(seed)
    f = rng.uniform(0.2, 0.8, B)
    mask = np.zeros((B, N, words), np.uint64)
    for i in range(N):
        p = np.minimum(np.floor(f * (i + rng.uniform(0, 1, 1))).astype(np.int64), i) - 1
        has = p >= 0
        mask[has, i] = mask[np.nonzero(has)[0], p[has]]
        mask[:, i, i // 64] |= np.uint64(1 << (i % 64))
    return torch.from_numpy(mask.view(np.int64)).to(DEV)


def _paths(case, seed=0):
    """Accepted paths: nodes in rising order, each either in its place already or behind all places of the path."""
    B, D = case["B"], case["D"]
    rng = np.random.default_rng(seed)
    n = np.array(_rows(case)) - 1
    length = np.minimum(1 + (np.arange(B) * 5 + max(0, D - 2)) % D, n)
    node = np.zeros((B, D), np.int64)
    for b in range(B):
        L = int(length[b])
        free = np.arange(D, max(D, n[b]))
        far = np.sort(rng.permutation(free)[:L])
        node[b, :L] = np.concatenate([np.arange(L - len(far)), far]) if len(far) < L else far
    return length, node


@functools.lru_cache(maxsize=None)
def _context(Nmax, B, D, dtype):
    from paper_2609_22098_b200 import binding
    return binding.TreeSpark(V=1024, D=D, r=8, K=4, Nmax=max(1, Nmax), max_batch=B, dtype=dtype)


def _layout(case, pages, columns, dtype):
    from paper_2609_22098_b200 import binding
    return binding.CacheLayout(Hq=case.get("Hq", case.get("Hkv", 1)), Hkv=case.get("Hkv", 1), Dh=case.get("Dh", 64), page_size=case["ps"], n_pages=pages,
                               max_pages=columns, dtype=dtype)


def prepare(case, seed):
    g = _gen(seed)
    B, R, ps = case["B"], case["Nmax"] + 1, case["ps"]
    order = torch.randperm(B, generator=torch.Generator().manual_seed(seed)).tolist()
    lens = [_lens(case)[i] for i in order] if "len_lo" in case else [0] * B
    rows = [_rows(case)[i] for i in order]
    s = dict(case=case, B=B, R=R, n_nodes=_ints([r - 1 for r in rows]) if case["Nmax"] else None, seq_len=_ints(lens))
    dtype = torch.bfloat16
    if case["op"] == "reserve":
        have = [0 if case["fresh"] else -(-n // ps) for n in lens]
        full, total = _pages(case, lens, rows, 64, g)
        held = torch.tensor(have, device=DEV)
        cols = torch.arange(full.shape[1], device=DEV)
        table = torch.where(cols[None] < held[:, None], full, NO_PAGE)
        used = torch.zeros(total + 1, dtype=torch.bool, device=DEV)
        used[table.flatten().long()] = True
        free = torch.nonzero(~used[:total]).flatten()
        free = free[torch.randperm(free.numel(), generator=g, device=DEV)]
        pages = torch.zeros(total, dtype=torch.int32, device=DEV)
        pages[:free.numel()] = free
        # a pool that is short of some pages now and then: the last requests are refused
        short = -3 if seed % 4 == 3 else 64
        s.update(table=table, held=held.to(torch.int32), free_pages=pages, free_count=_ints([max(0, free.numel() - 64 + short)]), pages=total)
        s["out"] = dict(held=torch.empty_like(s["held"]), free_count=torch.empty_like(s["free_count"]), slot_map=torch.empty(B, R, dtype=torch.int32, device=DEV),
                        status=torch.empty(B, dtype=torch.int32, device=DEV))
    else:
        table, total = _pages(case, lens, rows, 5, g)
        s.update(table=table, pages=total)
        if case["op"] == "append":
            dtype = _dtype(case)
            Hkv, Dh = case["Hkv"], case["Dh"]
            # keys and values as a projection leaves them, side by side in one row
            both = torch.stack([_kv((B, R, Hkv, Dh), g), _kv((B, R, Hkv, Dh), g)], 2).to(dtype)
            s.update(k=both[:, :, 0], v=both[:, :, 1], slot_map=_slots(table, lens, rows, R, ps), pool=torch.zeros(total, Hkv, ps // 16, 18 * Dh, dtype=torch.uint8, device=DEV))
            s["k_val"], s["v_val"] = (torch.zeros(B, R, Hkv, Dh, dtype=dtype, device=DEV) for _ in range(2)) if case["values"] else (None, None)
        elif case["op"] == "attn":
            dtype = _dtype(case)
            s["pool"] = _filled_pool(case, total, g)
            s["q"] = (1.5 * torch.randn(B, R, case["Hq"], case["Dh"], generator=g, device=DEV)).to(dtype)
            s["mask"] = _trees(case, rows, seed) if case["tree"] and case["Nmax"] else None
            s["o"] = torch.zeros_like(s["q"])
            s["lse"] = torch.zeros(B, R, case["Hq"], dtype=torch.float32, device=DEV)
        else:
            length, node = _paths(case, seed)
            length, node = length[order], node[order]
            s.update(acc_len=_ints(length.tolist()), acc_node=_ints(node.tolist()), seq_out=torch.empty(B, dtype=torch.int32, device=DEV))
            s["pool"] = torch.randint(0, 256, (case["layers"], total, case["Hkv"], ps // 16, 18 * case["Dh"]), generator=g, device=DEV, dtype=torch.uint8)
    if own:
        s["ts"] = _context(case["Nmax"], B, case.get("D", 4), dtype)
        s["lay"] = _layout(case, s["pages"], s["table"].shape[1], dtype)
        if case["op"] == "attn":
            s["ws"] = s["ts"].attention_workspace(s["lay"], B)
    return s


# ---------------------------------------------------------------------------------------------------------------------------
# the format, plainly
# ---------------------------------------------------------------------------------------------------------------------------
_PAIR = [0, 2, 4, 6, 1, 3, 5, 7]     # element of nibble 0..7 of a word
_ELEMENT = [0, 4, 1, 5, 2, 6, 3, 7]  # nibble of element 0..7


def _encode(x):
    """[..., Dh] -> codes [..., Dh / 2] and scales [..., Dh / 16], as bytes."""
    y = x.float().unflatten(-1, (-1, 16))
    top = y.abs().amax(-1)
    scale = (top / torch.full_like(top, 7)).clamp(max=448).to(torch.float8_e4m3fn)   # (by a number torch would multiply with 1 / 7: another value next to a border)
    s = scale.float()[..., None]
    c = torch.where(s > 0, (torch.round(y / s)).clamp(-8, 7) + 8, 8.0).to(torch.uint8)
    n = c.flatten(-2).unflatten(-1, (-1, 8))[..., _PAIR].unflatten(-1, (4, 2))
    return (n[..., 0] | (n[..., 1] << 4)).flatten(-2), scale.view(torch.uint8)


def _decode(codes, scales):
    """The values of codes [..., Dh / 2] and scales [..., Dh / 16]."""
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, 8))[..., _ELEMENT].flatten(-2)
    s = scales.view(torch.float8_e4m3fn).float()
    return ((n.float() - 8).unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2)


@functools.lru_cache(maxsize=None)
def _bytes_of_token(Dh):
    """Where the 18 * Dh / 16 bytes of each of a block's 16 tokens lie: K codes, V codes, K scales, V scales."""
    t, G = torch.arange(16)[:, None], Dh // 16
    kc = t * (Dh // 2) + torch.arange(Dh // 2)
    j = torch.arange(Dh // 2)
    vc = 8 * Dh + (t // 8) * (4 * Dh) + (j // 8) * 64 + (t % 8) * 8 + j % 8
    ks = 16 * Dh + t * G + torch.arange(G)
    vs = 17 * Dh + (t // 8) * (G * 8) + torch.arange(G) * 8 + t % 8
    return torch.cat([kc, vc, ks, vs], 1).to(DEV)


def _place(slot, ps, Dh):
    """(page, block, bytes) of slots."""
    return slot // ps, slot % ps // 16, _bytes_of_token(Dh)[slot % 16]


# ---------------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------------
def run(s):
    return {"reserve": _reserve, "append": _append, "attn": _attention, "commit": _commit}[s["case"]["op"]](s)


def _reserve(s):
    if own:
        o = s["ts"].cache_reserve(s["lay"], s["seq_len"], s["held"], s["free_pages"], s["free_count"], s["table"], n_nodes=s["n_nodes"], out=s["out"])
        return dict(o, table=s["table"])
    ps, table, held, count = s["case"]["ps"], s["table"], s["held"].long(), s["free_count"].long()
    seq = s["seq_len"].long()
    rows = (s["n_nodes"].long() if s["n_nodes"] is not None else 0) + torch.ones_like(seq)
    need = (seq + rows + ps - 1) // ps
    take = (need - held).clamp(min=0)
    start = torch.cumsum(take, 0) - take
    granted = (take == 0) | (start + take <= count)
    cols = torch.arange(table.shape[1], device=DEV)[None]
    new = (cols >= held[:, None]) & (cols < need[:, None]) & granted[:, None]
    page = s["free_pages"][(count - 1 - (start - held)[:, None] - cols).clamp(0, s["free_pages"].numel() - 1)]
    table = torch.where(new, page, table)
    i = torch.arange(s["R"], device=DEV)[None]
    pos = seq[:, None] + i
    slot = torch.gather(table, 1, (pos // ps).clamp(max=table.shape[1] - 1)) * ps + pos % ps
    slot = torch.where((i < rows[:, None]) & granted[:, None], slot, NO_PAGE).to(torch.int32)
    return dict(table=table, held=torch.where(granted, torch.maximum(held, need), held).to(torch.int32), free_count=(count - (take * granted).sum()).to(torch.int32),
                slot_map=slot, status=torch.where(granted, 0, REFUSED).to(torch.int32))


def _append(s):
    if own:
        s["ts"].cache_append(s["lay"], s["k"], s["v"], s["slot_map"], s["pool"], k_val=s["k_val"], v_val=s["v_val"])
        return dict(pool=s["pool"], k=s["k_val"], v=s["v_val"])
    case, slot = s["case"], s["slot_map"].flatten().long()
    used = slot >= 0
    k, v, slot = s["k"].flatten(0, 1)[used], s["v"].flatten(0, 1)[used], slot[used]
    (kc, ks), (vc, vs) = _encode(k), _encode(v)
    page, block, at = _place(slot, case["ps"], case["Dh"])
    head = torch.arange(case["Hkv"], device=DEV)
    s["pool"][page[:, None, None], head[None, :, None], block[:, None, None], at[:, None, :]] = torch.cat([kc, vc, ks, vs], -1)
    if case["values"]:
        s["k_val"].flatten(0, 1)[used] = _decode(kc, ks).to(k.dtype)
        s["v_val"].flatten(0, 1)[used] = _decode(vc, vs).to(v.dtype)
    return dict(pool=s["pool"], k=s["k_val"], v=s["v_val"])


def _attention(s):
    case = s["case"]
    scale = case["Dh"] ** -0.5
    if own:
        s["ts"].tree_attention(s["lay"], s["q"], s["pool"], s["table"], s["seq_len"], n_nodes=s["n_nodes"], mask=s["mask"], scale=scale, out=s["o"], lse=s["lse"], ws=s["ws"])
        return dict(o=s["o"], lse=s["lse"])
    B, R, Hkv, Dh, ps = s["B"], s["R"], case["Hkv"], case["Dh"], case["ps"]
    g = case["Hq"] // Hkv
    raw = s["pool"][s["table"].long().clamp(min=0)].transpose(1, 2).flatten(2, 3)                         # [B][Hkv][blocks][18 Dh]
    k = _decode(raw[..., :8 * Dh].unflatten(-1, (16, -1)), raw[..., 16 * Dh:17 * Dh].unflatten(-1, (16, -1))).flatten(2, 3)
    vc = raw[..., 8 * Dh:16 * Dh].unflatten(-1, (2, Dh // 16, 8, 8)).transpose(-3, -2).flatten(-2).flatten(-3, -2)
    vs = raw[..., 17 * Dh:].unflatten(-1, (2, Dh // 16, 8)).transpose(-2, -1).flatten(-3, -2)
    v = _decode(vc, vs).flatten(2, 3)                                                                     # [B][Hkv][T][Dh]
    T = k.shape[2]
    pos = torch.arange(T, device=DEV) - s["seq_len"].long()[:, None]                                      # [B][T]: row of this round, below 0 the prefix
    rows = (s["n_nodes"].long() if s["n_nodes"] is not None else torch.zeros(B, dtype=torch.long, device=DEV)) + 1
    i = torch.arange(R, device=DEV)
    if s["mask"] is None:
        sees = pos[:, None, :] <= i[None, :, None]
    else:
        bit = (pos - 1).clamp(0, case["Nmax"] - 1)[:, None, :].expand(B, case["Nmax"], T)
        on = ((torch.gather(s["mask"], 2, bit // 64) >> (bit % 64)) & 1).bool() & (pos >= 1)[:, None, :]
        sees = torch.cat([torch.zeros_like(on[:, :1]), on], 1) | (pos <= 0)[:, None, :]
    sees &= (pos < rows[:, None])[:, None, :]                                                             # [B][R][T]
    q = s["q"].float().unflatten(2, (Hkv, g)).permute(0, 2, 1, 3, 4).flatten(2, 3)                        # [B][Hkv][R g][Dh]
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(scale).unflatten(2, (R, g))
    x.masked_fill_(~sees[:, None, :, None, :], float("-inf"))
    m = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(m > float("-inf"), m, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (R, g)) / total.clamp(min=1e-38)
    lse = (m + total.log())[..., 0]
    used = (i[None] < rows[:, None])
    s["o"][used] = o.permute(0, 2, 1, 3, 4).flatten(2, 3).to(s["o"].dtype)[used]
    s["lse"][used] = lse.permute(0, 2, 1, 3).flatten(2, 3)[used]
    return dict(o=s["o"], lse=s["lse"])


def _commit(s):
    if own:
        s["ts"].cache_commit(s["lay"], s["pool"], s["table"], s["seq_len"], s["acc_len"], s["acc_node"], seq_len_out=s["seq_out"])
        return dict(pool=s["pool"], seq_len=s["seq_out"])
    case = s["case"]
    ps, D = case["ps"], case["D"]
    i = torch.arange(D, device=DEV)[None]
    seq, on = s["seq_len"].long()[:, None], i < s["acc_len"][:, None]
    move = lambda row: torch.gather(s["table"].long(), 1, ((seq + row) // ps).clamp(max=s["table"].shape[1] - 1)) * ps + (seq + row) % ps  # noqa: E731
    src, dst = move(1 + s["acc_node"].long())[on], move((1 + i).expand_as(on))[on]
    head = torch.arange(case["Hkv"], device=DEV)[None, :, None]
    page, block, at = _place(src, ps, case["Dh"])
    rows = s["pool"][:, page[:, None, None], head, block[:, None, None], at[:, None, :]]
    page, block, at = _place(dst, ps, case["Dh"])
    s["pool"][:, page[:, None, None], head, block[:, None, None], at[:, None, :]] = rows
    s["seq_out"].copy_(s["seq_len"] + 1 + s["acc_len"])
    return dict(pool=s["pool"], seq_len=s["seq_out"])


# ---------------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, request by request
# ---------------------------------------------------------------------------------------------------------------------------
_E4M3 = sorted({m * 2.0 ** -9 for m in range(8)} | {(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)} - {480.0})


def _nearest_scale(t):
    """The nearest of the 127 scales to t (float64), the even one of two as near."""
    grid = torch.tensor(_E4M3, dtype=torch.float64, device=DEV)
    hi = torch.searchsorted(grid, t.clamp(max=448.0)).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - t, t - grid[lo]
    return torch.where((up < down) | ((up == down) & (hi % 2 == 0)) | (t >= 448.0), grid[hi], grid[lo])


def _held_as(x):
    """What is held for x, in 64 bits."""
    y = x.double().reshape(*x.shape[:-1], -1, 16)
    top = y.abs().amax(-1)
    s = _nearest_scale(top / torch.full_like(top, 7))[..., None]
    return torch.where(s > 0, torch.clamp(torch.round(y / torch.where(s > 0, s, 1.0)), -8, 7) * s, 0.0).reshape(x.shape)


def _read_head(pool, pages, Dh):
    """K and V [tokens][Hkv][Dh] of a list of pages, in 64 bits: nibble by nibble from the bytes of each token."""
    raw = pool[pages].permute(0, 2, 1, 3)                       # [pages][blocks][Hkv][18 Dh]
    tok = raw[..., _bytes_of_token(Dh)]                         # [pages][blocks][Hkv][16][18 Dh / 16]
    tok = tok.permute(0, 1, 3, 2, 4).flatten(0, 2)              # [tokens][Hkv][bytes]
    out = []
    for c0, s0 in ((0, Dh), (Dh // 2, Dh + Dh // 16)):
        word = tok[..., c0:c0 + Dh // 2].unflatten(-1, (-1, 4)).long()
        word = word[..., 0] | word[..., 1] << 8 | word[..., 2] << 16 | word[..., 3] << 24
        value = torch.stack([(word >> 4 * (e // 2 + 4 * (e % 2))) & 15 for e in range(8)], -1).double() - 8
        scale = torch.tensor(_E4M3 + [float("nan")] * 129, dtype=torch.float64, device=DEV)[tok[..., s0:s0 + Dh // 16].long()]
        out.append(value.flatten(-2) * scale.repeat_interleave(16, -1))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("reserve", "commit"):
        return None
    if case["op"] == "append":
        if not case["values"]:
            return None
        used = (s["slot_map"] >= 0)[..., None, None]
        return dict(pool=None, k=torch.where(used, _held_as(s["k"]), 0.0), v=torch.where(used, _held_as(s["v"]), 0.0))
    B, R, Hq, Hkv, Dh, ps = case["B"], s["R"], case["Hq"], case["Hkv"], case["Dh"], case["ps"]
    o = torch.zeros(B, R, Hq, Dh, dtype=torch.float64, device=DEV)
    lse = torch.zeros(B, R, Hq, dtype=torch.float64, device=DEV)
    for b in range(B):
        n = int(s["seq_len"][b])
        rows = 1 + (int(s["n_nodes"][b]) if s["n_nodes"] is not None else 0)
        k, v = _read_head(s["pool"], s["table"][b, :-(-(n + rows) // ps)].long(), Dh)
        sees = torch.zeros(rows, n + rows, dtype=torch.bool, device=DEV)
        sees[:, :n + 1] = True
        if s["mask"] is None:
            sees[:, n:] = torch.ones(rows, rows, device=DEV).tril().bool()
        elif rows > 1:
            bits = torch.stack([(s["mask"][b, :rows - 1, j // 64] >> (j % 64)) & 1 for j in range(rows - 1)], 1)
            sees[1:, n + 1:] = bits.bool()
        for h in range(Hkv):
            kh, vh = k[:n + rows, h], v[:n + rows, h]
            g = Hq // Hkv
            x = torch.einsum("rgd,td->grt", s["q"][b, :rows, h * g:(h + 1) * g].double(), kh) / math.sqrt(Dh)
            x = torch.where(sees[None], x, float("-inf"))
            z = torch.logsumexp(x, -1)
            lse[b, :rows, h * g:(h + 1) * g] = z.T
            o[b, :rows, h * g:(h + 1) * g] = torch.einsum("grt,td->rgd", torch.exp(x - z[..., None]), vh)
    return dict(o=o, lse=lse)
