"""The 4-bit key/value cache around the target's forward -- TEST INFRASTRUCTURE.

Plain restatement in float64 / Python integers of the four calls around the cache: pages and slots of a round, the write into
the cache, the attention of a tree's rows (Section 3.2, item 3: row i attends to the prefix and to its root path), the move of
the accepted path.  Only the tests import this module; the product path never does.

Format (the paper fixes none): per page and head, blocks of 16 tokens, each 18 * Dh bytes: K codes row by row; V codes octet of
tokens by octet, group of 16 channels by group, token by token; K scales row by row; V scales octet, group, token.  Value =
(code - 8) * scale * 2**exp; channel 2j of a 32-bit word is nibble j, channel 2j + 1 nibble j + 4.
"""
from __future__ import annotations

import numpy as np

OVERFLOW = -6
NAN_SCALE = 0x7F


def _scale_values():
    v = []
    for byte in range(127):
        e, m = byte >> 3, byte & 7
        v.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(v)


SCALES = _scale_values()          # value of scale byte 0..126; 127 is NaN


def nearest_scale(t):
    """Byte of the scale nearest to t >= 0, the even byte of two as near, at most 448."""
    t = min(float(t), 448.0)
    hi = int(np.searchsorted(SCALES, t))
    if SCALES[hi] == t or hi == 0:
        return hi
    lo = hi - 1
    a, b = t - SCALES[lo], SCALES[hi] - t
    return lo if a < b or (a == b and lo % 2 == 0) else hi


def quantise(x, exp):
    """Codes [Dh] in 0..15 and scale bytes [Dh / 16] of a row x [Dh] (float64, finite)."""
    codes, scales = np.full(len(x), 8, np.int64), np.zeros(len(x) // 16, np.int64)
    for g in range(len(x) // 16):
        y = np.asarray(x[16 * g:16 * g + 16], np.float64) * 2.0 ** -exp
        byte = nearest_scale(np.max(np.abs(y)) / 7.0)
        scales[g] = byte
        if SCALES[byte] > 0:
            codes[16 * g:16 * g + 16] = np.clip(np.rint(y / SCALES[byte]), -8, 7) + 8
    return codes, scales


def _word_bytes(codes8):
    w = 0
    for e in range(8):
        w |= int(codes8[e]) << (4 * (e // 2 + 4 * (e % 2)))
    return [(w >> 8 * i) & 255 for i in range(4)]


def _row_bytes(codes):
    return [b for i in range(0, len(codes), 8) for b in _word_bytes(codes[i:i + 8])]


def token_bytes(Dh, tau):
    """Places in a block of the bytes of token tau: (K codes, V codes, K scales, V scales)."""
    kc = [tau * (Dh // 2) + i for i in range(Dh // 2)]
    vc = [8 * Dh + (tau // 8) * 4 * Dh + (i // 8) * 64 + (tau % 8) * 8 + i % 8 for i in range(Dh // 2)]
    ks = [16 * Dh + tau * (Dh // 16) + i for i in range(Dh // 16)]
    vs = [17 * Dh + (tau // 8) * (Dh // 2) + i * 8 + tau % 8 for i in range(Dh // 16)]
    return kc, vc, ks, vs


def append(pool, page_size, slots, k, v, k_exp=0, v_exp=0):
    """Write rows k, v [n][Hkv][Dh] to `slots` of pool [pages][Hkv][page_size/16][18 Dh] (uint8, in place); returns the values
    that the cache holds for them (float64; rows without a slot: untouched zeros)."""
    n, Hkv, Dh = k.shape
    kv, vv = np.zeros((n, Hkv, Dh)), np.zeros((n, Hkv, Dh))
    for i in range(n):
        if not 0 <= slots[i] < pool.shape[0] * page_size:
            continue
        page, at = divmod(int(slots[i]), page_size)
        kc, vc, ks, vs = token_bytes(Dh, at % 16)
        for h in range(Hkv):
            blk = pool[page, h, at // 16]
            if not (np.isfinite(k[i, h]).all() and np.isfinite(v[i, h]).all()):
                blk[kc] = blk[vc] = 0x88
                blk[ks] = blk[vs] = NAN_SCALE
                kv[i, h] = vv[i, h] = np.nan
                continue
            for row, c, s, exp, val in ((k[i, h], kc, ks, k_exp, kv), (v[i, h], vc, vs, v_exp, vv)):
                codes, scales = quantise(row, exp)
                blk[c] = _row_bytes(codes)
                blk[s] = scales
                val[i, h] = (codes - 8) * np.repeat(SCALES[scales], 16) * 2.0 ** exp
    return kv, vv


def read(pool, page_size, slot, h, Dh, k_exp=0, v_exp=0):
    """K and V [Dh] of a slot's head as the cache holds them (float64, NaN where the scale is)."""
    page, at = divmod(int(slot), page_size)
    blk = pool[page, h, at // 16]
    kc, vc, ks, vs = token_bytes(Dh, at % 16)
    out = []
    for c, s, exp in ((kc, ks, k_exp), (vc, vs, v_exp)):
        b = blk[c].astype(np.int64).reshape(-1, 4)
        w = b[:, 0] | b[:, 1] << 8 | b[:, 2] << 16 | b[:, 3] << 24
        codes = np.stack([(w >> 4 * (e // 2 + 4 * (e % 2))) & 15 for e in range(8)], 1).reshape(-1)
        sc = blk[s].astype(np.int64)
        val = np.where(sc & 0x7F == NAN_SCALE, np.nan, SCALES[np.minimum(sc & 0x7F, 126)])
        out.append((codes - 8) * np.repeat(val, 16) * 2.0 ** exp)
    return out


def reserve(page_size, n_pages, seq_len, rows, held, free_pages, free_count, table, R):
    """Pages and slots of a round, request by request.  Returns table, held, free list, free count, slots [B][R], status."""
    table, held, free, B = table.copy(), list(held), list(free_pages), len(seq_len)
    count, status, slots, back, short = int(free_count), [0] * B, np.full((B, R), -1, np.int64), [], False
    for b in range(B):
        if seq_len[b] < 0:
            back += [int(p) for p in table[b, :held[b]] if 0 <= p < n_pages]   # (other entries are no pages)
            table[b, :held[b]] = -1
            held[b] = 0
            continue
        need = -(-(int(seq_len[b]) + rows[b]) // page_size)
        take = max(0, need - held[b])
        if need > table.shape[1] or (take and (short or take > count)):
            status[b] = OVERFLOW
            short = short or need <= table.shape[1]
            continue
        for c in range(held[b], need):
            count -= 1
            table[b, c] = free[count]
        held[b] = max(held[b], need)
        for i in range(rows[b]):
            pos = int(seq_len[b]) + i
            page = int(table[b, pos // page_size])
            if 0 <= page < n_pages:
                slots[b, i] = page * page_size + pos % page_size
    for p in back:
        free[count] = p
        count += 1
    return table, held, free, count, slots, status


def sees(mask_words, i, rel):
    """Whether row i sees the token at place rel behind the prefix; mask_words None: a chain."""
    if mask_words is None:
        return rel <= i
    if rel == 0 or i == 0:
        return rel == 0
    return bool((int(mask_words[i - 1][(rel - 1) // 64]) >> ((rel - 1) % 64)) & 1)


def attention(pool, page_size, table_row, seq_len, rows, q, mask_words, scale, k_exp=0, v_exp=0):
    """Rows q [rows][Hq][Dh] of one request: (out [rows][Hq][Dh], lse [rows][Hq]) in float64."""
    rows_, Hq, Dh = q.shape
    Hkv = pool.shape[1]
    out, lse = np.zeros((rows, Hq, Dh)), np.full((rows, Hq), -np.inf)
    pos = [p for p in range(seq_len + rows)
           if p // page_size < len(table_row) and 0 <= table_row[p // page_size] < pool.shape[0]]
    if not pos:
        return out, lse
    visible = np.array([[p < seq_len or sees(mask_words, i, p - seq_len) for p in pos] for i in range(rows)])
    for h in range(Hkv):
        kv = [read(pool, page_size, int(table_row[p // page_size]) * page_size + p % page_size, h, Dh, k_exp, v_exp) for p in pos]
        K, V = np.array([x[0] for x in kv]), np.array([x[1] for x in kv])
        for i in range(rows):
            on = visible[i]
            if not on.any():
                continue
            for hq in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                x = scale * (K[on] @ q[i, hq].astype(np.float64))
                m = x.max()
                e = np.exp(x - m)
                out[i, hq] = e @ V[on] / e.sum()
                lse[i, hq] = m + np.log(e.sum())
                if np.isnan(x).any():   # a token that holds NaN makes the whole row NaN
                    out[i, hq], lse[i, hq] = np.nan, np.nan
    return out, lse


def commit(pool, page_size, table_row, seq_len, acc_len, acc_node, Nmax):
    """Move the rows of an accepted path in pool [layers][pages][Hkv][blocks][18 Dh] (in place); returns the new length."""
    if seq_len < 0:
        return seq_len
    Dh = pool.shape[-1] // 18

    def where(row):
        p = seq_len + row
        if p // page_size >= len(table_row) or not 0 <= table_row[p // page_size] < pool.shape[1]:
            return None
        return int(table_row[p // page_size]), p % page_size

    moves = []
    for i in range(acc_len):
        src, dst = (where(1 + int(acc_node[i])) if 0 <= acc_node[i] < Nmax else None), where(1 + i)
        if src is not None and dst is not None:
            at = np.concatenate(token_bytes(Dh, src[1] % 16))
            moves.append((dst, pool[:, src[0], :, src[1] // 16][..., at].copy()))
    for dst, data in moves:
        at = np.concatenate(token_bytes(Dh, dst[1] % 16))
        view = pool[:, dst[0], :, dst[1] // 16]
        view[..., at] = data
    return seq_len + 1 + acc_len
