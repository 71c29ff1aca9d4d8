"""The 8-bit KV cache in 64 bits: what a row is held as, where its bytes lie, and attention over what they stand for.

An element is an e4m3 code times a power of two 2^e that the 32 rows of a block share per kv head: e is the least whole number,
-100 at least, with max|x| <= 448 2^e; where later rows of a block raise it, the codes of the earlier ones are rounded once
more.  Codes are held to 240 at e = 120: 256 2^120 is no bf16 number.  NaN counts as 0, an infinity as the largest finite bf16.  Plain numpy, from the format's definition
(include/space.h, space_kvb_cache).
"""
import numpy as np

from .kvq import BF16_MAX, sanitise, visible
from .layout import SAME_GROUP

PAGE, BLOCK = 128, 32


def _values():
    """What the codes 0 .. 127 stand for (the last one: NaN)."""
    c = np.arange(128)
    e, m = c >> 3, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[127] = np.nan
    return v


VALUES = np.concatenate([_values(), -_values()])


def encode(x):
    """Nearest codes (ties to even), held to +-448."""
    a = np.minimum(np.abs(x), 448.0)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -20))), -6) - 3)
    a = np.round(a / step) * step
    code = np.searchsorted(VALUES[:127], a)
    assert (VALUES[code] == a).all()
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def exponent(top):
    e = -100
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


def head_bytes(d):
    return 2 * PAGE * d + 8 * (PAGE // BLOCK)


def _views(mem, d):
    """K codes [128, d], V codes [128, d] and scales [4, 2] of a page of one head (views of its bytes)."""
    n = PAGE * d
    k = mem[:n].reshape(d // 16, PAGE, 16)
    v = mem[n:2 * n].reshape(PAGE // 16, d, 16)
    return k, v, mem[2 * n:].view(np.float32).reshape(PAGE // BLOCK, 2)


def append(pool, table, head, L, k, v):
    """Rows k, v [n, d] (64 bits, finite) behind the L rows of a sequence; pool [n_pages, H, head_bytes] is changed.  Pages
    outside the pool are skipped."""
    n, d = k.shape
    k, v = (np.clip(x, -240 * 2.0 ** 120, 240 * 2.0 ** 120) for x in (k, v))
    for s0 in range(L // BLOCK * BLOCK, L + n, BLOCK):
        page = table[s0 // PAGE]
        if not 0 <= page < pool.shape[0]:
            continue
        lo, hi = max(L - s0, 0), min(L + n - s0, BLOCK)
        kc, vc, sc = _views(pool[page, head], d)
        row0 = s0 % PAGE
        for which, x in ((0, k), (1, v)):
            rows = x[s0 + lo - L:s0 + hi - L]
            e = exponent(np.abs(rows).max())
            old = sc[row0 // BLOCK, which]
            if lo > 0 and 2.0 ** e <= old:
                e = int(np.log2(old))
            at = lambda i: (kc[:, row0 + i, :].reshape(-1) if which == 0 else vc[(row0 + i) // 16, :, (row0 + i) % 16])

            def put(i, codes):
                if which == 0:
                    kc[:, row0 + i, :] = codes.reshape(-1, 16)
                else:
                    vc[(row0 + i) // 16, :, (row0 + i) % 16] = codes
            if lo > 0 and 2.0 ** e > old:
                for i in range(lo):
                    put(i, encode(VALUES[at(i)] * (float(old) / 2.0 ** e)))
            for i in range(lo, hi):
                put(i, encode(rows[i - lo] / 2.0 ** e))
            sc[row0 // BLOCK, which] = 2.0 ** e


def read_rows(pool, table, n, d):
    """Rows 0 .. n-1 of one sequence: K and V [H, n, d] in 64 bits; rows of a page outside the pool are NaN."""
    H = pool.shape[1]
    out = [np.full((H, n, d), np.nan) for _ in range(2)]
    for t in range((n + PAGE - 1) // PAGE):
        if not 0 <= table[t] < pool.shape[0]:
            continue
        m = min(PAGE, n - t * PAGE)
        for h in range(H):
            kc, vc, sc = _views(pool[table[t], h], d)
            s = np.repeat(sc.astype(np.float64), BLOCK, 0)
            out[0][h, t * PAGE:t * PAGE + m] = (VALUES[kc].transpose(1, 0, 2).reshape(PAGE, d) * s[:, :1])[:m]
            out[1][h, t * PAGE:t * PAGE + m] = (VALUES[vc].transpose(0, 2, 1).reshape(PAGE, d) * s[:, 1:])[:m]
    return out


def turn(x, table, pos, interleaved=False):
    """Rows x [n, ..., d] (fp32) at positions pos [n], by a table [n_pos, rot]: in fp32, each product and the sum rounded."""
    x = x.astype(np.float32)
    rot = table.shape[1]
    row = table[np.clip(pos, 0, table.shape[0] - 1)].astype(np.float32)
    row = row.reshape(row.shape[0], *([1] * (x.ndim - 2)), rot)
    c, s = row[..., :rot // 2], row[..., rot // 2:]
    y = x.copy()
    i = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., i[0]], x[..., i[1]]
    y[..., i[0]], y[..., i[1]] = a * c - b * s, b * c + a * s
    return y


def attention(q, pool, table, kv_len, k, scale, k_new=None, v_new=None, variant=SAME_GROUP):
    """q [B, n_q, H_q, d], k_new / v_new [B, n_q, H_kv, d] in 64 bits -> out [B, n_q, H_q, d], lse [B, H_q, n_q], and what
    their errors are held to: the bound's arithmetic is in bounds()."""
    B, n_q, H_q, d = q.shape
    H = pool.shape[1]
    out, lse = np.zeros(q.shape), np.full((B, H_q, n_q), -np.inf)
    tol, lse_tol = np.zeros(q.shape[:3]), np.zeros(lse.shape)
    for b in range(B):
        n = int(kv_len[b])
        if n < 0 or n > PAGE * table.shape[1]:
            continue
        K, V = read_rows(pool, table[b], n, d)
        there = ~np.isnan(K[0, :, 0]) if n else np.zeros(0, dtype=bool)
        page = np.arange(n)[there] // PAGE
        K, V = K[:, there], V[:, there]
        see = np.ones((n_q, K.shape[1]), dtype=bool)
        if k_new is not None:
            K = np.concatenate([K, sanitise(k_new[b]).transpose(1, 0, 2)], 1)
            V = np.concatenate([V, sanitise(v_new[b]).transpose(1, 0, 2)], 1)
            see = np.concatenate([see, visible(k, variant)], 1)
            page = np.concatenate([page, np.full(n_q, 1 << 30)])
        if not K.shape[1]:
            continue
        for hq in range(H_q):
            h = hq * H // H_q
            s = np.where(see, q[b, :, hq] @ K[h].T * scale, -np.inf)
            m = s.max(-1, keepdims=True)
            ok = np.isfinite(m[:, 0])
            p = np.where(see, np.exp(s - np.where(np.isfinite(m), m, 0.0)), 0.0)
            l = p.sum(-1, keepdims=True)
            p = p / np.where(l > 0, l, 1.0)
            out[b, :, hq] = p @ V[h]
            lse[b, hq] = np.where(ok, m[:, 0] + np.log(np.where(l > 0, l, 1.0))[:, 0], -np.inf)
            tol[b, :, hq], lse_tol[b, hq] = bounds(q[b, :, hq], K[h], V[h], p, see, page, scale)
    return out, lse, tol, lse_tol


def bounds(q, K, V, p, see, page, scale):
    """How far a row may be off before its rounding to bf16 (every channel), and its log sum.
    Scores: elements of a query row, and of a block's own row, are off by at most 2^-17 of the row's largest; sums of d products in
    fp32 by d 2^-24 of the products' magnitudes.  Only keys that count (p > 2^-40) do so.
    Weights: 2^-8 of themselves (two terms of four bits), and 2^-18 of the largest p |V| among 128 keys, for each of those keys;
    the exponential and the sums: 2^-20.  A block's own V rows: 2^-17 of their largest."""
    d = q.shape[1]
    aq, aK = np.abs(q), np.abs(K)
    e = 2.0 ** -17 * (aq.max(-1)[:, None] * aK.sum(-1)[None] + aq.sum(-1)[:, None] * aK.max(-1)[None]) + d * 2.0 ** -24 * (aq @ aK.T)
    delta = (np.where(see & (p > 2.0 ** -40), e, 0.0) * scale).max(-1)
    big = np.abs(V).max(-1)
    pv = p * big[None]
    floor = sum(128 * 2.0 ** -18 * pv[:, page == t].max(-1) for t in np.unique(page))
    tol = (2.0 ** -8 + 2.0 ** -17 + 2.0 ** -20 + 2 * delta) * pv.sum(-1) + floor
    return tol, delta + 2.0 ** -18
