"""The 4-bit KV cache in 64 bits: what a row is held as, where its bytes lie, and attention over what they stand for.

A row x of d channels: lo = min x, step = bf16(max((max x - lo) / 15, max|x| / 4096, 2^-100)), codes
u = min(round((x - lo) / step), 15) with ties to even; it stands for lo + step u.  NaN counts as 0, an infinity as the
largest finite bf16.  Plain numpy, element by element from the format's definition (include/space.h, space_kvq_cache).
"""
import numpy as np

from .bf16 import bf16_bits_to_f64 as to_f64
from .layout import SAME_GROUP, block_mask_rows

PAGE, BLOCK = 128, 32
BF16_MAX = float(np.uint32(0x7F7F0000).view(np.float32))


def round_bf16(x):
    """Nearest bf16 (ties to even) of 64-bit values, as 64-bit values."""
    m, e = np.frexp(x)
    return np.ldexp(np.round(np.ldexp(m, 8)), e - 8)


def bits_of(x):
    """Bit patterns of values that bf16 holds."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    assert not (u & 0xFFFF).any()
    return (u >> 16).astype(np.uint16)


def sanitise(x):
    x = np.where(np.isnan(x), 0.0, x)
    return np.clip(x, -BF16_MAX, BF16_MAX)


def quantise(x):
    """x [..., d] -> codes, step [..., 1], lo [..., 1]."""
    x = sanitise(x)
    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    step = round_bf16(np.maximum(np.maximum((hi - lo) / 15.0, np.maximum(-lo, hi) / 4096.0), 2.0 ** -100))
    return np.minimum(np.round((x - lo) / step), 15.0), step, lo


def values(x):
    u, step, lo = quantise(x)
    return lo + step * u


def block_bytes(d):
    return BLOCK * d + 8 * BLOCK


def _places(d):
    """Byte and shift of K and V codes in a block, [32, d] each."""
    r, c = np.arange(BLOCK)[:, None], np.arange(d)[None]
    k_at, k_sh = r * (d // 2) + c // 2, 4 * (c % 2) + 0 * r
    w, q, n = c // 32, c // 8 % 4, c % 8
    a, e, t, h = r // 16, r // 8 % 2, r // 2 % 4, r % 2
    v_at = BLOCK * d // 2 + 512 * w + 64 * n + 16 * t + 8 * a + 4 * e + 2 * h + q // 2
    return (k_at, k_sh), (v_at, 4 * (q % 2) + 0 * r)


def write_row(pool, page, head, row, k, v):
    """Row `row` of a page (pool [n_pages, H, 4 * block_bytes], uint8) from the channels of K and V."""
    d = k.shape[0]
    base, i = row // BLOCK * block_bytes(d), row % BLOCK
    mem = pool[page, head]
    for which, x in ((0, k), (1, v)):
        u, step, lo = quantise(x)
        at, sh = (p[i] for p in _places(d)[which])
        for c in range(d):
            b = base + int(at[c])
            mem[b] = (int(mem[b]) & ~(15 << int(sh[c])) & 255) | (int(u[c]) << int(sh[c]))
        p = base + BLOCK * d + which * 4 * BLOCK + 4 * i
        mem[p:p + 4] = np.concatenate([bits_of(step), bits_of(lo)]).view(np.uint8)


def read_rows(pool, table, n, d):
    """Rows 0 .. n-1 of one sequence: K and V [H, n, d] in 64 bits; rows of a page outside the pool are NaN."""
    H = pool.shape[1]
    out = [np.full((H, n, d), np.nan) for _ in range(2)]
    for t in range((n + PAGE - 1) // PAGE):
        if not 0 <= table[t] < pool.shape[0]:
            continue
        mem = pool[table[t]].reshape(H, PAGE // BLOCK, block_bytes(d))
        for which, (at, sh) in enumerate(_places(d)):
            code = (mem[:, :, at] >> sh.astype(np.uint8)) & 15
            par = np.ascontiguousarray(mem[:, :, BLOCK * d + which * 4 * BLOCK:BLOCK * d + (which + 1) * 4 * BLOCK]).view(np.uint16)
            par = to_f64(par.reshape(H, PAGE // BLOCK, BLOCK, 2))
            rows = (par[..., 1:] + par[..., :1] * code).reshape(H, PAGE, d)
            m = min(PAGE, n - t * PAGE)
            out[which][:, t * PAGE:t * PAGE + m] = rows[:, :m]
    return out


def visible(k, variant=SAME_GROUP):
    if k == 0:
        return np.ones((1, 1), dtype=bool)
    return np.array([[bool((m >> j) & 1) for j in range((k + 1) ** 2)] for m in block_mask_rows(k, variant)])


def attention(q, pool, table, kv_len, k, scale, k_new=None, v_new=None, variant=SAME_GROUP):
    """q [B, n_q, H_q, d], k_new / v_new [B, n_q, H_kv, d] in 64 bits; out [B, n_q, H_q, d], lse [B, H_q, n_q]."""
    B, n_q, H_q, d = q.shape
    H = pool.shape[1]
    out, lse = np.zeros(q.shape), np.full((B, H_q, n_q), -np.inf)
    for b in range(B):
        n = int(kv_len[b])
        if n < 0 or n > PAGE * table.shape[1]:
            continue
        K, V = read_rows(pool, table[b], n, d)
        there = ~np.isnan(K[0, :, 0]) if n else np.zeros(0, dtype=bool)
        K, V = K[:, there], V[:, there]
        m = K.shape[1]
        see = np.ones((n_q, m), dtype=bool)
        if k_new is not None:
            K = np.concatenate([K, sanitise(k_new[b]).transpose(1, 0, 2)], 1)
            V = np.concatenate([V, sanitise(v_new[b]).transpose(1, 0, 2)], 1)
            see = np.concatenate([see, visible(k, variant)], 1)
        if not K.shape[1]:
            continue
        for hq in range(H_q):
            h = hq // (H_q // H)
            s = np.where(see, scale * (q[b, :, hq] @ K[h].T), -np.inf)
            top = s.max(1, keepdims=True)
            with np.errstate(invalid="ignore"):
                e = np.exp(s - top)
            den = e.sum(1, keepdims=True)
            out[b, :, hq] = (e @ V[h]) / den
            lse[b, hq] = (np.log(den) + top)[:, 0]
    return out, lse
