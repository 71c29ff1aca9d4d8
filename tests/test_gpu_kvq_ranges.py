"""Attention over the 4-bit cache where its numbers are unusual.  Against the oracle in 64 bits, in every form of the
kernels."""
import math

import numpy as np
import pytest
import torch

from oracle import kvq
from oracle.bf16 import bf16_bits_to_f64, f32_to_bf16_bits
from test_gpu_kvq import B, P, WIDE, bits, check, dev, random_cache, run_attention, span_of  # noqa: F401 (B: a fixture)

pytestmark = pytest.mark.gpu

# G, k, pages per sequence in the table (0: as many as there are): 8, 16, 24-row items full to the last row, 24 and a rest,
# and the tensor-memory form's 64 rows (full, and full with a rest)
FORMS = [(8, 0, 0), (16, 0, 0), (8, 2, 0), (1, 5, 0), (16, 1, WIDE), (2, 6, WIDE)]


def params(pool, d, which):
    """{step, lo} of K (which = 0) or V (1) of every row, [pages, H, 128, 2] in 64 bits; NaN where nothing lives."""
    n = kvq.BLOCK * d + which * 4 * kvq.BLOCK
    mem = pool.reshape(pool.shape[0], pool.shape[1], 4, -1)
    raw = np.ascontiguousarray(mem[..., n:n + 128]).view(np.uint16)
    return bf16_bits_to_f64(raw).reshape(pool.shape[0], pool.shape[1], P, 2)


def set_params(pool, d, which, val):
    n = kvq.BLOCK * d + which * 4 * kvq.BLOCK
    mem = pool.reshape(pool.shape[0], pool.shape[1], 4, -1)
    new = f32_to_bf16_bits(val.astype(np.float32)).reshape(pool.shape[0], pool.shape[1], 4, 64).view(np.uint8)
    there = np.isfinite(val).all(-1).reshape(pool.shape[0], pool.shape[1], 4, kvq.BLOCK).repeat(4, -1)
    mem[..., n:n + 128] = np.where(there, new, mem[..., n:n + 128])


# ------------------------------------------------------------------------------------------------ scores far from zero

@pytest.mark.parametrize("level", [-20000.0, -1000.0, -100.0, -80.0, 1000.0])
@pytest.mark.parametrize("hole", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,k,pps", FORMS)
def test_scores_far_from_zero(B, d, G, k, pps, hole, level):
    """A softmax does not change with a shift of its scores: queries of one sign, keys of one sign, every score near
    `level`, also where the first page of a sequence is not in the pool."""
    rng = np.random.default_rng(31)
    H, lens, n_q = 8, [700, 650, 127, 300, 690, 513, 640, 699], (k + 1) ** 2
    pps = pps or 6
    pool, table = random_cache(rng, lens, H, d, pps)
    kp = params(pool, d, 0)
    step = 0.25 + 0.05 * rng.random(kp.shape[:-1])
    val = np.stack([step, level / math.sqrt(d) - 7.5 * step], -1)
    set_params(pool, d, 0, np.where(np.isfinite(kp), val, np.nan))
    if hole:
        table[:, 0] = -1
    q = f32_to_bf16_bits((1 + 0.2 * rng.standard_normal((len(lens), n_q, G * H, d))).astype(np.float32))
    out, lse, status = run_attention(B, q, pool, table, lens, k, None, None, H, d)
    want, want_lse = kvq.attention(bf16_bits_to_f64(q), pool, table, lens, k, 1 / math.sqrt(d))
    s = np.abs(want_lse[np.isfinite(want_lse)]).max() + 40.0
    # a score is two roundings at its own size (1.45 |score| in units of log2), which the weights follow
    spans = [np.nan_to_num(x) * (1 + 2048 * 8 * 2.0 ** -24 * s) for x in span_of(pool, table, lens, d, None)]
    check(out, lse, want, want_lse, spans, scores=s)
    assert status == [B.ST_BAD_PAGE if hole else 0] * len(lens)


@pytest.mark.parametrize("top", [12, 24, 40, 60])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,k,pps", FORMS)
def test_scores_that_are_large_and_grow(B, d, G, k, pps, top):
    """Pages of K that are up to 2^top as large as others, in any order: a reference is never below the scores it comes from,
    whatever the rounding of their size."""
    rng = np.random.default_rng(36)
    H, lens, n_q = 8, [1500, 1400, 1300, 700, 1500, 33, 128, 1450], (k + 1) ** 2
    pps = pps or 12
    pool, table = random_cache(rng, lens, H, d, pps)
    kp = params(pool, d, 0)
    kp *= 2.0 ** rng.integers(0, top + 1, size=(pool.shape[0], 1, 1, 1))
    set_params(pool, d, 0, kp)
    q = bits(rng, len(lens), n_q, G * H, d)
    kb, vb = bits(rng, len(lens), n_q, H, d, scale=2.0 ** (top // 2)), bits(rng, len(lens), n_q, H, d)
    out, lse, status = run_attention(B, q, pool, table, lens, k, kb, vb, H, d)
    assert not any(status) and np.isfinite(out).all() and np.isfinite(lse).all()
    q64, kb64, vb64, scale = bf16_bits_to_f64(q), bf16_bits_to_f64(kb), bf16_bits_to_f64(vb), 1 / math.sqrt(d)
    want, want_lse = kvq.attention(q64, pool, table, lens, k, scale, kb64, vb64)
    spans, sure = span_of(pool, table, lens, d, vb64), 0
    see = kvq.visible(k)
    for b, L in enumerate(lens):
        K, V = (np.concatenate([x, y[b].transpose(1, 0, 2)], 1) for x, y in zip(kvq.read_rows(pool, table[b], L, d), (kb64, vb64)))
        for hq in range(G * H):
            # a score: sums of 128 products and of a lowest value's, each off by 2^-24 of its terms' sizes
            a, h = q64[b, :, hq], hq // G
            s = np.where(np.concatenate([np.ones((n_q, L), bool), see], 1), scale * (a @ K[h].T), -np.inf)
            off = 128 * 2.0 ** -24 * 4 * scale * np.abs(a).sum(-1) * np.abs(K[h]).max()
            assert (np.abs(lse[b, hq] - want_lse[b, hq]) <= off + 1e-3).all()
            two = np.sort(s, -1)[:, -2:]
            one = two[:, 1] - two[:, 0] > 2 * off + 30                   # one key has all the weight
            sure += one.sum()
            err = np.abs(out[b, one, hq] - V[h][s.argmax(-1)[one]])
            assert (err <= np.abs(want[b, one, hq]) * 2.0 ** -8 + spans[b] * 2.0 ** -11 * 1.5).all(), err.max()
    assert sure > 0


# ------------------------------------------------------------------------------------------------ next to the largest number

@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,k,pps", FORMS + [(4, 0, 0), (4, 3, WIDE)])
def test_infinities_in_cached_rows(B, d, G, k, pps, which):
    """Rows with infinities and the largest numbers, appended (an infinity counts as the largest finite bf16): the outputs
    stay numbers, and are the softmax over what the cache holds."""
    rng = np.random.default_rng(32)
    H, lens, n_q = 2, [400, 300, 40, 333], (k + 1) ** 2
    n, pps = len(lens), pps or 5
    raw = bits(rng, n, 2, 400, H, d)                                     # K, V
    x = raw[:, 0 if which == "k" else 1]
    if which == "k":
        rows = [3, 70, 130, 131, 200, 260]                               # (sequence 2 has the first of them only)
        x[:, 3, :, 5], x[:, 70, :, 9] = 0x7F80, 0xFF80
        x[:, 130, :, 7], x[:, 131, :, 8] = 0x7F7F, 0xFF7F
        x[:, 200, :, ::2] = 0x7F80                                       # in many channels, and with both signs
        x[:, 260, :, ::16], x[:, 260, :, 8::16] = 0xFF80, 0x7F7F
        x[1, rows[1:]] = raw[1, 1, rows[1:]]                             # sequence 1: one element of one row
    else:
        x[:, 10:, :, 3] = 0x7F80                                         # a channel of which nearly every row is an infinity
        x[:, 5, :, 4] = 0xFF80
        x[3, 100:130, :, ::2] = 0x7F7F
    # scores: ordinary queries for V; for K small enough that c |k| |q| stays a number of 32 bits in most rows
    q = bits(rng, n, n_q, G * H, d, scale=2.0 if which == "v" else 0.05)
    pool = B.kvq_pool(n * 4 + 1, H, d)
    pool.fill_(255)
    table = np.full((n, pps), -1, np.int32)
    table[:, :4] = rng.permutation(4 * n).reshape(n, 4)
    ctx = B.Context(max_batch=n, n_q_heads=G * H, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=1 << 14)
    status = torch.zeros(n, dtype=torch.int32, device="cuda")
    kv, dt, count = dev(raw), dev(table), dev(np.array(lens, np.int32))
    ctx.space_kvq_append(ctx.kvq_append_args(kv[:, 0], kv[:, 1], pool, dt, torch.zeros_like(count), count=count, status=status))
    assert (status == B.ST_NONFINITE).all()
    held = pool.cpu().numpy()
    kb, vb = (bits(rng, n, n_q, H, d), bits(rng, n, n_q, H, d)) if k else (None, None)
    if which == "v" and k:
        vb[..., 3] = 0x7F80                                              # and of every row of the block
    out, lse, st = run_attention(B, q, held, table, lens, k, kb, vb, H, d)
    with np.errstate(over="ignore"):
        want, want_lse = kvq.attention(bf16_bits_to_f64(q), held, table, lens, k, 1 / math.sqrt(d),
                                       *((bf16_bits_to_f64(kb), bf16_bits_to_f64(vb)) if k else (None, None)))
    assert not any(st) and np.isfinite(out).all() and np.isfinite(lse).all()
    spans = span_of(held, table, lens, d, bf16_bits_to_f64(vb) if k else None)
    if which == "v":
        check(out, lse, want, want_lse, spans)
        # the other rows' channels: every weight is rounded, and multiplies the row's whole span; the channel itself is a number
        top = np.abs(want[..., 3]).max()
        assert top > 1e38 and (np.abs(out[..., 3] - want[..., 3]) <= 2.0 ** -8 * np.abs(want[..., 3]) + 2.0 ** -10 * max(spans)).all()
        return
    # one key takes the whole softmax of a row, or none of the unusual ones does
    held_to = 6.9e37                                                     # 1e38 in units of log2: larger scores are held to it
    clear = np.abs(want_lse) < held_to
    assert clear.mean() > 0.9 and (np.abs(want_lse) > 1e30).mean() > 0.2 and (np.abs(want_lse) < 100).any()
    rel = np.abs(lse - want_lse) / np.maximum(np.abs(want_lse), 1.0)
    assert rel[clear].max() <= 128 * 2.0 ** -23 * 40                     # (sums of up to 128 products with terms of both signs)
    sel = clear.transpose(0, 2, 1)
    for b in range(n):
        err = np.abs(out[b] - want[b])[sel[b]]
        assert (err <= np.abs(want[b])[sel[b]] * 2.0 ** -8 + spans[b] * 2.0 ** -11 * 1.5).all(), (b, err.max(), spans[b])
    # scores past the largest number: held to it
    out, lse, st = run_attention(B, bits(rng, n, n_q, G * H, d, scale=8.0), held, table, lens, k, kb, vb, H, d)
    assert not any(st) and np.isfinite(out).all() and np.isfinite(lse).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,k,pps", FORMS)
def test_ordinary_rows_behind_rows_far_below(B, d, G, k, pps):
    """The first keys score -1e36, all of them, the ones behind them as usual: those keep their bits."""
    rng = np.random.default_rng(35)
    H, lens, n_q = 8, [1, 130, 400, 650, 700, 257, 131, 690], (k + 1) ** 2
    n, pps = len(lens), pps or 6
    raw = bits(rng, n, 2, 700, H, d)
    raw[:, 0, :130, :, 11] = 0xFF80                                      # the first rows of K, and a few more
    raw[:, 0, 256:256 + 40, :, 11] = 0xFF80
    q = f32_to_bf16_bits((0.3 + 0.05 * rng.standard_normal((n, n_q, G * H, d))).astype(np.float32))
    pool = B.kvq_pool(n * 6 + 1, H, d)
    table = np.full((n, pps), -1, np.int32)
    table[:, :6] = rng.permutation(6 * n).reshape(n, 6)
    ctx = B.Context(max_batch=n, n_q_heads=G * H, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=1 << 14)
    kv, dt, count = dev(raw), dev(table), dev(np.array(lens, np.int32))
    ctx.space_kvq_append(ctx.kvq_append_args(kv[:, 0], kv[:, 1], pool, dt, torch.zeros_like(count), count=count))
    held = pool.cpu().numpy()
    kb, vb = bits(rng, n, n_q, H, d), bits(rng, n, n_q, H, d)
    for block in ((kb, vb), (None, None)):
        out, lse, st = run_attention(B, q, held, table, lens, k, *block, H, d)
        want, want_lse = kvq.attention(bf16_bits_to_f64(q), held, table, lens, k, 1 / math.sqrt(d),
                                       *(None if x is None else bf16_bits_to_f64(x) for x in block))
        assert not any(st)
        # keys that all score -1e36 lie apart by far more than a score's bits or are the same key's; the others are ordinary
        few = np.array(lens) <= 130
        if block[0] is None:
            assert np.isfinite(out).all() and (want_lse[few] < -1e30).all()
            rel = np.abs(lse[few] - want_lse[few]) / np.abs(want_lse[few])
            assert rel.max() <= 128 * 2.0 ** -23 * 40
        rest = ~few if block[0] is None else np.ones(n, bool)
        check(out[rest], lse[rest], want[rest], want_lse[rest],
              [s for s, r in zip(span_of(held, table, lens, d, None if block[0] is None else bf16_bits_to_f64(vb)), rest) if r])


# ------------------------------------------------------------------------------------------------ V far above the others

@pytest.mark.parametrize("factor", [2.0 ** 20, 2.0 ** 30])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,k,pps", [(8, 0, 0), (16, 0, 0), (1, 5, 0), (16, 1, WIDE), (2, 6, WIDE)])
def test_a_page_of_large_values_costs_rows_that_do_not_see_it_nothing(B, d, G, k, pps, factor):
    """Whole pages whose V is far above the rest, which one query row sees and the others hardly: those are as near to
    their values as without such pages."""
    rng = np.random.default_rng(33)
    H, lens, n_q = 8, [1500, 1400, 1300, 1500, 1500, 1100, 1500, 1450], (k + 1) ** 2
    pps = pps or 12
    pool, table = random_cache(rng, lens, H, d, pps)
    large = np.unique(table[:, [1, 6]])
    kp, vp = params(pool, d, 0), params(pool, d, 1)
    kp[large, ..., 0], kp[large, ..., 1] = 2.0 ** -7, 4.0                # keys of these pages: 4 and a little in every channel
    other = np.setdiff1d(np.arange(pool.shape[0]), large)
    there = np.sign(kp[other, ..., 0])                                   # (NaN where nothing lives)
    kp[other, ..., 0], kp[other, ..., 1] = 0.0625 * there, -0.46875 * there
    step = 0.25 + 0.05 * rng.random(vp.shape[:-1])                       # (steps within 2^6 of each other in every page)
    new = np.stack([step, -7.5 * step], -1)
    new[large] *= factor
    set_params(pool, d, 0, kp)
    set_params(pool, d, 1, np.where(np.isfinite(vp), new, np.nan))
    q = rng.standard_normal((len(lens), n_q, G * H, d)) * 0.3 - 1.0      # away from the large pages' keys
    row, head = n_q // 2, np.arange(H) * G + G // 2
    q[:, row, head] *= -0.9                                              # one row of every kv head: towards them
    q = f32_to_bf16_bits(q.astype(np.float32))
    out, lse, status = run_attention(B, q, pool, table, lens, k, None, None, H, d)
    want, want_lse = kvq.attention(bf16_bits_to_f64(q), pool, table, lens, k, 1 / math.sqrt(d))
    assert not any(status) and np.isfinite(out).all()
    sees = np.zeros(out.shape[1:3], bool)
    sees[row, head] = True
    assert np.abs(want[:, sees]).max() > factor / 100 and np.abs(want[:, ~sees]).max() < 10
    for rows, span in ((sees, 6.0 * factor), (~sees, 6.0)):
        err = np.abs(out[:, rows] - want[:, rows])
        assert (err <= np.abs(want[:, rows]) * 2.0 ** -8 + span * 2.0 ** -11 * 1.5).all(), (err.max(), span)
    assert np.abs(lse - want_lse).max() <= 128 * 2.0 ** -23 * (np.abs(want_lse).max() + 40) + 1e-6 * np.abs(want_lse).max()


# ------------------------------------------------------------------------------------------------ V of one sign

@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("d,H,G,k", [(64, 4, 8, 0), (128, 4, 8, 0), (64, 4, 16, 0), (128, 4, 4, 2), (128, 1, 16, 1), (64, 1, 1, 7), (128, 1, 16, 3)])
def test_values_of_one_sign(B, d, H, G, k, sign):
    """Tens of thousands of keys of nearly even weight in few pieces, with V on one side of zero: sums that only grow."""
    rng = np.random.default_rng(34)
    n, L, n_q = 128, 40000, (k + 1) ** 2
    pages = (L + P - 1) // P
    pool, one = random_cache(rng, [L], H, d, pages)
    vp = params(pool, d, 1)
    vp[..., 1] = vp[..., 0] * (2.0 if sign > 0 else -17.0)
    set_params(pool, d, 1, vp)
    table = np.repeat(one, n, 0)                                         # every sequence has the same pages
    q = bits(rng, n, n_q, G * H, d, scale=0.05)
    out, lse, status = run_attention(B, q, pool, table, [L] * n, k, None, None, H, d)
    assert not any(status)
    some = [0, 77, n - 1]
    want, want_lse = kvq.attention(bf16_bits_to_f64(q[some]), pool, table[some], [L] * 3, k, 1 / math.sqrt(d))
    check(out[some], lse[some], want, want_lse, span_of(pool, table[:1], [L], d, None) * 3)
