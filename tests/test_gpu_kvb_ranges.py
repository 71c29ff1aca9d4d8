"""The 8-bit cache where its numbers are unusual: rows next to the largest number, sums that pass it, block rows and query rows far
from one.  Against the oracle in 64 bits, in every form of the attention."""
import math

import numpy as np
import pytest
import torch

from oracle import kvb
from oracle.bf16 import bf16_bits_to_f64, f32_to_bf16_bits
from oracle.kvq import BF16_MAX, sanitise
from test_gpu_kvb import B, FORMS, P, WIDE, bits, check, context, dev, f64, i32, random_cache, run  # noqa: F401 (B: a fixture)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ items that are cut

@pytest.mark.parametrize("one_sign", [True, False])
@pytest.mark.parametrize("up", [100, 112, 126])
@pytest.mark.parametrize("d,k", FORMS)
def test_pieces_of_large_values(B, d, k, up, one_sign):
    """One sequence over all thread blocks, nearly even weights, V 2^up times as large as usual (2^126: up to the largest number that the
    format has): the mean of what the pieces hold, whatever their sums would be."""
    rng = np.random.default_rng(41)
    n_q, lens = (k + 1) ** 2, [3000]
    pool, table = random_cache(rng, lens, 1, d, WIDE if k == 6 else 25)
    for page in table[0, :24]:
        _, v, sc = kvb._views(pool[page, 0], d)
        sc[:, 1] = np.where(np.isnan(sc[:, 1]), sc[:, 1], np.float32(2.0 ** (up - 7)))
        if one_sign:
            v[v != 255] &= 127
    q = bits(rng, 1, n_q, 2, d, scale=0.05)
    out, lse, status = run(B, q, pool, table, lens, k, None, None, 1, d)
    check(out, lse, *kvb.attention(bf16_bits_to_f64(q), pool, table, lens, k, 1 / math.sqrt(d)))
    assert status == [0] and (not one_sign or np.abs(out).max() > 2.0 ** (up - 4))


@pytest.mark.parametrize("lens", [[700, 300, 40], [2500]])
@pytest.mark.parametrize("d,k", FORMS)
def test_infinities_in_appended_rows(B, d, k, lens):
    """V rows with infinities and the largest numbers, appended (an infinity counts as the largest finite bf16): one in a channel, nearly all
    of a channel, and pages of one sign behind pages of the other; pages of large rows that hardly any weight falls on."""
    rng = np.random.default_rng(42)
    n, n_q, most = len(lens), (k + 1) ** 2, max(lens)
    pps = WIDE if k == 6 else most // P + 2
    raw = bits(rng, n, 2, most, 1, d)                                    # K, V
    v = raw[:, 1]
    v[:, 17, :, 5] = 0x7F80                                              # one infinity in a channel
    v[:, 10:, :, 3] = 0x7F80                                             # nearly all of a channel
    at = np.arange(most) // P
    v[:, at % 2 == 0, :, 9], v[:, at % 2 == 1, :, 9] = 0x7F80, 0xFF80    # pages of one sign, then of the other
    v[:, at == 1, :, 32:] = 0xFF7F
    q = bits(rng, n, n_q, 2, d, scale=0.5)
    axis = f32_to_bf16_bits(np.where(np.arange(d) % 2, 1.0, -1.0).astype(np.float32))
    q[..., 1, :] = axis                                                  # the second head: page 1 scores 150 less than zero
    far = f32_to_bf16_bits((bf16_bits_to_f64(axis) * -150.0 / math.sqrt(d)).astype(np.float32))
    raw[:, 0][:, at == 1] = far
    rows = -(-most // P)
    pool, table = B.kvb_pool(n * rows + 1, 1, d), np.full((n, pps), -1, np.int32)
    table[:, :rows] = rng.permutation(n * rows).reshape(n, rows)
    ctx, status, kv, count = context(B, n, 2, 1, d), i32([0] * n), dev(raw), i32(lens)
    ctx.space_kvb_append(ctx.kvb_append_args(kv[:, 0], kv[:, 1], pool, dev(table), i32([0] * n), count=count, status=status))
    assert status.tolist() == [B.ST_NONFINITE] * n
    held = pool.cpu().numpy()
    for block in (True, False):
        kn, vn = (bits(rng, n, n_q, 1, d), bits(rng, n, n_q, 1, d)) if block else (None, None)
        if block:
            vn[..., 3] = 0x7F80
        out, lse, st = run(B, q, held, table, lens, k, kn, vn, 1, d)
        want = kvb.attention(bf16_bits_to_f64(q), held, table, lens, k, 1 / math.sqrt(d),
                             *((bf16_bits_to_f64(kn), bf16_bits_to_f64(vn)) if block else (None, None)))
        assert not any(st) and np.abs(want[0]).max() <= BF16_MAX
        check(out, lse, *want)


# ------------------------------------------------------------------------------------------------ rows next to the largest number

@pytest.mark.parametrize("d", [64, 128])
def test_what_is_read_back_is_finite(B, d):
    """Rows from 2^124 to the largest number and infinities, of both signs, as K and V: read back they are what the codes stand for, finite,
    and appended once more they are held as the same bytes."""
    rng = np.random.default_rng(43)
    n, H = 200, 2
    mag = np.linspace(2.0 ** 124, BF16_MAX, n * 2 * H * d).reshape(1, n, 2, H, d)
    raw = f32_to_bf16_bits((rng.permuted(mag, axis=1) * rng.choice([-1.0, 1.0], mag.shape)).astype(np.float32))
    raw[0, 40, 0, 0, 3], raw[0, 41, 1, 1, 5], raw[0, 150, :, :, 7] = 0x7F80, 0xFF80, 0x7F80
    raw[0, 42, :, :, :8] = np.array([0x7F6F, 0x7F70, 0x7F71, 0x7F77, 0x7F78, 0x7F79, 0x7F7F, 0xFF78], np.uint16)      # around 240 and 248 of 2^120
    x = sanitise(bf16_bits_to_f64(raw))
    table, ctx = np.array([[1, 0, -1]], np.int32), context(B, 1, H, H, d)
    first = np.zeros((2, H, kvb.head_bytes(d)), np.uint8)
    for h in range(H):
        kvb.append(first, table[0], h, 0, x[0, :, 0, h], x[0, :, 1, h])
    kv, status = dev(raw), i32([0])
    for again in (False, True):
        pool = B.kvb_pool(2, H, d)
        ctx.space_kvb_append(ctx.kvb_append_args(kv[:, :, 0], kv[:, :, 1], pool, dev(table), i32([0]), status=status))
        assert (pool.cpu().numpy() == first).all()
        assert status.tolist() == [0 if again else B.ST_NONFINITE]
        out = torch.empty_like(kv)
        status.zero_()
        ctx.space_kvb_read(ctx.kvb_read_args(pool, dev(table), i32([n]), out[:, :, 0], out[:, :, 1]))
        back = f64(out)
        assert np.isfinite(back).all()
        want = kvb.read_rows(first, table[0], n, d)
        assert (back[0, :, 0].transpose(1, 0, 2) == want[0]).all() and (back[0, :, 1].transpose(1, 0, 2) == want[1]).all()
        assert (np.abs(back - x) <= 2.0 ** -4 * np.abs(x)).all()         # (blocks' elements are within 2^4 of the largest: no steps near zero)
        kv = out
    # a block that such a row joins later: its codes of before are rounded once more, and stay below the largest number
    pool, want, kv = B.kvb_pool(2, H, d), np.zeros_like(first), dev(raw)
    rows = np.argsort(np.abs(x[0, :20]).max((1, 2, 3)))
    for i, r in enumerate([*rows, 42]):
        for h in range(H):
            kvb.append(want, table[0], h, i, x[0, r:r + 1, 0, h], x[0, r:r + 1, 1, h])
        ctx.space_kvb_append(ctx.kvb_append_args(kv[:, r:r + 1, 0], kv[:, r:r + 1, 1], pool, dev(table), i32([i])))
    assert (pool.cpu().numpy() == want).all() and np.isfinite(f64(read(B, ctx, pool, table, len(rows) + 1, H, d))).all()


def read(B, ctx, pool, table, n, H, d):
    out = torch.empty(1, n, 2, H, d, dtype=torch.bfloat16, device="cuda")
    ctx.space_kvb_read(ctx.kvb_read_args(pool, dev(table), i32([n]), out[:, :, 0], out[:, :, 1]))
    return out


# ------------------------------------------------------------------------------------------------ block rows and query rows far from one

@pytest.mark.parametrize("q_up,k_up", [(70, 70), (100, 100), (125, 125), (30, 100), (125, 10), (60, 50)])
@pytest.mark.parametrize("d,k", FORMS)
def test_products_beyond_the_largest_number(B, d, k, q_up, k_up):
    """Query rows times 2^q_up, block rows times 2^k_up, signs of all kinds: scores are held to 2^29 (log2 units), so that the keys
    above that, or where there are none all of those below -2^29, count the same."""
    rng = np.random.default_rng(44)
    n_q = (k + 1) ** 2
    pool, table = random_cache(rng, [0, 300], 1, d, WIDE if k == 6 else 3)
    q, kn, vn = bits(rng, 2, n_q, 2, d), bits(rng, 2, n_q, 1, d), bits(rng, 2, n_q, 1, d)
    q, kn = (f32_to_bf16_bits((bf16_bits_to_f64(x) * 2.0 ** up).astype(np.float32)) for x, up in ((q, q_up), (kn, k_up)))
    out, lse, status = run(B, q, pool, table, [0, 300], k, kn, vn, 1, d)
    assert status == [0, 0] and np.isfinite(out).all() and np.isfinite(lse).all()
    assert np.abs(lse).max() <= (2.0 ** 29 + 16) * math.log(2) * (1 + 2.0 ** -20)
    q64, k64, v64, see = bf16_bits_to_f64(q)[0], bf16_bits_to_f64(kn)[0, :, 0], bf16_bits_to_f64(vn)[0, :, 0], kvb.visible(k)
    clear = 0
    for hq in range(2):                                                  # sequence 0: the block's rows alone
        s = q64[:, hq] @ k64.T
        # a score's sign is known where it stands out of what products and their sums are rounded by
        known = (np.abs(s) > 2.0 ** -8 * (np.abs(q64[:, hq]) @ np.abs(k64).T)) | ~see
        for i in np.nonzero(known.all(-1))[0]:
            up = see[i] & (s[i] > 0)
            want = v64[up if up.any() else see[i]].mean(0)
            # even weights, each rounded by 2^-8; rows by 2^-17 of their largest; the output by 2^-8 of itself
            top = np.abs(v64).max()
            assert (np.abs(out[0, i, hq] - want) <= (2.0 ** -8 + 2.0 ** -17 + 2.0 ** -8) * top).all()
            clear += 1
    assert clear > n_q // 2


@pytest.mark.parametrize("q_up,k_up", [(64, -64), (-64, 64), (100, -100), (-90, 90), (30, -30)])
@pytest.mark.parametrize("d,k", FORMS)
def test_products_of_large_and_small_rows(B, d, k, q_up, k_up):
    """Ordinary scores between rows that are far from one."""
    rng = np.random.default_rng(45)
    n_q = (k + 1) ** 2
    pool, table = np.zeros((1, 1, kvb.head_bytes(d)), np.uint8), np.full((2, WIDE if k == 6 else 1), -1, np.int32)
    q, kn, vn = bits(rng, 2, n_q, 2, d), bits(rng, 2, n_q, 1, d), bits(rng, 2, n_q, 1, d)
    q, kn = (f32_to_bf16_bits((bf16_bits_to_f64(x) * 2.0 ** up).astype(np.float32)) for x, up in ((q, q_up), (kn, k_up)))
    out, lse, status = run(B, q, pool, table, [0, 0], k, kn, vn, 1, d)
    check(out, lse, *kvb.attention(bf16_bits_to_f64(q), pool, table, [0, 0], k, 1 / math.sqrt(d), bf16_bits_to_f64(kn), bf16_bits_to_f64(vn)))
    assert status == [0, 0]


@pytest.mark.parametrize("fill", [0x7FC0, 0x7F80, 0xFF80])
@pytest.mark.parametrize("d,k", FORMS)
def test_a_query_row_that_is_not_finite_and_sees_the_block_alone(B, d, k, fill):
    rng = np.random.default_rng(46)
    n_q = (k + 1) ** 2
    pool, table = np.zeros((1, 1, kvb.head_bytes(d)), np.uint8), np.full((2, WIDE if k == 6 else 1), -1, np.int32)
    q, kn, vn = bits(rng, 2, n_q, 2, d), bits(rng, 2, n_q, 1, d), bits(rng, 2, n_q, 1, d)
    base = run(B, q, pool, table, [0, 0], k, kn, vn, 1, d)
    for where in (slice(5, 6), slice(0, d)):
        q2 = q.copy()
        q2[0, n_q // 2, 1, where] = fill
        got = run(B, q2, pool, table, [0, 0], k, kn, vn, 1, d)
        bad = np.zeros((2, n_q, 2), bool)
        bad[0, n_q // 2, 1] = True
        assert np.isnan(got[0][bad]).all() and np.isnan(got[1].transpose(0, 2, 1)[bad]).all()
        assert (got[0][~bad] == base[0][~bad]).all() and (got[1].transpose(0, 2, 1)[~bad] == base[1].transpose(0, 2, 1)[~bad]).all()
