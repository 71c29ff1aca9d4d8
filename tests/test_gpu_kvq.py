"""The 4-bit KV cache on the GPU against its oracle: rows in and out, attention, page moves, refusals."""
import math

import numpy as np
import pytest
import torch

from oracle import kvq
from oracle.bf16 import bf16_bits_to_f64, f32_to_bf16_bits
from oracle.layout import EQ5_LITERAL, SAME_GROUP

pytestmark = pytest.mark.gpu
P = 128
WIDE = 5000                                          # pages of a table that names enough of them for the tensor-memory form (49 to 64 rows, 97 on)


@pytest.fixture(scope="module")
def B():
    from paper_2402_11809_b200 import binding
    return binding


def bits(rng, *shape, scale=1.0):
    return f32_to_bf16_bits((rng.standard_normal(shape) * scale).astype(np.float32))


def dev(a):
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).cuda().view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def f64(t):
    return t.detach().cpu().double().numpy()


def tables(rng, need_rows, pps, extra=2):
    """A shuffled page table for sequences of need_rows rows; unused entries point outside the pool."""
    need = [(n + P - 1) // P for n in need_rows]
    order = rng.permutation(sum(need) + extra)
    t = np.full((len(need), pps), -7, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = order[at:at + n]
        at += n
    return t, sum(need) + extra


def random_cache(rng, lens, H, d, pps, spread=1.0):
    """A pool whose rows below lens are plausible and whose every other byte is 0xFF (NaN steps)."""
    t, n_pages = tables(rng, lens, pps)
    bb = kvq.block_bytes(d)
    pool = np.full((n_pages, H, 4, bb), 255, dtype=np.uint8)
    n = kvq.BLOCK * d
    for b, L in enumerate(lens):
        for j in range((L + P - 1) // P):
            pg = pool[t[b, j]]
            pg[:, :, :n] = rng.integers(0, 256, size=(H, 4, n))
            step = np.abs(rng.standard_normal((H, 4, 2, 32)) * 0.1 + 0.25) * spread
            lo = -7.5 * step + 0.2 * rng.standard_normal(step.shape)
            par = np.stack([f32_to_bf16_bits(step.astype(np.float32)), f32_to_bf16_bits(lo.astype(np.float32))], -1)
            pg[:, :, n:] = par.reshape(H, 4, -1).view(np.uint8)
            for r in range(max(0, L - j * P), P):             # rows past the end: codes and steps of ones
                for which in (0, 1):
                    p0 = n + which * 128 + 4 * (r % 32)
                    pg[:, r // 32, p0:p0 + 4] = 255
    return pool.reshape(n_pages, H, 4 * bb), t


# ------------------------------------------------------------------------------------------------ rows in and out

@pytest.mark.parametrize("d,H,rows,step,lens,counts", [
    (128, 2, 1, 1, [0, 5, 127, 128, 640], [1, 1, 1, 1, 1]),             # one token
    (64, 3, 1, 1, [31, 32, 63, 0], None),
    (128, 4, 25, 5, [0, 100, 126, 380], [1, 5, 3, 4]),                   # the accepted rows of a step, k = 4
    (64, 1, 64, 8, [1, 129], [8, 2]),
    (128, 1, 16, 1, [17, 120], [16, 9]),
    (128, 3, 12, 1, [31, 127], [12, 11]), (64, 2, 13, 1, [31, 127], [13, 12]),   # the most that goes by rows, and one more
    (128, 2, 17, 1, [17, 120, 0], [17, 0, 9]),
    (64, 5, 300, 1, [0, 1, 31, 129, 500], [300, 299, 33, 1, 0]),         # prompts by blocks, odd everything
    (128, 2, 257, 1, [37, 0], [257, 200]),
    (64, 2, 99, 3, [5, 60], [33, 20]),
])
def test_append_and_read(B, d, H, rows, step, lens, counts):
    rng = np.random.default_rng(d + rows + H)
    n = len(lens)
    most = (rows - 1) // step + 1
    cnt = counts or [most] * n
    pps = max((a + c + P - 1) // P for a, c in zip(lens, cnt)) + 1
    table, n_pages = tables(rng, [a + c for a, c in zip(lens, cnt)], pps)
    # K and V as slices of one projection's output (strides of their own)
    raw = bits(rng, n, rows, 2, H, d, scale=1.5)
    raw[0, 0, 0, 0, :] = bits(rng, 1)[0]                                 # a constant row
    raw[0, 0, 1, 0, :] = 0                                               # and one of zeros
    kv = dev(raw)
    before = rng.integers(0, 256, size=(n_pages, H, 4 * kvq.block_bytes(d)), dtype=np.uint8)
    pool, want = dev(before), before.copy()
    x = bf16_bits_to_f64(raw)
    for b in range(n):
        for g in range(cnt[b]):
            for h in range(H):
                s = lens[b] + g
                kvq.write_row(want, table[b, s // P], h, s % P, x[b, g * step, 0, h], x[b, g * step, 1, h])
    ctx = B.Context(max_batch=n, n_q_heads=H, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=1 << 14)
    kv_len = dev(np.array(lens, np.int32))
    out_len, status = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    n0 = ctx.launch_count
    ctx.space_kvq_append(ctx.kvq_append_args(kv[:, :, 0], kv[:, :, 1], pool, dev(table), kv_len, row_step=step,
                                             count=None if counts is None else dev(np.array(counts, np.int32) - 1),
                                             count_bias=1, kv_len_out=out_len, status=status))
    assert ctx.launch_count == n0 + 1
    assert out_len.tolist() == [a + c for a, c in zip(lens, cnt)] and not status.any()
    assert (pool.cpu().numpy() == want).all()                            # every byte, those of other rows included
    # and back, from two rows before on, into a strided place
    first = np.array([a - 2 for a in lens], np.int32)
    m = max(cnt) + 5
    out = torch.full((n, m, H, 2, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    ctx.space_kvq_read(ctx.kvq_read_args(pool, dev(table), out_len, out[:, :, :, 0], out[:, :, :, 1], first=dev(first), status=status))
    got = f64(out)
    for b in range(n):
        for g in range(cnt[b]):
            for which in (0, 1):
                v = kvq.round_bf16(kvq.values(x[b, g * step, which]).astype(np.float32).astype(np.float64))
                assert (got[b, g + 2, :, which] == v).all()
        assert (got[b, cnt[b] + 2:] == 0).all()                          # past the length: zeros
        if lens[b] < 2:
            assert (got[b, :2 - lens[b]] == 0).all()                     # rows below 0
    assert not status.any()


def test_append_special_values(B):
    """NaN, infinities, the largest and the smallest magnitudes, ties."""
    d, H, n = 64, 1, 24
    rng = np.random.default_rng(9)
    raw = bits(rng, 1, n, H, d)
    raw[0, 0, 0, 3], raw[0, 1, 0, 5], raw[0, 2, 0, 7] = 0x7FC1, 0x7F80, 0xFF80
    raw[0, 3, 0, :] = np.where(np.arange(d) % 2, 0x7F7F, 0xFF7F)         # the whole range of bf16
    raw[0, 4, 0, :] = 0x0080                                             # the smallest normal number
    raw[0, 5] = bits(rng, H, d, scale=1e30)
    raw[0, 6] = bits(rng, H, d, scale=1e-25)
    # many ties: halves of an exact step
    for r in range(8, n):
        lo, s = -3.0 + r, 2.0 ** -(r % 5)
        v = lo + s * 0.5 * rng.integers(0, 31, size=d)
        v[0], v[1] = lo, lo + 15 * s
        raw[0, r, 0] = f32_to_bf16_bits(v.astype(np.float32))
    x = bf16_bits_to_f64(raw)
    table = np.zeros((1, 1), np.int32)
    for rows in (n, 8):                                                  # by blocks, and by rows
        pool = torch.zeros(1, H, 4 * kvq.block_bytes(d), dtype=torch.uint8, device="cuda")
        want = pool.cpu().numpy()
        for r in range(rows):
            kvq.write_row(want, 0, 0, r, x[0, r, 0], x[0, n - 1 - r, 0])
        ctx = B.Context(max_batch=1, n_q_heads=H, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=1 << 14)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        k = dev(raw)
        ctx.space_kvq_append(ctx.kvq_append_args(k[:, :rows], dev(raw[:, ::-1].copy())[:, :rows], pool, dev(table),
                                                 torch.zeros(1, dtype=torch.int32, device="cuda"), status=status))
        got = pool.cpu().numpy()
        assert (got == want).all(), np.argwhere(got != want)[:5]
        assert status.item() == B.ST_NONFINITE


def test_append_and_read_leave_bad_sequences_alone(B):
    d, H, n = 128, 2, 5
    rng = np.random.default_rng(3)
    raw = bits(rng, n, 40, H, d)
    for rows in (40, 4):
        pool = torch.full((4, H, 4 * kvq.block_bytes(d)), 170, dtype=torch.uint8, device="cuda")
        table = np.array([[0, 1], [2, 9], [-1, 3], [3, 3], [2, 3]], np.int32)
        lens = [-1, 126, 0, 256 - rows + 1, 2 ** 31 - 1]
        status = torch.zeros(n, dtype=torch.int32, device="cuda")
        out_len = torch.zeros(n, dtype=torch.int32, device="cuda")
        ctx = B.Context(max_batch=n, n_q_heads=H, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=1 << 14)
        k = dev(raw)[:, :rows]
        kv_len = dev(np.array(lens, np.int32))
        ctx.space_kvq_append(ctx.kvq_append_args(k, k, pool, dev(table), kv_len, kv_len_out=out_len, status=status))
        assert status.tolist() == [B.ST_CAPACITY, B.ST_BAD_PAGE, B.ST_BAD_PAGE, B.ST_CAPACITY, B.ST_CAPACITY]
        assert out_len.tolist() == [-1, 126 + rows, rows, lens[3], lens[4]]
        got = pool.cpu().numpy()
        want = np.full(got.shape, 170, dtype=np.uint8)
        x = bf16_bits_to_f64(raw)
        for g in range(2):                                               # rows 126, 127 of sequence 1 have their page
            for h in range(H):
                kvq.write_row(want, 2, h, 126 + g, x[1, g, h], x[1, g, h])
        assert (got == want).all()
        status.zero_()
        o = torch.ones(n, rows, H, d, dtype=torch.bfloat16, device="cuda")
        ctx.space_kvq_read(ctx.kvq_read_args(pool, dev(table), dev(np.array([0, 256, 256, 0, -5], np.int32)), o, o.clone(),
                                             first=dev(np.array([0, 130, 0, 5, 0], np.int32)), status=status))
        assert not o.any() and status.tolist() == [0, B.ST_BAD_PAGE, B.ST_BAD_PAGE, 0, 0]


# ------------------------------------------------------------------------------------------------ attention

def check(out, lse, want, want_lse, spans, scores=40.0):
    """Bounds from the arithmetic: out is rounded to bf16 (2^-9 of itself) once; every weight is rounded to 11 bits, off
    by at most 2^-11 of itself, and multiplies at most 8 steps of a V row or a whole row of the block: 2^-11 of the largest
    |V - centre| <= its span; weights below 2^-14 of the reference's scale are off by 2^-25 of it, 2^9 of which would be
    needed to matter.  Scores are fp32 sums of at most 128 products, each off by 2^-24 of |q||k|."""
    for b in range(out.shape[0]):
        err = np.abs(out[b] - want[b])
        assert np.isfinite(out[b]).all()
        assert (err <= np.abs(want[b]) * 2.0 ** -8 + spans[b] * 2.0 ** -11 * 1.5).all(), (b, err.max(), spans[b])
    fin = np.isfinite(want_lse)
    assert (fin == np.isfinite(lse)).all() and (lse[~fin] == -np.inf).all()
    if fin.any():
        assert np.abs(lse - want_lse)[fin].max() <= 128 * 2.0 ** -23 * scores + 1e-6 * np.abs(want_lse[fin]).max()


def span_of(pool, table, lens, d, v_new):
    out = []
    for b, L in enumerate(lens):
        _, v = kvq.read_rows(pool, table[b], max(L, 0), d)
        m = [np.nanmax(v) - np.nanmin(v)] if v.size else []
        if v_new is not None:
            m.append(2 * np.abs(kvq.sanitise(v_new[b])).max())
        out.append(max(m, default=0.0))
    return out


ATTN = [
    # d, H_kv, G, k, lens, block rows given
    (64, 1, 1, 0, [1], True), (128, 1, 1, 0, [1], False),
    (128, 2, 4, 0, [0, 1, 31, 32, 33, 127, 128, 129, 500], True),
    (64, 3, 1, 0, [0, 7, 64, 1000], False),
    (128, 3, 2, 1, [5, 128, 300], True), (64, 2, 16, 1, [77, 0], True),
    (128, 1, 8, 2, [0, 40, 400], True), (64, 5, 1, 3, [37, 1999], True),
    (128, 4, 1, 4, [128, 260], True), (128, 2, 1, 5, [2048, 1], True),
    (64, 2, 1, 5, [513, 640], True), (128, 1, 4, 5, [777], True),
    (64, 1, 8, 6, [129, 3], True), (128, 2, 8, 6, [600], True),
    (64, 2, 2, 7, [250, 0, 96], True), (128, 1, 16, 7, [300], True), (128, 1, 1, 7, [4000], True),
    (128, 1, 1, 3, [200, 64], False), (64, 1, 4, 7, [1030, 0], False),
    (128, 8, 1, 0, [9000], True), (64, 1, 16, 0, [20000, 3], False),
]


# more than 48 query rows in tables wide enough for the tensor-memory form
ATTN_WIDE = [
    (64, 1, 4, 4, [0, 1, 31, 32, 33, 127, 128, 129], True), (128, 1, 1, 6, [600, 0, 1], True),
    (128, 2, 1, 7, [250, 3000], True), (64, 3, 2, 5, [777, 130, 0], True), (128, 2, 4, 3, [384, 50], True),
    (128, 8, 2, 7, [1999, 37, 1200, 2048, 640], True),                   # several items and many pages per thread block
    (64, 4, 8, 5, [1500, 0, 900], True), (128, 1, 8, 7, [4000], True), (128, 16, 1, 6, [300] * 8, True),
    (64, 4, 2, 7, [3500, 2900, 3100], False), (128, 2, 16, 1, [5000], False), (64, 1, 16, 2, [1030, 0, 128], False),
    (64, 2, 16, 1, [77, 0], True), (64, 3, 4, 4, [777, 130, 0], True), (128, 1, 16, 3, [2300, 0, 128], False),
]
# long lists of pages: every warp's ring goes round several times, items end and begin within a thread block's share
ATTN_LONG = [
    (64, 32, 1, 1, [1500, 1900, 700, 2048, 1, 1300, 2000, 1111], True),  # 8 query rows at a time
    (64, 16, 1, 3, [2000, 1501, 2048, 900, 1999, 0, 1700, 1300], True),  # 16
    (64, 12, 4, 1, [2047, 1500, 1800, 1203, 640, 1290], False),
    (64, 8, 1, 4, [2500, 1501, 2048, 900, 1999, 40], True),              # 24 and a last row
    (128, 8, 4, 2, [1500, 1480, 2001], True),
]


@pytest.mark.parametrize("d,H,G,k,lens,block", ATTN + ATTN_LONG)
def test_attention(B, d, H, G, k, lens, block):
    attention_case(B, d, H, G, k, lens, block)


@pytest.mark.parametrize("d,H,G,k,lens,block", ATTN_WIDE)
def test_attention_in_wide_tables(B, d, H, G, k, lens, block):
    attention_case(B, d, H, G, k, lens, block, WIDE)


def attention_case(B, d, H, G, k, lens, block, pps=0):
    rng = np.random.default_rng(d + 100 * H + 10 * G + k)
    n, n_q, Hq = len(lens), (k + 1) ** 2, H * G
    pps = pps or max(1, max((L + P - 1) // P for L in lens) + 1)
    pool, table = random_cache(rng, lens, H, d, pps)
    qb = bits(rng, n, n_q, Hq + 1, d, scale=2.0)                         # a head more than is used: strided rows
    kb, vb = (bits(rng, n, n_q, H, d), bits(rng, n, n_q, H, d)) if block else (None, None)
    variant, name = ((B.MASK_EQ5_LITERAL, EQ5_LITERAL) if k % 2 else (B.MASK_SAME_GROUP, SAME_GROUP))
    scale = 1 / math.sqrt(d)
    want, want_lse = kvq.attention(bf16_bits_to_f64(qb[:, :, :Hq]), pool, table, lens, k, scale,
                                   bf16_bits_to_f64(kb) if block else None, bf16_bits_to_f64(vb) if block else None, name)
    ctx = B.Context(max_batch=n, n_q_heads=Hq, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=1 << 15)
    out = torch.full((n, n_q, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, Hq, n_q), float("nan"), device="cuda")
    status = torch.zeros(n, dtype=torch.int32, device="cuda")
    keep = [dev(qb), dev(pool), dev(table), dev(np.array(lens, np.int32)), None if kb is None else dev(kb), None if vb is None else dev(vb)]
    a = ctx.kvq_attn_args(keep[0][:, :, :Hq], keep[1], keep[2], keep[3], out, k, scale, k_new=keep[4], v_new=keep[5], lse=lse,
                          status=status, mask_variant=variant)
    ctx.space_kvq_attn_step(a)
    check(f64(out), f64(lse), want, want_lse, span_of(pool, table, lens, d, None if vb is None else bf16_bits_to_f64(vb)))
    assert not status.any()
    # the same bits a second time, also where pieces are joined
    first, first_lse = out.clone(), lse.clone()
    out.fill_(float("nan"))
    ctx.space_kvq_attn_step(a)
    assert torch.equal(first, out) and torch.equal(first_lse, lse)


def run_attention(B, q, pool, table, lens, k, kn=None, vn=None, H=1, d=64):
    n, n_q, Hq = q.shape[:3]
    ctx = B.Context(max_batch=n, n_q_heads=Hq, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=1 << 15)
    out = torch.full((n, n_q, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, Hq, n_q), float("nan"), device="cuda")
    status = torch.zeros(n, dtype=torch.int32, device="cuda")
    keep = [dev(q), dev(pool), dev(table), dev(np.array(lens, np.int32))] + [None if x is None else dev(x) for x in (kn, vn)]
    ctx.space_kvq_attn_step(ctx.kvq_attn_args(keep[0], keep[1], keep[2], keep[3], out, k, 1 / math.sqrt(d), k_new=keep[4],
                                              v_new=keep[5], lse=lse, status=status))
    torch.cuda.synchronize()
    return f64(out), f64(lse), status.tolist()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k,pps", [(1, 3), (5, WIDE), (6, WIDE)])
def test_sequences_that_do_not_fit_and_pages_outside_the_pool(B, d, k, pps):
    rng = np.random.default_rng(4)
    lens, n_q = [300, 40, 300, 50], (k + 1) ** 2
    pool, table = random_cache(rng, lens, 2, d, pps)
    q, kn, vn = bits(rng, 4, n_q, 4, d), bits(rng, 4, n_q, 2, d), bits(rng, 4, n_q, 2, d)
    given = [300, -3, pps * P + 1, 50]
    table[0, 1], table[3, 0] = pool.shape[0], -1
    for block in (True, False):
        kb, vb = (kn, vn) if block else (None, None)
        out, lse, status = run_attention(B, q, pool, table, given, k, kb, vb, 2, d)
        want, want_lse = kvq.attention(bf16_bits_to_f64(q), pool, table, [300, 0, 0, 50], k, 1 / math.sqrt(d),
                                       *((bf16_bits_to_f64(kb), bf16_bits_to_f64(vb)) if block else (None, None)))
        want[1:3], want_lse[1:3] = 0, -np.inf
        check(out, lse, want, want_lse, [30.0] * 4)
        assert status == [B.ST_BAD_PAGE, B.ST_CAPACITY, B.ST_CAPACITY, B.ST_BAD_PAGE]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k,pps", [(2, 2), (5, 2), (5, WIDE), (6, WIDE)])
def test_hidden_rows_have_no_influence(B, d, k, pps):
    """What one block row holds reaches only the rows that see it, whatever it is."""
    rng = np.random.default_rng(6)
    n_q = (k + 1) ** 2
    lens = [200, 0]
    pool, table = random_cache(rng, lens, 1, d, pps)
    q, kn, vn = bits(rng, 2, n_q, 2, d), bits(rng, 2, n_q, 1, d), bits(rng, 2, n_q, 1, d)
    base, base_lse, _ = run_attention(B, q, pool, table, lens, k, kn, vn, 1, d)
    see = kvq.visible(k)
    for fill in (0x7FC0, 0x7F80, 0xFF80, 0x7F7F, 0x0001):                # NaN, infinities, the largest, the smallest
        j = k + 2                                                        # a mask row of group 1
        k2, v2 = kn.copy(), vn.copy()
        k2[:, j, :, :d // 2] = fill
        v2[:, j, :, 1::2] = fill
        out, lse, _ = run_attention(B, q, pool, table, lens, k, k2, v2, 1, d)
        assert np.isfinite(out).all()
        blind = ~see[:, j]
        assert blind.sum() > n_q // 2
        assert (out[:, blind] == base[:, blind]).all() and (lse[:, :, blind] == base_lse[:, :, blind]).all()
        want, want_lse = kvq.attention(bf16_bits_to_f64(q), pool, table, lens, k, 1 / math.sqrt(d), bf16_bits_to_f64(k2), bf16_bits_to_f64(v2))
        for b in range(2):
            top = np.abs(want[b]).max(axis=(1, 2), keepdims=True)
            assert (np.abs(out[b] - want[b]) <= 2.0 ** -8 * np.abs(want[b]) + 2.0 ** -10 * np.maximum(top, 8.0)).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k,pps", [(2, 3), (6, WIDE)])
def test_query_rows_do_not_touch_each_other(B, d, k, pps):
    rng = np.random.default_rng(7)
    lens, n_q = [333], (k + 1) ** 2
    pool, table = random_cache(rng, lens, 1, d, pps)
    q, kn, vn = bits(rng, 1, n_q, 2, d), bits(rng, 1, n_q, 1, d), bits(rng, 1, n_q, 1, d)
    base, base_lse, _ = run_attention(B, q, pool, table, lens, k, kn, vn, 1, d)
    q2 = q.copy()
    q2[0, 1, 0, 3] = 0x7FC0
    q2[0, 4, 1, 9] = 0x7F80
    out, lse, _ = run_attention(B, q2, pool, table, lens, k, kn, vn, 1, d)
    hit = np.zeros((n_q, 2), bool)
    hit[1, 0] = hit[4, 1] = True
    assert np.isnan(out[0][hit]).all() and np.isnan(lse[0].T[hit]).all()
    assert (out[0][~hit] == base[0][~hit]).all() and (lse[0].T[~hit] == base_lse[0].T[~hit]).all()


@pytest.mark.parametrize("spread", [1e-6, 1e-3, 300.0, 1e6])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k,pps", [(1, 4), (4, WIDE)])
def test_value_scales(B, d, spread, k, pps):
    """V rows of other magnitudes, among them rows far larger and far smaller than the rest."""
    rng = np.random.default_rng(8)
    lens, n_q = [400, 90], (k + 1) ** 2
    pool, table = random_cache(rng, lens, 1, d, pps)
    mem = pool.reshape(pool.shape[0], 1, 4, -1)
    n = kvq.BLOCK * d
    par = mem[..., n + 128:].copy().view(np.uint16).reshape(-1, 64)
    val = bf16_bits_to_f64(par) * spread
    val[:, 10:14] *= 1e-4
    val[:, 20:22] *= 50
    ok = np.isfinite(val)
    par[ok] = f32_to_bf16_bits(val.astype(np.float32))[ok]
    mem[..., n + 128:] = par.view(np.uint8).reshape(mem[..., n + 128:].shape)
    q, kn, vn = bits(rng, 2, n_q, 4, d), bits(rng, 2, n_q, 1, d), bits(rng, 2, n_q, 1, d, scale=spread)
    out, lse, _ = run_attention(B, q, pool, table, lens, k, kn, vn, 1, d)
    want, want_lse = kvq.attention(bf16_bits_to_f64(q), pool, table, lens, k, 1 / math.sqrt(d), bf16_bits_to_f64(kn), bf16_bits_to_f64(vn))
    check(out, lse, want, want_lse, span_of(pool, table, lens, d, bf16_bits_to_f64(vn)))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k,pps", [(0, 12), (1, WIDE)])
def test_peaked_and_growing_scores(B, d, k, pps):
    """Scores that grow along the sequence by far more than 2^8 between pages, and fall again."""
    rng = np.random.default_rng(11)
    L = 1500
    pool, table = random_cache(rng, [L], 1, d, pps)
    mem = pool.reshape(pool.shape[0], 1, 4, -1)
    n = kvq.BLOCK * d
    par = mem[..., n:n + 128].copy().view(np.uint16).reshape(pool.shape[0], 4, 64)
    for t in range(12):
        f = [0.1, 1, 4, 10, 2, 0.5, 12, 0.1, 3, 1, 0.2, 5][t]
        v = bf16_bits_to_f64(par[table[0, t]]) * f
        ok = np.isfinite(v)
        par[table[0, t]][ok] = f32_to_bf16_bits(v.astype(np.float32))[ok]
    mem[..., n:n + 128] = par.view(np.uint8).reshape(mem[..., n:n + 128].shape)
    q = bits(rng, 1, (k + 1) ** 2, 16, d, scale=4.0)
    out, lse, _ = run_attention(B, q, pool, table, [L], k, None, None, 1, d)
    want, want_lse = kvq.attention(bf16_bits_to_f64(q), pool, table, [L], k, 1 / math.sqrt(d))
    s = np.abs(want_lse).max()
    # weights follow scores of several hundred: an error of 128 * 2^-23 of that in the exponent
    spans = [x * (1 + 2048 * 128 * 2.0 ** -23 * s) for x in span_of(pool, table, [L], d, None)]
    check(out, lse, want, want_lse, spans, scores=4 * s)


@pytest.mark.parametrize("k,pps", [(0, 6), (3, WIDE)])
def test_other_layers_in_one_allocation_and_past_32_bits(B, k, pps):
    """A pool whose pages are far apart (a layer among many), the last ones beyond 4 GB."""
    d, H, L, n_q = 128, 2, 700, (k + 1) ** 2
    rng = np.random.default_rng(12)
    small, table = random_cache(rng, [L], H, d, pps)
    head = small.shape[2]
    page_stride = 800_000_000 // 16 * 16
    big = torch.empty((small.shape[0] - 1) * page_stride + H * (head + 48), dtype=torch.uint8, device="cuda")
    pool = big.as_strided((small.shape[0], H, head), (page_stride, head + 48, 1))
    pool.copy_(dev(small))
    q = bits(rng, 1, n_q, 8, d)
    ctx = B.Context(max_batch=1, n_q_heads=8, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=1 << 14)
    out, status = torch.zeros(1, n_q, 8, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.zeros(1, 8, n_q, device="cuda")
    dt, dl, dq = dev(table), dev(np.array([L], np.int32)), dev(q)
    ctx.space_kvq_attn_step(ctx.kvq_attn_args(dq, pool, dt, dl, out, k, 0.1, lse=lse, status=status))
    want, want_lse = kvq.attention(bf16_bits_to_f64(q), small, table, [L], k, float(np.float32(0.1)))
    check(f64(out), f64(lse), want, want_lse, span_of(small, table, [L], d, None))
    # rows behind them, read back, and the pages copied where they stand
    new = bits(rng, 1, 20, H, d)
    kv = dev(new)
    out_len = torch.zeros_like(dl)
    ctx.space_kvq_append(ctx.kvq_append_args(kv, kv, pool, dt, dl, kv_len_out=out_len, status=status))
    back = torch.zeros(1, 20, H, d, dtype=torch.bfloat16, device="cuda")
    ctx.space_kvq_read(ctx.kvq_read_args(pool, dt, out_len, back, back.clone(), first=dl, status=status))
    assert (f64(back)[0] == kvq.round_bf16(kvq.values(bf16_bits_to_f64(new[0])).astype(np.float32).astype(np.float64))).all()
    free = [p for p in range(small.shape[0]) if p not in set(table[0].tolist())]
    assert len(free) == 2 and not status.any()
    B.space_pages_copy(B.page_pools([pool]), [[int(table[0, 5]), free[0], 128], [int(table[0, 0]), free[1], 33]])
    assert torch.equal(pool[free[0]], pool[int(table[0, 5])])
    assert torch.equal(pool[free[1]][:, :head // 2], pool[int(table[0, 0])][:, :head // 2])
    assert (pool[free[1]][:, head // 2:] == 255).all()


def test_streams_and_graphs(B):
    """On a stream of its own, and captured: append, attention over what it wrote, read."""
    d, H, G, k = 128, 2, 2, 2
    rng = np.random.default_rng(13)
    lens = np.array([130, 7], np.int32)
    pool, table = random_cache(rng, lens, H, d, 3)
    n_q = (k + 1) ** 2
    s = torch.cuda.Stream()
    ctx = B.Context(max_batch=2, n_q_heads=H * G, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=1 << 14)
    q, kn, vn = (dev(bits(rng, 2, n_q, h, d)) for h in (H * G, H, H))
    dp, dt, dl = dev(pool), dev(table), dev(lens)
    acc = dev(np.array([2, 0], np.int32))
    out, out2 = (torch.zeros(2, n_q, H * G, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    new_len = torch.zeros_like(dl)
    torch.cuda.synchronize()

    def step():
        ctx.space_kvq_attn_step(ctx.kvq_attn_args(q, dp, dt, dl, out, k, 0.09, k_new=kn, v_new=vn))
        ctx.space_kvq_append(ctx.kvq_append_args(kn, vn, dp, dt, dl, count=acc, count_bias=1, row_step=k + 1, kv_len_out=new_len))
        ctx.space_kvq_attn_step(ctx.kvq_attn_args(q, dp, dt, new_len, out2, k, 0.09))

    with torch.cuda.stream(s):
        step()
    s.synchronize()
    a, b = out.clone(), out2.clone()
    want, _ = kvq.attention(f64(q), dp.cpu().numpy(), table, [133, 8], k, float(np.float32(0.09)))
    assert np.abs(f64(b) - want).max() < 0.03 and new_len.tolist() == [133, 8]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    out.zero_(), out2.zero_(), new_len.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, a) and torch.equal(out2, b) and new_len.tolist() == [133, 8]


# ------------------------------------------------------------------------------------------------ page moves

@pytest.mark.parametrize("kind,H,d,layers,n_moves,rows", [
    ("kvq", 2, 128, 3, 5, (1, 128)), ("kvq", 1, 64, 1, 1, (33, 33)), ("bf16", 3, 64, 4, 40, (0, 128)),
    ("bf16", 8, 128, 40, 3, (1, 20)), ("kvq", 1, 64, 2, 1500, (1, 128)), ("bf16", 1, 64, 1, 130, (128, 128)),
])
def test_pages_copy(B, kind, H, d, layers, n_moves, rows):
    rng = np.random.default_rng(n_moves)
    n = 2 * n_moves + 3
    if kind == "kvq":
        pools = [torch.randint(0, 256, (n, H, 4 * kvq.block_bytes(d)), dtype=torch.uint8, device="cuda") for _ in range(layers)]
        group = 32
    else:
        pools = [torch.randint(0, 1 << 15, (n, H, P, d), dtype=torch.int16, device="cuda").view(torch.bfloat16) for _ in range(layers)]
        group = 1
    order = rng.permutation(n)
    moves = np.stack([order[:n_moves], order[n_moves:2 * n_moves], rng.integers(rows[0], rows[1] + 1, n_moves)], 1).astype(np.int32)
    raw = [p.view(torch.uint8).cpu().numpy().reshape(n, H, -1) for p in pools]
    B.space_pages_copy(B.page_pools(pools), moves)
    for p, r in zip(pools, raw):
        want = r.copy()
        for s, t, m in moves:
            e = (m + group - 1) // group * group * (r.shape[2] // P)
            want[t, :, :e] = r[s, :, :e]
        assert (p.view(torch.uint8).cpu().numpy().reshape(want.shape) == want).all()


def test_forked_sequences_decode_as_separate_ones(B):
    """Two samples forked from one prompt, their own tokens behind it, then a compacted pool: reads as if each had a cache
    of its own."""
    d, H = 64, 2
    rng = np.random.default_rng(20)
    prompt = bits(rng, 1, 200, H, d)
    tails = bits(rng, 2, 90, H, d)
    pool = B.kvq_pool(12, H, d)
    pg = B.Pager(12, 4, 4)
    ctx = B.Context(max_batch=2, n_q_heads=H, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=512)

    def append(slots, rows, first):
        t, x, n = dev(pg.batch_table(slots)), dev(rows), dev(np.array(first, np.int32))
        ctx.space_kvq_append(ctx.kvq_append_args(x, x, pool, t, n))
        torch.cuda.synchronize()

    junk = pg.admit()
    pg.reserve(junk, 3 * P)
    a = pg.admit()
    pg.reserve(a, 200)
    append([a], prompt, [0])
    b = pg.fork(a, 200)
    for s in (a, b):
        pg.reserve(s, 290)
        B.space_pages_copy(B.page_pools([pool]), pg.make_writable(s, 200, 90))
    append([a, b], tails, [200, 200])
    pg.release(junk)
    moves = pg.compact()
    assert len(moves) == 3
    B.space_pages_copy(B.page_pools([pool]), moves)
    out = torch.zeros(2, 290, H, d, dtype=torch.bfloat16, device="cuda")
    ctx.space_kvq_read(ctx.kvq_read_args(pool, dev(pg.batch_table([a, b])), dev(np.array([290, 290], np.int32)), out, out.clone()))
    for i in range(2):
        x = bf16_bits_to_f64(np.concatenate([prompt[0], tails[i]], 0))
        assert (f64(out[i]) == kvq.round_bf16(kvq.values(x).astype(np.float32).astype(np.float64))).all()
    assert pg.page_refs(0) in (1, 2) and pg.free_pages == 7
    pg.close()


# ------------------------------------------------------------------------------------------------ refusals

def test_refusals(B):
    d, H = 64, 2
    ctx = B.Context(max_batch=2, n_q_heads=4, n_kv_heads=H, head_dim=d, k_max=3, vocab=8, s_cap=512)
    pool = B.kvq_pool(4, H, d)
    table = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    kv = torch.zeros(2, 16, H, d, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(2, 16, 4, d, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    n0 = ctx.launch_count

    def refuse(make, call, code, **change):
        a = make()
        for name, v in change.items():
            o = a.cache if name in ("pool", "page_stride", "head_stride", "page_table", "pages_per_seq", "n_pages") else a
            setattr(o, name, v)
        with pytest.raises(B.SpaceError) as e:
            call(a)
        assert e.value.code == code, change

    attn = lambda: ctx.kvq_attn_args(q, pool, table, lens, out, 3, 0.1, k_new=kv, v_new=kv)
    app = lambda: ctx.kvq_append_args(kv, kv, pool, table, lens)
    read = lambda: ctx.kvq_read_args(pool, table, lens, kv, kv.clone())
    all3 = ((attn, ctx.space_kvq_attn_step), (app, ctx.space_kvq_append), (read, ctx.space_kvq_read))
    for make, call in all3:
        for change in (dict(pool=None), dict(page_table=None), dict(pages_per_seq=0), dict(pages_per_seq=1 << 24), dict(n_pages=0),
                       dict(kv_len=None), dict(head_stride=16), dict(page_stride=16)):
            refuse(make, call, B.E_INVALID_ARG, **change)
        for change in (dict(pool=pool.data_ptr() + 8), dict(page_stride=pool.stride(0) + 8), dict(head_stride=pool.stride(1) + 4)):
            refuse(make, call, B.E_ALIGNMENT, **change)
        refuse(make, call, B.E_WORKSPACE, batch=3)
        refuse(make, call, B.E_WORKSPACE, batch=-1)
    for change in (dict(k=-1), dict(mask_variant=2), dict(q=None), dict(out=None), dict(scale=0.0), dict(scale=float("nan")),
                   dict(k_new=None), dict(v_new=None)):
        refuse(attn, ctx.space_kvq_attn_step, B.E_INVALID_ARG, **change)
    refuse(attn, ctx.space_kvq_attn_step, B.E_WORKSPACE, k=4)
    for change in (dict(q=q.data_ptr() + 2), dict(out=out.data_ptr() + 8), dict(q_stride_r=12), dict(new_stride_h=4),
                   dict(k_new=kv.data_ptr() + 8)):
        refuse(attn, ctx.space_kvq_attn_step, B.E_ALIGNMENT, **change)
    for change in (dict(rows=-1), dict(rows=0), dict(row_step=0), dict(k_new=None), dict(v_new=None), dict(kv_len_out=lens.data_ptr())):
        refuse(app, ctx.space_kvq_append, B.E_INVALID_ARG, **change)
    refuse(app, ctx.space_kvq_append, B.E_ALIGNMENT, new_stride_b=100)
    for change in (dict(rows=-1), dict(k_out=None), dict(v_out=None)):
        refuse(read, ctx.space_kvq_read, B.E_INVALID_ARG, **change)
    refuse(read, ctx.space_kvq_read, B.E_ALIGNMENT, out_stride_r=9)
    for lib_call in (B.lib.space_kvq_attn_step, B.lib.space_kvq_append, B.lib.space_kvq_read):
        assert lib_call(None, None, None) == B.E_INVALID_ARG and lib_call(ctx._h, None, None) == B.E_INVALID_ARG
    assert ctx.launch_count == n0
    # a list of pages that does not fit 32 bits
    big = B.Context(max_batch=16, n_q_heads=4, n_kv_heads=4, head_dim=d, k_max=7, vocab=8, s_cap=512)
    bq = torch.zeros(16, 64, 4, d, dtype=torch.bfloat16, device="cuda")
    bp, bt, bl = B.kvq_pool(1, 4, d), torch.zeros(16, 1, dtype=torch.int32, device="cuda"), torch.zeros(16, dtype=torch.int32, device="cuda")
    a = big.kvq_attn_args(bq, bp, bt, bl, torch.empty_like(bq), 7, 0.1)
    a.cache.pages_per_seq = 1 << 23
    with pytest.raises(B.SpaceError) as e:
        big.space_kvq_attn_step(a)
    assert e.value.code == B.E_UNSUPPORTED and big.launch_count == 0
    a = attn()
    a.batch = 0
    ctx.space_kvq_attn_step(a)
    assert ctx.launch_count == n0
    assert B.kvq_page_bytes(2, 64) == 2 * 4 * (32 * 64 + 256) and B.kvq_page_bytes(2, 96) == 0 and B.kvq_page_bytes(0, 64) == 0


def test_page_move_refusals(B):
    pool = torch.zeros(6, 2, P, 64, dtype=torch.bfloat16, device="cuda")

    def refuse(code, moves, **change):
        d = B.page_pools([pool, pool.clone()])
        for name, v in change.items():
            setattr(d[1], name, v)
        with pytest.raises(B.SpaceError) as e:
            B.space_pages_copy(d, moves)
        assert e.value.code == code, (moves, change)

    good = [[0, 1, 5]]
    for moves in ([[0, 6, 1]], [[-1, 2, 1]], [[0, 1, 129]], [[0, 1, -1]], [[0, 1, 1], [2, 1, 1]], [[0, 1, 1], [1, 2, 1]], [[3, 3, 1]]):
        refuse(B.E_INVALID_ARG, moves)
    refuse(B.E_INVALID_ARG, [[4, 5, 1]], n_pages=5)
    for change in (dict(base=None), dict(parts=0), dict(group_rows=0), dict(group_rows=3), dict(group_bytes=0), dict(n_pages=0),
                   dict(part_stride=16), dict(page_stride=16)):
        refuse(B.E_INVALID_ARG, good, **change)
    for change in (dict(base=pool.data_ptr() + 2), dict(page_stride=pool.stride(0) * 2 + 8), dict(part_stride=pool.stride(1) * 2 + 8),
                   dict(group_bytes=24)):
        refuse(B.E_ALIGNMENT, good, **change)
    B.space_pages_copy(B.page_pools([pool]), np.zeros((0, 3), np.int32))
    B.space_pages_copy(B.page_pools([pool]), [[0, 1, 0]])
    assert B.lib.space_pages_copy(None, 1, None, 0, None) == B.E_INVALID_ARG
    assert not pool.any()


def test_struct_sizes(B):
    import ctypes
    import os
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ["space_kvq_cache", "space_kvq_append_args", "space_kvq_read_args", "space_kvq_attn_args", "space_page_pool", "space_page_move"]
    src = '#include <stdio.h>\n#include "space.h"\nint main(void){ printf("' + "%zu " * len(names) + '\\n", ' + \
          ", ".join(f"sizeof({n})" for n in names) + "); return 0; }\n"
    with tempfile.TemporaryDirectory() as t:
        open(os.path.join(t, "t.c"), "w").write(src)
        subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(root, "include"), os.path.join(t, "t.c"), "-o", os.path.join(t, "t")])
        out = subprocess.check_output([os.path.join(t, "t")]).decode().split()
    assert [int(x) for x in out] == [ctypes.sizeof(x) for x in (B.KvqCache, B.KvqAppendArgs, B.KvqReadArgs, B.KvqAttnArgs, B.PagePool, B.PageMove)]
