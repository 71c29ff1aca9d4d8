"""The 8-bit KV cache on the GPU against its oracle: rows in and out, attention, page moves, refusals."""
import math

import numpy as np
import pytest
import torch

from oracle import kvb
from oracle.bf16 import bf16_bits_to_f64, f32_to_bf16_bits
from oracle.kvq import sanitise
from oracle.layout import EQ5_LITERAL, SAME_GROUP

pytestmark = pytest.mark.gpu
P = 128


@pytest.fixture(scope="module")
def B():
    from paper_2402_11809_b200 import binding
    return binding


def bits(rng, *shape, scale=1.0):
    return f32_to_bf16_bits((rng.standard_normal(shape) * scale).astype(np.float32))


def dev(a):
    if a.dtype == np.uint16:
        return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda().view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def f64(t):
    return t.detach().cpu().double().numpy()


def i32(x):
    return dev(np.array(x, np.int32))


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


def random_cache(rng, lens, H, d, pps, spread=0.0):
    """A pool whose rows below lens are random codes under random powers of two; every other byte is 0xFF (codes and scales of
    NaN), the scales of a block that has rows excepted."""
    t, n_pages = tables(rng, lens, pps)
    pool = np.full((n_pages, H, kvb.head_bytes(d)), 255, dtype=np.uint8)
    codes = rng.integers(0, 127, size=(P, d)).astype(np.uint8)
    for b, L in enumerate(lens):
        for j in range((L + P - 1) // P):
            m = min(P, L - j * P)
            for h in range(H):
                kc, vc, sc = kvb._views(pool[t[b, j], h], d)
                for which, c in ((0, kc), (1, vc)):
                    x = rng.permutation(codes.reshape(-1)).reshape(P, d) | (128 * rng.integers(0, 2, size=(P, d))).astype(np.uint8)
                    if which == 0:
                        c[:, :m] = x[:m].reshape(m, d // 16, 16).transpose(1, 0, 2)
                    else:
                        for i in range(m):
                            c[i // 16, :, i % 16] = x[i]
                    e = -7 + np.round(spread * rng.standard_normal(4))
                    sc[:(m + 31) // 32, which] = (2.0 ** e)[:(m + 31) // 32]
    return pool, t


def context(B, n, Hq, H, d, **more):
    return B.Context(max_batch=n, n_q_heads=Hq, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=1 << 14, **more)


# ------------------------------------------------------------------------------------------------ rows in and out

APPEND = [
    (128, 2, 1, 1, [0, 5, 127, 128, 640], [1, 1, 1, 1, 1]),              # one token
    (64, 3, 1, 1, [31, 32, 63, 0], None),
    (128, 4, 25, 5, [0, 100, 126, 380], [1, 5, 3, 4]),                   # the accepted rows of a step, k = 4
    (64, 1, 64, 8, [1, 129], [8, 2]),
    (128, 1, 16, 1, [17, 120], [16, 9]),
    (128, 2, 17, 1, [17, 120, 0], [17, 0, 9]),
    (64, 5, 300, 1, [0, 1, 31, 129, 500], [300, 299, 33, 1, 0]),         # prompts, odd everything
    (128, 2, 257, 1, [37, 0], [257, 200]),
    (64, 2, 99, 3, [5, 60], [33, 20]),
]


@pytest.mark.parametrize("rot", [0, 1, 2])
@pytest.mark.parametrize("d,H,rows,step,lens,counts", APPEND)
def test_append_and_read(B, d, H, rows, step, lens, counts, rot):
    """rot 0: as they are; 1: turned by halves of all channels, queries too, positions given; 2: neighbours, 32 channels, cache rows."""
    rng = np.random.default_rng(d + rows + H + 1000 * rot)
    n, Hq = len(lens), 2 * H
    most = (rows - 1) // step + 1
    cnt = counts or [most] * n
    pps = max((a + c + P - 1) // P for a, c in zip(lens, cnt)) + 1
    table, n_pages = tables(rng, [a + c for a, c in zip(lens, cnt)], pps)
    raw = bits(rng, n, rows, 2, H, d, scale=1.5)                         # K and V as slices of one projection's output
    raw[0, 0, 0, 0, :] = 0
    raw[:, rows // 2] = bits(rng, n, 2, H, d, scale=40.0)                # some blocks' powers of two are raised
    kv, q = dev(raw), bits(rng, n, rows, Hq, d)
    qd, before = dev(q), rng.integers(0, 256, size=(n_pages, H, kvb.head_bytes(d)), dtype=np.uint8)
    want = before.copy()
    x = bf16_bits_to_f64(raw)
    # what is there already: rows of one append, whose codes may be rounded once more
    for b in range(n):
        old = bf16_bits_to_f64(bits(rng, lens[b], 2, H, d))
        for h in range(H):
            if lens[b]:
                kvb.append(want, table[b], h, 0, old[:, 0, h], old[:, 1, h])
    pool = dev(want)
    n_pos = max(lens) + rows - 3                                         # (the longest sequence runs out of positions)
    angles = rng.standard_normal((n_pos, (d if rot == 1 else 32) // 2)) * 3
    angle_rows = np.concatenate([np.cos(angles), np.sin(angles)], 1).astype(np.float32)
    pos = rng.integers(-2, n_pos + 2, size=(n, rows)).astype(np.int32) if rot == 1 else None
    rope = B.rope(dev(angle_rows), interleaved=rot == 2, pos=None if pos is None else dev(pos)) if rot else None
    q_want, turned, bad_pos = bf16_bits_to_f64(q), np.empty_like(x[:, :, 0]), np.zeros(n, bool)
    for b in range(n):
        src = np.arange(cnt[b]) * step
        at = lens[b] + np.arange(cnt[b]) if pos is None else pos[b, src]
        k = x[b, src, 0]
        if rot:
            bad_pos[b] = ((at < 0) | (at >= n_pos)).any()
            k = kvb.turn(k, angle_rows, at, rot == 2).astype(np.float64)
            q_want[b, src] = bf16_bits_to_f64(f32_to_bf16_bits(kvb.turn(q_want[b, src], angle_rows, at, rot == 2)))
        turned[b, :cnt[b]] = k
        for h in range(H):
            if cnt[b]:
                kvb.append(want, table[b], h, lens[b], k[:, h], x[b, src, 1, h])
    ctx = context(B, n, Hq, H, d)
    out_len, status = i32([0] * n), i32([0] * n)
    n0 = ctx.launch_count
    ctx.space_kvb_append(ctx.kvb_append_args(kv[:, :, 0], kv[:, :, 1], pool, dev(table), i32(lens), row_step=step,
                                             count=None if counts is None else i32(np.array(counts) - 1), count_bias=1, kv_len_out=out_len,
                                             status=status, rope=rope, **(dict(q=qd, q_out=qd) if rot else {})))
    assert ctx.launch_count == n0 + 1
    assert out_len.tolist() == [a + c for a, c in zip(lens, cnt)]
    assert status.tolist() == [B.ST_BAD_POSITION if p else 0 for p in bad_pos]
    got = pool.cpu().numpy()
    assert (got == want).all(), np.argwhere(got != want)[:5]             # every byte, those of other rows included
    assert (f64(qd) == q_want).all()
    # and back, from two rows before on, into a strided place
    first = np.array([a - 2 for a in lens], np.int32)
    m = max(cnt) + 5
    out = torch.full((n, m, H, 2, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    status.zero_()
    ctx.space_kvb_read(ctx.kvb_read_args(pool, dev(table), out_len, out[:, :, :, 0], out[:, :, :, 1], first=dev(first), status=status))
    back = f64(out)
    for b in range(n):
        K, V = kvb.read_rows(want, table[b], lens[b] + cnt[b], d)
        for g in range(m):
            s = lens[b] - 2 + g
            for which, v in ((0, K), (1, V)):
                assert (back[b, g, :, which] == (v[:, s] if 0 <= s < lens[b] + cnt[b] else 0)).all()      # (bf16 holds every code times its power)
    assert not status.any()


@pytest.mark.parametrize("d", [64, 128])
def test_a_later_row_raises_its_blocks_power(B, d):
    """Rows one at a time into one block, each larger or smaller than the ones before; the block beside it stays as it is."""
    rng = np.random.default_rng(d)
    n = 40
    raw = bits(rng, 1, n, 1, d)
    for i, e in enumerate(rng.integers(-30, 30, size=n)):
        raw[0, i] = f32_to_bf16_bits((bf16_bits_to_f64(raw[0, i]) * 2.0 ** e).astype(np.float32))
    raw[0, 33] = 0
    x = bf16_bits_to_f64(raw)
    pool, table = torch.zeros(1, 1, kvb.head_bytes(d), dtype=torch.uint8, device="cuda"), np.zeros((1, 1), np.int32)
    want = pool.cpu().numpy()
    ctx, k, v = context(B, 1, 1, 1, d), dev(raw), dev(raw[:, ::-1])
    for i in range(n):
        kvb.append(want, table[0], 0, i, x[0, i], x[0, n - 1 - i])
        ctx.space_kvb_append(ctx.kvb_append_args(k[:, i:i + 1], v[:, i:i + 1], pool, dev(table), i32([i])))
        got = pool.cpu().numpy()
        assert (got == want).all(), (i, np.argwhere(got != want)[:5])
    # a block whose first row is written anew starts over
    for i in (0, 1):
        kvb.append(want, table[0], 0, i, x[0, i] * 2.0 ** -40, x[0, i] * 2.0 ** -40)
        small = dev(f32_to_bf16_bits((x[:, i:i + 1] * 2.0 ** -40).astype(np.float32)))
        ctx.space_kvb_append(ctx.kvb_append_args(small, small, pool, dev(table), i32([i])))
    assert (pool.cpu().numpy() == want).all()


def test_append_special_values(B):
    """NaN, infinities, the largest and the smallest magnitudes, ties, and the largest numbers turned into one."""
    d, H, n = 64, 1, 128
    rng = np.random.default_rng(9)
    raw = bits(rng, 1, n, H, d)
    raw[0, 0, 0, 3], raw[0, 33, 0, 5], raw[0, 65, 0, 7] = 0x7FC1, 0x7F80, 0xFF80
    raw[0, 34, 0, :] = np.where(np.arange(d) % 2, 0x7F7F, 0xFF7F)
    raw[0, 1, 0, :] = 0x0080                                             # the smallest normal number, and one that is not
    raw[0, 2, 0, :] = 0x0001
    for r in range(96, n):                                               # ties: halves of a code's step
        raw[0, r, 0] = f32_to_bf16_bits((rng.integers(-31, 32, size=d) * 0.5 * 2.0 ** -(r % 5)).astype(np.float32))
    raw[0, 127, 0, 0] = f32_to_bf16_bits(np.float32([448.0]))[0]
    x = sanitise(bf16_bits_to_f64(raw))
    pool, table = torch.zeros(1, H, kvb.head_bytes(d), dtype=torch.uint8, device="cuda"), np.zeros((1, 1), np.int32)
    want = pool.cpu().numpy()
    kvb.append(want, table[0], 0, 0, x[0, :, 0], x[0, ::-1, 0])
    ctx, status = context(B, 1, H, H, d), i32([0])
    ctx.space_kvb_append(ctx.kvb_append_args(dev(raw), dev(raw[:, ::-1]), pool, dev(table), i32([0]), status=status))
    got = pool.cpu().numpy()
    assert (got == want).all(), np.argwhere(got != want)[:5]
    assert status.item() == B.ST_NONFINITE
    # turned by 45 degrees the largest numbers pass the largest: held to it
    c = np.float32(math.cos(math.pi / 4))
    rope = B.rope(dev(np.full((1, 64), c, np.float32)), pos=i32([[0] * n]))
    turned = np.clip(kvb.turn(x[0, :, 0], np.full((1, 64), c), np.zeros(n, int)).astype(np.float64), -kvb.BF16_MAX, kvb.BF16_MAX)
    kvb.append(want, table[0], 0, 0, turned[:, None][:, 0], x[0, ::-1, 0])
    ctx.space_kvb_append(ctx.kvb_append_args(dev(raw), dev(raw[:, ::-1]), pool, dev(table), i32([0]), status=status, rope=rope))
    assert (pool.cpu().numpy() == want).all()


def test_append_and_read_leave_bad_sequences_alone(B):
    d, H, n = 128, 2, 5
    rng = np.random.default_rng(3)
    raw = bits(rng, n, 40, H, d)
    for rows in (40, 4):
        pool = torch.full((4, H, kvb.head_bytes(d)), 0, dtype=torch.uint8, device="cuda")
        table = np.array([[0, 1], [2, 9], [-1, 3], [3, 3], [2, 3]], np.int32)
        lens = [-1, 126, 0, 256 - rows + 1, 2 ** 31 - 1]
        status, out_len = i32([0] * n), i32([0] * n)
        ctx = context(B, n, H, H, d)
        k = dev(raw)[:, :rows]
        q = dev(raw)[:, :rows]
        rope = B.rope(B.rope_table(4, 64), pos=torch.zeros(n, rows, dtype=torch.int32, device="cuda"))       # (position 0: nothing turns)
        q_out = torch.full_like(q, 7)
        ctx.space_kvb_append(ctx.kvb_append_args(k, k, pool, dev(table), i32(lens), kv_len_out=out_len, status=status, rope=rope, q=q, q_out=q_out))
        assert status.tolist() == [B.ST_CAPACITY, B.ST_BAD_PAGE, B.ST_BAD_PAGE, B.ST_CAPACITY, B.ST_CAPACITY]
        assert out_len.tolist() == [-1, 126 + rows, rows, lens[3], lens[4]]
        assert torch.equal(q_out[1:3], q[1:3]) and (q_out[[0, 3, 4]] == 7).all()
        want = np.zeros(tuple(pool.shape), np.uint8)
        x = bf16_bits_to_f64(raw)
        for h in range(H):                                               # rows 126, 127 of sequence 1 have their page
            kvb.append(want, table[1], h, 126, x[1, :2, h], x[1, :2, h])
        assert (pool.cpu().numpy() == want).all()
        status.zero_()
        o = torch.ones(n, rows, H, d, dtype=torch.bfloat16, device="cuda")
        ctx.space_kvb_read(ctx.kvb_read_args(pool, dev(table), i32([0, 256, 256, 0, -5]), o, o.clone(), first=i32([0, 130, 0, 5, 0]), status=status))
        assert not o.any() and status.tolist() == [0, B.ST_BAD_PAGE, B.ST_BAD_PAGE, 0, 0]


def test_nothing_to_do(B):
    ctx, d = context(B, 2, 2, 1, 64), 64
    pool, table = torch.full((2, 1, kvb.head_bytes(d)), 3, dtype=torch.uint8, device="cuda"), i32([[0], [1]])
    k = dev(bits(np.random.default_rng(0), 2, 3, 1, d))
    out_len = i32([9, 9])
    ctx.space_kvb_append(ctx.kvb_append_args(k, k, pool, table, i32([5, 128]), count=i32([0, -4]), kv_len_out=out_len))
    assert out_len.tolist() == [5, 128] and (pool == 3).all()
    ctx.space_kvb_append(ctx.kvb_append_args(k[:0], k[:0], pool, table, i32([0, 0])))
    n0 = ctx.launch_count
    ctx.space_kvb_read(ctx.kvb_read_args(pool, table, i32([5, 5]), k[:, :0], k[:, :0]))
    assert ctx.launch_count == n0


# ------------------------------------------------------------------------------------------------ attention

def check(out, lse, want, want_lse, tol, lse_tol):
    """Within the oracle's bounds, and half a step of the output's type: 2^-8 of the value."""
    assert np.isfinite(out).all()
    err = np.abs(out - want) - np.abs(want) * 2.0 ** -8
    assert (err <= tol[..., None]).all(), (err.max(), np.argwhere(err > tol[..., None])[:3])
    fin = np.isfinite(want_lse)
    assert (fin == np.isfinite(lse)).all() and (lse[~fin] == -np.inf).all()
    if fin.any():
        e = np.abs(np.where(fin, lse - np.where(fin, want_lse, 0), 0))
        assert (e <= lse_tol + 2.0 ** -21 * np.abs(np.where(fin, want_lse, 0))).all(), e.max()


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
    (64, 1, 2, 2, [0, 0, 0], True), (64, 1, 16, 0, [100, 0], True), (128, 1, 1, 4, [0, 0, 0, 0, 0], False),
    # long lists of pages: rings go round several times, items end and begin within a thread block's share
    (64, 32, 1, 1, [1500, 1900, 700, 2048, 1, 1300, 2000, 1111], True),  # 8 query rows at a time
    (64, 16, 1, 3, [2000, 1501, 2048, 900, 1999, 0, 1700, 1300], True),  # 16
    (64, 12, 2, 2, [2047, 1500, 1800, 1203, 640, 1290], False),          # 18
    (64, 8, 1, 4, [2500, 1501, 2048, 900, 1999, 40], True),              # 25
    (128, 8, 4, 2, [1500, 1480, 2001], True),                            # 36
    (128, 6, 1, 7, [33, 2000, 0, 129, 1, 64], True),                     # 64
    (64, 8, 4, 3, [1100, 0, 777, 5], True),                              # 64 and not a row more
    (128, 40, 1, 5, [0, 1, 3, 0, 120], True),                            # more items than pages
]


# 128 query rows at a time: tables that name many pages
ATTN_WIDE = [
    (64, 2, 16, 2, [1030, 0, 128], True), (128, 1, 8, 5, [777], False), (128, 4, 4, 6, [300, 1, 0, 2000], True), (64, 3, 16, 7, [129, 500], True),
    (128, 8, 2, 7, [1999, 37, 1200, 2048, 640], True), (64, 1, 16, 3, [4000, 31], True),
]


@pytest.mark.parametrize("d,H,G,k,lens,block", ATTN)
def test_attention(B, d, H, G, k, lens, block):
    attention_case(B, d, H, G, k, lens, block)


@pytest.mark.parametrize("d,H,G,k,lens,block", ATTN_WIDE)
def test_attention_in_wide_tables(B, d, H, G, k, lens, block):
    attention_case(B, d, H, G, k, lens, block, 6000)


def attention_case(B, d, H, G, k, lens, block, pps=0):
    rng = np.random.default_rng(d + 100 * H + 10 * G + k)
    n, n_q, Hq = len(lens), (k + 1) ** 2, H * G
    pps = pps or max(1, max((L + P - 1) // P for L in lens) + 1)
    pool, table = random_cache(rng, lens, H, d, pps, spread=1.0)
    qb = bits(rng, n, n_q, Hq + 1, d)                                    # a head more than is used: strided rows
    kb, vb = (bits(rng, n, n_q, H, d), bits(rng, n, n_q, H, d)) if block else (None, None)
    variant, name = ((B.MASK_EQ5_LITERAL, EQ5_LITERAL) if k % 2 else (B.MASK_SAME_GROUP, SAME_GROUP))
    scale = 1 / math.sqrt(d)
    want = kvb.attention(bf16_bits_to_f64(qb[:, :, :Hq]), pool, table, lens, k, scale,
                         bf16_bits_to_f64(kb) if block else None, bf16_bits_to_f64(vb) if block else None, name)
    ctx = context(B, n, Hq, H, d)
    out = torch.full((n, n_q, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, Hq, n_q), float("nan"), device="cuda")
    status = i32([0] * n)
    keep = [dev(qb), dev(pool), dev(table), i32(lens), None if kb is None else dev(kb), None if vb is None else dev(vb)]
    a = ctx.kvb_attn_args(keep[0][:, :, :Hq], keep[1], keep[2], keep[3], out, k, scale, k_new=keep[4], v_new=keep[5], lse=lse,
                          status=status, mask_variant=variant)
    ctx.space_kvb_attn_step(a)
    check(f64(out), f64(lse), *want)
    assert not status.any()
    # the same bits again and again, also where pieces are joined
    first, first_lse = out.clone(), lse.clone()
    for _ in range(4):
        out.fill_(float("nan"))
        ctx.space_kvb_attn_step(a)
        assert torch.equal(first, out) and torch.equal(first_lse, lse)


def run(B, q, pool, table, lens, k, kn=None, vn=None, H=1, d=64, scale=None):
    n, n_q, Hq = q.shape[:3]
    ctx = context(B, n, Hq, H, d)
    out = torch.full((n, n_q, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, Hq, n_q), float("nan"), device="cuda")
    status = i32([0] * n)
    keep = [dev(q), dev(pool), dev(table), i32(lens)] + [None if x is None else dev(x) for x in (kn, vn)]
    ctx.space_kvb_attn_step(ctx.kvb_attn_args(keep[0], keep[1], keep[2], keep[3], out, k, scale or 1 / math.sqrt(d), k_new=keep[4], v_new=keep[5],
                                              lse=lse, status=status))
    torch.cuda.synchronize()
    return f64(out), f64(lse), status.tolist()


FORMS = [(64, 1), (128, 1), (64, 3), (128, 3), (64, 4), (128, 5), (128, 7), (64, 6), (128, 6)]       # head size and k, two query heads to a kv head
WIDE = 6000                                          # pages that a table names: from 65 rows on, 128 at a time


@pytest.mark.parametrize("d,k", FORMS)
def test_sequences_that_do_not_fit_and_pages_outside_the_pool(B, d, k):
    rng = np.random.default_rng(4)
    lens, n_q, pps = [300, 40, 300, 50, 700], (k + 1) ** 2, WIDE if k == 6 else 6
    pool, table = random_cache(rng, lens, 2, d, pps)
    q, kn, vn = bits(rng, 5, n_q, 4, d), bits(rng, 5, n_q, 2, d), bits(rng, 5, n_q, 2, d)
    given = [300, -3, pps * P + 1, 50, 700]
    table[0, 1], table[3, 0], table[4, :] = pool.shape[0], -1, 2 ** 31 - 1
    for block in (True, False):
        kb, vb = (kn, vn) if block else (None, None)
        out, lse, status = run(B, q, pool, table, given, k, kb, vb, 2, d)
        want = kvb.attention(bf16_bits_to_f64(q), pool, table, [300, 0, 0, 50, 700], k, 1 / math.sqrt(d),
                             *((bf16_bits_to_f64(kb), bf16_bits_to_f64(vb)) if block else (None, None)))
        want[0][1:3], want[1][1:3] = 0, -np.inf
        check(out, lse, *want)
        assert status == [B.ST_BAD_PAGE, B.ST_CAPACITY, B.ST_CAPACITY, B.ST_BAD_PAGE, B.ST_BAD_PAGE]
        if not block:
            assert (out[4] == 0).all()


@pytest.mark.parametrize("d,k", [f for f in FORMS if f[1] > 1])
def test_hidden_rows_have_no_influence(B, d, k):
    """What one block row holds reaches only the rows that see it, whatever it is."""
    rng = np.random.default_rng(5)
    n_q, lens = (k + 1) ** 2, [130, 0]
    pool, table = random_cache(rng, lens, 1, d, WIDE if k == 6 else 2)
    q, kn, vn = bits(rng, 2, n_q, 2, d), bits(rng, 2, n_q, 1, d), bits(rng, 2, n_q, 1, d)
    see = kvb.visible(k)
    base = run(B, q, pool, table, lens, k, kn, vn, 1, d)
    for row in (1, n_q // 2, n_q - 1):
        for fill in (0x7FC0, 0x7F80, 0xFF80, 0x7F7F, 0x5F80):            # NaN, infinities, the largest, 2^64
            k2, v2 = kn.copy(), vn.copy()
            k2[:, row], v2[:, row] = fill, fill
            got = run(B, q, pool, table, lens, k, k2, v2, 1, d)
            blind = ~see[:, row]
            assert (got[0][:, blind] == base[0][:, blind]).all() and (got[1][:, :, blind] == base[1][:, :, blind]).all(), (row, hex(fill))
            assert np.isfinite(got[0]).all()


@pytest.mark.parametrize("d,k", FORMS)
def test_a_query_row_that_is_not_finite(B, d, k):
    rng = np.random.default_rng(6)
    n_q, lens = (k + 1) ** 2, [300]
    pool, table = random_cache(rng, lens, 1, d, WIDE if k == 6 else 3)
    q, kn, vn = bits(rng, 1, n_q, 2, d), bits(rng, 1, n_q, 1, d), bits(rng, 1, n_q, 1, d)
    base = run(B, q, pool, table, lens, k, kn, vn, 1, d)
    for fill in (0x7FC0, 0x7F80, 0xFF80):
        q2 = q.copy()
        q2[0, n_q // 2, 1, 5] = fill
        got = run(B, q2, pool, table, lens, k, kn, vn, 1, d)
        bad = np.zeros((n_q, 2), bool)
        bad[n_q // 2, 1] = True
        assert np.isnan(got[0][0][bad]).all() and np.isnan(got[1][0].T[bad]).all()
        assert (got[0][0][~bad] == base[0][0][~bad]).all() and (got[1][0].T[~bad] == base[1][0].T[~bad]).all()


@pytest.mark.parametrize("d,k", FORMS)
@pytest.mark.parametrize("size", [30.0, 3000.0, 3e9])
def test_large_scores(B, d, k, size):
    """Scores far apart: the largest key takes (nearly) all.  The cache's scores are exact differences times the factor; scores as large
    as these are known to d 2^-24 of themselves, which the bound counts."""
    rng = np.random.default_rng(7)
    n_q, lens = (k + 1) ** 2, [400, 31]
    pool, table = random_cache(rng, lens, 1, d, WIDE if k == 6 else 4)
    q, kn, vn = bits(rng, 2, n_q, 2, d, scale=size), bits(rng, 2, n_q, 1, d, scale=0.01), bits(rng, 2, n_q, 1, d)
    out, lse, status = run(B, q, pool, table, lens, k, kn, vn, 1, d)
    assert status == [0, 0] and np.isfinite(out).all() and np.isfinite(lse).all()
    if size < 1e9:
        want = kvb.attention(bf16_bits_to_f64(q), pool, table, lens, k, 1 / math.sqrt(d), bf16_bits_to_f64(kn), bf16_bits_to_f64(vn))
        check(out, lse, *want)


@pytest.mark.parametrize("d,k", FORMS)
def test_blocks_of_very_different_sizes(B, d, k):
    """V blocks 2^40 apart, K blocks 2^-60: what is large and hardly seen, and what is small and seen, in one row."""
    rng = np.random.default_rng(8)
    n_q, lens = (k + 1) ** 2, [500]
    pool, table = random_cache(rng, lens, 1, d, WIDE if k == 6 else 5)
    for j in range(4):
        sc = kvb._views(pool[table[0, j], 0], d)[2]
        sc[:, 1] *= np.float32(2.0 ** 20) if j == 1 else np.float32(2.0 ** -20) if j == 2 else 1
        sc[j, 1] *= np.float32(2.0 ** -30)
        if j == 3:
            sc[:2, 0] = np.float32(2.0 ** -60)
    q, kn, vn = bits(rng, 1, n_q, 2, d), bits(rng, 1, n_q, 1, d), bits(rng, 1, n_q, 1, d, scale=1e-4)
    out, lse, status = run(B, q, pool, table, lens, k, kn, vn, 1, d)
    want = kvb.attention(bf16_bits_to_f64(q), pool, table, lens, k, 1 / math.sqrt(d), bf16_bits_to_f64(kn), bf16_bits_to_f64(vn))
    check(out, lse, *want)


@pytest.mark.parametrize("k", [0, 2, 5])
def test_offsets_past_four_gigabytes(B, k):
    """Pages of a pool far apart: the second and third lie past 2^31 and 2^32 bytes."""
    d, H, L, n_q = 64, 1, 300, (k + 1) ** 2
    rng = np.random.default_rng(11)
    small, table = random_cache(rng, [L], H, d, 4)
    bytes_ = kvb.head_bytes(d)
    stride = (1 << 31) + 16 * 1001
    pages = 3
    order = [int(table[0, j]) for j in range(3)]
    big = torch.empty((pages - 1) * stride + bytes_, dtype=torch.uint8, device="cuda")
    pool = big.as_strided((pages, H, bytes_), (stride, bytes_, 1))
    for j, p in enumerate(order):
        pool[j].copy_(dev(small[p]))
    t = np.array([[0, 1, 2, -1]], np.int32)
    q, kn, vn = bits(rng, 1, n_q, 2, d), bits(rng, 1, n_q, H, d), bits(rng, 1, n_q, H, d)
    ctx = context(B, 1, 2, H, d)
    out = torch.empty(1, n_q, 2, d, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(1, 2, n_q, device="cuda")
    keep = [dev(q), dev(kn), dev(vn), dev(t)]
    ctx.space_kvb_attn_step(ctx.kvb_attn_args(keep[0], pool, keep[3], i32([L]), out, k, 0.125, k_new=keep[1], v_new=keep[2], lse=lse))
    check(f64(out), f64(lse), *kvb.attention(bf16_bits_to_f64(q), small, table, [L], k, 0.125, bf16_bits_to_f64(kn), bf16_bits_to_f64(vn)))
    ctx.space_kvb_append(ctx.kvb_append_args(keep[1], keep[2], pool, keep[3], i32([L])))
    o = torch.empty(1, n_q, H, d, dtype=torch.bfloat16, device="cuda")
    ctx.space_kvb_read(ctx.kvb_read_args(pool, keep[3], i32([L + n_q]), o, o.clone(), first=i32([L])))
    for h in range(H):
        kvb.append(small, table[0], h, L, bf16_bits_to_f64(kn)[0, :, h], bf16_bits_to_f64(vn)[0, :, h])
    assert (f64(o)[0].transpose(1, 0, 2) == kvb.read_rows(small, table[0], L + n_q, d)[0][:, L:]).all()


@pytest.mark.parametrize("k", [1, 4])
def test_captured_and_on_another_stream(B, k):
    """Two graphs of one context, replayed in turn on one stream with lengths that changed in between."""
    d, H, n, n_q = 128, 2, 3, (k + 1) ** 2
    rng = np.random.default_rng(12)
    lens = [300, 64, 500]
    pool, table = random_cache(rng, [600] * 3, H, d, 5)
    pd, td = dev(pool), dev(table)
    ctx, stream = context(B, n, 2 * H, H, d), torch.cuda.Stream()
    kv_len = i32(lens)
    graphs, outs, qs = [], [], []
    for i in range(2):
        q = bits(rng, n, n_q, 2 * H, d)
        qd, out = dev(q), torch.empty(n, n_q, 2 * H, d, dtype=torch.bfloat16, device="cuda")
        a = ctx.kvb_attn_args(qd, pd, td, kv_len, out, k, 0.09)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=stream):
            ctx.space_kvb_attn_step(a)
        graphs.append(g); outs.append(out); qs.append((q, a))
    for L in (lens, [1, 599, 128]):
        kv_len.copy_(i32(L))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for (q, _), out in zip(qs, outs):
            want = kvb.attention(bf16_bits_to_f64(q), pool, table, L, k, 0.09)
            check(f64(out), want[1], *want)


def test_two_contexts_on_two_streams_at_once(B):
    """Calls of both forms in turn on each stream, the streams not waiting for each other, behind appends that move the lengths on."""
    d, H, n, steps = 128, 4, 3, 12
    rng = np.random.default_rng(13)
    runs = []
    for i in range(2):
        pool, table = random_cache(rng, [900] * n, H, d, 8)
        runs.append(dict(ctx=context(B, n, 2 * H, H, d), stream=torch.cuda.Stream(), table=dev(table), first=pool))
    new = [dev(bits(rng, n, 16, h, d)) for h in (2 * H, H, H)]

    def go(r, pool, lens, outs):
        for j in range(steps):
            k = (1, 3, 2)[j % 3]
            n_q, out = (k + 1) ** 2, outs[j]
            q, kn, vn = (x[:, :n_q] for x in new)
            r["keep"].append(a := r["ctx"].kvb_attn_args(q, pool, r["table"], lens[j], out, k, 0.09, k_new=kn, v_new=vn))
            r["ctx"].space_kvb_attn_step(a)
            r["keep"].append(a := r["ctx"].kvb_append_args(kn, vn, pool, r["table"], lens[j], row_step=k + 1, kv_len_out=lens[j + 1]))
            r["ctx"].space_kvb_append(a)
    got = []
    for at_once in (False, True):
        work = []
        for r in runs:
            r["keep"] = []
            lens = [i32([700, 13, 0]) for _ in range(steps + 1)]
            outs = [torch.zeros(n, ((1, 3, 2)[j % 3] + 1) ** 2, 2 * H, d, dtype=torch.bfloat16, device="cuda") for j in range(steps)]
            work.append((r, dev(r["first"]), lens, outs))
        torch.cuda.synchronize()
        for w in work:
            with torch.cuda.stream(w[0]["stream"] if at_once else torch.cuda.current_stream()):
                go(*w)
            if not at_once:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        got.append([(w[1], w[2][-1], w[3]) for w in work])
    for (p0, l0, o0), (p1, l1, o1) in zip(*got):
        assert torch.equal(p0, p1) and torch.equal(l0, l1) and l0.tolist() == [L + 4 * (2 + 4 + 3) for L in (700, 13, 0)]
        assert all(torch.equal(x, y) for x, y in zip(o0, o1))


def test_page_moves(B):
    """space_pages_copy takes the 8-bit pool's pages whole or in rows of a page."""
    d, H = 64, 3
    pool = torch.randint(0, 256, (6, H, kvb.head_bytes(d)), dtype=torch.uint8, device="cuda")
    want = pool.clone()
    want[5], want[0] = pool[2], pool[3]
    B.space_pages_copy(B.page_pools([pool]), [(2, 5, P), (3, 0, P)])
    assert torch.equal(pool, want)


def test_refusals(B):
    """What the library itself refuses: nothing is launched."""
    d, H, Hq, k = 64, 2, 4, 1
    ctx = context(B, 2, Hq, H, d)
    pool, table, n_q = B.kvb_pool(4, H, d), i32([[0, 1], [2, 3]]), (k + 1) ** 2
    rows = lambda h=H: torch.zeros(2, n_q, h, d, dtype=torch.bfloat16, device="cuda")
    keep = [rows(Hq), rows(Hq), rows(), rows(), rows(), i32([0, 0]), i32([0, 0]), B.rope(B.rope_table(9, 32))]
    q, out, kn, vn, o2, kv_len, len2, rope = keep

    def attn():
        return ctx.kvb_attn_args(q, pool, table, kv_len, out, k, 0.1, k_new=kn, v_new=vn)

    def append():
        return ctx.kvb_append_args(kn, vn, pool, table, kv_len, kv_len_out=len2, rope=rope, q=q, q_out=out)

    def read():
        return ctx.kvb_read_args(pool, table, kv_len, kn, o2)
    cases = [(attn, "space_kvb_attn_step", "batch", 3, B.E_WORKSPACE), (attn, "space_kvb_attn_step", "k", 8, B.E_WORKSPACE),
             (attn, "space_kvb_attn_step", "k", -1, B.E_INVALID_ARG), (attn, "space_kvb_attn_step", "scale", 0.0, B.E_INVALID_ARG),
             (attn, "space_kvb_attn_step", "scale", float("nan"), B.E_INVALID_ARG), (attn, "space_kvb_attn_step", "q", 0, B.E_INVALID_ARG),
             (attn, "space_kvb_attn_step", "v_new", 0, B.E_INVALID_ARG), (attn, "space_kvb_attn_step", "q", q.data_ptr() + 2, B.E_ALIGNMENT),
             (attn, "space_kvb_attn_step", "q_stride_r", 4, B.E_ALIGNMENT), (attn, "space_kvb_attn_step", "mask_variant", 9, B.E_INVALID_ARG),
             (attn, "space_kvb_attn_step", "cache.n_pages", 0, B.E_INVALID_ARG), (attn, "space_kvb_attn_step", "cache.pool", pool.data_ptr() + 8, B.E_ALIGNMENT),
             (attn, "space_kvb_attn_step", "cache.head_stride", 16, B.E_INVALID_ARG), (attn, "space_kvb_attn_step", "cache.page_stride", 16, B.E_INVALID_ARG),
             (attn, "space_kvb_attn_step", "cache.pages_per_seq", 1 << 24, B.E_INVALID_ARG), (attn, "space_kvb_attn_step", "kv_len", 0, B.E_INVALID_ARG),
             (append, "space_kvb_append", "batch", 3, B.E_WORKSPACE), (append, "space_kvb_append", "rows", 0, B.E_INVALID_ARG),
             (append, "space_kvb_append", "row_step", 0, B.E_INVALID_ARG), (append, "space_kvb_append", "kv_len_out", kv_len.data_ptr(), B.E_INVALID_ARG),
             (append, "space_kvb_append", "q_out", 0, B.E_INVALID_ARG), (append, "space_kvb_append", "rope.rot_dim", 24, B.E_UNSUPPORTED),
             (append, "space_kvb_append", "rope.rot_dim", 80, B.E_UNSUPPORTED), (append, "space_kvb_append", "rope.n_pos", 0, B.E_INVALID_ARG),
             (append, "space_kvb_append", "rope.interleaved", 2, B.E_INVALID_ARG), (append, "space_kvb_append", "rope.table", 4, B.E_ALIGNMENT),
             (append, "space_kvb_append", "rope.table", 0, B.E_INVALID_ARG), (append, "space_kvb_append", "new_stride_h", 12, B.E_ALIGNMENT),
             (read, "space_kvb_read", "batch", 3, B.E_WORKSPACE), (read, "space_kvb_read", "rows", -1, B.E_INVALID_ARG),
             (read, "space_kvb_read", "k_out", 0, B.E_INVALID_ARG), (read, "space_kvb_read", "out_stride_b", 3, B.E_ALIGNMENT)]
    n0 = ctx.launch_count
    for make, call, field, value, code in cases:
        a = make()
        at, _, name = field.rpartition(".")
        setattr(getattr(a, at) if at else a, name, value)
        with pytest.raises(B.SpaceError) as e:
            getattr(ctx, call)(a)
        assert e.value.code == code, (call, field, value, e.value.code)
    assert ctx.launch_count == n0
