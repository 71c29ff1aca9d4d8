"""Rotation by position with the append to the bf16 cache (space_rope_append) on the GPU: every bit against fp32 arithmetic on the host."""
import numpy as np
import pytest
import torch

from oracle import kvb
from oracle.bf16 import bf16_bits_to_f64, f32_to_bf16_bits

pytestmark = pytest.mark.gpu
P = 128


@pytest.fixture(scope="module")
def B():
    from paper_2402_11809_b200 import binding
    return binding


def bits(rng, *shape):
    return f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))


def dev(a):
    if a.dtype == np.uint16:
        return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda().view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def i32(x):
    return dev(np.array(x, np.int32))


def f64(t):
    return t.detach().cpu().double().numpy()


def angles(rng, n_pos, rot):
    a = rng.standard_normal((n_pos, rot // 2)) * 5
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def turned(x, table, pos, inter):
    return bf16_bits_to_f64(f32_to_bf16_bits(kvb.turn(bf16_bits_to_f64(x), table, pos, inter)))


CASES = [
    # d, H_q, H_kv, rot, neighbours, rows, lens, counts, to (pages, rows, out), queries
    (128, 4, 4, 128, False, 1, [0, 5, 127, 128], None, "pages", True),
    (64, 8, 2, 64, False, 25, [0, 100, 126], [25, 0, 9], "pages", True),
    (64, 16, 1, 16, True, 3, [7], None, "rows", True),
    (128, 8, 8, 96, False, 36, [300, 0], [36, 40], "rows", False),
    (128, 1, 1, 32, True, 130, [1, 60, 0], [130, 64, -3], "pages", True),
    (64, 6, 3, 48, False, 7, [9, 2], None, "out", True),
    (128, 32, 4, 128, True, 64, [0, 0, 0, 0, 0], None, "out", True),
    (64, 5, 5, 32, False, 700, [3, 0, 0], [700, 1, 699], "pages", False),
    (128, 4, 1, 64, True, 2000, [0, 10], [2000, 1999], "rows", True),
]


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("d,Hq,H,rot,inter,rows,lens,counts,to,queries", CASES)
def test_rotation(B, d, Hq, H, rot, inter, rows, lens, counts, to, queries, given):
    rng = np.random.default_rng(d + rot + rows)
    n = len(lens)
    cnt = [min(max(c, 0), rows) for c in (counts or [rows] * n)]
    q, kv = bits(rng, n, rows, Hq + 1, d), bits(rng, n, rows, 2, H, d)           # a head more than is used; slices of one tensor
    qd, kvd = dev(q), dev(kv)
    n_pos = max(lens) + rows + 4
    table = angles(rng, n_pos, rot)
    pos = rng.integers(0, n_pos, size=(n, rows)).astype(np.int32) if given else None
    rope = B.rope(dev(table), interleaved=inter, pos=None if pos is None else dev(pos))
    cap = (max(a + c for a, c in zip(lens, cnt)) + P) // P * P
    ctx = B.Context(max_batch=n, n_q_heads=Hq, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=cap)
    out_len, status = i32([0] * n), i32([0] * n)
    fill = bits(rng, 1)[0]
    more = dict(v=kvd[:, :, 1])
    if to == "out":
        k_out = dev(np.full((n, rows, H, d), fill))
        more = dict(k_out=k_out)
    elif to == "rows":
        cache = dev(np.full((2, n, cap, H, d), fill)).transpose(2, 3)            # [2, n, H, cap, d] by strides
        more.update(k_cache=cache[0], v_cache=cache[1])
    else:
        pps = cap // P
        pages = rng.permutation(n * pps + 1)[:n * pps].reshape(n, pps).astype(np.int32)
        cache = dev(np.full((2, n * pps + 1, H, P, d), fill))
        more.update(k_cache=cache[0], v_cache=cache[1], page_table=dev(pages))
    q_out = dev(np.full((n, rows, Hq, d), fill)) if queries else None
    n0 = ctx.launch_count
    ctx.space_rope_append(ctx.rope_append_args(rope, qd[:, :, :Hq] if queries else None, q_out, kvd[:, :, 0], i32(lens),
                                               count=None if counts is None else i32(counts), kv_len_out=out_len, status=status, **more))
    assert ctx.launch_count == n0 + 1 and not status.any()
    assert out_len.tolist() == [a + c for a, c in zip(lens, cnt)]
    old = bf16_bits_to_f64(np.array([fill]))[0]
    if to != "out":
        want_c = np.full(tuple(cache.shape), old)
    for b in range(n):
        c, L = cnt[b], lens[b]
        at = pos[b, :c] if given else L + np.arange(c)
        if queries:
            got = f64(q_out[b])
            assert (got[:c] == turned(q[b, :c, :Hq], table, at, inter)).all() and (got[c:] == old).all()
        k, v = turned(kv[b, :c, 0], table, at, inter), bf16_bits_to_f64(kv[b, :c, 1])
        if to == "out":
            got = f64(k_out[b])
            assert (got[:c] == k).all() and (got[c:] == old).all()
            continue
        for g in range(c):
            s = L + g
            where = (b, slice(None), s) if to == "rows" else (pages[b, s // P], slice(None), s % P)
            want_c[(0, *where)], want_c[(1, *where)] = k[g], v[g]
    if to != "out":
        assert (f64(cache) == want_c).all()                              # everything else as it was
    if queries:                                                          # in place gives the same
        inplace = dev(q)
        ctx.space_rope_append(ctx.rope_append_args(rope, inplace[:, :, :Hq], inplace[:, :, :Hq], kvd[:, :, 0], i32(lens),
                                                   count=None if counts is None else i32(counts), k_out=kvd[:, :, 0]))
        for b in range(n):
            assert torch.equal(inplace[b, :cnt[b], :Hq], q_out[b, :cnt[b]])
            assert torch.equal(inplace[b, cnt[b]:], qd[b, cnt[b]:]) and torch.equal(inplace[b, :, Hq], qd[b, :, Hq])


def test_positions_outside_the_table_capacity_and_bad_pages(B):
    d, H, n, rows = 64, 2, 6, 3
    rng = np.random.default_rng(1)
    table = angles(rng, 10, 64)
    q, k, v = bits(rng, n, rows, H, d), bits(rng, n, rows, H, d), bits(rng, n, rows, H, d)
    pos = np.array([[0, 1, 2], [-1, 5, 6], [7, 10, 8], [1, 2, 3], [1, 2, 3], [1, 2, 3]], np.int32)
    ctx = B.Context(max_batch=n, n_q_heads=H, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=256)
    cache = torch.zeros(2, 8, H, P, d, dtype=torch.bfloat16, device="cuda")
    pages = np.array([[0, 1], [2, 3], [4, 5], [6, 9], [-1, 7], [6, 7]], np.int32)
    lens, status, out_len = [0, 10, 20, 126, 5, 254], i32([0] * n), i32([0] * n)
    q_out = torch.zeros(n, rows, H, d, dtype=torch.bfloat16, device="cuda")
    ctx.space_rope_append(ctx.rope_append_args(B.rope(dev(table), pos=dev(pos)), dev(q), q_out, dev(k), i32(lens), v=dev(v), k_cache=cache[0],
                                               v_cache=cache[1], page_table=dev(pages), kv_len_out=out_len, status=status))
    assert status.tolist() == [0, B.ST_BAD_POSITION, B.ST_BAD_POSITION, B.ST_BAD_PAGE, B.ST_BAD_PAGE, B.ST_CAPACITY]
    assert out_len.tolist() == [3, 13, 23, 129, 8, 254]
    want = np.zeros((2, 8, H, P, d))
    for b in range(n - 1):
        assert (f64(q_out[b]) == turned(q[b], table, pos[b], False)).all()
        for g in range(rows):
            s = lens[b] + g
            if 0 <= pages[b, s // P] < 8:
                want[0, pages[b, s // P], :, s % P] = turned(k[b], table, pos[b], False)[g]
                want[1, pages[b, s // P], :, s % P] = bf16_bits_to_f64(v[b])[g]
    assert (f64(cache) == want).all() and not q_out[n - 1].any()


def test_values_that_are_not_finite_stay_in_their_pairs(B):
    d = 64
    rng = np.random.default_rng(2)
    k = bits(rng, 1, 1, 2, d)
    k[0, 0, 0, 3], k[0, 0, 1, 40] = 0x7FC0, 0x7F80                       # NaN in a pair that turns, infinity in a channel that does not
    out = torch.zeros(1, 1, 2, d, dtype=torch.bfloat16, device="cuda")
    ctx = B.Context(max_batch=1, n_q_heads=2, n_kv_heads=2, head_dim=d, k_max=7, vocab=8, s_cap=128)
    ctx.space_rope_append(ctx.rope_append_args(B.rope(dev(angles(rng, 4, 32))), None, None, dev(k), i32([2]), k_out=out))
    got = f64(out)[0, 0]
    assert np.isnan(got[0]).nonzero()[0].tolist() == [3, 19] and np.isfinite(got[1]).sum() == d - 1 and got[1, 40] == np.inf


def test_captured_with_lengths_that_move_on(B):
    """A step that is captured once: the rows behind the cached ones, the lengths advanced by the call itself."""
    d, H, n = 64, 2, 3
    rng = np.random.default_rng(3)
    ctx = B.Context(max_batch=n, n_q_heads=H, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=256)
    cache = torch.zeros(2, n, H, 256, d, dtype=torch.bfloat16, device="cuda")
    table = angles(rng, 256, 64)
    k, v = bits(rng, n, 1, H, d), bits(rng, n, 1, H, d)
    kd, vd, lens, next_len = dev(k), dev(v), i32([0, 100, 5]), i32([0, 0, 0])
    a = ctx.rope_append_args(B.rope(dev(table)), None, None, kd, lens, v=vd, k_cache=cache[0], v_cache=cache[1], kv_len_out=next_len)
    g, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=stream):
        ctx.space_rope_append(a)
        lens.copy_(next_len)
    for _ in range(20):
        g.replay()
    torch.cuda.synchronize()
    assert lens.tolist() == [20, 120, 25]
    for b, L in enumerate([0, 100, 5]):
        want = np.stack([turned(k[b], table, np.array([L + i]), False)[0] for i in range(20)], 1)
        assert (f64(cache[0, b, :, L:L + 20]) == want).all() and (cache[1, b, :, L:L + 20] == vd[b, 0][:, None]).all()
    assert (cache != 0).any(-1).sum() == 2 * n * H * 20


def test_refusals(B):
    d, H = 64, 2
    ctx = B.Context(max_batch=2, n_q_heads=H, n_kv_heads=H, head_dim=d, k_max=7, vocab=8, s_cap=256)
    r = lambda: torch.zeros(2, 3, H, d, dtype=torch.bfloat16, device="cuda")
    keep = [r(), r(), r(), r(), i32([0, 0]), i32([0, 0]), torch.zeros(2, 2, H, 256, d, dtype=torch.bfloat16, device="cuda")]
    q, q_out, k, v, lens, out_len, cache = keep
    make = lambda: ctx.rope_append_args(B.rope(B.rope_table(9, 32)), q, q_out, k, lens, v=v, k_cache=cache[0], v_cache=cache[1], kv_len_out=out_len)
    cases = [("batch", 3, B.E_WORKSPACE), ("batch", -1, B.E_WORKSPACE), ("rows", -1, B.E_INVALID_ARG), ("rows", 0, B.E_INVALID_ARG), ("k", 0, B.E_INVALID_ARG),
             ("v", 0, B.E_INVALID_ARG), ("q_out", 0, B.E_INVALID_ARG), ("kv_len", 0, B.E_INVALID_ARG), ("kv_len_out", lens.data_ptr(), B.E_INVALID_ARG),
             ("k_out", k.data_ptr(), B.E_INVALID_ARG), ("v_cache", 0, B.E_INVALID_ARG), ("k_cache", 0, B.E_INVALID_ARG), ("rope.table", 0, B.E_INVALID_ARG),
             ("rope.rot_dim", 8, B.E_UNSUPPORTED), ("rope.rot_dim", 40, B.E_UNSUPPORTED), ("rope.rot_dim", 128, B.E_UNSUPPORTED),
             ("rope.n_pos", 0, B.E_INVALID_ARG), ("rope.interleaved", -1, B.E_INVALID_ARG), ("q", q.data_ptr() + 2, B.E_ALIGNMENT),
             ("kv_stride_s", 4, B.E_ALIGNMENT), ("kv_stride_s", 8, B.E_INVALID_ARG), ("new_stride_r", 12, B.E_ALIGNMENT)]
    n0 = ctx.launch_count
    for field, value, code in cases:
        a = make()
        at, _, name = field.rpartition(".")
        setattr(getattr(a, at) if at else a, name, value)
        with pytest.raises(B.SpaceError) as e:
            ctx.space_rope_append(a)
        assert e.value.code == code, (field, value, e.value.code)
    assert ctx.launch_count == n0
