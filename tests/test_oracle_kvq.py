"""The oracle of the 4-bit cache: quantisation, byte layout and attention pinned by independent statements."""
import math

import numpy as np
import pytest

from oracle import attention, brute, kvq  # noqa: F401
from oracle.bf16 import f32_to_bf16_bits


def rand_bf16(rng, *shape):
    return kvq.to_f64(f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32)))


@pytest.mark.parametrize("d", [64, 128])
def test_codes_are_the_nearest_of_sixteen_levels(d):
    rng = np.random.default_rng(0)
    x = rand_bf16(rng, 200, d) * np.exp2(rng.integers(-20, 20, size=(200, 1)))
    u, step, lo = kvq.quantise(x)
    assert u.min() == 0 and u.max() == 15 and (lo[:, 0] == x.min(1)).all()
    # within half a step of the value; the top one may lie past level 15 by what rounding the step took (2^-9 of 15 steps)
    assert (np.abs(kvq.values(x) - x) <= step * (0.5 + 15 * 2.0 ** -8)).all()
    levels = lo[..., None] + step[..., None] * np.arange(16)
    assert (np.abs(np.abs(levels - x[..., None]).min(-1) - np.abs(kvq.values(x) - x)) <= 1e-12 * np.abs(x)).all()


def test_special_rows():
    d = 64
    z = np.zeros(d)
    assert (kvq.values(z) == 0).all()
    c = np.full(d, 5.0)
    assert (kvq.values(c) == 5).all()
    big = np.where(np.arange(d) % 2, kvq.BF16_MAX, -kvq.BF16_MAX)
    v = kvq.values(big)
    assert np.isfinite(v).all() and (np.abs(v / big - 1) < 2.0 ** -7).all()
    odd = np.linspace(-1, 1, d)
    odd[3], odd[5], odd[7] = np.nan, np.inf, -np.inf
    v = kvq.values(odd)
    assert np.isfinite(v).all() and abs(v[5] / kvq.BF16_MAX - 1) < 2.0 ** -7 and abs(v[7] / kvq.BF16_MAX + 1) < 2.0 ** -7


@pytest.mark.parametrize("d", [64, 128])
def test_every_element_has_its_own_nibble(d):
    (k_at, k_sh), (v_at, v_sh) = kvq._places(d)
    seen = {(int(a), int(s)) for at, sh in ((k_at, k_sh), (v_at, v_sh)) for a, s in zip(at.ravel(), np.broadcast_to(sh, at.shape).ravel())}
    assert len(seen) == 2 * 32 * d and max(a for a, _ in seen) == 32 * d - 1 and {s for _, s in seen} == {0, 4}


@pytest.mark.parametrize("d,H", [(64, 2), (128, 1)])
def test_rows_come_back_as_their_values(d, H):
    rng = np.random.default_rng(1)
    pool = np.zeros((3, H, 4 * kvq.block_bytes(d)), dtype=np.uint8)
    table = np.array([2, 0], dtype=np.int32)
    n = 150
    x = rand_bf16(rng, 2, n, H, d)
    for s in rng.permutation(n):
        for h in range(H):
            kvq.write_row(pool, table[s // 128], h, s % 128, x[0, s, h], x[1, s, h])
    k, v = kvq.read_rows(pool, table, n, d)
    assert (k == kvq.values(x[0]).transpose(1, 0, 2)).all() and (v == kvq.values(x[1]).transpose(1, 0, 2)).all()
    assert not pool[1].any()


@pytest.mark.parametrize("k,G", [(0, 1), (2, 2), (3, 1)])
def test_attention_is_that_of_the_values(k, G):
    """Against the bf16 oracle over the values, rounded to bf16 where that changes nothing the tolerance sees."""
    rng = np.random.default_rng(2)
    d, H, L = 64, 2, 70
    n_q = (k + 1) ** 2
    pool = np.zeros((1, H, 4 * kvq.block_bytes(d)), dtype=np.uint8)
    for s in range(L):
        for h in range(H):
            kvq.write_row(pool, 0, h, s, *rand_bf16(rng, 2, d))
    q, kn, vn = rand_bf16(rng, 1, n_q, H * G, d), rand_bf16(rng, 1, n_q, H, d), rand_bf16(rng, 1, n_q, H, d)
    out, lse = kvq.attention(q, pool, np.array([[0]]), [L], k, 1 / math.sqrt(d), kn, vn)
    K, V = kvq.read_rows(pool, [0], L, d)
    for hq in range(H * G):
        for i in range(n_q):
            num, den = np.zeros(d), 0.0
            for j in range(L + n_q):
                if j >= L:
                    gi, oi, gj, oj = i // (k + 1), i % (k + 1), (j - L) // (k + 1), (j - L) % (k + 1)
                    if j - L > i or (oj and (not oi or gi != gj)):
                        continue
                kk, vv = (K[hq // G, j], V[hq // G, j]) if j < L else (kn[0, j - L, hq // G], vn[0, j - L, hq // G])
                e = math.exp(float(q[0, i, hq] @ kk) / math.sqrt(d))
                num, den = num + e * vv, den + e
            assert np.allclose(out[0, i, hq], num / den, rtol=1e-11, atol=1e-13)
            assert abs(lse[0, hq, i] - math.log(den)) < 1e-11
