"""The 8-bit cache's oracle against torch's e4m3 type and against hand-made bytes."""
import numpy as np
import pytest
import torch

from oracle import kvb


def test_codes_are_the_types():
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(kvb.VALUES, v, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(4000) * 2.0 ** rng.integers(-14, 9, 4000), np.arange(-1000, 1000) * 2.0 ** -11, [448.0, -448.0, 0.0]])
    x = np.clip(x, -448, 448).astype(np.float32)
    assert (kvb.encode(x.astype(np.float64)) == torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()).all()


@pytest.mark.parametrize("top,e", [(0.0, -100), (448.0, 0), (448.1, 1), (224.0, -1), (1.75, -8), (1.76, -7), (3.3895313892515355e38, 120)])
def test_exponent(top, e):
    assert kvb.exponent(top) == e


def test_rows_in_and_out():
    rng = np.random.default_rng(1)
    d, n = 64, 150
    k, v = rng.standard_normal((n, d)), rng.standard_normal((n, d))
    k[70:] *= 40                                             # raises the power of two of the block that row 64 opened
    pool, table = np.full((3, 2, kvb.head_bytes(d)), 7, np.uint8), np.array([2, 0])
    at = 0
    for m in (1, 31, 33, 5, 80):
        kvb.append(pool, table, 1, at, k[at:at + m], v[at:at + m])
        at += m
    K, V = kvb.read_rows(pool, table, n, d)
    for got, want in ((K[1], k), (V[1], v)):
        top = np.abs(want).reshape(-1)
        for s0 in range(0, n, 32):
            w, g = want[s0:s0 + 32], got[s0:s0 + 32]
            step = 2.0 ** kvb.exponent(np.abs(w).max())
            # two roundings at most: half a step of the code each (2^-4 of the value), half of 2^-9 near zero
            assert (np.abs(w - g) <= np.abs(w) * (2.0 ** -4 + 2.0 ** -4 * 1.07) + 2 * 2.0 ** -10 * step).all()
    assert (pool[:, 0] == 7).all() and (pool[1] == 7).all()
    # one rounding only where nothing raised it
    assert (np.abs(V[1] - v) <= np.abs(v) * 2.0 ** -4 + 2.0 ** -10 * np.repeat([2.0 ** kvb.exponent(np.abs(v[s:s + 32]).max()) for s in range(0, n, 32)], 32)[:n, None]).mean() > 0.9


def test_a_planted_mistake_is_seen():
    """Bounds of the attention test: a key left out, a scale off by one, a row's weight a sixteenth off."""
    rng = np.random.default_rng(2)
    d, L = 64, 200
    pool, table = np.zeros((2, 1, kvb.head_bytes(d)), np.uint8), np.array([[0, 1]])
    k, v = rng.standard_normal((L, d)), rng.standard_normal((L, d))
    kvb.append(pool, table[0], 0, 0, k, v)
    q = rng.standard_normal((1, 1, 1, d)) * 2
    out, lse, tol, lse_tol = kvb.attention(q, pool, table, [L], 0, d ** -0.5)
    assert tol.max() < 0.05 and lse_tol.max() < 1e-3
    one = kvb.attention(q, pool, table, [L - 1], 0, d ** -0.5)
    assert np.abs(one[1] - lse).max() > lse_tol.max()
    bad = pool.copy()
    bad[0, 0].view(np.float32)[-7] *= 2                      # V scale of rows 0 .. 31
    assert (np.abs(kvb.attention(q, bad, table, [L], 0, d ** -0.5)[0] - out) > tol[..., None] + np.abs(out) * 2.0 ** -8).any()


def test_turning_keeps_lengths_and_goes_back():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((5, 3, 64)).astype(np.float32)
    ang = rng.standard_normal((9, 16))
    table = np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)
    back = np.concatenate([np.cos(ang), -np.sin(ang)], 1).astype(np.float32)
    pos = np.array([0, 8, 3, 3, 1])
    for inter in (False, True):
        y = kvb.turn(x, table, pos, inter)
        assert (y[..., 32:] == x[..., 32:]).all() and np.abs(kvb.turn(y, back, pos, inter) - x).max() < 1e-6
        a = (slice(0, 32, 2), slice(1, 32, 2)) if inter else (slice(0, 16), slice(16, 32))
        assert np.abs(np.hypot(y[..., a[0]], y[..., a[1]]) - np.hypot(x[..., a[0]], x[..., a[1]])).max() < 1e-6
        assert (kvb.turn(x, table, np.array([-5, 99, 3, 3, 1]), inter)[:2] == kvb.turn(x, table, np.array([0, 8, 3, 3, 1]), inter)[:2]).all()
