"""Attention over the 4-bit cache where its numbers are unusual.  Against the oracle in 64 bits, in every form of the
kernels."""
import math

import numpy as np
import pytest

from oracle import kvq
from oracle.bf16 import bf16_bits_to_f64, f32_to_bf16_bits
from test_gpu_kvq import B, P, WIDE, check, random_cache, run_attention, span_of  # noqa: F401 (B: a fixture)

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

@pytest.mark.parametrize("level", [-1000.0, -100.0, -80.0, 1000.0])
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
