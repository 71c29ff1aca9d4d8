"""The 8-bit cache where its numbers are unusual: rows next to the largest number, sums that pass it, block rows and query rows far
from one.  Against the oracle in 64 bits, in every form of the attention."""
import math

import numpy as np
import pytest

from oracle import kvb
from oracle.bf16 import bf16_bits_to_f64
from test_gpu_kvb import B, FORMS, WIDE, bits, check, random_cache, run  # noqa: F401 (B: a fixture)

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
