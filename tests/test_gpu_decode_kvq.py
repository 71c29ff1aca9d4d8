"""Samples of one prompt decoded on a 4-bit cache with shared pages: paper_2402_11809_b200/decode_kvq.py."""
import numpy as np
import pytest
import torch

from oracle import kvq

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def D():
    from paper_2402_11809_b200 import build
    build.build()
    from paper_2402_11809_b200 import decode_kvq
    return decode_kvq


def decode(D, model, prompt, samples, k, share, temperature, steps=20):
    dec = D.Decoder(model, prompt, samples, k, max_tokens=100, temperature=temperature, seed=5, share=share)
    for _ in range(steps):
        dec.step()
    got = [dec.drop(1)]
    for _ in range(4):
        dec.step()
    return dec, got + [dec.tokens[i, :n].tolist() for i, n in enumerate(dec.n_tokens.tolist())]


@pytest.mark.parametrize("k,n_prompt,temperature", [(1, 130, 1.0), (3, 300, 1.0), (4, 257, 0.0), (2, 60, 0.7)])
def test_samples_with_shared_pages_equal_samples_with_their_own(D, k, n_prompt, temperature):
    m = D.Model(seed=k)
    prompt = torch.randint(0, m.vocab, (n_prompt,), generator=torch.Generator().manual_seed(k)).tolist()
    dec, got = decode(D, m, prompt, 3, k, True, temperature)
    own, want = decode(D, m, prompt, 3, k, False, temperature)
    assert got == want and not dec.status.any() and not own.status.any()
    assert dec.shared_pages == (n_prompt - 1 + 127) // 128 and own.shared_pages == 3 * dec.shared_pages
    assert all(len(t) >= 20 for t in got)
    if temperature == 0:
        n = len(got[0])
        assert got[1][:n] == got[0] and got[2][:n] == got[0]
    else:
        assert got[1] != got[2]
    # the first layer's rows are what the tokens' embeddings give, in 4 bits, in both caches
    for d in (dec, own):
        lens = d.kv_len.tolist()
        out = [torch.zeros(2, max(lens), m.h_kv, m.d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        d.ctx.space_kvq_read(d.ctx.kvq_read_args(d.pools[0], d.table, d.kv_len, *out))
        for i, L in enumerate(lens):
            seq = torch.tensor((prompt + got[1 + i])[:L], device="cuda")
            _, *kv = m.qkv(0, m.embed(seq[None], torch.arange(L, device="cuda")[None]))
            for x, o in zip(kv, out):
                x = x[0].double().cpu().numpy()
                v = kvq.values(x)
                # the projection's own rounding may differ by a unit of bf16 between calls of other shapes: 2^-8 of an element,
                # which moves a code by one at most
                step = (x.max(-1, keepdims=True) - x.min(-1, keepdims=True)) / 15
                assert np.abs(o[i, :L].double().cpu().numpy() - v).max() <= (1.1 * step + 2.0 ** -7 * np.abs(x).max(-1, keepdims=True)).max()
                assert (np.abs(o[i, :L].double().cpu().numpy() - v) <= 2.0 ** -8 * np.abs(v) + 1e-6).mean() > 0.9
