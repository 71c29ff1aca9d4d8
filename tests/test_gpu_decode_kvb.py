"""Samples of one prompt decoded on an 8-bit cache by a model that turns queries and keys, with penalties, biases and a mask on the
logits: paper_2402_11809_b200/decode_kvq.py.  The operators of a step one after another, against a step in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import kvb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def D():
    from paper_2402_11809_b200 import build
    build.build()
    from paper_2402_11809_b200 import decode_kvq
    return decode_kvq


CONTROLS = [dict(), dict(repetition=1.3, presence=0.4, frequency=0.1), dict(frequency=0.3, bias={3: 4.0, 17: -2.0}, allowed=[0, 3, 5, 17, 20, 21, 31])]


def decode(D, model, prompt, samples, k, share, temperature, controls, steps=20):
    dec = D.Decoder(model, prompt, samples, k, max_tokens=100, temperature=temperature, seed=5, share=share, bits=8, controls=controls)
    for _ in range(steps):
        dec.step()
    got = [dec.drop(1)]
    for _ in range(4):
        dec.step()
    return dec, got + [dec.tokens[i, :n].tolist() for i, n in enumerate(dec.n_tokens.tolist())]


@pytest.mark.parametrize("k,n_prompt,temperature,which", [(1, 130, 1.0, 0), (3, 300, 1.0, 1), (4, 257, 0.0, 1), (2, 60, 0.7, 2), (5, 129, 0.0, 2)])
def test_samples_with_shared_pages_equal_samples_with_their_own(D, k, n_prompt, temperature, which):
    m = D.Model(seed=k, rotary=True)
    c = D.Controls(**CONTROLS[which])
    prompt = torch.randint(0, m.vocab, (n_prompt,), generator=torch.Generator().manual_seed(k)).tolist()
    dec, got = decode(D, m, prompt, 3, k, True, temperature, c)
    own, want = decode(D, m, prompt, 3, k, False, temperature, c)
    assert got == want and not dec.status.any() and not own.status.any()
    assert dec.shared_pages == (n_prompt - 1 + 127) // 128
    counts = dec.counts.cpu().numpy()
    for i, row in enumerate(counts):                         # what is counted is what was taken
        times = np.bincount(got[1 + i], minlength=m.vocab)
        seen = np.bincount(prompt, minlength=m.vocab) > 0
        assert ((row & ~(1 << 30)) == times).all() and (((row >> 30) & 1) == seen).all()
    if c.allowed:
        assert set(sum(got, [])) <= set(c.allowed)


def plain_step(m, tokens, start, pools, table, scale):
    """Tokens of one sample behind `start` cached rows, in 64 bits: logits of every one, K and V rows of every layer (bf16)."""
    to64 = lambda t: t.double().cpu().numpy()
    b16 = lambda a: torch.from_numpy(a).to(torch.bfloat16).double().numpy()
    n, pos = len(tokens), start + np.arange(len(tokens))
    x, angles, rows = to64(m.emb)[tokens], m.angles.cpu().numpy(), []
    for i in range(m.layers):
        q = b16(x @ to64(m.wq[i])).reshape(n, m.h_q, m.d)
        kv = b16(x @ to64(m.wkv[i])).reshape(n, 2, m.h_kv, m.d)
        q, k = b16(kvb.turn(q, angles, pos).astype(np.float64)), b16(kvb.turn(kv[:, 0], angles, pos).astype(np.float64))
        K, V = kvb.read_rows(pools[i], table, start, m.d) if start else [np.zeros((m.h_kv, 0, m.d))] * 2
        K, V = np.concatenate([K, k.transpose(1, 0, 2)], 1), np.concatenate([V, kv[:, 1].transpose(1, 0, 2)], 1)
        out = np.zeros((n, m.h_q, m.d))
        for h in range(m.h_q):
            s = q[:, h] @ K[h * m.h_kv // m.h_q].T * scale
            s[np.arange(K.shape[1])[None] > start + np.arange(n)[:, None]] = -np.inf
            p = np.exp(s - s.max(-1, keepdims=True))
            out[:, h] = p / p.sum(-1, keepdims=True) @ V[h * m.h_kv // m.h_q]
        x = x + b16(out).reshape(n, -1) @ to64(m.wo[i])
        rows.append((k, kv[:, 1]))
    return x @ to64(m.head), rows


@pytest.mark.parametrize("k,n_prompt,which", [(1, 60, 1), (3, 140, 2), (2, 33, 0), (4, 20, 1)])
def test_greedy_steps_take_what_a_step_in_64_bits_takes(D, k, n_prompt, which):
    """Every token taken has, up to the arithmetic's error, the largest adjusted logit of its row.  Rows of the model are of unit size:
    an attention's output is off by 2^-8 of itself and by 2^-8 for its rounding, two layers and the head (sd 4 in all) make
    0.06 of that at worst in these sums of 512; 0.1 is allowed, where the best two logits are 1 apart."""
    m, c = D.Model(seed=20 + k, rotary=True), D.Controls(**CONTROLS[which])
    prompt = torch.randint(0, m.vocab, (n_prompt,), generator=torch.Generator().manual_seed(k)).tolist()
    dec = D.Decoder(m, prompt, 1, k, max_tokens=60, temperature=0.0, bits=8, controls=c)
    table, scale = dec.table.cpu().numpy()[0], m.d ** -0.5
    taken, gaps = [], []
    for _ in range(12):
        start, before = int(dec.kv_len[0]), int(dec.n_tokens[0])
        pools = [p.cpu().numpy() for p in dec.pools]
        dec.step()
        new = dec.tokens[0, before:int(dec.n_tokens[0])].tolist()
        logits, rows = plain_step(m, [(prompt + taken)[-1]] + new[:-1], start, pools, table, scale)
        for i, t in enumerate(new):
            z, past = logits[i].copy(), taken + new[:i]
            times = np.bincount(past, minlength=m.vocab) if past else np.zeros(m.vocab, int)
            seen = (np.bincount(prompt, minlength=m.vocab) > 0) | (times > 0)
            z = np.where(seen, np.where(z > 0, z / c.repetition, z * c.repetition), z) - c.frequency * times - c.presence * (times > 0)
            for b, v in c.bias.items():
                z[b] += v
            if c.allowed:
                z[[x for x in range(m.vocab) if x not in c.allowed]] = -np.inf
            gaps.append(z.max() - z[t])
            assert gaps[-1] <= 0.1, (i, t, z.max(), z[t])
        taken += new
        assert int(dec.kv_len[0]) == start + len(new)
        for layer, (k_rows, v_rows) in enumerate(rows):      # and the cache holds its rows, rounded to four bits twice at most
            K, V = kvb.read_rows(dec.pools[layer].cpu().numpy(), table, start + len(new), m.d)
            for got, want in ((K, k_rows), (V, v_rows)):
                got, want = got[:, start:], want.transpose(1, 0, 2)
                assert np.abs(got - want).max() <= 2.0 ** -3 * np.abs(want).max() + 0.05
    assert np.median(gaps) == 0 and not dec.status.any()
