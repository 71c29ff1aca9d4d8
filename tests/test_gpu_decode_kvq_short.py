"""Prompts of one token, and prompts that end with a page: paper_2402_11809_b200/decode_kvq.py."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_prompt,pages", [(1, 0), (2, 1), (129, 1), (130, 2)])
def test_short_prompts(n_prompt, pages):
    from paper_2402_11809_b200 import decode_kvq as D
    m, got = D.Model(), []
    prompt = torch.randint(0, m.vocab, (n_prompt,), generator=torch.Generator().manual_seed(3)).tolist()
    for share in (True, False):
        dec = D.Decoder(m, prompt, 3, 2, max_tokens=40, share=share)
        assert dec.shared_pages == (pages if share else 3 * pages)
        assert dec.copied == (2 if share and (n_prompt - 1) % D.PAGE else 0)           # every sample but the last to write
        for _ in range(8):
            dec.step()
        got.append([dec.drop(2)] + [dec.tokens[i, :n].tolist() for i, n in enumerate(dec.n_tokens.tolist())])
        assert not dec.status.any()
    assert got[0] == got[1] and all(len(t) >= 8 for t in got[0])
