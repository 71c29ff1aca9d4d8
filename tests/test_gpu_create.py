"""What a context costs: a program may make one per model, and a new one when its batch grows."""
import time

import pytest

pytestmark = pytest.mark.gpu


def test_further_contexts_are_cheap():
    """The device is asked for its properties (2.4 ms) with the first context only: what is left is an allocation."""
    import torch
    from paper_2402_11809_b200 import binding as B
    torch.cuda.synchronize()
    kept, took = [], []
    for _ in range(12):
        t = time.perf_counter()
        kept.append(B.Context(max_batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, k_max=3, vocab=8, s_cap=256))
        took.append(time.perf_counter() - t)
    assert min(took[1:]) < 1.5e-3, took
