"""space_attn_step on the bf16 cache that space_rope_append writes, and the commit behind it: a prompt, then steps at the block's
positions, against the 64-bit oracle."""
import math

import numpy as np
import pytest
import torch

import gpu_harness as H
from oracle import kvb
from oracle.attention import attention_step
from oracle.bf16 import bf16_bits_to_f64, f32_to_bf16_bits
from oracle.commit import commit_step
from oracle.layout import position_ids

pytestmark = pytest.mark.gpu
P = 128


@pytest.fixture(scope="module")
def B():
    from paper_2402_11809_b200 import binding
    return binding


def bits(rng, *shape):
    return f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))


def i32(x):
    return H.to_dev(np.array(x, np.int32))


def turned(x, table, pos, inter):
    return f32_to_bf16_bits(kvb.turn(bf16_bits_to_f64(x), table, pos, inter))


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("d,Hq,Hkv,k,rot,inter,impl,lens", [
    (128, 4, 4, 5, 128, False, "ATTN_TENSOR", [0, 92, 300]), (64, 8, 2, 3, 64, True, "ATTN_TENSOR", [127, 1, 128, 700]),
    (128, 8, 1, 6, 64, False, "ATTN_TENSOR_ROWS", [500]), (64, 2, 2, 1, 32, True, "ATTN_SIMT", [3, 126]), (128, 8, 2, 7, 96, False, "ATTN_TENSOR", [640, 63])])
def test_steps_on_the_cache_that_the_rotation_fills(B, d, Hq, Hkv, k, rot, inter, impl, lens, paged, captured):
    rng = np.random.default_rng(d + k)
    n, n_q, steps, scale = len(lens), (k + 1) ** 2, 3, 1 / math.sqrt(d)
    cap = (max(lens) + steps * (k + 1) + n_q + P) // P * P
    table = rng.standard_normal((cap + k, rot // 2)) * 3
    table = np.concatenate([np.cos(table), np.sin(table)], 1).astype(np.float32)
    ctx = B.Context(max_batch=n, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, k_max=k, vocab=8, s_cap=cap)
    pps, more = cap // P, {}
    if paged:
        pages = rng.permutation(n * pps + 1)[:n * pps].reshape(n, pps).astype(np.int32)
        cache = torch.full((2, n * pps + 1, Hkv, P, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        more = dict(page_table=H.to_dev(pages))
    else:
        cache = torch.full((2, n, Hkv, cap, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    angles = H.to_dev(table)
    status, kv_len, len2 = i32([0] * n), i32([0] * n), i32([0] * n)
    # the prompts, at positions 0, 1, ..: K and V as slices of one projection's output
    prompt = bits(rng, n, max(lens), 2, Hkv, d)
    pd = H.to_dev(prompt)
    want = np.zeros((2, n, Hkv, cap, d), np.uint16)
    ctx.space_rope_append(ctx.rope_append_args(B.rope(angles, inter), None, None, pd[:, :, 0], kv_len, v=pd[:, :, 1], k_cache=cache[0], v_cache=cache[1],
                                               count=i32(lens), kv_len_out=len2, status=status, **more))
    kv_len.copy_(len2)
    for b, L in enumerate(lens):
        want[0, b, :, :L] = turned(prompt[b, :L, 0], table, np.arange(L), inter).transpose(1, 0, 2)
        want[1, b, :, :L] = prompt[b, :L, 1].transpose(1, 0, 2)
    q, q_out = torch.empty(n, n_q, Hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(n, n_q, Hq, d, dtype=torch.bfloat16, device="cuda")
    kv, pos, accepted = torch.empty(n, n_q, 2, Hkv, d, dtype=torch.bfloat16, device="cuda"), i32(np.zeros((n, n_q))), i32([0] * n)
    out, lse = torch.empty(n, n_q, Hq, d, device="cuda"), torch.empty(n, Hq, n_q, device="cuda")
    args = (ctx.rope_append_args(B.rope(angles, inter, pos=pos), q, q_out, kv[:, :, 0], kv_len, v=kv[:, :, 1], k_cache=cache[0], v_cache=cache[1], status=status, **more),
            ctx.attn_args(q_out, cache[0], cache[1], kv_len, out, k, scale, lse=lse, status=status, impl=getattr(B, impl), **more),
            ctx.commit_args(cache[0], cache[1], accepted, kv_len, k, kv_len_out=len2, status=status, **more))

    def step():
        ctx.space_rope_append(args[0])
        ctx.space_attn_step(args[1])
        ctx.space_kv_commit(args[2])
    if captured:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            step()
    at = np.array(lens)
    for i in range(steps):
        qb, kb, got = bits(rng, n, n_q, Hq, d), bits(rng, n, n_q, 2, Hkv, d), rng.integers(0, k + 1, size=n)
        place = np.array([position_ids(k, int(L)) for L in at])
        q.copy_(H.to_dev(qb)); kv.copy_(H.to_dev(kb)); pos.copy_(i32(place)); accepted.copy_(i32(got))
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        turned_q = np.stack([turned(qb[b], table, place[b], inter) for b in range(n)])
        for b, L in enumerate(at):
            want[0, b, :, L:L + n_q] = turned(kb[b, :, 0], table, place[b], inter).transpose(1, 0, 2)
            want[1, b, :, L:L + n_q] = kb[b, :, 1].transpose(1, 0, 2)
        ref, ref_lse = attention_step(bf16_bits_to_f64(turned_q), bf16_bits_to_f64(want[0]), bf16_bits_to_f64(want[1]), at, k, scale)
        assert np.array_equal(H.bf16_to_bits(q_out), turned_q)
        H.check_attention(out.cpu().numpy().astype(np.float64), ref, f"step {i}")
        assert np.abs(lse.cpu().numpy() - ref_lse).max() <= 2e-3
        at, _, _ = commit_step(want[0], want[1], at, got, k)
        assert len2.tolist() == at.tolist() and not status.any()
        kv_len.copy_(len2)
    for b, L in enumerate(at):                                           # the verified rows, bit for bit
        rows = np.arange(L)
        for which in range(2):
            have = H.bf16_to_bits(cache[which])
            have = have[pages[b, rows // P], :, rows % P] if paged else have[b].transpose(1, 0, 2)[:L]
            assert np.array_equal(have, want[which, b, :, :L].transpose(1, 0, 2))
