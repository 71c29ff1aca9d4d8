"""Penalties, biases and masks on logits, and token counts, on the GPU: every bit against fp32 arithmetic on the host."""
import numpy as np
import pytest
import torch

from oracle.bf16 import bf16_bits_to_f64, f32_to_bf16_bits

pytestmark = pytest.mark.gpu
PROMPT = 1 << 30


@pytest.fixture(scope="module")
def B():
    from paper_2402_11809_b200 import binding
    return binding


def dev(a):
    if a.dtype == np.uint16:
        return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda().view(torch.bfloat16)
    if a.dtype == np.uint32:
        a = a.view(np.int32)
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def i32(x):
    return dev(np.array(x, np.int32))


def adjusted(z, k, counts=None, cand=None, rep=None, pres=None, freq=None, bias_tok=None, bias_val=None, bits=None, mask_row=None):
    """z [B, n, V] fp32, each operation rounded to it; -> z and which rows have no token left."""
    Bn, n, V = z.shape
    z, empty, f = z.copy(), np.zeros((Bn, n), bool), np.float32
    for b in range(Bn):
        c = np.zeros(V, np.int64) if counts is None else counts[b].astype(np.int64)
        for i in range(n):
            times, prompt = np.minimum(c & (PROMPT - 1), (1 << 24) - 1), (c & PROMPT) != 0
            for t in ([] if cand is None else cand[b, :i // (k + 1)]):
                if 0 <= t < V:
                    times[t] += 1
            times = np.minimum(times, (1 << 24) - 1)
            x = z[b, i]
            r = f(1) if rep is None else rep[b]
            x = np.where((times > 0) | prompt, np.where(x > 0, x / r, x * r), x).astype(f)
            with np.errstate(invalid="ignore"):
                y = (x - (f(0) if freq is None else freq[b]) * times.astype(f)).astype(f) - (f(0) if pres is None else pres[b])
            x = np.where(times > 0, y, x).astype(f)
            if bias_tok is not None:
                total = {}
                for t, v in zip(bias_tok[b], bias_val[b]):
                    if 0 <= t < V:
                        total[t] = f(total[t] + v) if t in total else v
                for t, v in total.items():
                    x[t] = f(x[t] + v)
            if bits is not None and 0 <= mask_row[b, i] < bits.shape[0]:
                allow = ((bits[mask_row[b, i]][np.arange(V) // 32] >> (np.arange(V) % 32)) & 1) != 0
                x = np.where(allow, x, f(-np.inf))
                empty[b, i] = not allow.any()
            z[b, i] = x
    return z, empty


# B, k, V, dtype, history, biases, masks, kept share
CASES = [
    (1, 0, 1, "f32", 0, 1, 1, 1.0), (3, 0, 7, "bf16", 4, 2, 0, 1.0), (2, 0, 5000, "f32", 300, 40, 0, 1.0), (5, 0, 4096, "bf16", 900, 0, 3, 0.3),
    (3, 0, 50257, "f32", 700, 300, 2, 0.01), (4, 0, 128256, "bf16", 2000, 16, 0, 1.0), (2, 1, 33, "f32", 20, 8, 4, 0.5),
    (3, 2, 1021, "bf16", 200, 1024, 5, 0.02), (2, 3, 32000, "f32", 400, 5, 0, 1.0), (4, 5, 2049, "bf16", 100, 3, 24, 0.02),
    (1, 7, 12345, "bf16", 500, 17, 9, 0.9), (2, 7, 4099, "f32", 50, 0, 64, 0.001), (9, 4, 300, "bf16", 0, 0, 7, 0.5), (2, 6, 2047, "f32", 3000, 0, 0, 1.0),
]


@pytest.mark.parametrize("place", ["out", "in place", "odd rows"])
@pytest.mark.parametrize("Bn,k,V,dtype,history,n_bias,n_masks,keep", CASES)
def test_adjust(B, Bn, k, V, dtype, history, n_bias, n_masks, keep, place):
    rng = np.random.default_rng(V + k + n_bias)
    n = (k + 1) ** 2
    z = (rng.standard_normal((Bn, n, V)) * 4).astype(np.float32)
    z[0, 0, V // 2] = -np.inf
    z[Bn - 1, n - 1, V // 3] = np.nan
    raw = z if dtype == "f32" else f32_to_bf16_bits(z)
    if dtype == "bf16":
        z = bf16_bits_to_f64(raw).astype(np.float32)
    a = {}
    if history:
        c = np.zeros((Bn, V), np.int32)
        for b in range(Bn):
            np.add.at(c[b], (V * rng.random(history) ** 3).astype(int), 1)
            c[b, rng.integers(0, V, size=history // 2)] |= PROMPT
        c[0, 0] = (1 << 25) + 5                                          # more than are counted
        a["counts"] = c
    if k:
        a["cand"] = (V * rng.random((Bn, k)) ** 3).astype(np.int32)
        a["cand"][0, 0] = -1
        a["cand"][-1, -1] = V
        if k > 2:
            a["cand"][:, 2] = a["cand"][:, 1]                            # the same candidate twice
    a["rep"], a["pres"], a["freq"] = (rng.uniform(lo, hi, Bn).astype(np.float32) for lo, hi in ((0.8, 1.6), (-0.5, 1.0), (0.0, 0.5)))
    if n_bias:
        a["bias_tok"] = rng.integers(-1, V + 1, size=(Bn, n_bias)).astype(np.int32)
        a["bias_tok"][:, n_bias // 2:] = np.where(rng.random((Bn, n_bias - n_bias // 2)) < 0.3, a["bias_tok"][:, :1], a["bias_tok"][:, n_bias // 2:])
        a["bias_val"] = rng.standard_normal((Bn, n_bias)).astype(np.float32)
        a["bias_val"][0, 0] = -np.inf
    if n_masks:
        words = (V + 31) // 32
        allow = rng.random((n_masks, words * 32)) < keep
        allow[0] = False                                                 # leaves nothing
        allow[0, V:] = True                                              # (bits behind the vocabulary allow no token)
        a["bits"] = (allow.reshape(n_masks, words, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
        a["mask_row"] = rng.integers(-1, n_masks, size=(Bn, n)).astype(np.int32)
    with np.errstate(invalid="ignore"):
        want, empty = adjusted(z, k, **a)
    ctx = B.Context(max_batch=Bn, n_q_heads=1, n_kv_heads=1, head_dim=64, k_max=max(k, 1), vocab=V, s_cap=128)
    if place == "odd rows":                                              # rows of another stride than the vocabulary's, not on the grid
        big = torch.zeros(Bn * n * (V + 3) + 1, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
        src = big[1:].view(Bn, n, V + 3)[:, :, :V]
        src.copy_(dev(raw))
        room = torch.full((Bn * n * (V + 5) + 3,), 7.0, dtype=src.dtype, device="cuda")
        out = room[3:].view(Bn, n, V + 5)[:, :, :V]
    else:
        src = dev(raw)
        out = src if place == "in place" else torch.full_like(src, 7.0)
    before = src.clone()
    status = i32([0] * Bn)
    names = dict(rep="repetition", pres="presence", freq="frequency", bits="mask_bits")
    keep_alive = {names.get(x, x): dev(v) for x, v in a.items()}
    call = lambda: ctx.space_logits_adjust(ctx.logits_adjust_args(src, out, k, status=status, **keep_alive))
    n0 = ctx.launch_count
    call()
    assert ctx.launch_count == n0 + 1
    got = out.float().cpu().numpy()
    if dtype == "bf16":
        w16 = torch.from_numpy(want).to(torch.bfloat16).float().numpy()  # nearest, ties to even
    else:
        w16 = want
    assert np.array_equal(got, w16, equal_nan=True), np.argwhere(~((got == w16) | (np.isnan(got) & np.isnan(w16))))[:5]
    assert status.tolist() == [B.ST_BAD_MASK if e.any() else 0 for e in empty]
    if place != "in place":
        assert torch.equal(src.view(torch.int32 if dtype == "f32" else torch.int16), before.view(torch.int32 if dtype == "f32" else torch.int16)) \
            if place == "out" else True
        out.fill_(7.0)
        call()                                                           # the same once more, the counters of before put back
        assert np.array_equal(out.float().cpu().numpy(), w16, equal_nan=True)
    if place == "odd rows":                                              # nothing beside the rows
        assert (room[:3] == 7).all() and (room[3:].view(Bn, n, V + 5)[:, :, V:] == 7).all()


def test_mask_numbers_and_no_status(B):
    V, k, Bn = 100, 1, 2
    ctx = B.Context(max_batch=Bn, n_q_heads=1, n_kv_heads=1, head_dim=64, k_max=1, vocab=V, s_cap=128)
    z = torch.randn(Bn, 4, V, device="cuda")
    bits = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    bits[0] = -1
    rows, status = i32([[0, -5, 2, 2 ** 31 - 1], [0, 0, -1, 0]]), i32([0, 0])
    out = torch.empty_like(z)
    ctx.space_logits_adjust(ctx.logits_adjust_args(z, out, k, mask_bits=bits, mask_row=rows, status=status))
    assert torch.equal(out, z) and status.tolist() == [B.ST_BAD_MASK, 0]         # a number from n_masks on: as without a mask
    rows[1, 3] = 1
    ctx.space_logits_adjust(ctx.logits_adjust_args(z, out, k, mask_bits=bits, mask_row=rows))
    assert torch.equal(out[0], z[0]) and torch.equal(out[1, :3], z[1, :3]) and (out[1, 3] == -float("inf")).all()


@pytest.mark.parametrize("mode", ["sample", "greedy"])
def test_rows_without_a_token_do_not_stop_verification(B, mode):
    """What the verification makes of adjusted logits: tokens that a mask forbids are never taken."""
    V, k, Bn = 300, 3, 4
    rng = np.random.default_rng(0)
    ctx = B.Context(max_batch=Bn, n_q_heads=1, n_kv_heads=1, head_dim=64, k_max=k, vocab=V, s_cap=128)
    n = (k + 1) ** 2
    z = dev(rng.standard_normal((Bn, n, V)).astype(np.float32))
    allow = np.zeros((1, 10 * 32), bool)
    allow[0, [5, 77, 299]] = True
    bits = dev((allow.reshape(1, 10, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32))
    ctx.space_logits_adjust(ctx.logits_adjust_args(z, z, k, mask_bits=bits, mask_row=i32(np.zeros((Bn, n)))))
    cand = i32(np.full((Bn, k), 5))
    f32 = lambda *s: torch.zeros(*s, device="cuda")
    outs = [i32(np.zeros(Bn)), i32(np.zeros((Bn, k + 1))), i32(np.zeros(Bn)), i32(np.zeros((Bn, k))), f32(Bn, k), torch.zeros(Bn, dtype=torch.uint8, device="cuda")]
    status = i32(np.zeros(Bn))
    ctx.space_verify(ctx.verify_args(z, cand, f32(Bn, k) + 0.5, i32(np.full(Bn, 10)), *outs, k, mode=B.MODE_SAMPLE if mode == "sample" else B.MODE_GREEDY,
                                     temperature=1.0, seed=3, seq_id=i32(np.arange(Bn)), status=status))
    taken = outs[1].cpu().numpy()
    for b in range(Bn):
        assert set(taken[b, :int(outs[2][b])]) <= {5, 77, 299} and set(outs[3][b].tolist()) <= {5, 77, 299}


COUNTS = [(1, 5, 1), (3, 100, 7), (2, 50257, 256), (2, 50257, 257), (4, 8192, 3000), (3, 8193, 2048), (2, 128256, 4001)]


@pytest.mark.parametrize("lens", [False, True])
@pytest.mark.parametrize("Bn,V,n", COUNTS)
def test_counts(B, Bn, V, n, lens):
    rng = np.random.default_rng(V + n)
    tokens = (V * rng.random((Bn, n + 3)) ** 3).astype(np.int32)
    tokens[:, 0], tokens[:, n // 2] = -1, V
    many = rng.integers(-3, n + 9, size=Bn).astype(np.int32)
    ctx = B.Context(max_batch=Bn, n_q_heads=1, n_kv_heads=1, head_dim=64, k_max=1, vocab=V, s_cap=128)
    td = dev(tokens)[:, :n]                                              # rows by stride
    want = np.zeros((Bn, V), np.int64)
    counts = torch.full((Bn, V), 99, dtype=torch.int32, device="cuda")
    for prompt, reset in ((False, True), (True, False), (False, False), (True, True), (False, False)):
        if reset:
            want[:] = 0
        for b in range(Bn):
            t = tokens[b, :min(max(many[b], 0), n) if lens else n]
            t = t[(t >= 0) & (t < V)]
            if prompt:
                want[b, t] |= PROMPT
            else:
                np.add.at(want[b], t, 1)
        ctx.space_token_counts(ctx.token_counts_args(td, counts, n_tokens=dev(many) if lens else None, prompt=prompt, reset=reset))
        assert (counts.cpu().numpy() == want).all()
    n0 = ctx.launch_count
    ctx.space_token_counts(ctx.token_counts_args(td[:, :0], counts))
    assert ctx.launch_count == n0
    ctx.space_token_counts(ctx.token_counts_args(td[:, :0], counts, reset=True))
    assert not counts.any()


def test_refusals(B):
    V, k, Bn = 40, 1, 2
    ctx = B.Context(max_batch=Bn, n_q_heads=1, n_kv_heads=1, head_dim=64, k_max=1, vocab=V, s_cap=128)
    z, f = torch.zeros(Bn, 4, V, device="cuda"), torch.zeros(Bn, 4, V, device="cuda")
    more = dict(bias_tok=i32(np.zeros((Bn, 3))), bias_val=torch.zeros(Bn, 3, device="cuda"), mask_bits=i32(np.zeros((2, 2))), mask_row=i32(np.zeros((Bn, 4))))
    adjust = lambda: ctx.logits_adjust_args(z, f, k, **more)
    tokens, counts = i32(np.zeros((Bn, 3))), i32(np.zeros((Bn, V)))
    count = lambda: ctx.token_counts_args(tokens, counts)
    cases = [(adjust, "space_logits_adjust", "batch", 3, B.E_WORKSPACE), (adjust, "space_logits_adjust", "k", 2, B.E_WORKSPACE),
             (adjust, "space_logits_adjust", "k", -1, B.E_INVALID_ARG), (adjust, "space_logits_adjust", "vocab", 41, B.E_WORKSPACE),
             (adjust, "space_logits_adjust", "vocab", 0, B.E_WORKSPACE), (adjust, "space_logits_adjust", "dtype", 7, B.E_INVALID_ARG),
             (adjust, "space_logits_adjust", "logits", 0, B.E_INVALID_ARG), (adjust, "space_logits_adjust", "out", 0, B.E_INVALID_ARG),
             (adjust, "space_logits_adjust", "logits", z.data_ptr() + 2, B.E_ALIGNMENT), (adjust, "space_logits_adjust", "out_row_stride", 39, B.E_INVALID_ARG),
             (adjust, "space_logits_adjust", "n_bias", 1025, B.E_INVALID_ARG), (adjust, "space_logits_adjust", "n_bias", -1, B.E_INVALID_ARG),
             (adjust, "space_logits_adjust", "bias_val", 0, B.E_INVALID_ARG), (adjust, "space_logits_adjust", "mask_row", 0, B.E_INVALID_ARG),
             (adjust, "space_logits_adjust", "n_masks", 0, B.E_INVALID_ARG), (count, "space_token_counts", "batch", 3, B.E_WORKSPACE),
             (count, "space_token_counts", "vocab", 41, B.E_WORKSPACE), (count, "space_token_counts", "n", -1, B.E_INVALID_ARG),
             (count, "space_token_counts", "tokens", 0, B.E_INVALID_ARG), (count, "space_token_counts", "counts", 0, B.E_INVALID_ARG)]
    n0 = ctx.launch_count
    for make, call, field, value, code in cases:
        a = make()
        setattr(a, field, value)
        with pytest.raises(B.SpaceError) as e:
            getattr(ctx, call)(a)
        assert e.value.code == code, (call, field, value, e.value.code)
    a = ctx.logits_adjust_args(z, z, k)
    a.out_row_stride = V + 4                                             # in place with another stride
    with pytest.raises(B.SpaceError):
        ctx.space_logits_adjust(a)
    assert ctx.launch_count == n0
