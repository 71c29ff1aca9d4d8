"""What the binding of the 8-bit cache, of the rotation and of the logits' adjustment refuses before it hands addresses to
the library.  Nothing is launched; tensors that say they are on a device stand in for such."""
import pytest
import torch

BATCH, HQ, HKV, D, PPS, PAGES, K, V = 3, 4, 2, 64, 2, 8, 1, 40
N_Q = (K + 1) ** 2


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)


def on_device(*shape, dtype=torch.int32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


def bf16(*shape):
    return on_device(*shape, dtype=torch.bfloat16)


def f32(*shape):
    return on_device(*shape, dtype=torch.float32)


@pytest.fixture(scope="module")
def B():
    from paper_2402_11809_b200 import build
    build.build()
    from paper_2402_11809_b200 import binding
    return binding


def context(B):
    ctx = B.Context.__new__(B.Context)               # (no device is asked for)
    ctx.cfg, ctx._h = B.Config(max_batch=BATCH, n_q_heads=HQ, n_kv_heads=HKV, head_dim=D, k_max=7, vocab=V, s_cap=256), None
    return ctx


def calls(B):
    """Each call with good arguments, by name."""
    pool = on_device(PAGES, HKV, B.kvb_page_bytes(1, D), dtype=torch.uint8)
    cache = dict(pool=pool, page_table=on_device(BATCH, PPS), kv_len=on_device(BATCH), status=on_device(BATCH))
    rope = B.rope(f32(100, 32), pos=on_device(BATCH, N_Q))
    rows = lambda h=HKV: bf16(BATCH, N_Q, h, D)
    return {
        "kvb_attn_args": dict(cache, q=rows(HQ), out=rows(HQ), k=K, scale=0.1, k_new=rows(), v_new=rows(), lse=f32(BATCH, HQ, N_Q)),
        "kvb_append_args": dict(cache, k_new=rows(), v_new=rows(), count=on_device(BATCH), kv_len_out=on_device(BATCH), rope=rope,
                                q=rows(HQ), q_out=rows(HQ)),
        "kvb_read_args": dict(cache, k_out=rows(), v_out=rows(), first=on_device(BATCH)),
        "rope_append_args": dict(rope=rope, q=rows(HQ), q_out=rows(HQ), k=rows(), v=rows(), kv_len=on_device(BATCH), status=on_device(BATCH),
                                 k_cache=bf16(PAGES, HKV, 128, D), v_cache=bf16(PAGES, HKV, 128, D), count=on_device(BATCH),
                                 kv_len_out=on_device(BATCH), page_table=on_device(BATCH, PPS)),
        "logits_adjust_args": dict(logits=f32(BATCH, N_Q, V), out=f32(BATCH, N_Q, V), k=K, counts=on_device(BATCH, V), cand=on_device(BATCH, K),
                                   repetition=f32(BATCH), presence=f32(BATCH), frequency=f32(BATCH), bias_tok=on_device(BATCH, 5),
                                   bias_val=f32(BATCH, 5), mask_bits=on_device(3, 2), mask_row=on_device(BATCH, N_Q), status=on_device(BATCH)),
        "token_counts_args": dict(tokens=on_device(BATCH, 7), counts=on_device(BATCH, V), n_tokens=on_device(BATCH)),
    }


NAMES = ["kvb_attn_args", "kvb_append_args", "kvb_read_args", "rope_append_args", "logits_adjust_args", "token_counts_args"]
OPTIONAL = ("status", "count", "kv_len_out", "first", "lse", "counts", "cand", "repetition", "presence", "frequency", "n_tokens")


@pytest.mark.parametrize("call", NAMES)
def test_good_arguments(B, call):
    args = calls(B)[call]
    a = getattr(context(B), call)(**args)
    assert a.batch == BATCH
    if "pool" in args:
        assert a.kv_len == args["kv_len"].data_ptr() and a.cache.pages_per_seq == PPS and a.cache.head_stride == B.kvb_page_bytes(1, D)
    if "rope" in args:
        assert (a.rope.n_pos, a.rope.rot_dim, a.rope.interleaved) == (100, 32, 0) and a.rope.pos
    for name in OPTIONAL:
        if name in args and not (call == "token_counts_args" and name == "counts"):
            assert not getattr(getattr(context(B), call)(**{**args, name: None}), name)


@pytest.mark.parametrize("call", NAMES)
def test_bad_arguments(B, call):
    ctx, args = context(B), calls(B)[call]
    bad = []
    for name, t in args.items():
        if not isinstance(t, torch.Tensor):
            continue
        bad.append((name, torch.zeros(t.shape, dtype=t.dtype)))                             # host memory
        bad.append((name, on_device(*t.shape, dtype=torch.int64 if t.dtype == torch.int32 else torch.float16)))
        if name in ("kv_len", "status", "count", "kv_len_out", "first", "n_tokens", "repetition"):
            bad.append((name, on_device(BATCH - 1, dtype=t.dtype)))
            bad.append((name, on_device(2 * BATCH, dtype=t.dtype)[::2]))
    if "pool" in args:
        bad += [("page_table", on_device(BATCH - 1, PPS)), ("page_table", on_device(BATCH, 2 * PPS)[:, ::2]), ("kv_len", None),
                ("pool", on_device(PAGES, HKV + 1, B.kvb_page_bytes(1, D), dtype=torch.uint8)),
                ("pool", on_device(PAGES, HKV, B.kvq_page_bytes(1, D), dtype=torch.uint8)),
                ("pool", on_device(PAGES, HKV, B.kvb_page_bytes(1, 128), dtype=torch.uint8))]
    if call == "kvb_attn_args":
        bad += [("lse", f32(BATCH, HQ, N_Q - 1)), ("lse", f32(BATCH, N_Q, HQ).transpose(1, 2)), ("q", bf16(BATCH, N_Q, HQ + 1, D)),
                ("out", bf16(BATCH - 1, N_Q, HQ, D)), ("k_new", bf16(BATCH - 1, N_Q, HKV, D)), ("k", K + 1), ("v_new", None), ("k_new", None)]
    if call in ("kvb_append_args", "rope_append_args"):
        bad += [("rope", B.rope(f32(100, 32), pos=on_device(BATCH, N_Q + 1))), ("rope", B.rope(f32(100, 32), pos=on_device(BATCH - 1, N_Q))),
                ("q", None), ("q_out", None), ("q", bf16(BATCH, N_Q, HQ - 1, D)), ("q_out", bf16(BATCH, N_Q + 1, HQ, D))]
    if call == "kvb_append_args":
        bad += [("rope", None)]                                                             # queries that nobody would turn
    if call == "rope_append_args":
        bad += [("k_out", bf16(BATCH, N_Q, HKV, D)), ("v_cache", None), ("v", None), ("page_table", None), ("kv_len", None),
                ("k_cache", bf16(PAGES, HKV, 64, D)), ("v_cache", bf16(PAGES, HKV + 1, 128, D))]
    if call == "logits_adjust_args":
        bad += [("k", K + 1), ("out", f32(BATCH, N_Q, V + 1)), ("out", bf16(BATCH, N_Q, V)), ("logits", f32(BATCH, V, N_Q).transpose(1, 2)),
                ("logits", f32(BATCH, N_Q + 1, V)[:, :N_Q]), ("counts", on_device(BATCH, V + 1)), ("cand", on_device(BATCH, K + 1)),
                ("bias_tok", None), ("bias_val", None), ("bias_val", f32(BATCH, 4)), ("mask_bits", None), ("mask_row", None),
                ("mask_bits", on_device(3, 3)), ("mask_row", on_device(BATCH, N_Q + 1))]
    if call == "token_counts_args":
        bad += [("tokens", on_device(7, BATCH).t()), ("counts", on_device(BATCH - 1, V)), ("counts", on_device(BATCH, 2 * V)[:, ::2])]
    for name, value in bad:
        with pytest.raises(AssertionError):
            getattr(ctx, call)(**{**args, name: value})
            pytest.fail(f"{call} takes {name} = {None if value is None else (value if isinstance(value, (int, B.Rope)) else (value.dtype, tuple(value.shape)))}", pytrace=False)


def test_rotation_tables(B):
    for t in (torch.zeros(4, 32), f32(4, 32).t(), f32(4), bf16(4, 32)):
        with pytest.raises(AssertionError):
            B.rope(t)
    for pos in (torch.zeros(2, 2, dtype=torch.int32), on_device(4), on_device(2, 2, dtype=torch.int64), on_device(2, 4)[:, ::2]):
        with pytest.raises(AssertionError):
            B.rope(f32(4, 32), pos=pos)
    t = B.rope_table(5, 16, device="cpu")
    assert t.shape == (5, 16) and (t[0, :8] == 1).all() and (t[0, 8:] == 0).all()
    assert torch.allclose(t[3, :8].double(), torch.cos(3 * 10000.0 ** (-torch.arange(8).double() / 8)), atol=1e-7)


def test_page_bytes_and_pools(B):
    assert [B.kvb_page_bytes(h, d) for h, d in ((1, 64), (1, 128), (5, 128), (0, 64), (1, 96), (-1, 64))] == [16416, 32800, 164000, 0, 0, 0]
    for d in (64, 128):
        p = B.page_pool(on_device(PAGES, HKV, B.kvb_page_bytes(1, d), dtype=torch.uint8))
        assert (p.n_pages, p.parts, p.group_rows, p.group_bytes) == (PAGES, HKV, 128, B.kvb_page_bytes(1, d))
        p = B.page_pool(on_device(PAGES, HKV, B.kvq_page_bytes(1, d), dtype=torch.uint8))
        assert (p.group_rows, p.group_bytes) == (32, B.kvq_page_bytes(1, d) // 4)


def test_sizes_are_the_headers(B, tmp_path):
    """The argument structs as a C compiler lays them out."""
    import ctypes
    import os
    import subprocess
    names = {"space_rope": B.Rope, "space_rope_args": B.RopeArgs, "space_kvb_append_args": B.KvbAppendArgs, "space_kvb_read_args": B.KvbReadArgs,
             "space_kvb_attn_args": B.KvbAttnArgs, "space_logits_args": B.LogitsArgs, "space_counts_args": B.CountsArgs}
    src = '#include <stddef.h>\n#include <stdio.h>\n#include "space.h"\nint main(void) {\n'
    for n, cls in names.items():
        src += f'printf("{n} %zu\\n", sizeof({n}));\n'
        for f, _ in cls._fields_:
            src += f'printf("{n}.{f} %zu\\n", offsetof({n}, {f}));\n'
    (tmp_path / "s.c").write_text(src + "return 0; }\n")
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.check_call(["gcc", "-I", include, str(tmp_path / "s.c"), "-o", str(tmp_path / "s")])
    for line in subprocess.check_output([str(tmp_path / "s")], text=True).splitlines():
        name, size = line.split()
        cls, _, field = name.partition(".")
        assert int(size) == (getattr(names[cls], field).offset if field else ctypes.sizeof(names[cls])), name
