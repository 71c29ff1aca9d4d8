"""What the binding of the 4-bit cache refuses before it hands addresses to the library: tensors of another type, fewer
elements than the batch, host memory.  Nothing is launched; tensors that say they are on a device stand in for such."""
import pytest
import torch

BATCH, HQ, HKV, D, PPS, PAGES, K = 3, 4, 2, 64, 2, 8, 1
N_Q = (K + 1) ** 2


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)


def on_device(*shape, dtype=torch.int32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture(scope="module")
def B():
    from paper_2402_11809_b200 import build
    build.build()
    from paper_2402_11809_b200 import binding
    return binding


def bf16(*shape):
    return on_device(*shape, dtype=torch.bfloat16)


def calls(B):
    """Each of the three calls with good arguments, by name."""
    pool = on_device(PAGES, HKV, B.kvq_page_bytes(1, D), dtype=torch.uint8)
    cache = dict(pool=pool, page_table=on_device(BATCH, PPS), kv_len=on_device(BATCH), status=on_device(BATCH))
    return {
        "kvq_attn_args": dict(cache, q=bf16(BATCH, N_Q, HQ, D), out=bf16(BATCH, N_Q, HQ, D), k=K, scale=0.1, k_new=bf16(BATCH, N_Q, HKV, D),
                              v_new=bf16(BATCH, N_Q, HKV, D), lse=on_device(BATCH, HQ, N_Q, dtype=torch.float32)),
        "kvq_append_args": dict(cache, k_new=bf16(BATCH, 5, HKV, D), v_new=bf16(BATCH, 5, HKV, D), count=on_device(BATCH),
                                kv_len_out=on_device(BATCH)),
        "kvq_read_args": dict(cache, k_out=bf16(BATCH, 5, HKV, D), v_out=bf16(BATCH, 5, HKV, D), first=on_device(BATCH)),
    }


def context(B):
    ctx = B.Context.__new__(B.Context)               # (no device is asked for)
    ctx.cfg, ctx._h = B.Config(max_batch=BATCH, n_q_heads=HQ, n_kv_heads=HKV, head_dim=D, k_max=7, vocab=8, s_cap=256), None
    return ctx


@pytest.mark.parametrize("call", ["kvq_attn_args", "kvq_append_args", "kvq_read_args"])
def test_good_arguments(B, call):
    args = calls(B)[call]
    a = getattr(context(B), call)(**args)
    assert a.batch == BATCH and a.kv_len == args["kv_len"].data_ptr() and a.cache.pages_per_seq == PPS
    for name in ("status", "count", "kv_len_out", "first", "lse"):
        if name in args:
            assert not getattr(getattr(context(B), call)(**{**args, name: None}), name)


@pytest.mark.parametrize("call", ["kvq_attn_args", "kvq_append_args", "kvq_read_args"])
def test_bad_arguments(B, call):
    ctx, args = context(B), calls(B)[call]
    bad = []
    for name, t in args.items():
        if not isinstance(t, torch.Tensor):
            continue
        bad.append((name, torch.zeros(t.shape, dtype=t.dtype)))                             # host memory
        bad.append((name, on_device(*t.shape, dtype=torch.int64 if t.dtype == torch.int32 else torch.float16)))
        if name in ("kv_len", "status", "count", "kv_len_out", "first"):
            bad.append((name, on_device(BATCH - 1)))
            bad.append((name, on_device(2 * BATCH)[::2]))
    bad += [("page_table", on_device(BATCH - 1, PPS)), ("page_table", on_device(BATCH, 2 * PPS)[:, ::2]), ("kv_len", None),
            ("pool", on_device(PAGES, HKV + 1, B.kvq_page_bytes(1, D), dtype=torch.uint8)),
            ("pool", on_device(PAGES, HKV, B.kvq_page_bytes(1, 128), dtype=torch.uint8))]
    if call == "kvq_attn_args":
        bad += [("lse", on_device(BATCH, HQ, N_Q - 1, dtype=torch.float32)), ("lse", on_device(BATCH, N_Q, HQ, dtype=torch.float32).transpose(1, 2)),
                ("q", bf16(BATCH, N_Q, HQ + 1, D)), ("out", bf16(BATCH - 1, N_Q, HQ, D)), ("k_new", bf16(BATCH - 1, N_Q, HKV, D)), ("k", K + 1),
                ("v_new", None), ("k_new", None)]
    for name, value in bad:
        with pytest.raises(AssertionError):
            getattr(ctx, call)(**{**args, name: value})
            pytest.fail(f"{call} takes {name} = {None if value is None else (value if isinstance(value, int) else (value.dtype, tuple(value.shape)))}", pytrace=False)


def test_page_pools(B):
    kvq, bf = on_device(PAGES, HKV, B.kvq_page_bytes(1, D), dtype=torch.uint8), bf16(PAGES, HKV, B.PAGE_SIZE, D)
    assert [p.n_pages for p in B.page_pools([kvq, bf])] == [PAGES, PAGES]
    for t in (torch.zeros(kvq.shape, dtype=kvq.dtype), torch.zeros(bf.shape, dtype=bf.dtype), bf.transpose(2, 3)):
        with pytest.raises(AssertionError):
            B.page_pool(t)
            pytest.fail(str((t.dtype, t.shape)), pytrace=False)
