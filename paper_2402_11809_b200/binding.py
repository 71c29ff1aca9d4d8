"""ctypes binding of libspace.so: the same names as include/space.h, argument
marshalling only.  Tensors are torch CUDA tensors (device memory and streams
are torch's); every step of the path runs inside the library's kernels.

Importing this module fails loudly when the compiled library is missing.
"""
import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libspace.so")

SPACE_MAX_K = 7
SPACE_MAX_ROWS = 64
OK = 0
E_INVALID_ARG, E_UNSUPPORTED, E_ALIGNMENT, E_WORKSPACE, E_CUDA, E_NO_DEVICE = -1, -2, -3, -4, -5, -6
E_STATIC_LIMIT = -7
NOALLOC_MAX_BATCH = 8
LMHEAD_MAX_ROWS = 256
MASK_SAME_GROUP, MASK_EQ5_LITERAL = 0, 1
MODE_GREEDY, MODE_SAMPLE = 0, 1
RESAMPLE_RESIDUAL_POINTMASS, RESAMPLE_PAPER_LITERAL, RESAMPLE_RESIDUAL_DRAFT = 0, 1, 2
DTYPE_BF16, DTYPE_F32 = 0, 1
ATTN_TENSOR, ATTN_SIMT, ATTN_TENSOR_ROWS = 0, 1, 2
ST_CAPACITY, ST_BAD_CANDIDATE, ST_TIMEOUT, ST_BAD_PAGE, ST_NONFINITE = 1, 2, 4, 8, 16
PAGE_SIZE = 128

EXPORTS = ["space_create", "space_destroy", "space_workspace_bytes", "space_layout",
           "space_attn_step", "space_verify", "space_verify_commit", "space_verify_greedy_noalloc",
           "space_kv_commit",
           "space_lmhead_verify", "space_sar_sft_transform", "space_decode_begin", "space_decode_advance",
           "space_step_host",
           "space_launch_count", "space_profile_enable", "space_profile_read",
           "space_debug_philox", "space_debug_wait_timeout", "space_strerror",
           "space_pager_create", "space_pager_destroy", "space_pager_admit", "space_pager_reserve",
           "space_pager_release", "space_pager_free_pages", "space_pager_rows", "space_pager_batch_table",
           "space_pager_fork", "space_pager_make_writable", "space_pager_truncate", "space_pager_compact",
           "space_pager_page_refs", "space_kvq_page_bytes", "space_kvq_append", "space_kvq_read",
           "space_kvq_attn_step", "space_pages_copy"]

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2402_11809_b200.build` "
        "(there is no CPU fallback)")
lib = C.CDLL(LIB_PATH)


class Config(C.Structure):
    _fields_ = [("device", C.c_int32), ("max_batch", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("k_max", C.c_int32),
                ("vocab", C.c_int32), ("host_staging", C.c_int32), ("s_cap", C.c_int64)]


class Layout(C.Structure):
    _fields_ = [("k", C.c_int32), ("n_q", C.c_int32),
                ("kind", C.c_uint8 * SPACE_MAX_ROWS), ("group", C.c_uint8 * SPACE_MAX_ROWS),
                ("offset", C.c_uint8 * SPACE_MAX_ROWS), ("relpos", C.c_int32 * SPACE_MAX_ROWS),
                ("mask", C.c_uint64 * SPACE_MAX_ROWS), ("target_rows", C.c_int32 * (SPACE_MAX_K + 1))]


class AttnArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("k", C.c_int32), ("mask_variant", C.c_int32),
                ("out_dtype", C.c_int32), ("impl", C.c_int32), ("scale", C.c_float),
                ("q", C.c_void_p), ("k_cache", C.c_void_p), ("v_cache", C.c_void_p),
                ("kv_stride_b", C.c_int64), ("kv_stride_h", C.c_int64), ("kv_stride_s", C.c_int64),
                ("kv_len", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p),
                ("status", C.c_void_p), ("page_table", C.c_void_p), ("pages_per_seq", C.c_int32),
                ("n_pages", C.c_int32)]


class VerifyArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("k", C.c_int32), ("vocab", C.c_int32),
                ("logits_dtype", C.c_int32), ("mode", C.c_int32), ("resample", C.c_int32),
                ("eos_id", C.c_int32), ("temperature", C.c_float), ("seed", C.c_uint64),
                ("logits", C.c_void_p), ("logits_row_stride", C.c_int64),
                ("cand", C.c_void_p), ("cand_prob", C.c_void_p), ("seq_id", C.c_void_p),
                ("kv_len", C.c_void_p), ("n_accept", C.c_void_p), ("out_tokens", C.c_void_p),
                ("n_out", C.c_void_p), ("next_cand", C.c_void_p), ("next_cand_prob", C.c_void_p),
                ("finished", C.c_void_p), ("status", C.c_void_p),
                ("top_k", C.c_int32), ("top_p", C.c_float),
                ("draft_tok", C.c_void_p), ("draft_prob", C.c_void_p),
                ("next_draft_tok", C.c_void_p), ("next_draft_prob", C.c_void_p)]


class CommitArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("k", C.c_int32), ("k_cache", C.c_void_p),
                ("v_cache", C.c_void_p), ("kv_stride_b", C.c_int64), ("kv_stride_h", C.c_int64),
                ("kv_stride_s", C.c_int64), ("n_accept", C.c_void_p), ("kv_len", C.c_void_p),
                ("kv_len_out", C.c_void_p), ("commit_src", C.c_void_p), ("commit_dst", C.c_void_p),
                ("status", C.c_void_p), ("page_table", C.c_void_p), ("pages_per_seq", C.c_int32),
                ("n_pages", C.c_int32)]


class LmHeadArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("k", C.c_int32), ("vocab", C.c_int32),
                ("hidden_dim", C.c_int32), ("eos_id", C.c_int32), ("mode", C.c_int32),
                ("resample", C.c_int32), ("temperature", C.c_float), ("seed", C.c_uint64),
                ("hidden", C.c_void_p), ("hidden_row_stride", C.c_int64),
                ("weight", C.c_void_p), ("weight_row_stride", C.c_int64),
                ("cand", C.c_void_p), ("cand_prob", C.c_void_p), ("seq_id", C.c_void_p),
                ("kv_len", C.c_void_p), ("n_accept", C.c_void_p), ("out_tokens", C.c_void_p),
                ("n_out", C.c_void_p), ("next_cand", C.c_void_p), ("next_cand_prob", C.c_void_p),
                ("finished", C.c_void_p), ("status", C.c_void_p), ("row_max", C.c_void_p),
                ("row_argmax", C.c_void_p)]


class DecodeState(C.Structure):
    _fields_ = [("batch", C.c_int32), ("k", C.c_int32), ("max_tokens", C.c_int32),
                ("mask_token_id", C.c_int32), ("mask_variant", C.c_int32), ("reserved", C.c_int32),
                ("tokens", C.c_void_p), ("n_tokens", C.c_void_p), ("last_token", C.c_void_p),
                ("cand", C.c_void_p), ("cand_prob", C.c_void_p), ("kv_len", C.c_void_p),
                ("finished", C.c_void_p), ("block_tokens", C.c_void_p), ("block_pos", C.c_void_p)]


class SarArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("seq_cap", C.c_int32), ("k", C.c_int32),
                ("mask_token_id", C.c_int32), ("pad_token_id", C.c_int32), ("ignore_index", C.c_int32),
                ("ar_threshold", C.c_uint32), ("reserved", C.c_int32),
                ("input_ids", C.c_void_p), ("labels", C.c_void_p), ("prompt_len", C.c_void_p),
                ("answer_len", C.c_void_p), ("rand_words", C.c_void_p), ("new_len", C.c_void_p),
                ("mask_start", C.c_void_p)]


class HostStepArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("k", C.c_int32), ("vocab", C.c_int32),
                ("logits_dtype", C.c_int32), ("mode", C.c_int32), ("resample", C.c_int32),
                ("eos_id", C.c_int32), ("mask_variant", C.c_int32), ("scale", C.c_float),
                ("temperature", C.c_float), ("seed", C.c_uint64),
                ("q", C.c_void_p), ("k_cache", C.c_void_p), ("v_cache", C.c_void_p),
                ("logits", C.c_void_p), ("cand", C.c_void_p), ("cand_prob", C.c_void_p),
                ("kv_len", C.c_void_p), ("out", C.c_void_p), ("n_accept", C.c_void_p),
                ("out_tokens", C.c_void_p), ("n_out", C.c_void_p), ("next_cand", C.c_void_p),
                ("next_cand_prob", C.c_void_p), ("finished", C.c_void_p), ("status", C.c_void_p),
                ("h2d_bytes", C.c_void_p), ("d2h_bytes", C.c_void_p),
                ("cache_resident", C.c_int32), ("reserved", C.c_int32)]


class KvqCache(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("page_stride", C.c_int64), ("head_stride", C.c_int64),
                ("page_table", C.c_void_p), ("pages_per_seq", C.c_int32), ("n_pages", C.c_int32)]


class KvqAppendArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("rows", C.c_int32), ("row_step", C.c_int32), ("count_bias", C.c_int32),
                ("k_new", C.c_void_p), ("v_new", C.c_void_p), ("new_stride_b", C.c_int64),
                ("new_stride_r", C.c_int64), ("new_stride_h", C.c_int64), ("cache", KvqCache),
                ("kv_len", C.c_void_p), ("count", C.c_void_p), ("kv_len_out", C.c_void_p), ("status", C.c_void_p)]


class KvqReadArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("rows", C.c_int32), ("cache", KvqCache), ("kv_len", C.c_void_p),
                ("first", C.c_void_p), ("k_out", C.c_void_p), ("v_out", C.c_void_p), ("out_stride_b", C.c_int64),
                ("out_stride_r", C.c_int64), ("out_stride_h", C.c_int64), ("status", C.c_void_p)]


class KvqAttnArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("k", C.c_int32), ("mask_variant", C.c_int32), ("scale", C.c_float),
                ("q", C.c_void_p), ("q_stride_b", C.c_int64), ("q_stride_r", C.c_int64), ("q_stride_h", C.c_int64),
                ("k_new", C.c_void_p), ("v_new", C.c_void_p), ("new_stride_b", C.c_int64),
                ("new_stride_r", C.c_int64), ("new_stride_h", C.c_int64), ("cache", KvqCache),
                ("kv_len", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p), ("status", C.c_void_p)]


class PagePool(C.Structure):
    _fields_ = [("base", C.c_void_p), ("page_stride", C.c_int64), ("part_stride", C.c_int64), ("parts", C.c_int32),
                ("group_rows", C.c_int32), ("group_bytes", C.c_int32), ("n_pages", C.c_int32)]


class PageMove(C.Structure):
    _fields_ = [("src", C.c_int32), ("dst", C.c_int32), ("rows", C.c_int32)]


lib.space_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(Config)]
lib.space_create.restype = C.c_int
lib.space_destroy.argtypes = [C.c_void_p]
lib.space_destroy.restype = None
lib.space_workspace_bytes.argtypes = [C.POINTER(Config)]
lib.space_workspace_bytes.restype = C.c_size_t
lib.space_layout.argtypes = [C.c_int, C.c_int, C.POINTER(Layout)]
lib.space_layout.restype = C.c_int
for _name, _arg in (("space_attn_step", AttnArgs), ("space_verify", VerifyArgs),
                    ("space_kv_commit", CommitArgs), ("space_step_host", HostStepArgs),
                    ("space_lmhead_verify", LmHeadArgs), ("space_kvq_append", KvqAppendArgs),
                    ("space_kvq_read", KvqReadArgs), ("space_kvq_attn_step", KvqAttnArgs)):
    getattr(lib, _name).argtypes = [C.c_void_p, C.POINTER(_arg), C.c_void_p]
    getattr(lib, _name).restype = C.c_int
lib.space_sar_sft_transform.argtypes = [C.POINTER(SarArgs), C.c_void_p]
lib.space_sar_sft_transform.restype = C.c_int
lib.space_decode_begin.argtypes = [C.c_void_p, C.POINTER(DecodeState), C.c_void_p, C.c_void_p]
lib.space_decode_begin.restype = C.c_int
lib.space_decode_advance.argtypes = [C.c_void_p, C.POINTER(DecodeState)] + [C.c_void_p] * 7
lib.space_decode_advance.restype = C.c_int
lib.space_verify_commit.argtypes = [C.c_void_p, C.POINTER(VerifyArgs), C.POINTER(CommitArgs), C.c_void_p]
lib.space_verify_commit.restype = C.c_int
lib.space_verify_greedy_noalloc.argtypes = [C.POINTER(VerifyArgs), C.c_void_p]
lib.space_verify_greedy_noalloc.restype = C.c_int
lib.space_launch_count.argtypes = [C.c_void_p]
lib.space_launch_count.restype = C.c_int64
lib.space_profile_enable.argtypes = [C.c_void_p, C.c_int]
lib.space_profile_enable.restype = C.c_int
lib.space_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_float), C.POINTER(C.c_int64)]
lib.space_profile_read.restype = C.c_int
lib.space_debug_philox.argtypes = [C.c_void_p, C.c_uint64, C.c_int64] + [C.c_void_p] * 6
lib.space_debug_philox.restype = C.c_int
lib.space_debug_wait_timeout.argtypes = [C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p]
lib.space_debug_wait_timeout.restype = C.c_int
lib.space_strerror.argtypes = [C.c_int]
lib.space_strerror.restype = C.c_char_p
lib.space_pager_create.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_void_p)]
lib.space_pager_create.restype = C.c_int
lib.space_pager_destroy.argtypes = [C.c_void_p]
lib.space_pager_destroy.restype = None
lib.space_pager_admit.argtypes = [C.c_void_p, C.POINTER(C.c_int32)]
lib.space_pager_admit.restype = C.c_int
lib.space_pager_reserve.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
lib.space_pager_reserve.restype = C.c_int
lib.space_pager_release.argtypes = [C.c_void_p, C.c_int32]
lib.space_pager_release.restype = C.c_int
lib.space_pager_free_pages.argtypes = [C.c_void_p]
lib.space_pager_free_pages.restype = C.c_int32
lib.space_pager_rows.argtypes = [C.c_void_p, C.c_int32]
lib.space_pager_rows.restype = C.c_int32
lib.space_pager_batch_table.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
lib.space_pager_batch_table.restype = C.c_int
lib.space_pager_fork.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
lib.space_pager_fork.restype = C.c_int
lib.space_pager_make_writable.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int32,
                                          C.POINTER(C.c_int32)]
lib.space_pager_make_writable.restype = C.c_int
lib.space_pager_truncate.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
lib.space_pager_truncate.restype = C.c_int
lib.space_pager_compact.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(C.c_int32)]
lib.space_pager_compact.restype = C.c_int
lib.space_pager_page_refs.argtypes = [C.c_void_p, C.c_int32]
lib.space_pager_page_refs.restype = C.c_int32
lib.space_kvq_page_bytes.argtypes = [C.c_int32, C.c_int32]
lib.space_kvq_page_bytes.restype = C.c_int64
lib.space_pages_copy.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p]
lib.space_pages_copy.restype = C.c_int


class SpaceError(RuntimeError):
    def __init__(self, code):
        self.code = code
        super().__init__(f"libspace error {code}: {lib.space_strerror(code).decode()}")


def _check(code):
    if code != OK:
        raise SpaceError(code)


def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = None


def _stream():
    """Handle of the current device's current stream.  The getters below torch.cuda.current_stream() are
    called directly: building its Stream object takes 3.5 us, more than a kernel launch (0.15 us this way)."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.current_stream()                          # initialises CUDA
        _raw_stream = (torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice)
    return _raw_stream[0](_raw_stream[1]())


def space_layout(k, mask_variant=MASK_SAME_GROUP):
    lay = Layout()
    _check(lib.space_layout(k, mask_variant, C.byref(lay)))
    return lay


def space_verify_greedy_noalloc(args):
    """Greedy verification with no context and no allocation (see include/space.h)."""
    _check(lib.space_verify_greedy_noalloc(C.byref(args), _stream()))


def space_sar_sft_transform(input_ids, labels, prompt_len, answer_len, rand_words, k, mask_token_id,
                            ar_threshold, pad_token_id=0, ignore_index=-100, new_len=None, mask_start=None):
    """SAR-SFT sample transform on int32 CUDA tensors, in place (see include/space.h)."""
    a = SarArgs(batch=input_ids.shape[0], seq_cap=input_ids.shape[1], k=k, mask_token_id=mask_token_id,
                pad_token_id=pad_token_id, ignore_index=ignore_index, ar_threshold=ar_threshold, reserved=0,
                input_ids=_ptr(input_ids), labels=_ptr(labels), prompt_len=_ptr(prompt_len),
                answer_len=_ptr(answer_len), rand_words=_ptr(rand_words), new_len=_ptr(new_len),
                mask_start=_ptr(mask_start))
    _check(lib.space_sar_sft_transform(C.byref(a), _stream()))


def space_strerror(code):
    return lib.space_strerror(code).decode()


def space_workspace_bytes(**cfg):
    return lib.space_workspace_bytes(C.byref(Config(**cfg)))


def kvq_page_bytes(n_kv_heads, head_dim):
    """Bytes of a page of the 4-bit cache: a pool is a uint8 tensor [n_pages, n_kv_heads, page_bytes(1, d)]."""
    return lib.space_kvq_page_bytes(n_kv_heads, head_dim)


def kvq_pool(n_pages, n_kv_heads, head_dim, device="cuda"):
    """An empty 4-bit page pool."""
    import torch
    return torch.zeros(n_pages, n_kv_heads, kvq_page_bytes(1, head_dim), dtype=torch.uint8, device=device)


def page_pool(t):
    """Descriptor of a page pool for space_pages_copy: a 4-bit pool (uint8 [n_pages, H_kv, bytes]), or one of the two
    pools of a bf16 cache ([n_pages, H_kv, PAGE_SIZE, d]).  Keep the tensor alive as long as the descriptor is used."""
    import torch
    assert t.is_cuda
    if t.dtype == torch.uint8:
        assert t.dim() == 3 and t.stride(2) == 1 and t.shape[2] % 4 == 0
        return PagePool(base=_ptr(t), page_stride=t.stride(0), part_stride=t.stride(1), parts=t.shape[1], group_rows=32,
                        group_bytes=t.shape[2] // 4, n_pages=t.shape[0])
    assert t.dim() == 4 and t.shape[2] == PAGE_SIZE and t.stride(3) == 1 and t.stride(2) == t.shape[3]
    e = t.element_size()
    return PagePool(base=_ptr(t), page_stride=t.stride(0) * e, part_stride=t.stride(1) * e, parts=t.shape[1], group_rows=1,
                    group_bytes=t.shape[3] * e, n_pages=t.shape[0])


def page_pools(tensors):
    """Descriptors of several pools, as space_pages_copy takes them (they keep the tensors alive)."""
    return _keeping((PagePool * len(tensors))(*map(page_pool, tensors)), *tensors)


def space_pages_copy(pools, moves):
    """Rows 0 .. rows-1 of page src to page dst in every pool.  pools: what page_pools returned, all on the current
    device; moves: int32 numpy array [n, 3] of (src, dst, rows), as Pager.make_writable and Pager.compact return it."""
    import numpy as np
    moves = np.ascontiguousarray(moves, dtype=np.int32).reshape(-1, 3)
    _check(lib.space_pages_copy(pools, len(pools), moves.ctypes.data, len(moves), _stream()))


def _keeping(args, *tensors):
    """The struct holds addresses only: the tensors live as long as it does."""
    args._tensors = tensors
    return args


def _check_i32(n, *tensors):
    """One int32 per sequence on the device, or None."""
    import torch
    for t in tensors:
        assert t is None or (t.dtype == torch.int32 and t.is_cuda and t.is_contiguous() and t.numel() >= n)


def _kvq_cache(pool, page_table, kv_len, batch):
    import torch
    assert pool.dtype == torch.uint8 and pool.is_cuda and pool.dim() == 3 and pool.stride(2) == 1
    assert page_table.dtype == torch.int32 and page_table.is_cuda and page_table.is_contiguous() and page_table.shape[0] >= batch
    assert kv_len is not None
    return KvqCache(pool=_ptr(pool), page_stride=pool.stride(0), head_stride=pool.stride(1), page_table=_ptr(page_table),
                    pages_per_seq=page_table.shape[1], n_pages=pool.shape[0])


class Context:
    """space_create / space_destroy plus the per-step entry points."""

    def __init__(self, device=0, max_batch=1, n_q_heads=32, n_kv_heads=32, head_dim=128, k_max=5,
                 vocab=32000, host_staging=0, s_cap=4096):
        self.cfg = Config(device=device, max_batch=max_batch, n_q_heads=n_q_heads,
                          n_kv_heads=n_kv_heads, head_dim=head_dim, k_max=k_max, vocab=vocab,
                          host_staging=host_staging, s_cap=s_cap)
        self._h = C.c_void_p()
        _check(lib.space_create(C.byref(self._h), C.byref(self.cfg)))

    def close(self):
        if self._h:
            lib.space_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def launch_count(self):
        return lib.space_launch_count(self._h)

    KERNELS = ("attn", "merge", "verify_target", "verify_emit", "commit", "lmhead")

    def space_profile_enable(self, on):
        _check(lib.space_profile_enable(self._h, int(on)))

    def space_profile_read(self):
        """{kernel: (summed ms, launches)} since profiling was enabled; clears the recording."""
        ms = (C.c_float * len(self.KERNELS))()
        n = (C.c_int64 * len(self.KERNELS))()
        _check(lib.space_profile_read(self._h, ms, n))
        return {name: (ms[i], n[i]) for i, name in enumerate(self.KERNELS)}

    # -- space_attn_step --------------------------------------------------
    def attn_args(self, q, k_cache, v_cache, kv_len, out, k, scale, lse=None, status=None,
                  mask_variant=MASK_SAME_GROUP, impl=ATTN_TENSOR, page_table=None):
        """page_table [B, pages_per_seq] int32: k_cache / v_cache are then pools [n_pages, H_kv, PAGE_SIZE, d]."""
        import torch
        assert q.is_contiguous() and out.is_contiguous()
        assert k_cache.stride() == v_cache.stride() and k_cache.stride(3) == 1
        return AttnArgs(batch=q.shape[0], k=k, mask_variant=mask_variant,
                        out_dtype=DTYPE_F32 if out.dtype == torch.float32 else DTYPE_BF16,
                        impl=impl, scale=scale, q=_ptr(q), k_cache=_ptr(k_cache), v_cache=_ptr(v_cache),
                        kv_stride_b=k_cache.stride(0), kv_stride_h=k_cache.stride(1),
                        kv_stride_s=k_cache.stride(2), kv_len=_ptr(kv_len), out=_ptr(out),
                        lse=_ptr(lse), status=_ptr(status), page_table=_ptr(page_table),
                        pages_per_seq=0 if page_table is None else page_table.shape[1],
                        n_pages=0 if page_table is None else k_cache.shape[0])

    def space_attn_step(self, args):
        _check(lib.space_attn_step(self._h, C.byref(args), _stream()))

    # -- space_verify -----------------------------------------------------
    def verify_args(self, logits, cand, cand_prob, kv_len, n_accept, out_tokens, n_out, next_cand,
                    next_cand_prob, finished, k, mode=MODE_GREEDY, temperature=1.0, seed=0,
                    resample=RESAMPLE_RESIDUAL_POINTMASS, eos_id=-1, seq_id=None, status=None,
                    top_k=0, top_p=1.0, draft_tok=None, draft_prob=None, next_draft_tok=None, next_draft_prob=None):
        import torch
        assert logits.stride(2) == 1 and logits.stride(0) == logits.shape[1] * logits.stride(1)
        return VerifyArgs(batch=logits.shape[0], k=k, vocab=logits.shape[2],
                          logits_dtype=DTYPE_F32 if logits.dtype == torch.float32 else DTYPE_BF16,
                          mode=mode, resample=resample, eos_id=eos_id, temperature=temperature,
                          seed=seed, logits=_ptr(logits), logits_row_stride=logits.stride(1),
                          cand=_ptr(cand), cand_prob=_ptr(cand_prob), seq_id=_ptr(seq_id),
                          kv_len=_ptr(kv_len), n_accept=_ptr(n_accept), out_tokens=_ptr(out_tokens),
                          n_out=_ptr(n_out), next_cand=_ptr(next_cand),
                          next_cand_prob=_ptr(next_cand_prob), finished=_ptr(finished),
                          status=_ptr(status), top_k=top_k, top_p=top_p,
                          draft_tok=_ptr(draft_tok), draft_prob=_ptr(draft_prob),
                          next_draft_tok=_ptr(next_draft_tok), next_draft_prob=_ptr(next_draft_prob))

    def space_verify(self, args):
        _check(lib.space_verify(self._h, C.byref(args), _stream()))

    def space_verify_commit(self, vargs, cargs):
        """space_verify + space_kv_commit in one launch less (see include/space.h)."""
        _check(lib.space_verify_commit(self._h, C.byref(vargs), C.byref(cargs), _stream()))

    # -- space_lmhead_verify ----------------------------------------------
    def lmhead_args(self, hidden, weight, cand, n_accept, out_tokens, n_out, next_cand, next_cand_prob,
                    finished, k, eos_id=-1, status=None, row_max=None, row_argmax=None, mode=MODE_GREEDY,
                    temperature=1.0, seed=0, resample=RESAMPLE_RESIDUAL_POINTMASS, cand_prob=None,
                    seq_id=None, kv_len=None):
        """hidden [B, n_q, D] and weight [V, D] bf16 CUDA tensors with contiguous last dimension."""
        assert hidden.stride(2) == 1 and weight.stride(1) == 1
        assert hidden.stride(0) == hidden.shape[1] * hidden.stride(1)
        return LmHeadArgs(batch=hidden.shape[0], k=k, vocab=weight.shape[0], hidden_dim=weight.shape[1],
                          eos_id=eos_id, mode=mode, resample=resample, temperature=temperature, seed=seed,
                          hidden=_ptr(hidden), hidden_row_stride=hidden.stride(1),
                          weight=_ptr(weight), weight_row_stride=weight.stride(0), cand=_ptr(cand),
                          cand_prob=_ptr(cand_prob), seq_id=_ptr(seq_id), kv_len=_ptr(kv_len),
                          n_accept=_ptr(n_accept), out_tokens=_ptr(out_tokens), n_out=_ptr(n_out),
                          next_cand=_ptr(next_cand), next_cand_prob=_ptr(next_cand_prob),
                          finished=_ptr(finished), status=_ptr(status), row_max=_ptr(row_max),
                          row_argmax=_ptr(row_argmax))

    def space_lmhead_verify(self, args):
        _check(lib.space_lmhead_verify(self._h, C.byref(args), _stream()))

    # -- space_kv_commit --------------------------------------------------
    def commit_args(self, k_cache, v_cache, n_accept, kv_len, k, kv_len_out=None, commit_src=None,
                    commit_dst=None, status=None, page_table=None):
        return CommitArgs(batch=n_accept.shape[0], k=k, k_cache=_ptr(k_cache), v_cache=_ptr(v_cache),
                          kv_stride_b=k_cache.stride(0), kv_stride_h=k_cache.stride(1),
                          kv_stride_s=k_cache.stride(2), n_accept=_ptr(n_accept), kv_len=_ptr(kv_len),
                          kv_len_out=_ptr(kv_len_out), commit_src=_ptr(commit_src),
                          commit_dst=_ptr(commit_dst), status=_ptr(status), page_table=_ptr(page_table),
                          pages_per_seq=0 if page_table is None else page_table.shape[1],
                          n_pages=0 if page_table is None else k_cache.shape[0])

    def space_kv_commit(self, args):
        _check(lib.space_kv_commit(self._h, C.byref(args), _stream()))

    # -- 4-bit cache ------------------------------------------------------
    def _check_rows(self, k, v):
        import torch
        assert k.dtype == v.dtype == torch.bfloat16 and k.is_cuda and v.is_cuda
        assert k.shape == v.shape and k.stride() == v.stride() and k.stride(3) == 1
        assert k.shape[2] == self.cfg.n_kv_heads and k.shape[3] == self.cfg.head_dim

    def _check_pool(self, pool):
        assert pool.shape[1] == self.cfg.n_kv_heads and pool.shape[2] == kvq_page_bytes(1, self.cfg.head_dim)

    def kvq_append_args(self, k_new, v_new, pool, page_table, kv_len, count=None, count_bias=0, row_step=1,
                        kv_len_out=None, status=None):
        """k_new / v_new [B, rows, H_kv, d] bf16 by strides.  A prompt or a token: row_step 1; the accepted rows of a
        step's block: row_step k + 1, count n_accept, count_bias 1."""
        n = k_new.shape[0]
        self._check_rows(k_new, v_new)
        self._check_pool(pool)
        _check_i32(n, kv_len, count, kv_len_out, status)
        return _keeping(KvqAppendArgs(batch=n, rows=k_new.shape[1], row_step=row_step, count_bias=count_bias,
                                      k_new=_ptr(k_new), v_new=_ptr(v_new), new_stride_b=k_new.stride(0),
                                      new_stride_r=k_new.stride(1), new_stride_h=k_new.stride(2),
                                      cache=_kvq_cache(pool, page_table, kv_len, n), kv_len=_ptr(kv_len), count=_ptr(count),
                                      kv_len_out=_ptr(kv_len_out), status=_ptr(status)),
                        k_new, v_new, pool, page_table, kv_len, count, kv_len_out, status)

    def space_kvq_append(self, args):
        _check(lib.space_kvq_append(self._h, C.byref(args), _stream()))

    def kvq_read_args(self, pool, page_table, kv_len, k_out, v_out, first=None, status=None):
        """k_out / v_out [B, rows, H_kv, d] bf16 by strides."""
        n = k_out.shape[0]
        self._check_rows(k_out, v_out)
        self._check_pool(pool)
        _check_i32(n, kv_len, first, status)
        return _keeping(KvqReadArgs(batch=n, rows=k_out.shape[1], cache=_kvq_cache(pool, page_table, kv_len, n),
                                    kv_len=_ptr(kv_len), first=_ptr(first), k_out=_ptr(k_out), v_out=_ptr(v_out),
                                    out_stride_b=k_out.stride(0), out_stride_r=k_out.stride(1), out_stride_h=k_out.stride(2),
                                    status=_ptr(status)),
                        pool, page_table, kv_len, first, k_out, v_out, status)

    def space_kvq_read(self, args):
        _check(lib.space_kvq_read(self._h, C.byref(args), _stream()))

    def kvq_attn_args(self, q, pool, page_table, kv_len, out, k, scale, k_new=None, v_new=None, lse=None, status=None,
                      mask_variant=MASK_SAME_GROUP):
        """q [B, (k+1)^2, H_q, d] and k_new / v_new [B, (k+1)^2, H_kv, d] bf16 by strides, out contiguous bf16."""
        import torch
        n = q.shape[0]
        assert q.dtype == out.dtype == torch.bfloat16 and q.is_cuda and out.is_cuda
        assert q.stride(3) == 1 and out.is_contiguous() and out.shape == q.shape
        assert q.shape[1:] == ((k + 1) ** 2, self.cfg.n_q_heads, self.cfg.head_dim)
        self._check_pool(pool)
        _check_i32(n, kv_len, status)
        assert lse is None or (lse.dtype == torch.float32 and lse.is_cuda and lse.is_contiguous() and
                               lse.numel() == n * q.shape[1] * q.shape[2])
        sb = sr = sh = 0
        assert (k_new is None) == (v_new is None)
        if k_new is not None:
            self._check_rows(k_new, v_new)
            assert k_new.shape[:2] == q.shape[:2]
            sb, sr, sh = k_new.stride()[:3]
        return _keeping(KvqAttnArgs(batch=n, k=k, mask_variant=mask_variant, scale=scale, q=_ptr(q),
                                    q_stride_b=q.stride(0), q_stride_r=q.stride(1), q_stride_h=q.stride(2), k_new=_ptr(k_new),
                                    v_new=_ptr(v_new), new_stride_b=sb, new_stride_r=sr, new_stride_h=sh,
                                    cache=_kvq_cache(pool, page_table, kv_len, n), kv_len=_ptr(kv_len), out=_ptr(out), lse=_ptr(lse),
                                    status=_ptr(status)),
                        q, k_new, v_new, pool, page_table, kv_len, out, lse, status)

    def space_kvq_attn_step(self, args):
        _check(lib.space_kvq_attn_step(self._h, C.byref(args), _stream()))

    # -- decoding loop state (Algorithm 1) ---------------------------------
    def decode_state(self, tokens, n_tokens, last_token, cand, cand_prob, kv_len, finished, block_tokens,
                     block_pos, k, mask_token_id, mask_variant=MASK_SAME_GROUP):
        return DecodeState(batch=tokens.shape[0], k=k, max_tokens=tokens.shape[1], mask_token_id=mask_token_id,
                           mask_variant=mask_variant, reserved=0, tokens=_ptr(tokens), n_tokens=_ptr(n_tokens),
                           last_token=_ptr(last_token), cand=_ptr(cand), cand_prob=_ptr(cand_prob),
                           kv_len=_ptr(kv_len), finished=_ptr(finished), block_tokens=_ptr(block_tokens),
                           block_pos=_ptr(block_pos))

    def space_decode_begin(self, state, last_prompt_token):
        _check(lib.space_decode_begin(self._h, C.byref(state), _ptr(last_prompt_token), _stream()))

    def space_decode_advance(self, state, out_tokens, n_out, next_cand, next_cand_prob, step_finished, kv_len_next):
        _check(lib.space_decode_advance(self._h, C.byref(state), _ptr(out_tokens), _ptr(n_out), _ptr(next_cand),
                                        _ptr(next_cand_prob), _ptr(step_finished), _ptr(kv_len_next), _stream()))

    # -- space_step_host --------------------------------------------------
    def space_step_host(self, args):
        _check(lib.space_step_host(self._h, C.byref(args), _stream()))

    def space_debug_wait_timeout(self, limit_ns, out4):
        """Let a bounded on-chip wait run out (see include/space.h); out4: int32 CUDA tensor of 4."""
        _check(lib.space_debug_wait_timeout(self._h, int(limit_ns), _ptr(out4), _stream()))

    def space_debug_philox(self, seed, c0, c1, c2, c3, out):
        _check(lib.space_debug_philox(self._h, seed, c0.numel(), _ptr(c0), _ptr(c1), _ptr(c2),
                                      _ptr(c3), _ptr(out), _stream()))


class Pager:
    """Page bookkeeping of a paged cache (space_pager_*): slots, pages, batch tables.  Host only."""

    def __init__(self, n_pages, pages_per_seq, max_slots):
        h = C.c_void_p()
        _check(lib.space_pager_create(n_pages, pages_per_seq, max_slots, C.byref(h)))
        self._h, self.pages_per_seq = h, pages_per_seq

    def close(self):
        if self._h:
            lib.space_pager_destroy(self._h)
            self._h = None

    __del__ = close

    def admit(self):
        s = C.c_int32(-1)
        _check(lib.space_pager_admit(self._h, C.byref(s)))
        return s.value

    def reserve(self, slot, n_rows):
        _check(lib.space_pager_reserve(self._h, slot, n_rows))

    def release(self, slot):
        _check(lib.space_pager_release(self._h, slot))

    @property
    def free_pages(self):
        return lib.space_pager_free_pages(self._h)

    def rows(self, slot):
        return lib.space_pager_rows(self._h, slot)

    def batch_table(self, slots):
        import numpy as np
        sl = np.ascontiguousarray(slots, dtype=np.int32)
        out = np.empty((len(sl), self.pages_per_seq), dtype=np.int32)
        _check(lib.space_pager_batch_table(self._h, sl.ctypes.data_as(C.c_void_p), len(sl),
                                           out.ctypes.data_as(C.c_void_p)))
        return out

    # forked slots that share pages (see include/space.h)
    def fork(self, parent, n_rows):
        s = C.c_int32(-1)
        _check(lib.space_pager_fork(self._h, parent, n_rows, C.byref(s)))
        return s.value

    def make_writable(self, slot, first_row, n_rows):
        """Moves [n, 3] (n <= 1) that space_pages_copy has to run before rows first_row .. are written."""
        return self._moves(1, lambda buf, n: lib.space_pager_make_writable(self._h, slot, first_row, n_rows, buf, 1, n))

    def truncate(self, slot, n_rows):
        _check(lib.space_pager_truncate(self._h, slot, n_rows))

    def compact(self, max_moves=1024):
        """Moves [n, 3] that space_pages_copy has to run before the next call on the cache."""
        return self._moves(max_moves, lambda buf, n: lib.space_pager_compact(self._h, buf, max_moves, n))

    def page_refs(self, page):
        return lib.space_pager_page_refs(self._h, page)

    @staticmethod
    def _moves(cap, call):
        import numpy as np
        buf, n = np.empty((max(cap, 1), 3), dtype=np.int32), C.c_int32(0)
        _check(call(buf.ctypes.data, C.byref(n)))
        return buf[:n.value]
