// Rotated rows into the bf16 cache (space_rope_append).
//
// Bytes read once and written once, 4 d per row and head, beside a table row of 4 rot_dim bytes per row that all its heads share:
// HBM bounds it.  A warp has a row (or, of few rows, a share of its heads) and keeps the row's cosines and sines; addresses go from
// head to head by a stride, products are taken in pairs.  4 x 5700 rows of 32 + 8 + 8 heads of 128: 90.5 us, 6.2 TB/s, 0.94 of the copy
// rate.  (A list of (row, head) pairs, table entries loaded for each: 193 us; a row of heads over a whole thread block, addresses worked
// out for every head: 125 us, bound by instructions, 175 a 16-byte vector instead of 79.)  16 x 36 rows of 32 + 32 + 32 heads: 7.9 us with eight warps
// to a row, 13.4 with two rows to a block.  (64 registers, 36 bytes of a thread spilled.)  The order is a projection's output's: q, then K, then V heads of a row.
#include "rope_common.cuh"

namespace {
using namespace rope;

constexpr int THREADS = 256, WARPS = THREADS / 32;

struct Params {
  Table t;
  int B, rows, H_q, H_kv;                            // (H_q 0: no queries)
  int share;                                         // warps that share a row
  int64_t cap;                                       // rows a sequence may have (no cache: no limit)
  const char* src[3]; int64_t sb[3], sr[3], sh[3];   // q, k, v; bytes
  char* dst[2]; int64_t db[2], dr[2], dh[2];         // q_out, k_out; bytes
  char* cache[2]; int64_t cb, ch, cs;                // K, V; bytes
  const int32_t* page_table; int pages_per_seq, n_pages;
  const int32_t* kv_len; const int32_t* count; int32_t* len_out; int32_t* status;
};

template <int DH>
__global__ void __launch_bounds__(THREADS, 4) rope_append_kernel(const __grid_constant__ Params p) {
  pdl_launch_dependents();
  pdl_wait();
  const uint32_t task = blockIdx.x * WARPS + (threadIdx.x >> 5), row_of_task = task / (uint32_t)p.share;
  const int b = blockIdx.y, part = (int)(task - row_of_task * (uint32_t)p.share);
  const int L = p.kv_len[b];
  const int want = p.count ? p.count[b] : p.rows;
  const int n = max(0, min(want, p.rows));
  const bool fits = !p.cache[0] || (L >= 0 && (int64_t)L + n <= p.cap);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (!fits && p.status) atomicOr(p.status + b, SPACE_ST_CAPACITY);
    if (p.len_out) p.len_out[b] = fits ? L + n : L;
  }
  if (!fits || row_of_task >= (uint32_t)n) return;
  const int r = (int)row_of_task;
  bool bad;
  const float* row = table_row(p.t, b, p.rows, r, (int64_t)L + r, bad);
  Turn u;
  load_turn(p.t, row, (threadIdx.x & 31) % (DH / 8), u);
  int64_t off = 0;                                   // of the cache row, head 0
  if (p.cache[0]) off = kv_row_offset(p.page_table, p.pages_per_seq, p.n_pages, p.cb, p.ch, p.cs, b, 0, L + r);
  if ((threadIdx.x & 31) == 0 && part == 0 && p.status && (bad || off < 0))
    atomicOr(p.status + b, (bad ? SPACE_ST_BAD_POSITION : 0) | (off < 0 ? SPACE_ST_BAD_PAGE : 0));
  if (p.H_q)
    row_heads<DH, true>(p.t, u, p.H_q, part, p.share, p.src[0] + (int64_t)b * p.sb[0] + (int64_t)r * p.sr[0], p.sh[0],
                        p.dst[0] + (int64_t)b * p.db[0] + (int64_t)r * p.dr[0], p.dh[0]);
  const int64_t from = (int64_t)b * p.sb[1] + (int64_t)r * p.sr[1];
  if (!p.cache[0]) {
    row_heads<DH, true>(p.t, u, p.H_kv, part, p.share, p.src[1] + from, p.sh[1], p.dst[1] + (int64_t)b * p.db[1] + (int64_t)r * p.dr[1], p.dh[1]);
  } else if (off >= 0) {
    row_heads<DH, true>(p.t, u, p.H_kv, part, p.share, p.src[1] + from, p.sh[1], p.cache[0] + off, p.ch);
    // (V heads from the other end of the warps: few heads leave some of them without K heads)
    row_heads<DH, false>(p.t, u, p.H_kv, p.share - 1 - part, p.share, p.src[2] + from, p.sh[1], p.cache[1] + off, p.ch);
  }
}

}  // namespace

int check_rope(const space_ctx* ctx, const space_rope& r) {
  if (!r.table || r.n_pos < 1 || (r.interleaved != 0 && r.interleaved != 1)) return SPACE_E_INVALID_ARG;
  if ((uintptr_t)r.table & 15u) return SPACE_E_ALIGNMENT;
  if (r.rot_dim < 16 || r.rot_dim > ctx->cfg.head_dim || r.rot_dim % 16) return SPACE_E_UNSUPPORTED;
  return SPACE_OK;
}

extern "C" int space_rope_append(space_ctx* ctx, const space_rope_args* a, void* stream) {
  if (!ctx || !a) return SPACE_E_INVALID_ARG;
  if (a->batch < 0 || a->batch > ctx->cfg.max_batch) return SPACE_E_WORKSPACE;
  if (a->rows < 0) return SPACE_E_INVALID_ARG;
  if (a->batch == 0) return SPACE_OK;
  const bool cached = a->k_cache != nullptr;
  if (a->rows < 1 || !a->k || !a->kv_len || a->kv_len_out == a->kv_len || (a->q != nullptr) != (a->q_out != nullptr) ||
      cached == (a->k_out != nullptr) || cached != (a->v_cache != nullptr) || (cached && !a->v))
    return SPACE_E_INVALID_ARG;
  const int rc = check_rope(ctx, a->rope);
  if (rc != SPACE_OK) return rc;
  const void* bases[] = {a->q, a->q_out, a->k, a->v, a->k_out, a->k_cache, a->v_cache};
  for (const void* p : bases)
    if ((uintptr_t)p & 15u) return SPACE_E_ALIGNMENT;
  const int64_t strides[] = {a->q_stride_b, a->q_stride_r, a->q_stride_h, a->q_out_stride_b, a->q_out_stride_r, a->q_out_stride_h,
                             a->new_stride_b, a->new_stride_r, a->new_stride_h, a->k_out_stride_b, a->k_out_stride_r, a->k_out_stride_h,
                             a->kv_stride_b, a->kv_stride_h, a->kv_stride_s};
  for (int64_t s : strides)
    if (s % 8) return SPACE_E_ALIGNMENT;
  if (cached && a->kv_stride_s < ctx->cfg.head_dim) return SPACE_E_INVALID_ARG;
  if (cached && a->page_table && (a->pages_per_seq < 1 || a->n_pages < 1 || (int64_t)a->pages_per_seq * SPACE_PAGE_SIZE > ctx->cfg.s_cap))
    return SPACE_E_INVALID_ARG;
  Params p;
  memset(&p, 0, sizeof(p));
  p.t = rope::table_of(a->rope);
  p.B = a->batch; p.rows = a->rows; p.H_q = a->q ? ctx->cfg.n_q_heads : 0; p.H_kv = ctx->cfg.n_kv_heads;
  if (cudaSetDevice(ctx->cfg.device) != cudaSuccess) return SPACE_E_CUDA;
  p.cap = a->page_table ? (int64_t)a->pages_per_seq * SPACE_PAGE_SIZE : ctx->cfg.s_cap;
  p.src[0] = (const char*)a->q; p.sb[0] = 2 * a->q_stride_b; p.sr[0] = 2 * a->q_stride_r; p.sh[0] = 2 * a->q_stride_h;
  p.src[1] = (const char*)a->k; p.src[2] = (const char*)a->v;
  for (int i = 1; i < 3; ++i) { p.sb[i] = 2 * a->new_stride_b; p.sr[i] = 2 * a->new_stride_r; p.sh[i] = 2 * a->new_stride_h; }
  p.dst[0] = (char*)a->q_out; p.db[0] = 2 * a->q_out_stride_b; p.dr[0] = 2 * a->q_out_stride_r; p.dh[0] = 2 * a->q_out_stride_h;
  p.dst[1] = (char*)a->k_out; p.db[1] = 2 * a->k_out_stride_b; p.dr[1] = 2 * a->k_out_stride_r; p.dh[1] = 2 * a->k_out_stride_h;
  p.cache[0] = (char*)a->k_cache; p.cache[1] = (char*)a->v_cache;
  p.cb = 2 * a->kv_stride_b; p.ch = 2 * a->kv_stride_h; p.cs = 2 * a->kv_stride_s;
  p.page_table = a->page_table; p.pages_per_seq = a->pages_per_seq; p.n_pages = a->n_pages;
  p.kv_len = a->kv_len; p.count = a->count; p.len_out = a->kv_len_out; p.status = a->status;
  p.share = rope::warps_per_row((int64_t)p.B * p.rows, ctx->sm_count, WARPS);
  const dim3 grid((unsigned)(((int64_t)p.rows * p.share + WARPS - 1) / WARPS), p.B);
  ctx->launches += 1;
  return cuda_ok(launch_pdl(ctx->cfg.head_dim == 128 ? rope_append_kernel<128> : rope_append_kernel<64>, grid, dim3(THREADS), 0, (cudaStream_t)stream, p));
}
