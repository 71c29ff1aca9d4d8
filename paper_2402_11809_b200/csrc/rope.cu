// Rotated rows into the bf16 cache (space_rope_append).
//
// Bytes read once and written once, 4 d per row and head, beside a table row of 4 rot_dim bytes per row that all its heads share (out of the
// first-level cache).  d / 8 lanes have a row of one head, a thread PAIRS of (row, head), whose loads are all on their way before the
// first is used.  The order is sequence, row, head: q, then K, then V heads of a row, as a projection's output lies.
#include "rope_common.cuh"

namespace {
using namespace rope;

constexpr int THREADS = 256, PAIRS = 4;

struct Params {
  Table t;
  int B, rows, H_q, H_kv, n_heads;                   // heads per row: H_q (or 0), H_kv, and H_kv again where values go to a cache
  int64_t cap;                                       // rows a sequence may have (no cache: no limit)
  const char* src[3]; int64_t sb[3], sr[3], sh[3];   // q, k, v; bytes
  char* dst[2]; int64_t db[2], dr[2], dh[2];         // q_out, k_out; bytes
  char* cache[2]; int64_t cb, ch, cs;                // K, V; bytes
  const int32_t* page_table; int pages_per_seq, n_pages;
  const int32_t* kv_len; const int32_t* count; int32_t* len_out; int32_t* status;
};

template <int DH>
__global__ void __launch_bounds__(THREADS) rope_append_kernel(const __grid_constant__ Params p) {
  constexpr int LANES = DH / 8, SLOTS = THREADS / LANES;
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.y, x = threadIdx.x % LANES;
  const int L = p.kv_len[b];
  const int want = p.count ? p.count[b] : p.rows;
  const int n = max(0, min(want, p.rows));
  const bool fits = !p.cache[0] || (L >= 0 && (int64_t)L + n <= p.cap);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (!fits && p.status) atomicOr(p.status + b, SPACE_ST_CAPACITY);
    if (p.len_out) p.len_out[b] = fits ? L + n : L;
  }
  const uint32_t pair0 = blockIdx.x * (uint32_t)(SLOTS * PAIRS) + threadIdx.x / LANES;
  if (!fits || blockIdx.x * (uint32_t)(SLOTS * PAIRS) >= (uint32_t)n * (uint32_t)p.n_heads) return;
  uint4 v[PAIRS];
  Turn u[PAIRS];
  char* to[PAIRS];
  bool turned[PAIRS];
#pragma unroll
  for (int j = 0; j < PAIRS; ++j) {
    const uint32_t pair = pair0 + j * SLOTS;
    const int r = (int)(pair / (uint32_t)p.n_heads), g = (int)(pair - (uint32_t)r * p.n_heads);
    v[j] = make_uint4(0, 0, 0, 0);
    to[j] = nullptr;
    turned[j] = false;
    if (r < n) {
      const int which = g < p.H_q ? 0 : g < p.H_q + p.H_kv ? 1 : 2;
      const int h = g - (which == 0 ? 0 : which == 1 ? p.H_q : p.H_q + p.H_kv);
      v[j] = *(reinterpret_cast<const uint4*>(p.src[which] + (int64_t)b * p.sb[which] + (int64_t)r * p.sr[which] + (int64_t)h * p.sh[which]) + x);
      if (which < 2) {
        bool bad;
        const float* row = table_row(p.t, b, p.rows, r, (int64_t)L + r, bad);
        if (bad && g == 0 && x == 0 && p.status) atomicOr(p.status + b, SPACE_ST_BAD_POSITION);
        load_turn(p.t, row, x, u[j]);
        turned[j] = true;
      }
      if (which == 0 || !p.cache[0]) {
        to[j] = p.dst[which] + (int64_t)b * p.db[which] + (int64_t)r * p.dr[which] + (int64_t)h * p.dh[which];
      } else {
        const int64_t off = kv_row_offset(p.page_table, p.pages_per_seq, p.n_pages, p.cb, p.ch, p.cs, b, h, L + r);
        if (off >= 0) to[j] = p.cache[which - 1] + off;
        else if (x == 0 && p.status) atomicOr(p.status + b, SPACE_ST_BAD_PAGE);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < PAIRS; ++j) {
    float y[8];
    turn_row<LANES>(p.t, v[j], x, u[j], y);
    if (to[j]) *(reinterpret_cast<uint4*>(to[j]) + x) = turned[j] ? pack8(y) : v[j];
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
  p.n_heads = p.H_q + p.H_kv * (cached ? 2 : 1);
  if ((int64_t)p.rows * p.n_heads > 0x7FFF0000ll) return SPACE_E_UNSUPPORTED;
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
  const int per_block = THREADS / (ctx->cfg.head_dim / 8) * PAIRS;
  const dim3 grid((unsigned)(((int64_t)p.rows * p.n_heads + per_block - 1) / per_block), p.B);
  ctx->launches += 1;
  return cuda_ok(launch_pdl(ctx->cfg.head_dim == 128 ? rope_append_kernel<128> : rope_append_kernel<64>, grid, dim3(THREADS), 0, (cudaStream_t)stream, p));
}
