// Entry points of the 8-bit cache: argument checks, then the launchers of kvb_rows.cu and kvb_attn.cu.
#include "common.cuh"
#include "rope_common.cuh"

namespace {
bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// What the three calls have in common.
int check_cache(const space_ctx* ctx, const space_kvb_cache& c) {
  if (!c.pool || !c.page_table || c.pages_per_seq < 1 || c.n_pages < 1 ||
      (int64_t)c.pages_per_seq * SPACE_PAGE_SIZE > (1ll << 30))
    return SPACE_E_INVALID_ARG;
  if (!aligned16(c.pool) || c.page_stride % 16 || c.head_stride % 16) return SPACE_E_ALIGNMENT;
  const int64_t head = space_kvb_page_bytes(1, ctx->cfg.head_dim);
  if ((ctx->cfg.n_kv_heads > 1 && c.head_stride < head) ||
      (c.n_pages > 1 && c.page_stride < (ctx->cfg.n_kv_heads - 1) * c.head_stride + head))
    return SPACE_E_INVALID_ARG;
  return SPACE_OK;
}
// Rows [B, r, H, d] by strides: two tensors of one shape.
int check_rows(const void* k, const void* v, int64_t sb, int64_t sr, int64_t sh) {
  if (!k || !v) return SPACE_E_INVALID_ARG;
  if (!aligned16(k) || !aligned16(v) || sb % 8 || sr % 8 || sh % 8) return SPACE_E_ALIGNMENT;
  return SPACE_OK;
}
}  // namespace

extern "C" {

int64_t space_kvb_page_bytes(int32_t n_kv_heads, int32_t head_dim) {
  if (n_kv_heads < 1 || (head_dim != 64 && head_dim != 128)) return 0;
  return (int64_t)n_kv_heads * (2 * SPACE_PAGE_SIZE * head_dim + 8 * (SPACE_PAGE_SIZE / 32));
}

int space_kvb_append(space_ctx* ctx, const space_kvb_append_args* a, void* stream) {
  if (!ctx || !a) return SPACE_E_INVALID_ARG;
  if (a->batch < 0 || a->batch > ctx->cfg.max_batch) return SPACE_E_WORKSPACE;
  if (a->rows < 0 || a->row_step < 1) return SPACE_E_INVALID_ARG;
  if (a->batch == 0) return SPACE_OK;
  if (a->rows < 1 || !a->kv_len || a->kv_len_out == a->kv_len) return SPACE_E_INVALID_ARG;
  int rc = check_rows(a->k_new, a->v_new, a->new_stride_b, a->new_stride_r, a->new_stride_h);
  if (rc == SPACE_OK) rc = check_cache(ctx, a->cache);
  if (rc == SPACE_OK && a->rope.table) rc = check_rope(ctx, a->rope);
  if (rc != SPACE_OK) return rc;
  if ((a->q != nullptr) != (a->q_out != nullptr) || (a->q && !a->rope.table)) return SPACE_E_INVALID_ARG;
  if (a->q) rc = check_rows(a->q, a->q_out, a->q_stride_b | a->q_out_stride_b, a->q_stride_r | a->q_out_stride_r, a->q_stride_h | a->q_out_stride_h);
  if (rc != SPACE_OK) return rc;
  if (cudaSetDevice(ctx->cfg.device) != cudaSuccess) return SPACE_E_CUDA;
  return launch_kvb_append(ctx, a, (cudaStream_t)stream);
}

int space_kvb_read(space_ctx* ctx, const space_kvb_read_args* a, void* stream) {
  if (!ctx || !a) return SPACE_E_INVALID_ARG;
  if (a->batch < 0 || a->batch > ctx->cfg.max_batch) return SPACE_E_WORKSPACE;
  if (a->rows < 0) return SPACE_E_INVALID_ARG;
  if (a->batch == 0 || a->rows == 0) return SPACE_OK;
  if (!a->kv_len) return SPACE_E_INVALID_ARG;
  int rc = check_rows(a->k_out, a->v_out, a->out_stride_b, a->out_stride_r, a->out_stride_h);
  if (rc == SPACE_OK) rc = check_cache(ctx, a->cache);
  if (rc != SPACE_OK) return rc;
  if (cudaSetDevice(ctx->cfg.device) != cudaSuccess) return SPACE_E_CUDA;
  return launch_kvb_read(ctx, a, (cudaStream_t)stream);
}

int space_kvb_attn_step(space_ctx* ctx, const space_kvb_attn_args* a, void* stream) {
  if (!ctx || !a) return SPACE_E_INVALID_ARG;
  if (a->batch < 0 || a->batch > ctx->cfg.max_batch || a->k > ctx->cfg.k_max) return SPACE_E_WORKSPACE;
  if (a->k < 0 || (a->mask_variant != SPACE_MASK_SAME_GROUP && a->mask_variant != SPACE_MASK_EQ5_LITERAL))
    return SPACE_E_INVALID_ARG;
  if (a->batch == 0) return SPACE_OK;
  if (!a->q || !a->out || !a->kv_len || !(a->scale > 0.f) || (a->k_new == nullptr) != (a->v_new == nullptr))
    return SPACE_E_INVALID_ARG;
  if (!aligned16(a->q) || !aligned16(a->out) || a->q_stride_b % 8 || a->q_stride_r % 8 || a->q_stride_h % 8)
    return SPACE_E_ALIGNMENT;
  int rc = a->k_new ? check_rows(a->k_new, a->v_new, a->new_stride_b, a->new_stride_r, a->new_stride_h) : SPACE_OK;
  if (rc == SPACE_OK) rc = check_cache(ctx, a->cache);
  if (rc != SPACE_OK) return rc;
  if (cudaSetDevice(ctx->cfg.device) != cudaSuccess) return SPACE_E_CUDA;
  space_layout_t lay;
  lay.mask[0] = 1;                                   // a single row sees itself
  if (a->k > 0 && (rc = space_layout(a->k, a->mask_variant, &lay)) != SPACE_OK) return rc;
  return launch_kvb_attn(ctx, a, lay.mask, (cudaStream_t)stream);
}

}  // extern "C"
