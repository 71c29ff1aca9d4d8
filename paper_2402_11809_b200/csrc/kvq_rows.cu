// Rows into the 4-bit cache and out of it (space_kvq_append, space_kvq_read).
//
// A row of d channels has d / 8 lanes, eight channels each.  Append: minimum and maximum by shuffles,
// step = bf16(max((hi - lo) / 15, max|x| / 4096, 2^-100)), u = round((x - lo) / step).  The quotient has to be the
// exact one at ties, which bf16 inputs meet often (a tie is a quotient n + 1/2 with few bits): one reciprocal per
// row, then per element a product and one residual step,
//   q0 = x inv,  q = q0 + (x - q0 step) inv,
// which is exact where the quotient has few bits, and off by at most an ulp elsewhere, where a quotient of these
// operands (8 bits over 8 bits) is further than 2^-16 of itself from a tie.  Everything in halves, so that
// hi - lo cannot overflow.
//
// Both kernels have two forms.  By blocks: a thread block per 32-row block of the cache; V codes, which lie transposed
// (the order of the attention's operand), are gathered in shared memory and leave in 16-byte pieces.  By rows: the
// lanes of a row store their V bytes two at a time where they belong; for the few rows of a step or a token, where
// a thread block per 32-row block would be nearly empty.
#include "kvq_common.cuh"

namespace {
using namespace kvq;

constexpr int THREADS = 256;

struct AppendParams {
  Cache cache;
  int B, H, max_count, step, bias;
  const char* src[2];                                // K, V
  int64_t sb, sr, sh;                                // bytes
  const int32_t* kv_len; const int32_t* count; int32_t* len_out; int32_t* status;
};

// Rows of sequence b that are appended, -1 where they do not fit.
__device__ __forceinline__ int append_count(const AppendParams& p, int b, int L) {
  const int64_t want = p.count ? (int64_t)p.count[b] + p.bias : (int64_t)p.max_count;
  const int n = (int)(want < 0 ? 0 : want > p.max_count ? p.max_count : want);
  return L >= 0 && (int64_t)L + n <= (int64_t)p.cache.pages_per_seq * SPACE_PAGE_SIZE ? n : -1;
}

// Codes of this lane's eight channels, channel n in bits 4n .. 4n+3, and the row's {step, lo}.
template <int LANES>
__device__ __forceinline__ uint32_t quantise(uint4 v, uint32_t& par, bool& bad) {
  bad = any_nonfinite(v);
  if (bad) v = make_uint4(finite_pair(v.x), finite_pair(v.y), finite_pair(v.z), finite_pair(v.w));
  const float x[8] = {bf_lo(v.x), bf_hi(v.x), bf_lo(v.y), bf_hi(v.y), bf_lo(v.z), bf_hi(v.z), bf_lo(v.w), bf_hi(v.w)};
  float lo = fminf(fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), fminf(fminf(x[4], x[5]), fminf(x[6], x[7])));
  float hi = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, o));
  }
  const float lo2 = 0.5f * lo;
  const float s = fmaxf(fmaxf((0.5f * hi - lo2) / 7.5f, fmaxf(-lo, hi) * (1.f / 4096.f)), 0x1p-100f);
  const __nv_bfloat16 sb = __float2bfloat16_rn(s);
  const float s2 = 0.5f * __bfloat162float(sb), inv = 1.f / s2;
  par = (uint32_t)__bfloat16_as_ushort(sb) | (__float_as_uint(lo) & 0xFFFF0000u);
  uint32_t w = 0;
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const float y = fmaf(x[n], 0.5f, -lo2);
    const float q0 = y * inv;
    const float q = fminf(fmaf(fmaf(-q0, s2, y), inv, q0), 15.f);
    w |= (__float_as_uint(q + 12582912.f) & 15u) << (4 * n);   // 1.5 * 2^23: the sum's last bit is a unit, ties to even
  }
  return w;
}

// Nibbles 0..3 of the low half as bytes.
__device__ __forceinline__ uint32_t spread(uint32_t a) {
  a = (a | a << 8) & 0x00FF00FFu;
  return (a | a << 4) & 0x0F0F0F0Fu;
}
// The lanes x, x^1, x^2, x^3 hold channels n = 0..7 of q = 0..3 (word w): this lane's two V byte pairs, those of
// n = vn, vn + 1 (low half first).
__device__ __forceinline__ uint32_t v_bytes(uint32_t w, int q, int& vn) {
  const uint32_t o = __shfl_xor_sync(0xFFFFFFFFu, w, 1);
  // the even lane joins n = 0..3, the odd one n = 4..7: low four bits from the even lane's channels
  const uint32_t even = (q & 1) ? o >> 16 : w & 0xFFFFu, odd = (q & 1) ? w >> 16 : o & 0xFFFFu;
  const uint32_t bytes = spread(even) | spread(odd) << 4;
  const uint32_t p = __shfl_xor_sync(0xFFFFFFFFu, bytes, 2);   // the same n, the other q / 2
  vn = 4 * (q & 1) + (q & 2);
  return (q & 2) ? __byte_perm(p, bytes, 0x7362) : __byte_perm(bytes, p, 0x5140);
}

template <int DH>
__global__ void __launch_bounds__(THREADS) append_rows_kernel(const AppendParams p) {
  constexpr int LANES = DH / 8;
  pdl_launch_dependents();
  pdl_wait();
  const int x = threadIdx.x % LANES;
  const int64_t idx = ((int64_t)blockIdx.x * THREADS + threadIdx.x) / LANES;
  const int which = (int)(idx & 1);
  const int64_t rest = idx >> 1;
  const int h = (int)(rest % p.H);
  const int bg = (int)(rest / p.H);
  const int b = bg / p.max_count, g = bg % p.max_count;
  int L = 0, n = 0;
  if (b < p.B) {
    L = p.kv_len[b];
    n = append_count(p, b, L);
    if (g == 0 && h == 0 && which == 0 && x == 0) {
      if (n < 0 && p.status) atomicOr(p.status + b, SPACE_ST_CAPACITY);
      if (p.len_out) p.len_out[b] = L + max(n, 0);
    }
  }
  const bool mine = g < n;
  char* blk = mine ? block_at<DH>(p.cache, b, h, L + g) : nullptr;
  if (mine && !blk && p.status && x == 0) atomicOr(p.status + b, SPACE_ST_BAD_PAGE);
  uint4 v = make_uint4(0, 0, 0, 0);
  if (blk) v = *(reinterpret_cast<const uint4*>((which ? p.src[1] : p.src[0]) + (int64_t)b * p.sb + (int64_t)g * p.step * p.sr + (int64_t)h * p.sh) + x);
  uint32_t par;
  bool bad;
  const uint32_t w = quantise<LANES>(v, par, bad);
  int vn;
  const uint32_t vb = v_bytes(w, x & 3, vn);
  if (!blk) return;
  if (bad && p.status) atomicOr(p.status + b, SPACE_ST_NONFINITE);
  const int i = (L + g) % BLOCK_ROWS;
  if (x == 0) *reinterpret_cast<uint32_t*>(blk + (which ? Fmt<DH>::V_PAR : Fmt<DH>::K_PAR) + 4 * i) = par;
  if (which == 0) {
    *reinterpret_cast<uint32_t*>(blk + i * (DH / 2) + 4 * x) = w;
  } else {
    char* at = blk + Fmt<DH>::CODES + 512 * (x >> 2) + v_row_at(i) + 64 * vn;
    *reinterpret_cast<uint16_t*>(at) = (uint16_t)vb;
    *reinterpret_cast<uint16_t*>(at + 64) = (uint16_t)(vb >> 16);
  }
}

template <int DH>
__global__ void __launch_bounds__(THREADS) append_blocks_kernel(const AppendParams p) {
  constexpr int LANES = DH / 8, ROWS = THREADS / LANES, PASSES = BLOCK_ROWS / ROWS;   // rows at a time
  __shared__ __align__(16) unsigned char vsm[Fmt<DH>::CODES];
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.z, h = blockIdx.y;
  const int L = p.kv_len[b], n = append_count(p, b, L);
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) {
    if (n < 0 && p.status) atomicOr(p.status + b, SPACE_ST_CAPACITY);
    if (p.len_out) p.len_out[b] = L + max(n, 0);
  }
  if (n <= 0) return;
  const int s0 = (L / BLOCK_ROWS + (int)blockIdx.x) * BLOCK_ROWS;      // first row of this block (may lie before L)
  if (s0 >= L + n) return;
  char* blk = block_at<DH>(p.cache, b, h, s0);
  if (!blk) {
    if (p.status && threadIdx.x == 0) atomicOr(p.status + b, SPACE_ST_BAD_PAGE);
    return;
  }
  const int x = threadIdx.x % LANES, r = threadIdx.x / LANES;
  const int i_lo = max(L - s0, 0), i_hi = min(L + n - s0, BLOCK_ROWS);  // rows of the block that are written
  uint4 v[2][PASSES];
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
      const int i = k * ROWS + r;
      v[which][k] = make_uint4(0, 0, 0, 0);
      if (i >= i_lo && i < i_hi)
        v[which][k] = *(reinterpret_cast<const uint4*>(p.src[which] + (int64_t)b * p.sb + (int64_t)(s0 + i - L) * p.step * p.sr + (int64_t)h * p.sh) + x);
    }
  bool bad_any = false;
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
      const int i = k * ROWS + r;
      const bool mine = i >= i_lo && i < i_hi;
      uint32_t par;
      bool bad;
      const uint32_t w = quantise<LANES>(v[which][k], par, bad);
      bad_any |= bad;
      if (mine && x == 0) *reinterpret_cast<uint32_t*>(blk + (which ? Fmt<DH>::V_PAR : Fmt<DH>::K_PAR) + 4 * i) = par;
      if (which == 0) {
        if (mine) *reinterpret_cast<uint32_t*>(blk + i * (DH / 2) + 4 * x) = w;
      } else {
        int vn;
        const uint32_t vb = v_bytes(w, x & 3, vn);
        unsigned char* at = vsm + 512 * (x >> 2) + v_row_at(i) + 64 * vn;
        *reinterpret_cast<uint16_t*>(at) = (uint16_t)vb;
        *reinterpret_cast<uint16_t*>(at + 64) = (uint16_t)(vb >> 16);
      }
    }
  if (bad_any && p.status) atomicOr(p.status + b, SPACE_ST_NONFINITE);
  __syncthreads();
  const int t = threadIdx.x;
  if (t * 16 < Fmt<DH>::CODES) {
    uint4* dst = reinterpret_cast<uint4*>(blk + Fmt<DH>::CODES) + t;
    const uint4 val = reinterpret_cast<const uint4*>(vsm)[t];
    if (i_lo == 0 && i_hi == BLOCK_ROWS) {
      *dst = val;
    } else {                                               // sixteen bytes are eight rows' pairs: 16a + 8e + 2t + h
      const uint32_t w[4] = {val.x, val.y, val.z, val.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = 16 * (j >> 2) + 8 * ((j >> 1) & 1) + 2 * (t & 3) + (j & 1);
        if (i >= i_lo && i < i_hi) reinterpret_cast<uint16_t*>(dst)[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
      }
    }
  }
}

struct ReadParams {
  Cache cache;
  int B, H, rows;
  char* dst[2];
  int64_t sb, sr, sh;                                // bytes
  const int32_t* kv_len; const int32_t* first; int32_t* status;
};

// Eight values lo + step * u as bf16; the codes are four bits apart in w.
__device__ __forceinline__ uint4 values(uint32_t w, uint32_t par) {
  const float s = bf_lo(par), lo = bf_hi(par);
  uint32_t r[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __nv_bfloat162 y = __floats2bfloat162_rn(fmaf((float)((w >> (8 * j)) & 15u), s, lo), fmaf((float)((w >> (8 * j + 4)) & 15u), s, lo));
    r[j] = *reinterpret_cast<const uint32_t*>(&y);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}
// Codes of V channels 32w + 8q + (0..7) of row i out of a block's V codes.
__device__ __forceinline__ uint32_t v_word(const unsigned char* codes, int x, int i) {
  const unsigned char* at = codes + 512 * (x >> 2) + v_row_at(i) + ((x >> 1) & 1);
  uint32_t w = 0;
#pragma unroll
  for (int n = 0; n < 8; ++n) w |= ((uint32_t)(at[64 * n] >> (4 * (x & 1))) & 15u) << (4 * n);
  return w;
}

template <int DH>
__global__ void __launch_bounds__(THREADS) read_rows_kernel(const ReadParams p) {
  constexpr int LANES = DH / 8;
  pdl_launch_dependents();
  pdl_wait();
  const int x = threadIdx.x % LANES;
  const int64_t idx = ((int64_t)blockIdx.x * THREADS + threadIdx.x) / LANES;
  const int which = (int)(idx & 1);
  const int64_t rest = idx >> 1;
  const int h = (int)(rest % p.H);
  const int bg = (int)(rest / p.H);
  const int b = bg / p.rows, g = bg % p.rows;
  if (b >= p.B) return;
  const int64_t s = (int64_t)(p.first ? p.first[b] : 0) + g;
  uint4 out = make_uint4(0, 0, 0, 0);
  if (s >= 0 && s < p.kv_len[b]) {
    const char* blk = block_at<DH>(p.cache, b, h, (int)s);
    const int i = (int)(s % BLOCK_ROWS);
    if (blk) {
      const uint32_t par = *reinterpret_cast<const uint32_t*>(blk + (which ? Fmt<DH>::V_PAR : Fmt<DH>::K_PAR) + 4 * i);
      const uint32_t w = which ? v_word(reinterpret_cast<const unsigned char*>(blk) + Fmt<DH>::CODES, x, i)
                               : *reinterpret_cast<const uint32_t*>(blk + i * (DH / 2) + 4 * x);
      out = values(w, par);
    } else if (p.status && x == 0) {
      atomicOr(p.status + b, SPACE_ST_BAD_PAGE);
    }
  }
  *(reinterpret_cast<uint4*>((which ? p.dst[1] : p.dst[0]) + (int64_t)b * p.sb + (int64_t)g * p.sr + (int64_t)h * p.sh) + x) = out;
}

template <int DH>
__global__ void __launch_bounds__(THREADS) read_blocks_kernel(const ReadParams p) {
  constexpr int LANES = DH / 8, ROWS = THREADS / LANES, PASSES = BLOCK_ROWS / ROWS;
  __shared__ __align__(16) unsigned char vsm[Fmt<DH>::CODES];
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.z, h = blockIdx.y;
  const int64_t first = p.first ? p.first[b] : 0;
  // blocks of the cache from the one that holds row `first` on (floor, also below row 0)
  const int64_t s0 = ((first >= 0 ? first : first - (BLOCK_ROWS - 1)) / BLOCK_ROWS + (int64_t)blockIdx.x) * BLOCK_ROWS;
  if (s0 >= first + p.rows) return;
  const int len = p.kv_len[b];
  const bool live = s0 >= 0 && s0 < len;
  const char* blk = live ? block_at<DH>(p.cache, b, h, (int)s0) : nullptr;
  if (live && !blk && p.status && threadIdx.x == 0) atomicOr(p.status + b, SPACE_ST_BAD_PAGE);
  const int x = threadIdx.x % LANES, r = threadIdx.x / LANES;
  if (blk && threadIdx.x * 16 < Fmt<DH>::CODES)
    reinterpret_cast<uint4*>(vsm)[threadIdx.x] = reinterpret_cast<const uint4*>(blk + Fmt<DH>::CODES)[threadIdx.x];
  uint32_t kw[PASSES], par[2][PASSES];
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    const int i = k * ROWS + r;
    kw[k] = par[0][k] = par[1][k] = 0;
    if (blk) {
      kw[k] = *reinterpret_cast<const uint32_t*>(blk + i * (DH / 2) + 4 * x);
      par[0][k] = *reinterpret_cast<const uint32_t*>(blk + Fmt<DH>::K_PAR + 4 * i);
      par[1][k] = *reinterpret_cast<const uint32_t*>(blk + Fmt<DH>::V_PAR + 4 * i);
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    const int i = k * ROWS + r;
    const int64_t g = s0 + i - first;
    if (g < 0 || g >= p.rows) continue;
    const bool there = blk && s0 + i < len;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const int64_t at = (int64_t)b * p.sb + g * p.sr + (int64_t)h * p.sh;
    *(reinterpret_cast<uint4*>(p.dst[0] + at) + x) = there ? values(kw[k], par[0][k]) : zero;
    *(reinterpret_cast<uint4*>(p.dst[1] + at) + x) = there ? values(v_word(vsm, x, i), par[1][k]) : zero;
  }
}

// Up to this many rows per sequence go by rows.
constexpr int FEW_ROWS = 16;

}  // namespace

int launch_kvq_append(space_ctx* ctx, const space_kvq_append_args* a, cudaStream_t st) {
  AppendParams p;
  p.cache = cache_of(a->cache);
  p.B = a->batch; p.H = ctx->cfg.n_kv_heads;
  p.max_count = (a->rows - 1) / a->row_step + 1;
  p.step = a->row_step; p.bias = a->count ? a->count_bias : 0;
  p.src[0] = (const char*)a->k_new; p.src[1] = (const char*)a->v_new;
  p.sb = 2 * a->new_stride_b; p.sr = 2 * a->new_stride_r; p.sh = 2 * a->new_stride_h;
  p.kv_len = a->kv_len; p.count = a->count; p.len_out = a->kv_len_out; p.status = a->status;
  const bool wide = ctx->cfg.head_dim == 128;
  cudaError_t e;
  if (p.max_count <= FEW_ROWS) {
    const int64_t threads = (int64_t)p.B * p.max_count * p.H * 2 * (ctx->cfg.head_dim / 8);
    const dim3 grid((unsigned)((threads + THREADS - 1) / THREADS));
    e = launch_pdl(wide ? append_rows_kernel<128> : append_rows_kernel<64>, grid, dim3(THREADS), 0, st, p);
  } else {
    const dim3 grid((unsigned)(((int64_t)p.max_count + 2 * BLOCK_ROWS - 2) / BLOCK_ROWS), p.H, p.B);
    e = launch_pdl(wide ? append_blocks_kernel<128> : append_blocks_kernel<64>, grid, dim3(THREADS), 0, st, p);
  }
  ctx->launches += 1;
  return cuda_ok(e);
}

int launch_kvq_read(space_ctx* ctx, const space_kvq_read_args* a, cudaStream_t st) {
  ReadParams p;
  p.cache = cache_of(a->cache);
  p.B = a->batch; p.H = ctx->cfg.n_kv_heads; p.rows = a->rows;
  p.dst[0] = (char*)a->k_out; p.dst[1] = (char*)a->v_out;
  p.sb = 2 * a->out_stride_b; p.sr = 2 * a->out_stride_r; p.sh = 2 * a->out_stride_h;
  p.kv_len = a->kv_len; p.first = a->first; p.status = a->status;
  const bool wide = ctx->cfg.head_dim == 128;
  cudaError_t e;
  if (p.rows <= FEW_ROWS) {
    const int64_t threads = (int64_t)p.B * p.rows * p.H * 2 * (ctx->cfg.head_dim / 8);
    const dim3 grid((unsigned)((threads + THREADS - 1) / THREADS));
    e = launch_pdl(wide ? read_rows_kernel<128> : read_rows_kernel<64>, grid, dim3(THREADS), 0, st, p);
  } else {
    const dim3 grid((unsigned)(((int64_t)p.rows + 2 * BLOCK_ROWS - 2) / BLOCK_ROWS), p.H, p.B);
    e = launch_pdl(wide ? read_blocks_kernel<128> : read_blocks_kernel<64>, grid, dim3(THREADS), 0, st, p);
  }
  ctx->launches += 1;
  return cuda_ok(e);
}
