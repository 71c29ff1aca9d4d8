// Rows into the 4-bit cache and out of it (space_kvq_append, space_kvq_read).
//
// Append: a row of d channels has d / 16 lanes; minimum and maximum by shuffles of one pair of bf16,
// step = bf16(max((hi - lo) / 15, max|x| / 4096, 2^-100)), u = round((x - lo) / step).  The quotient has to be the
// exact one at ties, which bf16 inputs meet often (a tie is a quotient n + 1/2 with few bits): one reciprocal per
// row, then per element a product and one residual step,
//   q0 = x inv,  q = q0 + (x - q0 step) inv,
// which is exact where the quotient has few bits, and off by at most an ulp elsewhere, where a quotient of these
// operands (8 bits over 8 bits) is further than 2^-16 of itself from a tie.  Everything in halves, so that
// hi - lo cannot overflow.
//
// Two forms.  By blocks: a thread block per 32-row block of the cache; V codes, which lie transposed (the order of the
// attention's operand), are gathered in shared memory and leave in 16-byte pieces.  By rows: the lanes of a row
// store their V bytes two at a time where they belong; for the few rows of a step or a token, where a thread block
// per 32-row block would be nearly empty.  Sixteen channels a lane, in pairs of floats and with one shuffle for both
// ends of the span, because the first form (eight channels, single floats) was held up by its instructions: 16 sequences
// of 512 to 4096 rows, 32 heads, d = 128, took it 257 us; now 156 (166 with three input sets in turn), of which the bytes (5 d + 8 a row and head, K and V)
// are 111.
//
// Read back: a thread block per 32-row block, V codes through shared memory; 204 us of 190 for the same rows (a second
// form by rows was never faster, also for one row, and is not kept).
#include "kvq_common.cuh"
#include "tc_common.cuh"

namespace {
using namespace kvq;
using namespace tc;

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

__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmin2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// {lo, -hi} of the row as a pair of bf16 (both are elements of it): one shuffle and one minimum per step.
template <int LANES>
__device__ __forceinline__ uint32_t row_span(const uint4& u, const uint4& v) {
  const uint32_t lo = min2_nan(min2_nan(min2_nan(u.x, u.y), min2_nan(u.z, u.w)), min2_nan(min2_nan(v.x, v.y), min2_nan(v.z, v.w)));
  const uint32_t hi = max2_nan(max2_nan(max2_nan(u.x, u.y), max2_nan(u.z, u.w)), max2_nan(max2_nan(v.x, v.y), max2_nan(v.z, v.w))) ^ 0x80008000u;
  uint32_t m = min2_nan(__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) m = min2_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  return m;
}
// A row has d / 16 lanes, sixteen channels each.  Codes of this lane's first and second eight channels, channel n in
// bits 4n .. 4n+3, and the row's {step, lo}.
template <int LANES>
__device__ __forceinline__ uint2 quantise(uint4 u, uint4 v, uint32_t& par, bool& bad) {
  uint32_t span = row_span<LANES>(u, v);
  bad = (span & 0x7F80u) == 0x7F80u || (span & 0x7F800000u) == 0x7F800000u;    // NaN or an infinity somewhere in the row
  if (__any_sync(0xFFFFFFFFu, bad)) {
    make_finite(u); make_finite(v);
    span = row_span<LANES>(u, v);
  }
  const float lo = bf_lo(span), hi = -bf_hi(span), lo2 = 0.5f * lo;
  // (hi - lo) / 15, in halves; the quotient by a product and a residual step, as below
  const float d = 0.5f * hi - lo2, d0 = d * (1.f / 7.5f);
  const float s = fmaxf(fmaxf(fmaf(fmaf(-d0, 7.5f, d), 1.f / 7.5f, d0), fmaxf(-lo, hi) * (1.f / 4096.f)), 0x1p-100f);
  const __nv_bfloat16 sb = __float2bfloat16_rn(s);
  const float s2 = 0.5f * __bfloat162float(sb);
  float r0;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(s2));
  const float inv = fmaf(fmaf(-s2, r0, 1.f), r0, r0);
  par = (uint32_t)__bfloat16_as_ushort(sb) | span << 16;
  const uint64_t inv2 = pack2(inv, inv), step2 = pack2(-s2, -s2), off2 = pack2(-lo2, -lo2), half2 = pack2(0.5f, 0.5f);
  const uint64_t magic = pack2(12582912.f, 12582912.f);                        // 1.5 * 2^23: a sum's last bit is a unit, ties to even
  const uint32_t x[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 7; i >= 0; --i) {
    const uint64_t y = fma2(pack2(bf_lo(x[i]), bf_hi(x[i])), half2, off2);
    const uint64_t q0 = fma2(y, inv2, 0ull);
    const uint64_t q = add2(fma2(fma2(q0, step2, y), inv2, q0), magic);
    // (at most 15 (1 + 2^-8) before it is rounded: no clamp)  Both words are 0x4B400000 + u: shifted and added up
    // modulo 2^32, with the constants' sum taken off at the end
    w[i >> 2] = w[i >> 2] * 256u + (uint32_t)(q >> 32) * 16u + (uint32_t)q;
  }
  return make_uint2(w[0] - 0x4B400000u * 0x11111111u, w[1] - 0x4B400000u * 0x11111111u);
}

// Nibbles 0..3 of the low half as bytes.
__device__ __forceinline__ uint32_t spread(uint32_t a) {
  a = (a | a << 8) & 0x00FF00FFu;
  return (a | a << 4) & 0x0F0F0F0Fu;
}
// Lane x has the channels n = 0..7 of q = 2 (x % 2) and of the next q, of word w = x / 2: its four V byte pairs, those of
// n = 4 (x % 2) + 0..3 (two in a word, low half first).
__device__ __forceinline__ uint2 v_bytes(const uint2& w, int x) {
  const uint32_t lo = spread(w.x & 0xFFFFu) | spread(w.y & 0xFFFFu) << 4, hi = spread(w.x >> 16) | spread(w.y >> 16) << 4;
  const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, (x & 1) ? lo : hi, 1);
  const uint32_t a = (x & 1) ? got : lo, b = (x & 1) ? hi : got;               // q / 2 = 0 and 1
  return make_uint2(__byte_perm(a, b, 0x5140), __byte_perm(a, b, 0x7362));
}
template <int PITCH>
__device__ __forceinline__ void store_v(char* granules, int x, int i, const uint2& vb) {
  char* at = granules + (8 * (x >> 1) + 4 * (x & 1)) * PITCH + v_row_at(i);
  *reinterpret_cast<uint16_t*>(at) = (uint16_t)vb.x;
  *reinterpret_cast<uint16_t*>(at + PITCH) = (uint16_t)(vb.x >> 16);
  *reinterpret_cast<uint16_t*>(at + 2 * PITCH) = (uint16_t)vb.y;
  *reinterpret_cast<uint16_t*>(at + 3 * PITCH) = (uint16_t)(vb.y >> 16);
}

template <int DH>
__global__ void __launch_bounds__(THREADS) append_rows_kernel(const AppendParams p) {
  constexpr int LANES = DH / 16;
  pdl_launch_dependents();
  pdl_wait();
  const int x = threadIdx.x % LANES;
  const uint32_t idx = (blockIdx.x * (uint32_t)THREADS + threadIdx.x) / LANES;
  const int which = (int)(idx & 1);
  const uint32_t rest = idx >> 1;
  const int h = (int)(rest % (uint32_t)p.H), bg = (int)(rest / (uint32_t)p.H);
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
  uint4 u = make_uint4(0, 0, 0, 0), v = u;
  if (blk) {
    const uint4* src = reinterpret_cast<const uint4*>((which ? p.src[1] : p.src[0]) + (int64_t)b * p.sb + (int64_t)g * p.step * p.sr + (int64_t)h * p.sh) + 2 * x;
    u = src[0]; v = src[1];
  }
  uint32_t par;
  bool bad;
  const uint2 w = quantise<LANES>(u, v, par, bad);
  const uint2 vb = v_bytes(w, x);
  if (!blk) return;
  const int i = (L + g) % BLOCK_ROWS;
  if (x == 0) {
    if (bad && p.status) atomicOr(p.status + b, SPACE_ST_NONFINITE);
    *reinterpret_cast<uint32_t*>(blk + (which ? Fmt<DH>::V_PAR : Fmt<DH>::K_PAR) + 4 * i) = par;
  }
  if (which == 0) *reinterpret_cast<uint2*>(blk + i * (DH / 2) + 8 * x) = w;
  else store_v<64>(blk + Fmt<DH>::CODES, x, i, vb);
}

template <int DH>
__global__ void __launch_bounds__(2 * DH) append_blocks_kernel(const AppendParams p) {
  constexpr int LANES = DH / 16;                     // 32 rows at a time
  constexpr int PITCH = 68;                          // of 64 bytes (a channel's granules): the lanes of a row reach different banks
  __shared__ __align__(16) char vsm[Fmt<DH>::CODES / 64 * PITCH];
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
  const int x = threadIdx.x % LANES, i = threadIdx.x / LANES;
  const int i_lo = max(L - s0, 0), i_hi = min(L + n - s0, BLOCK_ROWS);  // rows of the block that are written
  const bool mine = i >= i_lo && i < i_hi;
  uint4 u[2], v[2];
  u[0] = u[1] = v[0] = v[1] = make_uint4(0, 0, 0, 0);
  if (mine) {
    const int64_t at = (int64_t)b * p.sb + (int64_t)(s0 + i - L) * p.step * p.sr + (int64_t)h * p.sh + 32 * x;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const uint4* src = reinterpret_cast<const uint4*>(p.src[which] + at);
      u[which] = src[0]; v[which] = src[1];
    }
  }
  char* blk = block_at<DH>(p.cache, b, h, s0);
  if (!blk) {
    if (p.status && threadIdx.x == 0) atomicOr(p.status + b, SPACE_ST_BAD_PAGE);
    return;
  }
  uint32_t kp, vp;
  bool kbad, vbad;
  const uint2 kw = quantise<LANES>(u[0], v[0], kp, kbad);
  if (mine) *reinterpret_cast<uint2*>(blk + i * (DH / 2) + 8 * x) = kw;
  store_v<PITCH>(vsm, x, i, v_bytes(quantise<LANES>(u[1], v[1], vp, vbad), x));
  if (mine && x == 0) {
    *reinterpret_cast<uint32_t*>(blk + Fmt<DH>::K_PAR + 4 * i) = kp;
    *reinterpret_cast<uint32_t*>(blk + Fmt<DH>::V_PAR + 4 * i) = vp;
    if ((kbad || vbad) && p.status) atomicOr(p.status + b, SPACE_ST_NONFINITE);
  }
  __syncthreads();
  const int t = threadIdx.x;
  if (t * 16 < Fmt<DH>::CODES) {
    uint4* dst = reinterpret_cast<uint4*>(blk + Fmt<DH>::CODES) + t;
    const uint32_t* from = reinterpret_cast<const uint32_t*>(vsm + (t >> 2) * PITCH + (t & 3) * 16);
    const uint4 val = make_uint4(from[0], from[1], from[2], from[3]);
    if (i_lo == 0 && i_hi == BLOCK_ROWS) {
      *dst = val;
    } else {                                               // sixteen bytes are eight rows' pairs: 16a + 8e + 2t + h
      const uint32_t w[4] = {val.x, val.y, val.z, val.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int r = 16 * (j >> 2) + 8 * ((j >> 1) & 1) + 2 * (t & 3) + (j & 1);
        if (r >= i_lo && r < i_hi) reinterpret_cast<uint16_t*>(dst)[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
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

// Up to this many rows per sequence are appended by rows (16 sequences x 32 heads, d = 128, us by rows / by blocks:
// 4 rows 3.4 / 5.6, 12 rows 5.3 / 6.0, 16 rows 7.1 / 6.2, 64 rows 14.3 / 8.1).
constexpr int FEW_ROWS = 12;

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
    const int64_t threads = (int64_t)p.B * p.max_count * p.H * 2 * (ctx->cfg.head_dim / 16);
    const dim3 grid((unsigned)((threads + THREADS - 1) / THREADS));
    e = launch_pdl(wide ? append_rows_kernel<128> : append_rows_kernel<64>, grid, dim3(THREADS), 0, st, p);
  } else {
    const dim3 grid((unsigned)(((int64_t)p.max_count + 2 * BLOCK_ROWS - 2) / BLOCK_ROWS), p.H, p.B);
    e = launch_pdl(wide ? append_blocks_kernel<128> : append_blocks_kernel<64>, grid, dim3(2 * ctx->cfg.head_dim), 0, st, p);
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
  const dim3 grid((unsigned)(((int64_t)p.rows + 2 * BLOCK_ROWS - 2) / BLOCK_ROWS), p.H, p.B);
  const cudaError_t e = launch_pdl(ctx->cfg.head_dim == 128 ? read_blocks_kernel<128> : read_blocks_kernel<64>, grid, dim3(THREADS), 0, st, p);
  ctx->launches += 1;
  return cuda_ok(e);
}
