// Rows into the 8-bit cache and out of it (space_kvb_append, space_kvb_read).
//
// Append: a thread block has one 32-row block of one kv head, whose rows share a power of two, K and V: its new rows are
// loaded (and turned), their largest magnitudes meet, the codes are one conversion per pair of elements.  V codes lie sixteen rows to
// a channel (the attention's operand wants the keys of a channel side by side): they change places in shared memory and
// leave in 16-byte pieces.  Rows that the block had before are touched only where the power of two grows.
// Queries that are to be turned along have thread blocks of their own behind those.
// Read back: the same way round.
//
// What bounds them: 16 prompts of 512 to 4096 rows, 8 kv heads and 32 turned query heads of 128: 172 us, 4.3 TB/s of HBM and 68 % of the issue
// slots (the queries' 600 MB take half; K and V the rest of the instructions: rotation, largest magnitudes, codes, bytes
// that change places); read back 56 us, 5.0 TB/s.  Accepted rows of 64 sequences: a launch each, 5 us.
// (64 registers, 36 bytes of a thread spilled, for head size 128: four thread blocks an SM.)
#include "kvb_common.cuh"
#include "rope_common.cuh"

namespace {
using namespace kvb;

constexpr int THREADS = 256;
// Elements are held to 240 2^120 in magnitude: 256 2^120, to which larger ones would be rounded, is no bf16 number.
constexpr float ELEMENT_MAX = 0x1.Ep127f;
constexpr uint32_t ELEMENT_MAX_BITS = 0x7F70u;       // (as bf16)

struct AppendParams {
  Cache cache;
  int B, H, H_q, rows, max_count, step, bias, blocks;        // blocks: 32-row blocks a sequence's new rows may touch
  int64_t n_append;                                  // thread blocks that append
  int q_blocks, share;                               // thread blocks per sequence that turn queries; warps that share a row
  const char* src[2]; int64_t sb, sr, sh;            // K, V; bytes
  const char* q; int64_t q_sb, q_sr, q_sh;
  char* q_out; int64_t o_sb, o_sr, o_sh;
  rope::Table t;
  const int32_t* kv_len; const int32_t* count; int32_t* len_out; int32_t* status;
};

// Rows of sequence b that are appended, -1 where they do not fit.
__device__ __forceinline__ int append_count(const AppendParams& p, int b, int L) {
  const int64_t want = p.count ? (int64_t)p.count[b] + p.bias : (int64_t)p.max_count;
  const int n = (int)(want < 0 ? 0 : want > p.max_count ? p.max_count : want);
  return L >= 0 && (int64_t)L + n <= (int64_t)p.cache.pages_per_seq * SPACE_PAGE_SIZE ? n : -1;
}

// V codes of a 32-row block in shared memory: [2][DH] entries of sixteen rows, eight channels four bytes further on so that
// the lanes of a row reach different banks.
template <int DH>
struct VTile {
  static constexpr int GROUP = 16 * DH + 4 * (DH / 8), BYTES = 2 * GROUP;
  static __device__ __forceinline__ int at(int group, int c) { return group * GROUP + 16 * c + 4 * (c >> 3); }
};

__device__ __forceinline__ uint32_t held_pair(uint32_t w) {        // two finite bf16
  return __vminu2(w & 0x7FFF7FFFu, ELEMENT_MAX_BITS * 0x10001u) | (w & 0x80008000u);
}

// Four codes with their scale's power of two raised.  (From 2^119 to 2^120: 224 at most.)
__device__ __forceinline__ uint32_t coarser(uint32_t w, float ratio) {
  const uint32_t lo = halves2(w & 0xFFFFu), hi = halves2(w >> 16);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  return codes4(a.x * ratio, a.y * ratio, b.x * ratio, b.y * ratio);
}

// Queries of sequence b, beside the append.
template <int DH>
__device__ __forceinline__ void turn_queries(const AppendParams& p, int b, int block) {
  const uint32_t task = (uint32_t)block * (THREADS / 32) + (threadIdx.x >> 5), row = task / (uint32_t)p.share;
  const int L = p.kv_len[b], n = append_count(p, b, L), g = (int)row, part = (int)(task - row * (uint32_t)p.share);
  if (n <= 0 || row >= (uint32_t)n) return;
  const int64_t r = (int64_t)g * p.step;
  bool bad;
  rope::Turn u;
  rope::load_turn(p.t, rope::table_row(p.t, b, p.rows, (int)r, (int64_t)L + g, bad), (threadIdx.x & 31) % (DH / 8), u);
  rope::row_heads<DH, true>(p.t, u, p.H_q, part, p.share, p.q + (int64_t)b * p.q_sb + r * p.q_sr, p.q_sh, p.q_out + (int64_t)b * p.o_sb + r * p.o_sr, p.o_sh);
}

template <int DH>
__global__ void __launch_bounds__(THREADS, 4) kvb_append_kernel(const __grid_constant__ AppendParams p) {
  using F = Fmt<DH>;
  using VT = VTile<DH>;
  constexpr int LANES = DH / 8, ROWS = THREADS / LANES, PASSES = BLOCK_ROWS / ROWS;
  __shared__ __align__(16) unsigned char vsm[VT::BYTES];
  __shared__ uint32_t tops[2][THREADS / 32];
  pdl_launch_dependents();
  pdl_wait();
  if ((int64_t)blockIdx.x >= p.n_append) {
    const uint32_t rest = blockIdx.x - (uint32_t)p.n_append;
    turn_queries<DH>(p, (int)(rest / (uint32_t)p.q_blocks), (int)(rest % (uint32_t)p.q_blocks));
    return;
  }
  const uint32_t bh = blockIdx.x / (uint32_t)p.blocks;
  const int part = (int)(blockIdx.x - bh * (uint32_t)p.blocks), b = (int)(bh / (uint32_t)p.H), h = (int)(bh - (uint32_t)b * p.H);
  const int L = p.kv_len[b], n = append_count(p, b, L);
  if (part == 0 && h == 0 && threadIdx.x == 0) {
    if (n < 0 && p.status) atomicOr(p.status + b, SPACE_ST_CAPACITY);
    if (p.len_out) p.len_out[b] = L + max(n, 0);
  }
  if (n <= 0) return;
  const int s0 = (L / BLOCK_ROWS + part) * BLOCK_ROWS;       // first row of this block (may lie before L)
  if (s0 >= L + n) return;
  const int x = threadIdx.x % LANES, r = threadIdx.x / LANES;
  const int i_lo = max(L - s0, 0), i_hi = min(L + n - s0, BLOCK_ROWS);  // rows of the block that are written
  uint4 v[2][PASSES];
  rope::Turn u[PASSES];
  int bits = 0;
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    const int i = k * ROWS + r;
    v[0][k] = v[1][k] = make_uint4(0, 0, 0, 0);      // (rows that are not written: zeros, turned by zeros)
#pragma unroll
    for (int j = 0; j < 4; ++j) u[k].c[j] = u[k].s[j] = 0ull;
    if (i >= i_lo && i < i_hi) {
      const int64_t from = (int64_t)(s0 + i - L) * p.step;
#pragma unroll
      for (int which = 0; which < 2; ++which)
        v[which][k] = *(reinterpret_cast<const uint4*>(p.src[which] + (int64_t)b * p.sb + from * p.sr + (int64_t)h * p.sh) + x);
      if (p.t.table) {
        bool bad;
        rope::load_turn(p.t, rope::table_row(p.t, b, p.rows, (int)from, (int64_t)s0 + i, bad), x, u[k]);
        if (bad && h == 0) bits |= SPACE_ST_BAD_POSITION;
      }
    }
  }
  char* head = page_at(p.cache, b, h, s0);
  const int row0 = s0 % SPACE_PAGE_SIZE;
  float2* scales = reinterpret_cast<float2*>(head + F::SCALES) + row0 / BLOCK_ROWS;
  const float2 was = head && i_lo > 0 ? *scales : make_float2(0.f, 0.f);
  uint64_t y[PASSES][4];                             // the K rows, turned
  float top[2] = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    uint32_t most[2];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      most[which] = kvq::max_bits(v[which][k]);
      if (most[which] >= 0x7F80u) {
        bits |= SPACE_ST_NONFINITE;
        kvq::make_finite(v[which][k]);
        most[which] = kvq::max_bits(v[which][k]);
      }
    }
    if (most[1] > ELEMENT_MAX_BITS) {                // (K: once it is turned)
      v[1][k] = make_uint4(held_pair(v[1][k].x), held_pair(v[1][k].y), held_pair(v[1][k].z), held_pair(v[1][k].w));
      most[1] = ELEMENT_MAX_BITS;
    }
    top[1] = fmaxf(top[1], __uint_as_float(most[1] << 16));
    if (p.t.table) {
      rope::turn_row<LANES>(p.t, v[0][k], x, u[k], y[k]);
#pragma unroll
      for (int j = 0; j < 4; ++j) top[0] = fmaxf(top[0], fmaxf(fabsf(rope::first_of(y[k][j])), fabsf(rope::second_of(y[k][j]))));
    } else {
      const uint32_t w[4] = {v[0][k].x, v[0][k].y, v[0][k].z, v[0][k].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) y[k][j] = rope::pair_of(w[j]);
      top[0] = fmaxf(top[0], __uint_as_float(most[0] << 16));
    }
  }
  if (top[0] > ELEMENT_MAX) {                        // (two of the largest numbers turned into one can pass the largest)
    top[0] = ELEMENT_MAX;
#pragma unroll
    for (int k = 0; k < PASSES; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        y[k][j] = rope::pair(fminf(fmaxf(rope::first_of(y[k][j]), -ELEMENT_MAX), ELEMENT_MAX), fminf(fmaxf(rope::second_of(y[k][j]), -ELEMENT_MAX), ELEMENT_MAX));
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const uint32_t m = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top[which]));      // (not negative: ordered as numbers)
    if ((threadIdx.x & 31) == 0) tops[which][threadIdx.x >> 5] = m;
  }
  if (!head) {                                       // (the same for the whole block)
    if (p.status && threadIdx.x == 0) atomicOr(p.status + b, SPACE_ST_BAD_PAGE);
    return;
  }
  if (bits && p.status) atomicOr(p.status + b, bits);
  __syncthreads();
  float down[2], ratio[2];
  bool raised[2];
  float2 scale;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) m = max(m, tops[which][w]);
    int e = scale_exp(__uint_as_float(m));
    const int e0 = min(max((int)((__float_as_uint(which ? was.y : was.x) >> 23) & 255u) - 127, MIN_EXP), 120);
    raised[which] = i_lo > 0 && e > e0;
    ratio[which] = raised[which] ? pow2(max(e0 - e, -126)) : 1.f;
    if (i_lo > 0) e = max(e, e0);
    down[which] = pow2(-e);
    (which ? scale.y : scale.x) = pow2(e);
  }
  if (threadIdx.x == 0) *scales = scale;
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    const int i = k * ROWS + r;
    uint2* kc = reinterpret_cast<uint2*>(head + (x >> 1) * F::K_COLS + 16 * (row0 + i) + 8 * (x & 1));
    if (i >= i_lo && i < i_hi) {
      const uint32_t w[4] = {v[1][k].x, v[1][k].y, v[1][k].z, v[1][k].w};
      uint32_t kk[4], vv[4];                         // pairs of codes
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t a = rope::mul_pair(y[k][j], rope::pair(down[0], down[0])), c = rope::mul_pair(rope::pair_of(w[j]), rope::pair(down[1], down[1]));
        kk[j] = codes2(rope::first_of(a), rope::second_of(a));
        vv[j] = codes2(rope::first_of(c), rope::second_of(c));
      }
      *kc = make_uint2(kk[0] | kk[1] << 16, kk[2] | kk[3] << 16);
      unsigned char* at = vsm + VT::at(i >> 4, 8 * x) + (i & 15);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        at[32 * j] = (unsigned char)vv[j];
        at[32 * j + 16] = (unsigned char)(vv[j] >> 8);
      }
    } else if (raised[0] && i < i_lo) {
      const uint2 w = *kc;
      *kc = make_uint2(coarser(w.x, ratio[0]), coarser(w.y, ratio[0]));
    }
  }
  __syncthreads();
  for (int t = threadIdx.x; t < 2 * DH; t += THREADS) {
    const int group = t / DH, c = t % DH;
    const int lo = max(i_lo - 16 * group, 0), hi = min(i_hi - 16 * group, 16);           // new rows of these sixteen
    unsigned char* dst = reinterpret_cast<unsigned char*>(head) + F::CODES + (row0 / 16 + group) * F::V_ROWS + 16 * c;
    const uint32_t* from = reinterpret_cast<const uint32_t*>(vsm + VT::at(group, c));
    if (lo == 0 && hi == 16) {
      *reinterpret_cast<uint4*>(dst) = make_uint4(from[0], from[1], from[2], from[3]);
      continue;
    }
    if (raised[1] && i_lo > 16 * group) {            // these sixteen have rows from before
      uint4 w = *reinterpret_cast<const uint4*>(dst);
      const uint32_t o[4] = {coarser(w.x, ratio[1]), coarser(w.y, ratio[1]), coarser(w.z, ratio[1]), coarser(w.w, ratio[1])};
      uint32_t keep[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int m = min(max(i_lo - 16 * group - 4 * j, 0), 4);                         // bytes of this word that rows before L have
        const uint32_t mask = m == 4 ? 0xFFFFFFFFu : (1u << (8 * m)) - 1u;
        keep[j] = (o[j] & mask) | (keep[j] & ~mask);
      }
      *reinterpret_cast<uint4*>(dst) = make_uint4(keep[0], keep[1], keep[2], keep[3]);
    }
    for (int j = lo; j < hi; ++j) dst[j] = reinterpret_cast<const unsigned char*>(from)[j];
  }
}

struct ReadParams {
  Cache cache;
  int B, H, rows;
  char* dst[2];
  int64_t sb, sr, sh;                                // bytes
  const int32_t* kv_len; const int32_t* first; int32_t* status;
};

// Four codes times a power of two as bf16: exact.
__device__ __forceinline__ uint2 values(uint32_t w, float s) {
  const uint32_t lo = halves2(w & 0xFFFFu), hi = halves2(w >> 16);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  const __nv_bfloat162 u = __floats2bfloat162_rn(a.x * s, a.y * s), v = __floats2bfloat162_rn(b.x * s, b.y * s);
  return make_uint2(*reinterpret_cast<const uint32_t*>(&u), *reinterpret_cast<const uint32_t*>(&v));
}

template <int DH>
__global__ void __launch_bounds__(THREADS) kvb_read_kernel(const ReadParams p) {
  using F = Fmt<DH>;
  using VT = VTile<DH>;
  constexpr int LANES = DH / 8, ROWS = THREADS / LANES, PASSES = BLOCK_ROWS / ROWS;
  __shared__ __align__(16) unsigned char vsm[VT::BYTES];
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.z, h = blockIdx.y;
  const int64_t first = p.first ? p.first[b] : 0;
  // blocks of the cache from the one that holds row `first` on (floor, also below row 0)
  const int64_t s0 = ((first >= 0 ? first : first - (BLOCK_ROWS - 1)) / BLOCK_ROWS + (int64_t)blockIdx.x) * BLOCK_ROWS;
  if (s0 >= first + p.rows) return;
  const int len = p.kv_len[b];
  const bool live = s0 >= 0 && s0 < len;
  const char* head = live ? page_at(p.cache, b, h, (int)s0) : nullptr;
  if (live && !head && p.status && threadIdx.x == 0) atomicOr(p.status + b, SPACE_ST_BAD_PAGE);
  const int x = threadIdx.x % LANES, r = threadIdx.x / LANES, row0 = (int)(s0 & (SPACE_PAGE_SIZE - 1));
  uint2 kw[PASSES];
  float2 scale = make_float2(0.f, 0.f);
  if (head) {
    scale = *(reinterpret_cast<const float2*>(head + F::SCALES) + row0 / BLOCK_ROWS);
#pragma unroll
    for (int k = 0; k < PASSES; ++k)
      kw[k] = *reinterpret_cast<const uint2*>(head + (x >> 1) * F::K_COLS + 16 * (row0 + k * ROWS + r) + 8 * (x & 1));
    for (int t = threadIdx.x; t < 2 * DH; t += THREADS) {
      const uint4 w = *reinterpret_cast<const uint4*>(head + F::CODES + row0 / 16 * F::V_ROWS + 16 * t);
      uint32_t* to = reinterpret_cast<uint32_t*>(vsm + VT::at(t / DH, t % DH));
      to[0] = w.x; to[1] = w.y; to[2] = w.z; to[3] = w.w;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    const int i = k * ROWS + r;
    const int64_t g = s0 + i - first;
    if (g < 0 || g >= p.rows) continue;
    const bool there = head && s0 + i < len;
    uint4 kv = make_uint4(0, 0, 0, 0), vv = kv;
    if (there) {
      const uint2 a = values(kw[k].x, scale.x), c = values(kw[k].y, scale.x);
      kv = make_uint4(a.x, a.y, c.x, c.y);
      const unsigned char* at = vsm + VT::at(i >> 4, 8 * x) + (i & 15);
      const uint2 e = values(at[0] | at[16] << 8 | at[32] << 16 | (uint32_t)at[48] << 24, scale.y);
      const uint2 f = values(at[64] | at[80] << 8 | at[96] << 16 | (uint32_t)at[112] << 24, scale.y);
      vv = make_uint4(e.x, e.y, f.x, f.y);
    }
    const int64_t at = (int64_t)b * p.sb + g * p.sr + (int64_t)h * p.sh;
    *(reinterpret_cast<uint4*>(p.dst[0] + at) + x) = kv;
    *(reinterpret_cast<uint4*>(p.dst[1] + at) + x) = vv;
  }
}

}  // namespace

int launch_kvb_append(space_ctx* ctx, const space_kvb_append_args* a, cudaStream_t st) {
  AppendParams p;
  memset(&p, 0, sizeof(p));
  const int d = ctx->cfg.head_dim;
  p.cache = cache_of(a->cache);
  p.B = a->batch; p.H = ctx->cfg.n_kv_heads; p.H_q = ctx->cfg.n_q_heads; p.rows = a->rows;
  p.max_count = (a->rows - 1) / a->row_step + 1;
  p.step = a->row_step; p.bias = a->count ? a->count_bias : 0;
  p.src[0] = (const char*)a->k_new; p.src[1] = (const char*)a->v_new;
  p.sb = 2 * a->new_stride_b; p.sr = 2 * a->new_stride_r; p.sh = 2 * a->new_stride_h;
  p.kv_len = a->kv_len; p.count = a->count; p.len_out = a->kv_len_out; p.status = a->status;
  if (a->rope.table) p.t = rope::table_of(a->rope);
  p.blocks = (int)(((int64_t)p.max_count + 2 * BLOCK_ROWS - 2) / BLOCK_ROWS);
  p.n_append = (int64_t)p.B * p.H * p.blocks;
  int64_t grid = p.n_append;
  if (a->q) {
    p.q = (const char*)a->q; p.q_sb = 2 * a->q_stride_b; p.q_sr = 2 * a->q_stride_r; p.q_sh = 2 * a->q_stride_h;
    p.q_out = (char*)a->q_out; p.o_sb = 2 * a->q_out_stride_b; p.o_sr = 2 * a->q_out_stride_r; p.o_sh = 2 * a->q_out_stride_h;
    p.share = rope::warps_per_row((int64_t)p.B * p.max_count, ctx->sm_count, THREADS / 32);
    p.q_blocks = (int)(((int64_t)p.max_count * p.share + THREADS / 32 - 1) / (THREADS / 32));
    grid += (int64_t)p.B * p.q_blocks;
  }
  if (grid > 0x7FFFFFFFll) return SPACE_E_UNSUPPORTED;
  ctx->launches += 1;
  return cuda_ok(launch_pdl(d == 128 ? kvb_append_kernel<128> : kvb_append_kernel<64>, dim3((unsigned)grid), dim3(THREADS), 0, st, p));
}

int launch_kvb_read(space_ctx* ctx, const space_kvb_read_args* a, cudaStream_t st) {
  ReadParams p;
  p.cache = cache_of(a->cache);
  p.B = a->batch; p.H = ctx->cfg.n_kv_heads; p.rows = a->rows;
  p.dst[0] = (char*)a->k_out; p.dst[1] = (char*)a->v_out;
  p.sb = 2 * a->out_stride_b; p.sr = 2 * a->out_stride_r; p.sh = 2 * a->out_stride_h;
  p.kv_len = a->kv_len; p.first = a->first; p.status = a->status;
  const dim3 grid((unsigned)(((int64_t)p.rows + 2 * BLOCK_ROWS - 2) / BLOCK_ROWS), p.H, p.B);
  ctx->launches += 1;
  return cuda_ok(launch_pdl(ctx->cfg.head_dim == 128 ? kvb_read_kernel<128> : kvb_read_kernel<64>, grid, dim3(THREADS), 0, st, p));
}
