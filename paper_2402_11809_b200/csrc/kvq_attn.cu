// Attention of a step's block rows over the 4-bit cache (space_kvq_attn_step), up to 16 query rows at a time.
//
// The mathematics.  A cached row stands for lo + step u, so with the codes as they lie
//   score = c (step_k sum_c q_c u_c + lo_k sum_c q_c),     out = sum_j e_j step_j (u_j - 8) + sum_j e_j (lo_j + 8 step_j):
// the products take bare codes, steps and lowest values are two multiply-adds per score.  A code that is masked out of
// its 32-bit word is already an f16 number, the subnormal u 2^-24 (or u 2^-20 for the nibbles at bits 4..7), which
// the tensor cores take at full rate; the powers of two go into the query row (first product) and into the epilogue
// (second one, whose codes are centred by 8 first: sums of one sign would collect the tensor core's truncation).
// f16 holds a bf16 query row exactly, scaled by a power of two, and the weights e step to 11 bits.  The sums of e and of
// e (lo + 8 step) refer to the largest score so far, the weights to the largest e step of their row so far: a row of V
// that is large and hardly seen costs the others no bits.
//
// The work.  Everything is bound by the cache's bytes, (d + 8) per key and head, so: the keys of all (sequence, kv head,
// 16 query rows) items form one flat list of 128-key pages, every thread block takes an equal share of it, and a page's
// four blocks of 32 keys go to its four warps.  A warp streams its blocks (contiguous 32 d + 256 bytes each) into a ring of
// its own with bulk copies and never meets another warp until the item ends: 3 blocks per SM x 4 warps x 2 blocks in
// flight.  The cache is laid out in the order of the m16n8k16 operands, so that a lane's 16 bytes are what it feeds to
// the tensor core: nothing is shuffled or staged.  The pieces of an item that was cut are joined by the block that
// stores the last of them, always in the same order.
// Every wait is bounded; an expired wait sets SPACE_ST_TIMEOUT and the block drains and exits.
#include "common.cuh"
#include "tc_common.cuh"
#include "attn_common.cuh"
#include "kvq_common.cuh"
#include <cuda_fp16.h>
#include <math_constants.h>

namespace {
using namespace kvq;
using namespace tc;

constexpr int WARPS = PAGE_BLOCKS, THREADS = 32 * WARPS;   // a warp per 32-row block of a page
constexpr int RT = 16;                               // query rows of an item
constexpr int STAGES = 3;
constexpr int CTAS_PER_SM = 3;
constexpr int SHARE_COST = 1;                        // fixed cost of starting an item, in pages
constexpr uint64_t WAIT_NS = 1000000000ull;
constexpr float REF_SLACK = 8.f;                     // a row's reference moves when a score exceeds it by 2^8
constexpr float W_LIMIT = 16384.f;                   // weights of the second product stay below this (f16 ends at 65504)

struct Params {
  Cache cache;
  int B, n_q, H_q, H_kv, G, n_rt;                    // n_rt: items of 16 query rows per (sequence, kv head)
  int n_groups;                                      // thread blocks
  int has_new;
  float c;                                           // scale * log2(e)
  const char* q; int64_t q_sb, q_sr, q_sh;           // bytes
  const char* kn; const char* vn; int64_t n_sb, n_sr, n_sh;
  const int32_t* kv_len;
  __nv_bfloat16* out; float* lse; int32_t* status;
  float* part;                                       // [2 * n_groups][RT * (DH + 2)]
  int* arrived;                                      // [B * H_kv * n_rt], self-resetting
  int* err;
  uint64_t mask[SPACE_MAX_ROWS];                     // Eq. 5: bit j of word i: block row i sees block row j
};

template <int DH>
struct Smem {
  static constexpr int RING = STAGES * Fmt<DH>::BLOCK;       // of a warp
  static constexpr int O_PITCH = DH + 4;                     // floats
  static constexpr int OT = RT * O_PITCH * 4;                // a warp's accumulators, in its ring once that has run dry
  static_assert(OT <= RING, "the accumulators are parked in the ring");
  static constexpr int V_PITCH = DH * 2 + 16;                // bytes: the block's own V rows as f16
  static_assert(16 * V_PITCH <= RING, "so are the block's V rows");
  static constexpr int ML_OFF = WARPS * RING;                // [WARPS][RT] {reference, sum}
  static constexpr int BAR_OFF = ML_OFF + WARPS * RT * 8;
  static constexpr int MISC_OFF = BAR_OFF + WARPS * STAGES * 8;
  static constexpr int TABLE_OFF = MISC_OFF + 16;            // prefix[max_batch + 1] (64 bits), seq_len[max_batch]
};

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_h(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t h2sub(uint32_t a, uint32_t b) {
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 1));
  return fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 2));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
  return v + __shfl_xor_sync(0xFFFFFFFFu, v, 2);
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }     // -126 <= e <= 127

__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* err, int site) {
  return mbar_wait_bounded(bar, parity, abort_flag, err, site, WAIT_NS, 32);
}

// Where an item's query row r lies: block row and head.
__device__ __forceinline__ void row_of(const Params& p, int h, int r, int& i, int& hq) {
  i = r / p.G;
  hq = h * p.G + (r - i * p.G);
}

// State of a warp: two query rows per lane (lane / 4 and + 8).
template <int DH>
struct Acc {
  float o[DH / 8][4];
  float m[2], l[2], z[2];                            // reference (log2 units), sum of e, sum of e (lo + 8 step)
  float R[2], vinv[2];                               // reference of the accumulators, 2^(m - R + 6)
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < DH / 8; ++t) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.f;
    m[0] = m[1] = R[0] = R[1] = -CUDART_INF_F; l[0] = l[1] = z[0] = z[1] = 0.f;
    vinv[0] = vinv[1] = 0x1p126f;
  }
  __device__ __forceinline__ void scale_rows(float f0, float f1) {
#pragma unroll
    for (int t = 0; t < DH / 8; ++t) { o[t][0] *= f0; o[t][1] *= f0; o[t][2] *= f1; o[t][3] *= f1; }
  }
  // References raised to mx where that is more; the sums follow.  Returns the factor they took.
  __device__ __forceinline__ float2 raise(float mx0, float mx1) {
    const float n0 = fmaxf(m[0], mx0), n1 = fmaxf(m[1], mx1);
    const float f0 = m[0] == n0 ? 1.f : fast_exp2(m[0] - n0), f1 = m[1] == n1 ? 1.f : fast_exp2(m[1] - n1);
    m[0] = n0; m[1] = n1;
    l[0] *= f0; l[1] *= f1; z[0] *= f0; z[1] *= f1;
    return make_float2(f0, f1);
  }
  // 2^(m - R + 6), bounded: a weight of at least 2^-100 times the bound is over what set_scale lets through
  __device__ __forceinline__ void set_vinv() {
#pragma unroll
    for (int s = 0; s < 2; ++s) vinv[s] = R[s] == -CUDART_INF_F ? 0x1p126f : fast_exp2(fminf(m[s] - R[s] + 6.f, 126.f));
  }
  // The accumulators' reference moved up to a row's largest weight t (relative to m), where that would pass 2^14.
  __device__ __forceinline__ void set_scale(float t0, float t1) {
    const float t[2] = {quad_max(t0), quad_max(t1)};
    float f[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      f[s] = 1.f;
      if (t[s] * vinv[s] > W_LIMIT) {
        const float n = m[s] + (float)((int)(__float_as_uint(t[s]) >> 23) - 127);
        f[s] = fast_exp2(R[s] - n);
        R[s] = n;
      }
    }
    scale_rows(f[0], f[1]);
    set_vinv();
  }
};

// Query rows as operands: lane (n = lane / 4, t = lane % 4) holds of rows n and n + 8 the channels t * DH/4 .. ; the
// pair that a code word's mask brings out at bits 0..3 (4..7) of each half is a k-step's first (second) half.
template <int DH>
struct Query {
  uint32_t a[DH / 16][4];
  float sum[2];                                      // sum of the row's channels
  float c;                                           // scores = c * (products), with the rows' power of two undone
  __device__ __forceinline__ void load(const Params& p, int b, int h, int r0, int lane) {
    const int t = lane & 3;
    uint4 raw[2][DH / 32];
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int r = r0 + (lane >> 2) + 8 * s;
      int i, hq;
      row_of(p, h, r, i, hq);
      const bool there = i < p.n_q;
      const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)b * p.q_sb + (int64_t)i * p.q_sr + (int64_t)hq * p.q_sh) + t * (DH / 32);
      float sm = 0.f;
#pragma unroll
      for (int j = 0; j < DH / 32; ++j) {
        raw[s][j] = there ? src[j] : make_uint4(0, 0, 0, 0);
        const uint32_t w[4] = {raw[s][j].x, raw[s][j].y, raw[s][j].z, raw[s][j].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          sm += bf_lo(w[k]) + bf_hi(w[k]);
          // exponents; a row that is not finite does not set the scale of the others
          const uint32_t e0 = (w[k] >> 7) & 0xFFu, e1 = (w[k] >> 23) & 0xFFu;
          top = max(top, max(e0 == 255u ? 0u : e0, e1 == 255u ? 0u : e1));
        }
      }
      sum[s] = quad_sum(sm);
    }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    // largest element in [2^8, 2^9): what f16 drops lies 2^-32 below it
    const int e = top ? min(max(8 - ((int)top - 127), -100), 100) : 0;
    const float f = pow2(e), f16th = f * 0.0625f;
    c = p.c * pow2(-e);
    const float c0 = p.c;
    sum[0] *= c0; sum[1] *= c0;
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) {
      // k-step ks is half of code word ks / 2: pairs 2 (ks % 2) and 2 (ks % 2) + 1, channels 8 (ks/2) + pair (+ 4)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint4 v = raw[s][ks / 2];
        const uint32_t lo = (ks & 1) ? v.y : v.x, hi = (ks & 1) ? v.w : v.z;   // channels 2(ks%2), +1 and 4 + 2(ks%2), +1
        a[ks][s] = pack_h(bf_lo(lo) * f, bf_lo(hi) * f);
        a[ks][2 + s] = pack_h(bf_hi(lo) * f16th, bf_hi(hi) * f16th);
      }
    }
  }
};

// The state of several warps or pieces meets: nothing but sums in a fixed order.
template <int DH>
__device__ __forceinline__ void store_row4(const Params& p, int b, int h, int r, int c4, float4 o, float m, float l) {
  int i, hq;
  row_of(p, h, r, i, hq);
  const float rd = l > 0.f || l != l ? 1.f / l : 0.f;      // a row without keys: zeros
  const __nv_bfloat162 x = __floats2bfloat162_rn(o.x * rd, o.y * rd), y = __floats2bfloat162_rn(o.z * rd, o.w * rd);
  __nv_bfloat16* dst = p.out + (((int64_t)b * p.n_q + i) * p.H_q + hq) * DH + 4 * c4;
  *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
  if (c4 == 0 && p.lse) p.lse[((int64_t)b * p.H_q + hq) * p.n_q + i] = (m + log2f(l)) * 0.6931471805599453f;
}

template <int DH>
__global__ void __launch_bounds__(THREADS, CTAS_PER_SM) kvq_attn_kernel(const __grid_constant__ Params p, int max_batch) {
  using F = Fmt<DH>;
  using S = Smem<DH>;
  extern __shared__ __align__(128) unsigned char sm[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane & 3;
  const uint32_t base = smem_u32(sm);
  const uint32_t ring = base + warp * S::RING, bar = base + S::BAR_OFF + warp * STAGES * 8;
  float2* ml = reinterpret_cast<float2*>(sm + S::ML_OFF);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::MISC_OFF);
  int* last_flag = reinterpret_cast<int*>(sm + S::MISC_OFF + 4);
  long long* prefix = reinterpret_cast<long long*>(sm + S::TABLE_OFF);
  int* seq_len = reinterpret_cast<int*>(prefix + max_batch + 1);

  pdl_launch_dependents();
  if (threadIdx.x == 0) *abort_flag = 0;
  if (lane == 0) {
    for (int s = 0; s < STAGES; ++s) mbar_init(bar + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  pdl_wait();
  // Lengths, and the list's running sums: a (sequence, kv head, row block) has a page per 128 keys, one more where the
  // block's own rows are given, at least one (rows without any key still get their zeros), and SHARE_COST ahead.
  auto pages_of = [&](int L) { return max((L + SPACE_PAGE_SIZE - 1) / SPACE_PAGE_SIZE + p.has_new, 1); };
  if (warp == 0) {
    long long carry = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const int b = b0 + lane;
      int L = -1;
      long long n = 0;
      if (b < p.B) {
        L = p.kv_len[b];
        if (L < 0 || (int64_t)L > (int64_t)p.cache.pages_per_seq * SPACE_PAGE_SIZE) {
          if (blockIdx.x == 0 && p.status) atomicOr(p.status + b, SPACE_ST_CAPACITY);
          L = -1;
        }
        n = (long long)(pages_of(max(L, 0)) + SHARE_COST) * p.H_kv * p.n_rt;
      }
      long long incl = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += v;
      }
      if (b < p.B) { seq_len[b] = L; prefix[b] = carry + incl - n; }
      carry += __shfl_sync(0xFFFFFFFFu, incl, 31);
    }
    if (lane == 0) prefix[p.B] = carry;
  }
  __syncthreads();
  const long long W = prefix[p.B], NG = W < p.n_groups ? W : p.n_groups;
  if ((long long)blockIdx.x >= NG) return;
  long long cur = attn::muldiv(W, blockIdx.x, NG);
  const long long share0 = cur, end = attn::muldiv(W, (long long)blockIdx.x + 1, NG);
  const int per_head = p.n_rt;

  uint32_t step = 0;                                 // blocks of the ring used so far, by this warp
  Query<DH> q;
  Acc<DH> acc;
  int b = 0;
  while (cur < end) {
    while (prefix[b + 1] <= cur) ++b;
    const int L0 = seq_len[b], L = max(L0, 0);
    const int T = pages_of(L), Tv = T + SHARE_COST;
    const long long rem = cur - prefix[b];
    const int it = (int)(rem / Tv), x0 = (int)(rem - (long long)it * Tv);     // item h * n_rt + row block
    const int h = it / per_head, rt = it - h * per_head;
    const int n_list = (int)min((long long)(Tv - x0), end - cur);
    const long long seg_at = cur;
    cur += n_list;
    const int t0 = max(x0 - SHARE_COST, 0), t1 = x0 + n_list - SHARE_COST;
    if (t1 <= t0) continue;                          // only the cost of starting: no pages here
    const int r0 = rt * RT;
    const int rows = min(RT, p.n_q * p.G - r0);
    const int Tc = (L + SPACE_PAGE_SIZE - 1) / SPACE_PAGE_SIZE;        // pages of the cache; page Tc is the block's rows
    const int c1 = min(t1, Tc);

    // this warp's blocks: rows [32 warp, +32) of pages t0 .. c1-1; a sequence's last page may leave it none
    int n_blk = *abort_flag ? 0 : max(c1 - t0, 0);   // (after a wait that ran out: no more requests, but every item is counted)
    if (*abort_flag && p.status && threadIdx.x == 0) atomicOr(p.status + b, SPACE_ST_TIMEOUT);
    if (n_blk > 0 && L - (c1 - 1) * SPACE_PAGE_SIZE <= warp * BLOCK_ROWS) --n_blk;
    const int32_t* table = p.cache.page_table + (int64_t)b * p.cache.pages_per_seq;
    const char* head = p.cache.pool + (int64_t)h * p.cache.head_stride + warp * F::BLOCK;
    int pages = 0, pages0 = -32;                     // lane j: page of tile t0 + pages0 + j
    uint32_t good = 0;                               // bit j: that page is in the pool
    auto look = [&](int j) {                         // pages of the 32 tiles that tile j is among (converged warp)
      if (j - pages0 < 32) return;
      pages0 = j;
      const int at = t0 + j + lane;
      pages = (j + lane < n_blk && at < p.cache.pages_per_seq) ? table[at] : -1;
      const bool ok = pages >= 0 && pages < p.cache.n_pages;
      good = __ballot_sync(0xFFFFFFFFu, ok);
      if (!ok && j + lane < n_blk && p.status) atomicOr(p.status + b, SPACE_ST_BAD_PAGE);
    };
    // (requests run STAGES - 1 blocks ahead of the products, so they look pages up first; whether the page was good
    // travels with the request as a bit per stage)
    uint32_t staged = 0;
    auto request = [&](int j, uint32_t at) {
      if (j >= n_blk) return;
      look(j);
      const int pg = __shfl_sync(0xFFFFFFFFu, pages, j - pages0);
      const uint32_t s = at % STAGES;
      const bool ok = (good >> (j - pages0)) & 1u;
      staged = (staged & ~(1u << s)) | (uint32_t)ok << s;
      if (lane == 0) {
        if (ok) {
          mbar_expect_tx(bar + 8 * s, F::BLOCK);
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                       ::"r"(ring + s * F::BLOCK), "l"(head + (int64_t)pg * p.cache.page_stride), "r"(F::BLOCK), "r"(bar + 8 * s) : "memory");
        } else {
          mbar_arrive(bar + 8 * s);
        }
      }
    };
#pragma unroll
    for (int j = 0; j < STAGES - 1; ++j) request(j, step + j);

    q.load(p, b, h, r0, lane);
    acc.clear();
    for (int j = 0; j < n_blk; ++j, ++step) {
      request(j + STAGES - 1, step + STAGES - 1);
      const uint32_t s = step % STAGES, parity = (step / STAGES) & 1;
      if (!mbar_try(bar + 8 * s, parity) && !wait_long(bar + 8 * s, parity, abort_flag, p.err, 40 + warp)) {
        if (p.status && lane == 0) atomicOr(p.status + b, SPACE_ST_TIMEOUT);
        // what is on its way has to land before the ring is used for anything else
        const uint32_t issued = step + min(STAGES, n_blk - j);
        for (; step < issued; ++step) mbar_drain_bounded(bar + 8 * (step % STAGES), (step / STAGES) & 1, WAIT_NS);
        break;
      }
      if (!((staged >> s) & 1u)) continue;           // a page outside the pool: its keys are left out
      const uint32_t blk = ring + s * F::BLOCK;
      const int valid = min(L - (t0 + j) * SPACE_PAGE_SIZE - warp * BLOCK_ROWS, BLOCK_ROWS);   // keys of this block, >= 1

      // ---- S = Q U^T: keys 8 nt + lane / 4 of the block are the columns of product nt
      float sc[4][4];
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
        uint32_t w[DH / 32];
        const uint32_t at = blk + (8 * nt + (lane >> 2)) * (DH / 2) + t * (DH / 8);
        if (DH == 128) {
          const uint4 v = lds128(at);
          w[0] = v.x; w[1] = v.y; w[2 % (DH / 32)] = v.z; w[3 % (DH / 32)] = v.w;
        } else {
          const uint2 v = lds64(at);
          w[0] = v.x; w[1] = v.y;
        }
#pragma unroll
        for (int k = 0; k < DH / 32; ++k) {
          const uint32_t u = w[k] >> 8;
          mma(sc[nt], q.a[2 * k][0], q.a[2 * k][1], q.a[2 * k][2], q.a[2 * k][3], w[k] & 0x000F000Fu, w[k] & 0x00F000F0u);
          mma(sc[nt], q.a[2 * k + 1][0], q.a[2 * k + 1][1], q.a[2 * k + 1][2], q.a[2 * k + 1][3], u & 0x000F000Fu, u & 0x00F000F0u);
        }
      }
      // ---- steps and lowest values of keys 8 nt + 2t, + 1
      float ks[4][2], kz[4][2], vs[4][2], vz[4][2];
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        uint2 kp = lds64(blk + F::K_PAR + (8 * nt + 2 * t) * 4), vp = lds64(blk + F::V_PAR + (8 * nt + 2 * t) * 4);
        if (valid < BLOCK_ROWS) {                    // rows past the end may hold anything
          if (8 * nt + 2 * t >= valid) kp.x = vp.x = 0;
          if (8 * nt + 2 * t + 1 >= valid) kp.y = vp.y = 0;
        }
        const float c24 = q.c * 16777216.f;          // undoes the codes' 2^-24
        ks[nt][0] = bf_lo(kp.x) * c24; ks[nt][1] = bf_lo(kp.y) * c24;
        kz[nt][0] = bf_hi(kp.x); kz[nt][1] = bf_hi(kp.y);
        vs[nt][0] = bf_lo(vp.x); vs[nt][1] = bf_lo(vp.y);
        vz[nt][0] = fmaf(vs[nt][0], 8.f, bf_hi(vp.x)); vz[nt][1] = fmaf(vs[nt][1], 8.f, bf_hi(vp.y));
      }
      // ---- scores relative to the rows' references, which move when a score exceeds them by 2^8
      float ref0 = acc.m[0] == -CUDART_INF_F ? 0.f : acc.m[0], ref1 = acc.m[1] == -CUDART_INF_F ? 0.f : acc.m[1];
      float mx0 = -CUDART_INF_F, mx1 = -CUDART_INF_F;
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          sc[nt][e] = fmaf(sc[nt][e], ks[nt][e], fmaf(kz[nt][e], q.sum[0], -ref0));
          sc[nt][2 + e] = fmaf(sc[nt][2 + e], ks[nt][e], fmaf(kz[nt][e], q.sum[1], -ref1));
          if (valid < BLOCK_ROWS && 8 * nt + 2 * t + e >= valid) sc[nt][e] = sc[nt][2 + e] = -CUDART_INF_F;
          mx0 = fmaxf(mx0, sc[nt][e]); mx1 = fmaxf(mx1, sc[nt][2 + e]);
        }
      }
      const bool fresh = acc.m[0] == -CUDART_INF_F || acc.m[1] == -CUDART_INF_F;
      if (__any_sync(0xFFFFFFFFu, fresh || mx0 > REF_SLACK || mx1 > REF_SLACK)) {
        const float n0 = quad_max(mx0) + ref0, n1 = quad_max(mx1) + ref1;
        acc.raise(n0, n1);
        acc.set_vinv();
        const float s0 = ref0 - (acc.m[0] == -CUDART_INF_F ? 0.f : acc.m[0]), s1 = ref1 - (acc.m[1] == -CUDART_INF_F ? 0.f : acc.m[1]);
#pragma unroll
        for (int nt = 0; nt < 4; ++nt) { sc[nt][0] += s0; sc[nt][1] += s0; sc[nt][2] += s1; sc[nt][3] += s1; }
      }
      // ---- e, its sums, and the weights e step in f16
      float t0 = 0.f, t1 = 0.f;
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        const float e0 = fast_exp2(sc[nt][0]), e1 = fast_exp2(sc[nt][1]), e2 = fast_exp2(sc[nt][2]), e3 = fast_exp2(sc[nt][3]);
        acc.l[0] += e0 + e1; acc.l[1] += e2 + e3;
        acc.z[0] = fmaf(e0, vz[nt][0], fmaf(e1, vz[nt][1], acc.z[0]));
        acc.z[1] = fmaf(e2, vz[nt][0], fmaf(e3, vz[nt][1], acc.z[1]));
        sc[nt][0] = e0 * vs[nt][0]; sc[nt][1] = e1 * vs[nt][1]; sc[nt][2] = e2 * vs[nt][0]; sc[nt][3] = e3 * vs[nt][1];
        t0 = max3(t0, sc[nt][0], sc[nt][1]); t1 = max3(t1, sc[nt][2], sc[nt][3]);
      }
      if (__any_sync(0xFFFFFFFFu, t0 * acc.vinv[0] > W_LIMIT || t1 * acc.vinv[1] > W_LIMIT)) acc.set_scale(t0, t1);
      uint32_t pa[2][4];
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        pa[nt >> 1][2 * (nt & 1)] = pack_h(sc[nt][0] * acc.vinv[0], sc[nt][1] * acc.vinv[0]);
        pa[nt >> 1][2 * (nt & 1) + 1] = pack_h(sc[nt][2] * acc.vinv[1], sc[nt][3] * acc.vinv[1]);
      }
      // ---- O += P (U - 8): channels 8 (4 wd + qd) + lane / 4 are the columns
#pragma unroll
      for (int wd = 0; wd < DH / 32; ++wd) {
        const uint4 v = lds128(blk + F::CODES + 512 * wd + 16 * lane);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        const uint32_t c0 = 0x00080008u, c1_ = 0x00800080u;                    // 8 in units of 2^-24 and 2^-20
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const uint32_t x = w[2 * a], y = w[2 * a + 1], xs = x >> 8, ys = y >> 8;
          mma(acc.o[4 * wd + 0], pa[a][0], pa[a][1], pa[a][2], pa[a][3], h2sub(x & 0x000F000Fu, c0), h2sub(y & 0x000F000Fu, c0));
          mma(acc.o[4 * wd + 1], pa[a][0], pa[a][1], pa[a][2], pa[a][3], h2sub(x & 0x00F000F0u, c1_), h2sub(y & 0x00F000F0u, c1_));
          mma(acc.o[4 * wd + 2], pa[a][0], pa[a][1], pa[a][2], pa[a][3], h2sub(xs & 0x000F000Fu, c0), h2sub(ys & 0x000F000Fu, c0));
          mma(acc.o[4 * wd + 3], pa[a][0], pa[a][1], pa[a][2], pa[a][3], h2sub(xs & 0x00F000F0u, c1_), h2sub(ys & 0x00F000F0u, c1_));
        }
      }
      __syncwarp();                                  // the stage is free for the next request
    }
    // ---- accumulators in real units
    {
      float f[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) f[s] = acc.R[s] == -CUDART_INF_F ? 1.f : fast_exp2(acc.R[s] - acc.m[s] - 6.f);
#pragma unroll
      for (int nt = 0; nt < DH / 8; ++nt) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc.o[nt][e] = acc.o[nt][e] * ((nt & 1) ? 1048576.f : 16777216.f) * f[e >> 1];
      }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) { acc.l[s] = quad_sum(acc.l[s]); acc.z[s] = quad_sum(acc.z[s]); }
#pragma unroll
    for (int nt = 0; nt < DH / 8; ++nt) {
      acc.o[nt][0] += acc.z[0]; acc.o[nt][1] += acc.z[0]; acc.o[nt][2] += acc.z[1]; acc.o[nt][3] += acc.z[1];
    }
    acc.z[0] = acc.z[1] = 0.f;

    // ---- the block's own rows: keys 16 warp .. + 15 of it, as f16 scaled by a power of two per key
    if (t1 > Tc && p.has_new && 16 * warp < p.n_q && L0 >= 0) {
      const int k0 = 16 * warp;
      float sc[2][4], kf[2];
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
        sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
        const int key = k0 + 8 * nt + (lane >> 2);
        uint4 raw[DH / 32];
        uint32_t topk = 0;
        const uint4* src = reinterpret_cast<const uint4*>(p.kn + (int64_t)b * p.n_sb + (int64_t)key * p.n_sr + (int64_t)h * p.n_sh) + t * (DH / 32);
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) {
          raw[j] = key < p.n_q ? src[j] : make_uint4(0, 0, 0, 0);
          if (any_nonfinite(raw[j])) raw[j] = make_uint4(finite_pair(raw[j].x), finite_pair(raw[j].y), finite_pair(raw[j].z), finite_pair(raw[j].w));
          const uint32_t m2 = __vmaxu2(__vmaxu2(raw[j].x & 0x7FFF7FFFu, raw[j].y & 0x7FFF7FFFu), __vmaxu2(raw[j].z & 0x7FFF7FFFu, raw[j].w & 0x7FFF7FFFu));
          topk = max(topk, max(m2 & 0xFFFFu, m2 >> 16));
        }
        topk = max(topk, __shfl_xor_sync(0xFFFFFFFFu, topk, 1));
        topk = max(topk, __shfl_xor_sync(0xFFFFFFFFu, topk, 2));
        const int e = topk ? min(127 - (int)(topk >> 7), 120) : 0;           // largest element in [1, 2)
        const float f = pow2(max(e, -126)), f16x = f * 16.f;
        kf[nt] = pow2(-max(e, -126));
#pragma unroll
        for (int k = 0; k < DH / 32; ++k) {
          const uint4 v = raw[k];
          mma(sc[nt], q.a[2 * k][0], q.a[2 * k][1], q.a[2 * k][2], q.a[2 * k][3],
              pack_h(bf_lo(v.x) * f, bf_lo(v.z) * f), pack_h(bf_hi(v.x) * f16x, bf_hi(v.z) * f16x));
          mma(sc[nt], q.a[2 * k + 1][0], q.a[2 * k + 1][1], q.a[2 * k + 1][2], q.a[2 * k + 1][3],
              pack_h(bf_lo(v.y) * f, bf_lo(v.w) * f), pack_h(bf_hi(v.y) * f16x, bf_hi(v.w) * f16x));
        }
      }
      // V rows into the (dry) ring as f16, largest element of a row in [1, 2); eight channels a lane
      constexpr int LANES = DH / 8;
      int ve[16 / (32 / LANES)];                     // exponent of row 32/LANES * i + lane / LANES
#pragma unroll
      for (int i = 0; i < 16 * LANES / 32; ++i) {
        const int row = i * (32 / LANES) + lane / LANES, key = k0 + row;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (key < p.n_q) v = *(reinterpret_cast<const uint4*>(p.vn + (int64_t)b * p.n_sb + (int64_t)key * p.n_sr + (int64_t)h * p.n_sh) + lane % LANES);
        if (any_nonfinite(v)) v = make_uint4(finite_pair(v.x), finite_pair(v.y), finite_pair(v.z), finite_pair(v.w));
        const uint32_t m2 = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
        uint32_t topv = max(m2 & 0xFFFFu, m2 >> 16);
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) topv = max(topv, __shfl_xor_sync(0xFFFFFFFFu, topv, o));
        ve[i] = min(max((int)(topv >> 7) - 127, -110), 126);
        const float f = pow2(-ve[i]);
        const uint4 hv = make_uint4(pack_h(bf_lo(v.x) * f, bf_hi(v.x) * f), pack_h(bf_lo(v.y) * f, bf_hi(v.y) * f),
                                    pack_h(bf_lo(v.z) * f, bf_hi(v.z) * f), pack_h(bf_lo(v.w) * f, bf_hi(v.w) * f));
        const uint32_t at = ring + row * S::V_PITCH + (lane % LANES) * 16;
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(hv.x), "r"(hv.y), "r"(hv.z), "r"(hv.w) : "memory");
      }
      __syncwarp();
      // scores, Eq. 5; keys 8 nt + 2t + e of this warp's sixteen are this lane's columns
      float mx[2] = {-CUDART_INF_F, -CUDART_INF_F}, big[2] = {0.f, 0.f};
      int vx[2], kve[2][2];
      uint64_t see[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int r = r0 + (lane >> 2) + 8 * s;
        see[s] = r < p.n_q * p.G ? p.mask[r / p.G] : 0ull;
      }
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int col = 2 * t + e;                 // key 8 nt + col: its K factor sits in lane 4 col, its V exponent where its row was read
          const float f = __shfl_sync(0xFFFFFFFFu, kf[nt], 4 * col);
          const int row = 8 * nt + col;
          int vexp_k = 0;
#pragma unroll
          for (int i = 0; i < 16 * LANES / 32; ++i) {
            const int got = __shfl_sync(0xFFFFFFFFu, ve[i], (row % (32 / LANES)) * LANES);
            if (i == row / (32 / LANES)) vexp_k = got;
          }
          kve[nt][e] = vexp_k;
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            float& x = sc[nt][2 * s + e];
            const bool vis = (see[s] >> (k0 + row)) & 1ull;
            x *= fminf(f * q.c, 1e38f);              // (rows next to the largest number: a score stays one, and NaN NaN)
            x = !vis ? -CUDART_INF_F : x > 1e38f ? 1e38f : x < -1e38f ? -1e38f : x;
            mx[s] = fmaxf(mx[s], x);
          }
        }
      }
      const float2 down = acc.raise(quad_max(mx[0]), quad_max(mx[1]));
      acc.scale_rows(down.x, down.y);
#pragma unroll
      for (int nt = 0; nt < DH / 8; ++nt) {
        big[0] = fmaxf(big[0], fmaxf(fabsf(acc.o[nt][0]), fabsf(acc.o[nt][1])));
        big[1] = fmaxf(big[1], fmaxf(fabsf(acc.o[nt][2]), fabsf(acc.o[nt][3])));
      }
      // weights e 2^(exponent of the V row); they and the accumulators go down by the power of two of the row's largest
      float lb[2] = {0.f, 0.f};
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            float& x = sc[nt][2 * s + e];
            const float ex = x == -CUDART_INF_F ? 0.f : fast_exp2(x - acc.m[s]);
            lb[s] += ex;
            x = ex * pow2(kve[nt][e]);
            big[s] = fmaxf(big[s], x);
          }
        }
      }
      float wf[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        vx[s] = min(max((int)(__float_as_uint(quad_max(big[s])) >> 23) - 127, -110), 126);
        wf[s] = pow2(-vx[s]);
      }
      acc.scale_rows(wf[0] * 1024.f, wf[1] * 1024.f);
      uint32_t pa[4];
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
        pa[2 * nt] = pack_h(sc[nt][0] * wf[0] * 1024.f, sc[nt][1] * wf[0] * 1024.f);
        pa[2 * nt + 1] = pack_h(sc[nt][2] * wf[1] * 1024.f, sc[nt][3] * wf[1] * 1024.f);
      }
#pragma unroll
      for (int nt = 0; nt < DH / 8; ++nt) {
        uint32_t b0, b1;
        const uint32_t at = ring + (lane & 15) * S::V_PITCH + nt * 16;
        asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];" : "=r"(b0), "=r"(b1) : "r"(at) : "memory");
        mma(acc.o[nt], pa[0], pa[1], pa[2], pa[3], b0, b1);
      }
      acc.scale_rows(pow2(vx[0]) * 0.0009765625f, pow2(vx[1]) * 0.0009765625f);
      acc.l[0] += quad_sum(lb[0]); acc.l[1] += quad_sum(lb[1]);
      __syncwarp();
    }

    // ---- the four warps' states meet
    if (t == 0) {
      ml[warp * RT + (lane >> 2)] = make_float2(acc.m[0], acc.l[0]);
      ml[warp * RT + (lane >> 2) + 8] = make_float2(acc.m[1], acc.l[1]);
    }
    __syncthreads();
    const bool whole = t0 == 0 && t1 == T;
    {
      float f[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int r = (lane >> 2) + 8 * s;
        float M = -CUDART_INF_F;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) M = fmaxf(M, ml[w * RT + r].x);
        f[s] = acc.m[s] == -CUDART_INF_F ? 0.f : fast_exp2(acc.m[s] - M);
        // (a row that is not a number keeps no reference; its sums say so)
        if (acc.l[s] != acc.l[s]) f[s] = 1.f;
      }
      float* mine = reinterpret_cast<float*>(sm + warp * S::RING);
#pragma unroll
      for (int nt = 0; nt < DH / 8; ++nt) {
        *reinterpret_cast<float2*>(mine + (lane >> 2) * S::O_PITCH + 8 * nt + 2 * t) = make_float2(acc.o[nt][0] * f[0], acc.o[nt][1] * f[0]);
        *reinterpret_cast<float2*>(mine + ((lane >> 2) + 8) * S::O_PITCH + 8 * nt + 2 * t) = make_float2(acc.o[nt][2] * f[1], acc.o[nt][3] * f[1]);
      }
    }
    __syncthreads();
    int piece0 = 0, pieces = 1, slot = 0;
    const long long first_page = prefix[b] + (long long)it * Tv + SHARE_COST;   // the item's first page in the list
    if (!whole) {
      piece0 = attn::group_of(first_page, W, NG);
      pieces = attn::group_of(first_page + T - 1, W, NG) - piece0 + 1;
      slot = 2 * (int)blockIdx.x + (seg_at == share0 ? 0 : 1);
    }
    constexpr int C4 = DH / 4;
    constexpr int SLOT = RT * (DH + 2);
    for (int idx = threadIdx.x; idx < rows * C4; idx += THREADS) {
      const int r = idx / C4, c4 = idx % C4;
      float M = -CUDART_INF_F, l = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) M = fmaxf(M, ml[w * RT + r].x);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float2 v = ml[w * RT + r];
        l += v.y * (v.x == -CUDART_INF_F ? (v.y != v.y ? 1.f : 0.f) : fast_exp2(v.x - M));
        const float4 x = *reinterpret_cast<const float4*>(sm + w * S::RING + (r * S::O_PITCH + 4 * c4) * 4);
        o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
      }
      if (whole) {
        store_row4<DH>(p, b, h, r0 + r, c4, o, M, l);
      } else {
        float* ps = p.part + (int64_t)slot * SLOT;
        __stcg(reinterpret_cast<float4*>(ps + r * DH) + c4, o);
        if (c4 == 0) { __stcg(ps + RT * DH + r, M); __stcg(ps + RT * DH + RT + r, l); }
      }
    }
    if (!whole) {
      const int item = (b * p.H_kv + h) * p.n_rt + rt;
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) {
        const int last = atomicAdd(p.arrived + item, 1) == pieces - 1;
        if (last) p.arrived[item] = 0;               // ready for the next call
        __threadfence();
        *last_flag = last;
      }
      __syncthreads();
      if (*last_flag) {
        // piece 0 stands in the second slot of its block unless the item began with that block's share
        const long long begin0 = attn::muldiv(W, piece0, NG);
        const int first_slot = 2 * piece0 + (begin0 >= first_page - SHARE_COST ? 0 : 1);
        for (int idx = threadIdx.x; idx < rows * C4; idx += THREADS) {
          const int r = idx / C4, c4 = idx % C4;
          attn::MergeAcc ma;
          ma.clear();
          bool nan = false;
          for (int x0 = 0; x0 < pieces; x0 += 4) {
            float ms[4], ls[4];
            float4 ov[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              ms[j] = -CUDART_INF_F; ls[j] = 0.f; ov[j] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (x0 + j < pieces) {
                const float* ps = p.part + (int64_t)(x0 + j == 0 ? first_slot : 2 * (piece0 + x0 + j)) * SLOT;
                ms[j] = __ldcg(ps + RT * DH + r);
                ls[j] = __ldcg(ps + RT * DH + RT + r);
                ov[j] = __ldcg(reinterpret_cast<const float4*>(ps + r * DH) + c4);
              }
              nan |= ls[j] != ls[j];
            }
            ma.add4(ms, ls, ov);
          }
          if (nan) ma.den = CUDART_NAN_F;
          store_row4<DH>(p, b, h, r0 + r, c4, ma.a, ma.mx, ma.den);
        }
      }
    }
    __syncthreads();                                 // everybody has read the rings: the next item's requests may fill them
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
}

template <int DH>
size_t smem_bytes(int max_batch) { return Smem<DH>::TABLE_OFF + (size_t)(max_batch + 1) * 8 + (size_t)max_batch * 4; }

template <int DH>
cudaError_t launch_dim(const Params& p, int max_batch, cudaStream_t st) {
  static unsigned long long done_mask = 0;           // devices on which the kernel may have its shared memory
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 64 || !((done_mask >> dev) & 1ull)) {
    cudaFuncSetAttribute(kvq_attn_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<DH>(128));
    if (dev < 64) done_mask |= 1ull << dev;
  }
  return launch_pdl(kvq_attn_kernel<DH>, dim3(p.n_groups), dim3(THREADS), smem_bytes<DH>(max_batch), st, p, max_batch);
}

}  // namespace

size_t kvq_partial_floats(const space_config* c, int sm_count) {
  return (size_t)2 * CTAS_PER_SM * sm_count * RT * (c->head_dim + 2);
}
size_t kvq_items(const space_config* c) {
  const size_t rows = (size_t)(c->k_max + 1) * (c->k_max + 1) * (c->n_q_heads / c->n_kv_heads);
  return (size_t)c->max_batch * c->n_kv_heads * ((rows + RT - 1) / RT);
}

int launch_kvq_attn(space_ctx* ctx, const space_kvq_attn_args* a, const uint64_t* mask_rows, cudaStream_t st) {
  Params p;
  memset(&p, 0, sizeof(p));
  p.cache = cache_of(a->cache);
  p.B = a->batch; p.n_q = (a->k + 1) * (a->k + 1); p.H_q = ctx->cfg.n_q_heads; p.H_kv = ctx->cfg.n_kv_heads;
  p.G = p.H_q / p.H_kv;
  p.n_rt = (p.n_q * p.G + RT - 1) / RT;
  p.n_groups = CTAS_PER_SM * ctx->sm_count;
  p.has_new = a->k_new != nullptr;
  p.c = a->scale * 1.4426950408889634f;
  p.q = (const char*)a->q; p.q_sb = 2 * a->q_stride_b; p.q_sr = 2 * a->q_stride_r; p.q_sh = 2 * a->q_stride_h;
  p.kn = (const char*)a->k_new; p.vn = (const char*)a->v_new;
  p.n_sb = 2 * a->new_stride_b; p.n_sr = 2 * a->new_stride_r; p.n_sh = 2 * a->new_stride_h;
  p.kv_len = a->kv_len; p.out = (__nv_bfloat16*)a->out; p.lse = a->lse; p.status = a->status;
  p.part = ctx->attn_part; p.arrived = ctx->kvq_arrived; p.err = ctx->counters + 3 * ctx->cfg.max_batch;
  for (int i = 0; i < p.n_q; ++i) p.mask[i] = mask_rows[i];
  const cudaError_t e = ctx->cfg.head_dim == 128 ? launch_dim<128>(p, ctx->cfg.max_batch, st) : launch_dim<64>(p, ctx->cfg.max_batch, st);
  ctx->launches += 1;
  return cuda_ok(e);
}
