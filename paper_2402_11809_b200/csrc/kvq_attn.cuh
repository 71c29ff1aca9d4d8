// What the two attention kernels over the 4-bit cache share (kvq_attn.cu: items of 8, 16 or 24 query rows on mma.sync;
// kvq_attn_tc.cu: of 64 on tcgen05): parameters, addresses of query rows, the join of an item's pieces.
#pragma once
#include "common.cuh"
#include "tc_common.cuh"
#include "attn_common.cuh"
#include "kvq_common.cuh"
#include <cuda_fp16.h>
#include <math_constants.h>

namespace kvq {
using namespace tc;

constexpr float FAR_BELOW = -4096.f;                 // a reference below this is not taken into the scores of later keys, whose bits it would cost
// Keys whose step, times a score's factors, is beyond this (rows that hold numbers next to the largest one): their scores are
// taken 2^-64 times as large and held to the range of numbers.  The lowest value is 4096 steps at most and the sums of query
// rows are of 128 elements: below the limit no term of a score passes 2^104.
constexpr float K_LARGE = 0x1p100f;
constexpr float SCORE_MAX = 1e38f;                   // (log2 units; the difference of two of them is a number)
constexpr float W_LIMIT = 16384.f;                   // weights of the second product stay below this (f16 ends at 65504)
constexpr float V_UNIT = 0x1p-32f;                   // of sums of V rows: with rows next to the largest number they stay numbers (2^24 keys of weight 2^8)
constexpr uint64_t WAIT_NS = 1000000000ull;

struct Params {
  Cache cache;
  int B, n_q, H_q, H_kv, G, gsh, n_rt;               // G = 1 << gsh; n_rt: items per (sequence, kv head)
  int n_groups;                                      // thread blocks
  int has_new;
  float c;                                           // scale * log2(e)
  const char* q; int64_t q_sb, q_sr, q_sh;           // bytes
  const char* kn; const char* vn; int64_t n_sb, n_sr, n_sh;
  const int32_t* kv_len;
  __nv_bfloat16* out; float* lse; int32_t* status;
  float* part;                                       // [2 * n_groups][rows * (DH + 2)]: sums times V_UNIT, references, sums of e
  int* arrived;                                      // [B * H_kv * n_rt], self-resetting
  int* err;
  uint64_t mask[SPACE_MAX_ROWS];                     // Eq. 5: bit j of word i: block row i sees block row j
};

// Bounded wait on an mbarrier phase, small enough to stand inline at every site (roles that run with register counts of
// their own cannot call): after WAIT_NS, or once another wait of the block has given up, false and the abort flag.
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* err, int site) {
  if (mbar_try(bar, parity)) return true;
  const uint64_t t0 = global_ns();
#pragma unroll 1
  while (!mbar_try(bar, parity)) {
    if (*abort_flag || global_ns() - t0 > WAIT_NS) {
      *abort_flag = 1;
      atomicCAS(err, 0, site);
      return false;
    }
  }
  return true;
}

// The same by a whole warp: one answer for all of its lanes.  (Each tries for itself: while another wait runs out, some could find the
// phase there and others the flag, and the lanes of a warp that goes by it would part for good.)
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* err, int site) {
  return __all_sync(0xFFFFFFFFu, wait(bar, parity, abort_flag, err, site));
}

__device__ __forceinline__ uint32_t pack_h(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
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
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }     // -126 <= e <= 127
__device__ __forceinline__ float clamp_score(float x) {                         // (NaN stays)
  return x > SCORE_MAX ? SCORE_MAX : x < -SCORE_MAX ? -SCORE_MAX : x;
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
  return v + __shfl_xor_sync(0xFFFFFFFFu, v, 2);
}
__device__ __forceinline__ uint32_t h2sub(uint32_t a, uint32_t b) {
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// Where a kv head's query row r lies: block row and head.  (G is a power of two.)
__device__ __forceinline__ void row_of(const Params& p, int h, int r, int& i, int& hq) {
  i = r >> p.gsh;
  hq = (h << p.gsh) + (r & ((1 << p.gsh) - 1));
}

// The flat list of W pages over NG thread blocks: the first `rem` blocks take one page more.
struct Cut {
  uint32_t NG, per, rem;
  __device__ __forceinline__ Cut(uint32_t W, uint32_t groups) {
    NG = min(W, groups);
    per = NG ? W / NG : 0;
    rem = W - per * NG;
  }
  __device__ __forceinline__ uint32_t begin(uint32_t g) const { return g * per + min(g, rem); }
  __device__ __forceinline__ uint32_t owner(uint32_t f) const {                // block whose share page f is in
    const uint32_t wide = rem * (per + 1);
    return f < wide ? f / (per + 1) : rem + (f - wide) / per;
  }
};

// o: a row's sums, times V_UNIT
template <int DH>
__device__ __forceinline__ void store_row4(const Params& p, int b, int h, int r, int c4, float4 o, float m, float l) {
  int i, hq;
  row_of(p, h, r, i, hq);
  const float rd = l > 0.f || l != l ? 0x1p32f / l : 0.f;  // a row without keys: zeros
  const __nv_bfloat162 x = __floats2bfloat162_rn(o.x * rd, o.y * rd), y = __floats2bfloat162_rn(o.z * rd, o.w * rd);
  __nv_bfloat16* dst = p.out + (((int64_t)b * p.n_q + i) * p.H_q + hq) * DH + 4 * c4;
  *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
  if (c4 == 0 && p.lse) p.lse[((int64_t)b * p.H_q + hq) * p.n_q + i] = (m + log2f(l)) * 0.6931471805599453f;
}

// The pieces of an item that was cut over several thread blocks meet, always in the same order: called by the block
// that stored the last of them, by whole warps.  item_at: the item's place in the flat list; a block's share can hold the
// end of one cut item (its first slot) and the start of another (its second one).
// A thread has four channels of U query rows; the DH / 4 threads of a row look up the references and sums of as many
// pieces at once, one each, while BATCH pieces of the accumulators are on their way: what this costs is the latency of
// loads that follow each other.  131072 keys, 8 kv heads of 4 rows (74 pieces a head), us: U = 1, BATCH = 4 / 8 / 16:
// 47.5 / 45.3 / 43.5; 2048 keys, 32 heads of 36 rows (5 pieces), U, BATCH = 1, 8 / 2, 8 / 6, 4: 23.0 / 21.1 / 20.3.  (The
// tensor-memory form has registers for U = 1, BATCH = 4.)
template <int DH, int RT, int U, int BATCH>
__device__ __forceinline__ void join_pieces(const Params& p, const Cut& cut, int b, int h, int r0, int rows, uint32_t piece0,
                                            int pieces, uint32_t item_at, int tid, int threads) {
  constexpr int C4 = DH / 4, SLOT = RT * (DH + 2);
  const float* part = p.part + (int64_t)(2 * piece0) * SLOT;
  const int first = cut.begin(piece0) >= item_at ? 0 : SLOT, n = rows * C4, c4 = tid % C4;
  auto at = [&](int x) { return part + (x == 0 ? (int64_t)first : (int64_t)x * (2 * SLOT)); };
#pragma unroll 1
  for (int idx = tid - tid % 32; idx < n; idx += U * threads) {               // (warps stay whole)
    int r[U];
    float M[U], den[U];
    float4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u] = min((idx + tid % 32 + u * threads) / C4, rows - 1);
      M[u] = -CUDART_INF_F; den[u] = 0.f; o[u] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll 1
    for (int x0 = 0; x0 < pieces; x0 += C4) {
      float m[U], l[U], f[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool there = x0 + c4 < pieces;
        m[u] = there ? __ldcg(at(x0 + c4) + RT * DH + r[u]) : -CUDART_INF_F;
        l[u] = there ? __ldcg(at(x0 + c4) + RT * DH + RT + r[u]) : 0.f;
      }
#pragma unroll 1
      for (int y = 0; y < C4 && x0 + y < pieces; y += BATCH) {
        float4 v[U][BATCH];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < BATCH; ++j)
            v[u][j] = x0 + y + j < pieces ? __ldcg(reinterpret_cast<const float4*>(at(x0 + y + j) + r[u] * DH) + c4) : make_float4(0.f, 0.f, 0.f, 0.f);
        if (y == 0) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            float top = m[u], sum;
#pragma unroll
            for (int k = 1; k < C4; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, k));
            top = fmaxf(top, M[u]);
            const float down = M[u] == top ? 1.f : fast_exp2(M[u] - top);
            M[u] = top;
            f[u] = m[u] == -CUDART_INF_F ? (l[u] != l[u] ? 1.f : 0.f) : fast_exp2(m[u] - top);   // (a row that is not a number keeps no reference)
            sum = l[u] * f[u];
#pragma unroll
            for (int k = 1; k < C4; k <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, k);
            den[u] = fmaf(den[u], down, sum);
            o[u].x *= down; o[u].y *= down; o[u].z *= down; o[u].w *= down;
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < BATCH; ++j) {
            const float w = __shfl_sync(0xFFFFFFFFu, f[u], y + j, C4);
            o[u].x = fmaf(v[u][j].x, w, o[u].x); o[u].y = fmaf(v[u][j].y, w, o[u].y);
            o[u].z = fmaf(v[u][j].z, w, o[u].z); o[u].w = fmaf(v[u][j].w, w, o[u].w);
          }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (idx + tid % 32 + u * threads < n) store_row4<DH>(p, b, h, r0 + r[u], c4, o[u], M[u], den[u]);
  }
}

}  // namespace kvq

int launch_kvq_attn_tc(space_ctx* ctx, kvq::Params& p, cudaStream_t st);
