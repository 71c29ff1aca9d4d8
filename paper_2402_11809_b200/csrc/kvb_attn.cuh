// What the two attention kernels over the 8-bit cache share (kvb_attn.cu: items of 8 or 16 query rows on mma.sync;
// kvb_attn_tc.cu: of 32, 64 or 128 on tcgen05): parameters, the split into two e4m3 terms, the join of an item's pieces.
#pragma once
#include "kvq_attn.cuh"
#include "kvb_common.cuh"

namespace kvb {
using kvq::Cut;
using kvq::lds128;
using kvq::lds64;
using kvq::mul2;
using kvq::wait;
using kvq::warp_wait;
using kvq::WAIT_NS;
using namespace tc;

constexpr float F_MIN = 0x1p-120f, F_MAX = 0x1p75f;  // factor of a score: products stay numbers, and differ from 0
constexpr float SCORE_MAX = 0x1p29f;                 // scores are held to this (log2 units)

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
  float* part;                                       // [2 * n_groups][rows * (DH + 2)]: outputs of a piece, then M, l of its rows
  int* arrived;                                      // [B * H_kv * n_rt], self-resetting
  int* err;
  uint64_t mask[SPACE_MAX_ROWS];                     // Eq. 5: bit j of word i: block row i sees block row j
};

// One decision of several warps after a wait: `all` is a barrier of them that tells each whether all of them were told that it is there.
// (While another wait runs out, some can be told so and others that it was given up, and a barrier that only some of them reach has no end.)
#pragma nv_exec_check_disable
template <class Hold, class All>
__host__ __device__ __forceinline__ bool all_told(Hold hold, All all) { return all(hold()); }

// Where a kv head's query row r lies: block row and head.  (G is a power of two.)
__device__ __forceinline__ void row_of(const Params& p, int h, int r, int& i, int& hq) {
  i = r >> p.gsh;
  hq = (h << p.gsh) + (r & ((1 << p.gsh) - 1));
}

// Four numbers as two e4m3 terms each: w0 the codes nearest to them, w1 those of what is left (exact: its bits are the ones
// that the first term dropped).
__device__ __forceinline__ void split4(float a, float b, float c, float d, uint32_t& w0, uint32_t& w1) {
  const uint32_t x = codes2(a, b), y = codes2(c, d);
  const uint32_t hx = halves2(x), hy = halves2(y);
  asm("{\n\t.reg .b16 p, q, m;\n\tmov.b32 {p, q}, %4;\n\tmov.b16 m, 0xBC00;\n\t"       // -1
      "fma.rn.f32.f16 %0, p, m, %2;\n\tfma.rn.f32.f16 %1, q, m, %3;\n\t}" : "=f"(a), "=f"(b) : "f"(a), "f"(b), "r"(hx));
  asm("{\n\t.reg .b16 p, q, m;\n\tmov.b32 {p, q}, %4;\n\tmov.b16 m, 0xBC00;\n\t"
      "fma.rn.f32.f16 %0, p, m, %2;\n\tfma.rn.f32.f16 %1, q, m, %3;\n\t}" : "=f"(c), "=f"(d) : "f"(c), "f"(d), "r"(hy));
  w0 = x | y << 16;
  w1 = codes4(a, b, c, d);
}

// Four channels of a row's mean over an item's, or a piece's, keys.  A mean of V rows is a number of their type; weights are rounded, their
// sum is not, so that a mean of the largest ones would pass them.  (NaN stays.)
__device__ __forceinline__ float4 held(float4 o) {
  const float most = 3.3895313892515355e38f;
  auto one = [&](float v) { return v > most ? most : v < -most ? -most : v; };
  return make_float4(one(o.x), one(o.y), one(o.z), one(o.w));
}

// Four channels of a finished row.
template <int DH>
__device__ __forceinline__ void store_row4(const Params& p, int b, int h, int r, int c4, float4 o) {
  int i, hq;
  row_of(p, h, r, i, hq);
  const __nv_bfloat162 x = __floats2bfloat162_rn(o.x, o.y), y = __floats2bfloat162_rn(o.z, o.w);
  __nv_bfloat16* dst = p.out + (((int64_t)b * p.n_q + i) * p.H_q + hq) * DH + 4 * c4;
  *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
}
__device__ __forceinline__ void store_lse(const Params& p, int b, int h, int r, float M, float l) {
  if (!p.lse) return;
  int i, hq;
  row_of(p, h, r, i, hq);
  p.lse[((int64_t)b * p.H_q + hq) * p.n_q + i] = (M + log2f(l)) * 0.6931471805599453f;
}

// The pieces of an item that was cut over several thread blocks: outputs of their own keys, weighed by their share l 2^M of all keys,
// always in the same order (every factor is 1 at most, that of what has been joined so far among them: means of V rows stay as large as
// those, whatever their sums would be); called by the block that stored the last of them, by whole warps.  item_at: the item's place in the
// flat list; a block's share can hold the end of one cut item (its first slot) and the start of another (its second one).
// A thread has four channels of U query rows; the DH / 4 threads of a row look up that many pieces' M and l at
// once, while BATCH pieces' outputs are on their way.
template <int DH, int RT, int U, int BATCH>
__device__ __forceinline__ void join_pieces(const Params& p, const Cut& cut, int b, int h, int r0, int rows, uint32_t piece0, int pieces, uint32_t item_at, int tid, int threads) {
  constexpr int C4 = DH / 4, SLOT = RT * (DH + 2);
  const float* part = p.part + (int64_t)(2 * piece0) * SLOT;
  const int first = cut.begin(piece0) >= item_at ? 0 : SLOT, n = rows * C4, c4 = tid % C4;
  auto at = [&](int x) { return part + (x == 0 ? (int64_t)first : (int64_t)x * (2 * SLOT)); };
#pragma unroll 1
  for (int idx = tid - tid % 32; idx < n; idx += U * threads) {                // (warps stay whole)
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
      float m[U], l[U], w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool there = x0 + c4 < pieces;
        m[u] = there ? __ldcg(at(x0 + c4) + RT * DH + r[u]) : -CUDART_INF_F;
        l[u] = there ? __ldcg(at(x0 + c4) + RT * DH + RT + r[u]) : 0.f;
        w[u] = 0.f;
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
            float top = m[u];
#pragma unroll
            for (int k = 1; k < C4; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, k));
            top = fmaxf(top, M[u]);
            const float down = M[u] == -CUDART_INF_F ? 0.f : fast_exp2(M[u] - top);
            M[u] = top;
            w[u] = m[u] == -CUDART_INF_F ? 0.f : l[u] * fast_exp2(m[u] - top);
            float sum = w[u];
#pragma unroll
            for (int k = 1; k < C4; k <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, k);
            const float before = den[u] * down;
            den[u] = before + sum;
            const float rd = den[u] > 0.f ? __fdividef(1.f, den[u]) : 0.f;     // (a row without keys: zeros; NaN stays)
            const float f = before * rd;
            w[u] *= rd;
            o[u].x *= f; o[u].y *= f; o[u].z *= f; o[u].w *= f;
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < BATCH; ++j) {
            const float f = __shfl_sync(0xFFFFFFFFu, w[u], y + j, C4);         // (past the last piece: v is 0)
            o[u].x = fmaf(v[u][j].x, f, o[u].x); o[u].y = fmaf(v[u][j].y, f, o[u].y);
            o[u].z = fmaf(v[u][j].z, f, o[u].z); o[u].w = fmaf(v[u][j].w, f, o[u].w);
          }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (idx + tid % 32 + u * threads < n) {
        store_row4<DH>(p, b, h, r0 + r[u], c4, o[u]);
        if (c4 == 0) store_lse(p, b, h, r0 + r[u], M[u], den[u]);
      }
  }
}

}  // namespace kvb

int launch_kvb_attn_tc(space_ctx* ctx, kvb::Params& p, cudaStream_t st);
