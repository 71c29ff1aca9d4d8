// Rotation of query and key rows by position (space.h, space_rope), shared by the appends to the bf16 cache (rope.cu) and
// to the 8-bit one (kvb_rows.cu).
#pragma once
#include "common.cuh"

namespace rope {

struct Table {
  const float* table;
  const int32_t* pos;
  int n_pos, rot, interleaved;
};
static inline Table table_of(const space_rope& r) { return Table{r.table, r.pos, r.n_pos, r.rot_dim, r.interleaved}; }

// The table row of source row `row` of sequence b (rows per sequence in `pos`), which becomes cache row s.
__device__ __forceinline__ const float* table_row(const Table& t, int b, int rows, int row, int64_t s, bool& bad) {
  const int64_t want = t.pos ? (int64_t)t.pos[(int64_t)b * rows + row] : s;
  const int64_t p = want < 0 ? 0 : want >= t.n_pos ? t.n_pos - 1 : want;
  bad = p != want;
  return t.table + p * t.rot;
}

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Products and sums of pairs, each rounded by itself.  (A sum as add.rn.f32x2 is fused with the product before it, which then
// is not rounded.)
__device__ __forceinline__ uint64_t pair(float a, float b) {
  return (uint64_t)__float_as_uint(a) | (uint64_t)__float_as_uint(b) << 32;
}
__device__ __forceinline__ uint64_t pair_of(uint32_t w) { return pair(lo_f(w), hi_f(w)); }
__device__ __forceinline__ float first_of(uint64_t p) { return __uint_as_float((uint32_t)p); }
__device__ __forceinline__ float second_of(uint64_t p) { return __uint_as_float((uint32_t)(p >> 32)); }
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
  return pair(__fadd_rn(first_of(a), first_of(b)), __fadd_rn(second_of(a), second_of(b)));
}

// What a lane's eight channels 8x .. 8x + 7 are multiplied by, as pairs of neighbours: themselves by c, their partners by s, the
// sine with the sign of its place (a c - b s is a c + b (-s), rounding for rounding).
struct Turn { uint64_t c[4], s[4]; };
__device__ __forceinline__ void load_turn(const Table& t, const float* row, int x, Turn& u) {
  const int half = t.rot >> 1, c0 = 8 * x;
#pragma unroll
  for (int i = 0; i < 4; ++i) u.c[i] = u.s[i] = 0ull;
  if (c0 >= t.rot) return;
  if (t.interleaved) {
    const float4 c = __ldg(reinterpret_cast<const float4*>(row) + x), s = __ldg(reinterpret_cast<const float4*>(row + half) + x);
    u.c[0] = pair(c.x, c.x); u.c[1] = pair(c.y, c.y); u.c[2] = pair(c.z, c.z); u.c[3] = pair(c.w, c.w);
    u.s[0] = pair(-s.x, s.x); u.s[1] = pair(-s.y, s.y); u.s[2] = pair(-s.z, s.z); u.s[3] = pair(-s.w, s.w);
  } else {
    const int j = c0 < half ? c0 : c0 - half;
    const float sign = c0 < half ? -1.f : 1.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 c = __ldg(reinterpret_cast<const float4*>(row + j) + i), s = __ldg(reinterpret_cast<const float4*>(row + half + j) + i);
      u.c[2 * i] = pair(c.x, c.y); u.c[2 * i + 1] = pair(c.z, c.w);
      u.s[2 * i] = pair(sign * s.x, sign * s.y); u.s[2 * i + 1] = pair(sign * s.z, sign * s.w);
    }
  }
}

// The lane's eight channels of a row, turned (fp32).  All lanes of the warp take part; a row's lanes (LANES of them, this
// one is x) are neighbours.  Pairs that are rot/2 apart come from the lane that holds the other half: nothing is read
// a second time, so that a row may be written where it was read.
template <int LANES>
__device__ __forceinline__ void turn_row(const Table& t, const uint4& v, int x, const Turn& u, uint64_t (&y)[4]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  const int c0 = 8 * x, half = t.rot >> 1;
  uint32_t o[4];
  if (t.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __funnelshift_l(w[i], w[i], 16);
  } else {
    const int from = c0 >= t.rot ? x : c0 < half ? x + (half >> 3) : x - (half >> 3);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __shfl_sync(0xFFFFFFFFu, w[i], from, LANES);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = pair_of(w[i]);
  if (c0 < t.rot) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = add_pair(mul_pair(y[i], u.c[i]), mul_pair(pair_of(o[i]), u.s[i]));
  }
}
__device__ __forceinline__ uint4 pack8(const uint64_t (&y)[4]) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(first_of(y[i]), second_of(y[i]));
    r[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// Heads of one row by a warp: d / 8 lanes have one, the warp 256 / d of them side by side (a group), AHEAD groups on their way at a
// time; the row's cosines and sines stay with the lanes.  Where few rows are to be turned, several warps share a row's groups: this one
// has groups `first`, first + step, ...  turned: else copied as they are.
constexpr int AHEAD = 4;
template <int DH, bool TURNED>
__device__ __forceinline__ void row_heads(const Table& t, const Turn& u, int heads, int first, int step, const char* src, int64_t ss, char* dst, int64_t ds) {
  constexpr int LANES = DH / 8, GROUP = 32 / LANES;
  const int lane = threadIdx.x & 31, x = lane % LANES, sub = lane / LANES;
  src += (int64_t)(first * GROUP + sub) * ss + 16 * x;
  dst += (int64_t)(first * GROUP + sub) * ds + 16 * x;
  ss *= step * GROUP; ds *= step * GROUP;
  for (int h0 = first * GROUP; h0 < heads; h0 += AHEAD * step * GROUP) {
    uint4 v[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      v[j] = make_uint4(0, 0, 0, 0);
      if (h0 + j * step * GROUP + sub < heads) v[j] = *reinterpret_cast<const uint4*>(src);
      src += ss;
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (h0 + j * step * GROUP >= heads) break;     // (the same for the warp)
      if (TURNED) {
        uint64_t y[4];
        turn_row<LANES>(t, v[j], x, u, y);
        v[j] = pack8(y);
      }
      if (h0 + j * step * GROUP + sub < heads) *reinterpret_cast<uint4*>(dst) = v[j];
      dst += ds;
    }
  }
}
// Warps that share a row, a power of two up to `most`: until there are 32 for each SM.
static inline int warps_per_row(int64_t rows, int sm_count, int most) {
  int w = 1;
  while (w < most && rows * w < 32ll * sm_count) w *= 2;
  return w;
}

}  // namespace rope


// What both calls check of the rotation (rope.cu).
int check_rope(const space_ctx* ctx, const space_rope& r);
