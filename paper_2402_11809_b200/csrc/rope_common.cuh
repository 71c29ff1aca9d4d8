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

// Cosines and sines of a lane's eight channels 8x .. 8x + 7 (pairs of neighbours: of its four pairs).
struct Turn { float c[8], s[8]; };
__device__ __forceinline__ void load4(float* d, const float* src) {
  const float4 v = __ldg(reinterpret_cast<const float4*>(src));
  d[0] = v.x; d[1] = v.y; d[2] = v.z; d[3] = v.w;
}
__device__ __forceinline__ void load_turn(const Table& t, const float* row, int x, Turn& u) {
  const int half = t.rot >> 1, c0 = 8 * x;
  if (c0 >= t.rot) return;
  if (t.interleaved) {
    load4(u.c, row + 4 * x);
    load4(u.s, row + half + 4 * x);
  } else {
    const int j = c0 < half ? c0 : c0 - half;
    load4(u.c, row + j); load4(u.c + 4, row + j + 4);
    load4(u.s, row + half + j); load4(u.s + 4, row + half + j + 4);
  }
}

// The lane's eight channels of a row, turned (fp32).  All lanes of the warp take part; a row's lanes (LANES of them, this
// one is x) are neighbours.  Pairs that are rot/2 apart come from the lane that holds the other half: nothing is read
// a second time, so that a row may be written where it was read.
template <int LANES>
__device__ __forceinline__ void turn_row(const Table& t, const uint4& v, int x, const Turn& u, float (&y)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  const int c0 = 8 * x, half = t.rot >> 1;
#pragma unroll
  for (int i = 0; i < 4; ++i) { y[2 * i] = lo_f(w[i]); y[2 * i + 1] = hi_f(w[i]); }
  if (t.interleaved) {
    if (c0 >= t.rot) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = y[2 * i], b = y[2 * i + 1];
      y[2 * i] = __fsub_rn(__fmul_rn(a, u.c[i]), __fmul_rn(b, u.s[i]));
      y[2 * i + 1] = __fadd_rn(__fmul_rn(b, u.c[i]), __fmul_rn(a, u.s[i]));
    }
    return;
  }
  const bool first = c0 < half;
  const int from = c0 >= t.rot ? x : first ? x + (half >> 3) : x - (half >> 3);
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = __shfl_sync(0xFFFFFFFFu, w[i], from, LANES);
  if (c0 >= t.rot) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float other = __fmul_rn((i & 1) ? hi_f(o[i >> 1]) : lo_f(o[i >> 1]), u.s[i]), mine = __fmul_rn(y[i], u.c[i]);
    y[i] = first ? __fsub_rn(mine, other) : __fadd_rn(mine, other);
  }
}
__device__ __forceinline__ uint4 pack8(const float (&y)[8]) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
    r[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// Heads of one row: d / 8 lanes have a head, a thread HEADS of them at a time, whose loads are all on their way before the
// first is used; the row's cosines and sines serve them all.  src(g) and dst(g): where head g is and goes (nullptr: nowhere); heads
// from `plain` on are copied as they are.  By whole warps.
constexpr int HEADS = 4;
template <int DH, int THREADS, class Src, class Dst>
__device__ __forceinline__ void turn_heads(const Table& t, const float* row, int n_heads, int plain, Src src, Dst dst) {
  constexpr int LANES = DH / 8, SLOTS = THREADS / LANES;
  const int x = threadIdx.x % LANES, g0 = threadIdx.x / LANES;
  Turn u;
  load_turn(t, row, x, u);
  for (int g = g0; g - g0 < n_heads; g += HEADS * SLOTS) {     // (the same number of times for a warp)
    uint4 v[HEADS];
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
      const int h = g + j * SLOTS;
      v[j] = h < n_heads ? *(reinterpret_cast<const uint4*>(src(h)) + x) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
      const int h = g + j * SLOTS;
      if (g - g0 + j * SLOTS >= n_heads) break;
      float y[8];
      turn_row<LANES>(t, v[j], x, u, y);
      char* to = h < n_heads ? dst(h) : nullptr;
      if (to) *(reinterpret_cast<uint4*>(to) + x) = h < plain ? pack8(y) : v[j];
    }
  }
}

}  // namespace rope


// What both calls check of the rotation (rope.cu).
int check_rope(const space_ctx* ctx, const space_rope& r);
