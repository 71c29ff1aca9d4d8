// The 4-bit cache's format (space.h, space_kvq_cache) as the kernels address it.
#pragma once
#include "common.cuh"

namespace kvq {

constexpr int BLOCK_ROWS = 32;                       // rows that are laid out together
constexpr int PAGE_BLOCKS = SPACE_PAGE_SIZE / BLOCK_ROWS;
// Bytes inside a block of 32 rows.
template <int DH>
struct Fmt {
  static constexpr int CODES = BLOCK_ROWS * DH / 2;  // K codes, then as many V codes
  static constexpr int K_PAR = 2 * CODES;            // [32] {bf16 step, bf16 lo}
  static constexpr int V_PAR = K_PAR + 4 * BLOCK_ROWS;
  static constexpr int BLOCK = V_PAR + 4 * BLOCK_ROWS;
  static constexpr int HEAD = PAGE_BLOCKS * BLOCK;   // a page of one kv head
  static_assert(BLOCK % 128 == 0, "every block starts on a 16-byte boundary");
};

struct Cache {
  char* pool;
  int64_t page_stride, head_stride;
  const int32_t* page_table;
  int pages_per_seq, n_pages;
};
static inline Cache cache_of(const space_kvq_cache& c) {
  return Cache{(char*)c.pool, c.page_stride, c.head_stride, c.page_table, c.pages_per_seq, c.n_pages};
}

// The 32-row block that holds row s (s >= 0) of sequence b, kv head h; nullptr for a page outside the pool.
template <int DH>
__device__ __forceinline__ char* block_at(const Cache& c, int b, int h, int s) {
  const int t = s / SPACE_PAGE_SIZE;
  const int pg = t < c.pages_per_seq ? c.page_table[(int64_t)b * c.pages_per_seq + t] : -1;
  if (pg < 0 || pg >= c.n_pages) return nullptr;
  return c.pool + (int64_t)pg * c.page_stride + (int64_t)h * c.head_stride + (s % SPACE_PAGE_SIZE) / BLOCK_ROWS * Fmt<DH>::BLOCK;
}

// Where row i of a block has its two bytes of channels {8q + n of 32w ..}: 512w + 64n + 16t + 8a + 4e + 2h
__device__ __forceinline__ int v_row_at(int i) {
  return 16 * ((i >> 1) & 3) + 8 * (i >> 4) + 4 * ((i >> 3) & 1) + 2 * (i & 1);
}

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// A pair of bf16 with a NaN made 0 and an infinity the largest finite value.
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
  const uint32_t mag = w & 0x7FFF7FFFu, nan = __vcmpgtu2(mag, 0x7F807F80u);
  return (__vminu2(mag, 0x7F7F7F7Fu) | (w & 0x80008000u)) & ~nan;
}
__device__ __forceinline__ uint32_t max_bits(const uint4& v) {     // of eight magnitudes
  const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
  return max(m & 0xFFFFu, m >> 16);
}
__device__ __forceinline__ bool any_nonfinite(const uint4& v) { return max_bits(v) >= 0x7F80u; }
__device__ __forceinline__ void make_finite(uint4& v) {
  if (max_bits(v) >= 0x7F80u) v = make_uint4(finite_pair(v.x), finite_pair(v.y), finite_pair(v.z), finite_pair(v.w));
}
__device__ __forceinline__ uint4 scale_bf16(const uint4& v, float f) {         // f a power of two
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 y = __floats2bfloat162_rn(bf_lo(w[i]) * f, bf_hi(w[i]) * f);
    r[i] = *reinterpret_cast<const uint32_t*>(&y);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}
// The same, with the largest magnitude's bits.
__device__ __forceinline__ uint32_t top_bits(uint4& v) {
  const uint32_t m = max_bits(v);
  if (m < 0x7F80u) return m;
  v = make_uint4(finite_pair(v.x), finite_pair(v.y), finite_pair(v.z), finite_pair(v.w));
  return max_bits(v);
}

}  // namespace kvq
