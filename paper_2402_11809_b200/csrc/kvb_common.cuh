// The 8-bit cache's format (space.h, space_kvb_cache) as the kernels address it.
#pragma once
#include "kvq_common.cuh"
#include <cuda_fp16.h>

namespace kvb {

constexpr int BLOCK_ROWS = 32;                       // rows that share a power of two
constexpr int PAGE_BLOCKS = SPACE_PAGE_SIZE / BLOCK_ROWS;
constexpr int MIN_EXP = -100;                        // of a scale
template <int DH>
struct Fmt {
  static constexpr int CODES = SPACE_PAGE_SIZE * DH; // K codes, then as many V codes
  static constexpr int SCALES = 2 * CODES;
  static constexpr int HEAD = SCALES + 8 * PAGE_BLOCKS;
  static constexpr int K_COLS = 16 * SPACE_PAGE_SIZE;        // bytes of sixteen K channels of a page
  static constexpr int V_ROWS = 16 * DH;                     // bytes of sixteen V rows of a page
};
using kvq::Cache;
using kvq::cache_of;

// The page of kv head h that holds row s (s >= 0) of sequence b; nullptr for one outside the pool.
__device__ __forceinline__ char* page_at(const Cache& c, int b, int h, int s) {
  const int t = s / SPACE_PAGE_SIZE;
  const int pg = t < c.pages_per_seq ? c.page_table[(int64_t)b * c.pages_per_seq + t] : -1;
  if (pg < 0 || pg >= c.n_pages) return nullptr;
  return c.pool + (int64_t)pg * c.page_stride + (int64_t)h * c.head_stride;
}

__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }     // -126 <= e <= 127
// The least e, MIN_EXP at least, with top <= 448 2^e = 1.75 2^(e + 8); top finite, not negative.
__device__ __forceinline__ int scale_exp(float top) {
  const uint32_t w = __float_as_uint(top);
  return max((int)(w >> 23) - 127 - 8 + ((w & 0x7FFFFFu) > 0x600000u ? 1 : 0), MIN_EXP);
}
// Two numbers as e4m3 (to nearest even, held to +-448), the first in the low byte.
__device__ __forceinline__ uint32_t codes2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) { return codes2(a, b) | codes2(c, d) << 16; }
// Two codes as a pair of f16 (exact).
__device__ __forceinline__ uint32_t halves2(uint32_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes));
  return r;
}

}  // namespace kvb
