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
  uint32_t r = w;
#pragma unroll
  for (int s = 0; s < 32; s += 16) {
    const uint32_t x = (w >> s) & 0x7FFFu;
    if (x > 0x7F80u) r &= ~(0xFFFFu << s);
    else if (x == 0x7F80u) r -= 1u << s;
  }
  return r;
}
__device__ __forceinline__ bool any_nonfinite(const uint4& v) {
  const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
  return (m & 0xFFFFu) >= 0x7F80u || (m >> 16) >= 0x7F80u;
}

}  // namespace kvq
