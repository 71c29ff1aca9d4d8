// Penalties, biases and masks on a step's logits (space_logits_adjust), and the counts they go by (space_token_counts).
//
// Logits are read once and written once (in place: only what changes; what a mask leaves nothing of is not read). A thread has
// sixteen bytes of tokens of a sequence: which of them have a count, a bias or are candidates stays in a word while it
// goes through the sequence's rows, and arithmetic is done for those alone that the mask allows too, one after another: few
// are.  An odd vocabulary puts rows at any offset from the 16-byte grid: what is read is shifted into place, and what is written
// is shifted back with the next lane's, so that stores are whole 16-byte pieces, and a warp's two ends by its last lane.
//
// What bounds it: several rows off the grid about 200 instructions a 16-byte vector, most of them selects and shifts, which issue every other cycle:
// 16 x 36 x 50257 bf16 under masks 51 us (2.3 TB/s; the bytes: 18); as many rows ahead as registers hold, more thread blocks, tokens one by one where a
// mask leaves few, all measured the same within 10 %.  Single rows on the grid: 64 x 128256 fp32 with counts 22 us of 15 for the bytes.
// Counts of prompts of 2048 tokens, set anew: 9 us.
#include "common.cuh"

namespace {

constexpr int THREADS = 256;
constexpr int ROWS_BLOCKS = 5;                       // of the kernel for several rows, on an SM
constexpr int ROW_TOKENS = 8;                        // of a thread, where a sequence has one row (twice as many on the 16-byte grid)
constexpr int COUNT_MAX = (1 << 24) - 1;             // (an fp32 number exactly)

struct Params {
  int B, k, n, V, words;
  const void* logits; int64_t in_rs;
  void* out; int64_t out_rs;
  int in_place, per, groups, chunks;                 // rows of a group; row groups and token chunks of a sequence: thread blocks
  const int32_t* counts; const int32_t* cand;
  const float* rep; const float* pres; const float* freq;
  int n_bias, n_masks;
  const int32_t* bias_tok; const float* bias_val;
  const uint32_t* bits; const int32_t* mask_row;
  int32_t* status;
  unsigned long long* alive; int* arrived;           // per sequence: rows with a token left, thread blocks that have said so
};

// The elements [lo, hi) of a vector that holds those of `row` from x on.
template <typename T>
__device__ __forceinline__ void store_some(T* row, int64_t x, const uint4& v, int lo, int hi) {
  constexpr int N = 16 / (int)sizeof(T);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i < lo || i >= hi) continue;
    if (sizeof(T) == 4) reinterpret_cast<uint32_t*>(row)[x + i] = w[i % 4];
    else reinterpret_cast<uint16_t*>(row)[x + i] = (uint16_t)(w[(i >> 1) % 4] >> (16 * (i & 1)));
  }
}

// An element of a vector, wherever it lies, and the vector with another one there.
template <typename T> __device__ __forceinline__ float element(const uint4& v, int t);
template <> __device__ __forceinline__ float element<float>(const uint4& v, int t) {
  return __uint_as_float(t & 2 ? (t & 1 ? v.w : v.z) : (t & 1 ? v.y : v.x));
}
template <> __device__ __forceinline__ float element<__nv_bfloat16>(const uint4& v, int t) {
  const uint32_t w = t & 4 ? (t & 2 ? v.w : v.z) : (t & 2 ? v.y : v.x);
  return __uint_as_float(t & 1 ? w & 0xFFFF0000u : w << 16);
}
template <typename T>
__device__ __forceinline__ void set_element(uint4& v, int t, float z) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
  const uint32_t bits = sizeof(T) == 4 ? __float_as_uint(z) : (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(z)) << (16 * (t & 1));
  const uint32_t mask = sizeof(T) == 4 ? 0xFFFFFFFFu : 0xFFFFu << (16 * (t & 1));
  const int at = sizeof(T) == 4 ? t : t >> 1;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i == at) w[i] = (w[i] & ~mask) | bits;
  v = make_uint4(w[0], w[1], w[2], w[3]);
}
// Elements whose bit is 0 become -infinity.
template <typename T>
__device__ __forceinline__ void mask_out(uint4& v, uint32_t keep) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!((keep >> i) & 1u)) w[i] = 0xFF800000u;
  } else {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {                 // four bits to the tops of four bytes, each byte's top all over two bytes
      const uint32_t tops = ((keep >> (2 * i)) & 0xFu) * 0x10204080u & 0x80808080u;
      uint32_t m0, m1;
      asm("prmt.b32 %0, %1, 0, 0x9988;" : "=r"(m0) : "r"(tops));
      asm("prmt.b32 %0, %1, 0, 0xBBAA;" : "=r"(m1) : "r"(tops));
      w[i] = (w[i] & m0) | (0xFF80FF80u & ~m0);
      w[i + 1] = (w[i + 1] & m1) | (0xFF80FF80u & ~m1);
    }
  }
  v = make_uint4(w[0], w[1], w[2], w[3]);
}

// GRID: every row begins on the 16-byte grid.
// Sixteen bytes of a row, the first `there` elements from x on; nothing behind them is read.
template <bool GRID, typename T>
__device__ __forceinline__ Piece2 fetch(const T* row, int x, int there) {
  constexpr int N = 16 / (int)sizeof(T);
  if (there == N && !GRID) return load_pieces(row, x);
  if (there == N) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(row + x));
    return Piece2{v, v};
  }
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < there) {
      if (sizeof(T) == 4) w[e % 4] = reinterpret_cast<const uint32_t*>(row)[x + e];
      else w[(e >> 1) % 4] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[x + e] << (16 * (e & 1));
    }
  Piece2 r;
  r.a = r.b = make_uint4(w[0], w[1], w[2], w[3]);
  return r;
}
template <bool GRID, typename T>
__device__ __forceinline__ uint4 shifted(const Piece2& got, const T* row, int there) {
  return !GRID && there == 16 / (int)sizeof(T) ? shift_pieces(got, row) : got.a;
}
// Sixteen bytes: the first n of them to lo, the others to hi + n (lo and hi on the 16-byte grid).
template <typename T>
__device__ __forceinline__ void store_edges(char* lo, char* hi, const uint4& s, int n) {
  const uint32_t w[4] = {s.x, s.y, s.z, s.w};
  if (n & 8) *reinterpret_cast<uint2*>(lo) = make_uint2(w[0], w[1]);
  if (n & 4) *reinterpret_cast<uint32_t*>(lo + (n & 8)) = n & 8 ? w[2] : w[0];
  if (sizeof(T) == 2 && (n & 2)) {
    const uint32_t both = n & 8 ? (n & 4 ? w[3] : w[2]) : (n & 4 ? w[1] : w[0]);
    *reinterpret_cast<uint16_t*>(lo + (n & 12)) = (uint16_t)both;
    *reinterpret_cast<uint16_t*>(hi + n) = (uint16_t)(both >> 16);
  }
  const int at = (n + 3) & ~3;
  if (at & 4) *reinterpret_cast<uint32_t*>(hi + at) = at & 8 ? w[3] : w[1];
  if (at <= 8) *reinterpret_cast<uint2*>(hi + 8) = make_uint2(w[2], w[3]);
}
// The vectors of a warp (neighbouring lanes', the first `there` elements of each) to a row, by all of its lanes.
template <bool GRID, typename T>
__device__ __forceinline__ void store_vectors(T* dst, int x, const uint4& v, int there, int vocab) {
  constexpr int N = 16 / (int)sizeof(T);
  const int lane = threadIdx.x & 31;
  const uint32_t off = (uint32_t)((uintptr_t)dst & 15);
  if (x - lane * N + 32 * N > vocab) {               // the row's end
    store_some<T>(dst, x, v, 0, there);
  } else if (GRID || off == 0) {
    *reinterpret_cast<uint4*>(dst + x) = v;
  } else {
    // pieces of the grid: a vector's elements from 16 - off bytes on with the first ones of the next lane's; the last lane has the
    // warp's last elements and its first ones
    Piece2 two;
    const int next = (lane + 1) & 31;
    two.a = v;
    two.b.x = __shfl_sync(0xFFFFFFFFu, v.x, next); two.b.y = __shfl_sync(0xFFFFFFFFu, v.y, next);
    two.b.z = __shfl_sync(0xFFFFFFFFu, v.z, next); two.b.w = __shfl_sync(0xFFFFFFFFu, v.w, next);
    const uint4 piece = shift_pieces(two, reinterpret_cast<const T*>((uintptr_t)(16 - off)));
    char* at = reinterpret_cast<char*>(dst + x) + (16 - off);
    if (lane < 31) *reinterpret_cast<uint4*>(at) = piece;
    else store_edges<T>(at, at - 32 * 16, piece, (int)off);
  }
}

struct Penalty { float rep, pres, freq; };
__device__ __forceinline__ float penalized(float z, int count, int behind, const Penalty& f) {
  const int times = min(min(count & (SPACE_COUNT_PROMPT - 1), COUNT_MAX) + behind, COUNT_MAX);
  if (times > 0 || (count & SPACE_COUNT_PROMPT)) z = z > 0.f ? z / f.rep : z * f.rep;
  if (times > 0) z = __fsub_rn(__fsub_rn(z, __fmul_rn(f.freq, (float)times)), f.pres);
  return z;
}

// The biases of the tokens [t0, t0 + CHUNK): a bit per token that has some, and their sum (in the list's order, whoever adds it up).
// Starts with a barrier of the block (what the caller has written to shared memory is there), ends with one if a bit is set.
template <int CHUNK>
struct Biases {
  uint32_t some[CHUNK / 32], twice[CHUNK / 32];
  int again[SPACE_LOGITS_MAX_BIAS], n_again;         // entries of tokens that have several
  float sum[CHUNK];
  __device__ __forceinline__ bool collect(const Params& p, int b, int t0) {
    const int32_t* tok = p.bias_tok + (int64_t)b * p.n_bias;
    const float* val = p.bias_val + (int64_t)b * p.n_bias;
    auto mine = [&](int i) {
      const int t = __ldg(tok + i);
      return t >= t0 && t - t0 < CHUNK && t < p.V ? t - t0 : -1;
    };
    bool any = false;
    for (int i = threadIdx.x; i < p.n_bias; i += THREADS) any = any || mine(i) >= 0;
    for (int i = threadIdx.x; i < CHUNK / 32; i += THREADS) some[i] = twice[i] = 0;
    if (threadIdx.x == 0) n_again = 0;
    if (!__syncthreads_or(any)) return false;
    for (int i = threadIdx.x; i < p.n_bias; i += THREADS) {
      const int t = mine(i);
      if (t < 0) continue;
      const uint32_t bit = 1u << (t & 31);
      if (atomicOr(&some[t >> 5], bit) & bit) atomicOr(&twice[t >> 5], bit);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.n_bias; i += THREADS) {
      const int t = mine(i);
      if (t < 0) continue;
      if ((twice[t >> 5] >> (t & 31)) & 1u) again[atomicAdd(&n_again, 1)] = i;
      else sum[t] = __ldg(val + i);
    }
    __syncthreads();
    if (n_again == 0) return true;
    const int lane = threadIdx.x & 31;               // a warp for such an entry: the token's first one adds up all of them
    for (int e = threadIdx.x >> 5; e < n_again; e += THREADS / 32) {
      const int i = again[e], t = __ldg(tok + i);
      float total = 0.f;
      bool first = true;
      for (int j0 = 0; j0 < p.n_bias && first; j0 += 32) {
        const int j = j0 + lane;
        const bool same = j < p.n_bias && __ldg(tok + j) == t;
        const float v = same ? __ldg(val + j) : 0.f;
        uint32_t some_of = __ballot_sync(0xFFFFFFFFu, same);
        if (some_of && j0 + __ffs(some_of) - 1 < i) first = false;
        for (; some_of && first; some_of &= some_of - 1) {
          const int from = __ffs(some_of) - 1;
          const float add = __shfl_sync(0xFFFFFFFFu, v, from);
          total = j0 + from == i ? add : total + add;
        }
      }
      if (first && lane == 0) sum[t - t0] = total;
    }
    __syncthreads();
    return true;
  }
};

// What the masks leave of a sequence's rows, when all of its thread blocks have said so.
__device__ __forceinline__ void report(const Params& p, int b, int bad, unsigned long long alive, unsigned long long& all_of_block) {
  if (bad && p.status) atomicOr(p.status + b, bad);
  if (!p.status) return;
  if ((threadIdx.x & 31) == 0 && alive) atomicOr(&all_of_block, alive);
  __syncthreads();
  if (threadIdx.x != 0) return;
  if (all_of_block) atomicOr(p.alive + b, all_of_block);
  __threadfence();
  if (atomicAdd(p.arrived + b, 1) == p.chunks * p.groups - 1) {
    __threadfence();
    const unsigned long long all = p.n == 64 ? ~0ull : (1ull << p.n) - 1ull;
    if (atomicExch(p.alive + b, 0ull) != all) atomicOr(p.status + b, SPACE_ST_BAD_MASK);
    p.arrived[b] = 0;
  }
}

// Sequences of one row: a thread has UNITS vectors of it, all on their way at once with their counts.
template <typename T, bool GRID>
__global__ void __launch_bounds__(THREADS, 4) logits_row_kernel(const __grid_constant__ Params p) {
  constexpr int N = 16 / (int)sizeof(T), UNITS = (GRID ? 2 * ROW_TOKENS : ROW_TOKENS) / N, UNIT = THREADS * N, CHUNK = UNITS * UNIT;
  __shared__ Biases<CHUNK> biases;
  __shared__ unsigned long long alive_s;
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.z, chunk0 = blockIdx.x * CHUNK;
  const int x0 = chunk0 + (int)threadIdx.x * N;
  const T* row = reinterpret_cast<const T*>(p.logits) + (int64_t)b * p.in_rs;
  T* dst = reinterpret_cast<T*>(p.out) + (int64_t)b * p.out_rs;
  const float* counts = reinterpret_cast<const float*>(p.counts + (int64_t)b * p.V);
  auto there = [&](int u) { return min(max(p.V - (x0 + u * UNIT), 0), N); };
  int m = -1, bad = 0;
  if (p.bits) {
    m = p.mask_row[b];
    if (m >= p.n_masks) { bad = SPACE_ST_BAD_MASK; m = -1; }
  }
  Piece2 got[UNITS], cnt[UNITS][N / 4];
  uint32_t keep[UNITS];
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    const int x = x0 + u * UNIT, n = there(u);
    keep[u] = n == 0 ? 0u : m < 0 ? (1u << n) - 1u : (__ldg(p.bits + (int64_t)m * p.words + (x >> 5)) >> (x & 31)) & ((1u << n) - 1u);
    got[u].a = got[u].b = make_uint4(0, 0, 0, 0);
    if (keep[u]) got[u] = fetch<GRID>(row, x, n);          // (what the mask leaves nothing of is not read)
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      cnt[u][i].a = cnt[u][i].b = make_uint4(0, 0, 0, 0);
      if (p.counts && keep[u] && n > 4 * i) cnt[u][i] = fetch<GRID>(counts, x + 4 * i, min(n - 4 * i, 4));
    }
  }
  const Penalty f{p.rep ? p.rep[b] : 1.f, p.pres ? p.pres[b] : 0.f, p.freq ? p.freq[b] : 0.f};
  if (threadIdx.x == 0) alive_s = 0;
  const bool biased = p.n_bias && biases.collect(p, b, chunk0);
  if (!p.n_bias && p.bits) __syncthreads();
  unsigned long long alive = 0;
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    const int x = x0 + u * UNIT, n = there(u);
    if (chunk0 + u * UNIT >= p.V) break;             // (the same for the whole block)
    uint4 v = shifted<GRID>(got[u], row, n), c[N / 4];
    uint32_t hit = 0;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      c[i] = shifted<GRID>(cnt[u][i], counts, min(max(n - 4 * i, 0), 4));
      hit |= ((c[i].x ? 1u : 0u) | (c[i].y ? 2u : 0u) | (c[i].z ? 4u : 0u) | (c[i].w ? 8u : 0u)) << (4 * i);
    }
    const uint32_t bias = biased ? biases.some[(x - chunk0) >> 5] >> (x & 31) : 0u;
    if (p.bits && __any_sync(0xFFFFFFFFu, keep[u] != 0)) alive = 1;
    uint32_t act = (hit | bias) & keep[u];
    const bool touch = !p.in_place || __any_sync(0xFFFFFFFFu, act || (n && keep[u] != (1u << n) - 1u));
    for (; act; act &= act - 1) {
      const int t = __ffs(act) - 1;
      const int count = __float_as_int(element<float>(N == 4 || t < 4 ? c[0] : c[N / 4 - 1], t & 3));
      float z = penalized(element<T>(v, t), count, 0, f);
      if ((bias >> t) & 1u) z += biases.sum[x - chunk0 + t];
      set_element<T>(v, t, z);
    }
    if (!touch) continue;
    if (p.bits) mask_out<T>(v, keep[u]);
    store_vectors<GRID>(dst, x, v, n, p.V);
  }
  if (p.bits) report(p, b, bad, alive, alive_s);
}

// Sequences of n rows: a thread has one vector of tokens, whose counts, biases and candidates stay with it from row to row.
template <typename T, bool GRID>
__global__ void __launch_bounds__(THREADS, ROWS_BLOCKS) logits_rows_kernel(const __grid_constant__ Params p) {
  constexpr int N = 16 / (int)sizeof(T), CHUNK = THREADS * N;
  __shared__ Biases<CHUNK> biases;
  __shared__ int32_t mask_s[SPACE_MAX_ROWS];
  __shared__ unsigned long long alive_s;
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.z, chunk0 = blockIdx.x * CHUNK;
  const int x = chunk0 + (int)threadIdx.x * N;
  const int there = min(max(p.V - x, 0), N);         // tokens of this thread
  const uint32_t valid = (1u << there) - 1u;
  const int i0 = blockIdx.y * p.per, i1 = min(i0 + p.per, p.n);
  const T* in0 = reinterpret_cast<const T*>(p.logits) + ((int64_t)b * p.n + i0) * p.in_rs;
  T* out0 = reinterpret_cast<T*>(p.out) + ((int64_t)b * p.n + i0) * p.out_rs;
  const float* counts = reinterpret_cast<const float*>(p.counts + (int64_t)b * p.V);
  Piece2 cnt[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    cnt[i].a = cnt[i].b = make_uint4(0, 0, 0, 0);
    if (p.counts && there > 4 * i) cnt[i] = fetch<GRID>(counts, x + 4 * i, min(there - 4 * i, 4));
  }
  unsigned long long is_cand = 0;                    // bit 8 t + j: token x + t is candidate j + 1
  if (p.cand)
    for (int j = 0; j < p.k; ++j) {
      const int t = __ldg(p.cand + b * p.k + j) - x;
      if (t >= 0 && t < there) is_cand |= 1ull << (8 * t + j);
    }
  const Penalty f{p.rep ? p.rep[b] : 1.f, p.pres ? p.pres[b] : 0.f, p.freq ? p.freq[b] : 0.f};
  int bad = 0;
  if (p.bits && i0 + (int)threadIdx.x < i1) {
    const int m = p.mask_row[(int64_t)b * p.n + i0 + threadIdx.x];
    if (m >= p.n_masks) bad = SPACE_ST_BAD_MASK;
    mask_s[threadIdx.x] = m < p.n_masks ? m : -1;
  }
  if (threadIdx.x == 0) alive_s = 0;
  const bool biased = p.n_bias && biases.collect(p, b, chunk0);
  if (!p.n_bias && p.bits) __syncthreads();
  const uint32_t bias = biased ? biases.some[(x - chunk0) >> 5] >> (x & 31) : 0u;
  uint32_t hit = bias;                               // tokens with a bias, a count or a place among the candidates
  uint4 c[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    c[i] = shifted<GRID>(cnt[i], counts, min(max(there - 4 * i, 0), 4));
    hit |= ((c[i].x ? 1u : 0u) | (c[i].y ? 2u : 0u) | (c[i].z ? 4u : 0u) | (c[i].w ? 8u : 0u)) << (4 * i);
  }
#pragma unroll
  for (int t = 0; t < N; ++t) hit |= (is_cand >> (8 * t)) & 0xFFu ? 1u << t : 0u;

  unsigned long long alive = 0;
#pragma unroll 1
  for (int i = i0; i < i1; ++i, in0 += p.in_rs, out0 += p.out_rs) {
    const int m = p.bits ? mask_s[i - i0] : -1;
    const uint32_t keep = m < 0 || !there ? valid : (__ldg(p.bits + (int64_t)m * p.words + (x >> 5)) >> (x & 31)) & valid;
    if (p.bits && __any_sync(0xFFFFFFFFu, keep != 0)) alive |= 1ull << i;
    uint32_t act = hit & keep;
    // (what stays where it is is not read, nor what the mask leaves nothing of)
    if (p.in_place && !__any_sync(0xFFFFFFFFu, act || keep != valid)) continue;
    Piece2 got;
    got.a = got.b = make_uint4(0, 0, 0, 0);
    if (keep) got = fetch<GRID>(in0, x, there);
    uint4 v = shifted<GRID>(got, in0, there);
    for (; act; act &= act - 1) {
      const uint32_t seen = (1u << (i / (p.k + 1))) - 1u;      // candidates that this row has behind it
      const int t = __ffs(act) - 1;
      const int count = __float_as_int(element<float>(N == 4 || t < 4 ? c[0] : c[N / 4 - 1], t & 3));
      float z = penalized(element<T>(v, t), count, __popc((uint32_t)(is_cand >> (8 * t)) & seen & 0x7Fu), f);
      if ((bias >> t) & 1u) z += biases.sum[x - chunk0 + t];
      set_element<T>(v, t, z);
    }
    if (p.bits) mask_out<T>(v, keep);
    store_vectors<GRID>(out0, x, v, there, p.V);
  }
  if (p.bits) report(p, b, bad, alive, alive_s);
}

// ---- counts
// A few tokens are added where they are.  More of them, or counts that start anew: a thread block per 8192 tokens of the
// vocabulary goes through the list and counts its own in shared memory.
constexpr int COUNT_CHUNK = 8192, FEW_TOKENS = 256;

struct CountParams {
  int B, V, n, prompt, reset;
  const int32_t* tokens; int64_t stride;
  const int32_t* n_tokens;
  int32_t* counts;
};

__global__ void __launch_bounds__(FEW_TOKENS) count_few_kernel(const CountParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.x, n = p.n_tokens ? min(p.n_tokens[b], p.n) : p.n;
  if ((int)threadIdx.x >= n) return;
  const int t = p.tokens[(int64_t)b * p.stride + threadIdx.x];
  if (t < 0 || t >= p.V) return;
  int32_t* at = p.counts + (int64_t)b * p.V + t;
  if (p.prompt) atomicOr(at, SPACE_COUNT_PROMPT);
  else atomicAdd(at, 1);
}

__global__ void __launch_bounds__(THREADS) count_chunk_kernel(const CountParams p) {
  __shared__ __align__(16) int hist[COUNT_CHUNK];
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.y, t0 = blockIdx.x * COUNT_CHUNK, len = min(COUNT_CHUNK, p.V - t0);
  constexpr int FIRST = 8;
  const int32_t* tokens = p.tokens + (int64_t)b * p.stride;
  int first[FIRST];                                  // tokens that are on their way while the counts are cleared
#pragma unroll
  for (int u = 0; u < FIRST; ++u) first[u] = u * THREADS + (int)threadIdx.x < p.n ? __ldg(tokens + u * THREADS + threadIdx.x) : -1;
  const int n = p.n_tokens ? min(p.n_tokens[b], p.n) : p.n;
#pragma unroll
  for (int i = 0; i < COUNT_CHUNK / (4 * THREADS); ++i) reinterpret_cast<int4*>(hist)[i * THREADS + threadIdx.x] = make_int4(0, 0, 0, 0);
  __syncthreads();
  auto add = [&](int t) {
    if (t < t0 || t - t0 >= len) return;             // (below 0 or past the vocabulary: in no block's part)
    if (p.prompt) hist[t - t0] = SPACE_COUNT_PROMPT;
    else atomicAdd(&hist[t - t0], 1);
  };
#pragma unroll
  for (int u = 0; u < FIRST; ++u)
    if (u * THREADS + (int)threadIdx.x < n) add(first[u]);
#pragma unroll 4
  for (int i = FIRST * THREADS + threadIdx.x; i < n; i += THREADS) add(__ldg(tokens + i));
  __syncthreads();
  int32_t* out = p.counts + (int64_t)b * p.V + t0;
  if (p.reset && ((uintptr_t)out & 15) == 0) {
    for (int i = 4 * threadIdx.x; i + 4 <= len; i += 4 * THREADS) *reinterpret_cast<int4*>(out + i) = *reinterpret_cast<const int4*>(hist + i);
    for (int i = len / 4 * 4 + threadIdx.x; i < len; i += THREADS) out[i] = hist[i];
    return;
  }
  for (int i = threadIdx.x; i < len; i += THREADS) {
    const int h = hist[i];
    if (p.reset) out[i] = h;
    else if (h) out[i] = p.prompt ? out[i] | h : out[i] + h;
  }
}

}  // namespace

extern "C" {

int space_logits_adjust(space_ctx* ctx, const space_logits_args* a, void* stream) {
  if (!ctx || !a) return SPACE_E_INVALID_ARG;
  if (a->batch < 0 || a->batch > ctx->cfg.max_batch || a->k > ctx->cfg.k_max) return SPACE_E_WORKSPACE;
  if (a->vocab < 1 || a->vocab > ctx->cfg.vocab) return SPACE_E_WORKSPACE;
  if (a->k < 0 || (a->dtype != SPACE_DTYPE_F32 && a->dtype != SPACE_DTYPE_BF16)) return SPACE_E_INVALID_ARG;
  if (a->batch == 0) return SPACE_OK;
  if (!a->logits || !a->out || a->logits_row_stride < a->vocab || a->out_row_stride < a->vocab) return SPACE_E_INVALID_ARG;
  if (a->out == a->logits && a->out_row_stride != a->logits_row_stride) return SPACE_E_INVALID_ARG;
  if (a->n_bias < 0 || a->n_bias > SPACE_LOGITS_MAX_BIAS || (a->n_bias > 0 && (!a->bias_tok || !a->bias_val))) return SPACE_E_INVALID_ARG;
  if ((a->mask_bits == nullptr) != (a->mask_row == nullptr) || (a->mask_bits && a->n_masks < 1)) return SPACE_E_INVALID_ARG;
  const int esz = a->dtype == SPACE_DTYPE_F32 ? 4 : 2;
  if ((uintptr_t)a->logits % esz || (uintptr_t)a->out % esz) return SPACE_E_ALIGNMENT;
  if (cudaSetDevice(ctx->cfg.device) != cudaSuccess) return SPACE_E_CUDA;
  Params p;
  memset(&p, 0, sizeof(p));
  p.B = a->batch; p.k = a->k; p.n = (a->k + 1) * (a->k + 1); p.V = a->vocab; p.words = (a->vocab + 31) / 32;
  p.logits = a->logits; p.in_rs = a->logits_row_stride; p.out = a->out; p.out_rs = a->out_row_stride;
  p.in_place = a->out == a->logits;
  p.counts = a->counts; p.cand = a->k ? a->cand : nullptr;
  p.rep = a->repetition; p.pres = a->presence; p.freq = a->frequency;
  p.n_bias = a->n_bias; p.bias_tok = a->bias_tok; p.bias_val = a->bias_val;
  p.n_masks = a->n_masks; p.bits = a->mask_bits; p.mask_row = a->mask_row; p.status = a->status;
  p.alive = ctx->logits_alive; p.arrived = ctx->logits_arrived;
  const int64_t in_b = p.in_rs * esz, out_b = p.out_rs * esz;
  const bool grid = !(((uintptr_t)p.logits | (uintptr_t)p.out | (uintptr_t)p.counts | (uintptr_t)in_b | (uintptr_t)out_b) & 15) && (!p.counts || p.V % 4 == 0);
  const int chunk = THREADS * (p.n > 1 ? 16 / esz : grid ? 2 * ROW_TOKENS : ROW_TOKENS);
  p.chunks = (int)(((int64_t)p.V + chunk - 1) / chunk);
  // Rows are shared out so that the thread blocks, ROWS_BLOCKS to an SM at once, end together: what a block does before its first row is
  // worth about three of them.
  int64_t least = INT64_MAX;
  for (int per = 1; per <= p.n; ++per) {
    const int groups = (p.n + per - 1) / per;
    const int64_t slots = (int64_t)ROWS_BLOCKS * ctx->sm_count, turns = ((int64_t)p.chunks * p.B * groups + slots - 1) / slots;
    if (turns * (per + 3) < least) { least = turns * (per + 3); p.groups = groups; p.per = per; }
  }
  void (*kernel)(Params);
  if (p.n == 1)
    kernel = esz == 4 ? (grid ? logits_row_kernel<float, true> : logits_row_kernel<float, false>)
                      : (grid ? logits_row_kernel<__nv_bfloat16, true> : logits_row_kernel<__nv_bfloat16, false>);
  else
    kernel = esz == 4 ? (grid ? logits_rows_kernel<float, true> : logits_rows_kernel<float, false>)
                      : (grid ? logits_rows_kernel<__nv_bfloat16, true> : logits_rows_kernel<__nv_bfloat16, false>);
  ctx->launches += 1;
  return cuda_ok(launch_pdl(kernel, dim3(p.chunks, p.groups, p.B), dim3(THREADS), 0, (cudaStream_t)stream, p));
}

int space_token_counts(space_ctx* ctx, const space_counts_args* a, void* stream) {
  if (!ctx || !a) return SPACE_E_INVALID_ARG;
  if (a->batch < 0 || a->batch > ctx->cfg.max_batch) return SPACE_E_WORKSPACE;
  if (a->vocab < 1 || a->vocab > ctx->cfg.vocab) return SPACE_E_WORKSPACE;
  if (a->n < 0) return SPACE_E_INVALID_ARG;
  if (a->batch == 0 || (a->n == 0 && !a->reset)) return SPACE_OK;
  if (!a->counts || (a->n > 0 && !a->tokens)) return SPACE_E_INVALID_ARG;
  if (cudaSetDevice(ctx->cfg.device) != cudaSuccess) return SPACE_E_CUDA;
  const CountParams p{a->batch, a->vocab, a->n, a->prompt != 0, a->reset != 0, a->tokens, a->tokens_stride_b, a->n_tokens, a->counts};
  ctx->launches += 1;
  if (!p.reset && p.n <= FEW_TOKENS)
    return cuda_ok(launch_pdl(count_few_kernel, dim3(p.B), dim3((p.n + 31) / 32 * 32), 0, (cudaStream_t)stream, p));
  return cuda_ok(launch_pdl(count_chunk_kernel, dim3((unsigned)(((int64_t)p.V + COUNT_CHUNK - 1) / COUNT_CHUNK), p.B), dim3(THREADS), 0, (cudaStream_t)stream, p));
}

}  // extern "C"
