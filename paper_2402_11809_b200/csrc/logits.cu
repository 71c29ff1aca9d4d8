// Penalties, biases and masks on a step's logits (space_logits_adjust), and the counts they go by (space_token_counts).
//
// Logits are read once and written once (in place: only what changes). A thread has sixteen bytes of tokens of a sequence: their
// counts, biases and the candidates among them stay in registers while it goes through the sequence's rows, which
// differ in how many candidates count and in the mask.  Four rows are on their way at a time.  An odd vocabulary puts rows at any
// offset from the 16-byte grid: what is read is shifted into place, and what is written is put together from
// a lane and its neighbour, so that stores are whole 16-byte pieces but for the ends of a warp's part.
#include "common.cuh"

namespace {

constexpr int THREADS = 256, ROWS_AHEAD = 4;
constexpr int COUNT_MAX = (1 << 24) - 1;             // (an fp32 number exactly)

struct Params {
  int B, k, n, V, words;
  const void* logits; int64_t in_rs;
  void* out; int64_t out_rs;
  int in_place, groups, chunks;                      // row groups and token chunks of a sequence: thread blocks
  const int32_t* counts; const int32_t* cand;
  const float* rep; const float* pres; const float* freq;
  int n_bias, n_masks;
  const int32_t* bias_tok; const float* bias_val;
  const uint32_t* bits; const int32_t* mask_row;
  int32_t* status;
  unsigned long long* alive; int* arrived;           // per sequence: rows with a token left, thread blocks that have said so
};

template <typename T> __device__ __forceinline__ void unpack(const uint4& v, float* z);
template <> __device__ __forceinline__ void unpack<float>(const uint4& v, float* z) {
  z[0] = __uint_as_float(v.x); z[1] = __uint_as_float(v.y); z[2] = __uint_as_float(v.z); z[3] = __uint_as_float(v.w);
}
template <> __device__ __forceinline__ void unpack<__nv_bfloat16>(const uint4& v, float* z) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { z[2 * i] = __uint_as_float(w[i] << 16); z[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
template <typename T> __device__ __forceinline__ uint4 pack(const float* z);
template <> __device__ __forceinline__ uint4 pack<float>(const float* z) {
  return make_uint4(__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3]));
}
template <> __device__ __forceinline__ uint4 pack<__nv_bfloat16>(const float* z) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(z[2 * i], z[2 * i + 1]);
    r[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}
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

template <typename T>
__global__ void __launch_bounds__(THREADS) logits_adjust_kernel(const __grid_constant__ Params p) {
  constexpr int N = 16 / (int)sizeof(T), CHUNK = THREADS * N;
  constexpr uint32_t ALL = (1u << N) - 1u;
  __shared__ float bias_s[CHUNK];
  __shared__ int32_t tok_s[SPACE_LOGITS_MAX_BIAS];
  __shared__ float val_s[SPACE_LOGITS_MAX_BIAS];
  __shared__ unsigned long long alive_s;
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.z, chunk0 = blockIdx.x * CHUNK, lane = threadIdx.x & 31;
  const int x0 = chunk0 + (int)threadIdx.x * N;
  const int there = min(max(p.V - x0, 0), N);        // tokens of this thread
  float bias[N];
#pragma unroll
  for (int i = 0; i < N; ++i) bias[i] = 0.f;
  if (threadIdx.x == 0) alive_s = 0;
  if (p.n_bias) {
    for (int i = threadIdx.x; i < CHUNK; i += THREADS) bias_s[i] = 0.f;
    for (int i = threadIdx.x; i < p.n_bias; i += THREADS) {
      tok_s[i] = p.bias_tok[(int64_t)b * p.n_bias + i];
      val_s[i] = p.bias_val[(int64_t)b * p.n_bias + i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.n_bias; i += THREADS) {
      const int t = tok_s[i];
      if (t < chunk0 || t >= chunk0 + CHUNK || t >= p.V) continue;
      bool first = true;                             // the first entry of a token adds up all of them
      for (int j = 0; j < i && first; ++j) first = tok_s[j] != t;
      if (!first) continue;
      float sum = val_s[i];
      for (int j = i + 1; j < p.n_bias; ++j)
        if (tok_s[j] == t) sum += val_s[j];
      bias_s[t - chunk0] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) bias[i] = bias_s[threadIdx.x * N + i];
  } else {
    __syncthreads();
  }
  // counts, and which candidates a token is: bit j of nibble pair i: token x0 + i is candidate j + 1
  int count[N];
  unsigned long long is_cand = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) count[i] = 0;
  if (p.counts) {
    const int32_t* row = p.counts + (int64_t)b * p.V + x0;
    if (there == N && ((uintptr_t)row & 15) == 0) {
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        const int4 c = __ldg(reinterpret_cast<const int4*>(row) + i);
        count[4 * i] = c.x; count[4 * i + 1] = c.y; count[4 * i + 2] = c.z; count[4 * i + 3] = c.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) if (i < there) count[i] = __ldg(row + i);
    }
  }
  if (p.cand) {
    for (int j = 0; j < p.k; ++j) {
      const int t = p.cand[b * p.k + j] - x0;
      if (t >= 0 && t < there) is_cand |= 1ull << (8 * t + j);
    }
  }
  bool some = is_cand != 0;
#pragma unroll
  for (int i = 0; i < N; ++i) some = some || count[i] != 0 || bias[i] != 0.f;      // (NaN differs from 0)
  const float rep = p.rep ? p.rep[b] : 1.f, pres = p.pres ? p.pres[b] : 0.f, freq = p.freq ? p.freq[b] : 0.f;

  const int per = (p.n + p.groups - 1) / p.groups, i0 = blockIdx.y * per, i1 = min(i0 + per, p.n);
  const uint32_t valid = there == N ? ALL : (1u << there) - 1u;
  unsigned long long alive = 0;
  int bad = 0;
  for (int r0 = i0; r0 < i1; r0 += ROWS_AHEAD) {
    Piece2 got[ROWS_AHEAD];
    uint32_t keep[ROWS_AHEAD];
#pragma unroll
    for (int u = 0; u < ROWS_AHEAD; ++u) {
      const int i = r0 + u;
      keep[u] = valid;
      got[u].a = got[u].b = make_uint4(0, 0, 0, 0);
      if (i >= i1) continue;
      if (p.bits) {
        const int m = p.mask_row[(int64_t)b * p.n + i];
        if (m >= p.n_masks) bad = SPACE_ST_BAD_MASK;
        else if (m >= 0) keep[u] = there ? (__ldg(p.bits + (int64_t)m * p.words + (x0 >> 5)) >> (x0 & 31)) & valid : 0u;
      }
      const T* row = reinterpret_cast<const T*>(p.logits) + ((int64_t)b * p.n + i) * p.in_rs;
      const bool shifted = ((uintptr_t)row & 15) != 0;
      if (there && (keep[u] || !valid) && (!p.in_place || shifted || some || keep[u] != valid)) {
        if (there == N) got[u] = load_pieces(row, x0);
        else {                                       // the row's end: nothing behind it is read
          uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (e < there) {
              if (sizeof(T) == 4) w[e % 4] = reinterpret_cast<const uint32_t*>(row)[x0 + e];
              else w[(e >> 1) % 4] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[x0 + e] << (16 * (e & 1));
            }
          got[u].a = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < ROWS_AHEAD; ++u) {
      const int i = r0 + u;
      if (i >= i1) break;                            // (the same for the whole block)
      const T* row = reinterpret_cast<const T*>(p.logits) + ((int64_t)b * p.n + i) * p.in_rs;
      uint4 v = there == N ? shift_pieces(got[u], row) : got[u].a;
      if (__any_sync(0xFFFFFFFFu, keep[u] != 0)) alive |= 1ull << i;
      const bool touched = some || keep[u] != valid;
      if (touched) {
        float z[N];
        unpack<T>(v, z);
        const uint32_t behind = (1u << (i / (p.k + 1))) - 1u;                  // candidates that this row has seen
#pragma unroll
        for (int t = 0; t < N; ++t) {
          const int c = count[t], times = min((c & (SPACE_COUNT_PROMPT - 1)), COUNT_MAX) + __popc((uint32_t)(is_cand >> (8 * t)) & behind & 0x7Fu);
          if (times > 0 || (c & SPACE_COUNT_PROMPT)) z[t] = z[t] > 0.f ? z[t] / rep : z[t] * rep;
          if (times > 0) z[t] = __fsub_rn(__fsub_rn(z[t], __fmul_rn(freq, (float)min(times, COUNT_MAX))), pres);
          z[t] += bias[t];
          if (!((keep[u] >> t) & 1u)) z[t] = -__int_as_float(0x7F800000);
        }
        v = pack<T>(z);
      }
      T* dst = reinterpret_cast<T*>(p.out) + ((int64_t)b * p.n + i) * p.out_rs;
      const bool write = !p.in_place || touched;
      const uint32_t off = (uint32_t)((uintptr_t)dst & 15);
      if (off == 0) {
        if (write && there == N) *reinterpret_cast<uint4*>(dst + x0) = v;
        else if (write) store_some<T>(dst, x0, v, 0, there);
      } else {
        // own elements from `split` on lie in the next 16-byte piece, whose rest the next lane has
        const int split = N - (int)(off / sizeof(T));
        Piece2 two;
        two.a = v;
        two.b.x = __shfl_down_sync(0xFFFFFFFFu, v.x, 1); two.b.y = __shfl_down_sync(0xFFFFFFFFu, v.y, 1);
        two.b.z = __shfl_down_sync(0xFFFFFFFFu, v.z, 1); two.b.w = __shfl_down_sync(0xFFFFFFFFu, v.w, 1);
        const int next = __shfl_down_sync(0xFFFFFFFFu, there | (write ? 16 : 0), 1);
        const bool whole = lane < 31 && there == N && (next & 15) >= split;
        const int prev = __shfl_up_sync(0xFFFFFFFFu, (int)whole, 1);
        if (whole) {
          // bytes 16 - off .. of the two vectors, as shift_pieces takes them for a row at that offset
          if (write || (next & 16)) *reinterpret_cast<uint4*>(dst + x0 + split) = shift_pieces(two, reinterpret_cast<const T*>((uintptr_t)(16 - off)));
        } else if (write) {
          store_some<T>(dst, x0, v, split, there);
        }
        if (write && !(lane > 0 && prev)) store_some<T>(dst, x0, v, 0, min(split, there));
      }
    }
  }
  if (p.bits) {
    if (bad && p.status) atomicOr(p.status + b, bad);
    if (!p.status) return;
    if (lane == 0 && alive) atomicOr(&alive_s, alive);
    __syncthreads();
    if (threadIdx.x == 0) {
      if (alive_s) atomicOr(p.alive + b, alive_s);
      __threadfence();
      if (atomicAdd(p.arrived + b, 1) == p.chunks * p.groups - 1) {            // every other block has said what it found
        __threadfence();
        const unsigned long long all = p.n == 64 ? ~0ull : (1ull << p.n) - 1ull;
        if (atomicExch(p.alive + b, 0ull) != all) atomicOr(p.status + b, SPACE_ST_BAD_MASK);
        p.arrived[b] = 0;
      }
    }
  }
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
  __shared__ int hist[COUNT_CHUNK];
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.y, t0 = blockIdx.x * COUNT_CHUNK, len = min(COUNT_CHUNK, p.V - t0);
  for (int i = threadIdx.x; i < len; i += THREADS) hist[i] = 0;
  __syncthreads();
  const int n = p.n_tokens ? min(p.n_tokens[b], p.n) : p.n;
  const int32_t* tokens = p.tokens + (int64_t)b * p.stride;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const int t = __ldg(tokens + i);                 // (below 0 or past the vocabulary: in no block's part)
    if (t >= t0 && t < t0 + len) {
      if (p.prompt) hist[t - t0] = SPACE_COUNT_PROMPT;
      else atomicAdd(&hist[t - t0], 1);
    }
  }
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
  const int chunk = THREADS * 16 / esz;
  p.chunks = (int)(((int64_t)p.V + chunk - 1) / chunk);
  // rows are shared out until four thread blocks an SM have some
  const int64_t want = (4ll * ctx->sm_count + (int64_t)p.chunks * p.B - 1) / ((int64_t)p.chunks * p.B);
  const int steps = (p.n + ROWS_AHEAD - 1) / ROWS_AHEAD;
  const int per = ROWS_AHEAD * (int)((steps + (want < steps ? want : steps) - 1) / (want < steps ? want : steps));
  p.groups = (p.n + per - 1) / per;
  const dim3 grid(p.chunks, p.groups, p.B);
  ctx->launches += 1;
  if (esz == 4) return cuda_ok(launch_pdl(logits_adjust_kernel<float>, grid, dim3(THREADS), 0, (cudaStream_t)stream, p));
  return cuda_ok(launch_pdl(logits_adjust_kernel<__nv_bfloat16>, grid, dim3(THREADS), 0, (cudaStream_t)stream, p));
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
