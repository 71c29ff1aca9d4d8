// Attention of a step's block rows over the 8-bit cache (space_kvb_attn_step) on tcgen05, e4m3 operands.
//
// The mathematics.  The cache's codes are tensor-core operands as they lie; what they are multiplied with is split in two:
// a query row, scaled by a power of two of its own, is q0 + q1 with e4m3 numbers (four bits each: bf16 has eight), and so is a weight.
//   S = q0 K^T + q1 K^T,    O_page = w0 V + w1 V.
// A page's weights are taken relative to the page's largest (weight times V scale) of their row, so that V rows which are large and
// hardly seen cost the others no bits, and the page's result joins an fp32 sum in registers with its own factor:
//   chunk b of 32 keys (one K and one V scale 2^k_b, 2^v_b):   m_b = max_j s_j,   e_j = 2^(s_j - m_b),
//   w_j = e_j 2^((m_b - m) + v_b - E + 8),  m = max m_b,  E = max_b (m_b - m) + v_b,     l += sum_b 2^(m_b - M) sum_j e_j,
//   o = o 2^(R - R') + O_page 2^(E + (m - M) - R' - 8)   with R' the larger of R and E + (m - M), both relative to the running maximum M.
// Only differences of scores are ever added to exponents of scales: large scores cost no bits.
//
// The work.  Query rows are the MMA's M extent, a row per thread: 128 of them, or 64 or 32 held twice or four times over,
// each copy with keys of its own (32-key chunks), so that a row's softmax needs no other thread until the item ends and few rows
// keep four warps busy.  The flat list of 128-key pages over all (sequence, kv head, query rows) items is cut evenly
// over the thread blocks, two per SM: one's softmax runs under the other's products.  Pieces of a cut item are joined by the
// block that stores the last of them, always in the same order.
// The block's own rows are one more page: bf16 rows as two e4m3 terms each, the second ones as keys 64 ..; their scores are summed in
// pairs, their weights used twice.
//
// Warps: 0-3 softmax and sums, 4 copies and products (one thread), 5-7 only give their registers away.
// Every wait is bounded; an expired wait sets SPACE_ST_TIMEOUT, no role leaves its loop early, and the block drains and exits.
#include "kvq_attn.cuh"
#include "kvb_common.cuh"

namespace {
using kvq::Cut;
using kvq::lds128;
using kvq::mul2;
using kvq::wait;
using kvq::WAIT_NS;
using namespace kvb;
using namespace tc;

constexpr int TILE = SPACE_PAGE_SIZE;                // keys of a page, rows of an MMA
constexpr int SOFT = 128, THREADS = 2 * SOFT;      // (registers move by groups of four warps)
constexpr int CTAS = 2;                              // per SM
constexpr int SHARE_COST = 2;                        // fixed cost of an item, in pages
constexpr int RING = 8;                              // scales and flags of that many pages
constexpr float F_MIN = 0x1p-120f, F_MAX = 0x1p75f;  // factor of a score: products stay numbers, and differ from 0
constexpr float REF_EXACT = 0x1p23f;                 // up to this a reference's rounding moves weights by 2^0.5 at most

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

template <int DH>
struct Smem {
  using F = Fmt<DH>;
  static constexpr int STAGES = DH == 128 ? 2 : 4;
  static constexpr int Q_PIECE = TILE * DH;                  // [DH / 16][128][16] codes; two of them
  static constexpr int K_OFF = 2 * Q_PIECE;                  // [STAGES]
  static constexpr int V_OFF = K_OFF + STAGES * F::CODES;    // [STAGES]
  static constexpr int SCALE_OFF = V_OFF + STAGES * F::CODES;        // [RING][4] {K, V}
  static constexpr int OWN_OFF = SCALE_OFF + RING * 32;      // [64] {K factor, V exponent} of the block's own rows
  static constexpr int ML_OFF = OWN_OFF + 64 * 8;            // [128] {M, l}
  static constexpr int SRC_OFF = ML_OFF + 128 * 8;           // [RING] addresses of pages on their way
  static constexpr int BAD_OFF = SRC_OFF + RING * 8;         // [RING]
  static constexpr int BAR_OFF = BAD_OFF + RING * 4;
  static constexpr int N_BARS = 2 * STAGES + 4;
  static constexpr int MISC_OFF = BAR_OFF + N_BARS * 8;
  static constexpr int MASK_OFF = (MISC_OFF + 16 + 7) / 8 * 8;
  static constexpr int TABLE_OFF = MASK_OFF + SPACE_MAX_ROWS * 8;    // prefix[max_batch + 1], seq_len[max_batch]
  static_assert(CTAS * (TABLE_OFF + 129 * 4 + 128 * 4 + 1024) <= 228 * 1024, "two blocks per SM");
};

__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
template <int R> __device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R> __device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

#define KVB_R8(r, o) "=r"(r[o]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), "=r"(r[o + 7])
#define KVB_W8(r, o) "r"(r[o]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7])
__device__ __forceinline__ void tmem_ld32(uint32_t a, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
               "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : KVB_R8(r, 0), KVB_R8(r, 8), KVB_R8(r, 16), KVB_R8(r, 24) : "r"(a) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t a, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : KVB_R8(r, 0), KVB_R8(r, 8) : "r"(a) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t a, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(a), KVB_W8(r, 0), KVB_W8(r, 8) : "memory");
}
__device__ __forceinline__ void tmem_st4(uint32_t a, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
// e4m3 x e4m3 -> f32, both operands K-major, M = 128
__device__ __forceinline__ void mma8_ss(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma8_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ constexpr uint32_t instr_desc(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24); }
// Unswizzled K-major operand: 8 rows x 16 bytes lie together, lbo bytes to the next sixteen bytes of K, sbo to the next eight rows.
__device__ __forceinline__ uint64_t plain_desc(uint32_t addr, uint32_t lbo, uint32_t sbo) {
  return (uint64_t)((addr >> 4) & 0x3FFF) | (uint64_t)((lbo >> 4) & 0x3FFF) << 16 | (uint64_t)((sbo >> 4) & 0x3FFF) << 32 | (uint64_t)1 << 46;
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const char* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// Four numbers as two e4m3 terms each: w0 the codes nearest to them, w1 those of what is left.
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

__device__ __forceinline__ float max32(const uint32_t* s) {
  float m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = __uint_as_float(s[i]);
#pragma unroll
  for (int j = 4; j < 28; j += 8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = max3(m[i], __uint_as_float(s[j + 2 * i]), __uint_as_float(s[j + 2 * i + 1]));
  }
  m[0] = max3(m[0], __uint_as_float(s[28]), __uint_as_float(s[29]));
  m[1] = max3(m[1], __uint_as_float(s[30]), __uint_as_float(s[31]));
  return fmaxf(max3(m[0], m[1], m[2]), m[3]);
}

// The items of a block's share, in order: every role walks them for itself.
struct Walk {
  uint32_t cur, end, at;                             // at: the item's place in the list
  int b, it;                                         // item h * n_rt + block of query rows
  int L, t0, t1;                                     // pages [t0, t1) of it; cached rows (-1: the sequence does not fit)
  bool opens;                                        // the share begins with this item
  __device__ __forceinline__ int cached() const { return (max(L, 0) + TILE - 1) / TILE; }    // that page: the block's own rows
  __device__ __forceinline__ int pages(int has_new) const { return max(cached() + has_new, 1); }
  __device__ __forceinline__ bool next(const uint32_t* prefix, const int* seq_len, int has_new, uint32_t share0) {
    while (cur < end) {
      while (prefix[b + 1] <= cur) ++b;
      L = seq_len[b];
      const int Tv = pages(has_new) + SHARE_COST;
      const uint32_t rem = cur - prefix[b];
      it = (int)(rem / (uint32_t)Tv);
      const int x0 = (int)rem - it * Tv, n = min(Tv - x0, (int)(end - cur));
      opens = cur == share0;
      at = cur - x0;
      cur += n;
      t0 = max(x0 - SHARE_COST, 0); t1 = x0 + n - SHARE_COST;
      if (t1 > t0) return true;                      // (else only the cost of starting)
    }
    return false;
  }
};

__device__ __forceinline__ uint4 pack_row8(const float* y) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
    r[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// The pieces of an item that was cut over several thread blocks: outputs of their own keys, weighed by l 2^M.  A thread has
// four channels of a row; the DH / 4 threads of a row look up that many pieces' M and l at once.
template <int DH, int RT>
__device__ __forceinline__ void join_pieces(const Params& p, const Cut& cut, int b, int h, int r0, int rows, uint32_t piece0, int pieces, uint32_t item_at, int tid) {
  constexpr int C4 = DH / 4, SLOT = RT * (DH + 2), BATCH = 8;
  const float* part = p.part + (int64_t)(2 * piece0) * SLOT;
  const int first = cut.begin(piece0) >= item_at ? 0 : SLOT, n = rows * C4, c4 = tid % C4;
  auto at = [&](int x) { return part + (x == 0 ? (int64_t)first : (int64_t)x * (2 * SLOT)); };
#pragma unroll 1
  for (int idx = tid - tid % 32; idx < n; idx += SOFT) {                       // (warps stay whole)
    const int r = min((idx + tid % 32) / C4, rows - 1);
    float M = -CUDART_INF_F, den = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int x0 = 0; x0 < pieces; x0 += C4) {
      const bool there = x0 + c4 < pieces;
      const float m = there ? __ldcg(at(x0 + c4) + RT * DH + r) : -CUDART_INF_F;
      const float l = there ? __ldcg(at(x0 + c4) + RT * DH + RT + r) : 0.f;
      float w = 0.f;
#pragma unroll 1
      for (int y = 0; y < C4 && x0 + y < pieces; y += BATCH) {
        float4 v[BATCH];
#pragma unroll
        for (int j = 0; j < BATCH; ++j)
          v[j] = x0 + y + j < pieces && y + j < C4 ? __ldcg(reinterpret_cast<const float4*>(at(x0 + y + j) + r * DH) + c4) : make_float4(0.f, 0.f, 0.f, 0.f);
        if (y == 0) {
          float top = m;
#pragma unroll
          for (int k = 1; k < C4; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, k));
          top = fmaxf(top, M);
          const float down = M == -CUDART_INF_F ? 0.f : fast_exp2(M - top);
          M = top;
          w = m == -CUDART_INF_F ? 0.f : l * fast_exp2(m - top);
          float sum = w;
#pragma unroll
          for (int k = 1; k < C4; k <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, k);
          den = fmaf(den, down, sum);
          o.x *= down; o.y *= down; o.z *= down; o.w *= down;
        }
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
          const float f = __shfl_sync(0xFFFFFFFFu, w, (y + j) % C4, C4);       // (past the last: v is 0)
          o.x = fmaf(v[j].x, f, o.x); o.y = fmaf(v[j].y, f, o.y); o.z = fmaf(v[j].z, f, o.z); o.w = fmaf(v[j].w, f, o.w);
        }
      }
    }
    if (idx + tid % 32 < n) {
      const int i = (r0 + r) >> p.gsh, hq = (h << p.gsh) + ((r0 + r) & (p.G - 1));
      const float rd = den > 0.f ? 1.f / den : 0.f;  // a row without keys: zeros
      const __nv_bfloat162 x = __floats2bfloat162_rn(o.x * rd, o.y * rd), y = __floats2bfloat162_rn(o.z * rd, o.w * rd);
      __nv_bfloat16* dst = p.out + (((int64_t)b * p.n_q + i) * p.H_q + hq) * DH + 4 * c4;
      *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
      if (c4 == 0 && p.lse) p.lse[((int64_t)b * p.H_q + hq) * p.n_q + i] = (M + log2f(den)) * 0.6931471805599453f;
    }
  }
}

template <int DH, int REP>
__global__ void __launch_bounds__(THREADS, CTAS) kvb_attn_kernel(const __grid_constant__ Params p, int max_batch) {
  using F = Fmt<DH>;
  using S = Smem<DH>;
  constexpr int STAGES = S::STAGES, RT = TILE / REP, NC = 4 / REP;             // rows of an item, chunks of a copy of them
  extern __shared__ __align__(1024) unsigned char sm[];
  const uint32_t base = smem_u32(sm), bar0 = base + S::BAR_OFF;
  auto BAR = [&](int i) { return bar0 + 8u * i; };
  // GO: the softmax warps have come to a page, and what they bring for its products is there; SDONE: its scores are (or it has
  // none).  Both sides pass each page through these two, products or not: neither gets a phase ahead of the other.
  constexpr int FULLK = 0, FULLV = STAGES, GO = 2 * STAGES, SDONE = GO + 1, PREADY = GO + 2, ODONE = GO + 3;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + S::MISC_OFF);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::MISC_OFF + 4);
  volatile int* last_flag = reinterpret_cast<volatile int*>(sm + S::MISC_OFF + 8);
  uint32_t* prefix = reinterpret_cast<uint32_t*>(sm + S::TABLE_OFF);
  int* seq_len = reinterpret_cast<int*>(prefix + max_batch + 1);
  volatile int* bad = reinterpret_cast<volatile int*>(sm + S::BAD_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;

  if (tid == 0) {
    *abort_flag = 0;
    for (int s = 0; s < 2 * STAGES; ++s) mbar_init(BAR(s), 1);
    mbar_init(BAR(GO), 4); mbar_init(BAR(SDONE), 1); mbar_init(BAR(PREADY), 4); mbar_init(BAR(ODONE), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (tid < SPACE_MAX_ROWS) reinterpret_cast<uint64_t*>(sm + S::MASK_OFF)[tid] = p.mask[tid];
  // Tensor memory is taken when the kernel before has given its own back, and the next kernel's blocks may come when all of these
  // have theirs: nobody holds some while it waits for somebody who wants some.
  pdl_wait();
  if (warp == 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(256u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (warp == 0) {
    uint32_t carry = 0;                              // running sums of the list
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const int b = b0 + lane;
      int L = -1;
      uint32_t n = 0;
      if (b < p.B) {
        L = p.kv_len[b];
        if (L < 0 || (int64_t)L > (int64_t)p.cache.pages_per_seq * TILE) {
          if (blockIdx.x == 0 && p.status) atomicOr(p.status + b, SPACE_ST_CAPACITY);
          L = -1;
        }
        n = (uint32_t)((max((max(L, 0) + TILE - 1) / TILE + p.has_new, 1) + SHARE_COST) * p.H_kv * p.n_rt);
      }
      uint32_t incl = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += v;
      }
      if (b < p.B) { seq_len[b] = L; prefix[b] = carry + incl - n; }
      carry += __shfl_sync(0xFFFFFFFFu, incl, 31);
    }
    if (lane == 0) prefix[p.B] = carry;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_launch_dependents();
  const uint32_t tmem = *tmem_slot;
  const uint32_t TM_S = tmem, TM_O = tmem + TILE;    // S (its columns are the weights' afterwards), O
  const Cut cut(prefix[p.B], p.n_groups);
  Walk wk;
  const bool mine = blockIdx.x < cut.NG;
  const uint32_t share0 = mine ? cut.begin(blockIdx.x) : 0;
  wk.b = 0; wk.cur = share0;
  wk.end = mine ? cut.begin(blockIdx.x + 1) : 0;
  uint32_t g = 0, m = 0;                             // pages, and pages with products, so far
  auto hold = [&](int bar, uint32_t use, int site) { return wait(BAR(bar), use & 1, abort_flag, p.err, site); };

  if (warp >= 4) {
    regs_dec<48>();
    if (warp == 4 && elect_one()) {
      // ---- pages ahead: K, scales and V of page `fetched`, K as soon as a stage's K has been used, V when its V has been
      Walk pw = wk;
      uint32_t fetched = 0;
      volatile uint64_t* src_ring = reinterpret_cast<volatile uint64_t*>(sm + S::SRC_OFF);
      bool live = pw.next(prefix, seq_len, p.has_new, share0);
      int t = live ? pw.t0 : 0;
      auto page_of = [&]() { return live && t < pw.cached() ? __ldg(p.cache.page_table + (int64_t)pw.b * p.cache.pages_per_seq + t) : -1; };
      int pg = page_of();                            // (one page ahead of its use)
      auto fetch_k = [&]() {
        if (!live) return;
        const uint32_t s = fetched % STAGES, e = fetched % RING;
        const bool cached = t < pw.cached(), good = cached && pg >= 0 && pg < p.cache.n_pages;
        bad[e] = !good;
        uint64_t src = 0;
        if (good) {
          const char* head = p.cache.pool + (int64_t)pg * p.cache.page_stride + (int64_t)(pw.it / p.n_rt) * p.cache.head_stride;
          src = (uint64_t)head;
          mbar_expect_tx(BAR(FULLK + s), F::CODES + 32);
          bulk_copy(base + S::K_OFF + s * F::CODES, head, F::CODES, BAR(FULLK + s));
          bulk_copy(base + S::SCALE_OFF + e * 32, head + F::SCALES, 32, BAR(FULLK + s));
        } else {
          if (cached && p.status) atomicOr(p.status + pw.b, SPACE_ST_BAD_PAGE);
          mbar_arrive(BAR(FULLK + s));
        }
        src_ring[e] = src;
        ++fetched;
        if (++t == pw.t1) {
          live = pw.next(prefix, seq_len, p.has_new, share0);
          t = pw.t0;
        }
        pg = page_of();
      };
      auto fetch_v = [&](uint32_t j) {
        if (j >= fetched) return;
        const uint32_t s = j % STAGES;
        const char* head = reinterpret_cast<const char*>(src_ring[j % RING]);
        if (head) {
          mbar_expect_tx(BAR(FULLV + s), F::CODES);
          bulk_copy(base + S::V_OFF + s * F::CODES, head + F::CODES, F::CODES, BAR(FULLV + s));
        } else {
          mbar_arrive(BAR(FULLV + s));
        }
      };
      for (uint32_t j = 0; j < STAGES; ++j) { fetch_k(); fetch_v(j); }
      const uint64_t q0 = plain_desc(base, 16 * TILE, 128);
      bool ok = true;
      while (wk.next(prefix, seq_len, p.has_new, share0)) {
        const int Tc = wk.cached();
        for (int tt = wk.t0; tt < wk.t1; ++tt, ++g) {
          const uint32_t s = g % STAGES;
          ok = hold(FULLK + s, g / STAGES, 2) && ok;
          const bool own = tt >= Tc;
          const bool products = own ? p.has_new && wk.L >= 0 : !bad[g % RING];
          ok = hold(GO, g, 1) && ok;
          if (products && ok) {
            tc_fence_after();
            const uint64_t kd = plain_desc(base + S::K_OFF + s * F::CODES, 16 * TILE, 128);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int ks = 0; ks < DH / 32; ++ks)
                mma8_ss(TM_S, q0 + (uint64_t)((i * S::Q_PIECE + ks * 32 * TILE) >> 4), kd + (uint64_t)((ks * 32 * TILE) >> 4), instr_desc(TILE), i + ks > 0);
          }
          if (products) tc_commit(BAR(SDONE));
          else mbar_arrive(BAR(SDONE));
          ok = hold(SDONE, g, 3) && ok;
          fetch_k();
          ok = hold(FULLV + s, g / STAGES, 5) && ok;
          if (products) {
            ok = hold(PREADY, m, 6) && ok;
            if (ok) {
              tc_fence_after();
              const uint64_t vd = plain_desc(base + S::V_OFF + s * F::CODES, F::V_ROWS, 128);
#pragma unroll
              for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                  mma8_ts(TM_O, TM_S + 16 * b + 8 * i, vd + (uint64_t)((2 * b * F::V_ROWS) >> 4), instr_desc(DH), b + i > 0);
            }
            tc_commit(BAR(ODONE));
            ok = hold(ODONE, m, 7) && ok;
            ++m;
          }
          fetch_v(g + STAGES);
        }
      }
      // (every copy was waited for above; after a wait that ran out, here)
      if (*abort_flag)
        for (uint32_t j = fetched > STAGES ? fetched - STAGES : 0; j < fetched; ++j) {
          mbar_drain_bounded(BAR(FULLK + j % STAGES), (j / STAGES) & 1, WAIT_NS);
          mbar_drain_bounded(BAR(FULLV + j % STAGES), (j / STAGES) & 1, WAIT_NS);
        }
    }
  } else {
    regs_inc<208>();                                 // (128 threads x 208 + 128 x 48 = the 256 x 128 of the launch)
    const int rep = warp / (4 / REP), row = tid % RT;
    const uint32_t lanes = (uint32_t)(32 * warp) << 16;
    float2* ml = reinterpret_cast<float2*>(sm + S::ML_OFF);
    float2* own = reinterpret_cast<float2*>(sm + S::OWN_OFF);
    while (wk.next(prefix, seq_len, p.has_new, share0)) {
      const int h = wk.it / p.n_rt, r0 = (wk.it - h * p.n_rt) * RT, rows = min(p.n_q * p.G - r0, RT), Tc = wk.cached();
      const int qi = (r0 + row) >> p.gsh, hq = (h << p.gsh) + ((r0 + row) & (p.G - 1));
      const bool there = row < rows;
      // ---- the query row, as two terms
      float f;                                       // factor of a score
      bool nan = false;
      {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)wk.b * p.q_sb + (int64_t)qi * p.q_sr + (int64_t)hq * p.q_sh);
        uint4 v[DH / 8];
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < DH / 8; ++j) v[j] = there ? src[j] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < DH / 8; ++j) top = max(top, kvq::max_bits(v[j]));
        nan = top >= 0x7F80u;
        const int e = nan ? 0 : max((int)(top >> 7) - 127, -100) - 7;          // the largest element to [2^7, 2^8)
        const float up = pow2(-e);
        f = p.c * pow2(e);
#pragma unroll
        for (int j = 0; j < DH / 16; ++j) {
          uint32_t w0[4], w1[4];
          const uint32_t x[8] = {v[2 * j].x, v[2 * j].y, v[2 * j].z, v[2 * j].w, v[2 * j + 1].x, v[2 * j + 1].y, v[2 * j + 1].z, v[2 * j + 1].w};
#pragma unroll
          for (int k = 0; k < 4; ++k)
            split4(kvq::bf_lo(x[2 * k]) * up, kvq::bf_hi(x[2 * k]) * up, kvq::bf_lo(x[2 * k + 1]) * up, kvq::bf_hi(x[2 * k + 1]) * up, w0[k], w1[k]);
          const uint32_t to = base + j * (16 * TILE) + 16 * tid;
          asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(w0[0]), "r"(w0[1]), "r"(w0[2]), "r"(w0[3]) : "memory");
          asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to + S::Q_PIECE), "r"(w1[0]), "r"(w1[1]), "r"(w1[2]), "r"(w1[3]) : "memory");
        }
        fence_async();
      }
      uint64_t o2[DH / 2];
#pragma unroll
      for (int j = 0; j < DH / 2; ++j) o2[j] = 0ull;
      float M = -CUDART_INF_F, l = 0.f, R = 0.f, alpha = 1.f, beta = 0.f;
      bool pending = false;
      // the last page's result joins the sum
      auto take = [&]() {
        hold(ODONE, m - 1, 8);
        tc_fence_after();
        if (__any_sync(0xFFFFFFFFu, alpha != 1.f)) {
          const uint64_t a2 = pack2(alpha, alpha);
#pragma unroll
          for (int j = 0; j < DH / 2; ++j) o2[j] = mul2(o2[j], a2);
        }
        const uint64_t b2 = pack2(beta, beta);
#pragma unroll
        for (int c = 0; c < DH; c += 32) {
          uint32_t v[32];
          tmem_ld32(TM_O + lanes + c, v);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 16; ++j) o2[c / 2 + j] = fma2(pack2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), b2, o2[c / 2 + j]);
        }
        tc_fence_before();
        pending = false;
      };
      // a page's maximum pm, and E: the running ones, and the factors of the sums
      auto advance = [&](float pm, float E, float& lead) {
        lead = 0.f; alpha = 1.f; beta = 0.f;
        if (pm == -CUDART_INF_F) return;             // this row sees nothing of the page
        const float Mn = fmaxf(M, pm), d_old = M - Mn;
        lead = fast_exp2(pm - Mn);
        l *= fast_exp2(d_old);
        const float r_old = R + d_old, r_new = E + (pm - Mn), Rn = fmaxf(r_old, r_new);
        alpha = fast_exp2(r_old - Rn);
        beta = fast_exp2(r_new - Rn - 8.f);
        M = Mn; R = Rn;
      };
      for (int t = wk.t0; t < wk.t1; ++t, ++g) {
        const uint32_t s = g % STAGES;
        const bool is_own = t >= Tc;
        hold(FULLK + s, g / STAGES, 9);
        const bool products = is_own ? p.has_new && wk.L >= 0 : !bad[g % RING];
        if (!is_own || !products) {
          __syncwarp();
          if (lane == 0) mbar_arrive(BAR(GO));
        }
        if (!products) {
          hold(SDONE, g, 13);
          continue;
        }
        if (pending) take();
        if (!is_own) {
          const float2* sc = reinterpret_cast<const float2*>(sm + S::SCALE_OFF + (g % RING) * 32);
          const int vis0 = wk.L - t * TILE;          // visible keys of the page
          if (vis0 < TILE) {                         // what lies behind the last row must not count, whatever it is
            hold(FULLV + s, g / STAGES, 10);
            const int g0 = vis0 >> 4;
            for (int e = tid; e < (8 - g0) * DH; e += SOFT) {
              const int grp = g0 + e / DH, keep = min(max(vis0 - 16 * grp, 0), 16);
              unsigned char* at = sm + S::V_OFF + s * F::CODES + grp * F::V_ROWS + (e % DH) * 16;
              uint4 w = make_uint4(0, 0, 0, 0);
              if (keep) {
                w = *reinterpret_cast<const uint4*>(at);
                uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const int n = min(max(keep - 4 * j, 0), 4);
                  x[j] &= n == 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u;
                }
                w = make_uint4(x[0], x[1], x[2], x[3]);
              }
              *reinterpret_cast<uint4*>(at) = w;
            }
            fence_async();
          }
          hold(SDONE, g, 11);
          tc_fence_after();
          // ---- largest scores
          float fk[NC], mb[NC];
          uint32_t v[32];
          float pm = -CUDART_INF_F;
#pragma unroll
          for (int k = 0; k < NC; ++k) {
            const int cb = rep * NC + k, vis = vis0 - BLOCK_ROWS * cb;
            mb[k] = -CUDART_INF_F;
            fk[k] = fminf(fmaxf(f * sc[cb].x, F_MIN), F_MAX);
            if (vis > 0) {
              tmem_ld32(TM_S + lanes + 32 * cb, v);
              tmem_wait_ld();
              if (vis < BLOCK_ROWS) {
#pragma unroll
                for (int j = 0; j < 32; ++j) if (j >= vis) v[j] = 0xFF800000u;
              }
              mb[k] = max32(v) * fk[k];
            }
            pm = fmaxf(pm, mb[k]);
          }
          float x[NC], E = -CUDART_INF_F;
#pragma unroll
          for (int k = 0; k < NC; ++k) {
            const int ev = (int)((__float_as_uint(sc[rep * NC + k].y) >> 23) & 255u) - 127;
            x[k] = mb[k] == -CUDART_INF_F ? -CUDART_INF_F : (mb[k] - pm) + (float)ev;
            E = fmaxf(E, x[k]);
          }
          float lead;
          advance(pm, E, lead);
          // ---- weights
#pragma unroll
          for (int k = 0; k < NC; ++k) {
            const int cb = rep * NC + k, vis = vis0 - BLOCK_ROWS * cb;
            uint32_t w[16];
            if (vis > 0) {
              if (NC > 1) {
                tmem_ld32(TM_S + lanes + 32 * cb, v);
                tmem_wait_ld();
                if (vis < BLOCK_ROWS) {
#pragma unroll
                  for (int j = 0; j < 32; ++j) if (j >= vis) v[j] = 0xFF800000u;
                }
              }
              float nb = mb[k] == -CUDART_INF_F ? 0.f : -mb[k];
              if (__any_sync(0xFFFFFFFFu, fabsf(nb) > REF_EXACT)) {            // scores off the largest first, then times the factor
                const float top = max32(v);
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) - (nb == 0.f ? 0.f : top));
                nb = 0.f;
              }
              const float wf = mb[k] == -CUDART_INF_F ? 0.f : fast_exp2(x[k] - E + 8.f);
              const uint64_t f2 = pack2(fk[k], fk[k]), n2 = pack2(nb, nb), w2 = pack2(wf, wf);
              uint64_t sum0 = 0ull, sum1 = 0ull;
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                float a, b, c, d;
                unpack2(fma2(pack2(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1])), f2, n2), a, b);
                unpack2(fma2(pack2(__uint_as_float(v[4 * j + 2]), __uint_as_float(v[4 * j + 3])), f2, n2), c, d);
                const uint64_t e0 = pack2(fast_exp2(a), fast_exp2(b)), e1 = pack2(fast_exp2(c), fast_exp2(d));
                sum0 = add2(sum0, e0); sum1 = add2(sum1, e1);
                unpack2(mul2(e0, w2), a, b);
                unpack2(mul2(e1, w2), c, d);
                split4(a, b, c, d, w[j], w[8 + j]);
              }
              float a, b;
              unpack2(add2(sum0, sum1), a, b);
              if (mb[k] != -CUDART_INF_F) l = fmaf(a + b, lead * fast_exp2(mb[k] - pm), l);
            } else {
#pragma unroll
              for (int j = 0; j < 16; ++j) w[j] = 0;
            }
            tmem_st16(TM_S + lanes + 16 * cb, w);
          }
          if (REP > 1) {                             // keys that other copies of the row have
            const uint32_t zero[16] = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int b = 0; b < 4; ++b)
              if (b / NC != rep) tmem_st16(TM_S + lanes + 16 * b, zero);
          }
        } else {
          // ---- the block's own rows: keys j and 64 + j of the page are the two terms of row j
          {
            const int key = tid >> 1, c0 = (tid & 1) * (DH / 2);
            const bool real = key < p.n_q;
#pragma unroll 1
            for (int which = 0; which < 2; ++which) {
              const uint4* src = reinterpret_cast<const uint4*>((which ? p.vn : p.kn) + (int64_t)wk.b * p.n_sb + (int64_t)key * p.n_sr + (int64_t)h * p.n_sh) + c0 / 8;
              uint4 v[DH / 16];
              uint32_t top = 0;
#pragma unroll
              for (int j = 0; j < DH / 16; ++j) v[j] = real ? src[j] : make_uint4(0, 0, 0, 0);
#pragma unroll
              for (int j = 0; j < DH / 16; ++j) top = max(top, kvq::top_bits(v[j]));       // (and what is not finite made so)
              top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
              const int e = max((int)(top >> 7) - 127, -100) - 7;
              const float up = pow2(-e);
              if ((tid & 1) == 0) {
                if (which) own[key].y = (float)e;
                else own[key].x = pow2(e);
              }
#pragma unroll
              for (int j = 0; j < DH / 32; ++j) {
                uint32_t w0[4], w1[4];
                const uint32_t x[8] = {v[2 * j].x, v[2 * j].y, v[2 * j].z, v[2 * j].w, v[2 * j + 1].x, v[2 * j + 1].y, v[2 * j + 1].z, v[2 * j + 1].w};
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  split4(kvq::bf_lo(x[2 * k]) * up, kvq::bf_hi(x[2 * k]) * up, kvq::bf_lo(x[2 * k + 1]) * up, kvq::bf_hi(x[2 * k + 1]) * up, w0[k], w1[k]);
                if (which == 0) {
                  unsigned char* to = sm + S::K_OFF + s * F::CODES + (c0 / 16 + j) * F::K_COLS + 16 * key;
                  *reinterpret_cast<uint4*>(to) = make_uint4(w0[0], w0[1], w0[2], w0[3]);
                  *reinterpret_cast<uint4*>(to + 16 * 64) = make_uint4(w1[0], w1[1], w1[2], w1[3]);
                } else {
                  unsigned char* to = sm + S::V_OFF + s * F::CODES + (key >> 4) * F::V_ROWS + (c0 + 16 * j) * 16 + (key & 15);
#pragma unroll
                  for (int k = 0; k < 16; ++k) {
                    to[16 * k] = (unsigned char)(w0[k >> 2] >> (8 * (k & 3)));
                    to[16 * k + 4 * F::V_ROWS] = (unsigned char)(w1[k >> 2] >> (8 * (k & 3)));
                  }
                }
              }
            }
            fence_async();
            soft_sync();
            if (lane == 0) mbar_arrive(BAR(GO));
          }
          hold(SDONE, g, 12);
          tc_fence_after();
          // (the first copy of the rows has them all)
          const uint64_t see = rep == 0 && there ? reinterpret_cast<const uint64_t*>(sm + S::MASK_OFF)[qi] : 0ull;
          float pm = -CUDART_INF_F, E = -CUDART_INF_F;
          auto scores = [&](int j0, float* sc) {     // sixteen of them
            uint32_t a[16], b[16];
            tmem_ld16(TM_S + lanes + j0, a);
            tmem_ld16(TM_S + lanes + 64 + j0, b);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float fj = fminf(fmaxf(f * own[j0 + j].x, F_MIN), F_MAX);
              sc[j] = (see >> (j0 + j)) & 1ull ? (__uint_as_float(a[j]) + __uint_as_float(b[j])) * fj : -CUDART_INF_F;
            }
          };
          float sc[16];
          if (rep == 0) {
#pragma unroll 1
            for (int j0 = 0; j0 < 64; j0 += 16) {
              scores(j0, sc);
#pragma unroll
              for (int j = 0; j < 16; ++j) pm = fmaxf(pm, sc[j]);
            }
#pragma unroll 1
            for (int j0 = 0; j0 < 64; j0 += 16) {
              scores(j0, sc);
#pragma unroll
              for (int j = 0; j < 16; ++j) E = fmaxf(E, sc[j] == -CUDART_INF_F ? -CUDART_INF_F : (sc[j] - pm) + own[j0 + j].y);
            }
          }
          float lead, sum = 0.f;
          advance(pm, E, lead);
#pragma unroll 1
          for (int j0 = 0; j0 < 64; j0 += 16) {
            uint32_t w0[4], w1[4];
            if (rep == 0) {
              scores(j0, sc);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                float y[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const float d = sc[4 * j + k] - pm;
                  const bool vis = sc[4 * j + k] != -CUDART_INF_F;
                  sum += vis ? fast_exp2(d) : 0.f;
                  y[k] = vis ? fast_exp2(d + own[j0 + 4 * j + k].y - E + 8.f) : 0.f;
                }
                split4(y[0], y[1], y[2], y[3], w0[j], w1[j]);
              }
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j) w0[j] = w1[j] = 0;
            }
            // words of keys j0 .. of their chunk of 32, in columns whose scores have been read
            tmem_st4(TM_S + lanes + (j0 >> 5) * 16 + ((j0 >> 4) & 1) * 4, w0);
            tmem_st4(TM_S + lanes + (j0 >> 5) * 16 + ((j0 >> 4) & 1) * 4 + 8, w1);
          }
          l = fmaf(sum, lead, l);
          tmem_wait_st();
          {
            uint32_t w[32];
            tmem_ld32(TM_S + lanes, w);
            tmem_wait_ld();
            tmem_st16(TM_S + lanes + 32, w);
            tmem_st16(TM_S + lanes + 48, w + 16);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(PREADY));
        pending = true;
        ++m;
      }
      if (pending) take();

      // ---- the item's rows, or its piece of them
      const bool whole = wk.t0 == 0 && wk.t1 == wk.pages(p.has_new);
      const int slot = 2 * (int)blockIdx.x + (wk.opens ? 0 : 1);
      constexpr int SLOT = RT * (DH + 2);
      float* ps = p.part + (int64_t)slot * SLOT;
      __nv_bfloat16* dst = p.out + (((int64_t)wk.b * p.n_q + qi) * p.H_q + hq) * DH;
      const float NAN_F = __int_as_float(0x7FFFFFFF);
      float Mx = M, Lx = l;
      if (REP > 1) {
        ml[tid] = make_float2(M, l);
        soft_sync();
#pragma unroll
        for (int r = 0; r < REP; ++r) Mx = fmaxf(Mx, ml[r * RT + row].x);
        Lx = 0.f;
#pragma unroll
        for (int r = 0; r < REP; ++r) {
          const float2 v = ml[r * RT + row];
          Lx += v.x == -CUDART_INF_F ? 0.f : v.y * fast_exp2(v.x - Mx);
        }
      }
      float fac = M == -CUDART_INF_F ? 0.f : fast_exp2(M - Mx) / Lx * fast_exp2(R);
      if (nan && Mx != -CUDART_INF_F) { fac = NAN_F; Lx = NAN_F; }
      if (REP == 1) {
        if (there) {
#pragma unroll
          for (int c = 0; c < DH; c += 8) {
            float y[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              unpack2(o2[c / 2 + j], y[2 * j], y[2 * j + 1]);
              y[2 * j] *= fac; y[2 * j + 1] *= fac;
            }
            if (whole) *reinterpret_cast<uint4*>(dst + c) = pack_row8(y);
            else {
              __stcg(reinterpret_cast<float4*>(ps + row * DH + c), make_float4(y[0], y[1], y[2], y[3]));
              __stcg(reinterpret_cast<float4*>(ps + row * DH + c + 4), make_float4(y[4], y[5], y[6], y[7]));
            }
          }
        }
      } else {
        // copies of a row meet, half of the channels at a time, where the query rows were
        constexpr int CP = DH / 2, CS = CP / REP;
        float* buf = reinterpret_cast<float*>(sm);   // [CP][128]
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
          for (int c = 0; c < CP / 2; ++c) {
            float a, b;
            unpack2(o2[pass * (CP / 2) + c], a, b);
            buf[(2 * c) * TILE + tid] = a * fac;
            buf[(2 * c + 1) * TILE + tid] = b * fac;
          }
          soft_sync();
          if (there) {
#pragma unroll
            for (int c = 0; c < CS; c += 8) {
              float y[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                y[j] = 0.f;
#pragma unroll
                for (int r = 0; r < REP; ++r) y[j] += buf[(rep * CS + c + j) * TILE + r * RT + row];
              }
              const int ch = pass * CP + rep * CS + c;
              if (whole) *reinterpret_cast<uint4*>(dst + ch) = pack_row8(y);
              else {
                __stcg(reinterpret_cast<float4*>(ps + row * DH + ch), make_float4(y[0], y[1], y[2], y[3]));
                __stcg(reinterpret_cast<float4*>(ps + row * DH + ch + 4), make_float4(y[4], y[5], y[6], y[7]));
              }
            }
          }
          soft_sync();
        }
      }
      if (there && rep == 0) {
        if (!whole) { __stcg(ps + RT * DH + row, Mx); __stcg(ps + RT * DH + RT + row, Lx); }
        else if (p.lse) p.lse[((int64_t)wk.b * p.H_q + hq) * p.n_q + qi] = (Mx + log2f(Lx)) * 0.6931471805599453f;
      }
      if (*abort_flag && p.status && tid == 0) atomicOr(p.status + wk.b, SPACE_ST_TIMEOUT);
      if (!whole) {
        const int T = wk.pages(p.has_new);
        const uint32_t piece0 = cut.owner(wk.at + SHARE_COST);
        const int pieces = (int)(cut.owner(wk.at + SHARE_COST + T - 1) - piece0) + 1;
        soft_sync();
        if (tid == 0) {
          __threadfence();                           // (after the barrier: for all the stores)
          int* arrived = p.arrived + (wk.b * p.H_kv * p.n_rt + wk.it);
          const int last = atomicAdd(arrived, 1) == pieces - 1;
          if (last) *arrived = 0;                    // ready for the next call
          __threadfence();
          *last_flag = last;
        }
        soft_sync();
        if (*last_flag) join_pieces<DH, RT>(p, cut, wk.b, h, r0, rows, piece0, pieces, wk.at, tid);
        soft_sync();                                 // the flag is free for the next item
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 4) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(256u));
}

template <int DH>
size_t smem_bytes(int max_batch) { return Smem<DH>::TABLE_OFF + (size_t)(max_batch + 1) * 4 + (size_t)max_batch * 4; }

template <int DH, int REP>
cudaError_t launch_dim(Params& p, const space_ctx* ctx, cudaStream_t st) {
  static unsigned long long done_mask = 0;           // devices on which the kernel may have its shared memory
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 64 || !((done_mask >> dev) & 1ull)) {
    const cudaError_t e = cudaFuncSetAttribute(kvb_attn_kernel<DH, REP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<DH>(128));
    if (e != cudaSuccess) return e;
    if (dev < 64) done_mask |= 1ull << dev;
  }
  p.n_rt = (p.n_q * p.G + TILE / REP - 1) / (TILE / REP);
  p.n_groups = CTAS * ctx->sm_count;
  return launch_pdl(kvb_attn_kernel<DH, REP>, dim3(p.n_groups), dim3(THREADS), smem_bytes<DH>(ctx->cfg.max_batch), st, p, ctx->cfg.max_batch);
}

}  // namespace

int launch_kvb_attn(space_ctx* ctx, const space_kvb_attn_args* a, const uint64_t* mask_rows, cudaStream_t st) {
  Params p;
  memset(&p, 0, sizeof(p));
  p.cache = cache_of(a->cache);
  p.B = a->batch; p.n_q = (a->k + 1) * (a->k + 1); p.H_q = ctx->cfg.n_q_heads; p.H_kv = ctx->cfg.n_kv_heads;
  p.G = p.H_q / p.H_kv;
  while ((1 << p.gsh) < p.G) ++p.gsh;
  p.has_new = a->k_new != nullptr;
  p.c = a->scale * 1.4426950408889634f;
  p.q = (const char*)a->q; p.q_sb = 2 * a->q_stride_b; p.q_sr = 2 * a->q_stride_r; p.q_sh = 2 * a->q_stride_h;
  p.kn = (const char*)a->k_new; p.vn = (const char*)a->v_new;
  p.n_sb = 2 * a->new_stride_b; p.n_sr = 2 * a->new_stride_r; p.n_sh = 2 * a->new_stride_h;
  p.kv_len = a->kv_len; p.out = (__nv_bfloat16*)a->out; p.lse = a->lse; p.status = a->status;
  p.part = ctx->attn_part; p.arrived = ctx->kvb_arrived; p.err = ctx->counters + 3 * ctx->cfg.max_batch;
  for (int i = 0; i < p.n_q; ++i) p.mask[i] = mask_rows[i];
  const int rows = p.n_q * p.G;
  // the flat list is counted in 32 bits
  if ((double)p.B * p.H_kv * ((rows + 31) / 32) * ((double)p.cache.pages_per_seq + 8) > 2e9) return SPACE_E_UNSUPPORTED;
  ctx->launches += 1;
  const bool wide = ctx->cfg.head_dim == 128;
  const int rt = kvb_item_rows(rows);
  cudaError_t e;
  if (wide) e = rt == 32 ? launch_dim<128, 4>(p, ctx, st) : rt == 64 ? launch_dim<128, 2>(p, ctx, st) : launch_dim<128, 1>(p, ctx, st);
  else e = rt == 32 ? launch_dim<64, 4>(p, ctx, st) : rt == 64 ? launch_dim<64, 2>(p, ctx, st) : launch_dim<64, 1>(p, ctx, st);
  return cuda_ok(e);
}
