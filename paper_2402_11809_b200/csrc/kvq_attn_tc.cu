// Attention of a step's block rows over the 4-bit cache (space_kvq_attn_step), items of 64 query rows on tcgen05.
//
// The mathematics is kvq_attn.cu's but for one thing: products of bare K codes, steps and lowest values in the softmax,
// weights e step against a reference of their own; the V codes become (u + lo / step) 2^-9 on their way (one product and
// sum of the masked code, rounded to 11 bits once, as the weights are), so that there is no second sum of e (lo + 8 step)
// to keep per query row and key.  So is the work: (sequence, kv head, query rows) items, one flat list of 128-key pages, an
// equal share per thread block, cut items joined by the block that stores their last piece.
//
// The products are taken transposed, the 128 keys (channels) of a page on the MMA's M extent and the query rows on N:
//   S^T = U Q^T  (128 x N),      O^T += V^T P^T  (d x N).
// Both first operands come from tensor memory: the codes are unpacked in registers and stored there (tcgen05.st), because
// through shared memory the unpacked page would cost 4 d bytes written and as many read per key, more than the tensor
// core's products take.  The cache's order is that of the 16x256b store: a lane's 16 bytes are its registers.
//
// What bounds it is the softmax threads: a page of 64 rows takes 1.45 us, its products 0.2 us, the unpacking 0.5 beside
// them; left out one at a time, exponentials, products, unpacking or sums change it by 5 % at most, and what it follows
// is the number of instructions that the loops of all roles have, and whether the softmax warps run through theirs together.
// So (8 x 8 heads, 392 rows of 8192 keys; 451 us on mma.sync): sixteen softmax warps instead of eight (417 -> 396); whether
// a page's scores pass the limits is asked by an mbarrier under the exponentials, not by a barrier before them (349); block
// rows read their sums from a list of their own instead of a select per score (335); the unpacking in short loops (329); V
// in steps and one sum per row (323); scores in one read of tensor memory (320; 321 with all that keeps rows next to the
// largest number and references far below 0 right).  Slower were query rows on M (1.9 us a
// page), four groups of softmax warps, sixteen rows each, that do not wait for each other (+11 %), weights published, barriers asked
// for or parameters looked up a page ahead (+5 to 10 %), a factor common to all rows beside one each (+27 %).
//
// Warps (28, one thread block per SM):
//   0      bulk copies, a page of one kv head (4 (32 d + 256) contiguous bytes) per stage of the ring
//   1, 2   issue S^T and O^T products
//   4-7    query rows into shared memory (f16, one power of two per item); K codes -> tensor memory
//   8-11   V codes -> tensor memory
//   12-27  four threads per key, sixteen rows each: scores, e, its sums, weights as f16 into shared memory (second
//          operand); O^T out
// The block's own rows are one more page, whose K and V the code warps bring as f16 with a power of two per row instead.
// Every wait is bounded; an expired wait sets SPACE_ST_TIMEOUT, no role leaves its loop early (the named barriers stay
// matched), and the block drains and exits.
#include "kvq_attn.cuh"

namespace {
using namespace kvq;

constexpr int SOFT_WARPS = 16, SOFT = 32 * SOFT_WARPS;          // four threads per key
constexpr int THREADS = 12 * 32 + SOFT;
constexpr int TILE = SPACE_PAGE_SIZE;
constexpr int NP = 4;                                // sixteens of query rows of an item
constexpr int SHARE_COST = 5;                        // fixed cost of an item, in pages (8 us against 1.45 us a page)
constexpr int K_WARP0 = 4, V_WARP0 = 8, SOFT_WARP0 = 12;
constexpr float W_SHIFT = 2.f;                       // weights of a new reference lie in [2^2, 2^3) (below 2^-14 f16 has fewer bits)
// Where references are set, the scores that they come from are taken without any and then once more with them, which rounds
// otherwise: by 2^-22 of a score's largest term, 16 times the key's step times the score's factors at most.  Below this limit
// that is 4, which leaves the weights below 2^7; for steps beyond it the reference comes off the very same score.
constexpr float K_CAREFUL = 0x1p20f;
constexpr float X_LIMIT = 16.f;                      // a row's reference moves when a score exceeds it by 2^16

template <int DH>
struct Smem {
  static constexpr int N = 16 * NP;                          // query rows of an item (with padding)
  static constexpr int STAGES = DH == 128 ? 8 : 12;
  static constexpr int PAGE = Fmt<DH>::HEAD;
  static constexpr int Q_BYTES = N * DH * 2;                 // DH / 64 blocks [N][64] f16, 128-byte swizzle
  static constexpr int P_BYTES = TILE * 128;                 // [key][64 query rows] f16, 128-byte swizzle
  static constexpr int Q_OFF = 0;                            // two buffers each
  static constexpr int P_OFF = 2 * Q_BYTES;
  static constexpr int RING_OFF = P_OFF + 2 * P_BYTES;
  static constexpr int RC_OFF = RING_OFF + STAGES * PAGE;    // [N/2] {sum, sum, -m, -m} of query rows 2i, 2i + 1
  static constexpr int RC0_OFF = RC_OFF + 32 * 16;           // the same without references
  static constexpr int VINV_OFF = RC0_OFF + 32 * 16;         // [N] 2^(m - R + W_SHIFT)
  static constexpr int MREF_OFF = VINV_OFF + 256;            // [N] m
  static constexpr int RREF_OFF = MREF_OFF + 256;            // [N] R - m (m can be too large for the difference to show in R)
  static constexpr int FQ_OFF = RREF_OFF + 256;              // [N] factors
  static constexpr int GO_OFF = FQ_OFF + 256;                // [N] factors
  static constexpr int VSPAN_OFF = GO_OFF + 256;             // [2][4]
  static constexpr int ROFF_OFF = VSPAN_OFF + 32;            // [64]
  static constexpr int XQ_OFF = ROFF_OFF + 256;                // [4][64] per quarter
  static constexpr int XZ_OFF = XQ_OFF + 1024;               // [4][64]
  static constexpr int QSUM_OFF = XZ_OFF + 1024;             // [2][64] c * sum of a query row
  static constexpr int QTOP_OFF = QSUM_OFF + 512;            // [2][4] largest exponents, then [2] c with the power of two undone
  static constexpr int PAR_OFF = QTOP_OFF + 64;              // [STAGES][2][64] block rows' K and V factors
  static constexpr int BAD_OFF = PAR_OFF + STAGES * 512;     // [STAGES] page outside the pool
  static constexpr int BAR_OFF = (BAD_OFF + STAGES * 4 + 15) / 16 * 16;
  static constexpr int N_BARS = 2 * STAGES + 24;
  static constexpr int MISC_OFF = BAR_OFF + (N_BARS * 8 + 15) / 16 * 16;
  static constexpr int OVER_OFF = MISC_OFF + 16;             // [2] the last page (of those that ask) whose scores pass a limit
  static constexpr int LIMIT_OFF = MISC_OFF + 24;            // {score that the references move at, the largest vinv}
  static constexpr int RATIO_OFF = MISC_OFF + 32;            // [2][TILE] f16: lo / step of a page's V rows, times 2^-9
  static constexpr int MASK_OFF = RATIO_OFF + 2 * TILE * 2;             // [64] Eq. 5
  static constexpr int TABLE_OFF = MASK_OFF + SPACE_MAX_ROWS * 8;            // prefix[max_batch + 1], seq_len[max_batch]
  static constexpr int V_PITCH = DH * 2 + 16;                // bytes: the block's V rows as f16, in a stage
  static_assert(SPACE_MAX_ROWS * V_PITCH <= PAGE, "the block's V rows fit a stage");
  static_assert(TABLE_OFF + 129 * 4 + 128 * 4 <= 227 * 1024, "shared-memory plan too large");
};

__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, %0;" ::"n"(SOFT) : "memory"); }
__device__ __forceinline__ void k_sync() { asm volatile("bar.sync 2, 128;" ::: "memory"); }
__device__ __forceinline__ void v_sync() { asm volatile("bar.sync 3, 128;" ::: "memory"); }
template <int R> __device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R> __device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }

__device__ __forceinline__ void tmem_ld4(uint32_t a, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];" : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t a, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
                 "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]) : "r"(a) : "memory");
}
__device__ __forceinline__ void tmem_st4(uint32_t a, const float* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]) : "memory");
}
// 16 lanes x 32 columns: lane (n, t) of the warp holds of every eight columns {2t, 2t + 1} of rows n and n + 8
__device__ __forceinline__ void tmem_st_frag4(uint32_t a, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(a), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
               "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// Instruction descriptor: f16 x f16 -> f32, M = 128, N = n; first operand K-major, second one K-major or (b_mn) not.
__device__ __forceinline__ constexpr uint32_t instr_desc(int n, int b_mn) {
  return (1u << 4) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
}
// Masked codes as f16 (u 2^-24, or u 2^-20 for bits 4 .. 7 of each half) to (u + lo / step) 2^-9, rounded once.
__device__ __forceinline__ uint32_t h2fma(uint32_t x, uint32_t a, uint32_t c) {
  const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&c));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t value_even(uint32_t x, uint32_t r) { return h2fma(x & 0x000F000Fu, 0x78007800u, r); }    // 2^15
__device__ __forceinline__ uint32_t value_odd(uint32_t x, uint32_t r) { return h2fma(x & 0x00F000F0u, 0x68006800u, r); }     // 2^11
// Four values per lane joined over the warp: every lane ends with the one of column 2 (lane >> 4) + ((lane >> 3) & 1).
template <class J>
__device__ __forceinline__ float warp_join4(const float* v, int lane, J join) {
  const bool up = lane & 16, up2 = lane & 8;
  const float a = join(up ? v[2] : v[0], __shfl_xor_sync(0xFFFFFFFFu, up ? v[0] : v[2], 16));
  const float b = join(up ? v[3] : v[1], __shfl_xor_sync(0xFFFFFFFFu, up ? v[1] : v[3], 16));
  float r = join(up2 ? b : a, __shfl_xor_sync(0xFFFFFFFFu, up2 ? a : b, 8));
  r = join(r, __shfl_xor_sync(0xFFFFFFFFu, r, 4));
  r = join(r, __shfl_xor_sync(0xFFFFFFFFu, r, 2));
  return join(r, __shfl_xor_sync(0xFFFFFFFFu, r, 1));
}

// The items of a block's share, in order: every role walks them for itself.
struct Walk {
  uint32_t cur, end;
  int b, it;                                         // item h * n_rb + block of query rows
  int L, t0, t1;                                     // pages [t0, t1) of it; cached rows (-1: the sequence does not fit)
  bool opens;                                        // the share begins with this item
  __device__ __forceinline__ int cached() const { return (max(L, 0) + TILE - 1) / TILE; }   // that page: the block's own rows
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
      cur += n;
      t0 = max(x0 - SHARE_COST, 0); t1 = x0 + n - SHARE_COST;
      if (t1 > t0) return true;                      // (else only the cost of starting)
    }
    return false;
  }
};

template <int DH>
__global__ void __launch_bounds__(THREADS, 1) kvq_attn_tc_kernel(const __grid_constant__ Params p, int max_batch) {
  using F = Fmt<DH>;
  using S = Smem<DH>;
  constexpr int N = S::N, STAGES = S::STAGES;
  extern __shared__ __align__(1024) unsigned char sm[];
  const uint32_t base = smem_u32(sm), bar0 = base + S::BAR_OFF;
  auto BAR = [&](int i) { return bar0 + 8u * i; };
  constexpr int FULL = 0, EMPTY = STAGES, KTF = 2 * STAGES, KTE = KTF + 2, VTF = KTF + 4, VTE = KTF + 6, SF = KTF + 8, SE = KTF + 10,
                PF = KTF + 12, PE = KTF + 14, QF = KTF + 16, QE = KTF + 18, BLK = KTF + 20, DRAIN = KTF + 22, OVER = KTF + 23;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + S::MISC_OFF);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::MISC_OFF + 4);
  volatile int* last_flag = reinterpret_cast<volatile int*>(sm + S::MISC_OFF + 8);
  uint32_t* prefix = reinterpret_cast<uint32_t*>(sm + S::TABLE_OFF);
  int* seq_len = reinterpret_cast<int*>(prefix + max_batch + 1);
  volatile int* bad = reinterpret_cast<volatile int*>(sm + S::BAD_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    *abort_flag = (base & 1023u) ? 1 : 0;            // swizzled tiles need a 1024-byte aligned base
    for (int i = 0; i < 2; ++i) reinterpret_cast<volatile uint32_t*>(sm + S::OVER_OFF)[i] = 0;
    for (int s = 0; s < STAGES; ++s) { mbar_init(BAR(FULL + s), 1); mbar_init(BAR(EMPTY + s), 8 + SOFT_WARPS); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(BAR(KTF + i), 4); mbar_init(BAR(KTE + i), 1); mbar_init(BAR(VTF + i), 4); mbar_init(BAR(VTE + i), 1);
      mbar_init(BAR(SF + i), 1); mbar_init(BAR(SE + i), SOFT_WARPS); mbar_init(BAR(PF + i), SOFT_WARPS); mbar_init(BAR(PE + i), 1);
      mbar_init(BAR(QF + i), 4); mbar_init(BAR(QE + i), 2); mbar_init(BAR(BLK + i), 8);
    }
    mbar_init(BAR(DRAIN), 1);
    mbar_init(BAR(OVER), SOFT_WARPS);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (threadIdx.x < SPACE_MAX_ROWS) reinterpret_cast<uint64_t*>(sm + S::MASK_OFF)[threadIdx.x] = p.mask[threadIdx.x];
  if (warp == 3) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  if (warp == 0) {
    // the list's running sums, as in kvq_attn.cu
    uint32_t carry = 0;
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
  const uint32_t tmem = *tmem_slot;
  // columns: S^T two buffers, O^T, two buffers each of the unpacked K and V pages
  const uint32_t TM_S = tmem, TM_O = tmem + 128, TM_K = tmem + 192, TM_V = tmem + 320;
  const Cut cut(prefix[p.B], p.n_groups);
  Walk wk;
  const bool mine = blockIdx.x < cut.NG;
  const uint32_t share0 = mine ? cut.begin(blockIdx.x) : 0;
  wk.b = 0; wk.cur = share0;
  wk.end = mine ? cut.begin(blockIdx.x + 1) : 0;
  auto next = [&] { return wk.next(prefix, seq_len, p.has_new, share0); };
  uint32_t g = 0, items = 0;                         // pages and items so far
  // (a failed wait leaves no loop: what waits later returns at once, and the counts of arrivals stay matched)
  auto hold = [&](int bar, uint32_t use, int site) { return wait(BAR(bar), use & 1, abort_flag, p.err, site); };

  if (warp < 4) {
    regs_dec<24>();
    if (warp == 0) {
      // ================= bulk copies =========================================
      if (elect_one()) {
        bool ok = true;
        while (ok && next()) {
          const int32_t* table = p.cache.page_table + (int64_t)wk.b * p.cache.pages_per_seq;
          const char* head = p.cache.pool + (int64_t)(wk.it / p.n_rt) * p.cache.head_stride;
          const int Tc = wk.cached();
          for (int t = wk.t0; t < wk.t1; ++t, ++g) {
            const uint32_t s = g % STAGES;
            const int pg = t < Tc ? __ldg(table + t) : -1;
            if (g >= STAGES) ok = hold(EMPTY + s, g / STAGES - 1, 1);
            if (!ok) break;
            const bool good = pg >= 0 && pg < p.cache.n_pages;
            bad[s] = !good;
            if (good) {
              mbar_expect_tx(BAR(FULL + s), S::PAGE);
              asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                           ::"r"(base + S::RING_OFF + s * S::PAGE), "l"(head + (int64_t)pg * p.cache.page_stride), "r"(S::PAGE), "r"(BAR(FULL + s)) : "memory");
            } else {
              if (t < Tc && p.status) atomicOr(p.status + wk.b, SPACE_ST_BAD_PAGE);
              mbar_arrive(BAR(FULL + s));
            }
          }
        }
        // every copy has landed before the block may exit
        for (uint32_t i = g > STAGES ? g - STAGES : 0; i < g; ++i) mbar_drain_bounded(BAR(FULL + i % STAGES), (i / STAGES) & 1, WAIT_NS);
      }
    } else if (warp == 1) {
      // ================= S^T products ========================================
      if (elect_one()) {
        const uint64_t qdesc0 = smem_desc(base + S::Q_OFF, 16, 1024);
        bool ok = true;
        while (ok && next()) {
          const uint32_t qb = items & 1;
          ok = hold(QF + qb, items >> 1, 2);
          const uint64_t qd = qdesc0 + (uint64_t)((qb * S::Q_BYTES) >> 4);
          for (int t = wk.t0; t < wk.t1 && ok; ++t, ++g) {
            const uint32_t buf = g & 1;
            ok = hold(KTF + buf, g >> 1, 3);
            if (ok && g >= 2) ok = hold(SE + buf, (g - 2) >> 1, 4);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < DH / 16; ++kk)
              mma_ts(TM_S + buf * 64, TM_K + buf * 64 + kk * 8, qd + (uint64_t)(((kk >> 2) * (N * 128) + (kk & 3) * 32) >> 4), instr_desc(N, 0), kk > 0);
            tc_commit(BAR(SF + buf));
            tc_commit(BAR(KTE + buf));
            if (t == wk.t1 - 1) tc_commit(BAR(QE + qb));
          }
          ++items;
        }
        tc_commit(BAR(DRAIN));                       // all products done before tensor memory is released
        mbar_drain_bounded(BAR(DRAIN), 0, WAIT_NS);
      }
    } else if (warp == 2) {
      // ================= O^T products ========================================
      if (elect_one()) {
        const uint64_t pdesc0 = smem_desc(base + S::P_OFF, TILE * 128, 1024);
        bool ok = true;
        while (ok && next()) {
          for (int t = wk.t0; t < wk.t1 && ok; ++t, ++g) {
            const uint32_t buf = g & 1;
            ok = hold(VTF + buf, g >> 1, 5);
            if (ok) ok = hold(PF + buf, g >> 1, 6);
            if (!ok) break;
            tc_fence_after();
            const uint64_t pd = pdesc0 + (uint64_t)((buf * S::P_BYTES) >> 4);
#pragma unroll
            for (int kk = 0; kk < TILE / 16; ++kk)
              mma_ts(TM_O, TM_V + buf * 64 + kk * 8, pd + (uint64_t)((kk * 2048) >> 4), instr_desc(N, 1), (t == wk.t0 && kk == 0) ? 0u : 1u);
            tc_commit(BAR(VTE + buf));
            tc_commit(BAR(PE + buf));
          }
        }
        // (the last of these is waited for by the softmax threads; after a wait that ran out, here)
        if (*abort_flag) {
          for (uint32_t i = g > 2 ? g - 2 : 0; i < g; ++i) mbar_drain_bounded(BAR(VTE + (i & 1)), (i >> 1) & 1, WAIT_NS);
        }
      }
    }
  } else if (warp < V_WARP0) {
    regs_dec<64>();
    // ================= query rows, K codes -> tensor memory ====================
    const int w = warp - K_WARP0, n = lane >> 2, t4 = lane & 3;
    float* qsum = reinterpret_cast<float*>(sm + S::QSUM_OFF);
    uint32_t* qtop = reinterpret_cast<uint32_t*>(sm + S::QTOP_OFF);
    float* qc = reinterpret_cast<float*>(sm + S::QTOP_OFF + 32);
    float* par = reinterpret_cast<float*>(sm + S::PAR_OFF);
    while (next()) {
      const uint32_t qb = items & 1;
      const int h = wk.it / p.n_rt, rb = wk.it - h * p.n_rt, Tc = wk.cached();
      float c;                                       // scale, with the query rows' power of two undone
      {
        // (twice over the rows, in loops: what runs once per item should not push the pages' loops out of the
        // instruction cache; the second time they come out of the first-level cache)
        constexpr int ROWS = N / 4;                  // of this warp
        auto row = [&](int r, bool& there) {
          int i, hq;
          row_of(p, h, rb * N + w * ROWS + r, i, hq);
          there = r < ROWS && i < p.n_q;
          return reinterpret_cast<const uint4*>(p.q + (int64_t)wk.b * p.q_sb + (int64_t)i * p.q_sr + (int64_t)hq * p.q_sh) + t4 * (DH / 32);
        };
        uint32_t top = 0;
#pragma unroll 1
        for (int r = n; r < ROWS; r += 8) {
          bool there;
          const uint4* src = row(r, there);
#pragma unroll
          for (int j = 0; j < DH / 32; ++j) {
            const uint4 v = there ? src[j] : make_uint4(0, 0, 0, 0);
            const uint32_t m = max_bits(v);
            top = max(top, m);
            if (m >= 0x7F80u) top = 0x7F80u;
          }
        }
        top >>= 7;
        if (top >= 255u) {                           // something is not finite: the largest of what is
          top = 0;
#pragma unroll 1
          for (int r = n; r < ROWS; r += 8) {
            bool there;
            const uint16_t* src = reinterpret_cast<const uint16_t*>(row(r, there));
#pragma unroll 1
            for (int j = 0; j < DH / 4 && there; ++j) {
              const uint32_t e = (src[j] >> 7) & 0xFFu;
              if (e < 255u) top = max(top, e);
            }
          }
        }
        __syncwarp();
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (items >= 2) hold(QE + qb, (items >> 1) - 1, 7);
        if (lane == 0) qtop[qb * 4 + w] = top;
        k_sync();
        top = max(max(qtop[qb * 4], qtop[qb * 4 + 1]), max(qtop[qb * 4 + 2], qtop[qb * 4 + 3]));
        const int e = top ? min(max(8 - ((int)top - 127), -100), 100) : 0;   // largest element in [2^8, 2^9)
        const float f = pow2(e), f16th = f * 0.0625f;
        c = p.c * pow2(-e);
        if (threadIdx.x == K_WARP0 * 32) qc[qb] = c;
#pragma unroll 1
        for (int r0 = 0; r0 < ROWS; r0 += 8) {
          bool there;
          const uint4* src = row(r0 + n, there);
          const int r = w * ROWS + r0 + n;
          float sum = 0.f;
#pragma unroll
          for (int j = 0; j < DH / 32; ++j) {
            const uint4 v = there ? src[j] : make_uint4(0, 0, 0, 0);
            sum += ((bf_lo(v.x) + bf_hi(v.x)) + (bf_lo(v.y) + bf_hi(v.y))) + ((bf_lo(v.z) + bf_hi(v.z)) + (bf_lo(v.w) + bf_hi(v.w)));
#pragma unroll
            for (int half = 0; half < 2; ++half) {   // k-step 2 j + half: channels 8 j + {0, 4 | 1, 5} or {2, 6 | 3, 7}
              const int ks = 2 * j + half;
              const uint32_t lo = half ? v.y : v.x, hi = half ? v.w : v.z;
              const uint32_t a0 = pack_h(bf_lo(lo) * f, bf_lo(hi) * f), a1 = pack_h(bf_hi(lo) * f16th, bf_hi(hi) * f16th);
              const uint32_t at = base + S::Q_OFF + qb * S::Q_BYTES + (ks >> 2) * (N * 128) + r * 128 + (((2 * (ks & 3) + (t4 >> 1)) ^ (r & 7)) << 4) + (t4 & 1) * 8;
              if (r0 + n < ROWS) asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(at), "r"(a0), "r"(a1) : "memory");
            }
          }
          sum = quad_sum(sum) * p.c;
          if (t4 == 0 && r0 + n < ROWS) qsum[qb * 64 + r] = sum;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(QF + qb));
      }
      for (int t = wk.t0; t < wk.t1; ++t, ++g) {
        const uint32_t s = g % STAGES, buf = g & 1;
        hold(FULL + s, g / STAGES, 8);
        if (g >= 2) hold(KTE + buf, (g - 2) >> 1, 9);
        tc_fence_after();
        const uint32_t dst = TM_K + buf * 64 + ((uint32_t)(32 * w) << 16);
        const bool own = t >= Tc;                    // the block's own rows (or no rows at all)
        if (!own) {
          const uint32_t blk = base + S::RING_OFF + s * S::PAGE + w * F::BLOCK;
#pragma unroll 1
          for (int i = 0; i < 2 * (DH / 64); ++i) {  // sixteen keys, four k-steps
            const int i16 = i & 1, jj = i >> 1;
            const uint32_t at = blk + (16 * i16 + n) * (DH / 2) + t4 * (DH / 8) + 8 * jj;
            const uint2 x = lds64(at), y = lds64(at + 8 * (DH / 2));
            uint32_t r[16];
#pragma unroll
            for (int k = 0; k < 4; ++k) {            // eight columns: pairs 2 (k % 2), + 1 of word k / 2
              const uint32_t xw = k / 2 ? x.y : x.x, yw = k / 2 ? y.y : y.x;
              const uint32_t a = (k & 1) ? xw >> 8 : xw, d = (k & 1) ? yw >> 8 : yw;
              r[4 * k] = a & 0x000F000Fu; r[4 * k + 1] = a & 0x00F000F0u;
              r[4 * k + 2] = d & 0x000F000Fu; r[4 * k + 3] = d & 0x00F000F0u;
            }
            tmem_st_frag4(dst + ((uint32_t)(16 * i16) << 16) + 32 * jj, r);
          }
        } else if (p.has_new && wk.L >= 0 && 32 * w < p.n_q) {
#pragma unroll 1
          for (int i16 = 0; i16 < 2; ++i16) {
            uint4 raw[2][DH / 32];
            float f[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int key = 32 * w + 16 * i16 + 8 * i + n;
              const uint4* src = reinterpret_cast<const uint4*>(p.kn + (int64_t)wk.b * p.n_sb + (int64_t)key * p.n_sr + (int64_t)h * p.n_sh) + t4 * (DH / 32);
              uint32_t top = 0;
#pragma unroll
              for (int j = 0; j < DH / 32; ++j) {
                raw[i][j] = key < p.n_q ? src[j] : make_uint4(0, 0, 0, 0);
                top = max(top, top_bits(raw[i][j]));
              }
              top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
              top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
              const int e = max(min(127 - (int)(top >> 7), 120), -126);
              f[i] = pow2(e);
              if (t4 == 0) par[s * 128 + key] = fminf(pow2(-e) * c, 1e38f);
            }
#pragma unroll
            for (int jj = 0; jj < DH / 64; ++jj) {
              uint32_t r[16];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                  const uint4 v = raw[i][2 * jj + k / 2];
                  const uint32_t lo = (k & 1) ? v.y : v.x, hi = (k & 1) ? v.w : v.z;
                  r[4 * k + 2 * i] = pack_h(bf_lo(lo) * f[i], bf_lo(hi) * f[i]);
                  r[4 * k + 2 * i + 1] = pack_h(bf_hi(lo) * (f[i] * 16.f), bf_hi(hi) * (f[i] * 16.f));
                }
              }
              tmem_st_frag4(dst + ((uint32_t)(16 * i16) << 16) + 32 * jj, r);
            }
          }
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(BAR(KTF + buf));
          mbar_arrive(BAR(EMPTY + s));
          if (own) mbar_arrive(BAR(BLK + buf));
        }
      }
      ++items;
    }
  } else if (warp < SOFT_WARP0) {
    regs_dec<64>();
    // ================= V codes -> tensor memory ================================
    const int w = warp - V_WARP0;
    float* par = reinterpret_cast<float*>(sm + S::PAR_OFF);
    while (next()) {
      const int h = wk.it / p.n_rt, Tc = wk.cached();
      for (int t = wk.t0; t < wk.t1; ++t, ++g) {
        const uint32_t s = g % STAGES, buf = g & 1, stage = base + S::RING_OFF + s * S::PAGE;
        hold(FULL + s, g / STAGES, 10);
        const bool own = t >= Tc;
        __half* ratio = reinterpret_cast<__half*>(sm + S::RATIO_OFF) + buf * TILE;
        if (!own) {
          const uint32_t vp = lds32(stage + w * F::BLOCK + F::V_PAR + lane * 4);
          const bool gone = bad[s] != 0 || t * TILE + 32 * w + lane >= wk.L;   // (such a row may hold anything; its weights are 0)
          ratio[32 * w + lane] = __float2half_rn(gone ? 0.f : __fdividef(bf_hi(vp), bf_lo(vp)) * 0x1p-9f);
          v_sync();
        }
        if (g >= 2) hold(VTE + buf, (g - 2) >> 1, 11);
        tc_fence_after();
        const uint32_t dst = TM_V + buf * 64 + ((uint32_t)(32 * w) << 16);
        if (!own) {
          if (32 * w < DH) {
            const uint32_t rat = smem_u32(ratio) + (lane & 3) * 4;
#pragma unroll 1
            for (int r2 = 0; r2 < 2; ++r2) {         // two blocks of 32 rows, 32 columns
              uint32_t lo[16], hi[16];
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const uint4 v = lds128(stage + (2 * r2 + k) * F::BLOCK + F::CODES + 512 * w + 16 * lane);
                const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                  for (int e = 0; e < 2; ++e) {      // channels n and n + 8 of each 16: pairs 0 and 1 (2 and 3)
                    const uint32_t u = x[2 * a + e], u8 = u >> 8, r = lds32(rat + ((2 * r2 + k) * 32 + 16 * a + 8 * e) * 2);
                    lo[8 * k + 4 * a + e] = value_even(u, r); lo[8 * k + 4 * a + 2 + e] = value_odd(u, r);
                    hi[8 * k + 4 * a + e] = value_even(u8, r); hi[8 * k + 4 * a + 2 + e] = value_odd(u8, r);
                  }
              }
              tmem_st_frag4(dst + 32 * r2, lo);
              tmem_st_frag4(dst + (16u << 16) + 32 * r2, hi);
            }
          }
        } else {
          // the block's V rows as f16, largest element of a row in [1, 2), into the stage; eight channels a lane
          constexpr int LANES = DH / 8;
#pragma unroll 2
          for (int i = 0; i < 16 * LANES / 32; ++i) {
            const int key = 16 * w + i * (32 / LANES) + lane / LANES;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (p.has_new && wk.L >= 0 && key < p.n_q)
              v = *(reinterpret_cast<const uint4*>(p.vn + (int64_t)wk.b * p.n_sb + (int64_t)key * p.n_sr + (int64_t)h * p.n_sh) + lane % LANES);
            uint32_t top = top_bits(v);
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            const int e = min(max((int)(top >> 7) - 127, -110), 126);
            const float f = pow2(-e);
            const uint4 hv = make_uint4(pack_h(bf_lo(v.x) * f, bf_hi(v.x) * f), pack_h(bf_lo(v.y) * f, bf_hi(v.y) * f),
                                        pack_h(bf_lo(v.z) * f, bf_hi(v.z) * f), pack_h(bf_lo(v.w) * f, bf_hi(v.w) * f));
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};"
                         ::"r"(stage + key * S::V_PITCH + (lane % LANES) * 16), "r"(hv.x), "r"(hv.y), "r"(hv.z), "r"(hv.w) : "memory");
            if (lane % LANES == 0) par[s * 128 + 64 + key] = pow2(e) * 0x1p-9f;   // (as the cache's values)
          }
          v_sync();
          if (32 * w < DH) {
#pragma unroll 1
            for (int c = 0; c < 2; ++c) {            // sixteen channels
              uint32_t r[16];
#pragma unroll
              for (int k = 0; k < 4; ++k) {          // sixteen keys
                const uint32_t at = stage + (16 * k + 8 * (lane >> 4) + (lane & 7)) * S::V_PITCH + (32 * w + 16 * c) * 2 + ((lane >> 3) & 1) * 16;
                asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                             : "=r"(r[4 * k]), "=r"(r[4 * k + 2]), "=r"(r[4 * k + 1]), "=r"(r[4 * k + 3]) : "r"(at) : "memory");
              }
              tmem_st_frag4(dst + ((uint32_t)(16 * c) << 16), r);
#pragma unroll
              for (int k = 0; k < 16; ++k) r[k] = 0u;                            // a page has 128 rows, the block 64 at most
              tmem_st_frag4(dst + ((uint32_t)(16 * c) << 16) + 32, r);
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the next copy into this stage comes after
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(BAR(VTF + buf));
          mbar_arrive(BAR(EMPTY + s));
          if (own) mbar_arrive(BAR(BLK + buf));
        }
      }
    }
  } else {
    regs_inc<88>();
    // ================= softmax, output ==========================================
    constexpr int NC = 4 * NP;                       // query rows of a thread
    static_assert(NC == 16, "one read of tensor memory");
    const int quarter = warp & 3, part = (warp - SOFT_WARP0) >> 2;
    const int kl = quarter * 32 + lane;              // key of the page; channel in the epilogue
    const int sidx = part * 128 + kl, col0 = part * NC;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    // the key's place in the order in which the unpacked V lies: 16 a + 4 t + 2 e + h within 32 rows
    const int kp_row = (kl & 0x70) | ((kl & 6) << 1) | ((kl & 8) >> 2) | (kl & 1);
    const uint32_t prow = base + S::P_OFF + kp_row * 128, swz = (uint32_t)(kp_row & 7);
    const uint32_t rc_at = base + S::RC_OFF + col0 * 8, vinv_at = base + S::VINV_OFF + col0 * 4;
    float* rcf = reinterpret_cast<float*>(sm + S::RC_OFF);
    float* vinv = reinterpret_cast<float*>(sm + S::VINV_OFF);
    float* mref = reinterpret_cast<float*>(sm + S::MREF_OFF);
    float* rref = reinterpret_cast<float*>(sm + S::RREF_OFF);
    float* fq = reinterpret_cast<float*>(sm + S::FQ_OFF);
    float* go = reinterpret_cast<float*>(sm + S::GO_OFF);
    float* xq = reinterpret_cast<float*>(sm + S::XQ_OFF);
    float* xz = reinterpret_cast<float*>(sm + S::XZ_OFF);
    float* vspan = reinterpret_cast<float*>(sm + S::VSPAN_OFF);   // [2][4] largest and smallest V step of a quarter's keys
    int* roff = reinterpret_cast<int*>(sm + S::ROFF_OFF);         // [N] where a query row's output begins, in elements
    volatile float* limit = reinterpret_cast<volatile float*>(sm + S::LIMIT_OFF);
    const float* qsum = reinterpret_cast<const float*>(sm + S::QSUM_OFF);
    const volatile float* qc = reinterpret_cast<const volatile float*>(sm + S::QTOP_OFF + 32);
    const float* par = reinterpret_cast<const float*>(sm + S::PAR_OFF);
    const uint64_t* masks = reinterpret_cast<const uint64_t*>(sm + S::MASK_OFF);
    auto fmax2 = [](float a, float b) { return fmaxf(a, b); };
    auto fsum2 = [](float a, float b) { return a + b; };
    // every column joined over the warp's keys, into to[quarter]
    auto over_keys = [&](const float* v, float* to, auto join) {
#pragma unroll
      for (int i = 0; i < NC; i += 4) {
        const float r = warp_join4(v + i, lane, join);
        if ((lane & 7) == 0) to[quarter * 64 + col0 + i + (lane >> 3)] = r;
      }
    };
    auto fmin2 = [](float a, float b) { return fminf(a, b); };
    auto of_quarters_v = [&](const float* v, auto join) { return join(join(v[0], v[1]), join(v[2], v[3])); };
    auto of_quarters = [&](const float* v, auto join) { return join(join(v[sidx], v[64 + sidx]), join(v[128 + sidx], v[192 + sidx])); };
    uint32_t asked = 0;                              // pages whose scores were held against the limits so far
    volatile uint32_t* over_at = reinterpret_cast<volatile uint32_t*>(sm + S::OVER_OFF);
    uint32_t blocks = 0;                             // pages of block rows so far, per buffer
    while (next()) {
      const uint32_t qb = items & 1;
      const int h = wk.it / p.n_rt, rb = wk.it - h * p.n_rt, Tc = wk.cached();
      hold(QF + qb, items >> 1, 12);
      ++items;
      if (sidx < N) {
        float* r = rcf + 4 * (sidx >> 1) + (sidx & 1);
        r[0] = r[128] = qsum[qb * 64 + sidx]; r[2] = r[130] = 0.f;
        int qi, hq;
        row_of(p, h, rb * N + sidx, qi, hq);
        roff[sidx] = (qi * p.H_q + hq) * DH;
        mref[sidx] = rref[sidx] = -CUDART_INF_F;
        vinv[sidx] = 0x1p126f;
      }
      const float c24 = qc[qb] * 16777216.f;         // undoes the codes' 2^-24
      uint64_t l[NC / 2];
#pragma unroll
      for (int i = 0; i < NC / 2; ++i) l[i] = pack2(0.f, 0.f);
      soft_sync();
      if (sidx == 0) mbar_arrive(BAR(QE + qb));      // (with the last S^T product: the query buffer is free)
      const int r0 = rb * N, rows = min(N, p.n_q * p.G - r0);
      for (int t = wk.t0; t < wk.t1; ++t, ++g) {
        const uint32_t s = g % STAGES, buf = g & 1;
        const bool first = t == wk.t0, own = t >= Tc;
        // ---- this key's step and lowest value
        hold(FULL + s, g / STAGES, 13);
        float k1, k0, v1;
        uint32_t kp = 0;
        bool gone;
        if (!own) {
          const uint32_t blk = base + S::RING_OFF + s * S::PAGE + quarter * F::BLOCK + lane * 4;
          gone = bad[s] != 0 || t * TILE + kl >= wk.L;
          kp = gone ? 0u : lds32(blk + F::K_PAR);
          const uint32_t vp = gone ? 0u : lds32(blk + F::V_PAR);
          k1 = bf_lo(kp) * c24; k0 = bf_hi(kp); v1 = bf_lo(vp);
        } else {
          hold(BLK + buf, blocks >> (16 * buf), 14);
          blocks += 1u << (16 * buf);                // (only the low bit of each count is looked at)
          blocks &= 0x00010001u;
          gone = !p.has_new || wk.L < 0 || kl >= p.n_q;
          k1 = gone ? 0.f : par[s * 128 + (kl & 63)]; k0 = 0.f; v1 = gone ? 0.f : par[s * 128 + 64 + (kl & 63)];
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(EMPTY + s));
        hold(SF + buf, g >> 1, 15);
        tc_fence_after();
        const bool large = bf_lo(kp) * c24 > K_CAREFUL;                         // (2^-64 of its scores are taken first)
        const bool plain = !own && !__any_sync(0xFFFFFFFFu, gone || large);    // every row sees every key of this warp, none is large
        const bool careful = own || (!plain && __any_sync(0xFFFFFFFFu, large));
        if (!plain && large) { k1 = bf_lo(kp) * 0x1p-64f * c24; k0 *= 0x1p-64f; }
        // scores that settle are taken without references; where they are held to the range of numbers, references come after that
        uint32_t rc_page = rc_at + (careful ? S::RC0_OFF - S::RC_OFF : 0);
        float x[NC];
        uint32_t hw[NC / 2];
        // `fresh`: the references have to come from this page; `settled`: they have
        bool fresh = first, settled = first;
#pragma unroll 1
        for (;;) {
          // ---- scores less the rows' references, for this key and its rows
          tmem_ld16(TM_S + buf * 64 + lanes + col0, x);
          tmem_wait_ld();
          {
            const uint64_t k1p = pack2(k1, k1), k0p = pack2(k0, k0);
#pragma unroll
            for (int i = 0; i < NC / 2; ++i) {
              uint64_t sum, ref;
              asm volatile("ld.shared.v2.b64 {%0,%1}, [%2];" : "=l"(sum), "=l"(ref) : "r"(rc_page + 16 * i));
              unpack2(fma2(pack2(x[2 * i], x[2 * i + 1]), k1p, fma2(k0p, sum, ref)), x[2 * i], x[2 * i + 1]);
            }
          }
          if (careful) {                             // (rows next to the largest number: a score stays one)
            uint32_t see = own ? 0u : ~0u;           // (a loop: this code runs once an item, and is fetched for it)
            if (own && !gone) {
#pragma unroll 1
              for (int i = 0; i < NC; ++i)
                if (col0 + i < rows) see |= (uint32_t)((masks[(r0 + col0 + i) >> p.gsh] >> kl) & 1ull) << i;
            }
#pragma unroll
            for (int i = 0; i < NC; ++i) {
              const float y = clamp_score(large ? x[i] * 0x1p64f : x[i]) + (fresh ? 0.f : rcf[4 * ((col0 + i) >> 1) + 2 + (i & 1)]);
              x[i] = !gone && ((see >> i) & 1u) ? y : -CUDART_INF_F;
            }
          } else if (!plain && gone) {
#pragma unroll
            for (int i = 0; i < NC; ++i) x[i] = -CUDART_INF_F;
          }
          if (!fresh) {
            if (!settled) {
              // do scores or weights pass the limits?  (the weights by a bound: the largest score, the largest vinv; any score
              // does while a row has no reference, or one far below 0, which would cost the scores their bits)
              float a = fmaxf(x[0], x[1]), b = fmaxf(x[2], x[3]);
#pragma unroll
              for (int i = 4; i < NC; i += 4) { a = max3(a, x[i], x[i + 1]); b = max3(b, x[i + 2], x[i + 3]); }
              a = fmaxf(a, b);
              ++asked;
              const uint2 lim = lds64(base + S::LIMIT_OFF);
              if (a > __uint_as_float(lim.x) || fast_exp2(a) * v1 * __uint_as_float(lim.y) > W_LIMIT) over_at[asked & 1] = asked;
              __syncwarp();
              if (lane == 0) mbar_arrive(BAR(OVER));
            }
            // ---- e, and the weights e step as f16
            const uint64_t v1p = pack2(v1, v1);
#pragma unroll
            for (int i = 0; i < NC / 2; ++i) {
              x[2 * i] = fast_exp2(x[2 * i]); x[2 * i + 1] = fast_exp2(x[2 * i + 1]);
              uint64_t vi;
              asm volatile("ld.shared.b64 %0, [%1];" : "=l"(vi) : "r"(vinv_at + 8 * i));
              float w0, w1;
              unpack2(mul2(mul2(pack2(x[2 * i], x[2 * i + 1]), v1p), vi), w0, w1);
              hw[i] = pack_h(w0, w1);
            }
            if (settled) break;
            // What this waits for are the other softmax warps, each of which comes here whatever its own waits gave (they are
            // bounded, and short once one has run out).  So it does not look at the abort flag, and all read the same word.
            if (!mbar_try(BAR(OVER), (asked - 1) & 1)) {
              const uint64_t t0 = global_ns();
#pragma unroll 1
              while (!mbar_try(BAR(OVER), (asked - 1) & 1))
                if (global_ns() - t0 > 8 * WAIT_NS) { *abort_flag = 1; break; }
            }
            if (over_at[asked & 1] != asked) break;
            fresh = settled = true;                  // (from the scores again: they are still in tensor memory)
            rc_page = rc_at + S::RC0_OFF - S::RC_OFF;
            continue;
          }
          // ---- new references, from this page's largest scores and weights per query row
          fresh = false;
          if (!first) {                              // (P^T's buffers are idle then, and the products so far there to be scaled)
            hold(PE + ((g - 1) & 1), (g - 1) >> 1, 16);
            tc_fence_after();
          }
          over_keys(x, xq, fmax2);
          if (part == 0) {
            const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v1)), lo = __reduce_min_sync(0xFFFFFFFFu, gone ? 0x7F800000u : __float_as_uint(v1));
            if (lane == 0) { vspan[quarter] = __uint_as_float(hi); vspan[4 + quarter] = __uint_as_float(lo); }
          }
          soft_sync();
          const float vhi = of_quarters_v(vspan, fmax2), vlo = of_quarters_v(vspan + 4, fmin2);
          if (sidx < N) {
            const float mo = mref[sidx], mn = fmaxf(mo, of_quarters(xq, fmax2));
            fq[sidx] = mo == mn ? 1.f : fast_exp2(mo - mn);
            xz[sidx] = mn == -CUDART_INF_F ? 0.f : -mn;                        // what the scores move by
            mref[sidx] = mn;
            rref[sidx] -= mo == mn || mo == -CUDART_INF_F ? 0.f : mn - mo;
            rcf[4 * (sidx >> 1) + 2 + (sidx & 1)] = mn == -CUDART_INF_F ? 0.f : -mn;
          }
          // The rows' largest weights: each row's own, for rows that hardly see a V far above the rest should not follow it.  In a
          // first page whose steps are within 2^6 of each other the largest step serves for every row: each has a key of e = 1 there.
          const bool wide = !first || vhi > 64.f * vlo;
          if (wide) {
            soft_sync();
#pragma unroll
            for (int i = 0; i < NC; ++i) x[i] = fast_exp2(x[i] + xz[col0 + i]) * v1;
            over_keys(x, xq, fmax2);
            soft_sync();
          }
          if (sidx < N) {
            const float tm = wide ? of_quarters(xq, fmax2) : vhi;
            float D = rref[sidx], v = D == -CUDART_INF_F ? 0x1p126f : fast_exp2(fminf(W_SHIFT - D, 126.f)), f = 1.f;
            if (tm * v > W_LIMIT && mref[sidx] > -CUDART_INF_F) {
              const float nd = (float)((int)(__float_as_uint(tm) >> 23) - 127);
              f = fast_exp2(D - nd);
              rref[sidx] = D = nd;
              v = fast_exp2(fminf(W_SHIFT - D, 126.f));
            }
            go[sidx] = f; vinv[sidx] = v;
          }
          soft_sync();
          if (warp == SOFT_WARP0) {                  // (a row without any key so far, or with a reference far below 0: the next page settles again)
            float v = 0.f;
            bool none = false;
            for (int i = lane; i < rows; i += 32) { v = fmaxf(v, vinv[i]); none |= mref[i] < FAR_BELOW; }
            const uint32_t m = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v));
            none = __any_sync(0xFFFFFFFFu, none);
            if (lane == 0) { limit[0] = none ? -CUDART_INF_F : X_LIMIT; limit[1] = __uint_as_float(m); }
          }
          if (!first) {
#pragma unroll
            for (int i = 0; i < NC / 2; ++i) {
              const uint64_t f = *reinterpret_cast<const uint64_t*>(fq + col0 + 2 * i);
              l[i] = mul2(l[i], f);
            }
#pragma unroll 1
            for (int j = 0; j < NP; ++j) {
              float o[4];
              tmem_ld4(TM_O + lanes + col0 + 4 * j, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 4; ++e) o[e] *= go[col0 + 4 * j + e];
              tmem_st4(TM_O + lanes + col0 + 4 * j, o);
            }
            tmem_wait_st();
          }
          soft_sync();
          if (!careful) rc_page = rc_at;
        }
        // ---- S^T goes back; P^T out; sums of e
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(SE + buf));
        if (g >= 2) hold(PE + buf, (g - 2) >> 1, 17);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
          const int col = col0 + 4 * j;
          asm volatile("st.shared.v2.b32 [%0], {%1,%2};"
                       ::"r"(prow + buf * S::P_BYTES + ((((uint32_t)col >> 3) ^ swz) << 4) + (col & 4) * 2), "r"(hw[2 * j]), "r"(hw[2 * j + 1]) : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(PF + buf));
#pragma unroll
        for (int i = 0; i < NC / 2; ++i) l[i] = add2(l[i], pack2(x[2 * i], x[2 * i + 1]));
      }
      // ---- the item's (or piece's) end: sums over the keys, then O^T
      {
        float v[NC];
#pragma unroll
        for (int i = 0; i < NC / 2; ++i) unpack2(l[i], v[2 * i], v[2 * i + 1]);
        over_keys(v, xq, fsum2);
        soft_sync();
      }
      const int T = wk.pages(p.has_new);
      const bool whole = wk.t0 == 0 && wk.t1 == T;
      const uint32_t at = prefix[wk.b] + (uint32_t)(wk.it * (T + SHARE_COST));   // the item's place in the list
      uint32_t piece0 = 0;
      int pieces = 1;
      if (!whole) {
        piece0 = cut.owner(at + SHARE_COST);
        pieces = (int)(cut.owner(at + SHARE_COST + T - 1) - piece0) + 1;
      }
      constexpr int SLOT = N * (DH + 2);             // (a block's share can hold the end of one cut item and the start of another)
      float* ps = p.part + (int64_t)(2 * (int)blockIdx.x + (wk.opens ? 0 : 1)) * SLOT;
      if (sidx < N) {
        const float ls = of_quarters(xq, fsum2);
        const float m = mref[sidx], up = rref[sidx] - W_SHIFT + 9.f;           // (times V_UNIT before or after: neither 0 nor infinite)
        const float f = rref[sidx] == -CUDART_INF_F ? 1.f : up > 0.f ? fast_exp2(up - 32.f) : fast_exp2(up) * V_UNIT;
        const float rd = !whole ? 1.f : ls > 0.f || ls != ls ? 1.f / ls : 0.f;   // a row without keys: zeros
        fq[sidx] = f * rd;
        if (sidx < rows) {
          if (!whole) {
            __stcg(ps + N * DH + sidx, m);
            __stcg(ps + N * DH + N + sidx, ls);
          } else if (p.lse) {
            int i, hq;
            row_of(p, h, r0 + sidx, i, hq);
            p.lse[((int64_t)wk.b * p.H_q + hq) * p.n_q + i] = (m + log2f(ls)) * 0.6931471805599453f;
          }
        }
      }
      hold(PE + ((g - 1) & 1), (g - 1) >> 1, 18);
      tc_fence_after();
      soft_sync();
      __nv_bfloat16* dst = p.out + (int64_t)wk.b * p.n_q * p.H_q * DH + (kl & ~1);
#pragma unroll 1
      for (int j = 0; j < NP; ++j) {
        float o[4];
        tmem_ld4(TM_O + lanes + col0 + 4 * j, o);
        tmem_wait_ld();
        const int c = col0 + 4 * j;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] *= fq[c + e];
        if (whole) {
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] *= 0x1p32f;
          // two rows at a time: the even lane takes both channels of the first, the odd one of the second
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const float got = __shfl_xor_sync(0xFFFFFFFFu, (lane & 1) ? o[e] : o[e + 1], 1);
            const int r = c + e + (lane & 1);
            const __nv_bfloat162 y = (lane & 1) ? __floats2bfloat162_rn(got, o[e + 1]) : __floats2bfloat162_rn(o[e], got);
            if (kl < DH && r < rows) *reinterpret_cast<__nv_bfloat162*>(dst + roff[r]) = y;
          }
        } else if (kl < DH) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (c + e < rows) __stcg(ps + (c + e) * DH + kl, o[e]);
        }
      }
      tc_fence_before();
      if (*abort_flag && p.status && sidx == 0) atomicOr(p.status + wk.b, SPACE_ST_TIMEOUT);
      if (!whole) {
        soft_sync();
        if (sidx == 0) {
          __threadfence();                           // (after the barrier: for all the stores)
          int* arrived = p.arrived + ((wk.b * p.H_kv + h) * p.n_rt + rb);
          const int last = atomicAdd(arrived, 1) == pieces - 1;
          if (last) *arrived = 0;                    // ready for the next call
          __threadfence();
          *last_flag = last;
        }
        soft_sync();
        if (*last_flag) join_pieces<DH, N, 1, 4>(p, cut, wk.b, h, r0, rows, piece0, pieces, at, sidx, SOFT);
      }
      soft_sync();                                   // references, factors and the flag are free for the next item
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 3) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

template <int DH>
size_t smem_bytes(int max_batch) { return Smem<DH>::TABLE_OFF + (size_t)(max_batch + 1) * 4 + (size_t)max_batch * 4; }

template <int DH>
cudaError_t launch_dim(Params& p, const space_ctx* ctx, cudaStream_t st) {
  static unsigned long long done_mask = 0;           // devices on which the kernel may have its shared memory
  const int max_batch = ctx->cfg.max_batch;
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 64 || !((done_mask >> dev) & 1ull)) {
    cudaFuncSetAttribute(kvq_attn_tc_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<DH>(128));
    if (dev < 64) done_mask |= 1ull << dev;
  }
  static_assert(16 * NP <= KVQ_SM_ROWS, "a slot per block");
  p.n_groups = ctx->sm_count;
  return launch_pdl(kvq_attn_tc_kernel<DH>, dim3(p.n_groups), dim3(THREADS), smem_bytes<DH>(max_batch), st, p, max_batch);
}

}  // namespace

int launch_kvq_attn_tc(space_ctx* ctx, kvq::Params& p, cudaStream_t st) {
  p.n_rt = (p.n_q * p.G + 16 * NP - 1) / (16 * NP);
  return cuda_ok(ctx->cfg.head_dim == 128 ? launch_dim<128>(p, ctx, st) : launch_dim<64>(p, ctx, st));
}
