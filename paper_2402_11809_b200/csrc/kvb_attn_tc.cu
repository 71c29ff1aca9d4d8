// Attention of a step's block rows over the 8-bit cache (space_kvb_attn_step), items of up to 32, 64 or 128 query rows on tcgen05.
//
// The mathematics is kvb_attn.cu's (codes as operands as they lie, query rows and weights as two e4m3 terms each), with a page
// of 128 keys in the place of a block of 32:
//   S = q0 K^T + q1 K^T,    D = w0 V + w1 V,    chunk b of 32 keys (one K and one V scale 2^k_b, 2^v_b):   m_b = max_j s_j,
//   e_j = 2^(s_j - m_b),    w_j = e_j 2^((m_b - m) + v_b - E + 8),    m = max m_b,  E = max_b (m_b - m) + v_b,
//   l += sum_b 2^(m_b - M) sum_j e_j,    o = o 2^(R - R') + D 2^(E + (m - M) - R' - 8)     with R' the larger of R and E + (m - M).
// The block's own rows go through as one more page: a row, scaled by a power of two of its own, is two e4m3 terms as well (to 2^-18 of
// its largest element), which stand in for two rows of 64 with the same scores and the same weights:
//   S = (q0 + q1) (k0 + k1)^T,    D = (w0 + w1) (v0 + v1),    a mask bit and {2^k_j, v_j} for each key.
// (As bf16 products when an item ended they took 13,000 cycles there, of 25,000 between items: code that runs once an item comes
// from far away.  Two warps that have nothing else to do bring them an item ahead.)
//
// The work.  Query rows are the MMA's M extent: 128 of them, or 64 or 32 held twice or four times over, each copy with keys of its own
// (chunks of 32).  Both first operands, query rows and weights, are in tensor memory: an M = 128, K = 32 product takes 10 + N/2 cycles
// then, 43 + N/2 with the first operand in shared memory.  Two threads have a row (of a copy), half of its keys and half of the
// result's channels each; they tell each other their largest scores.  The flat list of 128-key pages over all (sequence, kv head,
// query rows) items is cut evenly over the thread blocks, one per SM.  A page's scores are there when the softmax of the page before ends,
// and its result is added up in the next page's time: the softmax never waits for products, nor they for each other.  Pieces of
// a cut item are joined by the block that stores the last of them, always in the same order.
//
// What bounds it: the softmax's chain of a page, about 2400 cycles with two warps to a scheduler (scores from tensor memory
// 370, weights 870 of which 512 are exponentials, the result 500, waits and meetings 500) against 1200 of products and 1300 of the page's bytes;
// between items 11,000 cycles.  16 sequences of up to 4096 keys, 32 heads, 36 rows: 127 us; 8 of 8192, 8 heads, 392 rows, 128 at a
// time: 272 us (387 TFLOP/s of the products that the formulas ask for, twice that of e4m3 ones).  With 128 rows a thread's scores and
// sums and a page's result are more than its registers: 286 bytes are spilled (with 64 rows 12, with 32 none; head size 128).
//
// Warps: 0-7 softmax and sums, 8 products (one thread), 9 copies (one thread), 10 and 11 ask L2 for the rows that items will want and
// bring blocks' own rows.  The copying thread walks the list and leaves out what has no keys (pages outside the pool); what
// there is it announces in order, and everybody else goes by that.
// Every wait is bounded; an expired wait sets SPACE_ST_TIMEOUT.  The warps that copy and that bring rows end there (of the latter both or
// neither), the others go through the rest of the share with waits that return at once, every warp as one; the block drains and exits.
#include "kvb_attn.cuh"

namespace {
using namespace kvb;

constexpr int TILE = SPACE_PAGE_SIZE;                // keys of a page, rows of an MMA
constexpr int GROUP = 128, SOFT = 2 * GROUP, THREADS = SOFT + GROUP;           // (registers move by groups of four warps)
constexpr int SHARE_COST = 5;                        // fixed cost of an item, in pages (2, 3, 4, 6 for 36 rows of 16 sequences: 148, 143, 135, 137 us)
constexpr int RING = 16;                             // scales and announcements of that many pages
enum { NO_MORE = 0x7FFFFFFF };                        // announced behind the last page
enum { OWN = 0x7FFFFFFE };                            // announced as an item's last page: the block's own rows
constexpr float REF_FAR = 0x1p22f;                   // up to this a reference's rounding moves weights by 2^0.25 at most

template <int DH>
struct Smem {
  using F = Fmt<DH>;
  static constexpr int STAGES = DH == 128 ? 4 : 8;           // pages on their way; behind them a place for a block's own rows
  static constexpr int MEET = DH / 4;                        // channels of a thread that copies of a row meet in at a time
  static constexpr int PITCH = SOFT + 1;                     // floats (four channels apart: another bank)
  static constexpr int MEET_OFF = 0;                         // [MEET][PITCH]
  static constexpr int MEET_BYTES = MEET * PITCH * 4 / 128 * 128 + 128;
  static constexpr int K_OFF = MEET_BYTES;                   // [STAGES + 1]
  static constexpr int V_OFF = K_OFF + (STAGES + 1) * F::CODES;      // [STAGES + 1]
  static constexpr int SCALE_OFF = V_OFF + (STAGES + 1) * F::CODES;        // [RING][4] {K, V}
  static constexpr int ML_OFF = SCALE_OFF + RING * 32;       // [2][SOFT] {M, l} of rows' halves and copies, by item
  static constexpr int OWN_OFF = ML_OFF + 2 * SOFT * 8;      // [64] of the block's own rows {K's power of two, V's exponent}
  static constexpr int XCH_OFF = OWN_OFF + SPACE_MAX_ROWS * 8;    // [2][SOFT] a page's {largest score, E} of a row's halves
  static constexpr int TOPS_OFF = XCH_OFF + 2 * SOFT * 8;    // [2][SOFT] largest elements of query rows' halves, by item
  static constexpr int DESC_OFF = TOPS_OFF + 2 * SOFT * 4;   // [RING] {item of the share, page of it}
  static constexpr int BAR_OFF = DESC_OFF + RING * 8;
  static constexpr int N_BARS = 4 * (STAGES + 1) + RING + 14;
  static constexpr int MISC_OFF = BAR_OFF + N_BARS * 8;
  static constexpr int MASK_OFF = (MISC_OFF + 16 + 7) / 8 * 8;
  static constexpr int TABLE_OFF = MASK_OFF + SPACE_MAX_ROWS * 8;    // prefix[max_batch + 1], seq_len[max_batch]
  static_assert(TABLE_OFF + 129 * 4 + 128 * 4 <= 227 * 1024, "shared-memory plan too large");
  static_assert(RING >= STAGES + 6, "an announcement outlives everybody who reads it");
};

__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, %0;" ::"n"(SOFT) : "memory"); }
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
// e4m3 x e4m3 -> f32, M = 128, first operand in tensor memory (a row per lane, four bytes of it per column), second one K-major
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

__device__ __forceinline__ float max16(const uint32_t* s) {
  const float* x = reinterpret_cast<const float*>(s);
  const float a = max3(max3(x[0], x[1], x[2]), x[3], x[4]), b = max3(max3(x[5], x[6], x[7]), x[8], x[9]);
  const float c = max3(max3(x[10], x[11], x[12]), x[13], x[14]);
  return fmaxf(max3(a, b, c), x[15]);
}

__device__ __forceinline__ void pair_sync() { asm volatile("bar.sync 2, 64;" ::: "memory"); }      // the warps that bring own rows
__device__ __forceinline__ bool pair_all(bool mine) {                                                // (and whether both may)
  int all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 2, 64, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
               : "=r"(all) : "r"((int)mine) : "memory");
  return all != 0;
}
__device__ __forceinline__ void prefetch_line(const char* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// The block's own rows as a page, by two warps: row j's K as two e4m3 terms in rows j and 64 + j of the stage, V likewise in sixteens
// j / 16 and 4 + j / 16; each row has powers of two of its own.  Row n_q and those behind it: zeros.
template <int DH>
__device__ __forceinline__ void bring_own(const Params& p, int b, int h, unsigned char* ks, unsigned char* vs, float2* sc, uint32_t full_k) {
  using F = Fmt<DH>;
  constexpr int LANES = DH / 4, PER = 64 / LANES, BATCH = 4;          // lanes of a row in the first pass, rows of both warps
  const int t = threadIdx.x & 63;
  const char* kn = p.kn + (int64_t)b * p.n_sb + (int64_t)h * p.n_sh;
  const char* vn = p.vn + (int64_t)b * p.n_sb + (int64_t)h * p.n_sh;
  const int x = t % LANES;
  const uint32_t lanes = LANES == 32 ? 0xFFFFFFFFu : 0xFFFFu << (t & 16);
#pragma unroll 1
  for (int r0 = t / LANES; r0 < SPACE_MAX_ROWS; r0 += BATCH * PER) {
    uint2 k[BATCH], v[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int r = r0 + j * PER;
      k[j] = v[j] = make_uint2(0, 0);
      if (r < p.n_q) {
        k[j] = *(reinterpret_cast<const uint2*>(kn + (int64_t)r * p.n_sr) + x);
        v[j] = *(reinterpret_cast<const uint2*>(vn + (int64_t)r * p.n_sr) + x);
      }
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int r = r0 + j * PER;
      unsigned char* at = ks + (x >> 2) * F::K_COLS + 16 * r + 4 * (x & 3);
      if (r >= p.n_q) {                              // (the same for a row's lanes)
        *reinterpret_cast<uint32_t*>(at) = 0;
        *reinterpret_cast<uint32_t*>(at + 16 * SPACE_MAX_ROWS) = 0;
        if (x == 0) sc[r] = make_float2(1.f, 0.f);
        continue;
      }
      k[j] = make_uint2(kvq::finite_pair(k[j].x), kvq::finite_pair(k[j].y));
      v[j] = make_uint2(kvq::finite_pair(v[j].x), kvq::finite_pair(v[j].y));
      const uint32_t kt = __reduce_max_sync(lanes, kvq::max_bits(make_uint4(k[j].x, k[j].y, 0, 0)));
      const uint32_t vt = __reduce_max_sync(lanes, kvq::max_bits(make_uint4(v[j].x, v[j].y, 0, 0)));
      const int ke = max((int)(kt >> 7) - 127, -100) - 7, ve = max((int)(vt >> 7) - 127, -100) - 7;      // the largest to [2^7, 2^8)
      const float up = pow2(-ke);
      uint32_t w0, w1;
      split4(kvq::bf_lo(k[j].x) * up, kvq::bf_hi(k[j].x) * up, kvq::bf_lo(k[j].y) * up, kvq::bf_hi(k[j].y) * up, w0, w1);
      *reinterpret_cast<uint32_t*>(at) = w0;
      *reinterpret_cast<uint32_t*>(at + 16 * SPACE_MAX_ROWS) = w1;
      if (x == 0) sc[r] = make_float2(pow2(ke), (float)ve);
    }
  }
  fence_async();
  pair_sync();
  if (t == 0) mbar_arrive(full_k);
  // a thread has two channels (of 64: with half of the keys), four keys at a time
  constexpr int PARTS = 128 / DH;
  const int c = 2 * (t % (DH / 2)), q0 = t / (DH / 2);
#pragma unroll 2
  for (int q = q0; q < SPACE_MAX_ROWS / 4; q += PARTS) {
    unsigned char* at = vs + (q >> 2) * F::V_ROWS + 16 * c + 4 * (q & 3);
    if (4 * q >= p.n_q) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        *reinterpret_cast<uint32_t*>(at + 16 * i) = 0;
        *reinterpret_cast<uint32_t*>(at + 16 * i + 4 * F::V_ROWS) = 0;
      }
      continue;
    }
    uint32_t w[4];
    float up[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = 4 * q + j;
      w[j] = r < p.n_q ? *reinterpret_cast<const uint32_t*>(vn + (int64_t)r * p.n_sr + 2 * c) : 0u;
      up[j] = pow2(-(int)sc[r].y);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = kvq::finite_pair(w[j]);
    uint32_t w0, w1;
    split4(kvq::bf_lo(w[0]) * up[0], kvq::bf_lo(w[1]) * up[1], kvq::bf_lo(w[2]) * up[2], kvq::bf_lo(w[3]) * up[3], w0, w1);
    *reinterpret_cast<uint32_t*>(at) = w0;
    *reinterpret_cast<uint32_t*>(at + 4 * F::V_ROWS) = w1;
    split4(kvq::bf_hi(w[0]) * up[0], kvq::bf_hi(w[1]) * up[1], kvq::bf_hi(w[2]) * up[2], kvq::bf_hi(w[3]) * up[3], w0, w1);
    *reinterpret_cast<uint32_t*>(at + 16) = w0;
    *reinterpret_cast<uint32_t*>(at + 16 + 4 * F::V_ROWS) = w1;
  }
  fence_async();
  pair_sync();
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

template <int DH, int REP>
__global__ void __launch_bounds__(THREADS, 1) kvb_attn_tc_kernel(const __grid_constant__ Params p, int max_batch) {
  using F = Fmt<DH>;
  using S = Smem<DH>;
  constexpr int STAGES = S::STAGES, RT = TILE / REP;                           // rows of an item
  constexpr int KEYS = TILE / REP / 2;               // of a page, that a thread has
  extern __shared__ __align__(1024) unsigned char sm[];
  const uint32_t base = smem_u32(sm), bar0 = base + S::BAR_OFF;
  auto BAR = [&](int i) { return bar0 + 8u * i; };
  // Of a stage: K, V are there / have been used.  SAID: page m is announced and its scales are there.  QREADY: an item's query rows are
  // there.  SDONE (two, by page): scores.  PREADY: weights (and the result before has been added up).  ODONE: a page's result.
  // XCH, QTOP (by pair of warps): largest scores, elements of both halves.  OVER: all products are done.
  constexpr int FULLK = 0, FULLV = STAGES + 1, FREEK = 2 * (STAGES + 1), FREEV = 3 * (STAGES + 1), SAID = 4 * (STAGES + 1), QREADY = SAID + RING,
                SDONE = QREADY + 1, PREADY = QREADY + 3, ODONE = QREADY + 4, XCH = QREADY + 5, QTOP = QREADY + 9, OVER = QREADY + 13;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + S::MISC_OFF);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::MISC_OFF + 4);
  volatile int* last_flag = reinterpret_cast<volatile int*>(sm + S::MISC_OFF + 8);
  uint32_t* prefix = reinterpret_cast<uint32_t*>(sm + S::TABLE_OFF);
  int* seq_len = reinterpret_cast<int*>(prefix + max_batch + 1);
  volatile int2* desc = reinterpret_cast<volatile int2*>(sm + S::DESC_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < 4 * (STAGES + 1) + RING; ++s) mbar_init(BAR(s), 1);
    mbar_init(BAR(QREADY), 8); mbar_init(BAR(SDONE), 1); mbar_init(BAR(SDONE + 1), 1); mbar_init(BAR(PREADY), 8); mbar_init(BAR(ODONE), 1);
    mbar_init(BAR(OVER), 1);
    for (int i = 0; i < 4; ++i) { mbar_init(BAR(XCH + i), 2); mbar_init(BAR(QTOP + i), 2); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (threadIdx.x < SPACE_MAX_ROWS) reinterpret_cast<uint64_t*>(sm + S::MASK_OFF)[threadIdx.x] = p.mask[threadIdx.x];
  // Tensor memory is taken when the kernel before has given its own back, and the next kernel's blocks may come when all of these
  // have theirs: nobody holds some while it waits for somebody who wants some.
  pdl_wait();
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
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
  // columns: scores (two buffers; those of 32 keys make way for their weights, 16 columns), a page's result, query rows (two buffers of
  // two terms)
  const uint32_t TM_S = tmem, TM_O = tmem + 2 * TILE, TM_Q = TM_O + TILE;
  const Cut cut(prefix[p.B], p.n_groups);
  Walk wk;
  const bool mine = blockIdx.x < cut.NG;
  const uint32_t share0 = mine ? cut.begin(blockIdx.x) : 0;
  wk.b = 0; wk.cur = share0;
  wk.end = mine ? cut.begin(blockIdx.x + 1) : 0;
  uint32_t m = 0;                                    // pages so far
  uint32_t cached = 0, own = 0;                      // of the cache, and blocks' own rows, among them
  uint32_t queries = 0;                              // items with pages so far: others' query rows nobody announces or waits for
  auto hold = [&](int bar, uint32_t use, int site) { return wait(BAR(bar), use & 1, abort_flag, p.err, site); };

  if (warp >= 8) {
    regs_dec<56>();
    if (warp == 9 && elect_one()) {
      // ---- copies: K of a page when the K of the page that had its stage has been used, V likewise
      bool ok = true;
      int item = 0;
      for (; ok && wk.next(prefix, seq_len, p.has_new, share0); ++item) {
        const int32_t* table = p.cache.page_table + (int64_t)wk.b * p.cache.pages_per_seq;
        const char* pool = p.cache.pool + (int64_t)(wk.it / p.n_rt) * p.cache.head_stride;
        const int end = min(wk.t1, wk.cached());
        int pg = wk.t0 < end ? __ldg(table + wk.t0) : -1;
        for (int t = wk.t0; t < end && ok; ++t) {
          const int page = pg;
          if (t + 1 < end) pg = __ldg(table + t + 1);        // (one page ahead of its use)
          if (page < 0 || page >= p.cache.n_pages) {
            if (p.status) atomicOr(p.status + wk.b, SPACE_ST_BAD_PAGE);
            continue;
          }
          const uint32_t s = cached % STAGES, use = cached / STAGES, e = m % RING;
          const char* head = pool + (int64_t)page * p.cache.page_stride;
          desc[e].x = item; desc[e].y = t;
          mbar_expect_tx(BAR(SAID + e), 32);
          bulk_copy(base + S::SCALE_OFF + e * 32, head + F::SCALES, 32, BAR(SAID + e));
          if (use) ok = hold(FREEK + s, use - 1, 1);
          if (ok) {
            mbar_expect_tx(BAR(FULLK + s), F::CODES);
            bulk_copy(base + S::K_OFF + s * F::CODES, head, F::CODES, BAR(FULLK + s));
            if (use) ok = hold(FREEV + s, use - 1, 2);
          }
          if (ok) {
            mbar_expect_tx(BAR(FULLV + s), F::CODES);
            bulk_copy(base + S::V_OFF + s * F::CODES, head + F::CODES, F::CODES, BAR(FULLV + s));
          }
          ++m; ++cached;
        }
        if (ok && p.has_new && wk.L >= 0 && wk.t1 > wk.cached()) {             // (two other warps bring them)
          desc[m % RING].x = item; desc[m % RING].y = OWN;
          mbar_arrive(BAR(SAID + m % RING));
          if (own) ok = hold(FREEV + STAGES, own - 1, 18);     // (so that announcements are not far ahead either)
          ++m; ++own;
        }
      }
      if (ok) {
        desc[m % RING].x = NO_MORE;
        mbar_arrive(BAR(SAID + m % RING));
      }
      // every copy has landed before the block may exit (a page whose copies a wait that ran out cut short is the last)
      for (uint32_t j = m >= RING ? m - RING + 1 : 0; j < m; ++j) mbar_drain_bounded(BAR(SAID + j % RING), (j / RING) & 1, WAIT_NS / 10);
      for (uint32_t j = cached > STAGES ? cached - STAGES : 0; j < cached; ++j) {
        mbar_drain_bounded(BAR(FULLK + j % STAGES), (j / STAGES) & 1, WAIT_NS / 10);
        mbar_drain_bounded(BAR(FULLV + j % STAGES), (j / STAGES) & 1, WAIT_NS / 10);
      }
    } else if (warp == 8 && elect_one()) {
      // ---- products: scores of page q, a page ahead of the result of page m
      uint32_t q = 0, q_cached = 0, q_own = 0;
      int item = -1;
      bool ok = true, more = true;
      while (true) {
        while (more && q < m + 2) {
          ok = hold(SAID + q % RING, q / RING, 3) && ok;
          const int it = ok ? desc[q % RING].x : NO_MORE;
          if (it == NO_MORE) { more = false; break; }
          if (it != item) {
            if (q > m) break;                        // (its query rows come when the weights of page m have)
            ok = hold(QREADY, queries++, 4) && ok;
            item = it;
          }
          const bool is_own = ok && desc[q % RING].y == OWN;
          const uint32_t s = is_own ? STAGES : q_cached % STAGES;
          ok = hold(FULLK + s, is_own ? q_own : q_cached / STAGES, 5) && ok;
          is_own ? ++q_own : ++q_cached;
          if (m && q > m) ok = hold(ODONE, m - 1, 6) && ok;                    // (the weights of page q - 2 lie where these scores go)
          tc_fence_after();
          const uint64_t kd = plain_desc(base + S::K_OFF + s * F::CODES, F::K_COLS, 128);
          const uint32_t qd = TM_Q + ((queries - 1) & 1) * 64;
          if (ok && !is_own) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int ks = 0; ks < DH / 32; ++ks)
                mma8_ts(TM_S + (q & 1) * TILE, qd + i * (DH / 4) + 8 * ks, kd + (uint64_t)((ks * 2 * F::K_COLS) >> 4), instr_desc(TILE), i + ks > 0);
          } else if (ok) {                           // both terms of 64 rows onto the same scores
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int ks = 0; ks < DH / 32; ++ks)
                mma8_ts(TM_S + (q & 1) * TILE, qd + (i & 1) * (DH / 4) + 8 * ks, kd + (uint64_t)((ks * 2 * F::K_COLS + (i >> 1) * 16 * SPACE_MAX_ROWS) >> 4),
                        instr_desc(SPACE_MAX_ROWS), i + ks > 0);
          }
          tc_commit(BAR(SDONE + (q & 1)));
          tc_commit(BAR(FREEK + s));
          ++q;
        }
        if (m == q) {
          if (more) continue;
          break;
        }
        const bool is_own = ok && desc[m % RING].y == OWN;
        const uint32_t s = is_own ? STAGES : cached % STAGES;
        ok = hold(FULLV + s, is_own ? own : cached / STAGES, 7) && ok;
        is_own ? ++own : ++cached;
        if (m) ok = hold(ODONE, m - 1, 8) && ok;     // (long since: whoever brings the weights has waited for it)
        ok = hold(PREADY, m, 9) && ok;
        tc_fence_after();
        const int chunks = is_own ? 1 : 3;          // (own rows: their second terms with the same weights)
        const uint64_t vd = plain_desc(base + S::V_OFF + s * F::CODES, F::V_ROWS, 128);
        if (ok) {
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              mma8_ts(TM_O, TM_S + (m & 1) * TILE + 32 * (b & chunks) + 8 * i, vd + (uint64_t)((2 * b * F::V_ROWS) >> 4), instr_desc(DH), b + i > 0);
        }
        tc_commit(BAR(ODONE));
        tc_commit(BAR(FREEV + s));
        ++m;
      }
      tc_commit(BAR(OVER));                          // all products done before tensor memory is released, after a wait that ran out too
      mbar_drain_bounded(BAR(OVER), 0, WAIT_NS);
    } else if (warp >= 10) {
      // ---- query rows, and the block's own, of all the share's items: out of HBM before somebody waits for them
      Walk ahead = wk;
      while (ahead.next(prefix, seq_len, p.has_new, share0)) {
        const int h = ahead.it / p.n_rt, r0 = (ahead.it - h * p.n_rt) * RT, rows = min(p.n_q * p.G - r0, RT), t = threadIdx.x & 63;
        for (int r = t; r < rows; r += 64) {
          int i, hq;
          row_of(p, h, r0 + r, i, hq);
          const char* at = p.q + (int64_t)ahead.b * p.q_sb + (int64_t)i * p.q_sr + (int64_t)hq * p.q_sh;
          prefetch_line(at);
          if (DH == 128) prefetch_line(at + 128);
        }
        if (!p.has_new || ahead.t1 <= ahead.cached()) continue;
        if (t < p.n_q) {
          const int64_t at = (int64_t)ahead.b * p.n_sb + (int64_t)t * p.n_sr + (int64_t)h * p.n_sh;
          prefetch_line(p.kn + at); prefetch_line(p.vn + at);
          if (DH == 128) { prefetch_line(p.kn + at + 128); prefetch_line(p.vn + at + 128); }
        }
      }
      // ---- the block's own rows, an item ahead
      while (wk.next(prefix, seq_len, p.has_new, share0)) {
        if (!p.has_new || wk.L < 0 || wk.t1 <= wk.cached()) continue;
        const auto place = [&] { return own == 0 || (hold(FREEK + STAGES, own - 1, 19) && hold(FREEV + STAGES, own - 1, 20)); };
        if (!all_told(place, pair_all)) break;       // (both warps or none: bring_own has barriers of the two)
        bring_own<DH>(p, wk.b, wk.it / p.n_rt, sm + S::K_OFF + STAGES * F::CODES, sm + S::V_OFF + STAGES * F::CODES,
                      reinterpret_cast<float2*>(sm + S::OWN_OFF), BAR(FULLK + STAGES));
        if ((threadIdx.x & 63) == 0) mbar_arrive(BAR(FULLV + STAGES));
        ++own;
      }
    }
  } else {
    regs_inc<224>();                                 // (256 threads x 224 + 128 x 56 = the 384 x 168 of the launch)
    const int half = warp >> 2, tid = threadIdx.x & (GROUP - 1), w4 = warp & 3;
    const int rep = w4 / (4 / REP), row = tid % RT;
    const uint32_t lanes = (uint32_t)(32 * w4) << 16;
    const int key0 = rep * (TILE / REP) + half * KEYS;       // first of this thread's keys of a page
    const uint32_t TM_C = TM_O + lanes + half * (DH / 2);
    // What is announced of page m, to whole warps: a warp goes round its loop together.
    int next_item, next_page;
    auto look = [&](uint32_t m) {
      const bool said = __all_sync(0xFFFFFFFFu, hold(SAID + m % RING, m / RING, 12));
      next_item = said ? desc[m % RING].x : NO_MORE;
      next_page = desc[m % RING].y;
    };
    // The query row of the item that wk stands at, this thread's half of it: as two terms into a buffer, if the item has pages.
    float f_next = 0.f;                              // factor of its scores
    bool nan_next = false;                           // it holds a NaN or an infinity
    auto bring_query = [&](int item) {
      const int h = wk.it / p.n_rt;
      int i, hq;
      row_of(p, h, (wk.it - h * p.n_rt) * RT + row, i, hq);
      const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)wk.b * p.q_sb + (int64_t)i * p.q_sr + (int64_t)hq * p.q_sh) + half * (DH / 16);
      uint4 v[DH / 16];
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < DH / 16; ++j) v[j] = i < p.n_q ? src[j] : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < DH / 16; ++j) top = max(top, kvq::max_bits(v[j]));
      uint32_t* tops = reinterpret_cast<uint32_t*>(sm + S::TOPS_OFF) + SOFT * (item & 1);
      tops[threadIdx.x] = top;
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(QTOP + w4));
      hold(QTOP + w4, item, 11);
      top = max(top, tops[threadIdx.x ^ GROUP]);
      nan_next = top >= 0x7F80u;
      const int e = nan_next ? 0 : max((int)(top >> 7) - 127, -100) - 7;       // the largest element to [2^7, 2^8)
      const float up = pow2(-e);
      f_next = p.c * pow2(e);
      if (item == 0) look(0);
      if (next_item != item) return;
      if (nan_next) {                                // (zeros for the products, so that it is known whether the row sees a key)
#pragma unroll
        for (int j = 0; j < DH / 16; ++j) v[j] = make_uint4(0, 0, 0, 0);
      }
      const uint32_t to0 = TM_Q + lanes + (queries++ & 1) * 64 + half * (DH / 8);
#pragma unroll
      for (int j = 0; j < DH / 16; j += 2) {
        uint32_t w0[4], w1[4];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint4 x = v[j + k];
          split4(kvq::bf_lo(x.x) * up, kvq::bf_hi(x.x) * up, kvq::bf_lo(x.y) * up, kvq::bf_hi(x.y) * up, w0[2 * k], w1[2 * k]);
          split4(kvq::bf_lo(x.z) * up, kvq::bf_hi(x.z) * up, kvq::bf_lo(x.w) * up, kvq::bf_hi(x.w) * up, w0[2 * k + 1], w1[2 * k + 1]);
        }
        tmem_st4(to0 + 2 * j, w0);
        tmem_st4(to0 + 2 * j + DH / 4, w1);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(QREADY));
    };
    bool live = wk.next(prefix, seq_len, p.has_new, share0);
    if (live) bring_query(0);
    for (int item = 0; live; ++item) {
      const int b = wk.b, it = wk.it, L = wk.L, T = wk.pages(p.has_new);
      const bool whole = wk.t0 == 0 && wk.t1 == T, opens = wk.opens;
      const uint32_t item_at = wk.at;
      const int h = it / p.n_rt, r0 = (it - h * p.n_rt) * RT, rows = min(p.n_q * p.G - r0, RT);
      const float f = f_next;
      const bool nan = nan_next;
      uint64_t o2[DH / 4];
#pragma unroll
      for (int j = 0; j < DH / 4; ++j) o2[j] = 0ull;
      float M = -CUDART_INF_F, l = 0.f, R = 0.f, alpha = 1.f, beta = 0.f;
      // A page's result joins the sum.  (A load from tensor memory and the wait for it stand side by side: its registers may not be
      // touched in between, which the compiler does not know.)
      bool pending = false;
      auto add = [&]() {
        hold(ODONE, m - 1, 13);
        tc_fence_after();
        if (__any_sync(0xFFFFFFFFu, alpha != 1.f)) {
          const uint64_t a2 = pack2(alpha, alpha);
#pragma unroll
          for (int j = 0; j < DH / 4; ++j) o2[j] = mul2(o2[j], a2);
        }
        const uint64_t b2 = pack2(beta, beta);
        uint32_t r[DH / 2];
#pragma unroll
        for (int c = 0; c < DH / 2; c += 32) tmem_ld32(TM_C + c, r + c);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < DH / 4; ++j) o2[j] = fma2(pack2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])), b2, o2[j]);
        tc_fence_before();
      };
      while (next_item == item) {
        const int t = next_page;
        const uint32_t s = cached % STAGES;          // (of a page of the cache)
        const uint32_t TM_SM = TM_S + lanes + (m & 1) * TILE;                  // the page's scores
        constexpr int NC = (KEYS + 31) / 32, N1 = KEYS < 32 ? KEYS : 32;       // 32 keys share their scales
        float2 sc[NC];
#pragma unroll
        for (int k = 0; k < NC; ++k) sc[k] = *(reinterpret_cast<const float2*>(sm + S::SCALE_OFF + (m % RING) * 32) + (key0 >> 5) + k);
        const int vis0 = L - (t == OWN ? 0 : t) * TILE, vis = vis0 - key0;            // visible keys of the page, and of this thread
        if (vis0 < TILE && t != OWN) {               // what lies behind the last row must not count, whatever it is
          hold(FULLV + s, cached / STAGES, 14);
          const int g0 = vis0 >> 4;
#pragma unroll 1
          for (int e = threadIdx.x; e < (8 - g0) * DH; e += SOFT) {
            const int sixteen = g0 + e / DH, keep = min(max(vis0 - 16 * sixteen, 0), 16);
            unsigned char* at = sm + S::V_OFF + s * F::CODES + sixteen * F::V_ROWS + (e % DH) * 16;
            const uint4 w = *reinterpret_cast<const uint4*>(at);
            uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int n = min(max(keep - 4 * j, 0), 4);
              x[j] &= n == 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u;
            }
            *reinterpret_cast<uint4*>(at) = make_uint4(x[0], x[1], x[2], x[3]);
          }
          fence_async();
        }
        hold(SDONE + (m & 1), m >> 1, 15);
        tc_fence_after();
        uint32_t v[KEYS];
#pragma unroll
        for (int k = 0; k < NC; ++k) {
          if (KEYS < 32) tmem_ld16(TM_SM + key0, v);
          else tmem_ld32(TM_SM + key0 + 32 * k, v + 32 * k);
        }
        tmem_wait_ld();
        float pm = -CUDART_INF_F, E = -CUDART_INF_F, top = 0.f, lower = 0.f, sum = 0.f;
        bool none = false;                           // this row sees nothing of the page
        // both halves of the row: the page's largest score, and E relative to it
        auto meet = [&]() {
          float2* xch = reinterpret_cast<float2*>(sm + S::XCH_OFF) + (m & 1) * SOFT;
          xch[threadIdx.x] = make_float2(pm, E);
          if (REP == 4) tc_fence_before();           // (both halves of 32 columns: a half's weights go where the other one's scores were)
          __syncwarp();
          if (lane == 0) mbar_arrive(BAR(XCH + w4));
          look(m + 1);                               // (meanwhile)
          if (pending) add();
          hold(XCH + w4, m, 16);
          if (REP == 4) tc_fence_after();
          const float2 other = xch[threadIdx.x ^ GROUP];
          top = fmaxf(pm, other.x); lower = pm - top;
          none = top == -CUDART_INF_F;
          E = none ? 0.f : fmaxf(E + lower, other.y + (other.x - top));
        };
        // (sixteen weights, first terms, then second ones: where scores of the same 32 keys were)
        auto put = [&](int u, uint32_t* w) {
          const int key = key0 + u;
          const uint32_t at = TM_SM + (key & ~31) + ((key >> 4) & 1) * 4;
          tmem_st4(at, w);
          tmem_st4(at + 8, w + 4);
        };
        if (t != OWN) {
          float fk[NC], ms[NC], mb[NC], x[NC], ev[NC];
          if (vis < KEYS) {
#pragma unroll
            for (int j = 0; j < KEYS; ++j) if (j >= vis) v[j] = 0xFF800000u;
          }
          bool far = false;
#pragma unroll
          for (int k = 0; k < NC; ++k) {
            ms[k] = max16(v + 32 * k);
            if (N1 > 16) ms[k] = fmaxf(ms[k], max16(v + 32 * k + 16));
            fk[k] = fminf(fmaxf(f * sc[k].x, F_MIN), F_MAX);
            x[k] = ms[k] * fk[k];
            mb[k] = ms[k] == -CUDART_INF_F ? 0.f : x[k];
            far = far || fabsf(mb[k]) > REF_FAR;
          }
          if (__any_sync(0xFFFFFFFFu, far)) {          // scores off the largest first, then times the factor
#pragma unroll
            for (int k = 0; k < NC; ++k) {
              const float top = ms[k] == -CUDART_INF_F ? 0.f : ms[k];
              if (fabsf(mb[k]) > SCORE_MAX) {
                fk[k] = SCORE_MAX / fabsf(top);
                x[k] = copysignf(SCORE_MAX, top);
              }
              mb[k] = 0.f;
#pragma unroll
              for (int j = 0; j < N1; ++j) v[32 * k + j] = __float_as_uint(__uint_as_float(v[32 * k + j]) - top);
            }
          }
#pragma unroll
          for (int k = 0; k < NC; ++k) pm = fmaxf(pm, x[k]);
#pragma unroll
          for (int k = 0; k < NC; ++k) {
            ev[k] = (float)((int)((__float_as_uint(sc[k].y) >> 23) & 255u) - 127);
            x[k] = x[k] == -CUDART_INF_F ? -CUDART_INF_F : x[k] - pm;
            E = fmaxf(E, x[k] + ev[k]);
          }
          meet();
          float wf[NC], part[NC];
#pragma unroll
          for (int k = 0; k < NC; ++k) {
            const float d = none || x[k] == -CUDART_INF_F ? -CUDART_INF_F : x[k] + lower;
            wf[k] = fast_exp2(d + (ev[k] + 8.f - E));
            part[k] = fast_exp2(d);
          }
#pragma unroll
          for (int k = 0; k < NC; ++k) {
            const uint64_t f2 = pack2(fk[k], fk[k]), n2 = pack2(-mb[k], -mb[k]), w2 = pack2(wf[k], wf[k]);
            uint64_t sum0 = 0ull, sum1 = 0ull;
#pragma unroll
            for (int u = 0; u < N1; u += 16) {
              uint32_t w[8];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t* y = v + 32 * k + u + 4 * j;
                float a, b, c, d;
                unpack2(fma2(pack2(__uint_as_float(y[0]), __uint_as_float(y[1])), f2, n2), a, b);
                unpack2(fma2(pack2(__uint_as_float(y[2]), __uint_as_float(y[3])), f2, n2), c, d);
                const uint64_t e0 = pack2(fast_exp2(a), fast_exp2(b)), e1 = pack2(fast_exp2(c), fast_exp2(d));
                sum0 = add2(sum0, e0); sum1 = add2(sum1, e1);
                unpack2(mul2(e0, w2), a, b);
                unpack2(mul2(e1, w2), c, d);
                split4(a, b, c, d, w[j], w[4 + j]);
              }
              put(32 * k + u, w);
            }
            float a, b;
            unpack2(add2(sum0, sum1), a, b);
            sum = fmaf(a + b, part[k], sum);
          }
        } else {
          // the block's own rows: a mask and powers of two for each key
          hold(FULLK + STAGES, own, 21);             // (long since; for those powers of two)
          const bool sees = key0 < SPACE_MAX_ROWS && row < rows;
          const uint64_t mask = sees ? reinterpret_cast<const uint64_t*>(sm + S::MASK_OFF)[(r0 + row) >> p.gsh] >> (key0 & 63) : 0ull;     // Eq. 5
          const float2* sc = reinterpret_cast<const float2*>(sm + S::OWN_OFF) + (key0 & 63);
#pragma unroll
          for (int j = 0; j < KEYS; ++j) {
            float y = __uint_as_float(v[j]) * fminf(fmaxf(f * sc[j].x, F_MIN), F_MAX);
            y = (mask >> j) & 1ull ? (y > SCORE_MAX ? SCORE_MAX : y < -SCORE_MAX ? -SCORE_MAX : y) : -CUDART_INF_F;
            pm = fmaxf(pm, y);
            v[j] = __float_as_uint(y);
          }
          const float from = pm == -CUDART_INF_F ? 0.f : pm;
#pragma unroll
          for (int j = 0; j < KEYS; ++j) E = fmaxf(E, __uint_as_float(v[j]) - from + sc[j].y);
          meet();
          const float ref = none ? 0.f : top, up = 8.f - E;
#pragma unroll
          for (int u = 0; u < KEYS; u += 16) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float y[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float off = __uint_as_float(v[u + 4 * j + i]) - ref;
                sum += fast_exp2(off);
                y[i] = fast_exp2(off + (sc[u + 4 * j + i].y + up));
              }
              split4(y[0], y[1], y[2], y[3], w[j], w[4 + j]);
            }
            put(u, w);
          }
        }
        if (REP > 1) {                               // keys that other copies of the row have: each half two of the four chunks
          const uint32_t zero[16] = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (c * REP / 4 != rep && (c & 1) == half) tmem_st16(TM_SM + 32 * c, zero);
        }
        // the weights are where the products want them
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(PREADY));
        // ---- the running maxima, and the factors of the results
        alpha = 1.f; beta = 0.f;
        if (!none) {
          const float Mn = fmaxf(M, top), down = M - Mn, up = top - Mn;
          l = fmaf(sum, fast_exp2(up), l * fast_exp2(down));
          const float r_old = R + down, r_new = E + up, Rn = fmaxf(r_old, r_new);
          alpha = fast_exp2(r_old - Rn);
          beta = fast_exp2(r_new - Rn - 8.f);
          M = Mn; R = Rn;
        }
        pending = true;
        ++m;
        t == OWN ? ++own : ++cached;
      }
      // the next item's query rows, while the last products run
      live = wk.next(prefix, seq_len, p.has_new, share0);
      if (live) bring_query(item + 1);

      if (pending) add();

      // ---- the item's rows, or its piece of them
      const int slot = 2 * (int)blockIdx.x + (opens ? 0 : 1);
      constexpr int SLOT = RT * (DH + 2);
      float* ps = p.part + (int64_t)slot * SLOT;
      const float NAN_F = __int_as_float(0x7FFFFFFF);
      float2* ml = reinterpret_cast<float2*>(sm + S::ML_OFF) + (item & 1) * SOFT;
      ml[threadIdx.x] = make_float2(M, l);
      soft_sync();
      auto total = [&](int r, float& Mx, float& Lx) {        // a row's largest score and sum over all that it has seen
        Mx = -CUDART_INF_F; Lx = 0.f;
#pragma unroll
        for (int k = 0; k < REP; ++k) Mx = fmaxf(Mx, ml[k * RT + r].x);
#pragma unroll
        for (int k = 0; k < REP; ++k) {
          const float2 v = ml[k * RT + r];
          Lx += v.x == -CUDART_INF_F ? 0.f : (v.y + ml[GROUP + k * RT + r].y) * fast_exp2(v.x - Mx);
        }
      };
      float Mx, Lx;
      total(row, Mx, Lx);
      float fac = M == -CUDART_INF_F ? 0.f : fast_exp2(M - Mx) / Lx * fast_exp2(R);
      if (nan && Mx != -CUDART_INF_F) fac = Lx = NAN_F;
      if (row < rows && rep == 0 && half == 0) {
        if (whole) {
          store_lse(p, b, h, r0 + row, Mx, Lx);
        } else {
          __stcg(ps + RT * DH + row, Mx); __stcg(ps + RT * DH + RT + row, Lx);
        }
      }
      // a row's copies meet, MEET channels of each half at a time
      float* buf = reinterpret_cast<float*>(sm + S::MEET_OFF);               // [MEET][PITCH]
#pragma unroll
      for (int c0 = 0; c0 < DH / 2; c0 += S::MEET) {
#pragma unroll
        for (int c = 0; c < S::MEET / 2; ++c) {
          float a, b;
          unpack2(o2[c0 / 2 + c], a, b);
          buf[(2 * c) * S::PITCH + threadIdx.x] = a * fac;
          buf[(2 * c + 1) * S::PITCH + threadIdx.x] = b * fac;
        }
        soft_sync();
        constexpr int QUADS = 2 * S::MEET / 4;       // of a row, both halves
#pragma unroll 1
        for (int e = threadIdx.x; e < rows * QUADS; e += SOFT) {
          const int r = e / QUADS, q = e % QUADS, hf = q / (QUADS / 2), c = 4 * (q % (QUADS / 2));
          float y[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            y[j] = 0.f;
#pragma unroll
            for (int k = 0; k < REP; ++k) y[j] += buf[(c + j) * S::PITCH + hf * GROUP + k * RT + r];
          }
          const int c4 = (hf * (DH / 2) + c0 + c) / 4;
          const float4 o = held(make_float4(y[0], y[1], y[2], y[3]));
          if (whole) store_row4<DH>(p, b, h, r0 + r, c4, o);
          else __stcg(reinterpret_cast<float4*>(ps + r * DH) + c4, o);
        }
        soft_sync();
      }
      if (*abort_flag && p.status && threadIdx.x == 0) atomicOr(p.status + b, SPACE_ST_TIMEOUT);
      if (!whole) {
        const uint32_t piece0 = cut.owner(item_at + SHARE_COST);
        const int pieces = (int)(cut.owner(item_at + SHARE_COST + T - 1) - piece0) + 1;
        if (threadIdx.x == 0) {
          __threadfence();                           // (after the barrier: for all the stores)
          int* arrived = p.arrived + (b * p.H_kv * p.n_rt + it);
          const int last = atomicAdd(arrived, 1) == pieces - 1;
          if (last) *arrived = 0;                    // ready for the next call
          __threadfence();
          *last_flag = last;
        }
        soft_sync();
        if (*last_flag) join_pieces<DH, RT, 4, 4>(p, cut, b, h, r0, rows, piece0, pieces, item_at, (int)threadIdx.x, SOFT);
        soft_sync();                                 // the flag is free for the next item
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

template <int DH>
size_t smem_bytes(int max_batch) { return Smem<DH>::TABLE_OFF + (size_t)(max_batch + 1) * 4 + (size_t)max_batch * 4; }

template <int DH, int REP>
cudaError_t launch_dim(Params& p, const space_ctx* ctx, cudaStream_t st) {
  static unsigned long long done_mask = 0;           // devices on which the kernel may have its shared memory
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 64 || !((done_mask >> dev) & 1ull)) {
    const cudaError_t e = cudaFuncSetAttribute(kvb_attn_tc_kernel<DH, REP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<DH>(128));
    if (e != cudaSuccess) return e;
    if (dev < 64) done_mask |= 1ull << dev;
  }
  static_assert(TILE / REP <= KVB_SM_ROWS, "a slot per block");
  p.n_rt = (p.n_q * p.G + TILE / REP - 1) / (TILE / REP);
  p.n_groups = ctx->sm_count;
  return launch_pdl(kvb_attn_tc_kernel<DH, REP>, dim3(p.n_groups), dim3(THREADS), smem_bytes<DH>(ctx->cfg.max_batch), st, p, ctx->cfg.max_batch);
}

}  // namespace

int launch_kvb_attn_tc(space_ctx* ctx, kvb::Params& p, cudaStream_t st) {
  const bool wide = ctx->cfg.head_dim == 128;
  // 128 rows of an item take 3600 cycles a page, 64 of them 2400: where they leave few enough of an item empty, and an SM gets enough pages (as many
  // as the table names) that coarser items do not cost more than that (us, 64 / 128 rows: 392 rows of 8 sequences of 8192 keys, 8 heads
  // 303 / 270, with head size 64 256 / 213, 1024 rows of 2 of 16384, 4 heads 178 / 150, 100 rows of 32 of up to 2048, 8 heads 113 / 102: 29 pages an
  // SM and more; 128 rows of 16 of up to 4096, 4 heads 53 / 70, 200 rows of 4 of up to 3000, 8 heads 55 / 62: 14 and 10).
  const int rows = p.n_q * p.G, n64 = (rows + 63) / 64, n128 = (rows + 127) / 128;
  const int64_t pages = (int64_t)p.B * p.H_kv * n128 * p.cache.pages_per_seq;
  const int rep = rows <= 32 ? 4 : 3 * n128 < 2 * n64 && pages >= 20 * (int64_t)ctx->sm_count ? 1 : 2;
  cudaError_t e;
  if (wide) e = rep == 4 ? launch_dim<128, 4>(p, ctx, st) : rep == 2 ? launch_dim<128, 2>(p, ctx, st) : launch_dim<128, 1>(p, ctx, st);
  else e = rep == 4 ? launch_dim<64, 4>(p, ctx, st) : rep == 2 ? launch_dim<64, 2>(p, ctx, st) : launch_dim<64, 1>(p, ctx, st);
  return cuda_ok(e);
}
