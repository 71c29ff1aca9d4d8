// Attention of a step's block rows over the 4-bit cache (space_kvq_attn_step), 8, 16 or 24 query rows at a time.
//
// The mathematics.  A cached row stands for lo + step u, so with the codes as they lie
//   score = c (step_k sum_c q_c u_c + lo_k sum_c q_c),     out = sum_j e_j step_j (u_j - 8) + sum_j e_j (lo_j + 8 step_j):
// the products take bare codes, steps and lowest values are two multiply-adds per score.  A code that is masked out of
// its 32-bit word is already an f16 number, the subnormal u 2^-24 (or u 2^-20 for the nibbles at bits 4..7), which
// the tensor cores take at full rate; the powers of two go into the query row (first product) and into the epilogue
// (second one, whose codes are centred by 8 first: sums of one sign would collect what the tensor core cuts off; without
// it 65536 keys in one piece with even weights were 1.4 % off, and 64 sequences, one input set, took 121 us instead of 127).
// f16 holds a bf16 query row exactly, scaled by a power of two, and the weights e step to 11 bits.  The sums of e and of
// e (lo + 8 step) refer to a bound on the scores so far, the weights to the largest e step of their row so far: a row of V
// that is large and hardly seen costs the others no bits.
//
// The work.  The cache's bytes, (d + 8) per key and head, bind up to 8 rows, unpacking, exponentials and products beyond:
// the keys of all (sequence, kv head, query rows) items form one flat list of 128-key pages, every thread block takes an
// equal share of it, and a page's four blocks of 32 keys go to its four warps.  A warp streams its blocks (contiguous
// 32 d + 256 bytes each) into a ring of its own with bulk copies and never meets another warp until the item ends: two
// of its three stages are in flight.  The products are taken transposed, keys and channels on the sixteen rows of
// m16n8k16 and query rows on its eight columns: the codes are the first operand, in the order in which the cache holds
// them, so a lane's 16 bytes are what it feeds to the tensor core, and nothing is padded beyond eights of query rows (with
// the query rows on the sixteen, the first form, one token of 64 sequences took 195 us).  The second operands lie in shared
// memory (query) or come out of the scores by an 8 x 8 transpose (weights).  Accumulators of 8, 16, 24 query rows and
// 32 keys leave registers for 4, 3, 2 blocks per SM.  The block's own rows are bf16 products, their weights two bf16
// terms each.  The pieces of an item that was cut are joined by the block that stores the last of them, always in the
// same order.
// Rows next to the largest number: where a block of keys holds one its scores are taken 2^-64 times as large and held to
// +-1e38, references are put above the scores, so that no weight passes 1, and sums of V rows are 2^-32 as large.
// Measured, d = 128, three input sets in turn: 64 sequences of 1024 to 16384 keys, 8 kv heads of 4 rows, 136.5 us (0.69 of
// the copy rate: four warps per scheduler issue 0.54 instructions a cycle); one sequence of 131071 keys 42 us, of which the
// pages are 26 (0.9), the start 5 and the join of 74 pieces a head 11; 16 sequences of 512 to 4096 keys, 32 heads, 36 rows 143 us,
// 1.7 us a page of 24 rows and block, two blocks per SM, of which the products are half and 0.37 instructions a cycle is
// what two warps per scheduler give; an item costs 8 us beside its pages.
// Every wait is bounded; an expired wait sets SPACE_ST_TIMEOUT and the block drains and exits.
#include "kvq_attn.cuh"

namespace {
using namespace kvq;
using namespace tc;

// A row's reference moves when a score exceeds it, to 2^8 above that: no e passes 1, so that no e step overflows.
constexpr float REF_SLACK = 8.f;
constexpr int WARPS = PAGE_BLOCKS, THREADS = 32 * WARPS;   // a warp per 32-row block of a page

// NT: query rows of an item in eights.
template <int DH, int NT>
struct Smem {
  static constexpr int RT = 8 * NT;
  // Fixed cost of an item, in pages of the list (16 sequences of 512 to 4096 keys, 32 heads, 36 rows: 168 us with 1, 153
  // with 2, 148 with 4; 16 x 8 heads, 32 rows of 1000 keys: 30.2 with 1, 27.0 with 3; eight rows: no difference).
  static constexpr int SHARE_COST = NT == 1 ? 1 : NT == 2 ? 3 : 4;
  static constexpr int STAGES = 3;
  static constexpr int CTAS = NT == 1 ? 4 : NT == 2 ? 3 : 2;           // per SM
  static constexpr int JOIN = NT == 1 ? 1 : NT == 2 ? 4 : 6;           // query rows of a thread in the join
  static constexpr int RING = STAGES * Fmt<DH>::BLOCK;       // of a warp
  static constexpr int O_PITCH = DH + 4;                     // floats
  static_assert(RT * O_PITCH * 4 <= RING, "a warp's accumulators are parked in its ring once that has run dry");
  static constexpr int V_PITCH = DH * 2 + 16;                // bytes: the block's own V rows
  static_assert(16 * V_PITCH <= RING, "so are the block's V rows");
  static constexpr int Q_OFF = WARPS * RING;                 // [NT][DH / 32][32 lanes] second operands of two k-steps
  static constexpr int SUM_OFF = Q_OFF + NT * (DH / 32) * 512;         // [RT] c * sum of a query row, then [WARPS] largest exponents
  static constexpr int ML_OFF = SUM_OFF + RT * 4 + WARPS * 4;          // [WARPS][RT] {reference, sum}
  static constexpr int BAR_OFF = ML_OFF + WARPS * RT * 8;
  static constexpr int MISC_OFF = BAR_OFF + WARPS * STAGES * 8;
  static constexpr int TABLE_OFF = MISC_OFF + 16;            // prefix[max_batch + 1], seq_len[max_batch]
  static_assert(CTAS * (TABLE_OFF + 129 * 4 + 128 * 4 + 1024) <= 228 * 1024, "blocks of the largest batch that an SM holds");
};

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 halves transposed over the warp
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// Over the eight lanes that hold a query row's keys.
__device__ __forceinline__ float col_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 4));
  v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 8));
  return fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 16));
}
__device__ __forceinline__ float col_sum(float v) {
  v += __shfl_xor_sync(0xFFFFFFFFu, v, 4);
  v += __shfl_xor_sync(0xFFFFFFFFu, v, 8);
  return v + __shfl_xor_sync(0xFFFFFFFFu, v, 16);
}

// State of a warp.  The products are taken transposed, keys (channels) on the sixteen rows of an m16n8k16 and query rows
// on its eight columns: lane (n = lane / 4, t = lane % 4) holds columns 2t and 2t + 1 of every eight query rows.
template <int DH, int NT>
struct Acc {
  float o[DH / 16][NT][4];                           // channels 16 ct + n (+ 8): {row 2t, 2t + 1} each
  float m[NT][2], D[NT][2];                          // reference of the sums (log2 units), that of the accumulators less it (m can be too large for the difference to show in a sum)
  uint64_t l[NT], z[NT];                             // sums of e, of e (lo + 8 step) V_UNIT; pairs of rows 2t, 2t + 1
  uint64_t nref[NT], vinv[NT];                       // -m (0 while there is none, or one far below 0), 2^(6 - D)
  float vtop;                                        // the largest of those
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int ct = 0; ct < DH / 16; ++ct) o[ct][nt][0] = o[ct][nt][1] = o[ct][nt][2] = o[ct][nt][3] = 0.f;
      m[nt][0] = m[nt][1] = D[nt][0] = D[nt][1] = -CUDART_INF_F;
      l[nt] = z[nt] = nref[nt] = pack2(0.f, 0.f);
      vinv[nt] = pack2(0x1p126f, 0x1p126f);
    }
    vtop = 0x1p126f;
  }
  __device__ __forceinline__ void scale_rows(int nt, float f0, float f1) {
#pragma unroll
    for (int ct = 0; ct < DH / 16; ++ct) { o[ct][nt][0] *= f0; o[ct][nt][1] *= f1; o[ct][nt][2] *= f0; o[ct][nt][3] *= f1; }
  }
  // Rows' references raised to 2^8 above mx where that is more than they are; the sums follow.  Returns the factors they took.
  __device__ __forceinline__ float2 raise(int nt, float mx0, float mx1) {
    const float mx[2] = {mx0, mx1};
    float f[2], r[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float n = mx[s] > m[nt][s] ? mx[s] + REF_SLACK : m[nt][s];
      f[s] = m[nt][s] == n ? 1.f : fast_exp2(m[nt][s] - n);
      D[nt][s] -= m[nt][s] == n ? 0.f : n - m[nt][s];
      m[nt][s] = n;
      r[s] = n < FAR_BELOW ? 0.f : -n;
    }
    nref[nt] = pack2(r[0], r[1]);
    const uint64_t f2 = pack2(f[0], f[1]);
    l[nt] = mul2(l[nt], f2); z[nt] = mul2(z[nt], f2);
    return make_float2(f[0], f[1]);
  }
  // 2^(6 - D), bounded: a weight of at least 2^-100 times the bound is over what set_scale lets through
  __device__ __forceinline__ void set_vinv(int nt) {
    float v[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) v[s] = fast_exp2(fminf(6.f - D[nt][s], 126.f));
    vinv[nt] = pack2(v[0], v[1]);
  }
  __device__ __forceinline__ void set_vtop() {
    float a, b;
    unpack2(vinv[0], a, b);
    vtop = fmaxf(a, b);
#pragma unroll
    for (int nt = 1; nt < NT; ++nt) { unpack2(vinv[nt], a, b); vtop = max3(vtop, a, b); }
  }
  // The accumulators' references moved up to the rows' largest weights (relative to m), where those would pass the limit.
  __device__ __forceinline__ void set_scale(int nt, float t0, float t1) {
    const float t[2] = {col_max(t0), col_max(t1)};
    float f[2], v[2];
    unpack2(vinv[nt], v[0], v[1]);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      f[s] = 1.f;
      if (t[s] * v[s] > W_LIMIT) {
        const float n = (float)((int)(__float_as_uint(t[s]) >> 23) - 127);
        f[s] = fast_exp2(D[nt][s] - n);
        D[nt][s] = n;
      }
    }
    scale_rows(nt, f[0], f[1]);
    set_vinv(nt);
  }
};

// The item's query rows as second operands, by all threads: lane (n, t) of a product needs of row n (+ 8 nt) the channels
// t * DH/4 ..; the pair that a code word's mask brings out at bits 0..3 (4..7) of each half is a k-step's first (second)
// half.  f16, scaled by one power of two; returns scale with that undone.
template <int DH, int NT>
struct Query {
  static constexpr int LANES = DH / 8, PER = THREADS / LANES, PASSES = (8 * NT + PER - 1) / PER;   // threads of a row, rows at a time
  uint4 v[PASSES];
  __device__ __forceinline__ void fetch(const Params& p, int b, int h, int r0) {
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
      const int r = k * PER + threadIdx.x / LANES;
      int i, hq;
      row_of(p, h, r0 + r, i, hq);
      v[k] = make_uint4(0, 0, 0, 0);
      if (r < 8 * NT && i < p.n_q)
        v[k] = *(reinterpret_cast<const uint4*>(p.q + (int64_t)b * p.q_sb + (int64_t)i * p.q_sr + (int64_t)hq * p.q_sh) + threadIdx.x % LANES);
    }
  }
};
template <int DH, int NT>
__device__ __forceinline__ float load_query(const Params& p, unsigned char* sm, const Query<DH, NT>& query) {
  using S = Smem<DH, NT>;
  constexpr int LANES = Query<DH, NT>::LANES, PER = Query<DH, NT>::PER, PASSES = Query<DH, NT>::PASSES;
  float* sums = reinterpret_cast<float*>(sm + S::SUM_OFF);
  uint32_t* tops = reinterpret_cast<uint32_t*>(sums + S::RT);
  const int x = threadIdx.x % LANES, lane = threadIdx.x & 31;
  const uint4 (&v)[PASSES] = query.v;
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    uint32_t m = max_bits(v[k]);
    if (m >= 0x7F80u) {                              // a row that is not finite does not set the scale of the others
      m = 0;
      const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
      for (int e = 0; e < 8; ++e) {
        const uint32_t y = (w[e >> 1] >> (16 * (e & 1))) & 0x7FFFu;
        if (y < 0x7F80u) m = max(m, y);
      }
    }
    top = max(top, m);
    float sum = ((bf_lo(v[k].x) + bf_hi(v[k].x)) + (bf_lo(v[k].y) + bf_hi(v[k].y))) + ((bf_lo(v[k].z) + bf_hi(v[k].z)) + (bf_lo(v[k].w) + bf_hi(v[k].w)));
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    const int r = k * PER + threadIdx.x / LANES;
    if (x == 0 && r < S::RT) sums[r] = sum * p.c;
  }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if (lane == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
  static_assert(WARPS == 4, "one word per warp");
  top = max(max(tops[0], tops[1]), max(tops[2], tops[3])) >> 7;
  // largest element in [2^8, 2^9): what f16 drops is 2^-29 of it at most
  const int e = top ? min(max(8 - ((int)top - 127), -100), 100) : 0;
  const float f = pow2(e), f16th = f * 0.0625f;
  const int t = x / (DH / 32), j = x % (DH / 32);    // piece: code word j of the lanes t, k-steps 2 j and 2 j + 1
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    const int r = k * PER + threadIdx.x / LANES;
    const uint4 q = make_uint4(pack_h(bf_lo(v[k].x) * f, bf_lo(v[k].z) * f), pack_h(bf_hi(v[k].x) * f16th, bf_hi(v[k].z) * f16th),
                               pack_h(bf_lo(v[k].y) * f, bf_lo(v[k].w) * f), pack_h(bf_hi(v[k].y) * f16th, bf_hi(v[k].w) * f16th));
    if (r < S::RT) reinterpret_cast<uint4*>(sm + S::Q_OFF)[((r >> 3) * (DH / 32) + j) * 32 + 4 * (r & 7) + t] = q;
  }
  __syncthreads();
  return p.c * pow2(-e);
}

template <int DH, int NT>
__global__ void __launch_bounds__(THREADS, Smem<DH, NT>::CTAS) kvq_attn_kernel(const __grid_constant__ Params p, int max_batch) {
  using F = Fmt<DH>;
  using S = Smem<DH, NT>;
  constexpr int STAGES = S::STAGES, RT = S::RT, SHARE_COST = S::SHARE_COST;
  extern __shared__ __align__(128) unsigned char sm[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane & 3;
  const uint32_t base = smem_u32(sm);
  const uint32_t ring = base + warp * S::RING, bar = base + S::BAR_OFF + warp * STAGES * 8;
  float2* ml = reinterpret_cast<float2*>(sm + S::ML_OFF);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::MISC_OFF);
  int* last_flag = reinterpret_cast<int*>(sm + S::MISC_OFF + 4);
  uint32_t* prefix = reinterpret_cast<uint32_t*>(sm + S::TABLE_OFF);
  int* seq_len = reinterpret_cast<int*>(prefix + max_batch + 1);
  const uint4* qs = reinterpret_cast<const uint4*>(sm + S::Q_OFF) + lane;
  const float* qsum = reinterpret_cast<const float*>(sm + S::SUM_OFF);

  pdl_launch_dependents();
  if (threadIdx.x == 0) *abort_flag = 0;
  if (lane == 0) {
    for (int s = 0; s < STAGES; ++s) mbar_init(bar + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  pdl_wait();
  // Lengths, and the list's running sums: a (sequence, kv head, row block) has a page per 128 keys, one more where the
  // block's own rows are given, at least one (rows without any key still get their zeros), and SHARE_COST ahead.
  auto pages_of = [&](int L) { return max((L + SPACE_PAGE_SIZE - 1) / SPACE_PAGE_SIZE + p.has_new, 1); };
  if (warp == 0) {
    uint32_t carry = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const int b = b0 + lane;
      int L = -1;
      uint32_t n = 0;
      if (b < p.B) {
        L = p.kv_len[b];
        if (L < 0 || (int64_t)L > (int64_t)p.cache.pages_per_seq * SPACE_PAGE_SIZE) {
          if (blockIdx.x == 0 && p.status) atomicOr(p.status + b, SPACE_ST_CAPACITY);
          L = -1;
        }
        n = (uint32_t)((pages_of(max(L, 0)) + SHARE_COST) * p.H_kv * p.n_rt);
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
  __syncthreads();
  const Cut cut(prefix[p.B], p.n_groups);
  if (blockIdx.x >= cut.NG) return;
  uint32_t cur = cut.begin(blockIdx.x);
  const uint32_t share0 = cur, end = cut.begin(blockIdx.x + 1);

  uint32_t step = 0;                                 // blocks of the ring used so far, by this warp
  Acc<DH, NT> acc;
  int b = 0;
  while (cur < end) {
    while (prefix[b + 1] <= cur) ++b;
    const int L0 = seq_len[b], L = max(L0, 0);
    const int T = pages_of(L), Tv = T + SHARE_COST;
    const uint32_t rem = cur - prefix[b];
    const int it = (int)(rem / (uint32_t)Tv), x0 = (int)rem - it * Tv;        // item h * n_rt + row block
    const int h = it / p.n_rt, rt = it - h * p.n_rt;
    const int n_list = min(Tv - x0, (int)(end - cur));
    const uint32_t item_at = cur - x0;               // the item's place in the list
    const bool opens = cur == share0;
    cur += n_list;
    const int t0 = max(x0 - SHARE_COST, 0), t1 = x0 + n_list - SHARE_COST;
    if (t1 <= t0) continue;                          // only the cost of starting: no pages here
    const int r0 = rt * RT;
    const int rows = min(RT, p.n_q * p.G - r0);
    const int Tc = (L + SPACE_PAGE_SIZE - 1) / SPACE_PAGE_SIZE;        // pages of the cache; page Tc is the block's rows
    const int c1 = min(t1, Tc);

    // this warp's blocks: rows [32 warp, +32) of pages t0 .. c1-1; a sequence's last page may leave it none
    const bool over = __any_sync(0xFFFFFFFFu, *abort_flag);
    int n_blk = over ? 0 : max(c1 - t0, 0);          // (after a wait that ran out: no more requests, but every item is counted)
    if (over && p.status && threadIdx.x == 0) atomicOr(p.status + b, SPACE_ST_TIMEOUT);
    if (n_blk > 0 && L - (c1 - 1) * SPACE_PAGE_SIZE <= warp * BLOCK_ROWS) --n_blk;
    const int32_t* table = p.cache.page_table + (int64_t)b * p.cache.pages_per_seq;
    const char* head = p.cache.pool + (int64_t)h * p.cache.head_stride + warp * F::BLOCK;
    int pages = 0, pages0 = -32;                     // lane j: page of tile t0 + pages0 + j
    uint32_t good = 0;                               // bit j: that page is in the pool
    auto look = [&](int j) {                         // pages of the 32 tiles that tile j is among (converged warp)
      if (j - pages0 < 32) return;
      pages0 = j;
      const int at = t0 + j + lane;
      pages = (j + lane < n_blk && at < p.cache.pages_per_seq) ? table[at] : -1;
      const bool ok = pages >= 0 && pages < p.cache.n_pages;
      good = __ballot_sync(0xFFFFFFFFu, ok);
      if (!ok && j + lane < n_blk && p.status) atomicOr(p.status + b, SPACE_ST_BAD_PAGE);
    };
    // (requests run STAGES - 1 blocks ahead of the products, so they look pages up first; whether the page was good
    // travels with the request as a bit per stage)
    uint32_t staged = 0;
    auto request = [&](int j, uint32_t at) {
      if (j >= n_blk) return;
      look(j);
      const int pg = __shfl_sync(0xFFFFFFFFu, pages, j - pages0);
      const uint32_t s = at % STAGES;
      const bool ok = (good >> (j - pages0)) & 1u;
      staged = (staged & ~(1u << s)) | (uint32_t)ok << s;
      if (lane == 0) {
        if (ok) {
          mbar_expect_tx(bar + 8 * s, F::BLOCK);
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                       ::"r"(ring + s * F::BLOCK), "l"(head + (int64_t)pg * p.cache.page_stride), "r"(F::BLOCK), "r"(bar + 8 * s) : "memory");
        } else {
          mbar_arrive(bar + 8 * s);
        }
      }
    };
    Query<DH, NT> query;
    query.fetch(p, b, h, r0);                        // (ahead of the requests, which wait for the page table)
#pragma unroll 1
    for (int j = 0; j < STAGES - 1; ++j) request(j, step + j);

    const float qc = load_query<DH, NT>(p, sm, query);
    uint64_t sum[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) sum[nt] = *reinterpret_cast<const uint64_t*>(qsum + 8 * nt + 2 * t);
    acc.clear();
    bool unset = true;                               // a row has no reference yet, or one far below 0
    for (int j = 0; j < n_blk; ++j, ++step) {
      request(j + STAGES - 1, step + STAGES - 1);
      const uint32_t s = step % STAGES, parity = (step / STAGES) & 1;
      if (!warp_wait(bar + 8 * s, parity, abort_flag, p.err, 40 + warp)) {
        if (p.status && lane == 0) atomicOr(p.status + b, SPACE_ST_TIMEOUT);
        // what is on its way has to land before the ring is used for anything else
        const uint32_t issued = step + min(STAGES, n_blk - j);
        for (; step < issued; ++step) mbar_drain_bounded(bar + 8 * (step % STAGES), (step / STAGES) & 1, WAIT_NS);
        break;
      }
      if (!((staged >> s) & 1u)) continue;           // a page outside the pool: its keys are left out
      const uint32_t blk = ring + s * F::BLOCK;
      const int valid = min(L - (t0 + j) * SPACE_PAGE_SIZE - warp * BLOCK_ROWS, BLOCK_ROWS);   // keys of this block, >= 1

      // ---- S^T = U Q^T: keys 16 mt + lane / 4 (+ 8) of the block are the rows of product mt
      float sc[2][NT][4];
      uint32_t kw[4][DH / 32];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t at = blk + (8 * i + (lane >> 2)) * (DH / 2) + t * (DH / 8);
        if (DH == 128) {
          const uint4 v = lds128(at);
          kw[i][0] = v.x; kw[i][1] = v.y; kw[i][2 % (DH / 32)] = v.z; kw[i][3 % (DH / 32)] = v.w;
        } else {
          const uint2 v = lds64(at);
          kw[i][0] = v.x; kw[i][1] = v.y;
        }
      }
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sc[mt][nt][0] = sc[mt][nt][1] = sc[mt][nt][2] = sc[mt][nt][3] = 0.f;
#pragma unroll
      for (int k = 0; k < DH / 32; ++k) {
        uint4 q[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) q[nt] = qs[(nt * (DH / 32) + k) * 32];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            const uint32_t x = half ? kw[2 * mt][k] >> 8 : kw[2 * mt][k], y = half ? kw[2 * mt + 1][k] >> 8 : kw[2 * mt + 1][k];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              mma(sc[mt][nt], x & 0x000F000Fu, y & 0x000F000Fu, x & 0x00F000F0u, y & 0x00F000F0u, half ? q[nt].z : q[nt].x, half ? q[nt].w : q[nt].y);
          }
      }
      // ---- steps and lowest values of keys 8 i + lane / 4; scores relative to the rows' references
      uint64_t vs[4], vz[4];
      float mx = -CUDART_INF_F, vmax = 0.f;
      const float c24 = qc * 16777216.f;            // undoes the codes' 2^-24
      uint32_t kp[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = 8 * i + (lane >> 2);
        kp[i] = lds32(blk + F::K_PAR + key * 4);
        const uint32_t vp = lds32(blk + F::V_PAR + key * 4);
        const float v1 = bf_lo(vp), v0 = fmaf(v1, 8.f * V_UNIT, bf_hi(vp) * V_UNIT);
        vs[i] = pack2(v1, v1); vz[i] = pack2(v0, v0);
      }
      if (__any_sync(0xFFFFFFFFu, fmaxf(max3(bf_lo(kp[0]), bf_lo(kp[1]), bf_lo(kp[2])), bf_lo(kp[3])) * c24 > K_LARGE)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float k1 = bf_lo(kp[i]) * 0x1p-64f * c24, k0 = bf_hi(kp[i]) * 0x1p-64f;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float s[2], r[2];
            unpack2(sum[nt], s[0], s[1]);
            unpack2(acc.nref[nt], r[0], r[1]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& x = sc[i >> 1][nt][2 * (i & 1) + e];
              x = clamp_score(fmaf(x, k1, k0 * s[e]) * 0x1p64f) + r[e];
            }
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float k1 = bf_lo(kp[i]) * c24, k0 = bf_hi(kp[i]);
          const uint64_t k1p = pack2(k1, k1), k0p = pack2(k0, k0);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float* x = &sc[i >> 1][nt][2 * (i & 1)];
            unpack2(fma2(pack2(x[0], x[1]), k1p, fma2(k0p, sum[nt], acc.nref[nt])), x[0], x[1]);
          }
        }
      }
      if (valid < BLOCK_ROWS) {                      // rows past the end may hold anything
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (8 * i + (lane >> 2) >= valid) {
            vs[i] = vz[i] = pack2(0.f, 0.f);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sc[i >> 1][nt][2 * (i & 1)] = sc[i >> 1][nt][2 * (i & 1) + 1] = -CUDART_INF_F;
          }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v1, v1_;
        unpack2(vs[i], v1, v1_);
        vmax = fmaxf(vmax, v1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mx = max3(mx, sc[i >> 1][nt][2 * (i & 1)], sc[i >> 1][nt][2 * (i & 1) + 1]);
      }
      // the references move when a score exceeds them, or while a row has none (or one far below 0)
      if (__any_sync(0xFFFFFFFFu, unset || mx > 0.f)) {
        unset = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float a0 = -CUDART_INF_F, a1 = -CUDART_INF_F, r0_, r1_;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            a0 = fmaxf(a0, sc[i >> 1][nt][2 * (i & 1)]); a1 = fmaxf(a1, sc[i >> 1][nt][2 * (i & 1) + 1]);
          }
          unpack2(acc.nref[nt], r0_, r1_);
          acc.raise(nt, col_max(a0) - r0_, col_max(a1) - r1_);
          acc.set_vinv(nt);
          unset |= acc.m[nt][0] < FAR_BELOW || acc.m[nt][1] < FAR_BELOW;
          // (without the old reference, then less the new one, whose scores are these: a difference of two references would
          // have the rounding of their size, and could leave the largest score above its own reference)
          float n0 = acc.m[nt][0] == -CUDART_INF_F ? 0.f : -acc.m[nt][0], n1 = acc.m[nt][1] == -CUDART_INF_F ? 0.f : -acc.m[nt][1];
          if (n0 == r0_) n0 = r0_ = 0.f;
          if (n1 == r1_) n1 = r1_ = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float &x0 = sc[i >> 1][nt][2 * (i & 1)], &x1 = sc[i >> 1][nt][2 * (i & 1) + 1];
            x0 = (x0 - r0_) + n0; x1 = (x1 - r1_) + n1;
          }
        }
        acc.set_vtop();
        mx = 0.f;                                    // (none is above its reference now; a first reference can also have moved the scores up)
      }
      // ---- could a weight pass the limit?  By a bound, the largest e times the largest step and factor of the lane; then
      // by the weights themselves
      if (__any_sync(0xFFFFFFFFu, fast_exp2(mx) * vmax * acc.vtop > W_LIMIT)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float t0 = 0.f, t1 = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v1, v1_;
            unpack2(vs[i], v1, v1_);
            t0 = fmaxf(t0, fast_exp2(sc[i >> 1][nt][2 * (i & 1)]) * v1); t1 = fmaxf(t1, fast_exp2(sc[i >> 1][nt][2 * (i & 1) + 1]) * v1);
          }
          acc.set_scale(nt, t0, t1);
        }
        acc.set_vtop();
      }
      // ---- e, its sums, and the weights e step in f16
      uint32_t pb[2][NT][2];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint64_t e = pack2(fast_exp2(sc[i >> 1][nt][2 * (i & 1)]), fast_exp2(sc[i >> 1][nt][2 * (i & 1) + 1]));
          acc.l[nt] = add2(acc.l[nt], e);
          acc.z[nt] = fma2(e, vz[i], acc.z[nt]);
          float w0, w1;
          unpack2(mul2(mul2(e, vs[i]), acc.vinv[nt]), w0, w1);
          pb[i >> 1][nt][i & 1] = transpose8(pack_h(w0, w1));
        }
      // ---- O^T += (U - 8)^T P^T: channels 16 (2 wd + ct) + lane / 4 (+ 8) are the rows
#pragma unroll
      for (int wd = 0; wd < DH / 32; ++wd) {
        const uint4 v = lds128(blk + F::CODES + 512 * wd + 16 * lane);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        const uint32_t c0 = 0x00080008u, c1_ = 0x00800080u;                    // 8 in units of 2^-24 and 2^-20
#pragma unroll
        for (int a = 0; a < 2; ++a) {
#pragma unroll
          for (int ct = 0; ct < 2; ++ct) {
            const uint32_t x = ct ? w[2 * a] >> 8 : w[2 * a], y = ct ? w[2 * a + 1] >> 8 : w[2 * a + 1];
            const uint32_t a0 = h2sub(x & 0x000F000Fu, c0), a1 = h2sub(x & 0x00F000F0u, c1_);
            const uint32_t a2 = h2sub(y & 0x000F000Fu, c0), a3 = h2sub(y & 0x00F000F0u, c1_);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma(acc.o[2 * wd + ct][nt], a0, a1, a2, a3, pb[a][nt][0], pb[a][nt][1]);
          }
        }
      }
      __syncwarp();                                  // the stage is free for the next request
    }
    // ---- sums over the lanes, accumulators in units of V_UNIT
    float ls[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float f[2], z[2];
      unpack2(acc.l[nt], ls[nt][0], ls[nt][1]);
      unpack2(acc.z[nt], z[0], z[1]);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        f[s] = acc.D[nt][s] == -CUDART_INF_F ? 1.f : fast_exp2(acc.D[nt][s] - 6.f);
        ls[nt][s] = col_sum(ls[nt][s]);
        z[s] = col_sum(z[s]);
      }
#pragma unroll
      for (int ct = 0; ct < DH / 16; ++ct)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc.o[ct][nt][e] = fmaf(acc.o[ct][nt][e] * ((e >= 2 ? 0x1p20f : 0x1p24f) * V_UNIT), f[e & 1], z[e & 1]);
    }

    // ---- the block's own rows: keys 16 warp .. + 15 of it, products in bf16 as they are (no code, no scale), weights as two
    // bf16 terms
    if (t1 > Tc && p.has_new && 16 * warp < p.n_q && L0 >= 0) {
      const int k0 = 16 * warp;
      constexpr int LANES = DH / 8, V_LOADS = 16 * LANES / 32;
      uint4 kr[2][DH / 32], vr[V_LOADS], qr[NT][DH / 32];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        int i, hq;
        row_of(p, h, r0 + 8 * nt + (lane >> 2), i, hq);
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)b * p.q_sb + (int64_t)i * p.q_sr + (int64_t)hq * p.q_sh) + t * (DH / 32);
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) qr[nt][j] = i < p.n_q ? src[j] : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int key = k0 + 8 * i + (lane >> 2);
        const uint4* src = reinterpret_cast<const uint4*>(p.kn + (int64_t)b * p.n_sb + (int64_t)key * p.n_sr + (int64_t)h * p.n_sh) + t * (DH / 32);
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) kr[i][j] = key < p.n_q ? src[j] : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < V_LOADS; ++i) {
        const int key = k0 + i * (32 / LANES) + lane / LANES;
        vr[i] = make_uint4(0, 0, 0, 0);
        if (key < p.n_q) vr[i] = *(reinterpret_cast<const uint4*>(p.vn + (int64_t)b * p.n_sb + (int64_t)key * p.n_sr + (int64_t)h * p.n_sh) + lane % LANES);
      }
      float sc[NT][4], kf[2] = {p.c, p.c};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) top = max(top, max_bits(kr[i][j]));
        if (__any_sync(0xFFFFFFFFu, top >= 0x7200u)) { // (from 2^101 on: what is not finite, and sums that fp32 would not hold)
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
#pragma unroll
          for (int j = 0; j < DH / 32; ++j) {
            make_finite(kr[i][j]);
            if (top >= 0x7200u) kr[i][j] = scale_bf16(kr[i][j], 0x1p-64f);
          }
          if (top >= 0x7200u) kf[i] = p.c * 0x1p64f;
        }
      }
#pragma unroll
      for (int k = 0; k < DH / 32; ++k) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint4 q = qr[nt][k];
          mma_bf16(sc[nt], kr[0][k].x, kr[1][k].x, kr[0][k].y, kr[1][k].y, q.x, q.y);
          mma_bf16(sc[nt], kr[0][k].z, kr[1][k].z, kr[0][k].w, kr[1][k].w, q.z, q.w);
        }
      }
#pragma unroll
      for (int i = 0; i < V_LOADS; ++i) {            // V rows into the (dry) ring
        make_finite(vr[i]);
        const uint32_t at = ring + (i * (32 / LANES) + lane / LANES) * S::V_PITCH + (lane % LANES) * 16;
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(vr[i].x), "r"(vr[i].y), "r"(vr[i].z), "r"(vr[i].w) : "memory");
      }
      __syncwarp();
      uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float mx[2] = {-CUDART_INF_F, -CUDART_INF_F}, lb[2] = {0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int r = r0 + 8 * nt + 2 * t + s;
          const uint64_t see = r < p.n_q * p.G ? p.mask[r >> p.gsh] : 0ull;    // Eq. 5
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float& x = sc[nt][2 * i + s];
            const bool vis = (see >> (k0 + 8 * i + (lane >> 2))) & 1ull;
            x *= kf[i];                              // (rows next to the largest number: a score stays one, and NaN NaN)
            x = vis ? clamp_score(x) : -CUDART_INF_F;
            mx[s] = fmaxf(mx[s], x);
          }
        }
        const float2 down = acc.raise(nt, col_max(mx[0]), col_max(mx[1]));
        ls[nt][0] *= down.x; ls[nt][1] *= down.y;
        if (__any_sync(0xFFFFFFFFu, down.x != 1.f || down.y != 1.f)) acc.scale_rows(nt, down.x, down.y);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float e0 = sc[nt][2 * i] == -CUDART_INF_F ? 0.f : fast_exp2(sc[nt][2 * i] - acc.m[nt][0]);
          const float e1 = sc[nt][2 * i + 1] == -CUDART_INF_F ? 0.f : fast_exp2(sc[nt][2 * i + 1] - acc.m[nt][1]);
          lb[0] += e0; lb[1] += e1;
          const float w0 = e0 * V_UNIT, w1 = e1 * V_UNIT;
          const __nv_bfloat162 hi = __floats2bfloat162_rn(w0, w1);
          const uint32_t hw = *reinterpret_cast<const uint32_t*>(&hi);
          float l0, l1;
          low_terms(hw, w0, w1, l0, l1);
          const __nv_bfloat162 lo = __floats2bfloat162_rn(l0, l1);
          ph[nt][i] = transpose8(hw);
          pl[nt][i] = transpose8(*reinterpret_cast<const uint32_t*>(&lo));
        }
        ls[nt][0] += col_sum(lb[0]); ls[nt][1] += col_sum(lb[1]);
      }
#pragma unroll
      for (int ct = 0; ct < DH / 16; ++ct) {
        uint32_t a0, a1, a2, a3;
        const uint32_t at = ring + (8 * (lane >> 4) + (lane & 7)) * S::V_PITCH + ct * 32 + ((lane >> 3) & 1) * 16;
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(a0), "=r"(a1), "=r"(a2), "=r"(a3) : "r"(at) : "memory");
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma_bf16(acc.o[ct][nt], a0, a1, a2, a3, ph[nt][0], ph[nt][1]);
          mma_bf16(acc.o[ct][nt], a0, a1, a2, a3, pl[nt][0], pl[nt][1]);
        }
      }
      __syncwarp();
    }

    // ---- the four warps' states meet
    if (lane < 4) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) ml[warp * RT + 8 * nt + 2 * t + e] = make_float2(acc.m[nt][e], ls[nt][e]);
    }
    __syncthreads();
    const bool whole = t0 == 0 && t1 == T;
    {
      float* mine = reinterpret_cast<float*>(sm + warp * S::RING);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = 8 * nt + 2 * t + e;
          float M = -CUDART_INF_F;
#pragma unroll
          for (int w = 0; w < WARPS; ++w) M = fmaxf(M, ml[w * RT + r].x);
          float f = acc.m[nt][e] == -CUDART_INF_F ? 0.f : fast_exp2(acc.m[nt][e] - M);
          if (ls[nt][e] != ls[nt][e]) f = 1.f;       // (a row that is not a number keeps no reference; its sums say so)
#pragma unroll
          for (int ct = 0; ct < DH / 16; ++ct) {
            mine[r * S::O_PITCH + 16 * ct + (lane >> 2)] = acc.o[ct][nt][e] * f;
            mine[r * S::O_PITCH + 16 * ct + 8 + (lane >> 2)] = acc.o[ct][nt][2 + e] * f;
          }
        }
    }
    __syncthreads();
    uint32_t piece0 = 0;
    int pieces = 1;
    if (!whole) {
      piece0 = cut.owner(item_at + SHARE_COST);
      pieces = (int)(cut.owner(item_at + SHARE_COST + T - 1) - piece0) + 1;
    }
    const int slot = 2 * (int)blockIdx.x + (opens ? 0 : 1);
    constexpr int C4 = DH / 4;
    constexpr int SLOT = RT * (DH + 2);
    for (int idx = threadIdx.x; idx < rows * C4; idx += THREADS) {
      const int r = idx / C4, c4 = idx % C4;
      float M = -CUDART_INF_F, l = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) M = fmaxf(M, ml[w * RT + r].x);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float2 v = ml[w * RT + r];
        l += v.y * (v.x == -CUDART_INF_F ? (v.y != v.y ? 1.f : 0.f) : fast_exp2(v.x - M));
        const float4 x = *reinterpret_cast<const float4*>(sm + w * S::RING + (r * S::O_PITCH + 4 * c4) * 4);
        o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
      }
      if (whole) {
        store_row4<DH>(p, b, h, r0 + r, c4, o, M, l);
      } else {
        float* ps = p.part + (int64_t)slot * SLOT;
        __stcg(reinterpret_cast<float4*>(ps + r * DH) + c4, o);
        if (c4 == 0) { __stcg(ps + RT * DH + r, M); __stcg(ps + RT * DH + RT + r, l); }
      }
    }
    if (!whole) {
      const int item = (b * p.H_kv + h) * p.n_rt + rt;
      __syncthreads();
      if (threadIdx.x == 0) {
        __threadfence();                             // (after the barrier: for the whole block's stores)
        const int last = atomicAdd(p.arrived + item, 1) == pieces - 1;
        if (last) p.arrived[item] = 0;               // ready for the next call
        __threadfence();
        *last_flag = last;
      }
      __syncthreads();
      if (*last_flag) {
        join_pieces<DH, RT, S::JOIN, NT == 1 ? 16 : 4>(p, cut, b, h, r0, rows, piece0, pieces, item_at, (int)threadIdx.x, THREADS);
      }
    }
    __syncthreads();                                 // everybody has read the rings: the next item's requests may fill them
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
}

template <int DH, int NT>
size_t smem_bytes(int max_batch) { return Smem<DH, NT>::TABLE_OFF + (size_t)(max_batch + 1) * 4 + (size_t)max_batch * 4; }

template <int DH, int NT>
cudaError_t launch_dim(Params& p, const space_ctx* ctx, cudaStream_t st) {
  static unsigned long long done_mask = 0;           // devices on which the kernel may have its shared memory
  const int max_batch = ctx->cfg.max_batch;
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 64 || !((done_mask >> dev) & 1ull)) {
    cudaFuncSetAttribute(kvq_attn_kernel<DH, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<DH, NT>(128));
    if (dev < 64) done_mask |= 1ull << dev;
  }
  static_assert(Smem<DH, NT>::CTAS * 8 * NT <= KVQ_SM_ROWS, "a slot per block");
  p.n_rt = (p.n_q * p.G + 8 * NT - 1) / (8 * NT);
  p.n_groups = Smem<DH, NT>::CTAS * ctx->sm_count;
  return launch_pdl(kvq_attn_kernel<DH, NT>, dim3(p.n_groups), dim3(THREADS), smem_bytes<DH, NT>(max_batch), st, p, max_batch);
}

}  // namespace

int launch_kvq_attn(space_ctx* ctx, const space_kvq_attn_args* a, const uint64_t* mask_rows, cudaStream_t st) {
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
  p.part = ctx->attn_part; p.arrived = ctx->kvq_arrived; p.err = ctx->counters + 3 * ctx->cfg.max_batch;
  for (int i = 0; i < p.n_q; ++i) p.mask[i] = mask_rows[i];
  const int rows = p.n_q * p.G;
  // the flat list is counted in 32 bits: items of eight rows at least, a page and the cost of starting more than a table names
  if ((double)p.B * p.H_kv * ((rows + 7) / 8) * ((double)p.cache.pages_per_seq + 4) > 2e9) return SPACE_E_UNSUPPORTED;
  ctx->launches += 1;
  // Which form.  A page costs 16 rows here 3 units, 24 rows 4, and in the tensor-memory form 64 rows 9 (what its items cost
  // beside their pages counted in; 48 rows would cost 8 and never be the cheapest); eight rows are the cheapest there are.  16 sequences x 16
  // heads of 2000 keys, us, by 8 / 16 / 24 rows: 8 rows 29.5 / 35 / 40, 16 rows 43 / 38 / 42, 18 rows 58 / 56 / 44, 32
  // rows 74 / 58 / 74, 36 rows 89 / 85 / 78; here / there: 50 rows 70 / 61 (1000 keys), 64 rows 109 / 85, 100 rows 170 / 149,
  // but 72 rows (8 x 8 heads, 3000 keys) 45 / 53 and 36 rows (16 x 32, up to 4096) 145 / 160.
  const int in16 = 3 * ((rows + 15) / 16), in24 = 4 * ((rows + 23) / 24);
  // It has one block per SM, so it also wants pages for each: at nine pages' worth an SM 54 / 52, at five 33 / 40.  (The
  // lengths are on the device: the table's width stands for them.)
  const int blocks = (rows + 63) / 64;
  if (9 * blocks < min(in16, in24) && (int64_t)p.B * p.H_kv * blocks * p.cache.pages_per_seq >= 8 * (int64_t)ctx->sm_count)
    return launch_kvq_attn_tc(ctx, p, st);
  const bool wide = ctx->cfg.head_dim == 128;
  const int nt = rows <= 8 ? 1 : in24 < in16 ? 3 : 2;
  cudaError_t e;
  if (wide) e = nt == 1 ? launch_dim<128, 1>(p, ctx, st) : nt == 2 ? launch_dim<128, 2>(p, ctx, st) : launch_dim<128, 3>(p, ctx, st);
  else e = nt == 1 ? launch_dim<64, 1>(p, ctx, st) : nt == 2 ? launch_dim<64, 2>(p, ctx, st) : launch_dim<64, 3>(p, ctx, st);
  return cuda_ok(e);
}
