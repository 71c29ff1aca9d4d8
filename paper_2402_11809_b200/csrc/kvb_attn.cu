// Attention of a step's block rows over the 8-bit cache (space_kvb_attn_step), up to sixteen query rows of a kv head.
//
// The mathematics.  The cache's codes are tensor-core operands as they lie (mma.sync m16n8k32, e4m3): nothing is unpacked.
// What they are multiplied with is split in two: a query row, scaled by a power of two of its own, is q0 + q1 with e4m3 numbers (four
// bits each: bf16 has eight), and so is a weight.
//   S = K q0 + K q1,   D = V^T w0 + V^T w1     for the 32 keys of a block, which share a K and a V scale 2^k, 2^v:
//   e_j = 2^(s_j - r), r the block's largest score less 8,   l += 2^(r - M) sum_j e_j,   o = o 2^(R - R') + D 2^(v + (r - M) - R')
// with M the running maximum of r and R' the larger of R and v + (r - M): weights are always taken relative to the largest of
// their own block, whatever other blocks hold, V rows that are large and hardly seen cost the others no bits, and only
// differences of scores are added to exponents of scales, so that large scores cost none.
//
// The work.  The keys of all (sequence, kv head, query rows) items form one flat list of 128-key pages, every thread block takes an
// equal share of it, and a page's four blocks of 32 keys go to its four warps.  A warp streams its blocks into a ring of its own with
// bulk copies and never meets another warp until the item ends.  The products are taken transposed, keys (channels) on
// the sixteen rows and query rows on the eight columns.  Which key and which channel stand where in a product is free as long as both
// operands agree: a lane takes 16 bytes of a K row at a time (four products' worth), 8 bytes of a V channel, and the
// weights' codes change lanes by an 8 x 8 transpose.  The block's own rows are bf16 products, their weights two bf16 terms each.
// The pieces of an item that was cut are joined by the block that stores the last of them, always in the same order.
// Every wait is bounded; an expired wait sets SPACE_ST_TIMEOUT and the block drains and exits.
//
// What bounds it: 64 sequences of up to 16384 keys, 8 heads of four rows: 227 us, 5.0 TB/s (0.76 of the copy rate), 54 % of the issue slots,
// the tensor pipe 31 % of its; with sixteen rows the chain of a block (products, maximum over the lanes, weights, products) with two warps
// to a scheduler (255 registers a thread, 16 bytes spilled; of up to eight rows 168 and 20).
#include "kvb_attn.cuh"

namespace {
using namespace kvb;

constexpr int WARPS = PAGE_BLOCKS, THREADS = 32 * WARPS;   // a warp per 32-row block of a page
constexpr float REF_FAR = 0x1p22f;                   // up to this a reference's rounding moves weights by 2^0.25 at most
constexpr int ROW_LARGE = 58;                        // (of smaller rows no sum of 128 products passes 2^123)
constexpr float ROW_DOWN = 0x1p-70f;

// NT: query rows of an item in eights.
template <int DH, int NT>
struct Smem {
  using F = Fmt<DH>;
  static constexpr int RT = 8 * NT;
  static constexpr int SHARE_COST = 2;                       // fixed cost of an item, in pages of the list
  static constexpr int STAGES = NT == 1 ? 2 : 3;
  static constexpr int CTAS = NT == 1 ? 3 : 2;               // per SM
  static constexpr int K_PITCH = 16 * BLOCK_ROWS + 16;       // bytes between sixteens of K channels: a lane quad reaches different banks
  static constexpr int V_PITCH = F::V_ROWS + 64;             // between sixteens of V rows
  static constexpr int V_AT = DH / 16 * K_PITCH;
  static constexpr int SCALE_AT = V_AT + 2 * V_PITCH;        // {K, V} scales of this block and its neighbour
  static constexpr int BLOCK = SCALE_AT + 16;
  static constexpr int RING = STAGES * BLOCK;                // of a warp
  static constexpr int O_PITCH = DH + 4;                     // floats
  static_assert(RT * O_PITCH * 4 <= RING, "a warp's accumulators are parked in its ring once that has run dry");
  static constexpr int OWN_PITCH = DH * 2 + 16;              // bytes: the block's own V rows
  static_assert(16 * OWN_PITCH <= RING, "so are the block's V rows");
  static constexpr int Q_PITCH = DH;                         // bytes: rows of one term (of 128 channels, odd rows with halves exchanged: eight lanes reach different banks)
  static constexpr int Q_OFF = WARPS * RING;                 // [2][RT]
  static constexpr int QF_OFF = Q_OFF + 2 * RT * Q_PITCH;    // [RT] factors of the rows' scores, NaN: the row holds a NaN or infinity
  static constexpr int ML_OFF = QF_OFF + RT * 4;             // [WARPS][RT] {M, l}
  static constexpr int BAR_OFF = ML_OFF + WARPS * RT * 8;
  static constexpr int MISC_OFF = BAR_OFF + WARPS * STAGES * 8;
  static constexpr int TABLE_OFF = MISC_OFF + 16;            // prefix[max_batch + 1], seq_len[max_batch]
  static_assert(CTAS * (TABLE_OFF + 129 * 4 + 128 * 4 + 1024) <= 228 * 1024, "blocks of the largest batch that an SM holds");
};

__device__ __forceinline__ void mma8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 halves transposed over the warp
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// Lane (n, t) has word n of the columns 2t and 2t + 1; it gets words 2t and 2t + 1 of column n.
__device__ __forceinline__ void transpose_words(uint32_t x, uint32_t y, uint32_t& a, uint32_t& b) {
  const uint32_t lo = transpose8(__byte_perm(x, y, 0x5410)), hi = transpose8(__byte_perm(x, y, 0x7632));
  a = __byte_perm(lo, hi, 0x5410);
  b = __byte_perm(lo, hi, 0x7632);
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

// State of a warp: lane (n = lane / 4, t = lane % 4) holds columns 2t and 2t + 1 of every eight query rows.
template <int DH, int NT>
struct Acc {
  float o[DH / 16][NT][4];                           // channels 16 ct + n (+ 8): {row 2t, 2t + 1} each
  float M[NT][2], R[NT][2], l[NT][2];                // (l: of this lane's keys)
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int ct = 0; ct < DH / 16; ++ct) o[ct][nt][0] = o[ct][nt][1] = o[ct][nt][2] = o[ct][nt][3] = 0.f;
#pragma unroll
      for (int s = 0; s < 2; ++s) { M[nt][s] = -CUDART_INF_F; R[nt][s] = l[nt][s] = 0.f; }
    }
  }
  // A block of keys with references r, this lane's sums of weights and V's exponent v joins: the accumulators move to the new
  // references, and beta are the factors of the block's results.  (r = -infinity: the row sees none of it.)
  __device__ __forceinline__ void join(const float (&r)[NT][2], const float (&sum)[NT][2], float v, float (&beta)[NT][2]) {
    float a[NT][2];
    bool move = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const float Mn = fmaxf(M[nt][s], r[nt][s]);
        const bool none = r[nt][s] == -CUDART_INF_F;
        const float down = M[nt][s] == Mn ? 0.f : M[nt][s] - Mn, up = none ? 0.f : r[nt][s] - Mn;
        l[nt][s] = fmaf(l[nt][s], fast_exp2(down), none ? 0.f : sum[nt][s] * fast_exp2(up));
        const float r_old = R[nt][s] + down, r_new = v + up, Rn = none ? r_old : fmaxf(r_old, r_new);
        a[nt][s] = r_old - Rn;
        move = move || a[nt][s] != 0.f;
        beta[nt][s] = none ? 0.f : fast_exp2(r_new - Rn);
        M[nt][s] = Mn; R[nt][s] = Rn;
      }
    if (__any_sync(0xFFFFFFFFu, move)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float f0 = fast_exp2(a[nt][0]), f1 = fast_exp2(a[nt][1]);
#pragma unroll
        for (int ct = 0; ct < DH / 16; ++ct) { o[ct][nt][0] *= f0; o[ct][nt][1] *= f1; o[ct][nt][2] *= f0; o[ct][nt][3] *= f1; }
      }
    }
  }
};

// The item's query rows as two terms in shared memory, by all threads: DH / 8 of them a row.
template <int DH, int NT>
struct Query {
  static constexpr int LANES = DH / 8, PER = THREADS / LANES, PASSES = (8 * NT + PER - 1) / PER;   // rows at a time
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
  __device__ __forceinline__ void store(const Params& p, unsigned char* sm) const {
    using S = Smem<DH, NT>;
    const int x = threadIdx.x % LANES;
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
      const int r = k * PER + threadIdx.x / LANES;
      uint32_t top = kvq::max_bits(v[k]);
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
      const bool nan = top >= 0x7F80u;
      const int e = nan ? 0 : max((int)(top >> 7) - 127, -100) - 7;            // the largest element to [2^7, 2^8)
      const float up = nan ? 0.f : pow2(-e);
      uint32_t w0[2], w1[2];
      split4(kvq::bf_lo(v[k].x) * up, kvq::bf_hi(v[k].x) * up, kvq::bf_lo(v[k].y) * up, kvq::bf_hi(v[k].y) * up, w0[0], w1[0]);
      split4(kvq::bf_lo(v[k].z) * up, kvq::bf_hi(v[k].z) * up, kvq::bf_lo(v[k].w) * up, kvq::bf_hi(v[k].w) * up, w0[1], w1[1]);
      if (r < S::RT) {
        unsigned char* to = sm + S::Q_OFF + r * S::Q_PITCH + (8 * x ^ (DH == 128 ? (r & 1) * 64 : 0));
        *reinterpret_cast<uint2*>(to) = nan ? make_uint2(0, 0) : make_uint2(w0[0], w0[1]);
        *reinterpret_cast<uint2*>(to + S::RT * S::Q_PITCH) = nan ? make_uint2(0, 0) : make_uint2(w1[0], w1[1]);
        if (x == 0) reinterpret_cast<float*>(sm + S::QF_OFF)[r] = nan ? __int_as_float(0x7FFFFFFF) : p.c * pow2(e);
      }
    }
  }
};

template <int DH, int NT>
__global__ void __launch_bounds__(THREADS, Smem<DH, NT>::CTAS) kvb_attn_kernel(const __grid_constant__ Params p, int max_batch) {
  using F = Fmt<DH>;
  using S = Smem<DH, NT>;
  constexpr int STAGES = S::STAGES, RT = S::RT, SHARE_COST = S::SHARE_COST;
  extern __shared__ __align__(128) unsigned char sm[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane & 3, n8 = lane >> 2;
  const uint32_t base = smem_u32(sm);
  const uint32_t ring = base + warp * S::RING, bar = base + S::BAR_OFF + warp * STAGES * 8;
  float2* ml = reinterpret_cast<float2*>(sm + S::ML_OFF);
  const float* qf = reinterpret_cast<const float*>(sm + S::QF_OFF);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::MISC_OFF);
  int* last_flag = reinterpret_cast<int*>(sm + S::MISC_OFF + 4);
  uint32_t* prefix = reinterpret_cast<uint32_t*>(sm + S::TABLE_OFF);
  int* seq_len = reinterpret_cast<int*>(prefix + max_batch + 1);

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
    // A block's pieces, one a lane: sixteens of K channels, sixteens of V rows, the scales of two blocks.
    const char* piece = p.cache.pool + (int64_t)h * p.cache.head_stride;
    uint32_t piece_at = 0, piece_bytes = 0;
    if (lane < DH / 16) {
      piece += lane * F::K_COLS + warp * (16 * BLOCK_ROWS);
      piece_at = lane * S::K_PITCH; piece_bytes = 16 * BLOCK_ROWS;
    } else if (lane < DH / 16 + 2) {
      piece += F::CODES + (2 * warp + lane - DH / 16) * F::V_ROWS;
      piece_at = S::V_AT + (lane - DH / 16) * S::V_PITCH; piece_bytes = F::V_ROWS;
    } else if (lane == DH / 16 + 2) {
      piece += F::SCALES + (warp >> 1) * 16;
      piece_at = S::SCALE_AT; piece_bytes = 16;
    }
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
      if (ok) {
        if (lane == 0) mbar_expect_tx(bar + 8 * s, 2 * BLOCK_ROWS * DH + 16);
        __syncwarp();
        if (piece_bytes)
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                       ::"r"(ring + s * S::BLOCK + piece_at), "l"(piece + (int64_t)pg * p.cache.page_stride), "r"(piece_bytes), "r"(bar + 8 * s) : "memory");
      } else if (lane == 0) {
        mbar_arrive(bar + 8 * s);
      }
    };
    Query<DH, NT> query;
    query.fetch(p, b, h, r0);                        // (ahead of the requests, which wait for the page table)
#pragma unroll 1
    for (int j = 0; j < STAGES - 1; ++j) request(j, step + j);
    query.store(p, sm);
    __syncthreads();
    float f[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float2 v = *reinterpret_cast<const float2*>(qf + 8 * nt + 2 * t);
      f[nt][0] = v.x; f[nt][1] = v.y;                // (NaN: fmaxf below takes the other one; the row is made NaN at the end)
    }
    acc.clear();
    const uint32_t qs = base + S::Q_OFF + n8 * S::Q_PITCH + 16 * t, swap = DH == 128 ? (n8 & 1) * 64 : 0;          // row n8 of every eight
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
      const uint32_t blk = ring + s * S::BLOCK;
      const int valid = min(L - (t0 + j) * SPACE_PAGE_SIZE - warp * BLOCK_ROWS, BLOCK_ROWS);   // keys of this block, >= 1

      // ---- S^T = K Q^T: rows n8 and n8 + 8 of product u are keys 4 n8 + 2u and + 1; a k-step has of each lane's sixteen channels
      // 64 cg + 16 t .. eight
      float sc[2][NT][4];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sc[u][nt][0] = sc[u][nt][1] = sc[u][nt][2] = sc[u][nt][3] = 0.f;
#pragma unroll
      for (int cg = 0; cg < DH / 64; ++cg) {
        uint4 k[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) k[i] = lds128(blk + (4 * cg + t) * S::K_PITCH + (4 * n8 + i) * 16);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int term = 0; term < 2; ++term) {
            const uint4 q = lds128(qs + (term * RT + 8 * nt) * S::Q_PITCH + (64 * cg ^ swap));
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              mma8(sc[u][nt], k[2 * u].x, k[2 * u + 1].x, k[2 * u].y, k[2 * u + 1].y, q.x, q.y);
              mma8(sc[u][nt], k[2 * u].z, k[2 * u + 1].z, k[2 * u].w, k[2 * u + 1].w, q.z, q.w);
            }
          }
      }
      const uint2 scales = lds64(blk + S::SCALE_AT + (warp & 1) * 8);
      const float ks = __uint_as_float(scales.x), ev = (float)((int)((scales.y >> 23) & 255u) - 127);
      // ---- weights: lane has of columns 2t, 2t + 1 the keys 4 n8 .. + 3.  (One thing after the other for all columns: they do not
      // wait for each other's latencies.)
      if (valid < BLOCK_ROWS) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (4 * n8 + i >= valid) sc[i >> 1][nt][2 * (i & 1)] = sc[i >> 1][nt][2 * (i & 1) + 1] = -CUDART_INF_F;
      }
      float ms[NT][2], fk[NT][2], r[NT][2], sum[NT][2], beta[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) ms[nt][c] = fmaxf(max3(sc[0][nt][c], sc[0][nt][2 + c], sc[1][nt][c]), sc[1][nt][2 + c]);
#pragma unroll
      for (int o = 4; o < 32; o <<= 1)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) ms[nt][c] = fmaxf(ms[nt][c], __shfl_xor_sync(0xFFFFFFFFu, ms[nt][c], o));     // (a number: the block has a key)
      bool far = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          fk[nt][c] = fminf(fmaxf(f[nt][c] * ks, F_MIN), F_MAX);
          const float mb = ms[nt][c] * fk[nt][c];
          r[nt][c] = mb - 8.f;
          far = far || fabsf(mb) > REF_FAR;
        }
      if (__any_sync(0xFFFFFFFFu, far)) {            // scores off the largest first, then times the factor
#pragma unroll 1
        for (int x = 0; x < 2 * NT; ++x)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              if (x != 2 * nt + c) continue;
              if (fabsf(ms[nt][c] * fk[nt][c]) > SCORE_MAX) {
                fk[nt][c] = SCORE_MAX / fabsf(ms[nt][c]);
                r[nt][c] = copysignf(SCORE_MAX, ms[nt][c]);
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                float& y = sc[i >> 1][nt][2 * (i & 1) + c];
                y = fast_exp2(fmaf(y - ms[nt][c], fk[nt][c], 8.f));
              }
            }
      } else {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[u][nt][e] = fast_exp2(fmaf(sc[u][nt][e], fk[nt][e & 1], -r[nt][e & 1]));
      }
      uint32_t w[NT][2][2], b0[NT][2], b1[NT][2];    // second operands of both terms
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          sum[nt][c] = (sc[0][nt][c] + sc[0][nt][2 + c]) + (sc[1][nt][c] + sc[1][nt][2 + c]);
          split4(sc[0][nt][c], sc[0][nt][2 + c], sc[1][nt][c], sc[1][nt][2 + c], w[nt][0][c], w[nt][1][c]);
        }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int term = 0; term < 2; ++term) transpose_words(w[nt][term][0], w[nt][term][1], b0[nt][term], b1[nt][term]);
      acc.join(r, sum, ev, beta);
      // ---- D^T = V^T W^T: the lane's keys of a channel are 8 t .. + 7
      const uint32_t vat = blk + S::V_AT + (t >> 1) * S::V_PITCH + n8 * 16 + 8 * (t & 1);
      uint32_t keep0 = 0xFFFFFFFFu, keep1 = 0xFFFFFFFFu;
      if (valid < BLOCK_ROWS) {                      // what lies behind the last row must not count, whatever it is
        const int a = min(max(valid - 8 * t, 0), 4), c = min(max(valid - 8 * t - 4, 0), 4);
        keep0 = a == 4 ? 0xFFFFFFFFu : (1u << (8 * a)) - 1u;
        keep1 = c == 4 ? 0xFFFFFFFFu : (1u << (8 * c)) - 1u;
      }
#pragma unroll
      for (int ct = 0; ct < DH / 16; ++ct) {
        uint2 x = lds64(vat + ct * 256), y = lds64(vat + ct * 256 + 128);
        x.x &= keep0; x.y &= keep1; y.x &= keep0; y.y &= keep1;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float d[4] = {0.f, 0.f, 0.f, 0.f};
          mma8(d, x.x, y.x, x.y, y.y, b0[nt][0], b1[nt][0]);
          mma8(d, x.x, y.x, x.y, y.y, b0[nt][1], b1[nt][1]);
          acc.o[ct][nt][0] = fmaf(d[0], beta[nt][0], acc.o[ct][nt][0]); acc.o[ct][nt][1] = fmaf(d[1], beta[nt][1], acc.o[ct][nt][1]);
          acc.o[ct][nt][2] = fmaf(d[2], beta[nt][0], acc.o[ct][nt][2]); acc.o[ct][nt][3] = fmaf(d[3], beta[nt][1], acc.o[ct][nt][3]);
        }
      }
      __syncwarp();                                  // everybody has read the stage: the next request may fill it
    }

    // ---- the block's own rows: keys 16 warp .. + 15 of it, products in bf16 as they are (no code, no scale), weights as two
    // bf16 terms, 2^-32 as large: sums of rows next to the largest number stay numbers
    if (t1 > Tc && p.has_new && 16 * warp < p.n_q && L0 >= 0) {
      const int k0 = 16 * warp;
      constexpr int LANES = DH / 8, V_LOADS = 16 * LANES / 32;
      uint4 kr[2][DH / 32], vr[V_LOADS], qr[NT][DH / 32];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        int i, hq;
        row_of(p, h, r0 + 8 * nt + n8, i, hq);
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)b * p.q_sb + (int64_t)i * p.q_sr + (int64_t)hq * p.q_sh) + t * (DH / 32);
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) qr[nt][j] = i < p.n_q ? src[j] : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int key = k0 + 8 * i + n8;
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
      float sc[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
      // Rows that hold a number of 2^ROW_LARGE or more, keys and queries (whose factors say so), are taken ROW_DOWN times as large: sums of
      // products stay numbers.
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < DH / 32; ++j) top = max(top, max(kvq::max_bits(kr[0][j]), kvq::max_bits(kr[1][j])));
#pragma unroll
      for (int k = 0; k < DH / 32; ++k) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint4 q = qr[nt][k];
          mma_bf16(sc[nt], kr[0][k].x, kr[1][k].x, kr[0][k].y, kr[1][k].y, q.x, q.y);
          mma_bf16(sc[nt], kr[0][k].z, kr[1][k].z, kr[0][k].w, kr[1][k].w, q.z, q.w);
        }
      }
      // Rows that hold a number of 2^ROW_LARGE or more, keys and queries (their factors say so), or one that is not finite: the
      // products once more, of such rows times ROW_DOWN, so that their sums are numbers; of a query row that is not finite with zeros, as over the cache: its keys are
      // known to be there, and it is made NaN at the end.  (Loaded anew: the rows that were there
      // have given their registers up.)
      const float f_large = p.c * pow2(ROW_LARGE - 7);
      constexpr uint32_t BITS_LARGE = (uint32_t)(ROW_LARGE + 127) << 7;        // (as bf16)
      if (__any_sync(0xFFFFFFFFu, top >= BITS_LARGE || !(qf[lane % RT] < f_large))) {
        const uint4* key_at[2];
        bool large[2];                               // such a key 8 i + n8
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int key = min(k0 + 8 * i + n8, p.n_q - 1);                     // (one behind the last: nobody sees it)
          key_at[i] = reinterpret_cast<const uint4*>(p.kn + (int64_t)b * p.n_sb + (int64_t)key * p.n_sr + (int64_t)h * p.n_sh) + t * (DH / 32);
          top = 0;
#pragma unroll 1
          for (int j = 0; j < DH / 32; ++j) {
            uint4 v = key_at[i][j];
            top = max(top, kvq::top_bits(v));
          }
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
          large[i] = top >= BITS_LARGE;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
#pragma unroll 1
        for (int j = 0; j < DH / 32; ++j) {
          uint4 v[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            v[i] = key_at[i][j];
            kvq::make_finite(v[i]);
            if (large[i]) v[i] = kvq::scale_bf16(v[i], ROW_DOWN);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            int i, hq;
            row_of(p, h, min(r0 + 8 * nt + n8, p.n_q * p.G - 1), i, hq);
            uint4 q = *(reinterpret_cast<const uint4*>(p.q + (int64_t)b * p.q_sb + (int64_t)i * p.q_sr + (int64_t)hq * p.q_sh) + t * (DH / 32) + j);
            const float of_row = qf[8 * nt + n8];
            if (of_row >= f_large) q = kvq::scale_bf16(q, ROW_DOWN);
            if (of_row != of_row) q = make_uint4(0, 0, 0, 0);
            mma_bf16(sc[nt], v[0].x, v[1].x, v[0].y, v[1].y, q.x, q.y);
            mma_bf16(sc[nt], v[0].z, v[1].z, v[0].w, v[1].w, q.z, q.w);
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const bool large_row = qf[8 * nt + 2 * t + c] >= f_large;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float x = sc[nt][2 * i + c];
              if (large[i]) x *= 1.f / ROW_DOWN;
              if (large_row) x *= 1.f / ROW_DOWN;
              sc[nt][2 * i + c] = x > 0x1p127f ? 0x1p127f : x < -0x1p127f ? -0x1p127f : x;
            }
          }
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < V_LOADS; ++i) {            // V rows into the (dry) ring
        kvq::make_finite(vr[i]);
        const uint32_t at = ring + (i * (32 / LANES) + lane / LANES) * S::OWN_PITCH + (lane % LANES) * 16;
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(vr[i].x), "r"(vr[i].y), "r"(vr[i].z), "r"(vr[i].w) : "memory");
      }
      __syncwarp();
      uint32_t ph[NT][2], pl[NT][2];
      float r[NT][2], sum[NT][2], beta[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float y[2][2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int row = r0 + 8 * nt + 2 * t + c;
          const uint64_t see = row < p.n_q * p.G ? p.mask[row >> p.gsh] : 0ull;                    // Eq. 5
          float top = -CUDART_INF_F;
          sum[nt][c] = 0.f;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const bool vis = (see >> (k0 + 8 * i + n8)) & 1ull;
            const float x = sc[nt][2 * i + c] * p.c;
            y[c][i] = vis ? (x > SCORE_MAX ? SCORE_MAX : x < -SCORE_MAX ? -SCORE_MAX : x) : -CUDART_INF_F;
            top = fmaxf(top, y[c][i]);
          }
          r[nt][c] = top = col_max(top);
          const float from = top == -CUDART_INF_F ? 0.f : top;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            y[c][i] = fast_exp2(y[c][i] - from);
            sum[nt][c] += y[c][i];
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float w0 = y[0][i] * 0x1p-32f, w1 = y[1][i] * 0x1p-32f;
          const __nv_bfloat162 hi = __floats2bfloat162_rn(w0, w1);
          const uint32_t hw = *reinterpret_cast<const uint32_t*>(&hi);
          float l0, l1;
          low_terms(hw, w0, w1, l0, l1);
          const __nv_bfloat162 lo = __floats2bfloat162_rn(l0, l1);
          ph[nt][i] = transpose8(hw);
          pl[nt][i] = transpose8(*reinterpret_cast<const uint32_t*>(&lo));
        }
      }
      acc.join(r, sum, 32.f, beta);
#pragma unroll
      for (int ct = 0; ct < DH / 16; ++ct) {
        uint32_t a0, a1, a2, a3;
        const uint32_t at = ring + (8 * (lane >> 4) + (lane & 7)) * S::OWN_PITCH + ct * 32 + ((lane >> 3) & 1) * 16;
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(a0), "=r"(a1), "=r"(a2), "=r"(a3) : "r"(at) : "memory");
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float d[4] = {0.f, 0.f, 0.f, 0.f};
          mma_bf16(d, a0, a1, a2, a3, ph[nt][0], ph[nt][1]);
          mma_bf16(d, a0, a1, a2, a3, pl[nt][0], pl[nt][1]);
          acc.o[ct][nt][0] = fmaf(d[0], beta[nt][0], acc.o[ct][nt][0]); acc.o[ct][nt][1] = fmaf(d[1], beta[nt][1], acc.o[ct][nt][1]);
          acc.o[ct][nt][2] = fmaf(d[2], beta[nt][0], acc.o[ct][nt][2]); acc.o[ct][nt][3] = fmaf(d[3], beta[nt][1], acc.o[ct][nt][3]);
        }
      }
      __syncwarp();
    }

    // ---- the four warps' states meet
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float sum = col_sum(acc.l[nt][e]);
        if (lane < 4) ml[warp * RT + 8 * nt + 2 * t + e] = make_float2(acc.M[nt][e], sum);
      }
    __syncthreads();
    const bool whole = t0 == 0 && t1 == T;
    auto total = [&](int r, float& M, float& l) {
      M = -CUDART_INF_F; l = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) M = fmaxf(M, ml[w * RT + r].x);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float2 v = ml[w * RT + r];
        l += v.x == -CUDART_INF_F ? 0.f : v.y * fast_exp2(v.x - M);
      }
    };
    {
      float* mine = reinterpret_cast<float*>(sm + warp * S::RING);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = 8 * nt + 2 * t + e;
          float M, l;
          total(r, M, l);
          float fac = acc.M[nt][e] == -CUDART_INF_F ? 0.f : fast_exp2(acc.M[nt][e] - M) / l * fast_exp2(acc.R[nt][e]);
          if (M != -CUDART_INF_F && f[nt][e] != f[nt][e]) fac = __int_as_float(0x7FFFFFFF);
#pragma unroll
          for (int ct = 0; ct < DH / 16; ++ct) {
            mine[r * S::O_PITCH + 16 * ct + n8] = acc.o[ct][nt][e] * fac;
            mine[r * S::O_PITCH + 16 * ct + 8 + n8] = acc.o[ct][nt][2 + e] * fac;
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
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(sm + w * S::RING + (r * S::O_PITCH + 4 * c4) * 4);
        o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
      }
      o = held(o);
      if (whole) store_row4<DH>(p, b, h, r0 + r, c4, o);
      else __stcg(reinterpret_cast<float4*>(p.part + (int64_t)slot * SLOT + r * DH) + c4, o);
      if (c4 == 0) {
        float M, l;
        total(r, M, l);
        if (M != -CUDART_INF_F && qf[r] != qf[r]) l = qf[r];
        if (whole) {
          store_lse(p, b, h, r0 + r, M, l);
        } else {
          __stcg(p.part + (int64_t)slot * SLOT + RT * DH + r, M);
          __stcg(p.part + (int64_t)slot * SLOT + RT * DH + RT + r, l);
        }
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
      if (*last_flag) join_pieces<DH, RT, NT, NT == 1 ? 16 : 4>(p, cut, b, h, r0, rows, piece0, pieces, item_at, (int)threadIdx.x, THREADS);
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
    const cudaError_t e = cudaFuncSetAttribute(kvb_attn_kernel<DH, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<DH, NT>(128));
    if (e != cudaSuccess) return e;
    if (dev < 64) done_mask |= 1ull << dev;
  }
  static_assert(Smem<DH, NT>::CTAS * 8 * NT <= KVB_SM_ROWS, "a slot per block");
  p.n_rt = (p.n_q * p.G + 8 * NT - 1) / (8 * NT);
  p.n_groups = Smem<DH, NT>::CTAS * ctx->sm_count;
  return launch_pdl(kvb_attn_kernel<DH, NT>, dim3(p.n_groups), dim3(THREADS), smem_bytes<DH, NT>(max_batch), st, p, max_batch);
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
  // the flat list is counted in 32 bits: items of eight rows at least, a page and the cost of starting more than a table names
  if ((double)p.B * p.H_kv * ((rows + 7) / 8) * ((double)p.cache.pages_per_seq + 4) > 2e9) return SPACE_E_UNSUPPORTED;
  ctx->launches += 1;
  // More query rows than sixteen go to tcgen05 (us, here / there: 32 rows of 64 sequences up to 8192 keys 395 / 217, 18 rows of 16 sequences
  // up to 4096 keys 143 / 121, 16 rows of those 107 / 123, 16 rows of 5 short sequences 16 / 22).
  if (rows > 16) return launch_kvb_attn_tc(ctx, p, st);
  const bool wide = ctx->cfg.head_dim == 128;
  cudaError_t e;
  if (rows <= 8) e = wide ? launch_dim<128, 1>(p, ctx, st) : launch_dim<64, 1>(p, ctx, st);
  else e = wide ? launch_dim<128, 2>(p, ctx, st) : launch_dim<64, 2>(p, ctx, st);
  return cuda_ok(e);
}
