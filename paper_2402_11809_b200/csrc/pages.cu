// Moves of rows between pages, over the pools of all layers in one launch (space_pages_copy).
//
// Nothing but bytes read once and written once: a thread block per 32 KB of a (move, pool) pair, eight 16-byte
// loads per thread in flight before its first store.  The lists travel as the launch's parameters: no copy to the
// device goes before the kernel.  700 pages of a bf16 pool in 4 layers (1.5 GB read, as much written): 445 us, 1.02 of the
// copy rate; sixteen last pages of 8 layers: 5.4 to 6.3 us, a launch.
#include "common.cuh"
#include <cstdlib>

namespace {

constexpr int THREADS = 256, UNROLL = 8;

struct Pool { char* base; int64_t page_stride, part_stride; int parts, group_rows, group_vecs, pad; };
template <int MAX_POOLS, int MAX_MOVES>
struct CopyParams {
  Pool pool[MAX_POOLS];
  space_page_move move[MAX_MOVES];
};

template <int MAX_POOLS, int MAX_MOVES>
__global__ void __launch_bounds__(THREADS) pages_copy_kernel(const __grid_constant__ CopyParams<MAX_POOLS, MAX_MOVES> p) {
  pdl_launch_dependents();
  pdl_wait();
  const space_page_move m = p.move[blockIdx.x];
  const Pool& pl = p.pool[blockIdx.y];
  const uint32_t seg = (uint32_t)((m.rows + pl.group_rows - 1) / pl.group_rows) * (uint32_t)pl.group_vecs;   // vectors of a part
  const uint32_t total = seg * (uint32_t)pl.parts;
  const uint32_t v0 = blockIdx.z * (uint32_t)(THREADS * UNROLL) + threadIdx.x;
  if (v0 >= total) return;
  const char* src = pl.base + (int64_t)m.src * pl.page_stride;
  char* dst = pl.base + (int64_t)m.dst * pl.page_stride;
  uint4 val[UNROLL];
  int64_t off[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const uint32_t v = v0 + u * THREADS;
    if (v < total) {
      const uint32_t part = v / seg;
      off[u] = (int64_t)part * pl.part_stride + (int64_t)(v - part * seg) * 16;
      val[u] = *reinterpret_cast<const uint4*>(src + off[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u)
    if (v0 + u * THREADS < total) *reinterpret_cast<uint4*>(dst + off[u]) = val[u];
}

// Whether some page is written twice, or both read and written: an open-addressed set of the pages written.
int check_overlap(const space_page_move* moves, int n) {
  size_t size = 16;
  while (size < 4 * (size_t)n) size *= 2;
  int32_t* set = (int32_t*)malloc(size * sizeof(int32_t));
  if (!set) return SPACE_E_WORKSPACE;
  memset(set, 0xFF, size * sizeof(int32_t));
  auto place = [&](int32_t page) {
    size_t i = ((uint32_t)page * 2654435761u) & (size - 1);
    while (set[i] >= 0 && set[i] != page) i = (i + 1) & (size - 1);
    return i;
  };
  int rc = SPACE_OK;
  for (int i = 0; i < n && rc == SPACE_OK; ++i) {
    const size_t at = place(moves[i].dst);
    if (set[at] >= 0) rc = SPACE_E_INVALID_ARG;
    set[at] = moves[i].dst;
  }
  for (int i = 0; i < n && rc == SPACE_OK; ++i)
    if (set[place(moves[i].src)] >= 0) rc = SPACE_E_INVALID_ARG;
  free(set);
  return rc;
}

template <int MAX_POOLS, int MAX_MOVES>
int launch_copy(const space_page_pool* pools, int n_pools, const space_page_move* moves, int n_moves, unsigned splits, cudaStream_t st) {
  CopyParams<MAX_POOLS, MAX_MOVES> p;
  for (int i = 0; i < n_pools; ++i)
    p.pool[i] = Pool{(char*)pools[i].base, pools[i].page_stride, pools[i].part_stride, pools[i].parts, pools[i].group_rows, pools[i].group_bytes / 16, 0};
  for (int i = 0; i < n_moves; ++i) p.move[i] = moves[i];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_moves, n_pools, splits); cfg.blockDim = dim3(THREADS); cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cuda_ok(cudaLaunchKernelEx(&cfg, pages_copy_kernel<MAX_POOLS, MAX_MOVES>, p));
}

}  // namespace

extern "C" int space_pages_copy(const space_page_pool* pools, int32_t n_pools, const space_page_move* moves, int32_t n_moves,
                                void* stream) {
  if (n_pools < 0 || n_moves < 0 || (n_pools > 0 && !pools) || (n_moves > 0 && !moves) || n_pools > SPACE_PAGES_MAX_POOLS)
    return SPACE_E_INVALID_ARG;
  if (n_pools == 0 || n_moves == 0) return SPACE_OK;
  int32_t n_pages = INT32_MAX, max_rows = 0;
  for (int i = 0; i < n_pools; ++i) {
    const space_page_pool& q = pools[i];
    if (!q.base || q.n_pages < 1 || q.parts < 1 || q.group_rows < 1 || SPACE_PAGE_SIZE % q.group_rows || q.group_bytes < 16)
      return SPACE_E_INVALID_ARG;
    if (((uintptr_t)q.base & 15) || q.page_stride % 16 || q.part_stride % 16 || q.group_bytes % 16) return SPACE_E_ALIGNMENT;
    // no part may reach into the next one, no page into the next one
    const int64_t part = (int64_t)(SPACE_PAGE_SIZE / q.group_rows) * q.group_bytes;
    if (part > (1 << 28) || (q.parts > 1 && q.part_stride < part) || q.parts > (1 << 30) / part ||
        (q.n_pages > 1 && q.page_stride < (q.parts - 1) * q.part_stride + part))
      return SPACE_E_INVALID_ARG;
    if (q.n_pages < n_pages) n_pages = q.n_pages;
  }
  for (int i = 0; i < n_moves; ++i) {
    if (moves[i].src < 0 || moves[i].src >= n_pages || moves[i].dst < 0 || moves[i].dst >= n_pages || moves[i].rows < 0 ||
        moves[i].rows > SPACE_PAGE_SIZE)
      return SPACE_E_INVALID_ARG;
    if (moves[i].rows > max_rows) max_rows = moves[i].rows;
  }
  const int rc = check_overlap(moves, n_moves);
  if (rc != SPACE_OK) return rc;
  if (max_rows == 0) return SPACE_OK;
  int64_t most = 0;                                        // vectors of the largest (move, pool) pair
  for (int i = 0; i < n_pools; ++i) {
    const int64_t v = (int64_t)((max_rows + pools[i].group_rows - 1) / pools[i].group_rows) * (pools[i].group_bytes / 16) * pools[i].parts;
    if (v > most) most = v;
  }
  const unsigned splits = (unsigned)((most + THREADS * UNROLL - 1) / (THREADS * UNROLL));
  if (splits > 65535u) return SPACE_E_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  for (int m0 = 0; m0 < n_moves; m0 += SPACE_PAGES_MAX_MOVES) {
    const int n = n_moves - m0 < SPACE_PAGES_MAX_MOVES ? n_moves - m0 : SPACE_PAGES_MAX_MOVES;
    // (a launch carries its parameters whole: 3 KB or 23 KB of them)
    const int e = n_pools <= 32 && n <= 128 ? launch_copy<32, 128>(pools, n_pools, moves + m0, n, splits, st)
                                            : launch_copy<SPACE_PAGES_MAX_POOLS, SPACE_PAGES_MAX_MOVES>(pools, n_pools, moves + m0, n, splits, st);
    if (e != SPACE_OK) return e;
  }
  return SPACE_OK;
}
