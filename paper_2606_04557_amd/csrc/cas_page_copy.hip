// Copies between pages of the paged cache: the first rows of the listed pages go to
// other pages, in the pools of every layer. A thread has U 16-byte loads in flight.
//
// Bound by HBM: every byte is read once (a page that several copies read comes from
// the cache after the first) and written once. 8,192 whole pages of 32 KB in two pools: 172 us,
// 6.2 TB/s; the ragged tails of 200 pages in 64 pools, 223 MB written of 174 MB: 82 us, 4.8 TB/s;
// four of them in two pools 2.7 us, a launch's latency.
#include "cas_device.h"

namespace cas {

namespace {

template <int T, int U>
__device__ __forceinline__ void copy_piece(const PageCopyParams &p, const cas_page_copy_t c, int piece) {
  constexpr int kStep = T * 16;   // bytes that the workgroup moves at a time
  const int64_t begin = (int64_t)piece * (U * kStep), end = (int64_t)c.rows * p.row_bytes;
  if (begin >= end) return;
  char *pool = p.pools[blockIdx.y];
  const char *src = pool + (int64_t)c.src * p.page_bytes + begin;
  char *dst = pool + (int64_t)c.dst * p.page_bytes + begin;
  const int left = (int)min(end - begin, (int64_t)(U * kStep)), at = threadIdx.x * 16;
  u32x4 v[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (at + u * kStep < left) v[u] = *reinterpret_cast<const u32x4 *>(src + at + u * kStep);
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (at + u * kStep < left) *reinterpret_cast<u32x4 *>(dst + at + u * kStep) = v[u];
}

template <int T, int U>
__global__ __launch_bounds__(T) void page_copy_kernel(PageCopyParams p) {
  const int which = blockIdx.x / p.pieces;
  copy_piece<T, U>(p, p.table[p.first + which], blockIdx.x - which * p.pieces);
}

template <int T, int U>
__global__ __launch_bounds__(T) void page_copy_args_kernel(PageCopyParams p, PageCopyList list) {
  const int which = blockIdx.x / p.pieces;
  copy_piece<T, U>(p, list.copies[p.first + which], blockIdx.x - which * p.pieces);
}

template <int T, int U>
void launch(const PageCopyParams &p, const PageCopyList *copies, dim3 grid, hipStream_t s) {
  if (copies) hipLaunchKernelGGL((page_copy_args_kernel<T, U>), grid, dim3(T), 0, s, p, *copies);
  else hipLaunchKernelGGL((page_copy_kernel<T, U>), grid, dim3(T), 0, s, p);
}

}  // namespace

hipError_t launch_page_copy(const PageCopyParams &p, const PageCopyList *copies, int n, int n_pools, hipStream_t s) {
  const dim3 grid((unsigned)(n * p.pieces), (unsigned)n_pools);
  if (p.piece == 512 * 16) launch<512, 1>(p, copies, grid, s);
  else if (p.piece == 512 * 32) launch<512, 2>(p, copies, grid, s);
  else launch<1024, 2>(p, copies, grid, s);
  return hipGetLastError();
}

}  // namespace cas
