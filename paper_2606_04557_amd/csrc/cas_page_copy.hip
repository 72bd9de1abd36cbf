// Copies between pages of the paged cache: y[dst][row] = x[dst's source][row] for
// the listed pages and rows, in the pools of every layer. Bound by HBM: every byte
// is read once and written once.
#include "cas_device.h"

namespace cas {

namespace {

constexpr int kPageCopyThreads = 256;

__device__ __forceinline__ void copy_piece(const PageCopyParams &p, const cas_page_copy_t c, int piece) {
  char *pool = p.pools[blockIdx.y];
  const int64_t begin = (int64_t)piece * p.piece, end = min(begin + p.piece, (int64_t)c.rows * p.row_bytes);
  const char *src = pool + (int64_t)c.src * p.page_bytes;
  char *dst = pool + (int64_t)c.dst * p.page_bytes;
  for (int64_t i = begin + threadIdx.x * 16; i < end; i += kPageCopyThreads * 16)
    *reinterpret_cast<u32x4 *>(dst + i) = *reinterpret_cast<const u32x4 *>(src + i);
}

__global__ __launch_bounds__(kPageCopyThreads) void page_copy_kernel(PageCopyParams p) {
  const int which = blockIdx.x / p.pieces;
  copy_piece(p, p.table[p.first + which], blockIdx.x - which * p.pieces);
}

__global__ __launch_bounds__(kPageCopyThreads) void page_copy_args_kernel(PageCopyParams p, PageCopyList list) {
  const int which = blockIdx.x / p.pieces;
  copy_piece(p, list.copies[p.first + which], blockIdx.x - which * p.pieces);
}

}  // namespace

hipError_t launch_page_copy(const PageCopyParams &p, const PageCopyList *copies, int n, int n_pools, hipStream_t s) {
  const dim3 grid((unsigned)(n * p.pieces), (unsigned)n_pools), threads(kPageCopyThreads);
  if (copies) hipLaunchKernelGGL(page_copy_args_kernel, grid, threads, 0, s, p, *copies);
  else hipLaunchKernelGGL(page_copy_kernel, grid, threads, 0, s, p);
  return hipGetLastError();
}

}  // namespace cas
