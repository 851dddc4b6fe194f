// Attention over a paged cache in 8 bits, many rows a request and few in one launch (paged_mixed_kernel, of codes).  Three workgroups to a CU up to head dim 64, where codes
// on their way through registers leave no room for four (3 prompts of 2500, 16 heads of 64: 71 us, 78 with four and spilled registers).
#pragma once
#include "paged8_few_impl.h"
#include "paged_tile_impl.h"

namespace fs {

template <typename T, class Code, int D, int NT, bool ONCE> __global__ __launch_bounds__(256, (D <= 64 && NT == 1 ? 3 : 2)) void paged8_mixed_kernel(const PagedArgs a) {
  __shared__ __align__(1024) union { Few8Lds<D, NT, 4> few; TileShared<D> tile; } lds;
  const int tiles = gridDim.x - a.few_grid, b = blockIdx.x;
  if (b < tiles) paged_tile<T, D, Code>(a, lds.tile, b);
  else paged8_few<T, Code, D, NT, 4, 32, ONCE>(a, lds.few, b - tiles);
}

template <typename T, class Code, int D, int NT, bool ONCE> hipError_t paged8_mixed_launch(const PagedArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((paged8_mixed_kernel<T, Code, D, NT, ONCE>), dim3(paged_mixed_grid(a)), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return (__is_same(T, f16_t) ? paged_mixed_join_launch_f16 : paged_mixed_join_launch_bf16)(a, D, NT, s);
}
template <typename T, class Code, int D, bool ONCE> hipError_t paged8_mixed_launch_rows(const PagedArgs& a, int row_tiles, hipStream_t s) {
  return row_tiles == 1 ? paged8_mixed_launch<T, Code, D, 1, ONCE>(a, s) : paged8_mixed_launch<T, Code, D, 2, ONCE>(a, s);
}
template <typename T, class Code> hipError_t paged8_mixed_launch_type(const PagedArgs& a, int dim, int row_tiles, hipStream_t s) {
  switch (dim) {
    case 32: return paged8_mixed_launch_rows<T, Code, 32, false>(a, row_tiles, s);
    case 64: return a.once ? paged8_mixed_launch_rows<T, Code, 64, true>(a, row_tiles, s) : paged8_mixed_launch_rows<T, Code, 64, false>(a, row_tiles, s);
    case 96: return a.once ? paged8_mixed_launch_rows<T, Code, 96, true>(a, row_tiles, s) : paged8_mixed_launch_rows<T, Code, 96, false>(a, row_tiles, s);
    default: return paged8_mixed_launch_rows<T, Code, 128, true>(a, row_tiles, s);
  }
}

}  // namespace fs
