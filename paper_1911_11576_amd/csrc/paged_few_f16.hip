// Attention over a paged cache, few rows a request: fp16.
#include "paged_few_impl.h"

namespace fs {
hipError_t paged_few_launch_f16(const PagedArgs& a, int dim, int row_tiles, hipStream_t s) { return paged_few_launch_type<f16_t>(a, dim, row_tiles, s); }
}  // namespace fs
