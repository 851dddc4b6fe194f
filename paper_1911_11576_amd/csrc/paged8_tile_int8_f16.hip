// Attention over a paged cache in 8 bits, many rows a request: int8 codes, f16.
#include "paged8_tile_impl.h"

namespace fs {
hipError_t paged8_mixed_launch_int8_f16(const PagedArgs& a, int dim, int row_tiles, hipStream_t s) { return paged8_mixed_launch_type<f16_t, Int8>(a, dim, row_tiles, s); }
}  // namespace fs
