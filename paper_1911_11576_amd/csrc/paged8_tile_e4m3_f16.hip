// Attention over a paged cache in 8 bits, many rows a request: e4m3 codes, f16.
#include "paged8_tile_impl.h"

namespace fs {
hipError_t paged8_mixed_launch_e4m3_f16(const PagedArgs& a, int dim, int row_tiles, hipStream_t s) { return paged8_mixed_launch_type<f16_t, E4m3>(a, dim, row_tiles, s); }
}  // namespace fs
