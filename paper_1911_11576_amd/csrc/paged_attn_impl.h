// Attention of new tokens over a paged cache (fs_plan_create_paged_attention): what its kernels share.
//
// A request's queries are rows of tiles: row r of request b and key head h is its token r / share, query head h * share + r %
// share, so that the query heads of a key head read its keys and values together.  Both dots run transposed on MFMA, as in
// the attention of whole groups: S^T = K . Q^T leaves every score of a row in four lanes, the softmax is a register
// reduction and two swaps, and the probabilities already are the second dot's operand, O^T = V^T . P^T.
#pragma once
#include "attn_stitch_impl.h"
#include "paged.h"

namespace fs {

struct PagedArgs {
  const void *q, *k, *v;
  const int *tables, *lengths, *starts;
  void* out;
  float* lse;
  float* partial;
  int64_t q_stride, out_stride;
  CacheLayout cache;
  int requests, tokens, q_heads, kv_heads, share, width, causal, window;
  float scale2;                    // scale times log2 e: scores are kept in units of log 2
  int unit_keys;                   // few rows: keys of a unit of work, a multiple of 128
  int log_groups;                  // few rows: workgroups = 1 << log_groups
  int few_rows;                    // requests of up to so many rows are the few-rows kernel's, the others the tile kernel's
  float* tile_partial;             // tiles of 128 rows: [slots][kv_heads][most_parts][128 * (D + 2)]
  int slots, most_parts, least_steps;      // places for tiles, parts that a tile's keys are split into at most, steps of 64 keys of a part at least
};

// A request as the kernels see it: its first row of q, its new tokens, its keys.
struct PagedRequest { int first, fresh, keys; };

__device__ __forceinline__ PagedRequest paged_request(const PagedArgs& a, int b) {
  PagedRequest r;
  r.first = min(max(a.starts[b], 0), a.tokens);
  r.fresh = max(0, min(max(a.starts[b + 1], 0), a.tokens) - r.first);
  r.keys = (int)min((int64_t)max(a.lengths[b], 0), (int64_t)a.width << a.cache.shift);
  return r;
}

// The first key that the first of a request's new tokens sees, down to a multiple of 32.
__device__ __forceinline__ int paged_first_key(const PagedArgs& a, const PagedRequest& r) {
  return a.window ? max(0, r.keys - r.fresh + 1 - a.window) & ~31 : 0;
}

// Values of a 16-byte piece that are infinite or NaN: the exponent's bits are all ones, which the addition carries into the sign's place.
template <typename T> struct Odd;
template <> struct Odd<f16_t> { static constexpr uint32_t kMask = 0x7c007c00u, kCarry = 0x04000400u; };
template <> struct Odd<bf16_t> { static constexpr uint32_t kMask = 0x7f807f80u, kCarry = 0x00800080u; };
template <typename T> __device__ __forceinline__ uint32_t odd_values(u32x4 v) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) any |= ((v[i] & Odd<T>::kMask) + Odd<T>::kCarry) & 0x80008000u;
  return any;
}
// ... and the piece with zeros in their places
template <typename T> __device__ __forceinline__ u32x4 without_odd(u32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t odd = ((v[i] & Odd<T>::kMask) + Odd<T>::kCarry) & 0x80008000u;      // bits 15 and 31
    v[i] &= ~((odd >> 15) * 0xffffu);
  }
  return v;
}

// few rows a request: the work split evenly over a fixed grid, then the parts joined
hipError_t paged_few_launch_f16(const PagedArgs&, int dim, int row_tiles, hipStream_t);
hipError_t paged_few_launch_bf16(const PagedArgs&, int dim, int row_tiles, hipStream_t);
// many rows a request: tiles of 128
hipError_t paged_tile_launch_f16(const PagedArgs&, int dim, hipStream_t);
hipError_t paged_tile_launch_bf16(const PagedArgs&, int dim, hipStream_t);

}  // namespace fs
