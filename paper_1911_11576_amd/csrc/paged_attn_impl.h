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
  int unit_keys;                   // few rows: keys of a unit of work, a multiple of 32 to a wavefront
  int log_groups, few_grid;        // few rows: workgroups, 1 << log_groups of them; log_groups -1: a unit each, which is a whole tile
  int log_heads, head_sets;        // few rows: log2 of the key heads of a set, and the sets
  int neighbours;                  // few rows: workgroups of an XCD have neighbouring runs
  int few_rows;                    // requests of up to so many rows are the few-rows kernel's, the others the tile kernel's
  float* tile_partial;             // tiles of 128 rows: up to 2 * kTileShares of [128 * (D + 2)]
  int slots;                       // places for tiles in the order of the rows
};

// Workgroups of the tile kernel that the chip holds, two to a CU: what is shared out evenly.
constexpr int kTileShares = 512;
// An even share has no fewer steps of 64 keys; parts may have, since a request's split tiles are all cut into as many even parts as its longest
// needs (of nine steps: four and five) (D 128, 32 / 8 heads, 128 tokens behind 1920: 26.6 us with 4, 28.9 with 8, 37.5 with
// 16; twice 64 behind 4032: 32.9, 30.0, 37.9; 512 and 256 behind 512 and 1792: 44.6, 44.1, 42.7).
constexpr int kLeastSteps = 8;
// Requests among which those of many rows are looked for, two times 256 (one of 512 tokens behind 32256 keys and 100 of one behind 4095: 772 us with
// tiles in the order of the rows, 500 with a line of them; for 1000 single tokens and 20 chunks, where nothing needs it, the looks cost 1283 -> 1320).
constexpr int kTileRequests = 512;

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

// The request to which place `at` of a line of tiles of 1 << log_rows rows belongs in which request b's begin at place
// first * share / rows + b: as many places as it can have tiles, whatever the lengths of the others.  -1: none.
__device__ __forceinline__ int paged_place(const PagedArgs& a, int b, int log_rows) {
  return (int)((int64_t)min(max(a.starts[b], 0), a.tokens) * a.share >> log_rows) + b;
}
__device__ __forceinline__ int paged_find(const PagedArgs& a, int at, int log_rows) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.requests;      // among n requests from lo on, 64 of them looked at at a time
  for (;;) {
    const int step = (n + 63) >> 6, b = lo + lane * step;
    const int here = __popcll(__ballot(b < lo + n && paged_place(a, min(b, a.requests - 1), log_rows) <= at));
    if (here == 0) return -1;
    lo += (here - 1) * step;
    if (step == 1) return lo;
    n = min(step, a.requests - lo);
  }
}

// Sum over the wavefront's lanes, the same in all of them.
__device__ __forceinline__ int wave_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, false);
  auto r = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
  v = (int)(r[0] + r[1]);
  r = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  return __builtin_amdgcn_readfirstlane((int)(r[0] + r[1]));
}
// Sum over the lanes up to and with this one: inside rows of 16 by shifts, then the last lane of the row before, and of the half before.
__device__ __forceinline__ int wave_upto(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}

// 2^x as the factor of what was summed up under a smaller maximum: no less than the least fp32 number, so that an infinity among it, a value's that the
// row sees, stays one where the power is none (0 times it would be NaN; of a number nothing is left either way).
__device__ __forceinline__ float sum_factor(float x) { return fmaxf(__builtin_amdgcn_exp2f(x), 0x1p-149f); }

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

// 16 bytes a lane from memory straight into LDS: piece I of 64 bytes of a lane's row to the wavefront's 1024 bytes at `lds` + 1024 I.
// (The instruction's offset counts on both sides.  As assembly, since the compiler makes every LDS read behind the builtin wait for
// all loads in flight, the next step's among them; there is no register that it writes.  The code waits by itself, below.)
// ONCE: read by nobody else, past the caches.
template <int I, bool ONCE> __device__ __forceinline__ void load_lds16(const uint16_t* from, uint32_t lds) {
  if constexpr (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off offset:%2 nt" ::"s"(lds + 960 * I), "v"(from), "n"(64 * I) : "memory");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off offset:%2" ::"s"(lds + 960 * I), "v"(from), "n"(64 * I) : "memory");
}
// 4 bytes a lane
__device__ __forceinline__ void load_lds4(const int* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(from) : "memory");
}
// until all but the last N loads are there (they come in order)
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// until LDS has been read: before a load writes there again
__device__ __forceinline__ void wait_lds_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }

// few rows a request: the work split evenly over a fixed grid, then the parts joined
hipError_t paged_few_launch_f16(const PagedArgs&, int dim, int row_tiles, hipStream_t);
hipError_t paged_few_launch_bf16(const PagedArgs&, int dim, int row_tiles, hipStream_t);
// many rows a request, in tiles of 128, and few rows, in one
hipError_t paged_mixed_launch_f16(const PagedArgs&, int dim, int row_tiles, hipStream_t);
hipError_t paged_mixed_launch_bf16(const PagedArgs&, int dim, int row_tiles, hipStream_t);

}  // namespace fs
