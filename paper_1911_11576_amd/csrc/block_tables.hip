// Block tables and slot maps from request lengths (fs_plan_create_block_tables).
//
// With c the cached and f the new tokens of a request, both cut as fs.h says, S the exclusive sum of f over the requests:
//   starts = min(S, T),  f' = the difference of its neighbours,  have = ceil(c / bs),  need = ceil((c + f') / bs)
//   request's first new block = free[exclusive sum of (need - have)]
// Both sums are scans of at most 4096 numbers: every workgroup makes them for itself in LDS (8 bytes a request read through
// the caches), which costs less than a kernel that hands them over, and then serves its run of rows, each row finding its
// request by bisection.  A block that a request gets new is written into the table by the row of its first token: no
// workgroup reads an entry that another writes, so the table is updated in place.  All of it is a launch and four dependent
// memory accesses (lengths -> entry or free list -> stores); no step's bytes come near a bandwidth.  2.2 us for 48 requests of one token, 4.6 for 515 of 32768.
#include "dev_common.h"
#include "paged.h"

namespace fs {
namespace {

struct TablesArgs {
  const int *cached, *fresh, *free;
  int *tables, *lengths, *starts, *positions, *slots, *taken;
  int requests, tokens, blocks, shift, width, n_free;
};

// Sums stop at 2^32 - 1: everything beyond `tokens` is cut to it anyway.
__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false); }

// Sum over the threads before this one, by shifts inside rows of 16 lanes, then the last lane of the row before and of the half before;
// `room` has a place per wavefront, and *all gets the workgroup's total.
template <int WG> __device__ __forceinline__ uint32_t block_exclusive(uint32_t v, uint32_t* room, uint32_t* all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t s = v;
  s = add(s, moved<0x111, 0xF>(s));
  s = add(s, moved<0x112, 0xF>(s));
  s = add(s, moved<0x114, 0xF>(s));
  s = add(s, moved<0x118, 0xF>(s));
  s = add(s, moved<0x142, 0xA>(s));
  s = add(s, moved<0x143, 0xC>(s));
  uint32_t before = __shfl_up(s, 1);
  if (lane == 0) before = 0;
  if constexpr (WG == 64) {
    *all = __builtin_amdgcn_readlane(s, 63);
    return before;
  }
  if (lane == 63) room[w] = s;
  __syncthreads();
  uint32_t total = 0;
#pragma unroll
  for (int k = 0; k < WG / 64; ++k) {
    const uint32_t n = room[k];
    if (k < w) before = add(before, n);
    total = add(total, n);
  }
  *all = total;
  __syncthreads();
  return before;
}

// E: requests of a thread, whose lengths it keeps.
template <int WG, int E> __global__ __launch_bounds__(WG) void block_tables_kernel(const TablesArgs a) {
  extern __shared__ uint32_t smem[];
  uint32_t* room = smem;                            // [16]
  uint32_t* starts = smem + 16;                     // [requests + 1]
  uint32_t* first_free = starts + a.requests + 1;   // [requests], place of a request's first new block in the free list
  uint32_t* in_cache = first_free + a.requests;     // [requests], its cached tokens
  const uint32_t T = (uint32_t)a.tokens;
  const int most = (int)min((int64_t)a.width << a.shift, (int64_t)0x7fffffff);
  const uint32_t in_block = (1u << a.shift) - 1;
  const int r0 = (int)threadIdx.x * E;
  uint32_t c[E], f[E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int r = min(r0 + i, a.requests - 1);
    c[i] = a.requests ? (uint32_t)max(0, min(a.cached[r], most)) : 0;
    f[i] = a.requests ? (uint32_t)max(a.fresh[r], 0) : 0;
  }
  uint32_t mine = 0, all;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    f[i] = r0 + i < a.requests ? min(f[i], (uint32_t)most - c[i]) : 0;
    mine = add(mine, f[i]);
  }
  uint32_t at = min(block_exclusive<WG>(mine, room, &all), T), blocks = 0, first[E];
  // the requests' rows, and the blocks they need new
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int r = r0 + i;
    const uint32_t next = min(T, add(at, f[i]));
    first[i] = blocks;
    blocks += ((c[i] + (next - at) + in_block) >> a.shift) - ((c[i] + in_block) >> a.shift);
    if (r < a.requests) {
      starts[r] = at;
      in_cache[r] = c[i];
      if (blockIdx.x == 0) {
        a.starts[r] = (int)at;
        a.lengths[r] = (int)(c[i] + (next - at));
      }
    }
    at = next;
  }
  if (threadIdx.x == WG - 1) starts[a.requests] = at;      // (behind the last request nothing is added)
  const uint32_t blocks_before = block_exclusive<WG>(blocks, room, &all);
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (r0 + i < a.requests) first_free[r0 + i] = blocks_before + first[i];
  __syncthreads();
  const uint32_t total = starts[a.requests];
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.starts[a.requests] = (int)total;
    a.taken[0] = (int)min(all, (uint32_t)a.n_free);
    a.taken[1] = (int)all;
  }
  for (uint32_t t = blockIdx.x * WG + threadIdx.x; t < T; t += gridDim.x * WG) {
    int position = 0, slot = -1;
    if (t < total) {
      int lo = 0, hi = a.requests;      // starts[lo] <= t < starts[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= t) lo = mid; else hi = mid;
      }
      const uint32_t c = in_cache[lo], p = c + (t - starts[lo]), entry = p >> a.shift, have = (c + in_block) >> a.shift;
      int* row = a.tables + (int64_t)lo * a.width;
      int block;
      if (entry < have) {
        block = row[entry];
      } else {
        const uint32_t k = first_free[lo] + entry - have;
        block = k < (uint32_t)a.n_free ? a.free[k] : -1;
        if ((p & in_block) == 0) row[entry] = block;
      }
      position = (int)p;
      if (block >= 0 && block < a.blocks) slot = (int)(((uint32_t)block << a.shift) + (p & in_block));
    }
    a.positions[t] = position;
    a.slots[t] = slot;
  }
}

}  // namespace

int block_tables_launch(const BlockTablesSpec& s, const void* const* in, void* const* out, void* stream, std::string* err) {
  const auto i = [&](int k) { return static_cast<const int*>(in[k]); };
  const auto o = [&](int k) { return static_cast<int*>(out[k]); };
  const TablesArgs a{i(0), i(1), i(2), o(0), o(1), o(2), o(3), o(4), o(5), s.d.requests, s.d.tokens, s.d.blocks, __builtin_ctz((unsigned)s.d.block_size), s.d.table_blocks, s.d.free_blocks};
  const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(s.grid), dim3(s.wg), (size_t)s.lds, static_cast<hipStream_t>(stream), a); };
  if (s.wg == 64) launch(block_tables_kernel<64, 1>);
  else if (s.wg == 256) launch(block_tables_kernel<256, 1>);
  else if (s.d.requests <= 1024) launch(block_tables_kernel<1024, 1>);
  else launch(block_tables_kernel<1024, 4>);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { *err = std::string("block_tables launch: ") + hipGetErrorString(e); return -1; }
  return 0;
}

}  // namespace fs
