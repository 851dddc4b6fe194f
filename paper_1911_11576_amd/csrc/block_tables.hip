// Block tables and slot maps from request lengths (fs_plan_create_block_tables).
//
// With c the cached and f the new tokens of a request, both cut as fs.h says, S the exclusive sum of f over the requests:
//   starts = min(S, T),  f' = the difference of its neighbours,  have = ceil(c / bs),  need = ceil((c + f') / bs)
//   request's first new block = free[exclusive sum of (need - have)]
// Both sums are scans of at most 4096 numbers: every workgroup makes them for itself in LDS (8 bytes a request read through
// the caches), which costs less than a kernel that hands them over, and then serves its run of rows, each row finding its
// request by bisection.  A block that a request gets new is written into the table by the row of its first token: no
// workgroup reads an entry that another writes, so the table is updated in place.  All of it is a launch and four dependent
// memory accesses (lengths -> entry or free list -> stores); no step's bytes come near a bandwidth.
#include "dev_common.h"
#include "paged.h"

namespace fs {
namespace {

struct TablesArgs {
  const int *cached, *fresh, *free;
  int *tables, *lengths, *starts, *positions, *slots, *taken;
  int requests, tokens, blocks, shift, width, n_free;
};

// Sum over the threads before this one; `room` has a place per wavefront, and *all gets the workgroup's total.
template <int WG> __device__ __forceinline__ uint64_t block_exclusive(uint64_t v, uint64_t* room, uint64_t* all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint64_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t t = __shfl_up((unsigned long long)s, d);
    if (lane >= d) s += t;
  }
  if constexpr (WG == 64) {
    *all = __shfl((unsigned long long)s, 63);
    return s - v;
  }
  if (lane == 63) room[w] = s;
  __syncthreads();
  uint64_t before = s - v, total = 0;
#pragma unroll
  for (int k = 0; k < WG / 64; ++k) {
    if (k < w) before += room[k];
    total += room[k];
  }
  *all = total;
  __syncthreads();
  return before;
}

template <int WG> __global__ __launch_bounds__(WG) void block_tables_kernel(const TablesArgs a) {
  extern __shared__ uint64_t smem[];
  uint64_t* room = smem;                            // [4]
  uint32_t* starts = reinterpret_cast<uint32_t*>(smem + 4);      // [requests + 1]
  uint32_t* first_free = starts + a.requests + 1;   // [requests], place of a request's first new block in the free list
  const uint32_t T = (uint32_t)a.tokens;
  const int most = (int)min((int64_t)a.width << a.shift, (int64_t)0x7fffffff);
  const uint32_t in_block = (1u << a.shift) - 1;
  const int each = (a.requests + WG - 1) / WG;
  const int r0 = min((int)threadIdx.x * each, a.requests), r1 = min(r0 + each, a.requests);
  auto cached_of = [&](int r) { return max(0, min(a.cached[r], most)); };
  auto fresh_of = [&](int r, int c) { return (uint32_t)min(max(a.fresh[r], 0), most - c); };
  uint64_t mine = 0, all;
  for (int r = r0; r < r1; ++r) mine += fresh_of(r, cached_of(r));
  uint32_t at = (uint32_t)min(block_exclusive<WG>(mine, room, &all), (uint64_t)T), blocks = 0;
  // the requests' rows, and the blocks they need new
  for (int r = r0; r < r1; ++r) {
    const int c = cached_of(r);
    const uint32_t next = (uint32_t)min((uint64_t)T, (uint64_t)at + fresh_of(r, c));
    starts[r] = at;
    first_free[r] = blocks;
    blocks += (((uint32_t)c + (next - at) + in_block) >> a.shift) - (((uint32_t)c + in_block) >> a.shift);
    if (blockIdx.x == 0) {
      a.starts[r] = (int)at;
      a.lengths[r] = c + (int)(next - at);
    }
    at = next;
  }
  if (threadIdx.x == WG - 1) starts[a.requests] = at;      // (the last thread's run ends where the requests do, or is empty behind them)
  const uint32_t blocks_before = (uint32_t)block_exclusive<WG>(blocks, room, &all);
  for (int r = r0; r < r1; ++r) first_free[r] += blocks_before;
  __syncthreads();
  const uint32_t total = starts[a.requests];
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.starts[a.requests] = (int)total;
    a.taken[0] = (int)min(all, (uint64_t)a.n_free);
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
      const uint32_t c = (uint32_t)cached_of(lo), p = c + (t - starts[lo]), entry = p >> a.shift, have = (c + in_block) >> a.shift;
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
  if (s.wg == 64) hipLaunchKernelGGL(block_tables_kernel<64>, dim3(s.grid), dim3(64), (size_t)s.lds, static_cast<hipStream_t>(stream), a);
  else hipLaunchKernelGGL(block_tables_kernel<256>, dim3(s.grid), dim3(256), (size_t)s.lds, static_cast<hipStream_t>(stream), a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { *err = std::string("block_tables launch: ") + hipGetErrorString(e); return -1; }
  return 0;
}

}  // namespace fs
