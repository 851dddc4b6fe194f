// Attention of new tokens over a paged cache (fs_plan_create_paged_attention).
//
// One wavefront a row (a token's query head): 64 keys at a time, a lane's dot product each, the running maximum and sum of a
// softmax over the wavefront, then every lane adds up its elements of the values that are seen.
#include <algorithm>

#include "dev_common.h"
#include "paged.h"

namespace fs {
namespace {

struct PagedArgs {
  const void *q, *k, *v;
  const int *tables, *lengths, *starts;
  void* out;
  float* lse;
  int64_t q_stride, out_stride;
  CacheLayout cache;
  int requests, tokens, q_heads, share, width, causal, window;
  float scale;
};

template <typename T, int D> __global__ __launch_bounds__(64) void paged_rows_kernel(const PagedArgs a) {
  constexpr int E = (D + 63) / 64;
  const int lane = threadIdx.x, token = blockIdx.x, head = blockIdx.y;
  __shared__ float qs[D];
  int lo = 0, hi = a.requests;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (min(max(a.starts[mid], 0), a.tokens) <= token) lo = mid; else hi = mid;
  }
  const int first = min(max(a.starts[lo], 0), a.tokens), end = min(max(a.starts[lo + 1], 0), a.tokens);
  if (token < first || token >= end) return;
  const int keys = (int)min((int64_t)max(a.lengths[lo], 0), (int64_t)a.width << a.cache.shift);
  const int position = keys - (end - first) + token - first;
  const int until = a.causal ? min(keys, position + 1) : keys, from = a.window ? max(0, position + 1 - a.window) : 0;
  const T* q = static_cast<const T*>(a.q) + token * a.q_stride + (int64_t)head * D;
  for (int d = lane; d < D; d += 64) qs[d] = Vec<T>::load1(q + d) * a.scale;
  __syncthreads();
  const int64_t head_at = (int64_t)(head / a.share) * a.cache.head;
  float m = -INFINITY, sum = 0.f, o[E] = {};
  for (int j0 = from; j0 < until; j0 += 64) {
    const int j = j0 + lane;
    int64_t at = -1;
    float s = -INFINITY;
    if (j < until) {
      const int block = a.tables[(int64_t)lo * a.width + (j >> a.cache.shift)];
      if (block >= 0 && block < a.cache.blocks) {
        at = block * a.cache.block + (int64_t)(j & ((1 << a.cache.shift) - 1)) * a.cache.slot + head_at;
        const T* k = static_cast<const T*>(a.k) + at;
        s = 0.f;
        for (int d = 0; d < D; d += 8) {
          float x[8];
          Vec<T>::load(k + d, x);
#pragma unroll
          for (int i = 0; i < 8; ++i) s = fmaf(qs[d + i], x[i], s);
        }
      }
    }
    const float top = fmaxf(m, group_allreduce<MaxOp, 64>(s));
    const float base = top == -INFINITY ? 0.f : top;
    const float p = at < 0 ? 0.f : __expf(s - base), keep = __expf(m - base);
    sum = sum * keep + group_allreduce<SumOp, 64>(p);
    m = top;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= keep;
    for (int i = 0; i < 64 && j0 + i < until; ++i) {
      const int64_t row = __shfl((long long)at, i);
      const float w = __shfl(p, i);
      if (row < 0) continue;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (lane + 64 * e < D) o[e] = fmaf(w, Vec<T>::load1(static_cast<const T*>(a.v) + row + lane + 64 * e), o[e]);
    }
  }
  T* out = static_cast<T*>(a.out) + token * a.out_stride + (int64_t)head * D;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (lane + 64 * e < D) Vec<T>::store1(out + lane + 64 * e, sum == 0.f ? 0.f : o[e] / sum);
  if (a.lse && lane == 0) a.lse[(int64_t)token * a.q_heads + head] = sum == 0.f ? -INFINITY : m + __logf(sum);
}

template <typename T> void launch_type(const PagedArgs& a, int dim, hipStream_t s) {
  const dim3 grid(a.tokens, a.q_heads);
  switch (dim) {
    case 32: hipLaunchKernelGGL((paged_rows_kernel<T, 32>), grid, dim3(64), 0, s, a); break;
    case 64: hipLaunchKernelGGL((paged_rows_kernel<T, 64>), grid, dim3(64), 0, s, a); break;
    case 96: hipLaunchKernelGGL((paged_rows_kernel<T, 96>), grid, dim3(64), 0, s, a); break;
    default: hipLaunchKernelGGL((paged_rows_kernel<T, 128>), grid, dim3(64), 0, s, a); break;
  }
}

}  // namespace

bool paged_attn_plan(PagedAttnSpec* s, int* n_kernels, int64_t* lds_bytes, std::string* err) {
  (void)err;
  s->partial_bytes = 0;
  *n_kernels = 1;
  *lds_bytes = 4 * s->d.head_dim;
  return true;
}

std::string paged_attn_describe(const PagedAttnSpec& s) {
  char buf[200];
  snprintf(buf, sizeof buf, "paged_attention[GRID-WARP,WARP] rows=%lld, cta_num=%lld, cta_size=64", (long long)s.d.tokens * s.d.q_heads, (long long)s.d.tokens * s.d.q_heads);
  return buf;
}

int paged_attn_launch(const PagedAttnSpec& s, const void* const* in, void* const* out, void* stream, std::string* err) {
  if (s.d.tokens == 0 || s.d.requests == 0) return 0;
  PagedArgs a{};
  a.q = in[0]; a.k = in[1]; a.v = in[2];
  a.tables = static_cast<const int*>(in[3]); a.lengths = static_cast<const int*>(in[4]); a.starts = static_cast<const int*>(in[5]);
  a.out = out[0];
  if (s.d.log_sum_exp) a.lse = static_cast<float*>(out[1]);
  a.q_stride = s.d.q_stride; a.out_stride = s.d.out_stride;
  a.cache = s.cache;
  a.requests = s.d.requests; a.tokens = s.d.tokens; a.q_heads = s.d.q_heads; a.share = s.share; a.width = s.d.table_blocks; a.causal = s.d.causal; a.window = s.d.window;
  a.scale = (float)s.d.scale;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (s.d.dtype == FS_F16) launch_type<f16_t>(a, s.d.head_dim, st);
  else launch_type<bf16_t>(a, s.d.head_dim, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { *err = std::string("paged_attention launch: ") + hipGetErrorString(e); return -1; }
  return 0;
}

}  // namespace fs
