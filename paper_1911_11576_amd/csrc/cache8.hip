// A paged cache in 8 bits: new keys and values quantised as they are written, and read back (fs_plan_create_cache_store8,
// fs_plan_create_cache_read8).  A code c of block b and head h stands for c * scales[b, h]; both kernels move bytes and little else.
#include <algorithm>

#include "cache8.h"

namespace fs {

struct Cache8Args {
  const void *k, *v;               // numbers: the store's, written by the read
  void *k_codes, *v_codes;
  float *k_scales, *v_scales;
  const int *tables, *lengths, *starts;
  int64_t k_stride, v_stride;
  CacheLayout cache;
  int requests, tokens, heads, width, pieces;      // pieces: of 16 codes of a head's row
  int groups;                      // store: workgroups of a place; read: rows of a workgroup
  int64_t items;                   // store: workgroups' worth of work
  uint32_t row_inv, piece_inv;     // read: items of a row, pieces of a head, as factors of a multiplication
};

// A request: its first row, its new tokens, its tokens; the position of the first row's token (below 0 where there are more rows than tokens).
struct Cache8Request { int first, fresh, keys; };
__device__ __forceinline__ Cache8Request cache8_request(const Cache8Args& a, int b) {
  Cache8Request r;
  r.first = min(max(a.starts[b], 0), a.tokens);
  r.fresh = max(0, min(max(a.starts[b + 1], 0), a.tokens) - r.first);
  r.keys = (int)min((int64_t)max(a.lengths[b], 0), (int64_t)a.width << a.cache.shift);
  return r;
}

// The last of the requests [lo, lo + n) for which at_most(b) holds, which holds for every one before it too; -1: for none.  64 of them looked at at a time.
template <class F> __device__ __forceinline__ int find_last(int lo, int n, F at_most) {
  const int lane = threadIdx.x & 63, end = lo + n;
  for (;;) {
    const int step = (n + 63) >> 6, b = lo + lane * step;
    const int here = __popcll(__ballot(b < lo + n && at_most(min(b, end - 1))));
    if (here == 0) return -1;
    lo += (here - 1) * step;
    if (step == 1) return lo;
    n = min(step, end - lo);
  }
}

// ---- store

// 16 numbers as they lie in memory: what a lane takes of a row
template <typename T> struct Raw16 { u32x4 w[2]; };
template <> struct Raw16<float> { u32x4 w[4]; };
template <typename T> __device__ __forceinline__ Raw16<T> load16(const T* p) {
  Raw16<T> r;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r.w) / 16); ++i) r.w[i] = stream_load16(reinterpret_cast<const u32x4*>(p) + i);
  return r;
}
// the largest of them without their signs, as bits that are ordered as the numbers are, infinities and NaN above all: of pairs in halves of a word
template <typename T> __device__ __forceinline__ uint32_t top_bits(uint32_t top, const Raw16<T>& r) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r.w) / 16); ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 4) {
        top = max(top, r.w[i][j] & 0x7fffffffu);
      } else {
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, r.w[i][j] & 0x7fff7fffu)));
      }
    }
  return top;
}
template <typename T> __device__ __forceinline__ float top_number(uint32_t bits) {
  if constexpr (sizeof(T) == 4) return as_f32(bits);
  else {
    const uint32_t b = max(bits & 0xffffu, bits >> 16);
    if constexpr (sizeof(T) == 2 && __is_same(T, bf16_t)) return bf16_to_f32(b);
    else return f16_to_f32(b);
  }
}
template <typename T> __device__ __forceinline__ void numbers(const Raw16<T>& r, float (&x)[16]) {
  constexpr int V = Vec<T>::V;
#pragma unroll
  for (int i = 0; i < 16 / V; ++i) {
    float y[V];
    Vec<T>::unpack(r.w[i], y);
#pragma unroll
    for (int j = 0; j < V; ++j) x[V * i + j] = y[j];
  }
}

// Codes of x * 2^power, rounded once, to the nearest and the even one of two.
template <class Code> __device__ __forceinline__ u32x4 codes_of(const float (&x)[16], int power) {
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = __builtin_ldexpf(x[4 * i + j], power);
    out[i] = Code::pack(y[0], y[1], y[2], y[3]);
  }
  return out;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, k));
  return v;
}
template <typename T> __device__ __forceinline__ uint32_t wave_top(uint32_t v) {      // halves apart, or whole words
  if constexpr (sizeof(T) == 4) return wave_max(v);
  else return wave_max(max(v & 0xffffu, v >> 16));
}

// W wavefronts do a block's part of one request and one head of K or of V: the new numbers, N pieces of 16 of a thread's in registers, their maximum, the
// block's scale, its codes from before in that scale where it grew, the new codes.  What registers do not hold is read twice.
template <typename T, class Code, int W, int N> __global__ __launch_bounds__(256) void cache8_store_kernel(const Cache8Args a) {
  __shared__ uint32_t tops[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int size = 1 << a.cache.shift;
  for (int64_t item = blockIdx.x; item < a.items; item += gridDim.x) {
    // ---- where: request b's blocks begin at place start / size + 2 b, as many places as it can touch blocks
    const int at = (int)(item / a.groups), unit = (int)(item - (int64_t)at * a.groups) * (4 / W) + wave / W;
    auto place = [&](int b) { return (min(max(a.starts[b], 0), a.tokens) >> a.cache.shift) + 2 * b; };
    const int b = find_last(0, a.requests, [&](int i) { return place(i) <= at; });
    bool work = b >= 0 && unit < 2 * a.heads;
    const bool values = unit >= a.heads;
    const int head = values ? unit - a.heads : unit;
    int lo = 0, n = 0, page = -1;
    int64_t row = 0;
    if (work) {
      const Cache8Request r = cache8_request(a, b);
      const int first = r.keys - r.fresh, j = (max(first, 0) >> a.cache.shift) + at - place(b);
      work = r.fresh > 0 && r.keys > 0 && j >= 0 && j <= (r.keys - 1) >> a.cache.shift;
      if (work) {
        page = a.tables[(int64_t)b * a.width + j];
        work = (unsigned)page < (unsigned)a.cache.blocks;
        const int begin = j << a.cache.shift;
        lo = max(0, max(first, 0) - begin);
        n = min(size, r.keys - begin) - lo;
        row = (int64_t)r.first + begin + lo - first;
        work = work && n > 0;
      }
    }
    if (!work) {
      if (W > 1) { __syncthreads(); __syncthreads(); }      // (W 4: the whole workgroup is here)
      continue;
    }
    const T* from = static_cast<const T*>(values ? a.v : a.k) + row * (values ? a.v_stride : a.k_stride) + (int64_t)head * a.pieces * 16;
    const int64_t stride = values ? a.v_stride : a.k_stride;
    uint8_t* codes = static_cast<uint8_t*>(values ? a.v_codes : a.k_codes) + (int64_t)page * a.cache.block + (int64_t)head * a.cache.head;
    float* scale_at = (values ? a.v_scales : a.k_scales) + (int64_t)page * a.heads + head;
    // ---- the thread's pieces: piece `p` of rows r0, r0 + rows, ...
    const int t = lane + 64 * (wave % W), rows = 64 * W / a.pieces, r0 = t / a.pieces, p = t - r0 * a.pieces;
    const int last = r0 < rows ? n : 0;      // (threads behind the last whole row have none)
    Raw16<T> x[N];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (r0 + i * rows < last) x[i] = load16(from + (r0 + i * rows) * stride + 16 * p);
    const float before = *scale_at;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (r0 + i * rows < last) top = top_bits<T>(top, x[i]);
    for (int r = r0 + N * rows; r < last; r += rows) top = top_bits<T>(top, load16(from + r * stride + 16 * p));
    top = wave_top<T>(top);
    if (W > 1) {
      if (lane == 0) tops[wave] = top;
      __syncthreads();
      top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
      __syncthreads();      // (before the next item's)
    }
    // ---- the scale, 2^power; NaN where a new number is none, or the scale from before
    const float most = top_number<T>(top);
    int power = max(-126, Code::power(most));
    bool nan = !(most < INFINITY);
    if (lo) {
      const uint32_t old = as_u32(before) & 0x7fffffffu;
      const int up = max(-126, (int)(old >> 23) - 127 + ((old & 0x7fffffu) != 0));
      power = max(power, up);
      nan |= up > 127;      // (infinities and NaN are 2^128 and more here)
    }
    const float now = nan ? __builtin_nanf("") : as_f32((uint32_t)(power + 127) << 23);
    const bool grown = lo && !nan && now != before;
    // ---- codes from before
    if (grown) {
      for (int r = r0; r < (r0 < rows ? lo : 0); r += rows) {
        u32x4* c = reinterpret_cast<u32x4*>(codes + (int64_t)r * a.cache.slot + 16 * p);
        const u32x4 was = *c;
        const float ratio = __builtin_ldexpf(before, -power);
        float y[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float z[4];
          Code::unpack(was[i], z);
#pragma unroll
          for (int j = 0; j < 4; ++j) y[4 * i + j] = z[j] * ratio;
        }
        *c = codes_of<Code>(y, 0);
      }
    }
    // ---- the new ones
    auto put = [&](int r, const Raw16<T>& raw) __attribute__((always_inline)) {
      float y[16];
      numbers(raw, y);
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = __builtin_amdgcn_fmed3f(y[i], -Code::template kMost<T>, Code::template kMost<T>);
      u32x4 c = codes_of<Code>(y, -power);
      if (nan) c = u32x4{0u, 0u, 0u, 0u};
      *reinterpret_cast<u32x4*>(codes + (int64_t)(lo + r) * a.cache.slot + 16 * p) = c;
    };
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (r0 + i * rows < last) put(r0 + i * rows, x[i]);
    for (int r = r0 + N * rows; r < last; r += rows) put(r, load16(from + r * stride + 16 * p));
    if (t == 0) *scale_at = now;
  }
}

template <typename T, class Code> void store_launch(const Cache8Args& a, int waves, int grid, hipStream_t s) {
  if (waves == 1) hipLaunchKernelGGL((cache8_store_kernel<T, Code, 1, 4>), dim3(grid), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((cache8_store_kernel<T, Code, 4, 4>), dim3(grid), dim3(256), 0, s, a);
}

// ---- read

// A workgroup has a.groups rows (tokens): where each one's codes lie is found once, by a thread a row, then 8 codes to a thread.
constexpr int kRowsMost = 64;
template <typename T, class Code> __global__ __launch_bounds__(256) void cache8_read_kernel(const Cache8Args a) {
  __shared__ int64_t where[kRowsMost];      // of a row: its place in the cache's codes; -1: it is written as zeros, -2: it is nobody's
  __shared__ int pages[kRowsMost];
  constexpr int U = 4;
  const int lane = threadIdx.x & 63, halves = 2 * a.pieces, each = 2 * a.heads * halves;      // 8 codes: of a head, of a row
  for (int t0 = blockIdx.x * a.groups; t0 < a.tokens; t0 += gridDim.x * a.groups) {
    const int rows = min(a.groups, a.tokens - t0);
    if (threadIdx.x < 64) {
      auto begins = [&](int t) { return [&, t](int b) { return min(max(a.starts[b], 0), a.tokens) <= t; }; };
      const int b0 = find_last(0, a.requests, begins(t0)), b1 = find_last(max(b0, 0), a.requests - max(b0, 0), begins(t0 + rows - 1));
      const int t = t0 + lane;
      int64_t at = -2;
      int page = 0;
      if (lane < rows && b1 >= 0) {
        int lo = b0, hi = b1;      // the last request that begins at or before t
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (begins(t)(mid)) lo = mid; else hi = mid - 1;
        }
        if (lo >= 0) {
          const Cache8Request r = cache8_request(a, lo);
          if (t >= r.first && t < r.first + r.fresh) {
            at = -1;
            const int p = r.keys - r.fresh + t - r.first;
            if (p >= 0) {
              page = a.tables[(int64_t)lo * a.width + (p >> a.cache.shift)];
              if ((unsigned)page < (unsigned)a.cache.blocks) at = (int64_t)page * a.cache.block + (int64_t)(p & ((1 << a.cache.shift) - 1)) * a.cache.slot;
            }
          }
        }
      }
      if (lane < kRowsMost) { where[lane] = at; pages[lane] = page; }
    }
    __syncthreads();
    const int items = rows * each;
      for (int i0 = threadIdx.x; i0 < items; i0 += 256 * U) {
      u32x2 c[U];
      float s[U];
      T* to[U];
      int kind[U];
  #pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + 256 * u;
        kind[u] = 0;
        if (i >= items) continue;
        const int r = a.groups == 1 ? 0 : (int)__umulhi((uint32_t)i, a.row_inv), rest = i - r * each, h = (int)__umulhi((uint32_t)rest, a.piece_inv), p = rest - h * halves;
        const int64_t at = where[r];
        if (at == -2) continue;
        const bool values = h >= a.heads;
        const int head = values ? h - a.heads : h;
        to[u] = static_cast<T*>(const_cast<void*>(values ? a.v : a.k)) + (t0 + r) * (values ? a.v_stride : a.k_stride) + (int64_t)head * a.pieces * 16 + 8 * p;
        kind[u] = 1;
        c[u] = u32x2{0u, 0u};
        s[u] = 0.f;
        if (at >= 0) {
          c[u] = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(values ? a.v_codes : a.k_codes) + at + (int64_t)head * a.cache.head + 8 * p);
          s[u] = (values ? a.v_scales : a.k_scales)[(int64_t)pages[r] * a.heads + head];
        }
      }
  #pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!kind[u]) continue;
        float x[8], y[4];
  #pragma unroll
        for (int i = 0; i < 2; ++i) {
          Code::unpack(c[u][i], y);
  #pragma unroll
          for (int j = 0; j < 4; ++j) x[4 * i + j] = y[j] * s[u];
        }
        if constexpr (sizeof(T) == 4) {
          reinterpret_cast<f32x4*>(to[u])[0] = f32x4{x[0], x[1], x[2], x[3]};
          reinterpret_cast<f32x4*>(to[u])[1] = f32x4{x[4], x[5], x[6], x[7]};
        } else {
          *reinterpret_cast<u32x4*>(to[u]) = pack16<T>(x);
        }
      }
    }
    __syncthreads();      // (before the next rows')
  }
}

// ---- geometry and launches

void cache8_geometry(Cache8Spec* s, bool store) {
  const fs_cache8_desc& d = s->d;
  const int pieces = d.head_dim / 16;
  if (store) {
    // a wavefront holds 4 * (64 / pieces) rows of a block, the others are read twice: four wavefronts where a block has more
    s->waves = d.block_size > 4 * (64 / pieces) ? 4 : 1;
    const int64_t places = ((int64_t)d.tokens >> s->cache.shift) + 2ll * d.requests;
    s->groups = (2 * d.kv_heads * s->waves + 3) / 4;
    s->items = places * s->groups;
    s->grid = (int)std::min<int64_t>(s->items, 1 << 23);
    return;
  }
  const int64_t each = 4ll * d.kv_heads * pieces;
  s->groups = (int)std::max<int64_t>(1, std::min<int64_t>(kRowsMost, 2048 / each));
  s->grid = (int)std::min<int64_t>(((int64_t)d.tokens + s->groups - 1) / s->groups, 1 << 23);
}

int cache8_launch(const Cache8Spec& s, bool store, const void* const* in, void* const* out, void* stream, std::string* err) {
  const fs_cache8_desc& d = s.d;
  if (d.tokens == 0 || d.requests == 0) return 0;
  Cache8Args a{};
  if (store) {
    a.k = in[0]; a.v = in[1];
    a.k_codes = out[0]; a.v_codes = out[1]; a.k_scales = static_cast<float*>(out[2]); a.v_scales = static_cast<float*>(out[3]);
  } else {
    a.k = out[0]; a.v = out[1];
    a.k_codes = const_cast<void*>(in[0]); a.v_codes = const_cast<void*>(in[1]);
    a.k_scales = static_cast<float*>(const_cast<void*>(in[2])); a.v_scales = static_cast<float*>(const_cast<void*>(in[3]));
  }
  const void* const* tables = in + (store ? 2 : 4);
  a.tables = static_cast<const int*>(tables[0]); a.lengths = static_cast<const int*>(tables[1]); a.starts = static_cast<const int*>(tables[2]);
  a.k_stride = d.k_stride; a.v_stride = d.v_stride;
  a.cache = s.cache;
  a.requests = d.requests; a.tokens = d.tokens; a.heads = d.kv_heads;
  a.width = d.blocks ? d.table_blocks : 0;      // (without a block there is no token to write or read)
  a.pieces = d.head_dim / 16;
  a.groups = s.groups; a.items = s.items;
  // i / n as the high half of i * ceil(2^32 / n), right while i * n <= 2^32: i < 2^11 where there are several rows, n <= 64 for the pieces of a head
  auto inverse = [](int64_t n) { return (uint32_t)(((1ll << 32) + n - 1) / n); };
  a.row_inv = inverse(4ll * d.kv_heads * a.pieces);
  a.piece_inv = inverse(2ll * a.pieces);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool e4m3 = d.code == FS_CODE_E4M3;
  if (store) {
    auto go = [&](auto type) {
      typedef decltype(type) T;
      if (e4m3) store_launch<T, E4m3>(a, s.waves, s.grid, st); else store_launch<T, Int8>(a, s.waves, s.grid, st);
    };
    if (d.dtype == FS_F32) go(float{}); else if (d.dtype == FS_F16) go(f16_t{}); else go(bf16_t{});
  } else {
    auto go = [&](auto type) {
      typedef decltype(type) T;
      if (e4m3) hipLaunchKernelGGL((cache8_read_kernel<T, E4m3>), dim3(s.grid), dim3(256), 0, st, a);
      else hipLaunchKernelGGL((cache8_read_kernel<T, Int8>), dim3(s.grid), dim3(256), 0, st, a);
    };
    if (d.dtype == FS_F32) go(float{}); else if (d.dtype == FS_F16) go(f16_t{}); else go(bf16_t{});
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { *err = std::string(store ? "cache_store8" : "cache_read8") + " launch: " + hipGetErrorString(e); return -1; }
  return 0;
}

}  // namespace fs
