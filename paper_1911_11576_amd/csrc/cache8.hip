// A paged cache in 8 bits: new keys and values quantised as they are written, and read back (fs_plan_create_cache_store8,
// fs_plan_create_cache_read8).  A code c of block b and head h stands for c * scales[b, h]; both kernels move bytes and little else.
#include <algorithm>
#include <type_traits>

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
  int places, piece_inv;           // store: places of requests' blocks; 2^16 over the pieces of 8 of a row, rounded up
};

// A request: its first row, its new tokens, its tokens.
struct Cache8Request { int b, first, fresh, keys; };
__device__ __forceinline__ int cache8_start(const Cache8Args& a, int b) { return min(max(a.starts[b], 0), a.tokens); }
__device__ __forceinline__ int cache8_keys(const Cache8Args& a, int b) { return (int)min((int64_t)max(a.lengths[b], 0), (int64_t)a.width << a.cache.shift); }

// The last request for which at_most(its first row, its number) holds, which holds for every one before it too (b -1: none).  64 of them are looked at at a
// time, one a lane, and what is known of the last 64 is requested with them: one access to memory, two from 65 requests on, three from 4097.
template <class F> __device__ __forceinline__ Cache8Request find_last(const Cache8Args& a, F at_most) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.requests;
  while (n > 64) {
    const int step = (n + 63) >> 6, b = lo + lane * step;
    const int here = __popcll(__ballot(b < lo + n && at_most(cache8_start(a, min(b, a.requests - 1)), b)));
    if (here == 0) return Cache8Request{-1, 0, 0, 0};
    n = min(step, n - (here - 1) * step);
    lo += (here - 1) * step;
  }
  const int b = min(lo + lane, a.requests - 1), first = cache8_start(a, b), end = cache8_start(a, b + 1), keys = cache8_keys(a, b);
  const int here = __popcll(__ballot(lane < n && at_most(first, b)));
  if (here == 0) return Cache8Request{-1, 0, 0, 0};
  const int f = __builtin_amdgcn_readlane(first, here - 1);
  return Cache8Request{lo + here - 1, f, max(0, __builtin_amdgcn_readlane(end, here - 1) - f), __builtin_amdgcn_readlane(keys, here - 1)};
}

// ---- store

// 8 numbers as they lie in memory: what a lane takes of a row at a time, whole lines by neighbouring lanes
template <typename T> struct Raw8 { u32x4 w[1]; };
template <> struct Raw8<float> { u32x4 w[2]; };
template <typename T, bool ONCE> __device__ __forceinline__ Raw8<T> load8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r.w) / 16); ++i) r.w[i] = ONCE ? stream_load16(reinterpret_cast<const u32x4*>(p) + i) : reinterpret_cast<const u32x4*>(p)[i];
  return r;
}
// the largest of them without their signs, as bits that are ordered as the numbers are, infinities and NaN above all: of pairs in halves of a word
template <typename T> __device__ __forceinline__ uint32_t top_bits(uint32_t top, const Raw8<T>& r) {
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
// The codes of 8 numbers over 2^power; CUT: those beyond `limit` as that, the largest number of T that such a code stands for.
template <typename T, class Code, bool CUT> __device__ __forceinline__ u32x2 codes_of(const Raw8<T>& r, int power, float limit) {
  if constexpr (sizeof(T) == 2 && !CUT) {
    return u32x2{Code::template pack_words<T>(r.w[0][0], r.w[0][1], power), Code::template pack_words<T>(r.w[0][2], r.w[0][3], power)};
  } else {
    constexpr int V = Vec<T>::V;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8 / V; ++i) {
      float y[V];
      Vec<T>::unpack(r.w[i], y);
#pragma unroll
      for (int j = 0; j < V; ++j) x[V * i + j] = CUT ? copysignf(fminf(fabsf(y[j]), limit), y[j]) : y[j];
    }
    return u32x2{Code::pack(x[0], x[1], x[2], x[3], power), Code::pack(x[4], x[5], x[6], x[7], power)};
  }
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false));
  auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(r[0], r[1]);
  r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)max(r[0], r[1]));
}
template <typename T> __device__ __forceinline__ uint32_t wave_top(uint32_t v) {      // halves apart, or whole words
  if constexpr (sizeof(T) == 4) return wave_max(v);
  else return wave_max(max(v & 0xffffu, v >> 16));
}

// W wavefronts do a block's part of one request and one head of K or V: the new numbers, N pieces of 8 of a thread's in registers, their maximum, the
// block's scale, its codes from before in that scale where it grew, the new codes.  What registers do not hold is read twice.  Bound by memory: 4.9 TB/s for 11014
// tokens, 8 heads of 128 in bf16 (13.8 us; with 16 numbers of a thread side by side and conversions by single instructions in fp32 18.5), 5.0 for 21253 tokens, 16 heads
// of 64 in fp16 side by side, into blocks of 64 (26.1 us; K and V by one wavefront 38, four wavefronts to a block 39).  ONCE: k and v past the caches where
// both are more than 64 MiB (those 26.1 us, 29.1 through the caches; the first 15.5 and 13.9).  The grid: all heads of a place one after the other on one XCD (workgroup n is
// dispatched to XCD n mod 8), eight places side by side; the 26.1 us are 27.1 where a place's heads go round the XCDs, 28.0 where all places of four heads come first.
template <typename T, class Code, int W, int N, bool ONCE> __global__ __launch_bounds__(256) void cache8_store_kernel(const Cache8Args a) {
  __shared__ uint32_t tops[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int size = 1 << a.cache.shift;
  for (int at = 8 * blockIdx.y + (blockIdx.x & 7); at < a.places; at += 8 * gridDim.y)
  for (int group = blockIdx.x >> 3; group < a.groups; group += gridDim.x >> 3) {
    // ---- where: request b's blocks begin at place start / size + 2 b, as many places as it can touch blocks
    const int unit = group * (4 / W) + wave / W;
    auto place = [&](int first, int b) { return (first >> a.cache.shift) + 2 * b; };
    const Cache8Request r = find_last(a, [&](int first, int b) { return place(first, b) <= at; });
    bool work = r.b >= 0 && unit < 2 * a.heads;
    const bool values = unit >= a.heads;
    const int head = values ? unit - a.heads : unit;
    int lo = 0, n = 0, page = -1;
    int64_t row = 0;
    if (work) {
      const int first = r.keys - r.fresh, j = (max(first, 0) >> a.cache.shift) + at - place(r.first, r.b);
      work = r.fresh > 0 && r.keys > 0 && j >= 0 && j <= (r.keys - 1) >> a.cache.shift;
      if (work) {
        page = a.tables[(int64_t)r.b * a.width + j];
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
    const int64_t stride = values ? a.v_stride : a.k_stride;
    const T* from = static_cast<const T*>(values ? a.v : a.k) + row * stride + (int64_t)head * a.pieces * 16;
    uint8_t* codes = static_cast<uint8_t*>(values ? a.v_codes : a.k_codes) + (int64_t)page * a.cache.block + (int64_t)head * a.cache.head;
    float* scale_at = (values ? a.v_scales : a.k_scales) + (int64_t)page * a.heads + head;
    // ---- the thread's pieces: piece `p` of rows r0, r0 + rows, ...
    const int t = lane + 64 * (wave % W), pieces = 2 * a.pieces, rows = 64 * W * a.piece_inv >> 16, r0 = t * a.piece_inv >> 16, p = t - r0 * pieces;
    const int last = r0 < rows ? n : 0;      // (threads behind the last whole row have none)
    Raw8<T> x[N];
    uint32_t top = 0;
    const float before = *scale_at;
    // (row r0 + r: a scalar base, and an offset of 32 bits that is the same for all of the thread's rows)
    const uint32_t in_row = (uint32_t)(r0 * (int)stride + 8 * p) * (uint32_t)sizeof(T);
    auto row_at = [&](int r) __attribute__((always_inline)) { return reinterpret_cast<const T*>(reinterpret_cast<const char*>(from + r * stride) + in_row); };
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (r0 + i * rows < last) x[i] = load8<T, ONCE>(row_at(i * rows));
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (r0 + i * rows < last) top = top_bits<T>(top, x[i]);
    for (int r = N * rows; r0 + r < last; r += rows) top = top_bits<T>(top, load8<T, ONCE>(row_at(r)));
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
    // ---- codes from before
    if (lo && !nan && now != before) {
      const float ratio = __builtin_ldexpf(before, -power);
      constexpr int U = 4;      // rows in flight
      for (int r = r0; r < (r0 < rows ? lo : 0); r += U * rows) {
        u32x2 was[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (r + u * rows < lo) was[u] = *reinterpret_cast<const u32x2*>(codes + (int64_t)(r + u * rows) * a.cache.slot + 8 * p);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (r + u * rows >= lo) continue;
          u32x2 codes_now;
#pragma unroll
          for (int i = 0; i < 2; ++i) codes_now[i] = Code::times(was[u][i], ratio);
          *reinterpret_cast<u32x2*>(codes + (int64_t)(r + u * rows) * a.cache.slot + 8 * p) = codes_now;
        }
      }
    }
    // ---- the new ones
    auto put = [&](auto cut) __attribute__((always_inline)) {
      const float limit = decltype(cut)::value ? Code::template most<T>(power) : 0.f;
      auto one = [&](int r, const Raw8<T>& raw) __attribute__((always_inline)) {
        u32x2 c = codes_of<T, Code, decltype(cut)::value>(raw, power, limit);
        if (decltype(cut)::value && nan) c = u32x2{0u, 0u};
        *reinterpret_cast<u32x2*>(codes + (int64_t)(lo + r) * a.cache.slot + 8 * p) = c;
      };
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (r0 + i * rows < last) one(r0 + i * rows, x[i]);
      for (int r = N * rows; r0 + r < last; r += rows) one(r0 + r, load8<T, ONCE>(row_at(r)));
    };
    // (no code stands for more than twice its number, whatever the scale)
    if (nan || most >= (__is_same(T, f16_t) ? 0x1p15f : 0x1p127f)) put(std::true_type{});
    else put(std::false_type{});
    if (t == 0) *scale_at = now;
  }
}

template <typename T, class Code, bool ONCE> void store_launch(const Cache8Args& a, int passes, int waves, dim3 grid, hipStream_t s) {
  if (waves == 4) hipLaunchKernelGGL((cache8_store_kernel<T, Code, 4, 8, ONCE>), grid, dim3(256), 0, s, a);
  else if (passes == 4) hipLaunchKernelGGL((cache8_store_kernel<T, Code, 1, 4, ONCE>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((cache8_store_kernel<T, Code, 1, 8, ONCE>), grid, dim3(256), 0, s, a);
}

// ---- read

// A wavefront has a.groups rows (tokens).  Where each one's codes lie is found a row a lane; then the wavefront goes over the columns, 8 codes to a lane, which
// are the same in all of its rows, K columns of U rows requested together.  WIDE: a token has 64 times 8 codes and more; else several rows lie side by side.
// 5.5 TB/s for 118997 tokens of 8 heads of 128, K and V (134 us, in some runs 129; with one column of 4 rows at a time 142, of 8 rows 146, a workgroup's rows found by one wavefront in
// LDS 140, its items one behind the other, each with divisions of its own, 182; stores through the caches 156 instead of 141).
template <typename T, class Code, bool WIDE> __global__ __launch_bounds__(256) void cache8_read_kernel(const Cache8Args a) {
  constexpr int U = 2, K = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int halves = 2 * a.pieces, each = 2 * a.heads * halves;      // 8 codes: of a head, of a row
  const int step = WIDE ? 1 : 64 / each, r0 = WIDE ? 0 : lane / each, col0 = lane - r0 * each;      // rows that are done together, the lane's among them
  for (int t0 = (blockIdx.x * 4 + wave) * a.groups; t0 < a.tokens; t0 += gridDim.x * 4 * a.groups) {
    const int rows = min(a.groups, a.tokens - t0);
    // ---- every row's request: mostly the first one's, else found from there on
    const int t = t0 + lane;
    const Cache8Request q = find_last(a, [&](int first, int) { return first <= t0; });
    int b = q.b, first = q.first, fresh = q.fresh, keys = q.keys;
    if (lane < rows && (b < 0 || t >= first + fresh)) {
      int lo = b, hi = a.requests - 1;      // the last request that begins at or before t: steps of 1, 2, 4 .. until one begins behind it, then bisection
      for (int step = 1; lo + step <= hi; step *= 2) {
        if (cache8_start(a, lo + step) > t) { hi = lo + step - 1; break; }
        lo += step;
      }
      while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (cache8_start(a, mid) <= t) lo = mid; else hi = mid - 1;
      }
      b = lo;
      if (b >= 0) { first = cache8_start(a, b); fresh = max(0, cache8_start(a, b + 1) - first); keys = cache8_keys(a, b); }
    }
    int64_t place = -2;      // of the row's codes; -1: it is written as zeros, -2: it is nobody's
    int page = 0;
    if (lane < rows && b >= 0 && t >= first && t < first + fresh) {
      place = -1;
      const int p = keys - fresh + t - first;
      if (p >= 0) {
        page = a.tables[(int64_t)b * a.width + (p >> a.cache.shift)];
        if ((unsigned)page < (unsigned)a.cache.blocks) place = (int64_t)page * a.cache.block + (int64_t)(p & ((1 << a.cache.shift) - 1)) * a.cache.slot;
      }
    }
    auto of_row = [&](int v, int r) __attribute__((always_inline)) { return WIDE ? __builtin_amdgcn_readlane(v, r) : __shfl(v, min(r, 63)); };
    // ---- the columns, K of a lane at a time
    const int ahead = WIDE ? 64 : each;
    for (int c0 = col0; c0 < each && r0 < step; c0 += K * ahead) {
      u32x2 c[K][U];
      float s[K][U];
      T* to[K];
      int64_t at[U];
      int in[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = r0 + u * step;
        at[u] = (int64_t)((uint64_t)(uint32_t)of_row((int)((uint64_t)place >> 32), r) << 32 | (uint32_t)of_row((int)place, r));
        in[u] = of_row(page, r);
        if (r >= rows) at[u] = -2;
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int col = c0 + k * ahead, h = col / halves, p = col - h * halves;
        const bool values = h >= a.heads;
        const int head = values ? h - a.heads : h;
        to[k] = nullptr;
        if (k == 0 || col < each) {
          const uint8_t* codes = static_cast<const uint8_t*>(values ? a.v_codes : a.k_codes) + (int64_t)head * a.cache.head + 8 * p;
          const float* scales = (values ? a.v_scales : a.k_scales) + head;
          to[k] = static_cast<T*>(const_cast<void*>(values ? a.v : a.k)) + (t0 + r0) * (values ? a.v_stride : a.k_stride) + (int64_t)head * a.pieces * 16 + 8 * p;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            c[k][u] = u32x2{0u, 0u};
            s[k][u] = 0.f;
            if (at[u] >= 0) {
              c[k][u] = *reinterpret_cast<const u32x2*>(codes + at[u]);
              s[k][u] = scales[(int64_t)in[u] * a.heads];
            }
          }
        }
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (k && !to[k]) continue;
        const int64_t stride = (c0 + k * ahead >= each / 2 ? a.v_stride : a.k_stride) * step;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (at[u] == -2) continue;
          T* out = to[k] + u * stride;
          float x[8], y[4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            Code::unpack(c[k][u][i], y);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = y[j] * s[k][u];
          }
          if constexpr (sizeof(T) == 4) {
            stream_store16(out, __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]}));
            stream_store16(out + 4, __builtin_bit_cast(u32x4, f32x4{x[4], x[5], x[6], x[7]}));
          } else {
            stream_store16(out, pack16<T>(x));
          }
        }
      }
    }
  }
}

template <typename T, class Code> void read_launch(const Cache8Args& a, bool wide, int grid, hipStream_t s) {
  if (wide) hipLaunchKernelGGL((cache8_read_kernel<T, Code, true>), dim3(grid), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((cache8_read_kernel<T, Code, false>), dim3(grid), dim3(256), 0, s, a);
}

// ---- geometry and launches

void cache8_geometry(Cache8Spec* s, bool store) {
  const fs_cache8_desc& d = s->d;
  if (store) {
    // as many wavefronts and registers as a block's new tokens take, where the call's are shared evenly by its requests: eight pieces of a thread, or four (single
    // tokens of 71 requests, 16 heads of 64, into blocks of 128: 4.4 us, 11.8 with what whole blocks take)
    const int rows = 64 / (d.head_dim / 8);      // of a wavefront at a time
    const int64_t most = std::min<int64_t>(d.block_size, d.requests ? (d.tokens + d.requests - 1) / d.requests : 0);
    s->waves = most > 8 * rows ? 4 : 1;
    s->passes = most > 4 * rows ? 8 : 4;
    s->once = 2ll * d.tokens * d.kv_heads * d.head_dim * (d.dtype == FS_F32 ? 4 : 2) > (64ll << 20);
    s->places = (int)(((int64_t)d.tokens >> s->cache.shift) + 2ll * d.requests);
    s->groups = (2 * d.kv_heads * s->waves + 3) / 4;
    s->grid_groups = std::min(s->groups, 1 << 10);
    // (eight times as many rows of a grid have less than 2^32 threads)
    s->grid = (int)std::min<int64_t>(((int64_t)s->places + 7) / 8, std::min(65535, (1 << 20) / s->grid_groups));
    return;
  }
  // two rows (or runs of rows side by side) to a wavefront where there are enough of them: each has four columns of both in flight
  const int64_t each = 4ll * d.kv_heads * (d.head_dim / 16);
  const int64_t side_by_side = each < 64 ? 64 / each : 1;
  s->groups = (int)(side_by_side * (d.tokens >= 4096 * side_by_side ? 2 : 1));
  s->wide = each >= 64;
  s->grid = (int)std::min<int64_t>(((int64_t)d.tokens + 4 * s->groups - 1) / (4 * s->groups), 1 << 23);
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
  a.groups = s.groups; a.places = s.places;
  a.piece_inv = (65536 + 2 * a.pieces - 1) / (2 * a.pieces);      // (right below 2^10: 256 threads, at most 64 pieces)
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool e4m3 = d.code == FS_CODE_E4M3;
  if (store) {
    const dim3 grid(8 * s.grid_groups, s.grid);
    auto go = [&](auto type) {
      typedef decltype(type) T;
      if (s.once) e4m3 ? store_launch<T, E4m3, true>(a, s.passes, s.waves, grid, st) : store_launch<T, Int8, true>(a, s.passes, s.waves, grid, st);
      else e4m3 ? store_launch<T, E4m3, false>(a, s.passes, s.waves, grid, st) : store_launch<T, Int8, false>(a, s.passes, s.waves, grid, st);
    };
    if (d.dtype == FS_F32) go(float{}); else if (d.dtype == FS_F16) go(f16_t{}); else go(bf16_t{});
  } else {
    auto go = [&](auto type) {
      typedef decltype(type) T;
      if (e4m3) read_launch<T, E4m3>(a, s.wide, s.grid, st); else read_launch<T, Int8>(a, s.wide, s.grid, st);
    };
    if (d.dtype == FS_F32) go(float{}); else if (d.dtype == FS_F16) go(f16_t{}); else go(bf16_t{});
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { *err = std::string(store ? "cache_store8" : "cache_read8") + " launch: " + hipGetErrorString(e); return -1; }
  return 0;
}

}  // namespace fs
