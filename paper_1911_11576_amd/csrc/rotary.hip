// Rotary positions (fs_plan_create_rotary), with and without the store into a paged cache.
//
// A head of D elements is D / (2 W) threads' work, W the elements of a vector: a thread has one vector of each half of the turned
// part (half layout), or two vectors of whole pairs (interleaved), and its angles are the same in every head of a token, so they
// are made once for several heads.  The angle position * frequency is formed in turns in 64 bits and
// reduced there to an eighth of a turn around a multiple of a quarter: positions of a million lose nothing.  Sine and cosine of
// the rest are the Taylor polynomials of degree 9 and 10 (remainders 2e-9 and 1e-10 at pi/4).
// Bound by HBM: every element is read and written once; no element goes through LDS.  5.6 to 6.2 TB/s for 130 to 340 MB, of the 6.6 of a copy.
#include <algorithm>

#include "dev_common.h"
#include "paged.h"

namespace fs {
namespace {

// n / d of numbers below 2^31 as a product: m = ceil(2^(31 + s) / d), s = ceil(log2 d), is off by less than d / 2^(31 + s) * n < 1 / d.
struct Divisor { uint32_t d = 1, m = 1, shift = 0; };
Divisor divisor(uint32_t d) {
  uint32_t s = 0;
  while ((1ull << s) < d) ++s;
  return Divisor{d, (uint32_t)(((1ull << (31 + s)) + d - 1) / d), 31 + s};
}
__device__ __forceinline__ uint32_t quotient(uint32_t n, const Divisor& d) { return (uint32_t)((uint64_t)n * d.m >> d.shift); }

struct RotaryArgs {
  const void *q, *k, *v;
  const int *positions, *slots;
  const double* frequencies;
  void *q_out, *k_out, *v_out;       // k_out and v_out: the caches where keys are stored
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
  CacheLayout cache;
  int64_t n_slots;
  int token0, tokens;                // of this launch: its first row, the rows behind it
  int q_heads, k_heads, heads, dim, rot, units, groups, inverse;      // groups: threads to a row and unit
  Divisor by_lanes, by_units, by_pairs;
  int most_angles;                   // of a workgroup's rows
  float magnitude;
  bool once;                         // of the launch: stores past the caches
};

// W elements at element alignment times W: one access of up to 16 bytes.
template <typename T, int W> struct Pack;
template <int BYTES> struct Raw;
template <> struct Raw<16> { typedef u32x4 type; };
template <> struct Raw<8> { typedef u32x2 type; };
template <> struct Raw<4> { typedef uint32_t type; };
template <> struct Raw<2> { typedef uint16_t type; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16_t v) { return bf16_to_f32(v.bits); }
__device__ __forceinline__ float to_float(f16_t v) { return f16_to_f32(v.bits); }
__device__ __forceinline__ void from_float(float f, float* v) { *v = f; }
__device__ __forceinline__ void from_float(float f, bf16_t* v) { v->bits = (uint16_t)f32_to_bf16(f); }
__device__ __forceinline__ void from_float(float f, f16_t* v) { v->bits = (uint16_t)f32_to_f16(f); }

template <typename T, int W> struct alignas(sizeof(T) * W) Pack {
  T v[W];
  typedef typename Raw<sizeof(T) * W>::type raw;
};
template <typename T, int W> __device__ __forceinline__ Pack<T, W> load_pack(const T* p) {
  return __builtin_bit_cast(Pack<T, W>, __builtin_nontemporal_load(reinterpret_cast<const typename Pack<T, W>::raw*>(p)));
}
template <bool ONCE, typename T, int W> __device__ __forceinline__ void store_pack(T* p, const Pack<T, W>& v) {
  typedef typename Pack<T, W>::raw raw;
  if constexpr (ONCE) __builtin_nontemporal_store(__builtin_bit_cast(raw, v), reinterpret_cast<raw*>(p));
  else *reinterpret_cast<raw*>(p) = __builtin_bit_cast(raw, v);
}

// cos and sin of `turns` whole turns
__device__ __forceinline__ void turned(double turns, float* c, float* s) {
  const double part = __builtin_amdgcn_fract(turns), quarters = __builtin_rint(4.0 * part);
  const float x = (float)(part - 0.25 * quarters) * 6.28318530717958647693f;
  const float y = x * x;
  const float sn = x * (1.f + y * (-1.f / 6 + y * (1.f / 120 + y * (-1.f / 5040 + y * (1.f / 362880)))));
  const float cs = 1.f + y * (-0.5f + y * (1.f / 24 + y * (-1.f / 720 + y * (1.f / 40320 + y * (-1.f / 3628800)))));
  const int n = (int)quarters & 3;
  const float a = n & 1 ? sn : cs, b = n & 1 ? cs : sn;
  *c = n == 1 || n == 2 ? -a : a;
  *s = n & 2 ? -b : b;
}

// kHalves, kInterleaved: two vectors of a head to a thread, as above.  kOneVector: halves, but a thread has one vector, whose results it stores, and reads
// the one that is turned with it too: neighbours' vectors are neighbours.  A head's threads are in one wavefront, which has read all of a head
// before it stores any of it (in place the buffers are the same).
enum { kHalves, kInterleaved, kOneVector };
constexpr double kTurn = 0.15915494309189533577;      // 1 / 2 pi

// H: heads of a thread, all of them requested before the angles are made.  With several of 8 elements a vector a workgroup makes the cosines and
// sines of its rows together, in LDS: every one once and not once a thread, which took more instructions than everything else.  ONCE: stores past the caches.
template <typename T, int W, int H, int LAYOUT, bool STORE, bool ONCE> __global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a) {
  const uint32_t n = blockIdx.x * 256u + threadIdx.x, row_in = quotient(n, a.by_lanes), r = n - row_in * a.by_lanes.d;
  constexpr bool INTER = LAYOUT == kInterleaved, ONE = LAYOUT == kOneVector, TOGETHER = H > 1 && W == 8;
  bool there = row_in < (uint32_t)a.tokens;
  if (!TOGETHER && !there) return;
  const int64_t token = (int64_t)a.token0 + (there ? row_in : 0);
  const int h0 = (int)quotient(r, a.by_units), u = (int)r - h0 * a.units;
  // the workgroup's first row, and the thread's first angle
  extern __shared__ float angles[];      // [row][pair]: cosines, then sines
  const int pairs = a.rot / 2;
  uint32_t row0 = 0, n_angles = 0;
  double turn0 = 0;
  auto turns = [&](uint32_t i) __attribute__((always_inline)) {
    const uint32_t k = quotient(i, a.by_pairs);
    return (double)a.positions[min((int64_t)a.token0 + row0 + k, (int64_t)a.token0 + a.tokens - 1)] * a.frequencies[i - k * pairs] * kTurn;
  };
  if constexpr (TOGETHER) {
    row0 = quotient(blockIdx.x * 256u, a.by_lanes);
    n_angles = (quotient(blockIdx.x * 256u + 255u, a.by_lanes) - row0 + 1) * pairs;
    turn0 = turns(min(threadIdx.x, n_angles - 1));
  }
  int64_t row = 0;
  if (STORE) {
    const int slot = a.slots[token];
    if (slot < 0 || slot >= a.n_slots) {
      if (!TOGETHER) return;
      there = false;
    }
    if (there) row = (int64_t)(slot >> a.cache.shift) * a.cache.block + (int64_t)(slot & ((1 << a.cache.shift) - 1)) * a.cache.slot;
  }
  // the thread's two vectors of a head, and whether they are turned
  int e0, e1;
  bool t0, t1, two = true;
  if constexpr (INTER) {
    e0 = u * W; e1 = (u + a.units) * W;
    t0 = e0 < a.rot; t1 = e1 < a.rot;
    two = e1 < a.dim;      // a head of an odd number of vectors: its last thread has one
  } else if constexpr (ONE) {
    e0 = u * W;
    t0 = t1 = e0 < a.rot;
    e1 = !t0 ? e0 : e0 < a.rot / 2 ? e0 + a.rot / 2 : e0 - a.rot / 2;
  } else {
    const int turned_units = a.rot / (2 * W);
    t0 = t1 = u < turned_units;
    e0 = t0 ? u * W : a.rot + (u - turned_units) * 2 * W;
    e1 = t0 ? a.rot / 2 + u * W : e0 + W;
  }
  Pack<T, W> p[H][2];
  T* to[H];
#pragma unroll
  for (int j = 0; j < H; ++j) {
    const int h = min(h0 + j * a.groups, a.heads - 1);
    const bool is_q = h < a.q_heads, is_v = STORE && h >= a.q_heads + a.k_heads;
    const int kh = h - a.q_heads - (is_v ? a.k_heads : 0);
    const T* x = static_cast<const T*>(is_q ? a.q : is_v ? a.v : a.k) + token * (is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride) + (int64_t)(is_q ? h : kh) * a.dim;
    p[j][0] = load_pack<T, W>(x + e0);
    p[j][1] = load_pack<T, W>(x + (two ? e1 : e0));
    if (is_q) to[j] = static_cast<T*>(a.q_out) + token * a.q_out_stride + (int64_t)h * a.dim;
    else if (STORE) to[j] = static_cast<T*>(is_v ? a.v_out : a.k_out) + row + (int64_t)kh * a.cache.head;
    else to[j] = static_cast<T*>(a.k_out) + token * a.k_out_stride + (int64_t)kh * a.dim;
  }
  float c[W], s[W];
  auto scaled = [&](double t, float* c, float* s) __attribute__((always_inline)) {
    turned(t, c, s);
    *c *= a.magnitude;
    *s *= a.inverse ? -a.magnitude : a.magnitude;
  };
  if constexpr (TOGETHER) {
    float* sines = angles + a.most_angles;
    for (uint32_t i = threadIdx.x; i < n_angles; i += 256) {
      float x, y;
      scaled(i == threadIdx.x ? turn0 : turns(i), &x, &y);
      angles[i] = x;
      sines[i] = y;
    }
    __syncthreads();
    if (!there) return;
  }
#pragma unroll
  for (int i = 0; i < W; ++i) {
    c[i] = 1.f; s[i] = 0.f;
    // interleaved: pairs of the first vector, then of the second
    const int pair = !INTER ? min(e0, e1) + i : i < W / 2 ? e0 / 2 + i : e1 / 2 + i - W / 2;
    if (!INTER ? t0 : i < W / 2 ? t0 : t1) {
      if constexpr (TOGETHER) {
        const uint32_t k = (row_in - row0) * pairs + pair;
        c[i] = angles[k];
        s[i] = angles[a.most_angles + k];
      } else {
        scaled((double)a.positions[token] * a.frequencies[pair] * kTurn, &c[i], &s[i]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < H; ++j) {
    const int h = h0 + j * a.groups;
    if (h >= a.heads) break;
    Pack<T, W> p0 = p[j][0], p1 = p[j][1];
    if (!STORE || h < a.q_heads + a.k_heads) {
      if constexpr (INTER) {
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
          const float x0 = to_float(p0.v[2 * i]), x1 = to_float(p0.v[2 * i + 1]), z0 = to_float(p1.v[2 * i]), z1 = to_float(p1.v[2 * i + 1]);
          if (t0) {
            from_float(x0 * c[i] - x1 * s[i], &p0.v[2 * i]);
            from_float(x1 * c[i] + x0 * s[i], &p0.v[2 * i + 1]);
          }
          if (t1) {
            from_float(z0 * c[i + W / 2] - z1 * s[i + W / 2], &p1.v[2 * i]);
            from_float(z1 * c[i + W / 2] + z0 * s[i + W / 2], &p1.v[2 * i + 1]);
          }
        }
      } else if (t0) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float x0 = to_float(p0.v[i]), x1 = to_float(p1.v[i]);
          from_float(ONE && e0 > e1 ? x0 * c[i] + x1 * s[i] : x0 * c[i] - x1 * s[i], &p0.v[i]);
          if constexpr (!ONE) from_float(x1 * c[i] + x0 * s[i], &p1.v[i]);
        }
      }
    }
    store_pack<ONCE>(to[j] + e0, p0);
    if (!ONE && two) store_pack<ONCE>(to[j] + e1, p1);
  }
}

template <typename T, int W, int H, int LAYOUT> void launch_heads(const RotaryArgs& a, const RotarySpec& s, unsigned wgs, hipStream_t stream) {
  const size_t lds = H > 1 && W == 8 ? 8 * (size_t)s.most_angles : 0;
  if (s.d.blocks > 0) hipLaunchKernelGGL((rotary_kernel<T, W, H, LAYOUT, true, false>), dim3(wgs), dim3(256), lds, stream, a);
  else if (a.once) hipLaunchKernelGGL((rotary_kernel<T, W, H, LAYOUT, false, true>), dim3(wgs), dim3(256), lds, stream, a);
  else hipLaunchKernelGGL((rotary_kernel<T, W, H, LAYOUT, false, false>), dim3(wgs), dim3(256), lds, stream, a);
}
template <typename T, int W, int LAYOUT> void launch_layout(const RotaryArgs& a, const RotarySpec& s, unsigned wgs, hipStream_t stream) {
  if constexpr (W == 8 && LAYOUT == kHalves)
    if (s.one) return launch_heads<T, W, 4, kOneVector>(a, s, wgs, stream);
  if (s.heads_each == 1) launch_heads<T, W, 1, LAYOUT>(a, s, wgs, stream);
  else if constexpr (W == 8) launch_heads<T, W, 2, LAYOUT>(a, s, wgs, stream);
  else if (s.heads_each == 4) launch_heads<T, W, 4, LAYOUT>(a, s, wgs, stream);
  else if constexpr (W * sizeof(T) != 8) launch_heads<T, W, 8, LAYOUT>(a, s, wgs, stream);
}

template <typename T, int W> hipError_t launch_width(RotaryArgs a, const RotarySpec& s, hipStream_t stream) {
  // threads are numbered in 31 bits: beyond that, several launches
  const int64_t lanes = (int64_t)s.units * s.groups, most = (0x7fffff00ll / lanes);
  for (int64_t t = 0; t < s.d.tokens; t += most) {
    a.token0 = (int)t;
    a.tokens = (int)std::min(most, s.d.tokens - t);
    const unsigned wgs = (unsigned)((a.tokens * lanes + 255) / 256);
    if (!s.d.interleaved) launch_layout<T, W, kHalves>(a, s, wgs, stream);
    else if constexpr (W >= 2) launch_layout<T, W, kInterleaved>(a, s, wgs, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T> hipError_t launch_type(const RotaryArgs& a, const RotarySpec& s, hipStream_t stream) {
  switch (s.width) {
    case 1: return launch_width<T, 1>(a, s, stream);
    case 2: return launch_width<T, 2>(a, s, stream);
    case 4: return launch_width<T, 4>(a, s, stream);
    default:
      if constexpr (sizeof(T) == 2) return launch_width<T, 8>(a, s, stream);
      else return hipErrorInvalidValue;
  }
}

}  // namespace

// Several heads to a thread are requested together and share its angles, where that leaves the chip two wavefronts a SIMD (32 rows of 48
// heads 4.0 us, with several 4.9).  16-bit vectors: two of them, angles made by the workgroup: 16384 rows of 40 heads of 128 in bf16 55.4 us (6.05 TB/s;
// 59.6 with four and angles of the thread's own, 79 with one; 55.7 with four), 24 + 24 + 24 heads of 64 into a cache 30.5.  fp32, whose vectors have half the angles:
// eight, angles of its own: 8192 rows of 32 heads of 64 21.6 us (22.2 with the workgroup's; 24.3 with four, 25.8 with one).  Where there are fewer than 16
// heads four, fewer than four one: a thread reads as many whatever there are (fp32, heads of 80 with 24 turned: 16384 rows of 8 heads 18.7 us, with eight 21.3;
// 65536 of two 21.3, with four 23.5, with eight 34.6).  Vectors of 8 bytes: four (bf16, 8192 rows of 40 heads of 128, strides of 4 more 32.1 us, with eight 34 to 37.6, with
// two 38.9, with one 43.8; of 80, 40 turned 25.9, 27.1, 27.1, 31.8: 4.05 TB/s); of 4 and 2 bytes eight as well (strides of 2 more 31.3, with four 32.6, with one 51.5).
// Interleaved, in vectors of 16 bytes: the gradient's sizes 56.0 us.
// Where a half of a head is no whole line of 128 bytes, or a part of it is not turned, a thread has one vector of a head: 8191 rows of those 72 heads of
// 64 in fp16, half of each turned, into a cache 26.9 us (5.6 TB/s), with two vectors 30.5; all of each turned 27.9 and 30.6.  Where halves are lines two are
// better: 55.4 and 57.8 for the first of these.  Stores go past the caches where two vectors fill whole lines each and are not for a cache, which attention reads next: 66.8 ->
// 60.0 us for the first (before the rest); with one vector 12286 rows of 48 heads of 64 25.8 -> 27.3, where lines are not filled 33 -> 41.  So not where the
// outputs' rows or buffers begin inside lines: the first with rows 16 bytes longer 67.0 us through the caches and 80.3 past them, its buffers 16 bytes behind a
// line 64.8 and 88.4, 64 bytes 61.0 and 63.2; the fp32 case 22.6 and 39.8, 22.7 and 38.2, 22.5 and 27.9.  Rows 64 bytes longer, of which every
// other one begins at a line: 68.4 and 58.7, in fp32 22.7 and 25.1.  Vectors of less than 16 bytes: 77.0 and 76.8, in fp32 26.5 and 27.2.
void rotary_geometry(RotarySpec* s) {
  const fs_rotary_desc& d = s->d;
  const int64_t threads = (int64_t)d.tokens * s->units * s->heads, bytes = (d.dtype == FS_F32 ? 4 : 2) * (int64_t)d.head_dim;
  const bool lines = bytes % 256 == 0 && (d.interleaved || d.rotary_dim == d.head_dim);
  s->heads_each = threads < 4 * 131072 ? 1 : s->width == 8 ? 2 : s->heads < 4 ? 1 : s->heads < 16 || s->width * (d.dtype == FS_F32 ? 4 : 2) == 8 ? 4 : 8;
  const int pieces = d.head_dim / 8;
  s->one = s->heads_each == 2 && !d.interleaved && !lines && (pieces & (pieces - 1)) == 0;
  if (s->one) {
    s->units = pieces;
    s->heads_each = 4;
  }
  const int64_t whole = 32;      // 128 bytes of fp32, 64 of the others
  s->once = lines && d.blocks == 0 && s->width == (d.dtype == FS_F32 ? 4 : 8) && d.q_out_stride % whole == 0 && (d.k_heads == 0 || d.k_out_stride % whole == 0);
  s->groups = (s->heads + s->heads_each - 1) / s->heads_each;
  s->most_angles = (254 / (s->units * s->groups) + 2) * (d.rotary_dim / 2);      // 256 threads are of no more rows
}

int rotary_launch(const RotarySpec& s, const void* const* in, void* const* out, void* stream, std::string* err) {
  if (s.d.tokens == 0) return 0;
  const bool store = s.d.blocks > 0;
  RotaryArgs a{};
  int i = 0;
  a.q = in[i++];
  if (s.d.k_heads) a.k = in[i++];
  if (store) a.v = in[i++];
  a.positions = static_cast<const int*>(in[i++]);
  a.frequencies = static_cast<const double*>(in[i++]);
  if (store) a.slots = static_cast<const int*>(in[i++]);
  a.q_out = out[0];
  if (s.d.k_heads) a.k_out = out[1];
  if (store) a.v_out = out[2];
  a.q_stride = s.d.q_stride; a.k_stride = s.d.k_stride; a.v_stride = s.d.v_stride; a.q_out_stride = s.d.q_out_stride; a.k_out_stride = s.d.k_out_stride;
  a.cache = s.cache;
  a.n_slots = (int64_t)s.d.blocks << s.cache.shift;
  a.q_heads = s.d.q_heads; a.k_heads = s.d.k_heads; a.heads = s.heads; a.dim = s.d.head_dim; a.rot = s.d.rotary_dim;
  a.units = s.units; a.groups = s.groups; a.by_units = divisor(s.units); a.by_lanes = divisor(s.units * s.groups); a.by_pairs = divisor(s.d.rotary_dim / 2);
  a.most_angles = s.most_angles; a.inverse = s.d.inverse;
  a.magnitude = (float)s.d.magnitude;
  a.once = s.once && ((reinterpret_cast<uintptr_t>(a.q_out) | reinterpret_cast<uintptr_t>(a.k_out)) & 127) == 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = s.d.dtype == FS_F32 ? launch_type<float>(a, s, st) : s.d.dtype == FS_F16 ? launch_type<f16_t>(a, s, st) : launch_type<bf16_t>(a, s, st);
  if (e != hipSuccess) { *err = std::string("rotary launch: ") + hipGetErrorString(e); return -1; }
  return 0;
}

}  // namespace fs
