// Rotary positions (fs_plan_create_rotary), with and without the store into a paged cache.
//
// A head of D elements is D / (2 W) threads' work, W the elements of a vector: a thread has one vector of each half of the turned
// part (half layout), or two vectors of whole pairs (interleaved), and its angles are the same in every head of a token, so it
// makes W cosines and sines once and then walks heads.  The angle position * frequency is formed in turns in 64 bits and
// reduced there to an eighth of a turn around a multiple of a quarter: positions of a million lose nothing.  Sine and cosine of
// the rest are the Taylor polynomials of degree 9 and 10 (remainders 2e-9 and 1e-10 at pi/4).
// Bound by HBM: every element is read and written once; nothing goes through LDS.
#include <algorithm>

#include "dev_common.h"
#include "paged.h"

namespace fs {
namespace {

struct RotaryArgs {
  const void *q, *k, *v;
  const int *positions, *slots;
  const double* frequencies;
  void *q_out, *k_out, *v_out;       // k_out and v_out: the caches where keys are stored
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
  CacheLayout cache;
  int64_t n_slots;
  int tokens, q_heads, k_heads, heads, dim, rot, units, heads_at_once, tokens_per_wg, inverse;
  float magnitude;
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
  return __builtin_bit_cast(Pack<T, W>, *reinterpret_cast<const typename Pack<T, W>::raw*>(p));
}
template <typename T, int W> __device__ __forceinline__ void store_pack(T* p, const Pack<T, W>& v) {
  *reinterpret_cast<typename Pack<T, W>::raw*>(p) = __builtin_bit_cast(typename Pack<T, W>::raw, v);
}

// cos and sin of `turns` whole turns
__device__ __forceinline__ void turned(double turns, float* c, float* s) {
  const double quarters = __builtin_rint(4.0 * turns);
  const float x = (float)(turns - 0.25 * quarters) * 6.28318530717958647693f;
  const float y = x * x;
  const float sn = x * (1.f + y * (-1.f / 6 + y * (1.f / 120 + y * (-1.f / 5040 + y * (1.f / 362880)))));
  const float cs = 1.f + y * (-0.5f + y * (1.f / 24 + y * (-1.f / 720 + y * (1.f / 40320 + y * (-1.f / 3628800)))));
  const int n = (int)(long long)quarters & 3;
  const float a = n & 1 ? sn : cs, b = n & 1 ? cs : sn;
  *c = n == 1 || n == 2 ? -a : a;
  *s = n & 2 ? -b : b;
}

template <typename T, int W, bool INTER, bool STORE> __global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a) {
  const int lanes = a.units * a.heads_at_once;
  const int in_wg = (int)threadIdx.x / lanes, r = (int)threadIdx.x - in_wg * lanes;
  const int64_t token = (int64_t)blockIdx.x * a.tokens_per_wg + in_wg;
  if (in_wg >= a.tokens_per_wg || token >= a.tokens) return;
  const int h0 = r / a.units, u = r - h0 * a.units;
  int64_t row = 0;
  if (STORE) {
    const int slot = a.slots[token];
    if (slot < 0 || slot >= a.n_slots) return;
    row = (int64_t)(slot >> a.cache.shift) * a.cache.block + (int64_t)(slot & ((1 << a.cache.shift) - 1)) * a.cache.slot;
  }
  // the thread's two vectors of a head, and whether they are turned
  int e0, e1;
  bool t0, t1, two = true;
  if constexpr (INTER) {
    e0 = u * W; e1 = (u + a.units) * W;
    t0 = e0 < a.rot; t1 = e1 < a.rot;
    two = e1 < a.dim;      // a head of an odd number of vectors: its last thread has one
  } else {
    const int turned_units = a.rot / (2 * W);
    t0 = t1 = u < turned_units;
    e0 = t0 ? u * W : a.rot + (u - turned_units) * 2 * W;
    e1 = t0 ? a.rot / 2 + u * W : e0 + W;
  }
  const double position = (double)a.positions[token];
  constexpr double kTurn = 0.15915494309189533577;      // 1 / 2 pi
  float c[W], s[W];
#pragma unroll
  for (int i = 0; i < W; ++i) {
    c[i] = 1.f; s[i] = 0.f;
    // interleaved: pairs of the first vector, then of the second
    const int pair = !INTER ? u * W + i : i < W / 2 ? e0 / 2 + i : e1 / 2 + i - W / 2;
    if (!INTER ? t0 : i < W / 2 ? t0 : t1) {
      turned(position * a.frequencies[pair] * kTurn, &c[i], &s[i]);
      c[i] *= a.magnitude;
      s[i] *= a.inverse ? -a.magnitude : a.magnitude;
    }
  }
  for (int h = h0; h < a.heads; h += a.heads_at_once) {
    const T* x;
    T* y;
    const bool is_q = h < a.q_heads, is_v = STORE && h >= a.q_heads + a.k_heads;
    const int kh = h - a.q_heads - (is_v ? a.k_heads : 0);
    if (is_q) {
      x = static_cast<const T*>(a.q) + token * a.q_stride + (int64_t)h * a.dim;
      y = static_cast<T*>(a.q_out) + token * a.q_out_stride + (int64_t)h * a.dim;
    } else {
      x = static_cast<const T*>(is_v ? a.v : a.k) + token * (is_v ? a.v_stride : a.k_stride) + (int64_t)kh * a.dim;
      if (STORE) y = static_cast<T*>(is_v ? a.v_out : a.k_out) + row + (int64_t)kh * a.cache.head;
      else y = static_cast<T*>(a.k_out) + token * a.k_out_stride + (int64_t)kh * a.dim;
    }
    Pack<T, W> p0 = load_pack<T, W>(x + e0), p1 = load_pack<T, W>(x + (two ? e1 : e0));
    if (!is_v) {
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
          from_float(x0 * c[i] - x1 * s[i], &p0.v[i]);
          from_float(x1 * c[i] + x0 * s[i], &p1.v[i]);
        }
      }
    }
    store_pack<T, W>(y + e0, p0);
    if (two) store_pack<T, W>(y + e1, p1);
  }
}

template <typename T, int W> hipError_t launch_width(const RotaryArgs& a, const RotarySpec& s, hipStream_t stream) {
  const dim3 grid((unsigned)s.grid), wg(s.wg);
  const bool store = s.d.blocks > 0;
  if constexpr (W >= 2) {
    if (s.d.interleaved) {
      if (store) hipLaunchKernelGGL((rotary_kernel<T, W, true, true>), grid, wg, 0, stream, a);
      else hipLaunchKernelGGL((rotary_kernel<T, W, true, false>), grid, wg, 0, stream, a);
      return hipGetLastError();
    }
  }
  if (store) hipLaunchKernelGGL((rotary_kernel<T, W, false, true>), grid, wg, 0, stream, a);
  else hipLaunchKernelGGL((rotary_kernel<T, W, false, false>), grid, wg, 0, stream, a);
  return hipGetLastError();
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

void rotary_geometry(RotarySpec* s) {
  // as many heads of a token at a time as a workgroup of 256 holds, all of them if it can
  s->heads_at_once = std::max(1, std::min(s->heads, 256 / s->units));
  const int lanes = s->units * s->heads_at_once;
  s->tokens_per_wg = std::max(1, 256 / lanes);
  s->wg = (lanes * s->tokens_per_wg + 63) / 64 * 64;
  s->grid = s->d.tokens ? (s->d.tokens + s->tokens_per_wg - 1) / s->tokens_per_wg : 0;
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
  a.tokens = s.d.tokens; a.q_heads = s.d.q_heads; a.k_heads = s.d.k_heads; a.heads = s.heads; a.dim = s.d.head_dim; a.rot = s.d.rotary_dim;
  a.units = s.units; a.heads_at_once = s.heads_at_once; a.tokens_per_wg = s.tokens_per_wg; a.inverse = s.d.inverse;
  a.magnitude = (float)s.d.magnitude;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = s.d.dtype == FS_F32 ? launch_type<float>(a, s, st) : s.d.dtype == FS_F16 ? launch_type<f16_t>(a, s, st) : launch_type<bf16_t>(a, s, st);
  if (e != hipSuccess) { *err = std::string("rotary launch: ") + hipGetErrorString(e); return -1; }
  return 0;
}

}  // namespace fs
