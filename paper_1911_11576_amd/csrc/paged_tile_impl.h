// Attention over a paged cache, many rows a request (chunks of prompts): bound by the matrix unit and the exponentials.
//
// A workgroup has 128 rows of one request and key head, 32 to a wavefront, and walks the keys that they see 64 at a time: keys
// and values go through registers into LDS, the next 64 in flight and written to the other half while these are worked on, one
// barrier a step.  Both dots are v_mfma_f32_32x32x16.  Where there are few tiles their keys are split over workgroups too, and
// paged_tile_join_kernel adds the parts in the order of the keys.
#pragma once
#include "paged_attn_impl.h"

namespace fs {

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <typename T> __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c);
template <> __device__ __forceinline__ f32x16 mfma32<f16_t>(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 mfma32<bf16_t>(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// 16 bytes a lane from memory straight into LDS: piece I of 64 bytes of a lane's row to the wavefront's 1024 bytes at `lds` + 1024 I.
// (The instruction's offset counts on both sides.  As assembly, since the compiler makes every LDS read behind the builtin wait for
// all loads in flight, the next step's among them; there is no register that it writes.)
template <int I> __device__ __forceinline__ void load_lds16(const uint16_t* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off offset:%2" ::"s"(lds + 960 * I), "v"(from), "n"(64 * I) : "memory");
}
// ... all of them there, before a barrier that hands them on
__device__ __forceinline__ void wait_lds_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }

template <class Op> __device__ __forceinline__ float halves_allreduce(float v) {
  const uint32_t u = as_u32(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return Op::apply(as_f32(r[0]), as_f32(r[1]));
}

// Which rows a tile kernel's workgroup has: tile `slot` of the line in which request b's tiles begin at first_b * share / 128 + b (as
// many places as it can have tiles, whatever the lengths), and which of its keys' parts.
struct TileWork {
  int b, row0, rows, key_first, steps, parts, per;      // steps of 64 keys; parts that they are split into, steps of a part
  PagedRequest r;
};
__device__ __forceinline__ bool tile_work(const PagedArgs& a, int slot, TileWork* t) {
  const int lane = threadIdx.x & 63;
  auto begin = [&](int b) { return (int)(((int64_t)min(max(a.starts[b], 0), a.tokens) * a.share >> 7)) + b; };
  int n = 0;
  for (int b0 = 0; b0 < a.requests; b0 += 64) {
    const int here = __popcll(__ballot(b0 + lane < a.requests && begin(b0 + lane) <= slot));
    n += here;
    if (here < 64) break;
  }
  if (n == 0) return false;
  t->b = n - 1;
  t->r = paged_request(a, t->b);
  t->rows = t->r.fresh * a.share;
  t->row0 = (slot - begin(t->b)) * 128;
  if (t->rows <= a.few_rows || t->row0 >= t->rows) return false;
  const int t1 = (min(t->row0 + 128, t->rows) - 1) / a.share, t0 = t->row0 / a.share, back = t->r.keys - t->r.fresh + 1;
  const int until = max(0, a.causal ? min(t->r.keys, back + t1) : t->r.keys);
  t->key_first = a.window ? min(max(0, back + t0 - a.window), until) & ~63 : 0;
  t->steps = (until - t->key_first + 63) / 64;
  t->parts = min(a.most_parts, max(1, t->steps / a.least_steps));
  t->per = (t->steps + t->parts - 1) / t->parts;
  t->parts = t->per ? (t->steps + t->per - 1) / t->per : 1;
  return true;
}

// 64 keys (or values) in LDS as the direct loads leave them: 16 keys to a wavefront's part, pieces of 64 bytes of them behind one
// another, [key / 16][64-byte piece][key % 16][4 x 16 bytes].  The 16 bytes x of a piece of key r stand in place x ^ (r / 4 % 4): eight lanes that
// read a 16-byte column, and the four rows of a transposing read, fall on different banks.
template <int D> struct TileLds {
  static constexpr int kPieces = D / 32, kKeys16 = 16 * D;      // halves of 16 keys
  uint16_t v[64 * D];
};

template <typename T, int D> __global__ __launch_bounds__(256, 2) void paged_tile_kernel(const PagedArgs a) {
  constexpr int KS = D / 16, DT = D / 32, CH = D / 32, K16 = 16 * D;
  __shared__ __align__(1024) TileLds<D> ksh[2], vsh[2];
  __shared__ uint32_t flags[2][4], odds[4];                 // which of a wavefront's 16 keys are there; whether a value of them is infinite or NaN
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 31, h = lane >> 5;
  const int head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads;
  const int part = rest % a.most_parts, slot = a.slots - 1 - rest / a.most_parts;      // the last tiles of a request have the most keys: first
  TileWork work;
  if (!tile_work(a, slot, &work) || part >= work.parts) return;
  const PagedRequest r = work.r;
  const int step0 = part * work.per, steps = min(work.per, work.steps - step0);
  const int key_first = work.key_first + 64 * step0;
  const int* table = a.tables + (int64_t)work.b * a.width;
  const int in_block = (1 << a.cache.shift) - 1;

  // ---- the lane's row: its query as B operands, the keys it sees
  const int row = work.row0 + 32 * w + c, there = min(row, work.rows - 1), token = there / a.share;
  u32x4 qf[KS];
  {
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + (r.first + token) * a.q_stride + (int64_t)(head * a.share + there - token * a.share) * D + 8 * h;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const u32x4*>(q + 16 * ks);
    if (a.scale2 < 0) {      // scores are compared before they are scaled
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[ks] ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
    }
  }
  const float scale2 = fabsf(a.scale2);
  const int back = r.keys - r.fresh + 1;
  const int until = a.causal ? min(r.keys, back + token) : r.keys, from = a.window ? back + token - a.window : 0;
  // ... of the wavefront's rows, uniform: no key from `most` on, every key before `least` and from `latest` on; none before `first`
  int most, least, latest, first;
  {
    const int w0 = min(work.row0 + 32 * w, work.rows - 1) / a.share, w1 = min(work.row0 + 32 * w + 31, work.rows - 1) / a.share;
    most = a.causal ? min(r.keys, back + w1) : r.keys;
    least = a.causal ? min(r.keys, back + w0) : r.keys;
    latest = a.window ? back + w1 - a.window : 0;
    first = a.window ? back + w0 - a.window : 0;
    if (work.row0 + 32 * w >= work.rows) most = 0;      // a wavefront without rows
  }
  const int edge = a.causal ? back + work.row0 / a.share : r.keys;                                       // the tile's rows see all keys before ...
  const int edge2 = a.window ? back + (min(work.row0 + 128, work.rows) - 1) / a.share - a.window : 0;    // ... and from here on

  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  float m = -INFINITY, l = 0.f;

  // ---- staging: wavefront w brings keys 16w .. 16w + 15, four lanes to a key
  const int srow = lane >> 2, skey = 16 * w + srow;
  const int64_t head_at = (int64_t)head * a.cache.head + 8 * ((lane & 3) ^ (srow >> 2 & 3));
  const uint16_t *kbase = static_cast<const uint16_t*>(a.k) + head_at, *vbase = static_cast<const uint16_t*>(a.v) + head_at;
  const int key_last = min(r.keys, key_first + 64 * steps);
  int block;
  auto request_block = [&](int key0) __attribute__((always_inline)) { block = table[max(0, min(key0 + skey, r.keys - 1)) >> a.cache.shift]; };
  auto request_rows = [&](int key0, int buf) __attribute__((always_inline)) {
    const int key = key0 + skey;
    const bool ok = key < key_last && (unsigned)block < (unsigned)a.cache.blocks;
    const int64_t at = (int64_t)(ok ? block : 0) * a.cache.block + (int64_t)(key & in_block) * a.cache.slot;
    const uint32_t kl = lds_address(&ksh[buf].v[w * K16]), vl = lds_address(&vsh[buf].v[w * K16]);
    load_lds16<0>(kbase + at, kl);
    load_lds16<0>(vbase + at, vl);
    if constexpr (CH > 1) { load_lds16<1>(kbase + at, kl); load_lds16<1>(vbase + at, vl); }
    if constexpr (CH > 2) { load_lds16<2>(kbase + at, kl); load_lds16<2>(vbase + at, vl); }
    if constexpr (CH > 3) { load_lds16<3>(kbase + at, kl); load_lds16<3>(vbase + at, vl); }
    const uint64_t good = __ballot(ok);
    uint32_t flag = 0xffffu;
    if (good != ~0ull) {
      flag = 0;
      for (int k = 0; k < 16; ++k) flag |= (uint32_t)(good >> (4 * k) & 1) << k;
    }
    if (lane == 0) flags[buf][w] = flag;
  };

  auto compute = [&](int key0, int buf) __attribute__((always_inline)) {
    const uint32_t valid0 = __builtin_amdgcn_readfirstlane(flags[buf][0] | flags[buf][1] << 16), valid1 = __builtin_amdgcn_readfirstlane(flags[buf][2] | flags[buf][3] << 16);
    const bool there = (valid0 & valid1) == 0xffffffffu;
    const bool idle = key0 >= most || key0 + 64 <= first;      // none of the wavefront's rows sees any
    if (!there || key0 + 64 > edge || key0 < edge2) {
      // not every row sees every key: values of keys that are none do not count, whatever lies there; an infinity or NaN of another
      // is added as it is in the rows that see it, and the dot runs without it
      const bool ok = (flags[buf][w] >> srow & 1) != 0;
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        u32x4* v = reinterpret_cast<u32x4*>(&vsh[buf].v[w * K16 + 512 * i + 8 * lane]);
        if (!ok) *v = u32x4{0u, 0u, 0u, 0u};
        else any |= odd_values<T>(*v);
      }
      const bool mine = __ballot(any != 0) != 0;
      if (lane == 0) odds[w] = mine;
      __syncthreads();
      if (__builtin_amdgcn_readfirstlane(odds[0] | odds[1] | odds[2] | odds[3])) {
        for (int k = 0; k < 64; ++k) {
          const bool seen = ((k < 32 ? valid0 >> k : valid1 >> (k - 32)) & 1) && key0 + k < until && key0 + k >= from;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const u32x2 v = *reinterpret_cast<const u32x2*>(&vsh[buf].v[(k >> 4) * K16 + 512 * dt + (k & 15) * 32 + 8 * (j ^ (k >> 2 & 3)) + 4 * h]);
              const float x[4] = {Mfma<T>::lo(v[0]), Mfma<T>::hi(v[0]), Mfma<T>::lo(v[1]), Mfma<T>::hi(v[1])};
#pragma unroll
              for (int i = 0; i < 4; ++i) o[dt][4 * j + i] += seen && !(fabsf(x[i]) < INFINITY) ? x[i] : 0.f;
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          u32x4* v = reinterpret_cast<u32x4*>(&vsh[buf].v[w * K16 + 512 * i + 8 * lane]);
          *v = without_odd<T>(*v);
        }
        __syncthreads();
      }
    }
    if (idle) return;
    const bool plain = there && key0 + 64 <= least && key0 >= latest;
    // ---- S^T: 64 keys x 32 rows
    f32x16 s[2];
    const uint16_t* klane = &ksh[buf].v[(c >> 4) * K16 + (c & 15) * 32];
    const int kx = c >> 2 & 3;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const u32x4 kf = *reinterpret_cast<const u32x4*>(klane + 2 * t * K16 + 512 * (ks / 2) + 8 * ((2 * (ks & 1) + h) ^ kx));
        s[t] = ks == 0 ? mfma32<T>(kf, qf[0], f32x16{}) : mfma32<T>(kf, qf[ks], s[t]);
      }
    // ---- softmax: the lane holds keys 32t + 8(i/4) + 4h + i%4 of its row
    if (!plain) {
      // a bit for every key that the row sees, from the lane's first on
      auto below = [](int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1; };
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int key = key0 + 32 * t;
        const uint32_t see = ((t ? valid1 : valid0) & below(until - key) & ~below(from - key)) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = see & 1u << (8 * (i / 4) + i % 4) ? s[t][i] : -INFINITY;
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
    top = halves_allreduce<MaxOp>(top);
    // the sums are rescaled where a maximum has grown by more than 2^8: below that the exponentials are as exact
    if (__ballot(top > m && !((top - m) * scale2 <= 8.f))) {
      const float grown = fmaxf(m, top);
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - grown) * scale2);
      m = grown;
      l *= keep;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] *= keep;
    }
    const float low = m == -INFINITY ? 0.f : m * scale2;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[t][i], scale2, -low));
        s[t][i] = e;
        sum += e;
      }
    l += sum;
    u32x4 pb[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) pb[k][i] = Mfma<T>::pack(s[k / 2][8 * (k & 1) + 2 * i], s[k / 2][8 * (k & 1) + 2 * i + 1]);
    // ---- O^T += V^T . P^T
    // (keys 16k + 4h + 0 .. 3, and 8 behind them: places x ^ h and x ^ (h + 2))
    const int cc = lane & 15;
    const uint16_t* vlane = &vsh[buf].v[(4 * h + (cc >> 2)) * 32 + 4 * (cc & 1)];
    const int vx = 2 * (lane >> 4 & 1) + (cc >> 1 & 1);
    auto vfrag = [&](int k, int dt) __attribute__((always_inline)) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const uint16_t* p = vlane + k * K16 + 512 * dt;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * (vx ^ h))));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 256 + 8 * (vx ^ (h + 2)))));
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    };
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] = mfma32<T>(vfrag(k, dt), pb[k], o[dt]);
  };

  if (steps > 0) {
    request_block(key_first);
    request_rows(key_first, 0);
    request_block(key_first + 64);
    wait_lds_loads();
    __syncthreads();
    for (int i = 0; i < steps; ++i) {
      const int key0 = key_first + 64 * i;
      if (i + 1 < steps) {
        request_rows(key0 + 64, (i + 1) & 1);
        request_block(key0 + 128);
      }
      compute(key0, i & 1);
      wait_lds_loads();
      __syncthreads();
    }
  }
  l = halves_allreduce<SumOp>(l);
  const float top = m == -INFINITY ? -INFINITY : m * scale2;      // in units of log 2
  if (work.parts > 1) {
    float* at = a.tile_partial + ((int64_t)(slot * a.kv_heads + head) * a.most_parts + part) * (128 * (D + 2));
    const int mine = 32 * w + c;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4*>(at + mine * D + 32 * dt + 8 * j + 4 * h) = f32x4{o[dt][4 * j], o[dt][4 * j + 1], o[dt][4 * j + 2], o[dt][4 * j + 3]};
    if (h == 0) { at[128 * D + mine] = top; at[128 * D + 128 + mine] = l; }
    return;
  }
  if (row >= work.rows) return;
  const int q_head = head * a.share + row - token * a.share;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint16_t* out = static_cast<uint16_t*>(a.out) + (int64_t)(r.first + token) * a.out_stride + (int64_t)q_head * D + 4 * h;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<u32x2*>(out + 32 * dt + 8 * j) = u32x2{Mfma<T>::pack(o[dt][4 * j] * inv, o[dt][4 * j + 1] * inv), Mfma<T>::pack(o[dt][4 * j + 2] * inv, o[dt][4 * j + 3] * inv)};
  if (a.lse && h == 0) a.lse[(int64_t)(r.first + token) * a.q_heads + q_head] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// 1024 values of a tile whose keys were split, four to a thread: the parts in the order of the keys.
template <typename T, int D> __global__ __launch_bounds__(256) void paged_tile_join_kernel(const PagedArgs a) {
  const int head = blockIdx.x % a.kv_heads, slot = blockIdx.x / a.kv_heads;
  TileWork work;
  if (!tile_work(a, slot, &work) || work.parts == 1) return;
  const int e = (blockIdx.y * 256 + threadIdx.x) * 4, mine = e / D, row = work.row0 + mine;
  if (row >= work.rows) return;
  const float* at = a.tile_partial + (int64_t)(slot * a.kv_heads + head) * a.most_parts * (128 * (D + 2));
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < work.parts; k0 += 4) {
    float pm[4], pl[4];
    f32x4 po[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* x = at + (int64_t)min(k0 + i, work.parts - 1) * (128 * (D + 2));
      pm[i] = x[128 * D + mine]; pl[i] = x[128 * D + 128 + mine];
      po[i] = *reinterpret_cast<const f32x4*>(x + e);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (k0 + i >= work.parts) continue;
      const float top = fmaxf(m, pm[i]), low = top == -INFINITY ? 0.f : top;
      const float f = __builtin_amdgcn_exp2f(m - low), g = __builtin_amdgcn_exp2f(pm[i] - low);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = o[j] * f + po[i][j] * g;
      l = l * f + pl[i] * g;
      m = top;
    }
  }
  const int token = row / a.share, q_head = head * a.share + row - token * a.share;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + (int64_t)(work.r.first + token) * a.out_stride + (int64_t)q_head * D + e % D) =
      u32x2{Mfma<T>::pack(o[0] * inv, o[1] * inv), Mfma<T>::pack(o[2] * inv, o[3] * inv)};
  if (a.lse && e % D == 0) a.lse[(int64_t)(work.r.first + token) * a.q_heads + q_head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <typename T, int D> hipError_t paged_tile_launch(const PagedArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((paged_tile_kernel<T, D>), dim3((unsigned)(a.slots * a.kv_heads * a.most_parts)), dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.most_parts == 1) return e;
  hipLaunchKernelGGL((paged_tile_join_kernel<T, D>), dim3((unsigned)(a.slots * a.kv_heads), D / 8), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T> hipError_t paged_tile_launch_type(const PagedArgs& a, int dim, hipStream_t s) {
  switch (dim) {
    case 32: return paged_tile_launch<T, 32>(a, s);
    case 64: return paged_tile_launch<T, 64>(a, s);
    case 96: return paged_tile_launch<T, 96>(a, s);
    default: return paged_tile_launch<T, 128>(a, s);
  }
}

}  // namespace fs
