// Attention over a paged cache, few rows a request (single tokens, a few guessed ones): bound by the reading of keys and values.
//
// The work of all requests is one line of units, (request, key head, tile of 16 * NT rows, run of keys), cut into as many equal
// runs as there are workgroups: each finds its own from the lengths on the device, whatever their spread.  A workgroup's four
// wavefronts take 32 keys each of every 128; a wavefront loads its keys straight into MFMA operands and its values through
// registers into LDS of its own (no barrier in the loop), the next 32 keys' in flight meanwhile.  At the end of a tile's run the
// wavefronts' maxima, sums and results meet in LDS; a tile that one workgroup does from end to end is stored, parts of others go to
// the partial results, which paged_few_join_kernel adds in the order of the keys.
#pragma once
#include "paged_attn_impl.h"

namespace fs {

constexpr int kFewGroups = 9;      // log2 of the workgroups: two to a CU

// Partial results of a workgroup: its first run of a tile and its last, each M rows of D sums, M maxima, M sums of exponentials.
template <int D, int NT> struct FewPart { static constexpr int kRows = 16 * NT, kFloats = kRows * (D + 2); };

// The line of units.  Every wavefront walks it for itself, 64 requests at a time, one a lane.
template <int NT> struct FewLine {
  const PagedArgs& a;
  uint32_t total = 0;
  // the 64 requests from `base` on: units before the first, and a lane's: those up to and with its own
  int base = 0;
  uint32_t before = 0, upto = 0, all = 0;
  PagedRequest mine{};
  uint32_t units = 0;

  __device__ __forceinline__ FewLine(const PagedArgs& args) : a(args) {}
  __device__ __forceinline__ int key_units(const PagedRequest& r) const {
    return max(1, (r.keys - paged_first_key(a, r) + a.unit_keys - 1) / a.unit_keys);
  }
  __device__ __forceinline__ void load(int from) {
    const int b = from + (int)(threadIdx.x & 63);
    base = from;
    units = 0;
    if (b < a.requests) {
      mine = paged_request(a, b);
      if (mine.fresh * a.share <= a.few_rows) units = (uint32_t)((mine.fresh * a.share + 16 * NT - 1) / (16 * NT)) * (uint32_t)key_units(mine) * (uint32_t)a.kv_heads;
    }
    upto = units;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t t = __shfl_up(upto, d);
      if ((int)(threadIdx.x & 63) >= d) upto += t;
    }
    all = __builtin_amdgcn_readlane(upto, 63);
  }
  __device__ __forceinline__ void count() {
    for (int from = 0; from < a.requests; from += 64) {
      load(from);
      total += all;
    }
    if (a.requests > 64) load(0);
    before = 0;
  }
  // where workgroup p's run begins
  __device__ __forceinline__ uint32_t cut(int p, int log_groups) const { return (uint32_t)((uint64_t)p * total >> log_groups); }
  // log2 of the workgroups that have work: at least a unit each
  __device__ __forceinline__ int groups() const { return min(a.log_groups, 31 - __clz((int)max(total, 1u))); }
  struct Tile { int b, head, row0, unit, n_units; uint32_t first; PagedRequest r; };      // first: the tile's first unit in the line
  __device__ __forceinline__ Tile find(uint32_t unit) {
    while (unit >= before + all && base + 64 < a.requests) {
      before += all;
      load(base + 64);
    }
    const uint64_t behind = __ballot(before + upto <= unit);
    const int lane = __popcll(behind);
    Tile t;
    t.b = base + lane;
    t.r = PagedRequest{__builtin_amdgcn_readlane(mine.first, lane), __builtin_amdgcn_readlane(mine.fresh, lane), __builtin_amdgcn_readlane(mine.keys, lane)};
    const uint32_t start = before + __builtin_amdgcn_readlane(upto, lane) - __builtin_amdgcn_readlane(units, lane);
    t.n_units = key_units(t.r);
    const uint32_t tile = (unit - start) / (uint32_t)t.n_units, tiles = (uint32_t)(t.r.fresh * a.share + 16 * NT - 1) / (16 * NT);
    t.unit = (int)(unit - start - tile * t.n_units);
    t.first = unit - t.unit;
    t.head = (int)(tile / tiles);
    t.row0 = (int)(tile - t.head * tiles) * 16 * NT;
    return t;
  }
};

template <typename T, int D, int NT> __global__ __launch_bounds__(256, 2) void paged_few_kernel(const PagedArgs a) {
  constexpr int KS = D / 32, DT = D / 16, M = 16 * NT;
  constexpr int VP = D + (D == 64 ? 8 : 16);       // row of V in LDS (halves), padded against bank conflicts
  constexpr int OP = D + 4;                        // row of results in LDS (floats)
  constexpr int kLds = 4 * 32 * VP * 2 > 4 * M * OP * 4 ? 4 * 32 * VP * 2 : 4 * M * OP * 4;
  __shared__ __align__(16) unsigned char smem[kLds];
  __shared__ float ms[4][M], ls[4][M];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int c = lane & 15, g = lane >> 4;
  uint16_t* vsh = reinterpret_cast<uint16_t*>(smem) + w * 32 * VP;
  float* osh = reinterpret_cast<float*>(smem);

  FewLine<NT> line(a);
  line.count();
  const int log_groups = line.groups(), p = blockIdx.x;
  if (p >> log_groups) return;
  const uint32_t u0 = line.cut(p, log_groups), u1 = line.cut(p + 1, log_groups);
  const uint16_t *kbase = static_cast<const uint16_t*>(a.k), *vbase = static_cast<const uint16_t*>(a.v);
  const int in_block = (1 << a.cache.shift) - 1;

  for (uint32_t cur = u0; cur < u1;) {
    const auto tile = line.find(cur);
    const int n = min(tile.n_units - tile.unit, (int)(u1 - cur));
    const PagedRequest r = tile.r;
    const int rows = r.fresh * a.share;
    const int* table = a.tables + (int64_t)tile.b * a.width;
    const int64_t head_at = (int64_t)tile.head * a.cache.head + 8 * g;
    // ---- the rows: their queries as B operands, and the keys they see
    u32x4 qf[NT][KS];
    int until[NT], from[NT];
    int most = 0, least = 0x7fffffff;      // over the tile's rows, uniform: no row sees keys from `most` on, every one sees those before `least` ...
    int latest = 0;                        // ... and from `latest` on
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = tile.row0 + 16 * nt + c, there = min(row, rows - 1), token = there / a.share;
      const uint16_t* q = static_cast<const uint16_t*>(a.q) + (r.first + token) * a.q_stride + (int64_t)(tile.head * a.share + there - token * a.share) * D + 8 * g;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[nt][ks] = *reinterpret_cast<const u32x4*>(q + 32 * ks);
      const int position = r.keys - r.fresh + token;
      until[nt] = a.causal ? min(r.keys, position + 1) : r.keys;
      from[nt] = a.window ? position + 1 - a.window : 0;
    }
    {
      const int t0 = tile.row0 / a.share, t1 = (min(tile.row0 + M, rows) - 1) / a.share, back = r.keys - r.fresh + 1;
      most = a.causal ? min(r.keys, back + t1) : r.keys;
      least = a.causal ? min(r.keys, back + t0) : r.keys;
      latest = a.window ? back + t1 - a.window : 0;
    }
    f32x4 o[NT][DT];
    float m[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt] = -INFINITY; l[nt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[nt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int key_first = paged_first_key(a, r) + tile.unit * a.unit_keys;
    const int key_end = min(most, key_first + n * a.unit_keys);
    u32x4 vf[2][KS];      // values on their way to LDS
    bool ok[2];           // the lane's two keys are there
    uint32_t valid = 0;   // of 32 keys those that are there
    bool plain, odd;      // every row sees every key; not so, and some value is infinite or NaN
    // ---- 32 keys: the block numbers of the lane's two keys, then their rows
    auto request_blocks = [&](int key0, int (&block)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) block[t] = table[min(key0 + 16 * t + c, r.keys - 1) >> a.cache.shift];
    };
    auto request_rows = [&](int key0, const int (&block)[2], u32x4 (&kf)[2][KS]) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int key = key0 + 16 * t + c;
        ok[t] = key < key_end && (unsigned)block[t] < (unsigned)a.cache.blocks;
        const int64_t at = (int64_t)(ok[t] ? block[t] : 0) * a.cache.block + (int64_t)(key & in_block) * a.cache.slot + head_at;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[t][ks] = *reinterpret_cast<const u32x4*>(kbase + at + 32 * ks);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) vf[t][ks] = *reinterpret_cast<const u32x4*>(vbase + at + 32 * ks);
      }
    };
    const uint16_t* vlane = vsh + (4 * g + (c >> 2)) * VP + 4 * (c & 3);
    auto stage = [&](int key0) __attribute__((always_inline)) {
      valid = (uint32_t)(__ballot(ok[0]) & 0xffffu) | (uint32_t)(__ballot(ok[1]) & 0xffffu) << 16;
      plain = valid == 0xffffffffu && key0 + 32 <= least && key0 >= latest;
      odd = false;
      if (!plain) {
        // keys that are none: their values do not count, whatever lies there; infinities and NaN of the others are for the rows that see them
        uint32_t any = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            if (!ok[t]) vf[t][ks] = u32x4{0u, 0u, 0u, 0u};
            any |= odd_values<T>(vf[t][ks]);
          }
        odd = __ballot(any != 0) != 0;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) *reinterpret_cast<u32x4*>(vsh + (16 * t + c) * VP + 32 * ks + 8 * g) = vf[t][ks];
    };
    auto work = [&](int key0, const u32x4 (&kf)[2][KS]) __attribute__((always_inline)) {
      f32x4 s[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          s[nt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) s[nt][t] = Mfma<T>::run(kf[t][ks], qf[nt][ks], s[nt][t]);
        }
      u32x4 pb[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float top = m[nt];
        bool seen[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = 16 * t + 4 * g + i;
            float z = s[nt][t][i] * a.scale2;
            seen[t][i] = true;
            if (!plain) {
              seen[t][i] = (valid >> k & 1) && key0 + k < until[nt] && key0 + k >= from[nt];
              z = seen[t][i] ? z : -INFINITY;
            }
            s[nt][t][i] = z;
            top = fmaxf(top, z);
          }
        top = rows_allreduce<MaxOp>(top);
        const float low = top == -INFINITY ? 0.f : top;
        const float keep = __builtin_amdgcn_exp2f(m[nt] - low);
        m[nt] = top;
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[nt][t][i] = __builtin_amdgcn_exp2f(s[nt][t][i] - low);
            sum += s[nt][t][i];
          }
        l[nt] = l[nt] * keep + sum;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[nt][dt][i] *= keep;
        pb[nt] = u32x4{Mfma<T>::pack(s[nt][0][0], s[nt][0][1]), Mfma<T>::pack(s[nt][0][2], s[nt][0][3]), Mfma<T>::pack(s[nt][1][0], s[nt][1][1]), Mfma<T>::pack(s[nt][1][2], s[nt][1][3])};
      }
      if (odd) {
        // rows that see an infinite or NaN value get it as it is; the second dot then runs without them
        for (int k = 0; k < 32; ++k) {
          if (!(valid >> k & 1)) continue;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const u32x2 v = *reinterpret_cast<const u32x2*>(vsh + k * VP + 16 * dt + 4 * g);
            const float x[4] = {Mfma<T>::lo(v[0]), Mfma<T>::hi(v[0]), Mfma<T>::lo(v[1]), Mfma<T>::hi(v[1])};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (key0 + k < until[nt] && key0 + k >= from[nt] && !(fabsf(x[i]) < INFINITY)) o[nt][dt][i] += x[i];
          }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            u32x4* v = reinterpret_cast<u32x4*>(vsh + (16 * t + c) * VP + 32 * ks + 8 * g);
            *v = without_odd<T>(*v);
          }
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vlane + 16 * dt)));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vlane + 16 * dt + 16 * VP)));
        const u32x4 vt = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[nt][dt] = Mfma<T>::run(vt, pb[nt], o[nt][dt]);
      }
    };
    // ---- the loop: this wavefront's 32 of every 128 keys, the next ones' loads in flight
    int key = key_first + 32 * w;
    if (key < key_end) {
      u32x4 kf[2][2][KS];
      int block[2];
      request_blocks(key, block);
      request_rows(key, block, kf[0]);
      request_blocks(key + 128, block);
      for (;;) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          stage(key);
          request_rows(key + 128, block, kf[half ^ 1]);
          request_blocks(key + 256, block);
          work(key, kf[half]);
          key += 128;
          if (key >= key_end) break;
        }
        if (key >= key_end) break;
      }
    }
    // ---- the four wavefronts' results together
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l[nt] = rows_allreduce<SumOp>(l[nt]);
      if (g == 0) { ms[w][16 * nt + c] = m[nt]; ls[w][16 * nt + c] = l[nt]; }
    }
    __syncthreads();      // (also: every wavefront is through with its V)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = 16 * nt + c;
      const float top = fmaxf(fmaxf(ms[0][row], ms[1][row]), fmaxf(ms[2][row], ms[3][row]));
      const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[nt] - top);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        f32x4 x = o[nt][dt];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] *= f;
        *reinterpret_cast<f32x4*>(osh + (w * M + row) * OP + 16 * dt + 4 * g) = x;
      }
    }
    __syncthreads();
    const bool whole = n == tile.n_units;
    float* part = whole ? nullptr : a.partial + (int64_t)(2 * p + (cur == u0 ? 0 : 1)) * FewPart<D, NT>::kFloats;
    for (int e = threadIdx.x; e < M * (D / 8); e += 256) {
      const int row = e / (D / 8), d = e % (D / 8) * 8;
      const float m0 = ms[0][row], m1 = ms[1][row], m2 = ms[2][row], m3 = ms[3][row], top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)), low = top == -INFINITY ? 0.f : top;
      const float sum = ls[0][row] * __builtin_amdgcn_exp2f(m0 - low) + ls[1][row] * __builtin_amdgcn_exp2f(m1 - low) + ls[2][row] * __builtin_amdgcn_exp2f(m2 - low) +
                        ls[3][row] * __builtin_amdgcn_exp2f(m3 - low);
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x4 y0 = *reinterpret_cast<const f32x4*>(osh + (k * M + row) * OP + d), y1 = *reinterpret_cast<const f32x4*>(osh + (k * M + row) * OP + d + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] += y0[i]; x[4 + i] += y1[i]; }
      }
      if (!whole) {
        *reinterpret_cast<f32x4*>(part + row * D + d) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4*>(part + row * D + d + 4) = f32x4{x[4], x[5], x[6], x[7]};
        if (d == 0) { part[M * D + row] = top; part[M * D + M + row] = sum; }
      } else if (tile.row0 + row < rows) {
        const int token = (tile.row0 + row) / a.share, head = tile.head * a.share + (tile.row0 + row) - token * a.share;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= inv;
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.out) + (int64_t)(r.first + token) * a.out_stride + (int64_t)head * D + d) =
            u32x4{Mfma<T>::pack(x[0], x[1]), Mfma<T>::pack(x[2], x[3]), Mfma<T>::pack(x[4], x[5]), Mfma<T>::pack(x[6], x[7])};
        if (a.lse && d == 0) a.lse[(int64_t)(r.first + token) * a.q_heads + head] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
      }
    }
    __syncthreads();      // (before the next tile's V)
    cur += n;
  }
}

// Tiles that several workgroups did: the workgroup of this kernel that stands at the first cut inside one joins its parts, 256 values of it, in the
// order of the keys; its wavefronts take every fourth part.
template <typename T, int D, int NT> __global__ __launch_bounds__(256) void paged_few_join_kernel(const PagedArgs a) {
  constexpr int M = 16 * NT;
  constexpr int64_t kFloats = FewPart<D, NT>::kFloats;
  __shared__ float ms[4][64], ls[4][64];
  __shared__ f32x4 os[4][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  FewLine<NT> line(a);
  line.count();
  const int log_groups = line.groups(), p = blockIdx.x + 1;
  if (p >> log_groups) return;
  const uint32_t at = line.cut(p, log_groups);
  if (at >= line.total) return;
  const auto tile = line.find(at);
  const uint32_t first = tile.first, end = first + tile.n_units, before = line.cut(p - 1, log_groups);
  if (at == first || before > first) return;      // no part before the cut, or another cut is the first
  int last = p;                                   // the workgroup that the last part is of
  while (line.cut(last + 1, log_groups) < end) ++last;
  const int e = blockIdx.y * 256 + lane * 4, row = e / D;
  const int n = last - p + 2;
  auto part = [&](int k) { return a.partial + (2 * (p - 1 + k) + (k == 0 && before != first ? 1 : 0)) * kFloats; };
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = w; k0 < n; k0 += 32) {
    float pm[8], pl[8];
    f32x4 po[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float* x = part(min(k0 + 4 * i, n - 1));
      pm[i] = x[M * D + row]; pl[i] = x[M * D + M + row];
      po[i] = *reinterpret_cast<const f32x4*>(x + e);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (k0 + 4 * i >= n) continue;
      const float top = fmaxf(m, pm[i]), low = top == -INFINITY ? 0.f : top;
      const float f = __builtin_amdgcn_exp2f(m - low), h = __builtin_amdgcn_exp2f(pm[i] - low);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = o[j] * f + po[i][j] * h;
      l = l * f + pl[i] * h;
      m = top;
    }
  }
  ms[w][lane] = m; ls[w][lane] = l; os[w][lane] = o;
  __syncthreads();
  if (w) return;
  const float top = fmaxf(fmaxf(ms[0][lane], ms[1][lane]), fmaxf(ms[2][lane], ms[3][lane])), low = top == -INFINITY ? 0.f : top;
  o = f32x4{0.f, 0.f, 0.f, 0.f};
  l = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float h = __builtin_amdgcn_exp2f(ms[k][lane] - low);
    l += ls[k][lane] * h;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] += os[k][lane][j] * h;
  }
  if (tile.row0 + row >= tile.r.fresh * a.share) return;
  const int token = (tile.row0 + row) / a.share, head = tile.head * a.share + (tile.row0 + row) - token * a.share;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + (int64_t)(tile.r.first + token) * a.out_stride + (int64_t)head * D + e % D) =
      u32x2{Mfma<T>::pack(o[0] * inv, o[1] * inv), Mfma<T>::pack(o[2] * inv, o[3] * inv)};
  if (a.lse && e % D == 0) a.lse[(int64_t)(tile.r.first + token) * a.q_heads + head] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <typename T, int D, int NT> hipError_t paged_few_launch(const PagedArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((paged_few_kernel<T, D, NT>), dim3(1 << a.log_groups), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((paged_few_join_kernel<T, D, NT>), dim3((1 << a.log_groups) - 1, 16 * NT * D / 256), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T> hipError_t paged_few_launch_type(const PagedArgs& a, int dim, int row_tiles, hipStream_t s) {
  switch (dim) {
    case 32: return row_tiles == 1 ? paged_few_launch<T, 32, 1>(a, s) : paged_few_launch<T, 32, 2>(a, s);
    case 64: return row_tiles == 1 ? paged_few_launch<T, 64, 1>(a, s) : paged_few_launch<T, 64, 2>(a, s);
    case 96: return row_tiles == 1 ? paged_few_launch<T, 96, 1>(a, s) : paged_few_launch<T, 96, 2>(a, s);
    default: return row_tiles == 1 ? paged_few_launch<T, 128, 1>(a, s) : paged_few_launch<T, 128, 2>(a, s);
  }
}

}  // namespace fs
