// Attention over a paged cache, few rows a request (single tokens, a few guessed ones): bound by the reading of keys and values.
//
// The work of all requests is one line of units, (request, set of key heads, tile of 16 * NT rows, run of keys), cut into equal
// runs, one to as many workgroups as a set has heads: each finds its own from the lengths on the device, whatever their spread.  The workgroups of a set walk the
// same keys of its heads at the same time behind one L2, which fetches lines that heads share once.  A workgroup's
// wavefronts take 32 keys each of a step; a wavefront brings keys and values into LDS of its own by direct loads of whole rows (no
// barrier in the loop), the next 32 keys as soon as the first dot is through with these, their values behind the second.  At the end of a tile's run the
// wavefronts' maxima, sums and results meet in LDS; a tile that one workgroup does from end to end is stored, parts of others go to
// the partial results, which paged_few_join_kernel adds in the order of the keys.  Where no request can be long a workgroup has
// one tile and all of its keys, and nothing is left to join.  6.5 TB/s for 64 requests of one token behind up to 24000 keys (32 / 8 heads of 128, 346 us; a copy of
// 1 GiB reaches 6.6), 5.5 for one behind 131072 (97 us); keys and values through the caches 397 and 108 (before the sets).
#pragma once
#include "paged_attn_impl.h"

namespace fs {


// Partial results of a workgroup: its first run of a tile and its last, each M rows of D sums, M maxima, M sums of exponentials.
template <int D, int NT> struct FewPart { static constexpr int kRows = 16 * NT, kFloats = kRows * (D + 2); };

// The line of units, of one key head of a set.  Every wavefront looks at it for itself, 64 requests at a time, one a lane.
template <int NT> struct FewLine {
  const PagedArgs& a;
  uint32_t total = 0;
  uint32_t chunks_upto = 0;      // units up to and with the lane's 64 requests, of the first 4096
  // the 64 requests from `base` on: units before the first, and a lane's: those up to and with its own
  int base = -1;
  uint32_t before = 0, upto = 0, all = 0;
  PagedRequest mine{};
  uint32_t units = 0;

  __device__ __forceinline__ FewLine(const PagedArgs& args) : a(args) {}
  __device__ __forceinline__ int key_units(const PagedRequest& r) const {
    return max(1, (r.keys - paged_first_key(a, r) + a.unit_keys - 1) / a.unit_keys);
  }
  __device__ __forceinline__ uint32_t units_of(const PagedRequest& r) const {
    if (r.fresh * a.share > a.few_rows) return 0;
    return (uint32_t)((r.fresh * a.share + 16 * NT - 1) / (16 * NT)) * (uint32_t)key_units(r) * (uint32_t)a.head_sets;
  }
  __device__ __forceinline__ PagedRequest request(int b) const { return b < a.requests ? paged_request(a, b) : PagedRequest{}; }
  __device__ __forceinline__ void load(int from) {
    base = from;
    mine = request(from + (int)(threadIdx.x & 63));
    units = units_of(mine);
    upto = (uint32_t)wave_upto((int)units);
    all = __builtin_amdgcn_readlane(upto, 63);
  }
  __device__ __forceinline__ void count() {
    if (a.requests <= 64) {
      load(0);
      total = all;
      return;
    }
    const int lane = threadIdx.x & 63;
    uint32_t sum = 0;
    for (int j = 0; j < a.requests; j += 256) {      // (four requests a lane in flight)
      PagedRequest r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = request(j + 64 * i + lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t n = (uint32_t)wave_sum((int)units_of(r[i]));
        total += n;
        if (lane == (j >> 6) + i) sum = n;
      }
    }
    chunks_upto = (uint32_t)wave_upto((int)sum);
  }
  // where workgroup p's run begins
  __device__ __forceinline__ uint32_t cut(int p, int log_groups) const { return (uint32_t)((uint64_t)p * total >> log_groups); }
  // log2 of the workgroups that have work, of one key head of a set: at least a unit each, so as many as the largest power of two among the units (32 / 8
  // heads of 128, one token behind 31 units of 256 keys 18.6 us, which 16 workgroups of a head do, behind 32 14.7, 33 17.5, 63 19.3, 64 19.4)
  __device__ __forceinline__ int groups() const { return min(a.log_groups - a.log_heads, 31 - __clz((int)max(total, 1u))); }
  struct Tile { int b, head, row0, unit, n_units; uint32_t first; PagedRequest r; bool there; };      // first: the tile's first unit in the line
  // the p-th tile, where a unit is one; of more than 64 requests the tile at place p, which takes fewer looks at their lengths
  __device__ __forceinline__ Tile whole(int p) {
    Tile t{};
    if (a.requests <= 64) {
      load(0);
      if ((uint32_t)p >= all) return t;
      return find((uint32_t)p);
    }
    const int at = p / a.head_sets;
    t.head = p - at * a.head_sets;
    t.b = paged_find(a, at, NT == 1 ? 4 : 5);
    t.there = t.b >= 0;
    if (!t.there) return t;
    t.r = paged_request(a, t.b);
    t.row0 = (at - paged_place(a, t.b, NT == 1 ? 4 : 5)) * 16 * NT;
    t.there = t.row0 < t.r.fresh * a.share && t.r.fresh * a.share <= a.few_rows;
    t.n_units = 1;
    return t;
  }
  __device__ __forceinline__ Tile find(uint32_t unit) {
    if (a.requests > 64) {
      const int chunk = __popcll(__ballot(chunks_upto <= unit));
      if (chunk < 64) {
        before = chunk ? __builtin_amdgcn_readlane(chunks_upto, chunk - 1) : 0;
        if (base != 64 * chunk) load(64 * chunk);
      } else {      // behind the first 4096 requests: one chunk behind the other
        if (base < 4096) {
          before = __builtin_amdgcn_readlane(chunks_upto, 63);
          load(4096);
        }
        while (unit >= before + all && base + 64 < a.requests) {
          before += all;
          load(base + 64);
        }
      }
    }
    const uint64_t behind = __ballot(before + upto <= unit);
    const int lane = min(63, (int)__popcll(behind));
    Tile t;
    t.b = base + lane;
    t.r = PagedRequest{__builtin_amdgcn_readlane(mine.first, lane), __builtin_amdgcn_readlane(mine.fresh, lane), __builtin_amdgcn_readlane(mine.keys, lane)};
    const uint32_t start = before + __builtin_amdgcn_readlane(upto, lane) - __builtin_amdgcn_readlane(units, lane);
    t.n_units = key_units(t.r);
    const uint32_t tile = (unit - start) / (uint32_t)t.n_units, tiles = (uint32_t)(t.r.fresh * a.share + 16 * NT - 1) / (16 * NT);
    t.unit = (int)(unit - start - tile * t.n_units);
    t.first = unit - t.unit;
    t.head = tiles ? (int)(tile / tiles) : 0;
    t.row0 = (int)(tile - t.head * tiles) * 16 * NT;
    // (requests whose rows overlap can be more units than 32 bits number: then what was found may be no tile)
    t.there = t.b < a.requests && (unsigned)t.head < (unsigned)a.head_sets && t.row0 >= 0 && t.row0 < t.r.fresh * a.share;
    return t;
  }
};

// 32 rows of D halves in LDS as direct loads of whole rows leave them, 16 bytes x of row r in place x ^ f(r): eight lanes that read the
// same 16 bytes of eight rows, and the four rows of a transposing read, fall on different banks.
template <int D> __device__ __forceinline__ int few_turn(int row) { return D == 128 ? 2 * (row & 7) : D == 64 ? row & 6 : row >> 1 & 2; }

// LDS of a workgroup of W wavefronts: keys and values of each while it reads them, then results.
template <int D, int NT, int W> struct FewLds {
  static constexpr int M = 16 * NT, OP = D + 4;      // OP: row of results (floats)
  union {
    uint16_t rows[W][2][32 * D];
    float results[W][M * OP];
  };
  int blocks[W][2][64];                              // block numbers of the keys to come
  float ms[W][M], ls[W][M];
};

// Workgroup p of 1 << log_groups (of as many as there are places for tiles where log_groups is -1).
template <typename T, int D, int NT, int W> __device__ __forceinline__ void paged_few(const PagedArgs& a, FewLds<D, NT, W>& lds, int p) {
  constexpr int KS = D / 32, DT = D / 16, M = 16 * NT, KEYS = 32 * W, C = D / 8, N = D / 16;      // C: 16-byte pieces of a row; N: direct loads of 32 rows
  constexpr int OP = FewLds<D, NT, W>::OP;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int c = lane & 15, g = lane >> 4;
  uint16_t *ksh = lds.rows[w][0], *vsh = lds.rows[w][1];
  const uint32_t k_lds = lds_address(ksh), v_lds = lds_address(vsh), b_lds = lds_address(&lds.blocks[w][0][0]);
  float* osh = &lds.results[0][0];
  auto& blocks = lds.blocks;
  auto& ms = lds.ms;
  auto& ls = lds.ls;

  FewLine<NT> line(a);
  uint32_t u0 = 0, u1 = 1;
  int head_in = 0;      // of its set
  if (a.log_groups >= 0) {
    if (a.neighbours) p = (p & 7) << (a.log_groups - 3) | p >> 3;      // (an XCD has every eighth workgroup)
    head_in = p & ((1 << a.log_heads) - 1);
    line.count();
    const int log_groups = line.groups(), run = p >> a.log_heads;
    if (run >> log_groups) return;
    u0 = line.cut(run, log_groups); u1 = line.cut(run + 1, log_groups);
  }
  const uint16_t *kbase = static_cast<const uint16_t*>(a.k), *vbase = static_cast<const uint16_t*>(a.v);
  const int in_block = (1 << a.cache.shift) - 1;

  for (uint32_t cur = u0; cur < u1;) {
    auto tile = a.log_groups < 0 ? line.whole(p) : line.find(cur);
    if (!tile.there) break;
    tile.head = tile.head << a.log_heads | head_in;
    const int n = min(tile.n_units - tile.unit, (int)(u1 - cur));
    const PagedRequest r = tile.r;
    const int rows = r.fresh * a.share;
    const int* table = a.tables + (int64_t)tile.b * a.width;
    const int64_t head_at = (int64_t)tile.head * a.cache.head;
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
    // ---- 32 keys: lane k's key has its row at `at`; load i brings piece (64 i + lane) % C of key (64 i + lane) / C
    int block;
    bool ok;
    int64_t at;
    auto block_of = [&](int key0) __attribute__((always_inline)) { return table + (min(key0 + lane, r.keys - 1) >> a.cache.shift); };
    auto locate = [&](int key0) __attribute__((always_inline)) {
      const int key = key0 + lane;
      ok = key < key_end && (unsigned)block < (unsigned)a.cache.blocks;
      at = head_at + (int64_t)(ok ? block : 0) * a.cache.block + (int64_t)(key & in_block) * a.cache.slot;
    };
    auto row_of = [&](int i) { return (64 * i + lane) / C; };
    auto bring = [&](const uint16_t* base, uint32_t lds) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = row_of(i), piece = (64 * i + lane) % C ^ few_turn<D>(row);
        load_lds16<0, true>(base + __shfl((long long)at, row) + 8 * piece, lds + 1024 * i);
      }
    };
    const int kturn = few_turn<D>(c), vturn = few_turn<D>(4 * g + (c >> 2));
    const uint16_t *klane = ksh + c * D, *vlane = vsh + (4 * g + (c >> 2)) * D + 4 * (c & 1);
    auto work = [&](int key0, int turn) __attribute__((always_inline)) {
      const uint32_t valid = (uint32_t)__ballot(ok);                                        // of 32 keys those that are there
      const bool plain = valid == 0xffffffffu && key0 + 32 <= least && key0 >= latest;      // every row sees every one
      const bool more = key0 + KEYS < key_end;
      wait_loads<N>();      // the keys are there (the values may not be)
      f32x4 s[NT][2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const u32x4 kf = *reinterpret_cast<const u32x4*>(klane + 16 * t * D + 8 * ((4 * ks + g) ^ kturn));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[nt][t] = Mfma<T>::run(kf, qf[nt][ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[nt][t]);
        }
      if (more) {
        block = blocks[w][turn][lane];
        locate(key0 + KEYS);
        wait_lds_reads();
        load_lds4(block_of(key0 + 2 * KEYS), b_lds + 256 * (turn ^ 1));
        bring(kbase, k_lds);
      }
      u32x4 pb[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float top = m[nt];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = 16 * t + 4 * g + i;
            float z = s[nt][t][i] * a.scale2;
            if (!plain) {
              z = (valid >> k & 1) && key0 + k < until[nt] && key0 + k >= from[nt] ? z : -INFINITY;
            }
            s[nt][t][i] = z;
            top = fmaxf(top, z);
          }
        top = rows_allreduce<MaxOp>(top);
        const float low = top == -INFINITY ? 0.f : top;
        const float keep = sum_factor(m[nt] - low);
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
        // rounded to T for the second dot alone: half a step of each weight, where fp32 weights would take that dot twice; the sum is of them unrounded
        pb[nt] = u32x4{Mfma<T>::pack(s[nt][0][0], s[nt][0][1]), Mfma<T>::pack(s[nt][0][2], s[nt][0][3]), Mfma<T>::pack(s[nt][1][0], s[nt][1][1]), Mfma<T>::pack(s[nt][1][2], s[nt][1][3])};
      }
      if (more) wait_loads<N + 1>();      // the values are there (the next keys may not be)
      else wait_loads<0>();
      if (!plain) {
        // values of keys that are none do not count, whatever lies there; an infinity or NaN of another is added as it is in the
        // rows that see it, and the second dot runs without it
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          u32x4* v = reinterpret_cast<u32x4*>(vsh + 8 * (64 * i + lane));
          if (!(valid >> row_of(i) & 1)) *v = u32x4{0u, 0u, 0u, 0u};
          else any |= odd_values<T>(*v);
        }
        if (__ballot(any != 0)) {
          for (int k = 0; k < 32; ++k)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              const u32x2 v = *reinterpret_cast<const u32x2*>(vsh + k * D + 8 * ((2 * dt + (g >> 1)) ^ few_turn<D>(k)) + 4 * (g & 1));
              const float x[4] = {Mfma<T>::lo(v[0]), Mfma<T>::hi(v[0]), Mfma<T>::lo(v[1]), Mfma<T>::hi(v[1])};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                const bool seen = (valid >> k & 1) && key0 + k < until[nt] && key0 + k >= from[nt];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[nt][dt][i] += seen && !(fabsf(x[i]) < INFINITY) ? x[i] : 0.f;
              }
            }
#pragma unroll
          for (int i = 0; i < N; ++i) {
            u32x4* v = reinterpret_cast<u32x4*>(vsh + 8 * (64 * i + lane));
            *v = without_odd<T>(*v);
          }
        }
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const uint16_t* v = vlane + 8 * ((2 * dt + (c >> 1 & 1)) ^ vturn);
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)v));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v + 16 * D)));
        const u32x4 vt = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[nt][dt] = Mfma<T>::run(vt, pb[nt], o[nt][dt]);
      }
      if (more) {
        wait_lds_reads();
        bring(vbase, v_lds);
      }
    };
    // ---- the loop: this wavefront's 32 of every 32 W keys, the next ones' loads in flight
    int key = key_first + 32 * w;
    if (key < key_end) {
      block = *block_of(key);
      locate(key);
      load_lds4(block_of(key + KEYS), b_lds);
      bring(kbase, k_lds);
      bring(vbase, v_lds);
      for (int turn = 0; key < key_end; key += KEYS, turn ^= 1) work(key, turn);
    }
    // ---- the wavefronts' results together
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l[nt] = rows_allreduce<SumOp>(l[nt]);
      if (g == 0) { ms[w][16 * nt + c] = m[nt]; ls[w][16 * nt + c] = l[nt]; }
    }
    __syncthreads();      // (also: every wavefront is through with its V)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = 16 * nt + c;
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < W; ++k) top = fmaxf(top, ms[k][row]);
      const float f = top == -INFINITY ? 0.f : sum_factor(m[nt] - top);
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
    for (int e = threadIdx.x; e < M * (D / 8); e += 64 * W) {
      const int row = e / (D / 8), d = e % (D / 8) * 8;
      float top = -INFINITY, sum = 0.f, x[8];
#pragma unroll
      for (int k = 0; k < W; ++k) top = fmaxf(top, ms[k][row]);
      const float low = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        sum += ls[k][row] * __builtin_amdgcn_exp2f(ms[k][row] - low);
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

template <typename T, int D, int NT, int W> __global__ __launch_bounds__(64 * W, 2) void paged_few_kernel(const PagedArgs a) {
  __shared__ __align__(1024) FewLds<D, NT, W> lds;
  paged_few<T, D, NT, W>(a, lds, blockIdx.x);
}

// The parts of a tile: running maximum, sum and 4 results of a thread, N parts requested at a time.
struct FewSum { float m, l; f32x4 o; };
__device__ __forceinline__ void few_add(FewSum& s, float m, float l, f32x4 o) {
  const float top = fmaxf(s.m, m), low = top == -INFINITY ? 0.f : top;
  const float f = sum_factor(s.m - low), h = sum_factor(m - low);
#pragma unroll
  for (int j = 0; j < 4; ++j) s.o[j] = s.o[j] * f + o[j] * h;
  s.l = s.l * f + l * h;
  s.m = top;
}
template <int N, int M, int D, class Part> __device__ __forceinline__ void few_add_parts(FewSum& s, int first, int step, Part part, int row, int e) {
  float m[N], l[N];
  f32x4 o[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float* x = part(first + i * step);
    m[i] = x[M * D + row]; l[i] = x[M * D + M + row];
    o[i] = *reinterpret_cast<const f32x4*>(x + e);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) few_add(s, m[i], l[i], o[i]);
}

// Tiles that several workgroups did, their parts added in the order of the keys: there is a workgroup here for every cut p of the line and head of a set, and
// those whose cuts lie in one tile share its rows, 256 values to a run.  A wavefront has a run, or takes turns with others at its parts where the
// runs are fewer (one token behind 131072 keys, 32 parts to a tile: 96.7 us with the first kernel, 99.2 where the workgroup
// of the first cut does all runs).
template <int D, int NT> struct FewJoin { static constexpr int kRuns = 16 * NT * D / 256, kWaves = kRuns > 8 ? kRuns : 16 / kRuns * kRuns, kThreads = 64 * kWaves; };
template <typename T, int D, int NT> __device__ __forceinline__ void paged_few_join(const PagedArgs& a, FewLine<NT>& line, int log_groups, int b) {
  constexpr int M = 16 * NT, W = FewJoin<D, NT>::kWaves;
  constexpr int64_t kFloats = FewPart<D, NT>::kFloats;
  __shared__ FewSum sums[W][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int p = (b >> a.log_heads) + 1, head_in = b & ((1 << a.log_heads) - 1);
  const uint32_t at = line.cut(p, log_groups);
  if (p >> log_groups || at >= line.total) return;
  auto tile = line.find(at);
  const uint32_t first = tile.first, end = first + tile.n_units;
  if (!tile.there || at == first) return;      // no part before the cut
  tile.head = tile.head << a.log_heads | head_in;
  // the first cut behind the tile's first unit, the last one before its end: p * total / groups > first, < end
  // (mostly this one is both, which costs no division)
  auto cut_behind = [&](uint32_t unit) { return (((uint64_t)unit << log_groups) + line.total - 1) / line.total; };
  const uint64_t cut0 = line.cut(p - 1, log_groups) <= first ? p : cut_behind(first + 1), behind = line.cut(p + 1, log_groups) >= end ? p + 1 : cut_behind(end);
  if (cut0 < 1 || cut0 > (uint64_t)p || behind <= (uint64_t)p) return;      // (not where rows of several requests are more units than 32 bits number)
  const int p0 = (int)cut0, last = (int)min(behind, (uint64_t)1 << log_groups) - 1;
  const int rows = min(M, tile.r.fresh * a.share - tile.row0), runs = (rows * D + 255) / 256;      // runs that have rows
  const int sharing = min(last - p0 + 1, runs), here = (runs + sharing - 1) / sharing, turns = W / here;
  if (p - p0 >= sharing) return;
  const int turn = wave / here, run = (p - p0) * here + wave - turn * here;
  const bool working = run < runs && turn < turns;
  const int e = run * 256 + lane * 4, row = e / D;
  const int n = last - p0 + 2;
  const bool whole = line.cut(p0 - 1, log_groups) == first;      // the first part is the first of its workgroup
  auto part = [&](int k) { return a.partial + (2 * ((p0 - 1 + k) << a.log_heads | head_in) + (k == 0 && !whole ? 1 : 0)) * kFloats; };
  FewSum s{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
  if (working) {
    int k = turn;
    for (; k + 7 * turns < n; k += 8 * turns) few_add_parts<8, M, D>(s, k, turns, part, row, e);
    if (k + 3 * turns < n) { few_add_parts<4, M, D>(s, k, turns, part, row, e); k += 4 * turns; }
    if (k + turns < n) { few_add_parts<2, M, D>(s, k, turns, part, row, e); k += 2 * turns; }
    if (k < n) few_add_parts<1, M, D>(s, k, turns, part, row, e);
  }
  if (turns > 1) {
    sums[wave][lane] = s;
    __syncthreads();
    if (!working || turn) return;
    for (int i = 1; i < min(turns, n); ++i) {
      const FewSum& x = sums[i * here + wave][lane];
      few_add(s, x.m, x.l, x.o);
    }
  }
  if (!working || row >= rows) return;
  const int r = tile.row0 + row, token = r / a.share, head = tile.head * a.share + r - token * a.share;
  const float inv = s.l == 0.f ? 0.f : 1.f / s.l;
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + (int64_t)(tile.r.first + token) * a.out_stride + (int64_t)head * D + e % D) =
      u32x2{Mfma<T>::pack(s.o[0] * inv, s.o[1] * inv), Mfma<T>::pack(s.o[2] * inv, s.o[3] * inv)};
  if (a.lse && e % D == 0) a.lse[(int64_t)(tile.r.first + token) * a.q_heads + head] = s.l == 0.f ? -INFINITY : (s.m + __builtin_amdgcn_logf(s.l)) * 0.6931471805599453f;
}

template <typename T, int D, int NT> __global__ __launch_bounds__((FewJoin<D, NT>::kThreads)) void paged_few_join_kernel(const PagedArgs a) {
  FewLine<NT> line(a);
  line.count();
  paged_few_join<T, D, NT>(a, line, line.groups(), blockIdx.x);
}

template <typename T, int D, int NT> hipError_t paged_few_launch(const PagedArgs& a, hipStream_t s) {
  // eight wavefronts fill a CU; whole tiles for more than every CU are done by four each, whose first loads pass while others work (D 128,
  // 32 / 8 heads: 32 requests of 500 keys 13.5 and 14.0 us, 64 27.3 and 23.8, 256 117 and 89; D 64, 256 of 100 50 and 21)
  if (a.log_groups < 0 && a.few_grid > 256) hipLaunchKernelGGL((paged_few_kernel<T, D, NT, 4>), dim3(a.few_grid), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_few_kernel<T, D, NT, 8>), dim3(a.few_grid), dim3(512), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.log_groups < 0) return e;
  hipLaunchKernelGGL((paged_few_join_kernel<T, D, NT>), dim3(a.few_grid - (1 << a.log_heads)), dim3(FewJoin<D, NT>::kThreads), 0, s, a);
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
