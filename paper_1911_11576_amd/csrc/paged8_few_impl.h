// Attention over a paged cache in 8 bits, few rows a request: bound by the reading of codes, half as many bytes as 16-bit keys and values have.
//
// The work is cut and joined as for a cache in 16 bits (FewLine, few_finish, paged_few_join).  A wavefront has 64 keys in LDS, as many bytes as 32
// there: KT of them are a step's, the others of the steps to come.  Codes come into LDS by direct loads of whole rows, scales with them, a key's to a lane; they become numbers of the storage type on their way from
// LDS to the matrix unit: keys' codes as they stand, exactly, and the scores get the scales; for values in bf16 the weights get them, in fp16, where these
// could leave the type's range, the numbers (powers of two exactly, of e4m3 the rest of a scale goes to the weights).  6.2 TB/s for 80 requests of one token behind up to
// 30000 keys (32 / 8 heads of 128, e4m3, 267 us; a copy of 1 GiB reaches 6.65), 4.5 for one behind 131072 (int8, 60 us, of which the reading takes 40: the start of table
// and keys 4, wavefronts that end after others 7, results 1, the second kernel 6).
#pragma once
#include <type_traits>

#include "cache8.h"
#include "paged_few_impl.h"

namespace fs {

// Rows of D codes in LDS, 16 bytes x of row r in place x ^ f(r): eight lanes that read the same 16 bytes of eight rows of keys, and the eight rows of
// a transposing read of values, 4g .. 4g + 3 and those 16 behind them, fall on different banks.
template <int D> __device__ __forceinline__ int few8_turn_k(int row) { return D == 128 ? row & 7 : D == 64 ? row >> 1 & 3 : row >> 2 & 1; }
template <int D> __device__ __forceinline__ int few8_turn_v(int row) { return D == 128 ? (row & 3) | (row >> 2 & 4) : D == 64 ? (row >> 1 & 1) | (row >> 3 & 2) : row >> 4 & 1; }

template <int D, int NT, int W> struct Few8Lds {
  FewLds<D, NT, W> few;            // (rows: 64 of D codes instead of 32 of D numbers)
  float scales[W][2][2][64];       // by turns: KT of the keys, KT of the values
};

// Workgroup p of 1 << log_groups (of as many as there are places for tiles where log_groups is -1).
template <typename T, class Code, int D, int NT, int W, int KT, bool ONCE> __device__ __forceinline__ void paged8_few(const PagedArgs& a, Few8Lds<D, NT, W>& lds, int p) {
  constexpr int KS = D / 32, DT = D / 16, M = 16 * NT, KEYS = KT * W, S = 64 / KT, TT = KT / 16, C = D / 16, N = KT * D / 1024;      // S: steps in LDS; C: 16-byte pieces of a row; N: direct loads of KT rows
  constexpr int E = 1 + KT / 32;      // loads of blocks to come and of scales
  constexpr bool kWeights = __is_same(T, bf16_t);                         // the scales of values go to the weights, else into the numbers ...
  constexpr bool kRest = !kWeights && __is_same(Code, E4m3);              // ... but for what is left of them beside a power of two
  typedef Numbers<Code, T> Num;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int c = lane & 15, g = lane >> 4;
  uint8_t *ksh = reinterpret_cast<uint8_t*>(lds.few.rows[w][0]), *vsh = reinterpret_cast<uint8_t*>(lds.few.rows[w][1]);
  const uint32_t k_lds = lds_address(ksh), v_lds = lds_address(vsh), b_lds = lds_address(&lds.few.blocks[w][0][0]), s_lds = lds_address(&lds.scales[w][0][0][0]);
  auto& blocks = lds.few.blocks;

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
  const uint8_t *kbase = static_cast<const uint8_t*>(a.k), *vbase = static_cast<const uint8_t*>(a.v);
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
    // ---- the rows: their queries as B operands, and the keys they see.  Two dots of 32 share 16 bytes of a key's row, so their k runs over d = 64 j + 16 g
    // + 0 .. 7 and + 8 .. 15; of 32 that are left as usual.
    u32x4 qf[NT][KS];
    int until[NT], from[NT];
    int most = 0, least = 0x7fffffff;      // over the tile's rows, uniform: no row sees keys from `most` on, every one sees those before `least` ...
    int latest = 0;                        // ... and from `latest` on
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = tile.row0 + 16 * nt + c, there = min(row, rows - 1), token = there / a.share;
      const uint16_t* q = static_cast<const uint16_t*>(a.q) + (r.first + token) * a.q_stride + (int64_t)(tile.head * a.share + there - token * a.share) * D;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[nt][ks] = *reinterpret_cast<const u32x4*>(q + (ks < KS / 2 * 2 ? 32 * (ks & ~1) + 16 * g + 8 * (ks & 1) : 32 * ks + 8 * g));
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
    const int key_first = paged_first_key(a, r) + max(0, tile.unit - a.tile_units) * a.unit_keys;
    const int key_end = min(most, paged_first_key(a, r) + (tile.unit + n - a.tile_units) * a.unit_keys);
    // ---- KT keys: lane k's key, k mod KT of them, has its row at `at`, its scales at `scale_at`; load i brings piece (64 i + lane) % C of key (64 i + lane) / C
    int block;
    int64_t at, scale_at;
    auto block_of = [&](int key0) __attribute__((always_inline)) { return table + (min(key0 + (lane & (KT - 1)), r.keys - 1) >> a.cache.shift); };
    auto locate = [&](int key0) __attribute__((always_inline)) {      // -> which of the keys are there
      const int key = key0 + (lane & (KT - 1));
      const bool ok = key < key_end && (unsigned)block < (unsigned)a.cache.blocks;
      at = head_at + (int64_t)(ok ? block : 0) * a.cache.block + (int64_t)(key & in_block) * a.cache.slot;
      scale_at = (int64_t)(ok ? block : 0) * a.kv_heads + tile.head;
      return __ballot(ok);
    };
    auto row_of = [&](int i) { return (64 * i + lane) / C; };
    // (turn: the place in LDS of a step)
    auto bring_blocks = [&](int key0, int turn) __attribute__((always_inline)) { load_lds4(block_of(key0), b_lds + 256 * turn); };
    auto bring_k = [&](int turn) __attribute__((always_inline)) {
      if constexpr (KT == 64) {
        load_lds4(reinterpret_cast<const int*>(a.k_scales) + scale_at, s_lds + 512 * turn);
        load_lds4(reinterpret_cast<const int*>(a.v_scales) + scale_at, s_lds + 512 * turn + 256);
      } else {
        load_lds4(reinterpret_cast<const int*>(lane < 32 ? a.k_scales : a.v_scales) + scale_at, s_lds + 512 * turn);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = row_of(i), piece = (64 * i + lane) % C ^ few8_turn_k<D>(row);
        load_lds16<0, ONCE>(reinterpret_cast<const uint16_t*>(kbase + __shfl((long long)at, row) + 16 * piece), k_lds + KT * D * turn + 1024 * i);
      }
    };
    auto bring_v = [&](int turn) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = row_of(i), piece = (64 * i + lane) % C ^ few8_turn_v<D>(row);
        load_lds16<0, ONCE>(reinterpret_cast<const uint16_t*>(vbase + __shfl((long long)at, row) + 16 * piece), v_lds + KT * D * turn + 1024 * i);
      }
    };
    const int kturn = few8_turn_k<D>(c), vrow = 4 * g + (c >> 1 & 3) + (c >> 3) * 16, vturn = few8_turn_v<D>(vrow);
    const uint8_t *klane = ksh + c * D, *vlane = vsh + vrow * D + 8 * (c & 1);
    uint64_t valid = 0, valid_next = 0;      // of the step's keys those that are there; S 2: of the next step's
    auto work = [&](int key0, auto at_turn) __attribute__((always_inline)) {
      constexpr int turn = decltype(at_turn)::value, ROWS = KT * D * turn;
      constexpr uint64_t kAll = KT == 64 ? ~0ull : 0xffffffffull;
      const bool plain = (valid & kAll) == kAll && key0 + KT <= least && key0 >= latest;      // every row sees every one
      const bool next = key0 + KEYS < key_end, more = key0 + S * KEYS < key_end;              // steps to come, and to be requested
      const float *kscales = &lds.scales[w][turn][0][0], *vscales = kscales + KT;
      // the keys and the scales are there (the values, and what was requested behind them, may not be)
      if (S == 1 || !next) wait_loads<N>();
      else wait_loads<3 * N + E>();
      f32x4 s[NT][TT];
      float kscale[TT], vscale[TT];      // of keys 16 t + 4 g + 0 .. 3, which are of one block
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const float f = kscales[16 * t + 4 * g] * a.scale2;
        kscale[t] = fmaf(f, 0.f, f);      // infinite: NaN, or a dot below 0 would leave the key without a weight and the result a number
        vscale[t] = vscales[16 * t + 4 * g];
      }
      // fp16, where a row may not see every key: also that of the values of key `lane`, since bring_k has the scales of a later step written to their place
      float lane_scale = 1.f;
      if (!kWeights && !plain) lane_scale = vscales[lane & (KT - 1)];
#pragma unroll
      for (int t = 0; t < TT; ++t) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < KS / 2; ++j) {
          const u32x4 kc = *reinterpret_cast<const u32x4*>(klane + ROWS + 16 * t * D + 16 * ((4 * j + g) ^ kturn));
          const u32x4 k0 = Num::plain(u32x2{kc[0], kc[1]}), k1 = Num::plain(u32x2{kc[2], kc[3]});
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            s[nt][t] = Mfma<T>::run(k0, qf[nt][2 * j], s[nt][t]);
            s[nt][t] = Mfma<T>::run(k1, qf[nt][2 * j + 1], s[nt][t]);
          }
        }
        if constexpr (KS & 1) {
          const u32x4 k0 = Num::plain(*reinterpret_cast<const u32x2*>(klane + ROWS + 16 * t * D + 16 * ((4 * (KS / 2) + (g >> 1)) ^ kturn) + 8 * (g & 1)));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[nt][t] = Mfma<T>::run(k0, qf[nt][KS - 1], s[nt][t]);
        }
      }
      uint64_t valid_new = 0;
      if (more) {
        block = blocks[w][turn][lane];
        valid_new = locate(key0 + S * KEYS);
        wait_lds_reads();
        bring_blocks(key0 + 2 * S * KEYS, turn);
        bring_k(turn);
      }
      u32x4 pb[NT][TT / 2];
      uint32_t see[NT][TT / 2];      // a bit for every key that the row sees, from the lane's first on
      if (!plain) {
        auto below = [](int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1; };
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int u = 0; u < TT / 2; ++u) {
            const int first = key0 + 32 * u;
            see[nt][u] = ((uint32_t)(valid >> 32 * u) & below(until[nt] - first) & ~below(from[nt] - first)) >> (4 * g);
          }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float top = m[nt];
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[nt][t][i] *= kscale[t];
        if (!plain) {
#pragma unroll
          for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][t][i] = see[nt][t / 2] & 1u << (16 * (t & 1) + i) ? s[nt][t][i] : -INFINITY;
        }
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, s[nt][t][i]);
        top = rows_allreduce<MaxOp>(top);
        const float low = top == -INFINITY ? 0.f : top;
        const float keep = sum_factor(m[nt] - low);
        m[nt] = top;
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < TT; ++t)
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
        if constexpr (kWeights || kRest) {
#pragma unroll
          for (int t = 0; t < TT; ++t) {
            const float f = kRest ? rest_of(vscale[t]) : vscale[t];
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][t][i] *= f;
          }
          if (!plain) {      // (a key that is not seen may have any scale)
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i) s[nt][t][i] = see[nt][t / 2] & 1u << (16 * (t & 1) + i) ? s[nt][t][i] : 0.f;
          }
        }
        // rounded to T for the second dot alone: half a step of each weight, where fp32 weights would take that dot twice; the sum is of them unrounded
#pragma unroll
        for (int u = 0; u < TT / 2; ++u)
          pb[nt][u] = u32x4{Mfma<T>::pack(s[nt][2 * u][0], s[nt][2 * u][1]), Mfma<T>::pack(s[nt][2 * u][2], s[nt][2 * u][3]), Mfma<T>::pack(s[nt][2 * u + 1][0], s[nt][2 * u + 1][1]),
                            Mfma<T>::pack(s[nt][2 * u + 1][2], s[nt][2 * u + 1][3])};
      }
      // what the numbers of values are multiplied by
      float into[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) into[t] = kWeights ? 1.f : kRest ? power_of(vscale[t]) : vscale[t];
      // the values are there (what was requested behind them may not be)
      if constexpr (S == 1) {
        if (more) wait_loads<N + E>();
        else wait_loads<0>();
      } else {
        if (more) wait_loads<3 * N + 2 * E>();
        else if (next) wait_loads<2 * N + E>();
        else wait_loads<0>();
      }
      if (!plain) {
        // values of keys that are none do not count, whatever lies there; a NaN of another, or a number beyond the type's range, is added as it is in the
        // rows that see it, and the second dot runs without it
        auto odd = [&](float code, float scale) __attribute__((always_inline)) {
          const float x = code * (kWeights ? 1.f : kRest ? power_of(scale) : scale);
          return !(fabsf(x) < (kWeights ? INFINITY : 65520.f));
        };
        bool any = false;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          u32x4* v = reinterpret_cast<u32x4*>(vsh + ROWS + 16 * (64 * i + lane));
          const int row = row_of(i);
          const float scale = kWeights ? 1.f : __shfl(lane_scale, row);
          if (!(valid >> row & 1)) {
            *v = u32x4{0u, 0u, 0u, 0u};
          } else {
            if constexpr (__is_same(Code, E4m3)) {
              const u32x4 x = *v;
#pragma unroll
              for (int j = 0; j < 4; ++j) any |= (((x[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
            }
            if (!kWeights) any |= !(fabsf(kRest ? power_of(scale) : scale) * (__is_same(Code, E4m3) ? 448.f : 128.f) < 65520.f);
          }
        }
        if (__ballot(any)) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll 1
            for (int k = 0; k < KT; ++k) {
              const float scale = kWeights ? 1.f : as_f32(__builtin_amdgcn_readlane(as_u32(lane_scale), k));
              float x[4];
              Code::unpack(*reinterpret_cast<const uint32_t*>(vsh + ROWS + k * D + 16 * (dt ^ few8_turn_v<D>(k)) + 4 * g), x);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                const bool seen = (valid >> k & 1) && key0 + k < until[nt] && key0 + k >= from[nt];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const float y = x[i] * scale;
                  o[nt][dt][i] += seen && odd(x[i], scale) ? (fabsf(y) < INFINITY ? copysignf(INFINITY, y) : y) : 0.f;
                }
              }
            }
#pragma unroll
          for (int i = 0; i < N; ++i) {
            u32x4* v = reinterpret_cast<u32x4*>(vsh + ROWS + 16 * (64 * i + lane));
            const float scale = kWeights ? 1.f : __shfl(lane_scale, row_of(i));
            u32x4 y = *v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float x[4];
              Code::unpack(y[j], x);
#pragma unroll
              for (int e = 0; e < 4; ++e) y[j] = odd(x[e], scale) ? y[j] & ~(0xffu << (8 * e)) : y[j];
            }
            *v = y;
          }
        }
        // a number's factor that is none would make NaN of a zero
        if (!kWeights)
#pragma unroll
          for (int t = 0; t < TT; ++t) into[t] = fabsf(into[t]) < INFINITY ? into[t] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < TT / 2; ++u)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          typedef int i32x2 __attribute__((ext_vector_type(2)));
          typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
          const u32x2 vc = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(vlane + ROWS + 32 * u * D + 16 * (dt ^ vturn))));
          const u32x4 vt = kWeights ? Num::plain(vc) : Num::scaled(vc, into[2 * u], into[2 * u + 1]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) o[nt][dt] = Mfma<T>::run(vt, pb[nt][u], o[nt][dt]);
        }
      if (more) {
        wait_lds_reads();
        bring_v(turn);
      }
      valid = S == 1 ? valid_new : valid_next;
      if (S > 1) valid_next = valid_new;
    };
    // ---- the loop: this wavefront's KT of every KT W keys, what LDS has room for in flight
    int key = key_first + KT * w;
    if (key < key_end) {
      block = *block_of(key);
      const int block1 = S > 1 ? *block_of(key + KEYS) : 0;
      valid = locate(key);
      // The queries are there (as the block is, which was requested behind them): used here, or the compiler, which knows nothing of the loads into LDS, would wait
      // for all loads where the loop uses them.
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[nt][ks]));
      bring_blocks(key + S * KEYS, 0);
      bring_k(0);
      bring_v(0);
      if constexpr (S > 1) {
        if (key + KEYS < key_end) {
          block = block1;
          valid_next = locate(key + KEYS);
          bring_blocks(key + 3 * KEYS, 1);
          bring_k(1);
          bring_v(1);
        }
      }
      for (;;) {
        work(key, std::integral_constant<int, 0>{});
        key += KEYS;
        if (key >= key_end) break;
        if constexpr (S > 1) {
          work(key, std::integral_constant<int, 1>{});
          key += KEYS;
          if (key >= key_end) break;
        }
      }
    }
    few_finish<T, D, NT, W>(a, lds.few, tile, n, 2 * p + (cur == u0 ? 0 : 1), o, m, l);
    __syncthreads();      // (before the next tile's V)
    cur += n;
  }
}

// Keys of a step: 64 at once cost fewer instructions for each; with two tiles of rows the registers hold the scores of 32 alone, and there is a step in flight
// behind this one.
constexpr int few8_keys(int nt) { return nt == 1 ? 64 : 32; }
template <typename T, class Code, int D, int NT, int W, bool ONCE> __global__ __launch_bounds__(64 * W, 2) void paged8_few_kernel(const PagedArgs a) {
  __shared__ __align__(1024) Few8Lds<D, NT, W> lds;
  paged8_few<T, Code, D, NT, W, few8_keys(NT), ONCE>(a, lds, blockIdx.x);
}

// Codes go past the caches (ONCE) where no other head has codes in their lines (a.once); heads of 128 fill lines, and those of 32 gain nothing from it.  (80 requests of up
// to 30000 keys, heads of 64, 16 of them: one behind the other 265 us, through the caches 294; side by side 420 and 363; 16 of 32 side by side 339 and 260.)
template <typename T, class Code, int D, int NT, bool ONCE> hipError_t paged8_few_launch(const PagedArgs& a, hipStream_t s) {
  if (a.log_groups < 0 && a.few_grid > 256) hipLaunchKernelGGL((paged8_few_kernel<T, Code, D, NT, 4, ONCE>), dim3(a.few_grid), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged8_few_kernel<T, Code, D, NT, 8, ONCE>), dim3(a.few_grid), dim3(512), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.log_groups < 0) return e;
  return (__is_same(T, f16_t) ? paged_few_join_launch_f16 : paged_few_join_launch_bf16)(a, D, NT, s);
}
template <typename T, class Code, int D, bool ONCE> hipError_t paged8_few_launch_rows(const PagedArgs& a, int row_tiles, hipStream_t s) {
  return row_tiles == 1 ? paged8_few_launch<T, Code, D, 1, ONCE>(a, s) : paged8_few_launch<T, Code, D, 2, ONCE>(a, s);
}

template <typename T, class Code> hipError_t paged8_few_launch_type(const PagedArgs& a, int dim, int row_tiles, hipStream_t s) {
  switch (dim) {
    case 32: return paged8_few_launch_rows<T, Code, 32, false>(a, row_tiles, s);
    case 64: return a.once ? paged8_few_launch_rows<T, Code, 64, true>(a, row_tiles, s) : paged8_few_launch_rows<T, Code, 64, false>(a, row_tiles, s);
    case 96: return a.once ? paged8_few_launch_rows<T, Code, 96, true>(a, row_tiles, s) : paged8_few_launch_rows<T, Code, 96, false>(a, row_tiles, s);
    default: return paged8_few_launch_rows<T, Code, 128, true>(a, row_tiles, s);
  }
}

}  // namespace fs
