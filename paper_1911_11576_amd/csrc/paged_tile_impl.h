// Attention over a paged cache, many rows a request (chunks of prompts): bound by the matrix unit and the exponentials.
//
// A workgroup has 128 rows of one request and key head, 32 to a wavefront, and walks the keys that they see 64 at a time: keys
// and values by direct loads into LDS, the next 64 in flight to the other half while these are worked on, one
// barrier a step.  Both dots are v_mfma_f32_32x32x16.  A tile of more than an even share of the work is split over workgroups
// by its keys, and paged_mixed_join_kernel adds the parts in their order.  850 to 930 TFLOP/s at D 128, by the card and its clock (8 chunks of 1 to 1024 tokens behind up to
// 12000 keys, 32 / 8 heads, 357 to 390 us; a bf16 product of 8192^3 1205 to 1240), 575 to 605 at D 64 (4 prompts of 2048 x 16 heads, 57 to 60 us).
#pragma once
#include <algorithm>

#include "cache8.h"
#include "paged_few_impl.h"

namespace fs {

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <typename T> __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c);
template <> __device__ __forceinline__ f32x16 mfma32<f16_t>(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 mfma32<bf16_t>(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <class Op> __device__ __forceinline__ float halves_allreduce(float v) {
  const uint32_t u = as_u32(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return Op::apply(as_f32(r[0]), as_f32(r[1]));
}

// What a workgroup of the tile kernel has: a tile of 128 rows, all of its keys or a part of them.
struct TileWork {
  int lane, b, head, tile;      // the lane that has the request (of a line), the request
  PagedRequest r;
  int rows, row0, key_first, steps;      // of the request, of the tile: steps of 64 keys
  int parts, part, partial;              // parts that the keys are split into, this one, and its place among the partial results
};

// The order of the work, made by every wavefront for itself from the lengths on the device, up to 64 requests of many rows one to a lane.  A tile's
// time goes with its steps, which differ up to the whole length of the longest request, and workgroups start in order as others end.
// So: the tiles of more steps than an even share of all work, that of few rows with it (63 requests of one token behind 2000 keys and one
// of 1000: 119 us, 155 where shares are of the tiles alone; 400 behind 200 and four of 256 behind 1744: 147, 162 where steps of short requests get lost), are split into parts of at most that and come first; the
// others follow by falling steps.  Steps do not fall along a request's tiles, so how many of them have at least s is a
// formula, and the k-th tile is found by bisection over s.  (Chunks of 1 to 1024 tokens behind contexts of up to 12000: the longest tile alone is 1.2
// times the even share; request by request the launch took 1.48 times it.)  A share is 1.25 times a 512th, so that parts of one length do
// not come out one more than places (512 tokens behind 7680: 99 us, 116 with 1.5, which makes 384 parts; 32768: 319 and 379).
struct TileLine {
  const PagedArgs& a;
  PagedRequest mine{};
  int id = 0;                                // the lane's request
  int tiles = 0, flat = -1;      // of the lane's request; with a window, or without the causal mask: steps of each of its tiles, as good as equal
  int share_steps = 0;           // an even share
  int split = 0, parts = 1;      // the lane's tiles of more steps than that (its last ones), and the parts of each
  int items = 0;                 // parts of all
  int64_t others = 0;            // steps of requests of few rows that the lane looked at, over all key heads

  __device__ __forceinline__ explicit TileLine(const PagedArgs& args) : a(args) {}
  __device__ __forceinline__ PagedRequest request(int b) const { return b < a.requests ? paged_request(a, b) : PagedRequest{}; }
  // those of many rows among up to kTileRequests, one a lane; false: there are more than 64
  __device__ __forceinline__ bool gather() {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int b0 = 0; b0 < a.requests; b0 += 256) {
      PagedRequest r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = request(b0 + 64 * i + lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        look(r[i]);
        const uint64_t many = __ballot(r[i].fresh * a.share > a.few_rows), below = (1ull << lane) - 1;
        if (!many) continue;
        const int here = __popcll(many);
        if (n + here > 64) return false;
        // the lanes that have one go behind those that are there, the others behind them
        const int to = n + (many >> lane & 1 ? __popcll(many & below) : here + __popcll(~many & below)) & 63;
        const int b = __builtin_amdgcn_ds_permute(4 * to, b0 + 64 * i + lane), first = __builtin_amdgcn_ds_permute(4 * to, r[i].first);
        const int fresh = __builtin_amdgcn_ds_permute(4 * to, r[i].fresh), keys = __builtin_amdgcn_ds_permute(4 * to, r[i].keys);
        if (lane >= n && lane < n + here) { id = b; mine = PagedRequest{first, fresh, keys}; }
        n += here;
      }
    }
    return true;
  }
  // 64 keys of a tile of few rows, which memory bounds, take a place on a CU as long as a step of 128 rows
  __device__ __forceinline__ void look(const PagedRequest& r) {
    const int rows = r.fresh * a.share;
    if (rows > 0 && rows <= a.few_rows) others += (int64_t)((r.keys - paged_first_key(a, r) + 63) >> 6) * a.kv_heads;
  }
  __device__ __forceinline__ void measure() {
    const int rows = mine.fresh * a.share;
    tiles = rows > a.few_rows ? (rows + 127) >> 7 : 0;
    flat = -1;
    if (!a.causal) flat = (mine.keys + 63) >> 6;
    else if (a.window && a.window < mine.keys) flat = (int)(((int64_t)a.window + 126 + 128 / a.share) >> 6);
  }
  // tiles of the lane's request with at least s steps: a tile's last token t has ceil((keys - fresh + 1 + t) / 64)
  __device__ __forceinline__ int at_least(int s) const {
    if (s <= 0) return tiles;
    if (s > (1 << 24) + 8) return 0;      // (2^30 keys are no more steps, and s times 64 would leave 32 bits)
    if (flat >= 0) return flat >= s ? tiles : 0;
    const int token = __builtin_elementwise_sub_sat((s - 1) << 6, mine.keys - mine.fresh);      // the first such token
    return token >= mine.fresh ? 0 : tiles - (max(token, 0) * a.share >> 7);
  }
  __device__ __forceinline__ int last_steps() const { return tiles == 0 ? 0 : flat >= 0 ? flat : (mine.keys + 63) >> 6; }
  // false: more than 64 requests of many rows, or of any more than the line looks at
  __device__ __forceinline__ bool order() {
    if (a.requests <= 64) {
      id = threadIdx.x & 63;
      mine = request(id);
      look(mine);
    } else if (a.requests > kTileRequests || !gather()) {
      return false;
    }
    measure();
    const int last = last_steps(), first = flat >= 0 || tiles == 0 ? last : max(0, mine.keys - mine.fresh + 64) >> 6;
    // in 64 steps, no more than 2^31 of them; what the lanes have beside whole 64s is summed up too (500 requests of seven steps and eight heads
    // are 28000 steps, none of which is 64 of one request)
    const int64_t halves = 2 * others + (int64_t)tiles * (first + last) * a.kv_heads;      // of steps
    const int total = wave_sum((int)min(halves >> 7, (int64_t)1 << 24)) + (wave_sum((int)(halves & 127)) >> 7);
    share_steps = min(1 << 23, max(kLeastSteps, (total + total / 4) / (kTileShares / 64)));      // (a tile has up to 2^24)
    for (;; share_steps *= 2) {      // (never more parts than there is room for)
      split = at_least(share_steps + 1);
      parts = split ? (last + share_steps - 1) / share_steps : 1;
      items = wave_sum((int)min((int64_t)split * parts * a.kv_heads, (int64_t)1 << 24));
      if (items <= 2 * kTileShares) return true;
    }
  }
  // the lane among whose `count` the number k falls, k counted from there on
  static __device__ __forceinline__ int among(int count, int* k) {
    const int upto = wave_upto(count);
    const int lane = min(63, (int)__popcll(__ballot(upto <= *k)));
    *k -= __builtin_amdgcn_readlane(upto, lane) - __builtin_amdgcn_readlane(count, lane);
    return lane;
  }
  __device__ __forceinline__ void fill(TileWork* t, int lane) const {
    t->lane = lane;
    t->b = __builtin_amdgcn_readlane(id, lane);
    t->r = PagedRequest{__builtin_amdgcn_readlane(mine.first, lane), __builtin_amdgcn_readlane(mine.fresh, lane), __builtin_amdgcn_readlane(mine.keys, lane)};
    t->rows = t->r.fresh * a.share;
    t->row0 = t->tile * 128;
    const int t1 = (min(t->row0 + 128, t->rows) - 1) / a.share, t0 = t->row0 / a.share, back = t->r.keys - t->r.fresh + 1;
    const int until = max(0, a.causal ? min(t->r.keys, back + t1) : t->r.keys);
    t->key_first = a.window ? min(max(0, back + t0 - a.window), until) & ~63 : 0;
    t->steps = (until - t->key_first + 63) >> 6;
  }
  // part k of the split tiles; `whole`: the k-th split tile instead, all of its parts
  __device__ __forceinline__ void find_split(int k, bool whole, TileWork* t) const {
    const int per = whole ? split * a.kv_heads : split * a.kv_heads * parts;
    int in = k;
    const int lane = among(per, &in);
    const int n = __builtin_amdgcn_readlane(split, lane) * a.kv_heads;      // tiles and heads of the request
    t->parts = __builtin_amdgcn_readlane(parts, lane);
    t->part = whole ? 0 : in / n;
    const int at = in - t->part * n;
    t->head = at % a.kv_heads;
    t->tile = __builtin_amdgcn_readlane(tiles, lane) - __builtin_amdgcn_readlane(split, lane) + at / a.kv_heads;
    int before = 0;      // parts of the requests before
    if (whole) {
      const int all = split * a.kv_heads * parts;
      before = wave_sum((int)(threadIdx.x & 63) < lane ? all : 0);
    }
    t->partial = whole ? before + at : k;
    fill(t, lane);
  }
  // the places of a tile's parts among the partial results are so far apart
  __device__ __forceinline__ int stride(const TileWork& t) const { return __builtin_amdgcn_readlane(split, t.lane) * a.kv_heads; }
  // the k-th of the tiles that are not split, by falling steps; false: there are not so many
  __device__ __forceinline__ bool find_whole(int k, TileWork* t) const {
    if (k >= wave_sum(tiles - split) * a.kv_heads) return false;
    // in eighths of an even share: tiles of about the same steps go request by request, whose keys the L2s then have (20 requests of 400
    // rows x 32 heads behind 3600 keys: 620 us, in the order of single steps 690)
    const int grain = max(1, share_steps >> 3);
    int lo = 0, hi = share_steps / grain + 1;      // more than k of at least lo eighths, no more than k of at least hi
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (wave_sum(max(0, at_least(mid * grain) - split)) * a.kv_heads > k) lo = mid; else hi = mid;
    }
    const int more = max(0, at_least(hi * grain) - split), here = at_least(lo * grain) - split - more;
    k -= wave_sum(more) * a.kv_heads;
    const int lane = among(here * a.kv_heads, &k);
    t->parts = 1; t->part = 0; t->partial = 0;
    t->head = k % a.kv_heads;
    t->tile = __builtin_amdgcn_readlane(tiles - split - more, lane) - 1 - k / a.kv_heads;
    fill(t, lane);
    return true;
  }
  // without a line: the tiles in the order of the rows, no one split
  __device__ __forceinline__ bool find_in_order(int k, TileWork* t) {
    const int at = a.slots - 1 - k / a.kv_heads, b = paged_find(a, at, 7);
    if (b < 0) return false;
    id = b;      // (the same in all lanes)
    mine = request(b);
    measure();
    t->tile = at - paged_place(a, b, 7);
    if (t->tile >= __builtin_amdgcn_readfirstlane(tiles)) return false;
    t->parts = 1; t->part = 0; t->partial = 0;
    t->head = k % a.kv_heads;
    fill(t, 0);
    return true;
  }
};

// 64 keys (or values) in LDS as the direct loads leave them: 16 keys to a wavefront's part, pieces of 64 bytes of them behind one
// another, [key / 16][64-byte piece][key % 16][4 x 16 bytes].  The 16 bytes x of a piece of key r stand in place x ^ (r / 4 % 4): eight lanes that
// read a 16-byte column, and the four rows of a transposing read, fall on different banks.
template <int D> struct TileLds {
  static constexpr int kPieces = D / 32, kKeys16 = 16 * D;      // halves of 16 keys
  uint16_t v[64 * D];
};

template <int D> struct TileShared {
  TileLds<D> k[2], v[2];
  uint32_t flags[2][4], odds[4];                            // which of a wavefront's 16 keys are there; whether a value of them is infinite or NaN
};

// A cache that holds numbers of the type itself, or one of the codes of 8 bits.
struct NoCode {};

// Workgroup k of the tile kernel.  Codes come into registers, 16 of a lane at a time, and go into LDS as numbers of T times their scales (powers of two: exactly), so that
// each is made once for four wavefronts; from there on both kinds are the same.
template <typename T, int D, class Code = NoCode> __device__ __forceinline__ void paged_tile(const PagedArgs& a, TileShared<D>& lds, int k) {
  constexpr bool kCodes = !__is_same(Code, NoCode);
  constexpr int KS = D / 16, DT = D / 32, CH = D / 32, K16 = 16 * D;
  auto &ksh = lds.k, &vsh = lds.v;
  auto& flags = lds.flags;
  auto& odds = lds.odds;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 31, h = lane >> 5;
  TileWork work;
  {
    TileLine line(a);
    if (!line.order()) {
      if (!line.find_in_order(k, &work)) return;
    } else {
      if (k < line.items) line.find_split(k, false, &work);
      else {
        // by turns forwards and backwards over 256 places, eight by eight (one to an XCD), so that what the CUs get one after the other adds up to
        // the same (prompts of 2048 rows x 16 heads of 64 60.8 -> 58.8 us)
        const int first = k & ~255, all = line.items + wave_sum(line.tiles - line.split) * a.kv_heads;
        if (first & 256 && first >= line.items && first + 256 <= all) k = first + (248 - (k & 248)) + (k & 7);
        if (!line.find_whole(k - line.items, &work)) return;
      }
    }
  }
  if (work.row0 < 0 || work.row0 >= work.rows) return;      // (requests whose rows overlap can be more tiles than 32 bits number)
  const PagedRequest r = work.r;
  const int head = work.head;
  // a part's steps: an even run of the tile's
  const int step0 = (int)((int64_t)work.steps * work.part / work.parts), steps = (int)((int64_t)work.steps * (work.part + 1) / work.parts) - step0;
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
    load_lds16<0, false>(kbase + at, kl);
    load_lds16<0, false>(vbase + at, vl);
    if constexpr (CH > 1) { load_lds16<1, false>(kbase + at, kl); load_lds16<1, false>(vbase + at, vl); }
    if constexpr (CH > 2) { load_lds16<2, false>(kbase + at, kl); load_lds16<2, false>(vbase + at, vl); }
    if constexpr (CH > 3) { load_lds16<3, false>(kbase + at, kl); load_lds16<3, false>(vbase + at, vl); }
    const uint64_t good = __ballot(ok);
    uint32_t flag = 0xffffu;
    if (good != ~0ull) {
      flag = 0;
      for (int k = 0; k < 16; ++k) flag |= (uint32_t)(good >> (4 * k) & 1) << k;
    }
    if (lane == 0) flags[buf][w] = flag;
  };

  // ---- staging of codes: four lanes to a key, lane q of them pieces q and q + 4 of 16 codes (where there are no such, one that another lane has too)
  constexpr int P = D / 16, PL = (P + 3) / 4;
  u32x4 kc[kCodes ? PL : 1], vc[kCodes ? PL : 1];
  float kscale = 0.f, vscale = 0.f;
  bool there_is = false;
  auto piece = [&](int i) { return (lane & (P - 4 * i >= 4 ? 3 : 1)) + 4 * i; };
  auto fetch = [&](int key0) __attribute__((always_inline)) {
    const int key = key0 + skey;
    there_is = key < key_last && (unsigned)block < (unsigned)a.cache.blocks;
    const int64_t at = (int64_t)head * a.cache.head + (int64_t)(there_is ? block : 0) * a.cache.block + (int64_t)(key & in_block) * a.cache.slot;
    const int64_t scale_at = (int64_t)(there_is ? block : 0) * a.kv_heads + head;
    const uint8_t *k8 = static_cast<const uint8_t*>(a.k) + at, *v8 = static_cast<const uint8_t*>(a.v) + at;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      kc[i] = *reinterpret_cast<const u32x4*>(k8 + 16 * piece(i));
      vc[i] = *reinterpret_cast<const u32x4*>(v8 + 16 * piece(i));
    }
    kscale = a.k_scales[scale_at];
    vscale = a.v_scales[scale_at];
  };
  auto put = [&](int buf, auto code) __attribute__((always_inline)) {
    typedef Numbers<decltype(code), T> Num;
    const bool even = __ballot(!Num::takes(kscale) || !Num::takes(vscale)) == 0;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      const int q = piece(i), at = w * K16 + 512 * (q / 2) + srow * 32, x = 2 * (q & 1), turn = srow >> 2 & 3;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const u32x4 c = v ? vc[i] : kc[i];
        const float scale = v ? vscale : kscale;
        const u32x2 c0 = {c[0], c[1]}, c1 = {c[2], c[3]};
        uint16_t* rows = (v ? vsh[buf].v : ksh[buf].v) + at;
        *reinterpret_cast<u32x4*>(rows + 8 * (x ^ turn)) = even ? Num::fast(c0, scale) : Num::rounded(c0, scale);
        *reinterpret_cast<u32x4*>(rows + 8 * ((x + 1) ^ turn)) = even ? Num::fast(c1, scale) : Num::rounded(c1, scale);
      }
    }
    const uint64_t good = __ballot(there_is);
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
      const float keep = m == -INFINITY ? 1.f : sum_factor((m - grown) * scale2);      // (of nothing but an infinity or NaN that was added: as it is)
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
    u32x4 pb[4];      // rounded to T for the second dot alone: half a step of each weight; their sum is of them unrounded
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
    if constexpr (kCodes) {
      fetch(key_first);
      request_block(key_first + 64);
      put(0, Code{});
      __syncthreads();
      for (int i = 0; i < steps; ++i) {
        const int key0 = key_first + 64 * i;
        if (i + 1 < steps) {
          fetch(key0 + 64);
          request_block(key0 + 128);
        }
        compute(key0, i & 1);
        if (i + 1 < steps) put((i + 1) & 1, Code{});
        __syncthreads();
      }
    } else {
      request_rows(key_first, 0);
      request_block(key_first + 64);
      wait_loads<0>();
      __syncthreads();
      for (int i = 0; i < steps; ++i) {
        const int key0 = key_first + 64 * i;
        if (i + 1 < steps) {
          request_rows(key0 + 64, (i + 1) & 1);
          request_block(key0 + 128);
        }
        compute(key0, i & 1);
        wait_loads<0>();
        __syncthreads();
      }
    }
  }
  l = halves_allreduce<SumOp>(l);
  const float top = m == -INFINITY ? -INFINITY : m * scale2;      // in units of log 2
  if (work.parts > 1) {
    float* at = a.tile_partial + (int64_t)work.partial * (128 * (D + 2));
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

// Tiles whose keys were split: workgroup b of `groups` joins every groups-th run of 4096 values of them, the parts in the order of the keys.
template <typename T, int D> __device__ __forceinline__ void paged_tile_join(const PagedArgs& a, int b, int groups) {
  TileLine line(a);
  if (!line.order()) return;
  const int runs = wave_sum(line.split) * a.kv_heads * (D / 32);
  for (; b < runs; b += groups) {
    const int k = b / (D / 32), run = b - k * (D / 32);
    TileWork work;
    line.find_split(k, true, &work);
    const int64_t stride = (int64_t)line.stride(work) * (128 * (D + 2));
    const float* at = a.tile_partial + (int64_t)work.partial * (128 * (D + 2));
    for (int i = threadIdx.x; i < 1024; i += blockDim.x) {
      const int e = (run * 1024 + i) * 4, mine = e / D, row = work.row0 + mine;
      if (row < 0 || row >= work.rows) continue;
      FewSum s{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
      auto part = [&](int n) { return at + n * stride; };
      int n = 0;
      for (; n + 4 <= work.parts; n += 4) few_add_parts<4, 128, D>(s, n, 1, part, mine, e);
      if (n + 2 <= work.parts) { few_add_parts<2, 128, D>(s, n, 1, part, mine, e); n += 2; }
      if (n < work.parts) few_add_parts<1, 128, D>(s, n, 1, part, mine, e);
      const int token = row / a.share, q_head = work.head * a.share + row - token * a.share;
      const float inv = s.l == 0.f ? 0.f : 1.f / s.l;
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + (int64_t)(work.r.first + token) * a.out_stride + (int64_t)q_head * D + e % D) =
          u32x2{Mfma<T>::pack(s.o[0] * inv, s.o[1] * inv), Mfma<T>::pack(s.o[2] * inv, s.o[3] * inv)};
      if (a.lse && e % D == 0) a.lse[(int64_t)(work.r.first + token) * a.q_heads + q_head] = s.l == 0.f ? -INFINITY : (s.m + __builtin_amdgcn_logf(s.l)) * 0.6931471805599453f;
    }
  }
}

// Requests of few rows and of many in one launch, and one that joins the parts of both: where there are none of one kind (whole prompts) it costs no
// launches of its own.  Those of few rows are numbered behind all tiles and begin as these run out, so that one kind reads memory while the other keeps
// the matrix unit busy at the tiles' end alone (512 tokens behind 32256 keys and 100 single ones behind 4095: 494 us, where the products take
// 226 and the reading 254; by turns of eight both ended up on shader engines of their own, chunks 378 -> 501).  Four workgroups to a CU up to head dim
// 64 (prompts of 2048 rows x 16 heads of 64: 60.5 us, 66.6 with three); beyond, two is what the LDS holds.
template <typename T, int D, int NT> __global__ __launch_bounds__(256, (D <= 64 && NT == 1 ? 4 : 2)) void paged_mixed_kernel(const PagedArgs a) {
  __shared__ __align__(1024) union { FewLds<D, NT, 4> few; TileShared<D> tile; } lds;
  const int tiles = gridDim.x - a.few_grid, b = blockIdx.x;
  if (b < tiles) paged_tile<T, D>(a, lds.tile, b);
  else paged_few<T, D, NT, 4>(a, lds.few, b - tiles);
}
template <typename T, int D, int NT> __global__ __launch_bounds__((FewJoin<D, NT>::kThreads)) void paged_mixed_join_kernel(const PagedArgs a) {
  // 256 workgroups for either kind: what there is to join is known on the device alone, mostly little
  if (blockIdx.x >= 256) {
    paged_tile_join<T, D>(a, blockIdx.x - 256, 256);
    return;
  }
  FewLine<NT> line(a);
  line.count();
  if (line.total == 0) return;
  const int log_groups = line.groups();
  for (int b = blockIdx.x; b < a.few_grid - (1 << a.log_heads); b += 256) {
    paged_few_join<T, D, NT>(a, line, log_groups, b);
    __syncthreads();
  }
}

inline unsigned paged_mixed_grid(const PagedArgs& a) {
  return (unsigned)(a.few_grid + std::max(a.few_grid, a.slots * a.kv_heads + (a.requests <= kTileRequests ? 2 * kTileShares : 0)));
}
template <typename T, int D, int NT> hipError_t paged_mixed_join_launch(const PagedArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((paged_mixed_join_kernel<T, D, NT>), dim3(a.requests <= kTileRequests ? 512 : 256), dim3(FewJoin<D, NT>::kThreads), 0, s, a);
  return hipGetLastError();
}
template <typename T, int D, int NT> hipError_t paged_mixed_launch(const PagedArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((paged_mixed_kernel<T, D, NT>), dim3(paged_mixed_grid(a)), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return paged_mixed_join_launch<T, D, NT>(a, s);
}

template <typename T, int D> hipError_t paged_mixed_launch_rows(const PagedArgs& a, int row_tiles, hipStream_t s) {
  return row_tiles == 1 ? paged_mixed_launch<T, D, 1>(a, s) : paged_mixed_launch<T, D, 2>(a, s);
}
template <typename T, int D> hipError_t paged_mixed_join_launch_rows(const PagedArgs& a, int row_tiles, hipStream_t s) {
  return row_tiles == 1 ? paged_mixed_join_launch<T, D, 1>(a, s) : paged_mixed_join_launch<T, D, 2>(a, s);
}
template <typename T> hipError_t paged_mixed_join_launch_type(const PagedArgs& a, int dim, int row_tiles, hipStream_t s) {
  switch (dim) {
    case 32: return paged_mixed_join_launch_rows<T, 32>(a, row_tiles, s);
    case 64: return paged_mixed_join_launch_rows<T, 64>(a, row_tiles, s);
    case 96: return paged_mixed_join_launch_rows<T, 96>(a, row_tiles, s);
    default: return paged_mixed_join_launch_rows<T, 128>(a, row_tiles, s);
  }
}
template <typename T> hipError_t paged_mixed_launch_type(const PagedArgs& a, int dim, int row_tiles, hipStream_t s) {
  switch (dim) {
    case 32: return paged_mixed_launch_rows<T, 32>(a, row_tiles, s);
    case 64: return paged_mixed_launch_rows<T, 64>(a, row_tiles, s);
    case 96: return paged_mixed_launch_rows<T, 96>(a, row_tiles, s);
    default: return paged_mixed_launch_rows<T, 128>(a, row_tiles, s);
  }
}

}  // namespace fs
