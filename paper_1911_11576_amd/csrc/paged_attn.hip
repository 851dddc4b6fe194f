// Attention of new tokens over a paged cache (fs_plan_create_paged_attention): the choice of kernels and the launch.
#include <algorithm>

#include "paged_attn_impl.h"

namespace fs {

bool paged_attn_plan(PagedAttnSpec* s, int* n_kernels, int64_t* lds_bytes, std::string* err) {
  const fs_paged_attention_desc& d = s->d;
  const int64_t keys = (int64_t)d.table_blocks << s->cache.shift;
  if (keys > (1ll << 30)) { *err = "more than 2^30 keys in a row of the table"; return false; }
  const int64_t rows = (int64_t)(d.max_new ? std::min(d.max_new, d.tokens) : d.tokens) * s->share;      // of a request
  // Up to 32 rows are one tile of the kernel that reads each key once.  Beyond, tiles of 128 (D 128, 32 / 8 heads, 30 requests of 4000 keys: 36
  // rows 119 us, with two of these tiles 179; 32 rows 100, as a tile of 128 120; D 64, 16 / 16: 30 rows 90 and 106, 60 rows 167 and 107).
  // (max_new 0 counts all rows of the call as one request's: single tokens are done by the mixed launch then, 64 behind up to 24000 keys in 261 us instead of
  // 250, 48 behind up to 900 in 25.1 instead of 20.9, 256 behind up to 500 in 62.9 instead of 44.2)
  const bool many = rows > 32;
  // rows to a tile of the few-rows kernel: 16 where that is what a request has (64 of 4000 keys 168 us, 184 in tiles of 32), else 32
  s->row_tiles = (many ? s->share : rows) <= 16 ? 1 : 2;
  s->few_rows = many ? 16 * s->row_tiles : 1 << 30;
  const int64_t tiles = ((int64_t)d.tokens * s->share / (16 * s->row_tiles) + d.requests) * d.kv_heads;      // at most
  const int64_t m = 16 * s->row_tiles;
  int64_t waves = many ? 4 : 8;      // of a workgroup
  const bool any = d.tokens && d.requests;
  if (!many && keys <= 1024 && tiles <= 65536) {
    // No request is longer than four steps of 256 keys: a workgroup each tile, nothing to join (32 / 8 heads of 128: 8 requests of 100 keys 7.0 us, in
    // equal runs 9.6; of 500 10.8 and 12.9; of 1000 14.6 and 13.9; 64 of 1000 43.7 and 48.3; with 4096 one of 2000 would take 25.5 and 13.6).
    s->log_groups = -1;
    s->unit_keys = 1024;
    s->few_grid = (int)tiles;
    if (tiles > 256) waves = 4;
  } else {
    // as many wavefronts as the chip holds, eight to a CU
    s->log_groups = many ? 9 : 8;
    s->few_grid = 1 << s->log_groups;
    s->unit_keys = 32 * (int)waves;
    // units are numbered in 31 bits
    while (tiles * (keys / s->unit_keys + 1) > 0x7fffffffll) {
      if (s->unit_keys >= (1 << 29)) { *err = "too many rows"; return false; }
      s->unit_keys *= 2;
    }
    // Sets of key heads.  Where a head's rows of a block follow one another: as large a power of two as divides the heads, up to the CUs of an XCD (64
    // requests of up to 24000 keys, 32 / 8 heads of 128: 345 us, 355 with sets of two, 361 without sets and neighbours).
    // Where heads lie side by side and share lines of 128 bytes: two (64 of 16000, 16 / 8 heads of 32: 209 us, 226 with eight, 323 without; 24 / 4 of
    // 96, 8000: 143 and 160).  Where they lie side by side in whole lines: none (256 of 4000, 32 / 8 of 128: 628 us, 676 with eight; 32 of 8000, 16 / 16 of 64: 170
    // and 195; one of 131072 alone gains, 97 -> 94).
    const int most = s->cache.slot < s->cache.head ? 5 : s->cache.head % 64 ? 1 : 0;
    s->log_heads = std::min(most, __builtin_ctz((unsigned)d.kv_heads));
    s->neighbours = most > 0;
    if (any) s->few_bytes = (2ll << s->log_groups) * m * (d.head_dim + 2) * 4;
  }
  s->partial_bytes = s->few_bytes;
  *n_kernels = s->log_groups < 0 ? 1 : 2;
  *lds_bytes = std::max<int64_t>(waves * 128 * d.head_dim, waves * m * (d.head_dim + 4) * 4) + waves * (512 + 8 * m);
  if (many) {
    s->slots = ((int64_t)d.tokens * s->share >> 7) + d.requests;
    if (s->slots * d.kv_heads > (1 << 24) - 2048) {      // (a grid has less than 2^32 threads)
      *err = "too many tiles for one grid"; return false; }
    if (any && d.requests <= kTileRequests) s->partial_bytes += 2ll * kTileShares * 128 * (d.head_dim + 2) * 4;
    *lds_bytes = std::max<int64_t>(*lds_bytes, 512 * d.head_dim + 48);
  }
  return true;
}

std::string paged_attn_describe(const PagedAttnSpec& s) {
  char buf[320];
  int n = snprintf(buf, sizeof buf, "paged_attention[GRID,WARP,CTA] rows to a tile=%d, keys to a unit=%d; cta_num=%d, cta_size=%d%s", 16 * s.row_tiles, s.unit_keys, s.few_grid, s.slots || (s.log_groups < 0 && s.few_grid > 256) ? 256 : 512,
                   s.log_groups < 0 ? "" : "; join[GRID,CTA]");
  if (s.slots) snprintf(buf + n, sizeof buf - n, "; requests of more than %d rows: rows to a tile=128, cta_num=%lld", s.few_rows, (long long)(s.slots * s.d.kv_heads));
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
  if (s.partial_bytes) a.partial = static_cast<float*>(out[s.d.log_sum_exp ? 2 : 1]);
  a.requests = s.d.requests; a.tokens = s.d.tokens; a.q_heads = s.d.q_heads; a.kv_heads = s.d.kv_heads; a.share = s.share; a.causal = s.d.causal; a.window = std::min(s.d.window, 1 << 30);      // (no request has more keys)
  a.width = s.d.blocks ? s.d.table_blocks : 0;      // (without a block there is no key to see, and no address to read)
  a.scale2 = (float)(s.d.scale * 1.4426950408889634);
  if (a.scale2 == 0.f) a.scale2 = 1.17549435e-38f;      // (what is not seen is -inf times the scale)
  a.unit_keys = s.unit_keys; a.log_groups = s.log_groups; a.few_grid = s.few_grid;
  hipStream_t st = static_cast<hipStream_t>(stream);
  a.few_rows = s.few_rows;
  a.log_heads = s.log_heads; a.neighbours = s.neighbours;
  a.head_sets = s.d.kv_heads >> a.log_heads;
  if (s.partial_bytes) a.tile_partial = a.partial + s.few_bytes / 4;
  a.slots = (int)s.slots;
  const bool f16 = s.d.dtype == FS_F16;
  const hipError_t e = s.slots ? (f16 ? paged_mixed_launch_f16 : paged_mixed_launch_bf16)(a, s.d.head_dim, s.row_tiles, st)
                               : (f16 ? paged_few_launch_f16 : paged_few_launch_bf16)(a, s.d.head_dim, s.row_tiles, st);
  if (e != hipSuccess) { *err = std::string("paged_attention launch: ") + hipGetErrorString(e); return -1; }
  return 0;
}

}  // namespace fs
