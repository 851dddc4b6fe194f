// Attention of new tokens over a paged cache (fs_plan_create_paged_attention): the choice of kernels and the launch.
#include <algorithm>

#include "paged_attn_impl.h"

namespace fs {

bool paged_attn_plan(PagedAttnSpec* s, int* n_kernels, int64_t* lds_bytes, std::string* err) {
  const fs_paged_attention_desc& d = s->d;
  const int64_t keys = (int64_t)d.table_blocks << s->cache.shift;
  if (keys > (1ll << 30)) { *err = "more than 2^30 keys in a row of the table"; return false; }
  const int64_t rows = (int64_t)(d.max_new ? std::min(d.max_new, d.tokens) : d.tokens) * s->share;      // of a request
  const bool many = rows > 32;
  // rows to a tile of the few-rows kernel: 16 where that is what a request has, else 32
  s->row_tiles = (many ? s->share : rows) <= 16 ? 1 : 2;
  s->few_rows = many ? 16 * s->row_tiles : 1 << 30;
  s->log_groups = 9;
  s->unit_keys = 128;
  // units are numbered in 31 bits
  const int64_t tiles = ((int64_t)d.tokens * s->share / (16 * s->row_tiles) + d.requests) * d.kv_heads;
  while (tiles * (keys / s->unit_keys + 1) > 0x7fffffffll) {
    if (s->unit_keys >= (1 << 29)) { *err = "too many rows"; return false; }
    s->unit_keys *= 2;
  }
  const int64_t m = 16 * s->row_tiles;
  s->few_bytes = d.tokens && d.requests ? (2ll << s->log_groups) * m * (d.head_dim + 2) * 4 : 0;
  s->partial_bytes = s->few_bytes;
  *n_kernels = 2;
  const int64_t pad = d.head_dim == 64 ? 8 : 16;
  *lds_bytes = std::max<int64_t>(4 * 32 * (d.head_dim + pad) * 2, 4 * m * (d.head_dim + 4) * 4) + 32 * m;
  s->slots = 0;
  s->most_parts = 1;
  s->least_steps = 8;
  if (many) {
    s->slots = ((int64_t)d.tokens * s->share >> 7) + d.requests;
    const int64_t wgs = s->slots * d.kv_heads;
    // few tiles: their keys are split too, to about two workgroups a CU
    s->most_parts = (int)std::max<int64_t>(1, std::min<int64_t>(512 / std::max<int64_t>(wgs, 1), (keys >> 6) / s->least_steps));
    if (wgs * s->most_parts > 0x7fffffffll) { *err = "too many tiles for one grid"; return false; }
    if (s->most_parts > 1 && s->partial_bytes) s->partial_bytes += wgs * s->most_parts * 128 * (d.head_dim + 2) * 4;
    *n_kernels = s->most_parts > 1 ? 4 : 3;
    *lds_bytes = std::max<int64_t>(*lds_bytes, 2ll * 64 * 2 * 2 * d.head_dim + 48);
  }
  return true;
}

std::string paged_attn_describe(const PagedAttnSpec& s) {
  char buf[320];
  int n = snprintf(buf, sizeof buf, "paged_attention[GRID,WARP,CTA] rows to a tile=%d, keys to a unit=%d; cta_num=%d, cta_size=256; join[GRID,CTA]", 16 * s.row_tiles, s.unit_keys, 1 << s.log_groups);
  if (s.slots) snprintf(buf + n, sizeof buf - n, "; requests of more than %d rows: rows to a tile=128, cta_num=%lld, parts=%d", s.few_rows, (long long)(s.slots * s.d.kv_heads * s.most_parts), s.most_parts);
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
  a.partial = static_cast<float*>(out[s.d.log_sum_exp ? 2 : 1]);
  a.requests = s.d.requests; a.tokens = s.d.tokens; a.q_heads = s.d.q_heads; a.kv_heads = s.d.kv_heads; a.share = s.share; a.causal = s.d.causal; a.window = s.d.window;
  a.width = s.d.blocks ? s.d.table_blocks : 0;      // (without a block there is no key to see, and no address to read)
  a.scale2 = (float)(s.d.scale * 1.4426950408889634);
  if (a.scale2 == 0.f) a.scale2 = 1.17549435e-38f;      // (what is not seen is -inf times the scale)
  a.unit_keys = s.unit_keys; a.log_groups = s.log_groups;
  hipStream_t st = static_cast<hipStream_t>(stream);
  a.few_rows = s.few_rows;
  a.tile_partial = a.partial + s.few_bytes / 4;
  a.slots = (int)s.slots; a.most_parts = s.most_parts; a.least_steps = s.least_steps;
  const bool f16 = s.d.dtype == FS_F16;
  hipError_t e = hipSuccess;
  if (s.slots) e = (f16 ? paged_tile_launch_f16 : paged_tile_launch_bf16)(a, s.d.head_dim, st);
  if (e == hipSuccess) e = (f16 ? paged_few_launch_f16 : paged_few_launch_bf16)(a, s.d.head_dim, s.row_tiles, st);
  if (e != hipSuccess) { *err = std::string("paged_attention launch: ") + hipGetErrorString(e); return -1; }
  return 0;
}

}  // namespace fs
