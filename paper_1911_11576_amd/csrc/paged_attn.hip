// Attention of new tokens over a paged cache (fs_plan_create_paged_attention): the choice of kernels and the launch.
#include <algorithm>

#include "paged_attn_impl.h"

namespace fs {

bool paged_attn_plan(PagedAttnSpec* s, int* n_kernels, int64_t* lds_bytes, std::string* err) {
  const fs_paged_attention_desc& d = s->d;
  const int64_t keys = (int64_t)d.table_blocks << s->cache.shift;
  if (keys > (1ll << 30)) { *err = "more than 2^30 keys in a row of the table"; return false; }
  // rows to a tile: 16 where that is what a request has, else 32
  const int64_t rows = (int64_t)(d.max_new ? std::min(d.max_new, d.tokens) : d.tokens) * s->share;
  s->row_tiles = rows <= 16 ? 1 : 2;
  s->log_groups = 9;
  s->unit_keys = 128;
  // units are numbered in 31 bits
  const int64_t tiles = ((int64_t)d.tokens * s->share / (16 * s->row_tiles) + d.requests) * d.kv_heads;
  while (tiles * (keys / s->unit_keys + 1) > 0x7fffffffll) {
    if (s->unit_keys >= (1 << 29)) { *err = "too many rows"; return false; }
    s->unit_keys *= 2;
  }
  const int64_t m = 16 * s->row_tiles;
  s->partial_bytes = d.tokens && d.requests ? (2ll << s->log_groups) * m * (d.head_dim + 2) * 4 : 0;
  *n_kernels = 2;
  const int64_t pad = d.head_dim == 64 ? 8 : 16;
  *lds_bytes = std::max<int64_t>(4 * 32 * (d.head_dim + pad) * 2, 4 * m * (d.head_dim + 4) * 4) + 32 * m;
  return true;
}

std::string paged_attn_describe(const PagedAttnSpec& s) {
  char buf[240];
  snprintf(buf, sizeof buf, "paged_attention[GRID,WARP,CTA] rows to a tile=%d, keys to a unit=%d; cta_num=%d, cta_size=256; join[GRID,CTA], partials=%lld", 16 * s.row_tiles, s.unit_keys,
           1 << s.log_groups, (long long)s.partial_bytes);
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
  a.unit_keys = s.unit_keys; a.log_groups = s.log_groups;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = (s.d.dtype == FS_F16 ? paged_few_launch_f16 : paged_few_launch_bf16)(a, s.d.head_dim, s.row_tiles, st);
  if (e != hipSuccess) { *err = std::string("paged_attention launch: ") + hipGetErrorString(e); return -1; }
  return 0;
}

}  // namespace fs
