// The C entry points of the operators around a paged cache (fs.h): arguments checked, geometry fixed, the plan's buffers
// listed for the check of every launch.  Host work alone.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <memory>
#include <new>

#include "paged.h"
#include "plan.h"

namespace {

using fs::CacheLayout;
using fs::set_error;

constexpr int64_t kMostTokens = 1ll << 30, kMostKeys = 0x7fffffffll;

int64_t size_of(int dtype) { return dtype == FS_F32 ? 4 : 2; }

fs_status invalid(const char* what, const std::string& why) { return set_error(FS_ERR_INVALID, std::string(what) + ": " + why); }

// block_size = 1 << *shift, and as many slots as 31 bits number
bool blocks_fit(int64_t blocks, int64_t block_size, int* shift, std::string* err) {
  if (block_size < 1 || block_size > 1024 || (block_size & (block_size - 1))) { *err = "block_size must be a power of two from 1 to 1024"; return false; }
  *shift = __builtin_ctzll((unsigned long long)block_size);
  if (blocks * block_size > kMostKeys) { *err = "more than 2^31 - 1 tokens in blocks"; return false; }
  return true;
}

// The cache's layout from the three strides (all 0: dense).  Rows of one cache must not overlap: sorted by stride, every
// dimension steps over all that the smaller ones cover.  *bytes: from its first element to behind its last.
bool cache_layout(int64_t blocks, int64_t heads, int64_t block_size, int64_t dim, int64_t sb, int64_t sh, int64_t ss, int64_t esize, CacheLayout* c, int64_t* bytes,
                  std::string* err) {
  if (sb < 0 || sh < 0 || ss < 0) { *err = "negative stride of the cache"; return false; }
  if (!sb && !sh && !ss) { ss = dim; sh = block_size * dim; sb = heads * sh; }
  int64_t stride[3] = {sb, sh, ss}, extent[3] = {blocks, heads, block_size};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j + 1 < 3; ++j)
      if (stride[j] > stride[j + 1]) { std::swap(stride[j], stride[j + 1]); std::swap(extent[j], extent[j + 1]); }
  __int128 covered = dim;
  for (int i = 0; i < 3; ++i) {
    if (extent[i] <= 1) continue;
    if (stride[i] < covered) { *err = "rows of the cache overlap (strides smaller than what they step over)"; return false; }
    covered += (__int128)stride[i] * (extent[i] - 1);
  }
  if (covered * esize > ((__int128)1 << 62)) { *err = "cache too large"; return false; }
  c->block = sb; c->head = sh; c->slot = ss; c->blocks = (int)blocks;
  *bytes = blocks ? (int64_t)covered * esize : 0;
  return true;
}

// A stride from token to token (0: dense) over heads x dim elements.
bool token_stride(int64_t* stride, int64_t heads, int64_t dim, const char* name, std::string* err) {
  if (!*stride) *stride = heads * dim;
  if (*stride < heads * dim || *stride > (1ll << 40)) { *err = std::string(name) + " is smaller than a token's heads, or beyond 2^40"; return false; }
  return true;
}

// bytes from the first element to behind the last of `tokens` rows
int64_t rows_bytes(int64_t tokens, int64_t stride, int64_t row, int64_t esize) { return tokens && row ? ((tokens - 1) * stride + row) * esize : 0; }

std::string numbers(const char* format, long long a, long long b = 0, long long c = 0, long long d = 0, long long e = 0, long long f = 0) {
  char buf[256];
  snprintf(buf, sizeof buf, format, a, b, c, d, e, f);
  return buf;
}

// The plan that `build` fills in; what it throws becomes a status.
template <class Build> fs_status create(fs_plan** out, const char* what, Build build) {
  if (!out) return set_error(FS_ERR_INVALID, "out is NULL");
  *out = nullptr;
  try {
    std::unique_ptr<fs_plan> p(new fs_plan);
    std::string err;
    int status = FS_ERR_INVALID;
    if (!build(p.get(), &status, &err)) return set_error((fs_status)status, std::string(what) + ": " + err);
    p->mode = FS_MODE_STITCHED;
    p->schedule = p->paged.kind;
    p->moved_bytes = p->paged.bytes;
    *out = p.release();
  } catch (const std::bad_alloc&) {
    return set_error(FS_ERR_NOMEM, "out of host memory");
  } catch (...) {
    return set_error(FS_ERR_INVALID, "internal error while planning");
  }
  return FS_OK;
}

bool known_code(int code) { return code == FS_CODE_E4M3 || code == FS_CODE_INT8; }

// What the kernels of a cache in 8 bits take: four neighbouring keys in one block, rows on 16 bytes.
bool codes_fit(const CacheLayout& c, int64_t block_size, std::string* err) {
  if (block_size < 8) { *err = "block_size must be at least 8"; return false; }
  for (int64_t n : {c.block, c.head, c.slot})
    if (n % 16) { *err = "strides of the cache must be multiples of 16 codes"; return false; }
  return true;
}

// Attention over a cache of numbers of the type (code -1) or of codes of 8 bits.
fs_status create_attention(const char* what, const fs_paged_attention_desc& desc, int code, int64_t* partial_bytes, fs_plan** out) {
  if (!partial_bytes) return invalid(what, "partial_bytes is NULL");
  *partial_bytes = 0;
  return create(out, what, [&](fs_plan* p, int* status, std::string* err) {
    fs::PagedAttnSpec& s = p->paged.attn;
    s.d = desc;
    s.code = code;
    fs_paged_attention_desc& d = s.d;
    const bool coded = code >= 0;
    const int64_t e = coded ? 1 : 2;      // bytes of the cache's elements
    if (d.reserved) { *err = "reserved must be 0"; return false; }
    if (d.dtype != FS_F32 && d.dtype != FS_F16 && d.dtype != FS_BF16) { *err = "unknown dtype"; return false; }
    if (d.requests < 0 || d.requests > 65536) { *err = "requests out of range [0,65536]"; return false; }
    if (d.q_heads < 1 || d.kv_heads < 1 || d.q_heads % d.kv_heads || d.q_heads > 65536) { *err = "q_heads must be a multiple of kv_heads, both above 0 and up to 65536"; return false; }
    if (d.tokens < 0 || (int64_t)d.tokens * d.q_heads > kMostTokens) { *err = "tokens below 0, or tokens * q_heads beyond 2^30"; return false; }
    if (d.head_dim < 1) { *err = "head_dim must be above 0"; return false; }
    if (d.blocks < 0 || d.table_blocks < 0) { *err = "negative number of blocks"; return false; }
    if (!blocks_fit(d.blocks, d.block_size, &s.cache.shift, err) || !blocks_fit(d.table_blocks, d.block_size, &s.cache.shift, err)) return false;
    if ((d.causal | 1) != 1 || (d.log_sum_exp | 1) != 1) { *err = "causal and log_sum_exp are 0 or 1"; return false; }
    if (d.window < 0 || (d.window && !d.causal)) { *err = "window below 0, or without causal"; return false; }
    if (d.max_new < 0) { *err = "max_new below 0"; return false; }
    if (!std::isfinite((float)(d.scale * 1.4426950408889634))) { *err = "scale must be finite in fp32"; return false; }
    const int64_t t = d.tokens, dim = d.head_dim, row = d.q_heads * dim;
    if (!token_stride(&d.q_stride, d.q_heads, dim, "q_stride", err) || !token_stride(&d.out_stride, d.q_heads, dim, "out_stride", err)) return false;
    int64_t cache_bytes = 0;
    const int shift = s.cache.shift;
    if (!cache_layout(d.blocks, d.kv_heads, d.block_size, dim, d.block_stride, d.head_stride, d.slot_stride, e, &s.cache, &cache_bytes, err)) return false;
    s.cache.shift = shift;
    *status = FS_ERR_UNSUPPORTED;
    if (d.dtype == FS_F32) { *err = "f16 and bf16 alone"; return false; }
    if (dim != 32 && dim != 64 && dim != 96 && dim != 128) { *err = "head_dim must be 32, 64, 96 or 128"; return false; }
    for (int64_t n : {d.q_stride, d.out_stride, s.cache.block, s.cache.head, s.cache.slot})
      if (n % 8) { *err = "strides must be multiples of 8 elements"; return false; }
    if (coded && !codes_fit(s.cache, d.block_size, err)) return false;
    s.share = d.q_heads / d.kv_heads;
    if (!fs::paged_attn_plan(&s, &p->n_kernels, &p->lds_bytes, err)) return false;
    fs::PagedPlan& g = p->paged;
    const int64_t b = t ? d.requests : 0;        // (no rows: nothing is launched)
    const bool cached = t && d.requests;
    const int64_t scales = 4ll * d.blocks * d.kv_heads;
    g.kind = coded ? FS_SCHED_PAGED_ATTENTION8 : FS_SCHED_PAGED_ATTENTION;
    g.in = {{"q", rows_bytes(t, d.q_stride, row, 2), -1}, {"k_cache", cached ? cache_bytes : 0, -1}, {"v_cache", cached ? cache_bytes : 0, -1}};
    if (coded) {
      g.in.push_back({"k_scales", cached ? scales : 0, -1});
      g.in.push_back({"v_scales", cached ? scales : 0, -1});
    }
    g.in.push_back({"tables", 4 * b * d.table_blocks, -1});
    g.in.push_back({"lengths", 4 * b, -1});
    g.in.push_back({"starts", b ? 4 * (b + 1) : 0, -1});
    g.out = {{"out", rows_bytes(t, d.out_stride, row, 2), -1}};
    if (d.log_sum_exp) g.out.push_back({"lse", 4 * t * d.q_heads, -1});
    if (s.partial_bytes) g.out.push_back({"partials", s.partial_bytes, -1});
    const int64_t keys = std::min<int64_t>((int64_t)d.requests * d.table_blocks * d.block_size, (int64_t)d.blocks * d.block_size);
    g.bytes = 4 * t * row + 2 * e * keys * d.kv_heads * dim + (coded ? 8 * (keys >> shift) * d.kv_heads : 0) + 4ll * d.requests * (d.table_blocks + 2) + (d.log_sum_exp ? 4 * t * d.q_heads : 0);
    p->description = fs::paged_attn_describe(s);
    *partial_bytes = s.partial_bytes;
    return true;
  });
}

// The store into a cache in 8 bits, and the reading back.
fs_status create_cache8(const char* what, const fs_cache8_desc* desc, bool store, fs_plan** out) {
  if (out) *out = nullptr;
  if (!desc) return invalid(what, "desc is NULL");
  return create(out, what, [&](fs_plan* p, int* status, std::string* err) {
    fs::Cache8Spec& s = p->paged.cache8;
    s.d = *desc;
    fs_cache8_desc& d = s.d;
    if (d.reserved) { *err = "reserved must be 0"; return false; }
    if (d.dtype != FS_F32 && d.dtype != FS_F16 && d.dtype != FS_BF16) { *err = "unknown dtype"; return false; }
    if (!known_code(d.code)) { *err = "unknown code"; return false; }
    if (d.requests < 0 || d.requests > 65536) { *err = "requests out of range [0,65536]"; return false; }
    if (d.tokens < 0 || d.tokens > kMostTokens) { *err = "tokens out of range [0,2^30]"; return false; }
    if (d.kv_heads < 1 || d.kv_heads > 65536) { *err = "kv_heads out of range [1,65536]"; return false; }
    if (d.head_dim < 1) { *err = "head_dim must be above 0"; return false; }
    if (d.blocks < 0 || d.table_blocks < 0) { *err = "negative number of blocks"; return false; }
    if (!blocks_fit(d.blocks, d.block_size, &s.cache.shift, err) || !blocks_fit(d.table_blocks, d.block_size, &s.cache.shift, err)) return false;
    const int64_t t = d.tokens, dim = d.head_dim, row = d.kv_heads * dim, e = size_of(d.dtype);
    if (!token_stride(&d.k_stride, d.kv_heads, dim, "k_stride", err) || !token_stride(&d.v_stride, d.kv_heads, dim, "v_stride", err)) return false;
    int64_t cache_bytes = 0;
    const int shift = s.cache.shift;
    if (!cache_layout(d.blocks, d.kv_heads, d.block_size, dim, d.block_stride, d.head_stride, d.slot_stride, 1, &s.cache, &cache_bytes, err)) return false;
    s.cache.shift = shift;
    *status = FS_ERR_UNSUPPORTED;
    if (dim % 16 || dim > 512) { *err = "head_dim must be a multiple of 16 up to 512"; return false; }
    if (d.k_stride * e % 16 || d.v_stride * e % 16) { *err = "rows of k and v must lie on 16 bytes"; return false; }
    if (d.k_stride > (1 << 22) || d.v_stride > (1 << 22)) { *err = "k_stride or v_stride beyond 2^22"; return false; }
    if (!codes_fit(s.cache, d.block_size, err)) return false;
    fs::cache8_geometry(&s, store);
    fs::PagedPlan& g = p->paged;
    const int64_t b = t ? d.requests : 0;        // (no rows: nothing is launched)
    const bool any = t && d.requests;
    const int64_t scales = 4ll * d.blocks * d.kv_heads;
    g.kind = store ? FS_SCHED_CACHE_STORE8 : FS_SCHED_CACHE_READ8;
    const std::vector<fs::PagedBuffer> rows = {{"k", any ? rows_bytes(t, d.k_stride, row, e) : 0, -1}, {"v", any ? rows_bytes(t, d.v_stride, row, e) : 0, -1}};
    const std::vector<fs::PagedBuffer> cache = {{"k_cache", any ? cache_bytes : 0, -1}, {"v_cache", any ? cache_bytes : 0, -1}, {"k_scales", any ? scales : 0, -1}, {"v_scales", any ? scales : 0, -1}};
    g.in = store ? rows : cache;
    g.in.push_back({"tables", 4 * b * d.table_blocks, -1});
    g.in.push_back({"lengths", 4 * b, -1});
    g.in.push_back({"starts", b ? 4 * (b + 1) : 0, -1});
    g.out = store ? cache : rows;
    const int64_t touched = std::min<int64_t>((t >> shift) + 2 * b, d.blocks);
    g.bytes = 2 * t * row * (e + 1) + 8 * touched * d.kv_heads + 4 * (2 * b + touched);
    if (store && s.waves > 1) p->lds_bytes = 16;      // a maximum of each
    p->description = store ? numbers("cache_store8[GRID-CTA,WARP] wavefronts to a block and head=%lld; cta_num=%lld, cta_size=256", s.waves, 8ll * s.grid_groups * s.grid)
                           : numbers("cache_read8[GRID-CTA,THREAD] rows=%lld; cta_num=%lld, cta_size=256", s.groups, s.grid);
    return true;
  });
}

}  // namespace

extern "C" {

fs_status fs_plan_create_block_tables(const fs_block_tables_desc* desc, fs_plan** out) {
  const char* what = "fs_plan_create_block_tables";
  if (out) *out = nullptr;
  if (!desc) return invalid(what, "desc is NULL");
  return create(out, what, [&](fs_plan* p, int*, std::string* err) {
    const fs_block_tables_desc& d = *desc;
    int shift;
    if (d.requests < 0 || d.requests > 4096) { *err = "requests out of range [0,4096]"; return false; }
    if (d.tokens < 0 || d.tokens > kMostTokens) { *err = "tokens out of range [0,2^30]"; return false; }
    if (d.blocks < 0 || d.free_blocks < 0 || d.table_blocks < 0) { *err = "negative number of blocks"; return false; }
    if (!blocks_fit(d.blocks, d.block_size, &shift, err) || !blocks_fit(d.table_blocks, d.block_size, &shift, err)) return false;
    fs::BlockTablesSpec& s = p->paged.tables;
    s.d = d;
    // Every workgroup scans all requests for itself and serves a row a thread.  One wavefront for a decode step (the kernel of 48 requests
    // 2.2 us, of 256 threads 2.4); else a thread a request, in as small a workgroup as has so many (256 requests, 32768 rows: 3.5 us, of 1024
    // threads 4.5; 515 requests: 4.6, of 256 threads, with three requests and two rows each, 5.7), and beyond 1024 four.
    s.wg = d.requests <= 64 && d.tokens <= 64 ? 64 : d.requests <= 256 ? 256 : 1024;
    s.grid = (int)std::min<int64_t>(std::max<int64_t>(1, ((int64_t)d.tokens + s.wg - 1) / s.wg), 2048);
    s.lds = 12ll * (d.requests + 1) + 64;
    p->lds_bytes = s.lds;
    const int64_t b = d.requests, t = d.tokens;
    p->paged.kind = FS_SCHED_BLOCK_TABLES;
    p->paged.in = {{"cached", 4 * b, -1}, {"fresh", 4 * b, -1}, {"free", 4ll * d.free_blocks, -1}};
    p->paged.out = {{"tables", 4 * b * d.table_blocks, -1}, {"lengths", 4 * b, -1}, {"starts", 4 * (b + 1), -1}, {"positions", 4 * t, -1}, {"slots", 4 * t, -1}, {"taken", 8, -1}};
    p->paged.bytes = 8 * b + 4 * (2 * b + 1) + 8 * t + 8 + 8 * ((t >> shift) + b);
    p->description = numbers("block_tables[GRID-CTA] requests=%lld, tokens=%lld, block_size=%lld; cta_num=%lld, cta_size=%lld, lds=%lld", b, t, d.block_size, s.grid, s.wg, s.lds);
    return true;
  });
}

fs_status fs_rotary_frequencies(int32_t rotary_dim, double base, double factor, double low, double high, double original, double* out) {
  const char* what = "fs_rotary_frequencies";
  if (!out || rotary_dim < 2 || (rotary_dim & 1)) return invalid(what, "out is NULL, or rotary_dim not even and above 0");
  const bool blend = low != 0 || high != 0;
  if (!(base > 0) || !std::isfinite(base) || !(factor >= 1) || !std::isfinite(factor)) return invalid(what, "base must be above 0 and factor at least 1");
  if (blend && (!(low > 0) || !(high > low) || !std::isfinite(high) || !(original > 0) || !std::isfinite(original)))
    return invalid(what, "0 < low < high and original above 0, or low and high both 0");
  for (int i = 0; i < rotary_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / rotary_dim);
    double keep = 0;      // the share of the frequency as it is
    if (blend) keep = std::fmin(1.0, std::fmax(0.0, (original * f / 6.283185307179586476925 - low) / (high - low)));
    out[i] = (1 - keep) * (f / factor) + keep * f;
  }
  return FS_OK;
}

fs_status fs_plan_create_rotary(const fs_rotary_desc* desc, fs_plan** out) {
  const char* what = "fs_plan_create_rotary";
  if (out) *out = nullptr;
  if (!desc) return invalid(what, "desc is NULL");
  return create(out, what, [&](fs_plan* p, int*, std::string* err) {
    fs::RotarySpec& s = p->paged.rotary;
    s.d = *desc;
    fs_rotary_desc& d = s.d;
    const bool store = d.blocks > 0;
    if (d.dtype != FS_F32 && d.dtype != FS_F16 && d.dtype != FS_BF16) { *err = "unknown dtype"; return false; }
    if (d.tokens < 0 || d.tokens > kMostTokens) { *err = "tokens out of range [0,2^30]"; return false; }
    if (d.q_heads < 1 || d.k_heads < 0 || d.q_heads > 65536 || d.k_heads > 65536) { *err = "q_heads out of range [1,65536], or k_heads out of [0,65536]"; return false; }
    if (d.head_dim < 2 || d.head_dim > 512 || (d.head_dim & 1)) { *err = "head_dim must be even, 2 to 512"; return false; }
    if (d.rotary_dim < 2 || d.rotary_dim > d.head_dim || (d.rotary_dim & 1)) { *err = "rotary_dim must be even, 2 to head_dim"; return false; }
    if ((d.interleaved | 1) != 1 || (d.inverse | 1) != 1) { *err = "interleaved and inverse are 0 or 1"; return false; }
    if (!std::isfinite(d.magnitude) || !std::isfinite((float)d.magnitude)) { *err = "magnitude must be finite in fp32"; return false; }
    if (d.blocks < 0) { *err = "negative number of blocks"; return false; }
    if (store && d.k_heads == 0) { *err = "a cache needs k_heads"; return false; }
    if (!store && (d.block_size || d.v_stride || d.block_stride || d.head_stride || d.slot_stride)) { *err = "fields of a cache without blocks"; return false; }
    if (store && d.k_out_stride) { *err = "k_out_stride with a cache"; return false; }
    const int64_t e = size_of(d.dtype), t = d.tokens, dim = d.head_dim;
    if (!token_stride(&d.q_stride, d.q_heads, dim, "q_stride", err) || !token_stride(&d.q_out_stride, d.q_heads, dim, "q_out_stride", err)) return false;
    if (d.k_heads && !token_stride(&d.k_stride, d.k_heads, dim, "k_stride", err)) return false;
    if (d.k_heads && !store && !token_stride(&d.k_out_stride, d.k_heads, dim, "k_out_stride", err)) return false;
    int64_t cache_bytes = 0;
    if (store) {
      if (!token_stride(&d.v_stride, d.k_heads, dim, "v_stride", err)) return false;
      if (!blocks_fit(d.blocks, d.block_size, &s.cache.shift, err)) return false;
      const int shift = s.cache.shift;
      if (!cache_layout(d.blocks, d.k_heads, d.block_size, dim, d.block_stride, d.head_stride, d.slot_stride, e, &s.cache, &cache_bytes, err)) return false;
      s.cache.shift = shift;
    }
    // The widest vector, up to 16 bytes, that every part of a head and every stride is a whole number of.
    int w = (int)(16 / e);
    auto whole = [&](int v) {
      for (int64_t n : {d.q_stride, d.q_out_stride, d.k_heads ? d.k_stride : 0, d.k_heads ? d.k_out_stride : 0, d.v_stride, s.cache.block, s.cache.head, s.cache.slot})
        if (n % v) return false;
      if (d.interleaved) return dim % v == 0 && d.rotary_dim % v == 0;
      return d.rotary_dim % (2 * v) == 0 && (dim - d.rotary_dim) % (2 * v) == 0;
    };
    while (w > 1 && !whole(w)) w >>= 1;
    if (!whole(w) || (d.interleaved && w < 2)) { *err = "strides must be even"; return false; }
    s.width = w;
    s.units = (int)((dim + 2 * w - 1) / (2 * w));
    s.heads = d.q_heads + d.k_heads * (store ? 2 : 1);
    fs::rotary_geometry(&s);
    if (w == 8 && s.heads_each > 1) p->lds_bytes = 8ll * s.most_angles;
    const int64_t q_row = d.q_heads * dim, k_row = d.k_heads * dim;
    fs::PagedPlan& g = p->paged;
    g.kind = FS_SCHED_ROTARY;
    g.in = {{"q", rows_bytes(t, d.q_stride, q_row, e), -1}};
    if (d.k_heads) g.in.push_back({"k", rows_bytes(t, d.k_stride, k_row, e), -1});
    if (store) g.in.push_back({"v", rows_bytes(t, d.v_stride, k_row, e), -1});
    g.in.push_back({"positions", 4 * t, -1});
    g.in.push_back({"frequencies", t ? 4ll * d.rotary_dim : 0, -1});
    if (store) g.in.push_back({"slots", 4 * t, -1});
    g.out = {{"q_out", rows_bytes(t, d.q_out_stride, q_row, e), d.q_stride == d.q_out_stride ? 0 : -1}};
    if (store) {
      g.out.push_back({"k_cache", t ? cache_bytes : 0, -1});
      g.out.push_back({"v_cache", t ? cache_bytes : 0, -1});
    } else if (d.k_heads) {
      g.out.push_back({"k_out", rows_bytes(t, d.k_out_stride, k_row, e), d.k_stride == d.k_out_stride ? 1 : -1});
    }
    g.bytes = 2 * t * dim * s.heads * e + t * (store ? 8 : 4) + 4ll * d.rotary_dim;
    p->description = numbers("rotary[GRID-WARP,THREAD] width=%lld, units=%lld, heads_each=%lld; cta_num=%lld, cta_size=256", s.width, s.units, s.heads_each,
                             (t * s.units * s.groups + 255) / 256) + (store ? ", stores k and v in the cache" : s.once ? ", stores past the caches" : "");
    return true;
  });
}

fs_status fs_plan_create_paged_attention(const fs_paged_attention_desc* desc, int64_t* partial_bytes, fs_plan** out) {
  const char* what = "fs_plan_create_paged_attention";
  if (out) *out = nullptr;
  if (!desc) return invalid(what, "desc is NULL");
  return create_attention(what, *desc, -1, partial_bytes, out);
}

fs_status fs_plan_create_paged_attention8(const fs_paged_attention8_desc* desc, int64_t* partial_bytes, fs_plan** out) {
  const char* what = "fs_plan_create_paged_attention8";
  if (out) *out = nullptr;
  if (!desc) return invalid(what, "desc is NULL");
  if (!known_code(desc->code)) return invalid(what, "unknown code");
  const fs_paged_attention8_desc& d = *desc;
  const fs_paged_attention_desc same = {d.dtype, d.requests, d.tokens, d.q_heads, d.kv_heads, d.head_dim, d.blocks, d.block_size, d.table_blocks, d.causal, d.window, d.max_new,
                                        d.log_sum_exp, 0, d.q_stride, d.out_stride, d.block_stride, d.head_stride, d.slot_stride, d.scale};
  return create_attention(what, same, d.code, partial_bytes, out);
}

fs_status fs_plan_create_cache_store8(const fs_cache8_desc* desc, fs_plan** out) { return create_cache8("fs_plan_create_cache_store8", desc, true, out); }
fs_status fs_plan_create_cache_read8(const fs_cache8_desc* desc, fs_plan** out) { return create_cache8("fs_plan_create_cache_read8", desc, false, out); }

}  // extern "C"

// Counts, NULL and alignment, identical pointers: as for all plans, on the plan's own list of buffers.
fs_status fs::paged_check_args(const PagedPlan& p, const void* const* in, int32_t n_in, void* const* out, int32_t n_out) {
  if (n_in != (int32_t)p.in.size()) return set_error(FS_ERR_INVALID, "n_in differs from the number of inputs");
  if (n_out != (int32_t)p.out.size()) return set_error(FS_ERR_INVALID, "n_out differs from the number of outputs");
  if (!in || !out) return set_error(FS_ERR_INVALID, "inputs/outputs is NULL");
  for (int i = 0; i < n_in; ++i)
    if (p.in[i].bytes && (!in[i] || (reinterpret_cast<uintptr_t>(in[i]) & 15)))
      return set_error(FS_ERR_INVALID, std::string("input ") + p.in[i].name + " is NULL or not 16-byte aligned");
  for (int i = 0; i < n_out; ++i) {
    if (!p.out[i].bytes) continue;
    if (!out[i] || (reinterpret_cast<uintptr_t>(out[i]) & 15)) return set_error(FS_ERR_INVALID, std::string("output ") + p.out[i].name + " is NULL or not 16-byte aligned");
    for (int k = 0; k < i; ++k)
      if (out[k] == out[i] && p.out[k].bytes) return set_error(FS_ERR_INVALID, std::string("outputs ") + p.out[k].name + " and " + p.out[i].name + " share one buffer");
    for (int k = 0; k < n_in; ++k)
      if (in[k] == out[i] && p.in[k].bytes && k != p.out[i].may_share)
        return set_error(FS_ERR_INVALID, std::string("output ") + p.out[i].name + " shares its buffer with input " + p.in[k].name);
  }
  return FS_OK;
}

int fs::paged_launch(const PagedPlan& p, const void* const* in, void* const* out, void* stream, std::string* err) {
  switch (p.kind) {
    case FS_SCHED_BLOCK_TABLES: return block_tables_launch(p.tables, in, out, stream, err);
    case FS_SCHED_ROTARY: return rotary_launch(p.rotary, in, out, stream, err);
    case FS_SCHED_CACHE_STORE8: return cache8_launch(p.cache8, true, in, out, stream, err);
    case FS_SCHED_CACHE_READ8: return cache8_launch(p.cache8, false, in, out, stream, err);
    default: return paged_attn_launch(p.attn, in, out, stream, err);
  }
}
