// The operators around a paged cache of keys and values (fs.h): what a plan of one of them holds, and their launches.
#pragma once
#include <stdint.h>
#include <string>
#include <vector>
#include "../../include/fs.h"

namespace fs {

// A buffer of a launch: its name for messages, its size (0: the pointer is not looked at) and, for an output, the input whose
// very buffer it may take (-1: none).
struct PagedBuffer { const char* name; int64_t bytes; int may_share; };

// Where a row of the cache begins: strides in elements, block_size = 1 << shift.
struct CacheLayout { int64_t block = 0, head = 0, slot = 0; int blocks = 0, shift = 0; };

struct BlockTablesSpec { fs_block_tables_desc d{}; int wg = 256, grid = 1; int64_t lds = 0; };
struct RotarySpec {
  fs_rotary_desc d{};
  CacheLayout cache;
  int width = 1;                   // elements of a vector
  int units = 1, heads = 1;        // threads to a head, heads in all (of q, k and stored v)
  int heads_each = 1, groups = 1;  // heads of a thread, threads that share the heads
  bool once = false;               // stores past the caches, where the outputs begin at lines of 128 bytes
  bool one = false;                // a vector of a head to a thread
  int most_angles = 0;             // several heads to a thread: angles of a workgroup's rows
};
struct PagedAttnSpec {
  fs_paged_attention_desc d{};
  CacheLayout cache;
  int share = 1;                   // query heads to a key head
  // requests of up to few_rows rows: tiles of 16 * row_tiles, units of unit_keys keys, 1 << log_groups workgroups
  int few_rows = 0, row_tiles = 1, unit_keys = 256, log_groups = 0, few_grid = 0;
  int log_heads = 0;               // key heads of a set, 1 << log_heads
  bool neighbours = false;         // workgroups of an XCD have neighbouring runs
  // the others: places for tiles of 128 rows (0: there are none)
  int64_t slots = 0, few_bytes = 0, partial_bytes = 0;
};

struct PagedPlan {
  int kind = 0;                    // fs_schedule, 0: the plan is none of these
  std::vector<PagedBuffer> in, out;
  int64_t bytes = 0;               // algorithmic
  BlockTablesSpec tables;
  RotarySpec rotary;
  PagedAttnSpec attn;
};

int block_tables_launch(const BlockTablesSpec&, const void* const* in, void* const* out, void* stream, std::string* err);
void rotary_geometry(RotarySpec*);
int rotary_launch(const RotarySpec&, const void* const* in, void* const* out, void* stream, std::string* err);

// Kernels, geometry and partial results of an attention plan; false: FS_ERR_UNSUPPORTED with *err.
bool paged_attn_plan(PagedAttnSpec*, int* n_kernels, int64_t* lds_bytes, std::string* err);
std::string paged_attn_describe(const PagedAttnSpec&);
int paged_attn_launch(const PagedAttnSpec&, const void* const* in, void* const* out, void* stream, std::string* err);

fs_status paged_check_args(const PagedPlan&, const void* const* in, int32_t n_in, void* const* out, int32_t n_out);
int paged_launch(const PagedPlan&, const void* const* in, void* const* out, void* stream, std::string* err);

}  // namespace fs
