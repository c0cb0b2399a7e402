// The steps around the cache: places for new tokens, their queries, keys and values, attention of sequences that share a prefix.
#pragma once
#include "../../include/unique.h"
#include "kernels.hpp"
#include "prefix_plan.hpp"

namespace unique {

// c.seq_lens and c.page_table are the descriptor's.
size_t place_bytes(const CacheView& c, int max_new_tokens);
hipError_t launch_place(const CacheView& c, const unique_placement& p, void* workspace, hipStream_t stream);

struct AppendArgs {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;  // elements from row to row
  const int32_t* positions;
  const int64_t* slots;
  void* q_out;
  int rows;
  unique_head_transform how;
};
hipError_t launch_append(const CacheView& c, const AppendArgs& a, hipStream_t stream);

// A prefix of a group, or a member's own pages.
struct PrefixSource {
  int32_t kind;                   // its items' class
  int32_t first_row;              // of their partial results
  int32_t begin, end;             // pages,
  int32_t each, count;            // those of an item, and items along them
  int32_t blocks;                 // of query rows; items of a block follow those of the next, a run of pages after the other
  int32_t place, rows;            // its first member, and its query rows
};
struct PrefixItem {
  int32_t place, rows;   // first member, query rows
  int32_t begin, end;    // pages
  int32_t seq;           // the sequence whose row of the page table it goes by
  int32_t own;           // 1: a member's own pages
  int32_t part;          // first row of its partial results
  int32_t reserved;
};
struct PrefixMember {
  int32_t seq;                  // < 0: left out
  int32_t count, part, step;    // of the group's items: how many, the row of the first's partial results, rows from one to the next
  int32_t own_count, own_part;  // of its own
  int32_t reserved[2];
};
struct PrefixWork {
  int32_t* num_items;    // one number
  PrefixSource* source;  // [groups + batch], and the items of each class before theirs, where they are more than the kernel that makes
  int32_t* first;        // [3][groups + batch]   the items holds
  PrefixItem* item;      // [max_items]
  PrefixMember* member;  // [batch]
  float* part_o;         // [kv_heads][max_rows][D]
  float* part_ml;        // [kv_heads][max_rows][2]
};
struct PrefixArgs {
  unique_prefix_groups groups;
  const void* q;
  float scale_log2;
  int32_t streams;  // keys and values are more than the caches hold
  void* out;
  float* lse_out;
  PrefixShape shape;
  PrefixWork work;
};
bool prefix_fits(const CacheView& c, const unique_prefix_groups& g);  // bounds that a launch can serve
size_t prefix_bytes(const CacheView& c, const unique_prefix_groups& g);
hipError_t launch_prefix(const CacheView& c, const unique_prefix_groups& g, const void* q, float scale_log2, void* out, float* lse_out, void* workspace,
                         hipStream_t stream);

template <typename T, int D>
hipError_t launch_prefix_of(const CacheView& c, const PrefixArgs& a, hipStream_t stream);
#define UNIQUE_DECLARE(T, D) template <> hipError_t launch_prefix_of<T, D>(const CacheView&, const PrefixArgs&, hipStream_t);
UNIQUE_DECLARE(float, 64) UNIQUE_DECLARE(float, 128) UNIQUE_DECLARE(uint16_t, 64) UNIQUE_DECLARE(uint16_t, 128)
#undef UNIQUE_DECLARE

}  // namespace unique
