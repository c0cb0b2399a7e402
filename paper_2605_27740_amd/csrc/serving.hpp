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

struct PrefixArgs {
  unique_prefix_groups groups;
  const void* q;
  float scale_log2;
  void* out;
  float* lse_out;
  float* partials;  // prefix_floats
};
size_t prefix_floats(const CacheView& c, const unique_prefix_groups& g);
hipError_t launch_prefix(const CacheView& c, const PrefixArgs& a, hipStream_t stream);

template <typename T, int D>
hipError_t launch_prefix_of(const CacheView& c, const PrefixArgs& a, const PrefixPlan& plan, float* part_ml, bool nt, hipStream_t stream);
#define UNIQUE_DECLARE(T, D) \
  template <> hipError_t launch_prefix_of<T, D>(const CacheView&, const PrefixArgs&, const PrefixPlan&, float*, bool, hipStream_t);
UNIQUE_DECLARE(float, 64) UNIQUE_DECLARE(float, 128) UNIQUE_DECLARE(uint16_t, 64) UNIQUE_DECLARE(uint16_t, 128)
#undef UNIQUE_DECLARE

}  // namespace unique
