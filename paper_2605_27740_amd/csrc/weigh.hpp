// Accounts of pages: attention that tells each page's share, and the eviction of the pages with the smallest accounts.
#pragma once
#include "dense_plan.hpp"
#include "kernels.hpp"

namespace unique {

// Attention over every page, as launch_decode's, which also adds to the account of every (sequence, KV head, page) the sum over the
// group's heads and the page's tokens of the attention weights: out[p] = decay * in[p] + that; in == nullptr: nothing so far.
struct WeighArgs {
  const void* q;
  float scale_log2, decay;
  const float* weights_in;
  float* weights_out;
  int weight_stride;  // floats from one (sequence, KV head) to the next
  void* out;
  float* lse_out;
  float* partials;    // weigh_floats(c)
};
size_t weigh_floats(const CacheView& c);
hipError_t launch_weigh(const CacheView& c, const WeighArgs& a, hipStream_t stream);

// How the batch is cut: by the lengths on the device into at most max_chunks chunks (dense_plan.hpp), or, where that is 0, by a plan.
struct WeighCut {
  SplitPlan plan;
  int max_chunks;
  DenseRound round;
};
template <typename T, int D>
hipError_t launch_weigh_of(const CacheView& c, const WeighArgs& a, const WeighCut& cut, float* part_ml, float* shares, hipStream_t stream);
#define UNIQUE_DECLARE(T, D) \
  template <> hipError_t launch_weigh_of<T, D>(const CacheView&, const WeighArgs&, const WeighCut&, float*, float*, hipStream_t);
UNIQUE_DECLARE(float, 64) UNIQUE_DECLARE(float, 128) UNIQUE_DECLARE(uint16_t, 64) UNIQUE_DECLARE(uint16_t, 128)
#undef UNIQUE_DECLARE

// Sequences of more than `budget` pages keep their first `sinks`, their last `recent` and the others with the largest accounts.
struct EvictArgs {
  int budget, sinks, recent;
  const float* weights_in;
  float* weights_out;
  int weight_stride;
  int32_t* page_table_out;
  int32_t* seq_lens_out;
  int32_t* freed_pages;  // [B][freed_stride]
  int32_t* freed_count;
  int freed_stride;
  void* workspace;       // evict_bytes(c)
};
size_t evict_bytes(const CacheView& c);
hipError_t launch_evict(const CacheView& c, const EvictArgs& a, hipStream_t stream);

}  // namespace unique
