// Pages of 4-bit numbers: the launches that write, read back and attend over records.
#pragma once
#include "kernels.hpp"
#include "quant_plan.hpp"

namespace unique {

// Full-precision pages on one side (c: the cache's table, strides and lengths), records on the other, found by a table of their own.
struct QuantPool {
  char* records;          // [num][Hkv][QuantTile::bytes()]
  const int32_t* table;   // [B][max_pages] of c
  int64_t num;
};

hipError_t launch_quantise(const CacheView& c, const QuantPool& pool, const int32_t* d_tok_begin, const int32_t* d_tok_end,
                           int max_pages_touched, hipStream_t stream);
hipError_t launch_restore(const CacheView& c, const QuantPool& pool, void* k_out, void* v_out, const int32_t* d_tok_begin,
                          const int32_t* d_tok_end, int max_pages_touched, hipStream_t stream);

// Attention over records, which c.page_table and c.num_phys describe. d_sel_pages == nullptr: every page, cut by the lengths (quant_plan.hpp)
// where that is worth while and the partial results that it may have, quant_cut_floats(c), find room.
size_t quant_cut_floats(const CacheView& c);
inline QuantBatch quant_batch(const CacheView& c) {
  return {c.B, c.Hkv, c.max_pages_hint, QuantTile{c.S, c.D}.bytes(), c.dtype == 1 || c.D == 64};
}
hipError_t launch_quant_decode(const CacheView& c, const void* records, const void* d_q, const int32_t* d_sel_pages, const int32_t* d_sel_count,
                               int sel_stride, int max_list_len, float sm_scale, void* d_out, float* d_lse_out, float* d_partials,
                               size_t partial_floats, hipStream_t stream);

struct QuantDecodeArgs {
  const char* records;
  const void* q;
  const int32_t* sel_pages;
  const int32_t* sel_count;
  int sel_stride;
  float scale_log2;
  float* part_o;
  float* part_ml;
  void* out;
  float* lse_out;
};
// plan.num_splits == 0: cut by the lengths into at most plan.pages_per_split chunks, and merged.
template <typename T, int D>
hipError_t launch_quant_partial(const CacheView& c, const QuantDecodeArgs& a, const SplitPlan& plan, bool stream_nt, hipStream_t stream);
template <> hipError_t launch_quant_partial<float, 64>(const CacheView&, const QuantDecodeArgs&, const SplitPlan&, bool, hipStream_t);
template <> hipError_t launch_quant_partial<float, 128>(const CacheView&, const QuantDecodeArgs&, const SplitPlan&, bool, hipStream_t);
template <> hipError_t launch_quant_partial<uint16_t, 64>(const CacheView&, const QuantDecodeArgs&, const SplitPlan&, bool, hipStream_t);
template <> hipError_t launch_quant_partial<uint16_t, 128>(const CacheView&, const QuantDecodeArgs&, const SplitPlan&, bool, hipStream_t);

}  // namespace unique
