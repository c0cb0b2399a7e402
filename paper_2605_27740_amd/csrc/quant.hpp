// Pages of 4-bit numbers: the layout of a page's record and the launches that write, read back and attend over records.
#pragma once
#include "dense_plan.hpp"
#include "kernels.hpp"

namespace unique {

constexpr int kQuantBlock = 32;  // channels that share a scale

// The part of one KV head in a page's record: K codes [S][D], two to a byte, the even channel in the low half | V codes
// [S/8][16][8][D/16]: groups of eight tokens, of D/16 channels | K scales [D/32][S] | V scales [D/32][S].
// V is stored the way the p.V product wants it: its lanes hold D/16 channels of four consecutive tokens, here 16 (D = 128) or 8
// consecutive bytes, where rows of channels would make it four loads of 4 or 2 bytes. A token is whole bytes in both, so that
// tokens can be added one by one.
struct QuantTile {
  int S, D;
  constexpr int k_codes() const { return 0; }
  constexpr int v_codes() const { return S * D / 2; }
  constexpr int k_scales() const { return S * D; }
  constexpr int v_scales() const { return S * D + S * (D / kQuantBlock); }
  constexpr int bytes() const { return S * D + 2 * S * (D / kQuantBlock); }
  constexpr int v_unit_bytes() const { return D / 32; }  // D/16 channels of a token
  constexpr int v_at(int tok, int unit) const { return v_codes() + ((tok / 8 * 16 + unit) * 8 + tok % 8) * v_unit_bytes(); }
};

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

// Attention over records, which c.page_table and c.num_phys describe. d_sel_pages == nullptr: every page.
hipError_t launch_quant_decode(const CacheView& c, const void* records, const void* d_q, const int32_t* d_sel_pages, const int32_t* d_sel_count,
                               int sel_stride, int max_list_len, float sm_scale, void* d_out, float* d_lse_out, float* d_partials,
                               hipStream_t stream);

// Every page of a batch whose sequences may differ in length is cut by the lengths on the device, as for full-precision pages
// (dense_plan.hpp). Three workgroups run on a compute unit where there is a chunk for each; with fewer chunks than that
// two have equal shares. us with 512 / 768 workgroups at a time (8 KV heads, G = 4, D = 128): 32 sequences of 4K to 131K tokens, pages
// of 32 275 / 226, 16 x 131072 366 / 356; 12 of 2K to 50K, G = 8, which may be 672 chunks, 62.9 / 67.3. More rounds than one
// cost more than they balance: from 256, 512 or 768 pages of a chunk on 372, 360 and 356 for 16 x 131072.
inline DenseRound quant_round(int rows, int max_pages) {
  return {rows * most_splits(rows, max_pages).num_splits >= 768 ? 768 : 512, 768};
}
constexpr int64_t kQuantLeastBytes = 24ll << 20;

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
