// The layout of a page's 4-bit record, and how attention over records is cut. Whole numbers only (no HIP), so that both can be checked without
// a GPU.
#pragma once
#include <stdint.h>

#include "dense_plan.hpp"

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

// Every page of a batch whose sequences may differ in length is cut by the lengths on the device, as for full-precision pages
// (dense_plan.hpp). Three workgroups run on a compute unit where there is a chunk for each; with fewer chunks than that
// two have equal shares. us with 512 / 768 workgroups at a time (8 KV heads, G = 4, D = 128): 32 sequences of 4K to 131K tokens, pages
// of 32 275 / 226, 16 x 131072 366 / 356; 12 of 2K to 50K, G = 8, which may be 672 chunks, 62.9 / 67.3. More rounds than one
// cost more than they balance: from 256, 512 or 768 pages of a chunk on 372, 360 and 356 for 16 x 131072.
inline DenseRound quant_round(int rows, int max_pages) {
  return {rows * most_splits(rows, max_pages).num_splits >= 768 ? 768 : 512, 768};
}
// (Batches that can read less than this are cut as if all were as long as the longest: 8 x 4000 tokens, 22 MB, 14.9 us either way.)
constexpr int64_t kQuantLeastBytes = 24ll << 20;

}  // namespace unique
