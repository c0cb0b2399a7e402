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

// Every page of a batch whose sequences may differ in length is cut by the lengths on the device, as for full-precision pages (dense_plan.hpp),
// into as many chunks as workgroups run at the same time, or a multiple that is two to a row. us without / with a cut (8 KV heads, G = 4, D = 128,
// pages of 16): 40 sequences of 1K to 4K tokens 32.5 / 27.2, even 38.2 / 39.3; 60 of 500 to 20K 80.4 / 75.7; 40 of 500 to 6K, D = 64, 27.3 / 21.5. With
// more than 256 rows a row that is short is soon done, and the merge is another launch: 64 x 2000 27.1 / 37.2, 64 of 100 to 700 11.1 / 19.6.
// Three workgroups run on a compute unit, two of fp32 outputs with D = 128, and two have enough to do where there is little (and no more rows than 256): with
// 512 / 768 at a time 32 sequences of 4K to 131K tokens, pages of 32, 275 / 226, 16 x 131072 366 / 356; 16 of 400 to 1500 14.2 / 15.1, 4 of 6K to 30K 21.4 / 21.9; fp32,
// 8 of 1K to 30K 33.4 / 36.4. More rounds than one cost more than they balance: from 256, 512 or 768 pages of a chunk on 372, 360 and 356 for 16 x 131072.
constexpr int kQuantMostRows = 1024;
constexpr int64_t kQuantLeastBytes = 24ll << 20, kQuantLeastRow = 384ll << 10, kQuantThreeBytes = 256ll << 20;
struct QuantBatch {
  int batch, kv_heads, max_pages, page_bytes;  // of the part of a KV head
  bool three_fit;
  constexpr int rows() const { return batch * kv_heads; }
  constexpr int64_t row_bytes() const { return (int64_t)max_pages * page_bytes; }
  DenseRound round() const {
    const int slots = three_fit && (rows() > 256 || rows() * row_bytes() >= kQuantThreeBytes) ? 768 : 512;
    return {(2 * rows() + slots - 1) / slots * slots, 768};
  }
  int max_chunks() const { return (int)dense_wanted_chunks(rows(), max_pages, round()); }
  bool balances() const {
    if (batch < 2 || batch > kDenseMaxBatch || rows() > kQuantMostRows || (int64_t)rows() * max_pages > INT32_MAX) return false;
    return rows() * row_bytes() >= kQuantLeastBytes && (rows() <= 256 || row_bytes() >= kQuantLeastRow);
  }
};

}  // namespace unique
