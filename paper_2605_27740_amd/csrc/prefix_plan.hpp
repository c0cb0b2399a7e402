// How attention over shared prefixes is cut into work items. Whole numbers only (no HIP), so that it can be checked without a GPU; the kernel that
// makes the items uses the same functions. (constexpr functions are compiled for the device, too.)
#pragma once
#include <stdint.h>

#include <algorithm>

namespace unique {

// Every group is a source of items, its prefix's pages times the blocks of its members' query rows, and every member one, its own pages.
constexpr int kPrefixSlots = 512;  // workgroups that run at a time, two to a compute unit

constexpr int kPrefixMostPages = 512;  // of an item of a prefix, whose page ids are held in registers
constexpr int kPrefixMostWorkgroups = (1 << 24) - 1;  // of 256 threads, of which a launch has fewer than 2^32

// Where there is little to read, every member reads its prefix for itself, in chunks that the host cuts, mostly out of the caches: there is no plan, and nothing to join if a chunk is all. Shared / each
// for itself, us: 2 x 2148 tokens (fp32, 2 heads of 64, 4 MB) 15.6 / 9.4, 2 x 300 (8 heads, bf16) 12.5 / 6.8, 8 x 1100 (34 MB) 14.3 / 10.8, 16 x 1500 (94 MB) 15.8 / 17.4, 4 x 8500 (133 MB) 21.7 / 24.4.
// If a chunk is all, up to 256 MB: 245 x 57 tokens (32 heads, 245 MB) 70.4 / 59.1, 64 x 768 in 8 groups (192 MB) 21.6 / 19.2, 128 x 520 (264 MB) 27.2 / 25.8. In fp32, whose products take long, up to 160:
// 57 x 1769 (one head, 99 MB) 24.0 / 20.7, 67 x 2039 in 5 groups (134 MB) 25.4 / 25.5, 4 x 4500 (141 MB) 35.2 / 28.7, 20 x 2865 of 64 channels (225 MB) 23.2 / 29.1, 2 x 14065 (220 MB) 57.3 / 45.7.
constexpr int64_t prefix_alone_bytes(bool one_chunk, int elem) { return (one_chunk ? 256ll : (elem == 4 ? 160ll : 64ll)) << 20; }
// Tokens of such a chunk at least, and half as many again if that is all of them: 2 x 600 tokens in one chunk or two 9.5 / 10.5 us, 900 12.3 / 11.9; chunks of 256, 512 and 1024 tokens at least, 8 x 1100
// 13.4 / 11.5 / 13.8. fp32, 2 x 2148 tokens of 64 channels, by 128 and 512: 9.8 / 12.7.
constexpr int prefix_alone_tokens(int elem) { return elem == 4 ? 128 : 512; }
// Every workgroup goes through the groups' starts, 64 at a time, for its member's: shared / each for itself 1024 x 70 tokens in 512 groups 50.4 / 27.7 us, 4096 in 2048 (or one more) 175 / 159.
constexpr int kPrefixAloneGroups = 2048;

struct PrefixShape {
  int32_t rows;         // query rows of a workgroup's block
  int32_t tile_pages;   // pages of a tile of tokens, a power of two
  int32_t wanted;       // items per KV head
  int32_t row_tokens;   // tokens of an item at least, for four of its rows
  int32_t max_items;    // there are at most, per KV head
  int32_t max_rows;     // rows of partial results at most, per KV head
  int32_t fits;         // a launch has room for that many; if not, the call is refused
  int32_t plans;        // every workgroup of the attention kernel makes the plan for itself
  int32_t chunks;       // of a member's pages, at most, where every member reads the prefix for itself; 0: it is shared
  int32_t chunk_pages;  // pages of such a chunk
};

// page_bytes: keys and values of a page and head; max_pages: the most that a sequence has.
inline PrefixShape prefix_shape(int batch, int kv_heads, int group, int elem, int page_size, int page_bytes, int max_pages, int num_groups, int max_members,
                                int max_prefix_pages, int max_own_pages) {
  PrefixShape s = {};
  const int64_t pages = std::max<int64_t>(std::min<int64_t>((int64_t)max_prefix_pages + max_own_pages, max_pages), 1), members = (int64_t)batch * kv_heads;
  const int64_t least = prefix_alone_tokens(elem) / page_size;
  const bool one = 2 * pages <= 3 * least;
  if (num_groups <= kPrefixAloneGroups && members * pages * page_bytes <= prefix_alone_bytes(one, elem)) {
    const int64_t n = one ? 1 : std::min((pages + least - 1) / least, std::max<int64_t>(2 * kPrefixSlots / members, 1));
    s.chunk_pages = (int32_t)((pages + n - 1) / n);
    s.chunks = (int32_t)((pages + s.chunk_pages - 1) / s.chunk_pages);
    s.max_rows = (int32_t)((int64_t)batch * s.chunks * group);
    s.fits = 1;
    return s;
  }
  const int64_t most = (int64_t)max_members * group;
  s.rows = elem == 4 ? 128 : (most <= 64 ? 64 : 128);
  s.tile_pages = (elem == 4 ? 32 : 64) / page_size;
  s.row_tokens = elem == 4 ? 2 : 8;
  const int64_t blocks = std::min<int64_t>(num_groups * ((most + s.rows - 1) / s.rows), (int64_t)batch * group / s.rows + num_groups);
  // An eighth fewer items than fit leave room for the short ones, unless a prefix's items are many blocks' anyway. 512 / 448, us: 16 x 131072 tokens 110.6 / 107.8, 24 x 100000 107 / 110, 32 x 8192 40.4 / 41.6,
  // 60 rows in 6 groups 106.4 / 105.9 (with one bf16 part of a probability instead of three 108.5 / 101.8, 103.7 / 97.2, 40.2 / 38.8, 107.2 / 105.1; 256 x 32768, eight blocks, 182 / 193).
  s.wanted = std::max((blocks > 2 * num_groups ? kPrefixSlots : kPrefixSlots / 8 * 7) / kv_heads, 1);
  // A source's items are one more than its share of the wanted ones at most, and hold a tile each. A member who is alone in a group has its prefix as their own.
  const int64_t longest = blocks * max_prefix_pages / kPrefixMostPages, prefix_tiles = blocks * ((max_prefix_pages + s.tile_pages - 1) / s.tile_pages);
  const int64_t tiles = prefix_tiles + (int64_t)batch * ((max_own_pages + s.tile_pages - 1) / s.tile_pages);
  const int64_t of_prefixes = std::min(std::max<int64_t>(s.wanted, longest) + blocks, prefix_tiles);
  // Prefixes may have to be cut for their page ids, when items would be longer.
  const int64_t cost = blocks * max_prefix_pages + batch * (max_own_pages + 96 / page_size + 1ll);
  const int64_t most_items = s.wanted + (cost > (int64_t)kPrefixMostPages * s.wanted ? longest : 0) + blocks + batch;
  const int64_t items = std::max<int64_t>(std::min(most_items, tiles), 1), all_rows = of_prefixes * s.rows + std::min<int64_t>(s.wanted + batch, tiles) * group;
  s.fits = items <= kPrefixMostWorkgroups / kv_heads && all_rows <= INT32_MAX;
  s.max_items = s.fits ? (int32_t)items : 0;
  s.max_rows = s.fits ? (int32_t)all_rows : 0;
  // The plan takes a workgroup 2.5 us, and a kernel of its own 5. By a kernel / by all, us (512 items wanted): 2 x 2148 tokens (fp32, 2 heads) 17.5 / 15.0, 32 x 8192 (8 heads, with 1000 of their own) 47.6 /
  // 43.6, 16 x 131072 108.1 / 105.8, 60 rows in 6 groups of 20000 tokens 158.9 / 157.8.
  s.plans = num_groups + batch < 256 && (int64_t)s.max_items * kv_heads <= 2 * kPrefixSlots;
  return s;
}

// (Page sizes are powers of two, and divisions in 64 bits take a workgroup as long as a trip to memory.)
constexpr int prefix_pages_of(int tokens, int page_size) { return tokens <= 0 ? 0 : (int)(((uint32_t)tokens + page_size - 1) >> __builtin_ctz(page_size)); }

// Kinds of items, in the order in which they are started: the long ones first.
enum PrefixKind { kPrefixRun = 0, kOwnRun = 1, kShortOwn = 2, kPrefixKinds = 3 };
constexpr int prefix_kind(bool own, int pages, int item_pages) { return !own ? kPrefixRun : (2 * pages >= item_pages ? kOwnRun : kShortOwn); }

// What a source costs, in pages. An item of few rows takes 3.5 us whatever there is to read, as long as 100 tokens of an 8-headed bf16 cache.
constexpr int64_t prefix_cost(int pages, int blocks, bool own, int page_size) {
  return pages <= 0 ? 0 : (int64_t)pages * blocks + (own ? prefix_pages_of(96, page_size) : 0);
}

// Pages of an item, before the items of a source are made equal: such that there are at most `wanted` items and one for each source's block. (No source has 2^29 pages.)
constexpr int prefix_item_pages(int64_t all_pages, int wanted) {
  if (all_pages <= INT32_MAX / 2) return (int)(((uint32_t)all_pages + (uint32_t)wanted - 1) / (uint32_t)wanted);
  const int64_t each = (all_pages + wanted - 1) / wanted;
  return each < (1 << 29) ? (int)each : 1 << 29;
}

// Items along a source's pages, and the pages of each. A block of many rows gets longer ones: its partial results, 4 bytes times D a row, are written and
// read again, and tokens are 4 bytes times D (bf16) each as well. In fp32, whose products take four times as long for each byte, a quarter as long: 70 rows behind 4722 tokens (one KV head) 50.7 / 28.2 us.
struct PrefixCut {
  int32_t count, pages;
};
constexpr PrefixCut prefix_cut(int pages, int item_pages, int live_rows, int row_tokens, int page_size, int tile_pages, bool own) {
  if (pages <= 0) return PrefixCut{0, tile_pages};
  const int least = prefix_pages_of((live_rows * row_tokens + 3) >> 2, page_size);
  uint32_t p = item_pages > least ? item_pages : least;
  if (!own && p > kPrefixMostPages) p = kPrefixMostPages;
  const uint32_t n = (pages + p - 1) / p;
  uint32_t each = (pages + n - 1) / n;
  each = (each + tile_pages - 1) & ~(uint32_t)(tile_pages - 1);
  return PrefixCut{(int32_t)((pages + each - 1) / each), (int32_t)each};
}

}  // namespace unique
