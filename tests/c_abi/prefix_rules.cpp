// C interface of the cut of attention over shared prefixes for the CPU tests.
#include "../../paper_2605_27740_amd/csrc/prefix_plan.hpp"

// Where every member reads for itself: chunks of a member, their pages, rows of partial results per KV head; chunks is 0 where prefixes are shared.
extern "C" void prefix_alone(int batch, int kv_heads, int group, int elem, int page_size, int page_bytes, int max_pages, int max_prefix, int max_own, int* out) {
  const unique::PrefixShape s = unique::prefix_shape(batch, kv_heads, group, elem, page_size, page_bytes, max_pages, 1, batch, max_prefix, max_own);
  out[0] = s.chunks; out[1] = s.chunk_pages; out[2] = s.max_rows;
}

// Sources (pages, rows, own) of a KV head -> items' sources and pages; the shape's bounds. Pages are so large that prefixes are shared.
extern "C" int prefix_items(int batch, int kv_heads, int group, int elem, int page_size, int num_groups, int max_members, int max_prefix, int max_own, int sources,
                            const int* pages, const int* rows, const int* own, int* shape, int* count, int* each, int* blocks) {
  const unique::PrefixShape s = unique::prefix_shape(batch, kv_heads, group, elem, page_size, 1 << 30, 1 << 30, num_groups, max_members, max_prefix, max_own);
  if (!s.fits) return 1;
  if (s.chunks) return 2;
  int64_t cost = 0;
  for (int i = 0; i < sources; ++i) {
    blocks[i] = (rows[i] + s.rows - 1) / s.rows;
    cost += unique::prefix_cost(pages[i], blocks[i], own[i], page_size);
  }
  const int item_pages = unique::prefix_item_pages(cost, s.wanted);
  for (int i = 0; i < sources; ++i) {
    const unique::PrefixCut cut = unique::prefix_cut(pages[i], item_pages, rows[i] < s.rows ? rows[i] : s.rows, s.row_tokens, page_size, s.tile_pages, own[i]);
    count[i] = cut.count;
    each[i] = cut.pages;
  }
  const int out[] = {s.rows, s.tile_pages, s.wanted, s.max_items, s.max_rows, s.plans, unique::kPrefixSlots, unique::kPrefixMostPages};
  for (int i = 0; i < 8; ++i) shape[i] = out[i];
  return 0;
}
