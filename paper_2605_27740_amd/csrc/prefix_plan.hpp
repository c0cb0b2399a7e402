// How attention over shared prefixes is cut into workgroups. Host arithmetic on the launch's bounds only (no HIP), so that it can be checked
// without a GPU.
#pragma once
#include <stdint.h>

#include <algorithm>

namespace unique {

struct PrefixPlan {
  int32_t rows;            // query rows of a workgroup: members times heads of the group
  int32_t blocks;          // of them in a group, at most
  int32_t chunk_pages;     // prefix pages of a workgroup
  int32_t chunks;          // of them in a prefix, at most
  int32_t own_pages;       // a sequence's own pages of a workgroup
  int32_t own_chunks;
  constexpr int32_t parts() const { return chunks + own_chunks; }  // of a row, at most
};

inline PrefixPlan prefix_plan(int batch, int kv_heads, int group, int elem, int page_size, int num_groups, int max_members, int max_prefix_pages,
                              int max_own_pages) {
  constexpr int64_t kWorkgroups = 512;
  PrefixPlan p;
  const int64_t rows = (int64_t)std::min(max_members, batch) * group;
  p.rows = elem == 4 ? 128 : (rows <= 64 ? 64 : 128);
  p.blocks = (int)((rows + p.rows - 1) / p.rows);
  const int64_t units = (int64_t)num_groups * p.blocks * kv_heads;
  const int per_tile = std::max(64 / page_size, 1);
  int64_t chunks = std::max<int64_t>(kWorkgroups / units, 1);
  int64_t pages = (max_prefix_pages + chunks - 1) / chunks;
  pages = std::max<int64_t>((pages + per_tile - 1) / per_tile * per_tile, per_tile);
  p.chunk_pages = (int)pages;
  p.chunks = (int)((max_prefix_pages + pages - 1) / pages);
  const int64_t own_units = (int64_t)batch * kv_heads;
  int64_t own = std::max<int64_t>(kWorkgroups / own_units, 1);
  own = std::max<int64_t>((max_own_pages + own - 1) / own, 4);
  own = std::min<int64_t>((own + 3) / 4 * 4, 256);
  p.own_pages = (int)own;
  p.own_chunks = (int)((max_own_pages + own - 1) / own);
  return p;
}

}  // namespace unique
