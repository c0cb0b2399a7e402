// The work items of attention over shared prefixes, and which instance of the kernels in prefix.hip a call takes.
#include "decode_core.hpp"
#include "serving.hpp"

namespace unique {
namespace {

constexpr int kItemThreads = 1024, kItemWaves = kItemThreads / kWave;
constexpr int kHeldSources = 2048;  // sources whose first items are searched in the LDS

// One workgroup makes the items: what each source has to read, how long items have to be for the chip to be full, where each source's items and
// partial results begin, and the items. Groups come first, as theirs have the most to do.
__global__ __launch_bounds__(kItemThreads) void prefix_items_kernel(CacheView c, PrefixArgs a) {
  __shared__ int s_first[kHeldSources + 1];
  __shared__ int64_t s_pages[kItemWaves];
  __shared__ int s_scan[2][kItemWaves];
  const int t = threadIdx.x, lane = t % kWave, wave = t / kWave;
  const int n = a.groups.num_groups, sources = n + c.B, G = c.H / c.Hkv;
  const unique_prefix_groups& g = a.groups;
  const PrefixWork& w = a.work;
  const bool held = sources <= kHeldSources;
  auto start_of = [&](int i) { return min(max(g.starts[i], 0), c.B); };
  auto prefix_of = [&](int i) { return min(max(g.prefix_pages[i], 0), g.max_prefix_pages); };
  auto size_of = [&](int i) { return min(max(start_of(i + 1) - start_of(i), 0), g.max_members); };
  if (held) {  // ends of the groups, to find the members' in
    for (int i = t; i < n; i += kItemThreads) s_first[i] = g.starts[i + 1];
    __syncthreads();
  }

  int64_t pages = 0;
  for (int i = t; i < sources; i += kItemThreads) {
    PrefixSource s = {};
    if (i < n) {
      const int size = size_of(i);
      s.place = start_of(i);
      s.rows = size * G;
      s.end = size > 1 ? prefix_of(i) : 0;  // (nobody to share it with: all pages are the member's own)
      s.blocks = (s.rows + a.shape.rows - 1) / a.shape.rows;
    } else {
      const int at = i - n;
      int lo = 0, hi = n;  // the first group that ends behind it
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if ((held ? s_first[mid] : g.starts[mid + 1]) > at) hi = mid;
        else lo = mid + 1;
      }
      PrefixMember m = {};
      m.seq = -1;
      if (lo < n && at >= g.starts[lo] && at - g.starts[lo] < g.max_members) {
        const int seq = g.members ? g.members[at] : at;
        if (seq >= 0 && seq < c.B) {
          m.seq = seq;
          m.reserved[0] = lo;
          s.place = at;
          s.rows = G;
          s.blocks = 1;
          const int prefix = prefix_of(lo);
          s.begin = size_of(lo) > 1 ? prefix : 0;
          s.end = min(min((c.seq_lens[seq] + c.S - 1) / c.S, c.max_pages_hint), prefix + g.max_own_pages);
        }
      }
      w.member[at] = m;
    }
    w.source[i] = s;
    pages += (int64_t)max(s.end - s.begin, 0) * s.blocks;
  }
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) pages += __shfl_xor(pages, d, kWave);
  if (lane == 0) s_pages[wave] = pages;
  __syncthreads();
  pages = 0;
  for (int i = 0; i < kItemWaves; ++i) pages += s_pages[i];
  const int64_t item_pages = prefix_item_pages(pages, a.shape.wanted);

  int items = 0, rows = 0;  // before the strip
  for (int i0 = 0; i0 < sources; i0 += kItemThreads) {
    const int i = i0 + t;
    PrefixSource s = {};
    if (i < sources) s = w.source[i];
    const PrefixCut cut = prefix_cut(s.end - s.begin, item_pages, min(s.rows, a.shape.rows), c.S, a.shape.tile_pages, i >= n);
    const int mine = cut.count * s.blocks;
    int x[2] = {mine, mine * (i < n ? a.shape.rows : G)}, upto[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) upto[k] = wave_inclusive_scan(x[k]);
    __syncthreads();
    if (lane == kWave - 1) {
      s_scan[0][wave] = upto[0];
      s_scan[1][wave] = upto[1];
    }
    __syncthreads();
    int all[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int waves = wave_inclusive_scan(lane < kItemWaves ? s_scan[k][lane] : 0);
      if (wave > 0) upto[k] += __builtin_amdgcn_readlane(waves, wave - 1);
      all[k] = __builtin_amdgcn_readlane(waves, kWave - 1);
    }
    s.first_item = items + upto[0] - x[0];
    s.first_row = rows + upto[1] - x[1];
    s.each = cut.pages;
    if (i < sources) {
      w.source[i] = s;
      if (held) s_first[i] = s.first_item;
    }
    items += all[0];
    rows += all[1];
  }
  if (t == 0) *w.num_items = items;
  __threadfence_block();
  __syncthreads();

  for (int at = t; at < c.B; at += kItemThreads) {
    PrefixMember m = w.member[at];
    if (m.seq < 0) continue;
    const PrefixSource s = w.source[m.reserved[0]], own = w.source[n + at];
    const int row = (at - s.place) * G;
    m.count = s.end > 0 ? (s.end + s.each - 1) / s.each : 0;
    m.part = s.first_row + row;  // blocks follow one another
    m.step = s.blocks * a.shape.rows;
    m.own_count = own.end > own.begin ? (own.end - own.begin + own.each - 1) / own.each : 0;
    m.own_part = own.first_row;
    w.member[at] = m;
  }
  for (int i = t; i < items; i += kItemThreads) {
    int lo = 0, hi = sources - 1;  // the last source that begins at or before it and has items
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if ((held ? s_first[mid] : w.source[mid].first_item) <= i) lo = mid;
      else hi = mid - 1;
    }
    const PrefixSource s = w.source[lo];
    const int k = i - s.first_item, run = k / s.blocks, block = k - run * s.blocks;
    PrefixItem item = {};
    item.place = s.place + block * (a.shape.rows / G);
    item.rows = min(s.rows - block * a.shape.rows, a.shape.rows);
    item.begin = s.begin + run * s.each;
    item.end = min(item.begin + s.each, s.end);
    item.seq = g.members ? g.members[s.place] : s.place;
    item.own = lo >= n;
    item.part = s.first_row + k * (lo < n ? a.shape.rows : G);
    w.item[i] = item;
  }
}

size_t aligned(size_t x) { return (x + 255) / 256 * 256; }

PrefixShape shape_of(const CacheView& c, const unique_prefix_groups& g) {
  return prefix_shape(c.B, c.Hkv, c.H / c.Hkv, c.dtype == 0 ? 4 : 2, c.S, g.num_groups, g.max_members, g.max_prefix_pages);
}

// Where everything lies in the workspace; -> its size.
size_t lay_out(const CacheView& c, const unique_prefix_groups& g, const PrefixShape& s, char* base, PrefixWork* w) {
  size_t at = 0;
  auto take = [&](auto** p, size_t count) {
    *p = reinterpret_cast<std::remove_reference_t<decltype(*p)>>(base + at);
    at += aligned(count * sizeof(**p));
  };
  take(&w->num_items, 1);
  take(&w->source, (size_t)g.num_groups + c.B);
  take(&w->item, (size_t)s.max_items);
  take(&w->member, (size_t)c.B);
  take(&w->part_o, (size_t)c.Hkv * s.max_rows * c.D);
  take(&w->part_ml, (size_t)c.Hkv * s.max_rows * 2);
  return at;
}

}  // namespace

size_t prefix_bytes(const CacheView& c, const unique_prefix_groups& g) {
  PrefixWork w;
  return lay_out(c, g, shape_of(c, g), nullptr, &w);
}

hipError_t launch_prefix(const CacheView& c, const unique_prefix_groups& g, const void* q, float scale_log2, void* out, float* lse_out, void* workspace,
                         hipStream_t st) {
  // The most that the bounds allow, all groups and members alike.
  const int64_t pages = std::min<int64_t>((int64_t)g.num_groups * g.max_prefix_pages + (int64_t)c.B * g.max_own_pages, c.num_phys);
  const bool streams = pages * c.Hkv * c.S * c.D * 2 * (c.dtype == 0 ? 4 : 2) > kStreamNtBytes;
  PrefixArgs a = {g, q, scale_log2, streams, out, lse_out, shape_of(c, g), {}};
  lay_out(c, g, a.shape, reinterpret_cast<char*>(workspace), &a.work);
  prefix_items_kernel<<<dim3(1), dim3(kItemThreads), 0, st>>>(c, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (c.dtype == 0) return c.D == 64 ? launch_prefix_of<float, 64>(c, a, st) : launch_prefix_of<float, 128>(c, a, st);
  return c.D == 64 ? launch_prefix_of<uint16_t, 64>(c, a, st) : launch_prefix_of<uint16_t, 128>(c, a, st);
}

}  // namespace unique
