// The work items of attention over shared prefixes, and which instance of the kernels in prefix.hip a call takes.
#include "decode_core.hpp"
#include "serving.hpp"

namespace unique {
namespace {

constexpr int kItemThreads = 1024, kItemWaves = kItemThreads / kWave;
constexpr int kHeldSources = kItemThreads;  // sources that are kept in the LDS
constexpr int kClasses = 3;                 // items come in this order: prefixes', long ones of members, short ones of members

// One workgroup makes the items: what each source has to read, how long items have to be for the chip to be full, where each source's items and
// partial results begin, and the items. kHeld: there is a thread for every source, and their number is the only loop.
template <bool kHeld>
__global__ __launch_bounds__(kItemThreads) void prefix_items_kernel(CacheView c, PrefixArgs a) {
  __shared__ PrefixSource s_source[kHeld ? kHeldSources : 1];
  __shared__ int s_first[kClasses][kHeld ? kHeldSources : 1];  // items of a class before each source's
  __shared__ int64_t s_cost[kItemWaves];
  __shared__ int s_scan[kClasses + 1][kItemWaves];
  const int t = threadIdx.x, lane = t % kWave, wave = t / kWave;
  const int n = a.groups.num_groups, sources = n + c.B, G = c.H / c.Hkv;
  const unique_prefix_groups& g = a.groups;
  const PrefixWork& w = a.work;
  PrefixSource* const source = kHeld ? s_source : w.source;
  auto first_of = [&](int k, int i) -> int& { return kHeld ? s_first[k][i] : w.first[(int64_t)k * sources + i]; };
  auto bound = [&](int at) { return min(max(at, 0), c.B); };
  auto prefix_of = [&](int pages) { return min(max(pages, 0), g.max_prefix_pages); };
  auto size_of = [&](int from, int to) { return min(max(bound(to) - bound(from), 0), g.max_members); };

  // What a source has to read. A member's group is the first that ends behind it.
  auto look_at = [&](int i, PrefixMember& m) {
    PrefixSource s = {};
    if (i < n) {
      const int from = g.starts[i], to = g.starts[i + 1], pages = g.prefix_pages[i], size = size_of(from, to);
      s.place = bound(from);
      s.rows = size * G;
      s.end = size > 1 ? prefix_of(pages) : 0;  // (nobody to share it with: all pages are the member's own)
      s.blocks = (s.rows + a.shape.rows - 1) / a.shape.rows;
      return s;
    }
    const int at = i - n, seq = g.members ? g.members[at] : at;
    int lo = 0, hi = n;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (g.starts[mid + 1] > at) hi = mid;
      else lo = mid + 1;
    }
    m = {};
    m.seq = -1;
    if (lo == n) return s;
    const int from = g.starts[lo], to = g.starts[lo + 1], prefix = prefix_of(g.prefix_pages[lo]);
    if (at < from || at - from >= g.max_members || seq < 0 || seq >= c.B) return s;
    m.seq = seq;
    m.group = lo;
    s.place = at;
    s.rows = G;
    s.blocks = 1;
    s.begin = size_of(from, to) > 1 ? prefix : 0;
    s.end = min(min((c.seq_lens[seq] + c.S - 1) / c.S, c.max_pages_hint), prefix + g.max_own_pages);
    return s;
  };
  auto cost_of = [&](int i, const PrefixSource& s) { return prefix_cost(s.end - s.begin, s.blocks, i >= n, c.S); };

  PrefixSource s = {};
  PrefixMember m = {};
  int64_t cost = 0;
  for (int i = t; i < sources; i += kItemThreads) {
    s = look_at(i, m);
    cost += cost_of(i, s);
    if constexpr (!kHeld) {
      w.source[i] = s;
      if (i >= n) w.member[i - n] = m;
    }
  }
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) cost += __shfl_xor(cost, d, kWave);
  if (lane == 0) s_cost[wave] = cost;
  __syncthreads();
  cost = lane < kItemWaves ? s_cost[lane] : 0;
#pragma unroll
  for (int d = 1; d < kItemWaves; d *= 2) cost += __shfl_xor(cost, d, kWave);
  const int64_t item_pages = prefix_item_pages(__shfl(cost, 0, kWave), a.shape.wanted);

  int before[kClasses + 1] = {0, 0, 0, 0};  // items of each class and rows before the strip
  for (int i0 = 0; i0 < sources; i0 += kItemThreads) {
    const int i = i0 + t;
    if constexpr (!kHeld) s = i < sources ? w.source[i] : PrefixSource{};
    const PrefixCut cut = prefix_cut(s.end - s.begin, item_pages, min(s.rows, a.shape.rows), c.S, a.shape.tile_pages, i >= n);
    const int mine = cut.count * s.blocks;
    s.kind = i < n ? 0 : (2 * (int64_t)min(cut.pages, s.end - s.begin) >= item_pages ? 1 : 2);
    int x[kClasses + 1], upto[kClasses + 1];
#pragma unroll
    for (int k = 0; k < kClasses; ++k) x[k] = s.kind == k ? mine : 0;
    x[kClasses] = mine * (i < n ? a.shape.rows : G);
#pragma unroll
    for (int k = 0; k <= kClasses; ++k) upto[k] = wave_inclusive_scan(x[k]);
    __syncthreads();
    if (lane == kWave - 1) {
#pragma unroll
      for (int k = 0; k <= kClasses; ++k) s_scan[k][wave] = upto[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k <= kClasses; ++k) {
      const int waves = wave_inclusive_scan(lane < kItemWaves ? s_scan[k][lane] : 0);
      upto[k] += before[k] + (wave > 0 ? __builtin_amdgcn_readlane(waves, wave - 1) : 0);
      before[k] += __builtin_amdgcn_readlane(waves, kWave - 1);
    }
    s.first_row = upto[kClasses] - x[kClasses];
    s.count = cut.count;
    s.each = cut.pages;
    if (i < sources) {
      source[i] = s;
#pragma unroll
      for (int k = 0; k < kClasses; ++k) first_of(k, i) = upto[k] - x[k];
    }
  }
  const int items = before[0] + before[1] + before[2];
  if (t == 0) *w.num_items = items;
  if constexpr (!kHeld) __threadfence_block();
  __syncthreads();

  for (int i = n + t % kItemThreads - (kHeld ? n : 0); i < sources; i += kItemThreads) {
    if (i < n) continue;
    if constexpr (!kHeld) m = w.member[i - n];
    if (m.seq >= 0) {
      const PrefixSource of = source[m.group], own = source[i];
      m.count = of.count;
      m.part = of.first_row + (i - n - of.place) * G;  // blocks follow one another
      m.step = of.blocks * a.shape.rows;
      m.own_count = own.count;
      m.own_part = own.first_row;
    }
    w.member[i - n] = m;
  }
  for (int i = t; i < items; i += kItemThreads) {
    int k = 0, y = i;
    if (y >= before[0]) {
      y -= before[0];
      k = 1;
      if (y >= before[1]) {
        y -= before[1];
        k = 2;
      }
    }
    int lo = 0, hi = sources - 1;  // the last source whose items of this class begin at or before it
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (first_of(k, mid) <= y) lo = mid;
      else hi = mid - 1;
    }
    const PrefixSource of = source[lo];
    const int z = y - first_of(k, lo), run = z / of.blocks, block = z - run * of.blocks;
    PrefixItem item = {};
    item.place = of.place + block * (a.shape.rows / G);
    item.rows = min(of.rows - block * a.shape.rows, a.shape.rows);
    item.begin = of.begin + run * of.each;
    item.end = min(item.begin + of.each, of.end);
    item.seq = g.members ? g.members[of.place] : of.place;
    item.own = k != 0;
    item.part = of.first_row + z * (k == 0 ? a.shape.rows : G);
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
  const size_t sources = (size_t)g.num_groups + c.B, kept = sources > kHeldSources ? sources : 0;
  take(&w->source, kept);
  take(&w->first, kept * kClasses);
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
  if (g.num_groups + c.B <= kHeldSources) prefix_items_kernel<true><<<dim3(1), dim3(kItemThreads), 0, st>>>(c, a);
  else prefix_items_kernel<false><<<dim3(1), dim3(kItemThreads), 0, st>>>(c, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (c.dtype == 0) return c.D == 64 ? launch_prefix_of<float, 64>(c, a, st) : launch_prefix_of<float, 128>(c, a, st);
  return c.D == 64 ? launch_prefix_of<uint16_t, 64>(c, a, st) : launch_prefix_of<uint16_t, 128>(c, a, st);
}

}  // namespace unique
