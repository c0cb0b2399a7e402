// The work items of attention over shared prefixes, and which instance of the kernels in prefix.hip a call takes.
#include "prefix_items.hpp"

namespace unique {
namespace {

constexpr int kItemThreads = 1024, kFewThreads = 256;
constexpr int kHeldSources = kItemThreads - 1;  // sources that are kept in the LDS

// One workgroup makes the items.
template <int kThreads, bool kHeld>
__global__ __launch_bounds__(kThreads) void prefix_items_kernel(CacheView c, PrefixArgs a) {
  __shared__ ItemsShared<kThreads, kHeld> sh;
  ItemsPlan<kThreads, kHeld> plan = {c, a, sh};
  plan.make();
  if (kHeld && plan.t < plan.sources) plan.keep(plan.t);
  const int n = plan.n, items = plan.items();
  if (plan.t == 0) *a.work.num_items = items;
  if constexpr (!kHeld) __threadfence_block();
  __syncthreads();

  if constexpr (kHeld) {
    if (plan.t >= n && plan.t < plan.sources) plan.tell_member(plan.t - n, plan.m);
  } else {
    for (int i = plan.t; i < c.B; i += kThreads) plan.tell_member(i, a.work.member[i]);
  }
  for (int i = plan.t; i < items; i += kThreads) {
    int y = i;
    const int k = plan.class_of(y);
    int lo = 0, hi = plan.sources - 1;  // the last source whose items of this class begin at or before it
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (plan.first_of(k, mid) <= y) lo = mid;
      else hi = mid - 1;
    }
    const PrefixSource of = plan.source()[lo];
    a.work.item[i] = plan.item_of(of, y - plan.first_of(k, lo), plan.leader_of(of));
  }
}

size_t aligned(size_t x) { return (x + 255) / 256 * 256; }

PrefixShape shape_of(const CacheView& c, const unique_prefix_groups& g) {
  return prefix_shape(c.B, c.Hkv, c.H / c.Hkv, c.dtype == 0 ? 4 : 2, c.S, c.S * c.D * 2 * (c.dtype == 0 ? 4 : 2), c.max_pages_hint, g.num_groups, g.max_members, g.max_prefix_pages, g.max_own_pages);
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

bool prefix_fits(const CacheView& c, const unique_prefix_groups& g) { return shape_of(c, g).fits; }

size_t prefix_bytes(const CacheView& c, const unique_prefix_groups& g) {
  PrefixWork w;
  return lay_out(c, g, shape_of(c, g), nullptr, &w);
}

hipError_t launch_prefix(const CacheView& c, const unique_prefix_groups& g, const void* q, float scale_log2, void* out, float* lse_out, void* workspace,
                         hipStream_t st) {
  // The most that the bounds allow, all groups and members alike.
  const int64_t pages = std::min<int64_t>((int64_t)g.num_groups * g.max_prefix_pages + (int64_t)c.B * g.max_own_pages, c.num_phys);
  const bool streams = pages * c.Hkv * c.S * c.D * 2 * (c.dtype == 0 ? 4 : 2) > kStreamNtBytes;
  const int sources = g.num_groups + c.B;
  PrefixArgs a = {g, q, scale_log2, streams, out, lse_out, shape_of(c, g), {}};
  lay_out(c, g, a.shape, reinterpret_cast<char*>(workspace), &a.work);
  if (!a.shape.plans && !a.shape.chunks) {
    auto make = [&](auto kernel, int threads) { kernel<<<dim3(1), dim3(threads), 0, st>>>(c, a); };
    if (sources < kFewThreads) make(prefix_items_kernel<kFewThreads, true>, kFewThreads);
    else if (sources <= kHeldSources) make(prefix_items_kernel<kItemThreads, true>, kItemThreads);
    else make(prefix_items_kernel<kItemThreads, false>, kItemThreads);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (c.dtype == 0) return c.D == 64 ? launch_prefix_of<float, 64>(c, a, st) : launch_prefix_of<float, 128>(c, a, st);
  return c.D == 64 ? launch_prefix_of<uint16_t, 64>(c, a, st) : launch_prefix_of<uint16_t, 128>(c, a, st);
}

}  // namespace unique
