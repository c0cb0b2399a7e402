// Which instance of the kernels in prefix.hip a call takes, and the workspace that it needs.
#include "prefix_plan.hpp"
#include "serving.hpp"

namespace unique {
namespace {

PrefixPlan plan_of(const CacheView& c, const unique_prefix_groups& g) {
  return prefix_plan(c.B, c.Hkv, c.H / c.Hkv, c.dtype == 0 ? 4 : 2, c.S, g.num_groups, g.max_members, g.max_prefix_pages, g.max_own_pages);
}
size_t part_floats(const CacheView& c, const PrefixPlan& p) { return (size_t)c.B * c.H * p.parts() * c.D; }

}  // namespace

size_t prefix_floats(const CacheView& c, const unique_prefix_groups& g) {
  const PrefixPlan p = plan_of(c, g);
  return part_floats(c, p) + (size_t)c.B * c.H * p.parts() * 2;
}

hipError_t launch_prefix(const CacheView& c, const PrefixArgs& a, hipStream_t st) {
  const PrefixPlan p = plan_of(c, a.groups);
  float* part_ml = a.partials + part_floats(c, p);
  const bool nt = decode_streams(c, a.groups.max_own_pages);
  if (c.dtype == 0) return c.D == 64 ? launch_prefix_of<float, 64>(c, a, p, part_ml, nt, st) : launch_prefix_of<float, 128>(c, a, p, part_ml, nt, st);
  return c.D == 64 ? launch_prefix_of<uint16_t, 64>(c, a, p, part_ml, nt, st) : launch_prefix_of<uint16_t, 128>(c, a, p, part_ml, nt, st);
}

}  // namespace unique
