// Attention over every page that also says how much of it went to each: the decode kernels' chunk code with PageShares, which
// writes, for every page and head, the log2 of the sum of the page's exponentials while they are in registers. K and V are read
// once, as without; the shares are G floats per page beside 2 S D elements of it. The weights need the sums over all chunks
// and come from a pass over the shares behind the merge.
#include <type_traits>

#include "decode_core.hpp"
#include "weigh.hpp"

namespace unique {
namespace {

template <typename T, int D, int S, int G, bool kNT>
__global__ __launch_bounds__(kDecWaves* kWave) void weigh_partial_kernel(CacheView c, const T* __restrict__ q, SplitPlan plan, float scale_log2,
                                                                         float* __restrict__ part_o, float* __restrict__ part_ml,
                                                                         float* __restrict__ shares) {
  __shared__ DecodeShared<T, D, G> sh;
  int split, hkv, b;
  locate_chunk(c, plan, split, hkv, b);
  const int row = b * c.Hkv + hkv;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int begin = split * plan.pages_per_split;
  const int N = c.seq_lens[b];
  const int P = min((N + S - 1) / S, c.max_pages_hint);
  if (begin >= P) return;
  const ChunkOut<T> to = {part_o, part_ml, nullptr, nullptr, 2};
  const Chunk chunk = {hkv, b, begin, min(begin + plan.pages_per_split, P), N, (int64_t)row * plan.num_splits + split};
  auto lookup = [&](int e, bool, int& phys, int& ntok) {
    const int ph = c.page_table[(int64_t)b * c.max_pages + e];
    if (ph >= 0 && (int64_t)ph < c.num_phys) {
      phys = ph;
      ntok = min(S, N - e * S);
    }
  };
  const PageShares<G> tell = {shares + (int64_t)row * c.max_pages_hint * G};
  decode_chunk<D, S, G, kNT>(c, q, chunk, wave, lane, lookup, scale_log2, to, sh, tell);
}

template <typename T, int D, int S, int G>
hipError_t launch_t(const CacheView& c, const WeighArgs& a, const SplitPlan& plan, float* part_ml, float* shares, hipStream_t st) {
  auto go = [&](auto kernel) {
    const dim3 grid = plan.rotate ? dim3(c.Hkv, c.B, plan.num_splits) : dim3(plan.num_splits, c.Hkv, c.B);
    kernel<<<grid, dim3(kDecWaves * kWave), 0, st>>>(c, reinterpret_cast<const T*>(a.q), plan, a.scale_log2, a.partials, part_ml, shares);
  };
  if (decode_streams(c, c.max_pages_hint)) go(weigh_partial_kernel<T, D, S, G, true>);
  else go(weigh_partial_kernel<T, D, S, G, false>);
  return hipGetLastError();
}

template <typename T, int D, int S>
hipError_t dispatch_g(const CacheView& c, const WeighArgs& a, const SplitPlan& plan, float* part_ml, float* shares, hipStream_t st) {
  switch (c.H / c.Hkv) {
    case 1: return launch_t<T, D, S, 1>(c, a, plan, part_ml, shares, st);
    case 2: return launch_t<T, D, S, 2>(c, a, plan, part_ml, shares, st);
    case 4: return launch_t<T, D, S, 4>(c, a, plan, part_ml, shares, st);
    case 8: return launch_t<T, D, S, 8>(c, a, plan, part_ml, shares, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

// One translation unit per element type and head dimension: UNIQUE_ELEM, UNIQUE_DIM.
template <>
hipError_t launch_weigh_partial<UNIQUE_ELEM, UNIQUE_DIM>(const CacheView& c, const WeighArgs& a, const SplitPlan& plan, float* part_ml, float* shares,
                                                         hipStream_t st) {
  switch (c.S) {
    case 8: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 8>(c, a, plan, part_ml, shares, st);
    case 16: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 16>(c, a, plan, part_ml, shares, st);
    case 32: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 32>(c, a, plan, part_ml, shares, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace unique
