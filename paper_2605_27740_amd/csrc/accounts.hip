// Accounts of pages from the shares that weigh.hip's kernels write, and the eviction of pages by them.
#include <algorithm>
#include <type_traits>

#include "decode_core.hpp"
#include "weigh.hpp"

namespace unique {
namespace {

constexpr int kAccountThreads = 256;

// The weights of a row's pages: the maximum M and the sum L of its chunks' (m, l) for every head, then, a thread a page,
// sum over the heads of 2^(share - M) / L.
template <int G>
__global__ __launch_bounds__(kAccountThreads) void account_kernel(CacheView c, SplitPlan plan, const float* __restrict__ part_ml,
                                                                  const float* __restrict__ shares, const float* weights_in, float* weights_out,
                                                                  int weight_stride, float decay) {
  __shared__ float s_m[G], s_r[G];
  const int b = blockIdx.z, row = b * c.Hkv + blockIdx.y;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int P = min((c.seq_lens[b] + c.S - 1) / c.S, c.max_pages_hint);
  if ((int)blockIdx.x * kAccountThreads >= P) return;
  const int ns = (P + plan.pages_per_split - 1) / plan.pages_per_split;
  for (int g = wave; g < G; g += kAccountThreads / kWave) {
    const float2* ml = reinterpret_cast<const float2*>(part_ml) + (int64_t)row * plan.num_splits * G + g;
    float M = kNegBig;
    for (int s = lane; s < ns; s += kWave) M = fmaxf(M, ml[(int64_t)s * G].x);
    M = group_allreduce<kWave>(M, OpMax());
    float L = 0.f;
    for (int s = lane; s < ns; s += kWave) {
      const float2 p = ml[(int64_t)s * G];
      L = fmaf(p.y, fast_exp2(p.x - M), L);
    }
    L = group_allreduce<kWave>(L, OpSum());
    if (lane == 0) {
      s_m[g] = M;
      s_r[g] = L > 0.f ? 1.f / L : 0.f;
    }
  }
  __syncthreads();
  const int p = blockIdx.x * kAccountThreads + threadIdx.x;
  if (p >= P) return;
  const float* share = shares + ((int64_t)row * c.max_pages_hint + p) * G;
  float w = 0.f;
#pragma unroll
  for (int g = 0; g < G; ++g) w = fmaf(fast_exp2(share[g] - s_m[g]), s_r[g], w);
  const int64_t at = (int64_t)row * weight_stride + p;
  weights_out[at] = weights_in ? fmaf(decay, weights_in[at], w) : w;
}

// What a page is ranked by: the sum of its accounts over the KV heads in 64 bits, rounded once. First pages: +inf.
__global__ __launch_bounds__(kAccountThreads) void rank_kernel(CacheView c, const float* weights, int weight_stride, int sinks, float* rank,
                                                               int rank_stride, int32_t* pages) {
  const int b = blockIdx.y, p = blockIdx.x * kAccountThreads + threadIdx.x;
  const int P = min((c.seq_lens[b] + c.S - 1) / c.S, c.max_pages_hint);
  if (p == 0) pages[b] = max(P, 0);
  if (p >= P) return;
  double sum = 0.0;
  for (int h = 0; h < c.Hkv; ++h) sum += (double)weights[((int64_t)b * c.Hkv + h) * weight_stride + p];
  rank[(int64_t)b * rank_stride + p] = p < sinks ? INFINITY : (float)sum;
}

constexpr int kCloseThreads = 1024;

// Closes a sequence's rows up to the kept pages, in place or not: kept[] ascends, so that entry i comes from kept[i] >= i and
// a round of the workgroup, which reads before it writes, leaves what later rounds read. blockIdx.x < Hkv: the accounts of a KV
// head; else the page table, the length and the list of freed pages.
__global__ __launch_bounds__(kCloseThreads) void close_kernel(CacheView c, EvictArgs a, const int32_t* __restrict__ kept, int kept_stride,
                                                              const int32_t* __restrict__ kept_count, const int32_t* __restrict__ pages) {
  const int b = blockIdx.y, t = threadIdx.x;
  const int P = pages[b], n = kept_count[b];
  const int32_t* from = kept + (int64_t)b * kept_stride;
  auto close = [&](const auto* in, auto* out, auto vacant) {
    for (int i0 = 0; i0 < P; i0 += kCloseThreads) {
      const int i = i0 + t;
      auto v = vacant;
      if (i < n) v = in[from[i]];
      __syncthreads();
      if (i < P) out[i] = v;
    }
  };
  if ((int)blockIdx.x < c.Hkv) {
    const int64_t row = ((int64_t)b * c.Hkv + blockIdx.x) * a.weight_stride;
    close(a.weights_in + row, a.weights_out + row, 0.f);
    return;
  }
  const int32_t* table = c.page_table + (int64_t)b * c.max_pages;
  int32_t* freed = a.freed_pages + (int64_t)b * a.freed_stride;
  for (int p = t; p < P; p += kCloseThreads) {  // kept pages below p
    int lo = 0, hi = n;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (from[mid] < p) lo = mid + 1;
      else hi = mid;
    }
    if ((lo == n || from[lo] != p) && p - lo < a.freed_stride) freed[p - lo] = table[p];
  }
  for (int i = P - n + t; i < a.freed_stride; i += kCloseThreads) freed[i] = -1;
  const int N = c.seq_lens[b];
  __syncthreads();
  close(table, a.page_table_out + (int64_t)b * c.max_pages, (int32_t)-1);
  if (t == 0) {
    a.freed_count[b] = P - n;
    a.seq_lens_out[b] = N - (P - n) * c.S;
  }
}

size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }
int rank_stride_of(const CacheView& c) { return (c.max_pages_hint + kScoreStrideAlign - 1) / kScoreStrideAlign * kScoreStrideAlign; }

}  // namespace

size_t weigh_floats(const CacheView& c) {
  return decode_partial_floats(c, c.max_pages_hint) + (size_t)c.B * c.H * c.max_pages_hint;
}

hipError_t launch_weigh(const CacheView& c, const WeighArgs& a, hipStream_t stream) {
  const SplitPlan plan = most_splits(c.B * c.Hkv, c.max_pages_hint);
  const int G = c.H / c.Hkv;
  float* part_ml = a.partials + (size_t)c.B * c.Hkv * plan.num_splits * G * c.D;
  float* shares = a.partials + plan_partial_floats(c, plan);
  auto run = [&](auto launch) { return launch(c, a, plan, part_ml, shares, stream); };
  hipError_t e = c.dtype == 0 ? (c.D == 64 ? run(launch_weigh_partial<float, 64>) : run(launch_weigh_partial<float, 128>))
                              : (c.D == 64 ? run(launch_weigh_partial<bf16_t, 64>) : run(launch_weigh_partial<bf16_t, 128>));
  if (e != hipSuccess) return e;
  e = launch_merge(c, nullptr, c.max_pages_hint, plan, a.partials, a.out, a.lse_out, stream);
  if (e != hipSuccess) return e;
  const dim3 grid((c.max_pages_hint + kAccountThreads - 1) / kAccountThreads, c.Hkv, c.B);
  auto account = [&](auto kernel) {
    kernel<<<grid, dim3(kAccountThreads), 0, stream>>>(c, plan, part_ml, shares, a.weights_in, a.weights_out, a.weight_stride, a.decay);
    return hipGetLastError();
  };
  switch (G) {
    case 1: return account(account_kernel<1>);
    case 2: return account(account_kernel<2>);
    case 4: return account(account_kernel<4>);
    case 8: return account(account_kernel<8>);
    default: return hipErrorInvalidValue;
  }
}

size_t evict_bytes(const CacheView& c) {
  return aligned((size_t)c.B * rank_stride_of(c) * sizeof(float)) + aligned((size_t)c.B * c.max_pages_hint * sizeof(int32_t)) +
         2 * aligned((size_t)c.B * sizeof(int32_t));
}

hipError_t launch_evict(const CacheView& c, const EvictArgs& args, hipStream_t stream) {
  EvictArgs a = args;
  a.budget = std::min(a.budget, c.max_pages_hint);
  char* ws = reinterpret_cast<char*>(a.workspace);
  const int rank_stride = rank_stride_of(c);
  float* rank = reinterpret_cast<float*>(ws);
  ws += aligned((size_t)c.B * rank_stride * sizeof(float));
  int32_t* kept = reinterpret_cast<int32_t*>(ws);
  ws += aligned((size_t)c.B * c.max_pages_hint * sizeof(int32_t));
  int32_t* pages = reinterpret_cast<int32_t*>(ws);
  int32_t* kept_count = reinterpret_cast<int32_t*>(ws + aligned((size_t)c.B * sizeof(int32_t)));
  const dim3 grid((c.max_pages_hint + kAccountThreads - 1) / kAccountThreads, c.B);
  rank_kernel<<<grid, dim3(kAccountThreads), 0, stream>>>(c, a.weights_in, a.weight_stride, a.sinks, rank, rank_stride, pages);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  CacheView one = c;  // a row per sequence
  one.Hkv = one.H = 1;
  one.force_recent = a.recent;
  e = launch_select(one, rank, nullptr, rank_stride, a.budget, kept, kept_count, stream);
  if (e != hipSuccess) return e;
  close_kernel<<<dim3(c.Hkv + 1, c.B), dim3(kCloseThreads), 0, stream>>>(c, a, kept, a.budget, kept_count, pages);
  return hipGetLastError();
}

}  // namespace unique
