// Attention over every page that also says how much of it went to each: the decode kernels' chunk code with PageShares, which
// writes, for every page and head, the log2 of the sum of the page's exponentials while they are in registers. K and V are read
// once, as without; the shares are G floats per page beside 2 S D elements of it. The weights need the sums over all chunks: they
// come from the shares in the kernel that merges the chunks, in workgroups of their own.
#include <type_traits>

#include "dense_cut.hpp"
#include "weigh.hpp"

namespace unique {
namespace {

// A page's part of the attention weights of a head: its share, the log2 of a sum, over the head's whole sum 2^M L; inverse: 1 / L.
__device__ __forceinline__ float add_weight(float w, float share, float M, float inverse) { return fmaf(fast_exp2(share - M), inverse, w); }

// With one chunk to a row there is nothing to merge: the workgroup writes the output and the row's accounts itself.
template <typename T, int D, int S, int G, bool kNT>
__global__ __launch_bounds__(kDecWaves* kWave) void weigh_partial_kernel(CacheView c, WeighArgs a, WeighCut cut, float* __restrict__ part_ml,
                                                                         float* shares) {
  __shared__ DecodeShared<T, D, G> sh;
  const bool alone = cut.max_chunks == 0 && cut.plan.num_splits == 1;
  const ChunkOut<T> to = {a.partials, part_ml, reinterpret_cast<T*>(a.out), a.lse_out, alone ? 1 : 2};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  Chunk chunk;
  if (cut.max_chunks > 0) {
    const int w = blockIdx.x;
    BatchChunks bc;
    if (!cut_batch(c, S, cut.max_chunks, w, bc, cut.round)) return;
    const unsigned long long here = sequence_of(c, bc, w);
    if (here == 0) return;
    chunk = chunk_of(c, bc, here, w);
  } else {
    int split, hkv, b;
    locate_chunk(c, cut.plan, split, hkv, b);
    const int N = c.seq_lens[b], begin = split * cut.plan.pages_per_split;
    const int P = min((N + S - 1) / S, c.max_pages_hint);
    if (begin >= P) {
      write_empty<T, D, G>(c, to, b, hkv);
      return;
    }
    chunk = {hkv, b, begin, min(begin + cut.plan.pages_per_split, P), N, (int64_t)(b * c.Hkv + hkv) * cut.plan.num_splits + split};
  }
  const int b = chunk.b, N = chunk.N;
  auto lookup = [&](int e, bool, int& phys, int& ntok) {
    const int ph = c.page_table[(int64_t)b * c.max_pages + e];
    if (ph >= 0 && (int64_t)ph < c.num_phys) {
      phys = ph;
      ntok = min(S, N - e * S);
    }
  };
  const int64_t row = b * c.Hkv + chunk.hkv;
  const PageShares<G> tell = {shares + row * c.max_pages_hint * G};
  decode_chunk<D, S, G, kNT>(c, reinterpret_cast<const T*>(a.q), chunk, wave, lane, lookup, a.scale_log2, to, sh, tell);
  if (!alone) return;
  float M[G], inverse[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    M[g] = fmaxf(fmaxf(sh.m[0][g], sh.m[1][g]), fmaxf(sh.m[2][g], sh.m[3][g]));
    float L = 0.f;
#pragma unroll
    for (int w = 0; w < kDecWaves; ++w) L = fmaf(sh.l[w][g], fast_exp2(sh.m[w][g] - M[g]), L);
    inverse[g] = L > 0.f ? 1.f / L : 0.f;
  }
  __syncthreads();  // the shares of all waves are written
  for (int p = threadIdx.x; p < chunk.end; p += kDecWaves * kWave) {
    float w = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) w = add_weight(w, tell.at[(int64_t)p * G + g], M[g], inverse[g]);
    const int64_t at = row * a.weight_stride + p;
    a.weights_out[at] = a.weights_in ? fmaf(a.decay, a.weights_in[at], w) : w;
  }
}

constexpr int kFinishThreads = kMergeWaves * kWave;
constexpr int kPagesEach = 2;  // of a thread

// The first H workgroups of a sequence merge a head's chunks, the others add up accounts: of a KV head, kPagesEach pages a thread,
// the sum over its heads of 2^(share - M) / L (add_weight) with the maximum M and the sum L of the chunks' (m, l), which every workgroup forms for itself.
template <typename T, int D, int G>
__global__ __launch_bounds__(kFinishThreads) void weigh_finish_kernel(CacheView c, WeighArgs a, WeighCut cut, const float* __restrict__ part_ml,
                                                                      const float* __restrict__ shares, int parts /*workgroups of a KV head*/) {
  __shared__ MergeShared<kMergeWaves, D> sh;
  __shared__ float s_m[G], s_r[G];
  const int b = blockIdx.y, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const bool merges = (int)blockIdx.x < c.H;
  const int part = merges ? 0 : (blockIdx.x - c.H) % parts, hkv = merges ? blockIdx.x / G : (blockIdx.x - c.H) / parts;
  const int row = b * c.Hkv + hkv, first = part * kFinishThreads * kPagesEach;
  const int P = min((c.seq_lens[b] + c.S - 1) / c.S, c.max_pages_hint);
  if (!merges && first >= P) return;
  int64_t base;
  int n, have;
  if (cut.max_chunks > 0) {
    BatchChunks bc;
    cut_batch(c, c.S, cut.max_chunks, 0, bc, cut.round);
    n = have = __builtin_amdgcn_readlane(bc.chunks, b);
    base = (int64_t)__builtin_amdgcn_readlane(bc.before, b) * c.Hkv + (int64_t)hkv * n;
  } else {
    n = (max(P, 0) + cut.plan.pages_per_split - 1) / cut.plan.pages_per_split;
    have = cut.plan.num_splits;
    base = (int64_t)row * have;
  }
  if (merges) {
    merge_chunks<T, D, G, kMergeWaves>(c, b, blockIdx.x, base, have, [&] { return n; }, a.partials, part_ml, reinterpret_cast<T*>(a.out), a.lse_out, sh);
    return;
  }
  float share[kPagesEach][G], old[kPagesEach];
#pragma unroll
  for (int u = 0; u < kPagesEach; ++u) {  // requested before anything else; the last page again behind it
    const int p = min(first + u * kFinishThreads + (int)threadIdx.x, P - 1);
    const float* from = shares + ((int64_t)row * c.max_pages_hint + p) * G;
#pragma unroll
    for (int g = 0; g < G; ++g) share[u][g] = from[g];
    old[u] = a.weights_in ? a.weights_in[(int64_t)row * a.weight_stride + p] : 0.f;
  }
  for (int g = wave; g < G; g += kMergeWaves) {
    const float2* ml = reinterpret_cast<const float2*>(part_ml) + base * G + g;
    float M = kNegBig;
    for (int s = lane; s < n; s += kWave) M = fmaxf(M, ml[(int64_t)s * G].x);
    M = group_allreduce<kWave>(M, OpMax());
    float L = 0.f;
    for (int s = lane; s < n; s += kWave) {
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
#pragma unroll
  for (int u = 0; u < kPagesEach; ++u) {
    const int p = first + u * kFinishThreads + threadIdx.x;
    float w = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) w = add_weight(w, share[u][g], s_m[g], s_r[g]);
    if (p < P) a.weights_out[(int64_t)row * a.weight_stride + p] = a.weights_in ? fmaf(a.decay, old[u], w) : w;
  }
}

template <typename T, int D, int S, int G>
hipError_t launch_t(const CacheView& c, const WeighArgs& a, const WeighCut& cut, float* part_ml, float* shares, hipStream_t st) {
  auto go = [&](auto kernel) {
    const dim3 grid = cut.max_chunks > 0 ? dim3(cut.max_chunks) : dim3(cut.plan.num_splits, c.Hkv, c.B);
    kernel<<<grid, dim3(kDecWaves * kWave), 0, st>>>(c, a, cut, part_ml, shares);
  };
  if (decode_streams(c, c.max_pages_hint)) go(weigh_partial_kernel<T, D, S, G, true>);
  else go(weigh_partial_kernel<T, D, S, G, false>);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (cut.max_chunks == 0 && cut.plan.num_splits == 1)) return e;
  const int parts = (c.max_pages_hint + kFinishThreads * kPagesEach - 1) / (kFinishThreads * kPagesEach);
  weigh_finish_kernel<T, D, G><<<dim3(c.H + c.Hkv * parts, c.B), dim3(kFinishThreads), 0, st>>>(c, a, cut, part_ml, shares, parts);
  return hipGetLastError();
}

template <typename T, int D, int S>
hipError_t dispatch_g(const CacheView& c, const WeighArgs& a, const WeighCut& cut, float* part_ml, float* shares, hipStream_t st) {
  switch (c.H / c.Hkv) {
    case 1: return launch_t<T, D, S, 1>(c, a, cut, part_ml, shares, st);
    case 2: return launch_t<T, D, S, 2>(c, a, cut, part_ml, shares, st);
    case 4: return launch_t<T, D, S, 4>(c, a, cut, part_ml, shares, st);
    case 8: return launch_t<T, D, S, 8>(c, a, cut, part_ml, shares, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

// One translation unit per element type and head dimension: UNIQUE_ELEM, UNIQUE_DIM.
template <>
hipError_t launch_weigh_of<UNIQUE_ELEM, UNIQUE_DIM>(const CacheView& c, const WeighArgs& a, const WeighCut& cut, float* part_ml, float* shares,
                                                    hipStream_t st) {
  switch (c.S) {
    case 8: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 8>(c, a, cut, part_ml, shares, st);
    case 16: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 16>(c, a, cut, part_ml, shares, st);
    case 32: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 32>(c, a, cut, part_ml, shares, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace unique
