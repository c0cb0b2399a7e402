// Dense decode of batches whose sequences may differ in length: chunks of nearly equal size from the lengths on the device.
//
// The host knows only the longest sequence, so most_splits cuts every row at the same multiples of 256 pages, and a ragged batch
// leaves some compute units with two full chunks and others with one: 8 sequences of 2000 to 60000 tokens read 811 MB in 142 us,
// 5.7 TB/s, where an even batch reaches 6.7. Here every workgroup adds up the pages of the batch, finds the smallest
// chunk with which the chunks fit the workgroups that run at the same time (or a multiple of them), cuts every row into
// equal chunks not longer than that, and takes the chunk of its index. That batch now takes 128 us, 6.3 TB/s; 32 sequences of 4K
// to 131K tokens (5.7 GB) 1832 before, 911 now. Other sizes: dense_plan.hpp.
#include <type_traits>

#include "dense_cut.hpp"

namespace unique {
namespace {

template <typename T, int D, int S, int G, bool kNT>
__global__ __launch_bounds__(kDecWaves* kWave) void paged_decode_dense_kernel(CacheView c, const T* __restrict__ q, int max_chunks,
                                                                              float scale_log2, float* __restrict__ part_o,
                                                                              float* __restrict__ part_ml) {
  __shared__ DecodeShared<T, D, G> sh;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;  // wave: scalar
  const int w = blockIdx.x;
  BatchChunks bc;
  if (!cut_batch(c, S, max_chunks, w, bc)) return;
  const unsigned long long here = sequence_of(c, bc, w);
  if (here == 0) return;
  const Chunk chunk = chunk_of(c, bc, here, w);
  const int b = chunk.b, N = chunk.N;
  const ChunkOut<T> to = {part_o, part_ml, nullptr, nullptr, 2};
  auto lookup = [&](int e, bool, int& phys, int& ntok) {
    const int ph = c.page_table[(int64_t)b * c.max_pages + e];
    if (ph >= 0 && (int64_t)ph < c.num_phys) {
      phys = ph;
      ntok = min(S, N - e * S);
    }
  };
  decode_chunk<D, S, G, kNT>(c, q, chunk, wave, lane, lookup, scale_log2, to, sh);
}

template <typename T, int D, int G, int kWaves>
__global__ __launch_bounds__(kWaves* kWave) void paged_decode_dense_merge_kernel(CacheView c, int max_chunks,
                                                                                  const float* __restrict__ part_o,
                                                                                  const float* __restrict__ part_ml, T* __restrict__ out,
                                                                                  float* __restrict__ lse_out) {
  __shared__ MergeShared<kWaves, D> sh;
  merge_cut<T, D, G, kWaves>(c, blockIdx.y, blockIdx.x, max_chunks, {}, part_o, part_ml, out, lse_out, sh);
}

template <typename T, int D, int S, int G>
hipError_t launch_t(const CacheView& c, const void* q, float sm_scale, void* out, float* lse, float* partials, hipStream_t st) {
  const int max_chunks = dense_max_chunks(c.B * c.Hkv, c.max_pages_hint);
  float* part_ml = partials + (size_t)max_chunks * G * D;
  auto go = [&](auto kernel) {
    kernel<<<dim3(max_chunks), dim3(kDecWaves * kWave), 0, st>>>(c, reinterpret_cast<const T*>(q), max_chunks,
                                                                 decode_scale_log2(c, sm_scale), partials, part_ml);
  };
  if (decode_streams(c, c.max_pages_hint)) go(paged_decode_dense_kernel<T, D, S, G, true>);
  else go(paged_decode_dense_kernel<T, D, S, G, false>);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  auto merge = [&](auto kernel, int waves) {
    kernel<<<dim3(c.H, c.B), dim3(waves * kWave), 0, st>>>(c, max_chunks, partials, part_ml, reinterpret_cast<T*>(out), lse);
    return hipGetLastError();
  };
  return dense_merge_alone(c.B * c.Hkv) ? merge(paged_decode_dense_merge_kernel<T, D, G, 1>, 1)
                                        : merge(paged_decode_dense_merge_kernel<T, D, G, kMergeWaves>, kMergeWaves);
}

template <typename T, int D, int S>
hipError_t dispatch_g(const CacheView& c, const void* q, float sm_scale, void* out, float* lse, float* partials, hipStream_t st) {
  switch (c.H / c.Hkv) {
    case 1: return launch_t<T, D, S, 1>(c, q, sm_scale, out, lse, partials, st);
    case 2: return launch_t<T, D, S, 2>(c, q, sm_scale, out, lse, partials, st);
    case 4: return launch_t<T, D, S, 4>(c, q, sm_scale, out, lse, partials, st);
    case 8: return launch_t<T, D, S, 8>(c, q, sm_scale, out, lse, partials, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

// One translation unit per element type and head dimension: UNIQUE_ELEM, UNIQUE_DIM.
template <>
hipError_t launch_dense<UNIQUE_ELEM, UNIQUE_DIM>(const CacheView& c, const void* d_q, float sm_scale, void* d_out, float* d_lse_out,
                                                 float* d_partials, hipStream_t st) {
  switch (c.S) {
    case 8: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 8>(c, d_q, sm_scale, d_out, d_lse_out, d_partials, st);
    case 16: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 16>(c, d_q, sm_scale, d_out, d_lse_out, d_partials, st);
    case 32: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 32>(c, d_q, sm_scale, d_out, d_lse_out, d_partials, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace unique
