// The cut of a batch by its lengths (dense_plan.hpp), found on the device by every wave that asks.
#pragma once
#include "decode_core.hpp"
#include "dense_plan.hpp"

namespace unique {
namespace {

// The chunks of a batch, the same in every wave that asks: lane b holds those of sequence b.
struct BatchChunks {
  int len;     // tokens of sequence `lane`
  int pages;
  int chunks;  // per row of that sequence
  int before;  // chunks per head of the sequences before it
};

__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_inclusive_scan(x), kWave - 1); }

// false: no chunk has the index w, or a larger one
__device__ __forceinline__ bool cut_batch(const CacheView& c, int S, int max_chunks, int w, BatchChunks& bc, DenseRound round = {}) {
  const int lane = threadIdx.x % kWave;
  bc.len = lane < c.B ? c.seq_lens[lane] : 0;
  bc.pages = max(0, min((bc.len + S - 1) / S, c.max_pages_hint));
  const int rows = c.B * c.Hkv;
  const int total = wave_sum(bc.pages) * c.Hkv, slots = dense_slots(total, max_chunks, round);
  const bool room = dense_has_room(rows, slots, max_chunks);
  if (w >= (room ? slots + rows : slots)) return false;  // most workgroups of a launch whose bound is far above the lengths
  if (__ballot(lane < c.B && bc.pages != __builtin_amdgcn_readfirstlane(bc.pages)) == 0) {
    bc.chunks = lane < c.B ? dense_even_chunks(bc.pages, rows, slots) : 0;
  } else {
    bc.chunks = dense_row_chunks(bc.pages, dense_rate(total, rows, slots, [&](uint32_t rate) {
      return wave_sum(dense_row_weight(bc.pages, rate, room)) * c.Hkv;
    }));
  }
  bc.before = wave_inclusive_scan(bc.chunks) - bc.chunks;
  return true;
}

// The sequence whose chunks hold the index w as a bit; 0 beyond the last chunk.
__device__ __forceinline__ unsigned long long sequence_of(const CacheView& c, const BatchChunks& bc, int w) {
  return __ballot(w >= bc.before * c.Hkv && w < (bc.before + bc.chunks) * c.Hkv);
}
// The chunk with the index w, of that sequence.
__device__ __forceinline__ Chunk chunk_of(const CacheView& c, const BatchChunks& bc, unsigned long long sequence, int w) {
  const int b = __ffsll(sequence) - 1;
  const int P = __builtin_amdgcn_readlane(bc.pages, b), n = __builtin_amdgcn_readlane(bc.chunks, b);
  const int i = w - __builtin_amdgcn_readlane(bc.before, b) * c.Hkv;  // chunk `split` of head hkv
  const int hkv = i / n, split = i % n, len = (P + n - 1) / n;
  const int begin = split * len, end = min(begin + len, P);
  const int N = __builtin_amdgcn_readlane(bc.len, b);
  return {hkv, b, begin, max(begin, end), N, w};
}

// The merge of a head's chunks.
template <typename T, int D, int G, int kWaves>
__device__ __forceinline__ void merge_cut(const CacheView& c, int b, int h, int max_chunks, DenseRound round, const float* __restrict__ part_o,
                                          const float* __restrict__ part_ml, T* __restrict__ out, float* __restrict__ lse_out,
                                          MergeShared<kWaves, D>& sh) {
  BatchChunks bc;
  cut_batch(c, c.S, max_chunks, 0, bc, round);
  const int n = __builtin_amdgcn_readlane(bc.chunks, b);
  const int64_t base = (int64_t)__builtin_amdgcn_readlane(bc.before, b) * c.Hkv + (int64_t)(h / G) * n;
  merge_chunks<T, D, G, kWaves>(c, b, h, base, n, [&] { return n; }, part_o, part_ml, out, lse_out, sh);
}

}  // namespace
}  // namespace unique
