// Attention of one new token per sequence where groups of sequences share the pages that their contexts begin with.
//
// softmax(q K^T) V over a prefix and a sequence's own tokens is joined from parts (o, m, l): sums relative to the part's own reference m. The parts of the
// prefix are products: all query heads of a group's members that use a KV head, up to hundreds of rows, times the prefix's keys, read once for all of them; a
// sequence's own pages are the decode kernels' chunks (decode_core.hpp), and their merge joins both.
//
// bf16 caches. A workgroup of four waves takes a chunk of a prefix for a KV head and a tile of rows. Tiles of 64 tokens go straight into the LDS. Both
// products run on v_mfma_f32_32x32x16_bf16 with the queries as columns: S^T = K Q^T leaves a lane with 16 tokens' logits of ONE query (column lane % 32, rows 8 (i / 4) + 4
// (lane / 32) + i % 4), so its softmax needs no other lane but lane ^ 32, and these are the k that the lane supplies to O^T = V^T P^T: probabilities never
// leave their lane. V^T comes out of the LDS by its transposing read. A row of the LDS holds its 16-byte pieces in the order piece ^ f(row), f
// distinct for 8 consecutive rows and even numbers for 4, so neither read meets a bank twice; the pieces are permuted where they are loaded, within a row of memory.
// Probabilities enter the second product rounded to bf16, and their sum does not: 24 bits, in three products, would double the arithmetic, which bounds
// groups of 32 sequences and more, for an error that is of the size of the output's own rounding.
// fp32 caches: the same on v_mfma_f32_32x32x2_f32, whose probabilities stay fp32.
#include <type_traits>

#include "decode_core.hpp"
#include "prefix_plan.hpp"
#include "serving.hpp"

namespace unique {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef const __attribute__((address_space(1))) void* global_ptr_t;
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;

struct Member {
  int seq, group, prefix;  // its sequence, group and the group's prefix pages; seq < 0: none
};

// The member at place i of the batch. Every lane looks at a group's end.
__device__ __forceinline__ Member member_at(const CacheView& c, const unique_prefix_groups& g, int i) {
  const int lane = threadIdx.x % kWave;
  int group = 0;
  for (int g0 = 0; g0 < g.num_groups; g0 += kWave) {
    const bool before = g0 + lane < g.num_groups && g.starts[min(g0 + lane, g.num_groups - 1) + 1] <= i;
    group += __popcll(__ballot(before));
  }
  Member m = {-1, group, 0};
  if (group >= g.num_groups || i - g.starts[group] >= g.max_members) return m;
  m.seq = g.members ? g.members[i] : i;
  if (m.seq >= c.B) m.seq = -1;
  m.prefix = min(max(g.prefix_pages[group], 0), min(g.max_prefix_pages, c.max_pages_hint));
  return m;
}

__device__ __forceinline__ int swizzle(int row) { return (row & 3) * 2 + (row >> 2 & 1); }

// A tile of keys or values in the LDS: kTokens rows of D elements, the pieces of a row permuted.
template <typename T, int D>
struct Tile {
  static constexpr int kRowBytes = D * (int)sizeof(T), kTokens = sizeof(T) == 2 ? 64 : 32;
  static constexpr int kBytes = kTokens * kRowBytes, kLoads = kBytes / (kDecWaves * kWave * 16);  // of a wave
  static constexpr int kLoadTokens = kWave * 16 / kRowBytes;                                      // tokens of a load
  static constexpr int kPieces = kRowBytes / 16;
};

template <typename T, int D>
struct PrefixShared {
  __attribute__((aligned(1024))) char k[2][Tile<T, D>::kBytes];
  __attribute__((aligned(1024))) char v[2][Tile<T, D>::kBytes];
};

// kAcross: waves that share the rows of the workgroup; the others take other tokens of a tile.
template <typename T, int D, int kAcross>
__global__ __launch_bounds__(kDecWaves* kWave, sizeof(T) == 2 ? 2 : 1) void prefix_kernel(CacheView c, PrefixArgs a, PrefixPlan plan,
                                                                                       float* __restrict__ part_ml) {
  using L = Tile<T, D>;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kSteps = D / 16;         // q.k products of a 32-token block (bf16)
  constexpr int kBlocks = D / 32;        // of channels
  constexpr int kAlong = kDecWaves / kAcross;
  constexpr int kHalves = L::kTokens / 32 / kAlong;  // 32-token blocks of a wave in a tile
  static_assert(kHalves >= 1, "a block for every wave");
  constexpr float kRoom = 6.f;           // log2: how far above the largest logit the reference is put
  __shared__ PrefixShared<T, D> sh;

  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 32, half = lane / 32;
  const int across = wave % kAcross, along = wave / kAcross;
  const int hkv = blockIdx.y, G = c.H / c.Hkv, split = blockIdx.z;
  const int group = blockIdx.x / plan.blocks, block = blockIdx.x - group * plan.blocks;
  const int start = max(a.groups.starts[group], 0), size = min(min(a.groups.starts[group + 1], c.B) - start, a.groups.max_members);
  const int prefix = min(max(a.groups.prefix_pages[group], 0), min(plan.chunks * plan.chunk_pages, min(a.groups.max_prefix_pages, c.max_pages_hint)));
  const int begin = split * plan.chunk_pages, end = min(begin + plan.chunk_pages, prefix);
  if (begin >= end || block * plan.rows >= size * G) return;
  const int first = a.groups.members ? a.groups.members[start] : start;

  // this lane's query row
  const int row = block * plan.rows + across * 32 + col;
  const int place = start + row / G;
  const bool live = row < size * G;
  const int seq = live ? (a.groups.members ? a.groups.members[place] : place) : -1;
  const bool mine = seq >= 0 && seq < c.B;
  const int tokens = mine ? c.seq_lens[seq] : 0;  // of this row's sequence
  const T* q = reinterpret_cast<const T*>(a.q) + ((int64_t)(mine ? seq : 0) * c.H + hkv * G + row % G) * D;
  bf16x8_t qb[kBf16 ? kSteps : 1];
  float qf[kBf16 ? 1 : D / 2];
  if constexpr (kBf16) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) qb[s] = as_bf16x8(mine ? load_raw(q + (2 * s + half) * 8) : zero_raw());
  } else {
#pragma unroll
    for (int s = 0; s < D / 8; ++s) {
      const float4 x = mine ? *reinterpret_cast<const float4*>(q + half * (D / 2) + 4 * s) : make_float4(0.f, 0.f, 0.f, 0.f);
      qf[4 * s] = x.x; qf[4 * s + 1] = x.y; qf[4 * s + 2] = x.z; qf[4 * s + 3] = x.w;
    }
  }
  const bool idle = block * plan.rows + across * 32 >= size * G;  // no row of this wave (uniform)

  const int shift = __builtin_ctz(c.S), tile_pages = L::kTokens >> shift;
  const int tiles = (end - begin + tile_pages - 1) / tile_pages;
  const int32_t* table = c.page_table + (int64_t)(first >= 0 && first < c.B ? first : 0) * c.max_pages;

  // Loads of a tile: wave w takes every fourth kilobyte. A page that there is not reads the pool's first page, and does not count.
  const int load_row = lane * 16 / L::kRowBytes, load_piece = lane % L::kPieces;
  auto issue = [&](int t) {
    char* to_k = sh.k[t % 2];
    char* to_v = sh.v[t % 2];
#pragma unroll
    for (int j = 0; j < L::kLoads; ++j) {
      const int at = (j * kDecWaves + wave) * L::kLoadTokens;  // token of the tile
      const int e = begin + t * tile_pages + (at >> shift);
      int page = e < end ? table[e] : 0;
      if (page < 0 || (int64_t)page >= c.num_phys) page = 0;
      const int64_t from = (int64_t)page * c.kv_page_stride + (int64_t)hkv * c.kv_head_stride + (int64_t)((at & (c.S - 1)) + load_row) * D;
      const int piece = load_piece ^ (swizzle(at + load_row) & (L::kPieces - 1));
      const char* k = reinterpret_cast<const char*>(reinterpret_cast<const T*>(c.k_cache) + from) + piece * 16;
      const char* v = reinterpret_cast<const char*>(reinterpret_cast<const T*>(c.v_cache) + from) + piece * 16;
      __builtin_amdgcn_global_load_lds((global_ptr_t)k, (lds_ptr_t)(to_k + at * L::kRowBytes), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((global_ptr_t)v, (lds_ptr_t)(to_v + at * L::kRowBytes), 16, 0, 0);
    }
  };

  float m = kNegBig, l = 0.f;
  f32x16_t acc[kBlocks];
#pragma unroll
  for (int e = 0; e < kBlocks; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;

  issue(0);
  for (int t = 0; t < tiles; ++t) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // the tile has arrived, and everyone is done with the one before
    if (t + 1 < tiles) issue(t + 1);
    if (idle) continue;
    const char* tk = sh.k[t % 2];
    const char* tv = sh.v[t % 2];
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      const int t0 = (along * kHalves + h) * 32;  // the block's first token in the tile
      const int at0 = ((begin + t * tile_pages) << shift) + t0;
      f32x16_t x;
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.f;
      const int krow = t0 + col;
      const char* kr = tk + krow * L::kRowBytes;
      const int sw = swizzle(krow) & (L::kPieces - 1);
      if constexpr (kBf16) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const bf16x8_t ka = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(kr + ((2 * s + half) ^ sw) * 16));
          x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qb[s], x, 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int s = 0; s < D / 8; ++s) {
          const float4 ka = *reinterpret_cast<const float4*>(kr + ((half * (D / 8) + s) ^ sw) * 16);
          x = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.x, qf[4 * s], x, 0, 0, 0);
          x = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.y, qf[4 * s + 1], x, 0, 0, 0);
          x = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.z, qf[4 * s + 2], x, 0, 0, 0);
          x = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.w, qf[4 * s + 3], x, 0, 0, 0);
        }
      }
      // Tokens that do not count: behind the chunk or the row's sequence, or of a page that there is not (pages are whole eights of tokens).
      bool there[4];  // uniform
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int e = (at0 + 8 * n) >> shift;
        const int page = e < end ? table[e] : -1;
        there[n] = page >= 0 && (int64_t)page < c.num_phys;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * n + i] = there[n] && at0 + 8 * n + 4 * half + i < tokens ? x[4 * n + i] * a.scale_log2 : -INFINITY;
      }
      float top = x[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
      if (__any(top > m)) {
        const float mnew = fmaxf(m, with_lane_xor32(top, OpMax()) + kRoom);
        const float alpha = fast_exp2(m - mnew);
        m = mnew;
        l *= alpha;
#pragma unroll
        for (int e = 0; e < kBlocks; ++e)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[e][i] *= alpha;
      }
      float p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = fast_exp2(x[i] - m);
        l += p[i];
      }
      if constexpr (kBf16) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {  // 16 tokens each: 4 half + 0..3 and 8 + 4 half + 0..3 of them are this lane's
          bf16x8_t pb;
#pragma unroll
          for (int i = 0; i < 8; ++i) pb[i] = (__bf16)p[8 * s + i];
#pragma unroll
          for (int e = 0; e < kBlocks; ++e) {
            // lane i of 16 asks for token i / 4, channels 4 (i % 4) + ..., and gets channel i of the four tokens
            s16x4_t part[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              const int token = t0 + 16 * s + 8 * n + 4 * half + lane % 16 / 4;
              const int channel = e * 32 + lane % 32 / 16 * 16 + lane % 4 * 4;
              const char* from = tv + token * L::kRowBytes + ((channel / 8) ^ (swizzle(token) & (L::kPieces - 1))) * 16 + channel % 8 * 2;
              part[n] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)from);
              if (!there[2 * s + n]) part[n] = s16x4_t{0, 0, 0, 0};  // whatever the pool's first page holds
            }
            typedef short s16x8_t __attribute__((ext_vector_type(8)));
            const s16x8_t va = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
            acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, va), pb, acc[e], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int token = t0 + 8 * (i / 4) + 4 * half + i % 4;
          const char* vr = tv + token * L::kRowBytes;
#pragma unroll
          for (int e = 0; e < kBlocks; ++e) {
            const int channel = e * 32 + col;
            const float there_v = *reinterpret_cast<const float*>(vr + ((channel / 4) ^ swizzle(token)) * 16 + channel % 4 * 4);
            const float va = there[i / 4] ? there_v : 0.f;
            acc[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(va, p[i], acc[e], 0, 0, 0);
          }
        }
      }
    }
  }

  l = with_lane_xor32(l, OpSum());
  if constexpr (kAlong > 1) {  // the waves that took other tokens of the same rows
    static_assert(kAlong == 2, "two waves");
    __syncthreads();
    float* o = reinterpret_cast<float*>(&sh) + across * (32 * D + 64);
    if (along == 1) {
#pragma unroll
      for (int e = 0; e < kBlocks; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[(e * 16 + i) * 64 + lane] = acc[e][i];
      if (half == 0) { o[32 * D + col] = m; o[32 * D + 32 + col] = l; }
    }
    __syncthreads();
    if (along == 1) return;
    const float m2 = o[32 * D + col], l2 = o[32 * D + 32 + col], M = fmaxf(m, m2);
    const float s1 = fast_exp2(m - M), s2 = fast_exp2(m2 - M);
    m = M;
    l = l * s1 + l2 * s2;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[e][i] = acc[e][i] * s1 + o[(e * 16 + i) * 64 + lane] * s2;
  }
  if (!live) return;
  const int64_t slot = (((int64_t)place * c.Hkv + hkv) * plan.parts() + split) * G + row % G;
  float* out = a.partials + slot * D;
#pragma unroll
  for (int e = 0; e < kBlocks; ++e)
#pragma unroll
    for (int n = 0; n < 4; ++n)
      *reinterpret_cast<float4*>(out + e * 32 + 8 * n + 4 * half) =
          make_float4(acc[e][4 * n], acc[e][4 * n + 1], acc[e][4 * n + 2], acc[e][4 * n + 3]);
  if (half == 0) *reinterpret_cast<float2*>(part_ml + slot * 2) = make_float2(m, l);
}

// A member's own pages, as the decode kernels take them.
template <typename T, int D, int S, int G, bool kNT>
__global__ __launch_bounds__(kDecWaves* kWave) void prefix_own_kernel(CacheView c, PrefixArgs a, PrefixPlan plan, float* __restrict__ part_ml) {
  __shared__ DecodeShared<T, D, G> sh;
  const int split = blockIdx.x, hkv = blockIdx.y, i = blockIdx.z;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const Member of = member_at(c, a.groups, i);
  if (of.seq < 0) return;
  const int b = of.seq, N = c.seq_lens[b], P = min((N + S - 1) / S, c.max_pages_hint);
  const int begin = of.prefix + split * plan.own_pages, end = min(begin + plan.own_pages, P);
  if (begin >= end) return;
  const int shared = (of.prefix + plan.chunk_pages - 1) / plan.chunk_pages;
  const ChunkOut<T> to = {a.partials, part_ml, reinterpret_cast<T*>(a.out), a.lse_out, 2};
  const Chunk chunk = {hkv, b, begin, end, N, ((int64_t)i * c.Hkv + hkv) * plan.parts() + shared + split};
  auto lookup = [&](int e, bool, int& phys, int& ntok) {
    const int ph = c.page_table[(int64_t)b * c.max_pages + e];
    if (ph >= 0 && (int64_t)ph < c.num_phys) {
      phys = ph;
      ntok = min(S, N - e * S);
    }
  };
  decode_chunk<D, S, G, kNT>(c, reinterpret_cast<const T*>(a.q), chunk, wave, lane, lookup, a.scale_log2, to, sh);
}

template <typename T, int D, int G>
__global__ __launch_bounds__(kMergeWaves* kWave) void prefix_merge_kernel(CacheView c, PrefixArgs a, PrefixPlan plan, const float* __restrict__ part_ml) {
  __shared__ MergeShared<kMergeWaves, D> sh;
  const int h = blockIdx.x, i = blockIdx.y;
  const Member of = member_at(c, a.groups, i);
  if (of.seq < 0) return;
  const int P = min((c.seq_lens[of.seq] + c.S - 1) / c.S, c.max_pages_hint);
  const int parts = (of.prefix + plan.chunk_pages - 1) / plan.chunk_pages +
                    min((max(P - of.prefix, 0) + plan.own_pages - 1) / plan.own_pages, plan.own_chunks);
  const int have = plan.parts();
  merge_chunks<T, D, G, kMergeWaves>(c, of.seq, h, ((int64_t)i * c.Hkv + h / G) * have, have, [&] { return parts; }, a.partials, part_ml,
                                     reinterpret_cast<T*>(a.out), a.lse_out, sh);
}

template <typename T, int D, int S, int G>
hipError_t launch_t(const CacheView& c, const PrefixArgs& a, const PrefixPlan& plan, float* part_ml, bool nt, hipStream_t st) {
  if (plan.chunks > 0) {
    auto go = [&](auto kernel) {
      kernel<<<dim3(a.groups.num_groups * plan.blocks, c.Hkv, plan.chunks), dim3(kDecWaves * kWave), 0, st>>>(c, a, plan, part_ml);
      return hipGetLastError();
    };
    hipError_t e;
    if constexpr (sizeof(T) == 2) e = plan.rows == 64 ? go(prefix_kernel<T, D, 2>) : go(prefix_kernel<T, D, 4>);
    else e = go(prefix_kernel<T, D, 4>);
    if (e != hipSuccess) return e;
  }
  if (plan.own_chunks > 0) {
    auto go = [&](auto kernel) { kernel<<<dim3(plan.own_chunks, c.Hkv, c.B), dim3(kDecWaves * kWave), 0, st>>>(c, a, plan, part_ml); };
    if (nt) go(prefix_own_kernel<T, D, S, G, true>);
    else go(prefix_own_kernel<T, D, S, G, false>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  prefix_merge_kernel<T, D, G><<<dim3(c.H, c.B), dim3(kMergeWaves * kWave), 0, st>>>(c, a, plan, part_ml);
  return hipGetLastError();
}

template <typename T, int D, int S>
hipError_t dispatch_g(const CacheView& c, const PrefixArgs& a, const PrefixPlan& plan, float* part_ml, bool nt, hipStream_t st) {
  switch (c.H / c.Hkv) {
    case 1: return launch_t<T, D, S, 1>(c, a, plan, part_ml, nt, st);
    case 2: return launch_t<T, D, S, 2>(c, a, plan, part_ml, nt, st);
    case 4: return launch_t<T, D, S, 4>(c, a, plan, part_ml, nt, st);
    case 8: return launch_t<T, D, S, 8>(c, a, plan, part_ml, nt, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

// One translation unit per element type and head dimension: UNIQUE_ELEM, UNIQUE_DIM.
template <>
hipError_t launch_prefix_of<UNIQUE_ELEM, UNIQUE_DIM>(const CacheView& c, const PrefixArgs& a, const PrefixPlan& plan, float* part_ml, bool nt,
                                                     hipStream_t st) {
  switch (c.S) {
    case 8: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 8>(c, a, plan, part_ml, nt, st);
    case 16: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 16>(c, a, plan, part_ml, nt, st);
    case 32: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 32>(c, a, plan, part_ml, nt, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace unique
