// Attention of one new token per sequence where groups of sequences share the pages that their contexts begin with.
//
// softmax(q K^T) V over a prefix and a sequence's own tokens is joined from parts (o, m, l): sums relative to the part's own reference m. The parts of the
// prefix are products: all query heads of a group's members that use a KV head, up to hundreds of rows, times the prefix's keys, read once for all of them. A
// sequence's own pages are the same with the few rows of one member. What a workgroup takes is an item (prefix_launch.hip): a run of pages times a block of rows.
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

typedef short s16x8_t __attribute__((ext_vector_type(8)));

// kAcross: waves that share the rows of the workgroup; the others take other tokens of a tile.
template <typename T, int D, int kAcross>
__global__ __launch_bounds__(kDecWaves* kWave, 2) void prefix_kernel(CacheView c, PrefixArgs a) {
  using L = Tile<T, D>;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kSteps = D / 16;         // q.k products of a 32-token block (bf16)
  constexpr int kBlocks = D / 32;        // of channels
  constexpr int kAlong = kDecWaves / kAcross;
  constexpr int kHalves = L::kTokens / 32 / kAlong;  // 32-token blocks of a wave in a tile
  static_assert(kHalves >= 1, "a block for every wave");
  constexpr float kRoom = 6.f;           // log2: how far above the largest logit the reference is put
  __shared__ PrefixShared<T, D> sh;

  const int hkv = blockIdx.x & (c.Hkv - 1), index = blockIdx.x / c.Hkv, G = c.H / c.Hkv;
  const PrefixItem item = a.work.item[index];
  if (index >= *a.work.num_items) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 32, half = lane / 32;
  const int across = wave % kAcross, along = wave / kAcross;

  // pages of the item, 64 at a time in the lanes
  const int shift = __builtin_ctz(c.S), tile_pages = L::kTokens >> shift;
  const int tiles = (item.end - item.begin + tile_pages - 1) / tile_pages;
  const int32_t* table = c.page_table + (int64_t)(item.seq >= 0 && item.seq < c.B ? item.seq : 0) * c.max_pages;
  auto window = [&](int e0) { return e0 + lane < item.end ? table[e0 + lane] : -1; };
  int ids = window(item.begin), ids_next = window(item.begin + kWave);

  // this lane's query row
  const int row = across * 32 + col;
  const bool live = row < item.rows;
  const int place = item.place + (live ? row : 0) / G;
  const int seq = a.groups.members ? a.groups.members[place] : place;
  const bool mine = live && seq >= 0 && seq < c.B;
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
  const bool idle = across * 32 >= item.rows;  // no row of this wave (uniform)
  // tokens that all rows of the wave have
  const int all_have = (int)wave_allreduce_minmax<false>((uint32_t)(live ? min(tokens, item.limit) : INT32_MAX));

  // Loads of a tile: wave w takes every fourth kilobyte. A page that there is not reads the pool's first page, and does not count. The pieces' order in a row is
  // the same in all of a wave's loads.
  const int load_row = lane * 16 / L::kRowBytes;
  const int load_off = load_row * L::kRowBytes + ((lane % L::kPieces) ^ (swizzle(wave * L::kLoadTokens + load_row) & (L::kPieces - 1))) * 16;
  const char* k_head = reinterpret_cast<const char*>(reinterpret_cast<const T*>(c.k_cache) + (int64_t)hkv * c.kv_head_stride);
  const char* v_head = reinterpret_cast<const char*>(reinterpret_cast<const T*>(c.v_cache) + (int64_t)hkv * c.kv_head_stride);
  const int64_t page_bytes = c.kv_page_stride * (int64_t)sizeof(T);
  unsigned long long valid = 0, valid_ahead = 0;  // of the pages in the lanes, which are there: of the tile in work and of the one ahead
  auto issue = [&](int t) {
    const int at_page = t * tile_pages;
    if (at_page > 0 && at_page % kWave == 0) {  // uniform
      ids = ids_next;
      ids_next = window(item.begin + at_page + kWave);
    }
    valid_ahead = __ballot(ids >= 0 && (int64_t)ids < c.num_phys);
    valid_ahead = (valid_ahead >> (at_page % kWave)) & ((1ull << tile_pages) - 1);
    char* to_k = sh.k[t % 2];
    char* to_v = sh.v[t % 2];
#pragma unroll
    for (int j = 0; j < L::kLoads; ++j) {
      const int at = (j * kDecWaves + wave) * L::kLoadTokens, e = at >> shift;  // token and page of the tile
      const int id = __builtin_amdgcn_readlane(ids, (at_page + e) % kWave);
      const int64_t from = (valid_ahead >> e & 1 ? id : 0) * page_bytes + (at & (c.S - 1)) * L::kRowBytes;
      __builtin_amdgcn_global_load_lds((global_ptr_t)(k_head + from + load_off), (lds_ptr_t)(to_k + at * L::kRowBytes), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((global_ptr_t)(v_head + from + load_off), (lds_ptr_t)(to_v + at * L::kRowBytes), 16, 0, 0);
    }
  };

  float m = kNegBig, l = 0.f;
  f32x16_t acc[kBlocks];
#pragma unroll
  for (int e = 0; e < kBlocks; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;

  // 32 tokens from t0 of the tile on; at0: the first one's number. kFull: all of them count for all rows.
  auto block = [&](auto full, const char* tk, const char* tv, int t0, int at0) {
    constexpr bool kFull = decltype(full)::value;
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
    bool there[4];  // pages are whole eights of tokens
    if constexpr (!kFull) {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        there[n] = valid >> ((t0 + 8 * n) >> shift) & 1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = at0 + 8 * n + 4 * half + i;
          x[4 * n + i] = there[n] && at < tokens && at < item.limit ? x[4 * n + i] : -INFINITY;
        }
      }
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
    top *= a.scale_log2;
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
      p[i] = fast_exp2(fmaf(x[i], a.scale_log2, -m));
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
            if constexpr (!kFull) {  // slots without a token may hold anything
#pragma unroll
              for (int i = 0; i < 4; ++i)
                part[n][i] = there[2 * s + n] && at0 + 16 * s + 8 * n + 4 * half + i < item.limit ? part[n][i] : (short)0;
            }
          }
          const s16x8_t va = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
          acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, va), pb, acc[e], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int token = 8 * (i / 4) + 4 * half + i % 4;
        const char* vr = tv + (t0 + token) * L::kRowBytes;
#pragma unroll
        for (int e = 0; e < kBlocks; ++e) {
          const int channel = e * 32 + col;
          float va = *reinterpret_cast<const float*>(vr + ((channel / 4) ^ swizzle(t0 + token)) * 16 + channel % 4 * 4);
          if constexpr (!kFull) va = there[i / 4] && at0 + token < item.limit ? va : 0.f;
          acc[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(va, p[i], acc[e], 0, 0, 0);
        }
      }
    }
  };

  issue(0);
  for (int t = 0; t < tiles; ++t) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // the tile has arrived, and everyone is done with the one before
    valid = valid_ahead;
    if (t + 1 < tiles) issue(t + 1);
    if (idle) continue;
    const char* tk = sh.k[t % 2];
    const char* tv = sh.v[t % 2];
    const int tile0 = (item.begin + t * tile_pages) << shift;
    const bool full = valid == (1ull << tile_pages) - 1 && tile0 + L::kTokens <= all_have;
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      const int t0 = (along * kHalves + h) * 32;
      if (full) block(std::true_type(), tk, tv, t0, tile0 + t0);
      else block(std::false_type(), tk, tv, t0, tile0 + t0);
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
  const int64_t slot = (int64_t)hkv * a.shape.max_rows + item.part + row;
  float* out = a.work.part_o + slot * D;
#pragma unroll
  for (int e = 0; e < kBlocks; ++e)
#pragma unroll
    for (int n = 0; n < 4; ++n)
      *reinterpret_cast<float4*>(out + e * 32 + 8 * n + 4 * half) =
          make_float4(acc[e][4 * n], acc[e][4 * n + 1], acc[e][4 * n + 2], acc[e][4 * n + 3]);
  if (half == 0) *reinterpret_cast<float2*>(a.work.part_ml + slot * 2) = make_float2(m, l);
}

// A wave joins the parts of a (member, query head): o = sum of 2^(m_j - M) o_j over sum of 2^(m_j - M) l_j. Lane s takes the pair (m, l) of part s; D / 4 lanes
// read a part's row, so that a load covers 2 or 4 parts, and eight loads are in flight.
template <typename T, int D>
__global__ __launch_bounds__(kMergeWaves* kWave) void prefix_merge_kernel(CacheView c, PrefixArgs a) {
  constexpr int kLanes = D / 4, kParts = kWave / kLanes, kAhead = 8;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t item = (int64_t)blockIdx.x * kMergeWaves + wave;
  if (item >= (int64_t)c.B * c.H) return;  // (no barrier below)
  const int i = (int)(item / c.H), h = (int)(item - (int64_t)i * c.H), G = c.H / c.Hkv, hkv = h / G;
  const PrefixMember of = a.work.member[i];
  if (of.seq < 0) return;
  const int n = of.count + of.own_count;
  const int64_t base = (int64_t)hkv * a.shape.max_rows + h % G;
  auto row_of = [&](int s) { return base + (s < of.count ? of.part + (int64_t)s * of.step : of.own_part + (int64_t)(s - of.count) * G); };
  const float2* ml = reinterpret_cast<const float2*>(a.work.part_ml);
  const float2 none = make_float2(kNegBig, 0.f);

  const float2 first = lane < n ? ml[row_of(lane)] : none;
  float M = first.x;
  for (int s0 = kWave; s0 < n; s0 += kWave) M = fmaxf(M, s0 + lane < n ? ml[row_of(s0 + lane)].x : kNegBig);
  M = group_allreduce<kWave>(M, OpMax());
  float L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  const int sub = lane / kLanes, channel = lane % kLanes * 4;
  for (int s0 = 0; s0 < n; s0 += kWave) {
    const float2 p = s0 == 0 ? first : (s0 + lane < n ? ml[row_of(s0 + lane)] : none);
    const float scale = fast_exp2(p.x - M);
    L = fmaf(p.y, scale, L);
    const int here = min(kWave, n - s0);
    for (int j0 = 0; j0 < here; j0 += kParts * kAhead) {
      float4 v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) v[u] = *reinterpret_cast<const float4*>(a.work.part_o + row_of(min(s0 + j0 + u * kParts + sub, n - 1)) * D + channel);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int j = j0 + u * kParts + sub;
        const float of_j = __shfl(scale, j % kWave, kWave);  // by all lanes, as any may be asked for its own
        const float sc = j < here ? of_j : 0.f;
        o[0] = fmaf(v[u].x, sc, o[0]);
        o[1] = fmaf(v[u].y, sc, o[1]);
        o[2] = fmaf(v[u].z, sc, o[2]);
        o[3] = fmaf(v[u].w, sc, o[3]);
      }
    }
  }
  L = group_allreduce<kWave>(L, OpSum());
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = cross_group_allreduce<kLanes>(o[k], OpSum());
  const bool any = L > 0.f;
  if (sub == 0) {
    T* dst = reinterpret_cast<T*>(a.out) + ((int64_t)of.seq * c.H + h) * D + channel;
#pragma unroll
    for (int k = 0; k < 4; ++k) store_elem(dst + k, any ? o[k] / L : 0.f);
    if (a.lse_out && lane == 0) a.lse_out[(int64_t)of.seq * c.H + h] = any ? (M + log2f(L)) * kLn2 : -INFINITY;
  }
}

}  // namespace

// One translation unit per element type and head dimension: UNIQUE_ELEM, UNIQUE_DIM.
template <>
hipError_t launch_prefix_of<UNIQUE_ELEM, UNIQUE_DIM>(const CacheView& c, const PrefixArgs& a, hipStream_t st) {
  using T = UNIQUE_ELEM;
  auto go = [&](auto kernel) {
    kernel<<<dim3(c.Hkv * a.shape.max_items), dim3(kDecWaves * kWave), 0, st>>>(c, a);
    return hipGetLastError();
  };
  hipError_t e;
  if constexpr (sizeof(T) == 2) e = a.shape.rows == 64 ? go(prefix_kernel<T, UNIQUE_DIM, 2>) : go(prefix_kernel<T, UNIQUE_DIM, 4>);
  else e = go(prefix_kernel<T, UNIQUE_DIM, 4>);
  if (e != hipSuccess) return e;
  const int64_t outs = (int64_t)c.B * c.H;
  prefix_merge_kernel<T, UNIQUE_DIM><<<dim3((unsigned)((outs + kMergeWaves - 1) / kMergeWaves)), dim3(kMergeWaves * kWave), 0, st>>>(c, a);
  return hipGetLastError();
}

}  // namespace unique
