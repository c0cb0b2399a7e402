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
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t lds_addr_t;  // byte address in the LDS
typedef const __attribute__((address_space(3))) char* lds_char_t;
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;

__device__ __forceinline__ int swizzle(int row) { return (row & 3) * 2 + (row >> 2 & 1); }

// 16 bytes a lane from base + off into the LDS, lane after lane from `to` on. In assembly, as the compiler would otherwise wait for all loads before every
// transposing read; nothing is written but the LDS, and who reads that waits by wait_units.
template <bool kNT>
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t off, lds_addr_t to) {
  if constexpr (kNT) asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(off), "s"(base), "s"(to) : "memory");
  else asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(to) : "memory");
}

// A unit is a tile of keys or of values: kTokens rows of D elements, the 16-byte pieces of a row permuted.
template <typename T, int D>
struct Unit {
  static constexpr int kRowBytes = D * (int)sizeof(T), kTokens = sizeof(T) == 2 ? 64 : 32;
  static constexpr int kBytes = kTokens * kRowBytes, kLoads = kBytes / (kDecWaves * kWave * 16);  // of a wave
  static constexpr int kLoadTokens = kWave * 16 / kRowBytes;                                      // tokens of a load
  static constexpr int kPieces = kRowBytes / 16;
  static constexpr int kRing = 80 * 1024 / kBytes < 6 ? 80 * 1024 / kBytes : 6;                   // units in the LDS
};

// Until all but the newest `left` units (kMost at most) have arrived.
template <int kMost, int kLoads>
__device__ __forceinline__ void wait_units(int left) {
  if (left >= kMost) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMost * kLoads) : "memory");
  else if constexpr (kMost > 0) wait_units<kMost - 1, kLoads>(left);
}

// kAcross: waves that share the rows of the workgroup; the others take other tokens of a tile.
template <typename T, int D, int kAcross, bool kNT>
__global__ __launch_bounds__(kDecWaves* kWave, 2) void prefix_kernel(CacheView c, PrefixArgs a) {
  using L = Unit<T, D>;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kSteps = D / 16;         // q.k products of a 32-token block (bf16)
  constexpr int kBlocks = D / 32;        // of channels
  constexpr int kAlong = kDecWaves / kAcross;
  constexpr int kHalves = L::kTokens / 32 / kAlong;  // 32-token blocks of a wave in a tile
  static_assert(kHalves >= 1, "a block for every wave");
  constexpr float kRoom = 6.f;           // log2: how far above the largest logit the reference is put
  constexpr int kIds = 4;                // page ids in a lane
  __shared__ __attribute__((aligned(1024))) char ring[L::kRing * L::kBytes];

  const int hkv = blockIdx.x & (c.Hkv - 1), index = blockIdx.x / c.Hkv, G = c.H / c.Hkv;
  const PrefixItem item = a.work.item[index];
  if (index >= *a.work.num_items) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 32, half = lane / 32;
  const int across = wave % kAcross, along = wave / kAcross;

  // pages of the item, kIds * 64 at a time in the lanes
  const int shift = __builtin_ctz(c.S), tile_pages = L::kTokens >> shift;
  const int tiles = (item.end - item.begin + tile_pages - 1) / tile_pages;
  const int32_t* table = c.page_table + (int64_t)(item.seq >= 0 && item.seq < c.B ? item.seq : 0) * c.max_pages;
  int held[kIds], ids = -1;
  auto look_up = [&](int e0) {
#pragma unroll
    for (int i = 0; i < kIds; ++i) held[i] = e0 + i * kWave + lane < item.end ? table[e0 + i * kWave + lane] : -1;
    // The wait is here and not where an id is used, where all that is on its way to the LDS would be waited for as well.
    asm volatile("" : "+v"(held[0]), "+v"(held[1]), "+v"(held[2]), "+v"(held[3]));
  };
  look_up(item.begin);

  // Loads of a unit: wave w takes every fourth kilobyte. A page that there is not reads the pool's first page, and does not count. The pieces' order in a
  // row is the same in all of a wave's loads.
  const int load_row = lane * 16 / L::kRowBytes;
  const uint32_t load_off = load_row * L::kRowBytes + ((lane % L::kPieces) ^ (swizzle(wave * L::kLoadTokens + load_row) & (L::kPieces - 1))) * 16;
  const char* heads[2] = {reinterpret_cast<const char*>(reinterpret_cast<const T*>(c.k_cache) + (int64_t)hkv * c.kv_head_stride),
                          reinterpret_cast<const char*>(reinterpret_cast<const T*>(c.v_cache) + (int64_t)hkv * c.kv_head_stride)};
  const int64_t page_bytes = c.kv_page_stride * (int64_t)sizeof(T);
  const lds_addr_t ring_at = (lds_addr_t)(uintptr_t)(lds_char_t)ring;
  auto pages_there = [&](int t) {  // of tile t, one bit each (uniform)
    const int at_page = t * tile_pages;
    if (at_page % kWave == 0) {
      if (at_page > 0 && at_page % (kIds * kWave) == 0) look_up(item.begin + at_page);
      const int i = at_page / kWave % kIds;
      ids = i == 0 ? held[0] : (i == 1 ? held[1] : (i == 2 ? held[2] : held[3]));
    }
    return (uint32_t)(__ballot((uint32_t)ids < (uint32_t)min(c.num_phys, (int64_t)INT32_MAX)) >> (at_page % kWave)) & ((1u << tile_pages) - 1);
  };
  uint32_t there_ahead = 0;  // of the newest tile
  auto issue = [&](int unit, int slot) {
    const int t = unit / 2;
    if (unit % 2 == 0) there_ahead = pages_there(t);
    const lds_addr_t to = ring_at + slot * L::kBytes;
#pragma unroll
    for (int j = 0; j < L::kLoads; ++j) {
      const int at = (j * kDecWaves + wave) * L::kLoadTokens, e = at >> shift;  // token and page of the tile
      const int id = __builtin_amdgcn_readlane(ids, (t * tile_pages + e) % kWave);
      const int64_t from = (there_ahead >> e & 1 ? id : 0) * page_bytes + (at & (c.S - 1)) * L::kRowBytes;
      load_to_lds<kNT>(heads[unit % 2] + from, load_off, to + at * L::kRowBytes);
    }
  };

  // This lane's query row; one that there is not takes another's query, and nobody reads what becomes of it (a column of the products is for itself).
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
    for (int s = 0; s < kSteps; ++s) qb[s] = as_bf16x8(load_raw(q + (2 * s + half) * 8));
  } else {
#pragma unroll
    for (int s = 0; s < D / 8; ++s) {
      const float4 x = *reinterpret_cast<const float4*>(q + half * (D / 2) + 4 * s);
      qf[4 * s] = x.x; qf[4 * s + 1] = x.y; qf[4 * s + 2] = x.z; qf[4 * s + 3] = x.w;
    }
  }
  // The queries are waited for here, not in every turn of the loop.
  if constexpr (kBf16) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) asm volatile("" : "+v"(qb[s]));
  } else {
#pragma unroll
    for (int s = 0; s < D / 2; ++s) asm volatile("" : "+v"(qf[s]));
  }
  const bool idle = across * 32 >= item.rows;  // no row of this wave (uniform)
  // tokens that all rows of the wave have
  const int all_have =
      __builtin_amdgcn_readfirstlane((int)wave_allreduce_minmax<false>((uint32_t)(live ? min(tokens, item.limit) : INT32_MAX)));

  float m = kNegBig, l = 0.f;
  f32x16_t acc[kBlocks];
#pragma unroll
  for (int e = 0; e < kBlocks; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;

  // Where a lane reads, behind a unit's beginning. Keys: token `col`, pieces (2 s + half) of step s, of which four follow from each
  // other by the permutation (fp32: pieces half * D / 8 + s, eight). Values, bf16: lane i of 16 asks for token i / 4, channels 4 (i % 4) + ..., and gets
  // channel i of the four tokens; blocks of channels two apart follow from each other. fp32: channels `col` of each block, token i % 4 + 4 half.
  constexpr int kWays = kBf16 ? 4 : 8;
  const int mine0 = along * kHalves * 32;  // the wave's first token in a tile
  lds_addr_t k_at[kWays], v_at[kBf16 ? 2 : 4];
#pragma unroll
  for (int s = 0; s < kWays; ++s) {
    const int piece = (kBf16 ? 2 * s + half : half * (D / 8) + s) ^ (swizzle(col) & (L::kPieces - 1));
    k_at[s] = ring_at + (mine0 + col) * L::kRowBytes + piece * 16;
  }
  if constexpr (kBf16) {
    const int token = 4 * half + lane % 16 / 4;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int channel = e * 32 + lane % 32 / 16 * 16 + lane % 4 * 4;
      v_at[e] = ring_at + (mine0 + token) * L::kRowBytes + ((channel / 8) ^ (swizzle(token) & (L::kPieces - 1))) * 16 + channel % 8 * 2;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int token = 4 * half + i;
      v_at[i] = ring_at + (mine0 + token) * L::kRowBytes + ((col / 4) ^ swizzle(token)) * 16 + col % 4 * 4;
    }
  }

  float p[kHalves][16];  // logits, then probabilities
  bf16x8_t pb[kBf16 ? kHalves : 1][2];
  // Products take their operands from the LDS in groups, the next group on its way while one is multiplied (left to itself the compiler reads one operand
  // at a time and waits for it).
  auto keys = [&](int slot) {
    constexpr int kGroup = kBf16 ? 4 : 2, kGroups = (kBf16 ? kSteps : D / 8) / kGroup;  // reads of 16 bytes
    u32x4_t ka[2][kGroup];
    lds_char_t at[kWays];
#pragma unroll
    for (int s = 0; s < kWays; ++s) at[s] = (lds_char_t)(uintptr_t)(k_at[s] + slot * L::kBytes);
    auto read = [&](int n, u32x4_t(&to)[kGroup]) {
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        const int s = n % kGroups * kGroup + u;
        to[u] = *(__attribute__((address_space(3))) const u32x4_t*)(at[s % kWays] + n / kGroups * 32 * L::kRowBytes + s / kWays * 128);
      }
    };
    read(0, ka[0]);
    f32x16_t x;
#pragma unroll
    for (int n = 0; n < kHalves * kGroups; ++n) {
      if (n + 1 < kHalves * kGroups) read(n + 1, ka[(n + 1) % 2]);
      __builtin_amdgcn_sched_barrier(0);
      if (n % kGroups == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
      }
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        const int s = n % kGroups * kGroup + u;
        if constexpr (kBf16) {
          x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, ka[n % 2][u]), qb[s], x, 0, 0, 0);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) x = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(ka[n % 2][u][i]), qf[4 * s + i], x, 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (n % kGroups == kGroups - 1) {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[n / kGroups][i] = x[i];
      }
    }
  };
  // Softmax of the tile. at0: the number of the wave's first token in it; full: all of its tokens count for all rows (uniform).
  auto weights = [&](bool full, uint32_t there, int at0) {
    if (!full) {
#pragma unroll
      for (int h = 0; h < kHalves; ++h)
#pragma unroll
        for (int n = 0; n < 4; ++n) {  // pages are whole eights of tokens
          const int end = there >> ((mine0 + h * 32 + 8 * n) >> shift) & 1 ? min(tokens, item.limit) : 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) p[h][4 * n + i] = at0 + h * 32 + 8 * n + 4 * half + i < end ? p[h][4 * n + i] : -INFINITY;
        }
    }
    float top = p[0][0];
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, p[h][i]);
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
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[h][i] = fast_exp2(fmaf(p[h][i], a.scale_log2, -m));
        l += p[h][i];
      }
      if constexpr (kBf16) {
#pragma unroll
        for (int i = 0; i < 16; ++i) pb[h][i / 8][i % 8] = (__bf16)p[h][i];
      }
    }
  };
  // Slots without a token may hold anything, so their values are set to zero.
  auto values = [&](bool full, uint32_t there, int at0, int slot) {
    auto end_of = [&](int token) { return there >> ((mine0 + token) >> shift) & 1 ? item.limit : 0; };
    lds_char_t at[kBf16 ? 2 : 4];
#pragma unroll
    for (int i = 0; i < (kBf16 ? 2 : 4); ++i) at[i] = (lds_char_t)(uintptr_t)(v_at[i] + slot * L::kBytes);
    if constexpr (kBf16) {  // a step is 16 tokens, of which 4 half + 0..3 and 8 + 4 half + 0..3 are this lane's
      s16x4_t va[2][kBlocks][2];
      auto read = [&](int n, s16x4_t(&to)[kBlocks][2]) {
#pragma unroll
        for (int e = 0; e < kBlocks; ++e)
#pragma unroll
          for (int u = 0; u < 2; ++u)
            to[e][u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(at[e % 2] + e / 2 * 128 + (16 * n + 8 * u) * L::kRowBytes));
      };
      read(0, va[0]);
#pragma unroll
      for (int n = 0; n < 2 * kHalves; ++n) {
        if (n + 1 < 2 * kHalves) read(n + 1, va[(n + 1) % 2]);
        __builtin_amdgcn_sched_barrier(0);
        if (!full) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int end = end_of(16 * n + 8 * u) - (at0 + 16 * n + 8 * u + 4 * half);  // of the lane's four tokens
#pragma unroll
            for (int e = 0; e < kBlocks; ++e)
#pragma unroll
              for (int i = 0; i < 4; ++i) va[n % 2][e][u][i] = i < end ? va[n % 2][e][u][i] : (short)0;
          }
        }
#pragma unroll
        for (int e = 0; e < kBlocks; ++e) {
          const s16x8_t v = __builtin_shufflevector(va[n % 2][e][0], va[n % 2][e][1], 0, 1, 2, 3, 4, 5, 6, 7);
          acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), pb[n / 2][n % 2], acc[e], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      constexpr int kGroup = 2;  // tokens at a time, of each half
      float va[2][kGroup][kBlocks];
      auto read = [&](int n, float(&to)[kGroup][kBlocks]) {
#pragma unroll
        for (int u = 0; u < kGroup; ++u) {
          const int i = n * kGroup + u;
#pragma unroll
          for (int e = 0; e < kBlocks; ++e)
            to[u][e] = *(__attribute__((address_space(3))) const float*)(at[i % 4] + 8 * (i / 4) * L::kRowBytes + e * 128);
        }
      };
      constexpr int kTurns = 16 * kHalves / kGroup;
      read(0, va[0]);
#pragma unroll
      for (int n = 0; n < kTurns; ++n) {
        if (n + 1 < kTurns) read(n + 1, va[(n + 1) % 2]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < kGroup; ++u) {
          const int i = n * kGroup + u, token = 8 * (i / 4) + i % 4;
          if (!full) {
            const bool here = at0 + token + 4 * half < end_of(token);
#pragma unroll
            for (int e = 0; e < kBlocks; ++e) va[n % 2][u][e] = here ? va[n % 2][u][e] : 0.f;
          }
#pragma unroll
          for (int e = 0; e < kBlocks; ++e) acc[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(va[n % 2][u][e], p[i / 16][i % 16], acc[e], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  // Unit 2 t holds the keys of tile t, unit 2 t + 1 its values. kRing - 1 units are on their way or in work: a unit that has been worked on by all waves, which the
  // barrier tells, is loaded again.
  const int units = 2 * tiles;
  uint32_t there = 0, there_next[L::kRing / 2 + 1];  // pages of the tile in work, and of those behind it
#pragma unroll
  for (int u = 0; u < L::kRing - 1; ++u) {
    if (u < units) issue(u, u);
    if (u % 2 == 0) there_next[u / 2] = there_ahead;
  }
  constexpr int kAhead = L::kRing - 1;             // units in flight, with the one that is waited for
  constexpr int kTilesAhead = (kAhead + 1) / 2;    // tiles whose pages have been looked at
  auto arrive = [&](int unit) {
    wait_units<kAhead - 1, L::kLoads>(units - 1 - unit);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  int slot = 0;
  auto next = [&](int s) { return s + 1 == L::kRing ? 0 : s + 1; };
  auto free_slot = [&](int s) { return s == 0 ? L::kRing - 1 : s - 1; };
  for (int t = 0; t < tiles; ++t) {
    there = there_next[0];
#pragma unroll
    for (int i = 0; i + 1 < kTilesAhead; ++i) there_next[i] = there_next[i + 1];
    const int at0 = ((item.begin + t * tile_pages) << shift) + mine0;
    const bool full = there == (1u << tile_pages) - 1 && at0 - mine0 + L::kTokens <= all_have;
    arrive(2 * t);
    if (2 * t + kAhead < units) issue(2 * t + kAhead, free_slot(slot));
    if (kAhead % 2 == 0) there_next[kTilesAhead - 1] = there_ahead;
    if (!idle) {
      keys(slot);
      weights(full, there, at0);
    }
    slot = next(slot);
    arrive(2 * t + 1);
    if (2 * t + 1 + kAhead < units) issue(2 * t + 1 + kAhead, free_slot(slot));
    if (kAhead % 2 == 1) there_next[kTilesAhead - 1] = there_ahead;
    if (!idle) values(full, there, at0, slot);
    slot = next(slot);
  }

  l = with_lane_xor32(l, OpSum());
  if constexpr (kAlong > 1) {  // the waves that took other tokens of the same rows
    static_assert(kAlong == 2, "two waves");
    static_assert(L::kRing * L::kBytes >= 2 * 4 * (32 * D + 64), "their results fit the ring");
    __syncthreads();
    float* o = reinterpret_cast<float*>(ring) + across * (32 * D + 64);
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
  const int64_t part = (int64_t)hkv * a.shape.max_rows + item.part + row;
  float* out = a.work.part_o + part * D;
#pragma unroll
  for (int e = 0; e < kBlocks; ++e)
#pragma unroll
    for (int n = 0; n < 4; ++n)
      *reinterpret_cast<float4*>(out + e * 32 + 8 * n + 4 * half) =
          make_float4(acc[e][4 * n], acc[e][4 * n + 1], acc[e][4 * n + 2], acc[e][4 * n + 3]);
  if (half == 0) *reinterpret_cast<float2*>(a.work.part_ml + part * 2) = make_float2(m, l);
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
  const bool nt = a.streams != 0;
  if constexpr (sizeof(T) == 2) {
    if (a.shape.rows == 64) e = nt ? go(prefix_kernel<T, UNIQUE_DIM, 2, true>) : go(prefix_kernel<T, UNIQUE_DIM, 2, false>);
    else e = nt ? go(prefix_kernel<T, UNIQUE_DIM, 4, true>) : go(prefix_kernel<T, UNIQUE_DIM, 4, false>);
  } else {
    e = nt ? go(prefix_kernel<T, UNIQUE_DIM, 4, true>) : go(prefix_kernel<T, UNIQUE_DIM, 4, false>);
  }
  if (e != hipSuccess) return e;
  const int64_t outs = (int64_t)c.B * c.H;
  prefix_merge_kernel<T, UNIQUE_DIM><<<dim3((unsigned)((outs + kMergeWaves - 1) / kMergeWaves)), dim3(kMergeWaves * kWave), 0, st>>>(c, a);
  return hipGetLastError();
}

}  // namespace unique
