// Attention of one new token per sequence where groups of sequences share the pages that their contexts begin with.
//
// softmax(q K^T) V over a prefix and a sequence's own tokens is joined from parts (o, m, l): sums relative to the part's own reference m. The parts of the
// prefix are products: all query heads of a group's members that use a KV head, up to hundreds of rows, times the prefix's keys, read once for all of them. A
// sequence's own pages are the same with the few rows of one member, and the decode kernels' chunk code takes them. What a workgroup takes is an item (prefix_items.hpp): a run of
// pages times a block of up to 128 query rows, or of a member's own pages.
//
// bf16 caches. Tiles of 64 tokens go straight into the LDS, 80 KB of them on their way at a time. Both
// products run on v_mfma_f32_32x32x16_bf16 with the queries as columns: S^T = K Q^T leaves a lane with 16 tokens' logits of ONE query (column lane % 32, rows 8 (i / 4) + 4
// (lane / 32) + i % 4), so its softmax needs no other lane but lane ^ 32, and these are the k that the lane supplies to O^T = V^T P^T: probabilities never
// leave their lane. V^T comes out of the LDS by its transposing read.
// Probabilities enter the second product with all 24 bits, as three parts of 8 (exactly), three products instead of one: with 8 bits an output whose terms cancel was off by 2^-9 of the
// terms, and two tokens of opposite values whose weights are nearly the same gave 0. us with one product / three: 256 sequences behind 32768 tokens 182 / 271 to 281, 16 behind 131072 100.5 / 108 to 110, 32 behind 8192
// 37.2 / 41.6, six groups of 10 102 / 106. The parts are made just before they are used, for 8 of a lane's 16 tokens at a time; between the products before, where registers end at 64 rows,
// 119 instead of 112 us behind 131072 tokens, 284 instead of 291 behind 32768.
// fp32 caches: the same on v_mfma_f32_32x32x2_f32, whose probabilities stay fp32, with tiles of 32 tokens.
//
// What bounds it, at 8 KV heads of 128 channels, bf16, pages of 16 or 32: the stream of keys and values up to some 30 sequences in a group (16 behind 131072 tokens: 552 MB in 97 us with the plan in
// front, 5.7 TB/s, matrix cores and vector units 36 % busy; six groups of 10 with 8 heads each, 1000 to 50000 tokens, 100 us, 5.4 TB/s), behind it the matrix cores and vector units together (256 behind 32768 tokens:
// 138 GFLOP, with three parts of a probability 276 of products, in 265 to 280 us, of which the last 20 are the members' own 128 MB; matrix cores 58 % busy, vector units 52, and the clock falls with the power that
// they take: 312 us in a long run).
// Own pages by the same way through the LDS as prefixes (measured with one part): 32 x 8192 tokens with 50 to 2000 of their own 39.4 / 45.0 us; four members with few pages in a workgroup: 39.3 / 43.5.
#include <type_traits>

#include "prefix_items.hpp"

namespace unique {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t lds_addr_t;  // byte address in the LDS
typedef const __attribute__((address_space(3))) char* lds_char_t;
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;

// How the eight 16-byte pieces of a row of 128 bytes are permuted (by exclusive or). Two rows lie in the 256 bytes that all banks of the LDS hold: 16 rows at the same
// piece, and 4 rows at four, then meet no bank twice.
__device__ __forceinline__ int swizzle(int row) { return (row >> 1 & 1) * 4 + (row >> 2 & 3); }

// 16 bytes a lane from base + off into the LDS, lane after lane from `to` on. In assembly, as the compiler would otherwise wait for all loads before every
// transposing read; nothing is written but the LDS, and who reads that waits by wait_units.
// The address comes out of lanes by a vector instruction, after which a memory instruction would have to keep a distance that the compiler does not keep for it here;
// a scalar one need not, and its copy of the address is also the step between m0 and its use. (Nothing else in these kernels uses m0: accesses to the LDS do not here.)
template <bool kNT>
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t off, lds_addr_t to) {
  uint64_t copy;
  if constexpr (kNT)
    asm volatile("s_mov_b32 m0, %3\n\ts_mov_b64 %0, %2\n\tglobal_load_lds_dwordx4 %1, %0 nt" : "=&s"(copy) : "v"(off), "s"(base), "s"(to) : "memory");
  else
    asm volatile("s_mov_b32 m0, %3\n\ts_mov_b64 %0, %2\n\tglobal_load_lds_dwordx4 %1, %0" : "=&s"(copy) : "v"(off), "s"(base), "s"(to) : "memory");
}

// A unit is a tile of keys or of values: kTokens rows of D elements, in planes of 128 bytes of each row. kAcross: waves that share the rows of the
// workgroup; the others take other tokens, 32 each.
template <typename T, int D, int kAcross>
struct Unit {
  static constexpr int kPlanes = D * (int)sizeof(T) / 128, kTokens = sizeof(T) == 2 ? 64 : 32;
  static constexpr int kPlaneBytes = kTokens * 128, kBytes = kPlanes * kPlaneBytes;
  static constexpr int kRuns = kTokens / 8 / kDecWaves;  // of eight tokens, which a wave loads a kilobyte of each plane of
  static constexpr int kLoads = kRuns * kPlanes;         // of a wave
  static constexpr int kRing = 80 * 1024 / kBytes;       // units in the LDS
  static constexpr int kHalves = kTokens * kAcross / kDecWaves / 32;  // blocks of 32 tokens of a tile that a wave takes, one or two
};

// Until all but the newest `left` units (kMost at most) have arrived.
template <int kMost, int kLoads>
__device__ __forceinline__ void wait_units(int left) {
  if (left >= kMost) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMost * kLoads) : "memory");
  else if constexpr (kMost > 0) wait_units<kMost - 1, kLoads>(left);
}

// A run of a prefix's pages for a block of query rows. Every wave goes through the tiles, 32 tokens at a time, in steps: the products S = K Q^T of tile t, the softmax
// of tile t - 1 and O += V P of tile t - 2 do not wait for each other, so that the matrix cores and the vector units both have something to do (bf16:
// they stand between each other in the code).
// -> true: nothing has been written, and each member has to be attended by itself. A sum is not finite, and some rows have tokens here that others have not: a product of the others'
// probability, 0, with an infinity or NaN among the values is not 0. (Looking at the values of such tiles beforehand took 216 us for 105, 16 sequences behind 131072 tokens, one of
// them of one token. Where such a value is, behind the end of one of them: 588 us; 256 behind 32768 tokens 2175 for 287.)
template <typename T, int D, int S, int kAcross, bool kNT>
__device__ __forceinline__ bool attend_prefix(const CacheView& c, const PrefixArgs& a, const PrefixItem& item, int hkv, char* ring) {
  using L = Unit<T, D, kAcross>;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kBlocks = D / 32;                    // of channels
  constexpr int kAlong = kDecWaves / kAcross;
  constexpr int kTilePages = L::kTokens / S;
  constexpr int kLag = 3 - L::kHalves;
  constexpr float kRoom = 6.f;                       // log2: how far above the largest logit the reference is put
  constexpr int kIds = kPrefixMostPages / kWave;     // page ids in a lane
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 32, half = lane / 32;
  const int across = wave % kAcross, along = wave / kAcross, G = c.H / c.Hkv;

  // The item's pages, looked up once. One that there is not is read from the pool's first page, and does not count.
  const int pages = item.end - item.begin, tiles = (pages + kTilePages - 1) / kTilePages;
  const int32_t* table = c.page_table + (int64_t)(item.seq >= 0 && item.seq < c.B ? item.seq : 0) * c.max_pages + item.begin;
  const uint32_t pool = (uint32_t)min(c.num_phys, (int64_t)INT32_MAX);
  int ids[kIds];
#pragma unroll
  for (int i = 0; i < kIds; ++i) ids[i] = table[min(i * kWave + lane, pages - 1)];
  // The wait is here and not where an id is used, where all that is on its way to the LDS would be waited for as well.
#pragma unroll
  for (int i = 0; i < kIds; ++i) asm volatile("" : "+v"(ids[i]));
  bool holes = false;
#pragma unroll
  for (int i = 0; i < kIds; ++i) holes |= (uint32_t)ids[i] >= pool;
  holes = __any(holes);
  auto ids_of = [&](int window) {
    int x = 0;
#pragma unroll
    for (int i = 0; i < kIds; ++i) x |= ids[i] & -(int)(window == i);  // (a choice becomes an array in memory)
    return x;
  };
  constexpr uint32_t kAll = (1u << kTilePages) - 1;
  auto there_at = [&](int t) {  // pages of tile t that there are, a bit each
    uint32_t bits = t == tiles - 1 ? (2u << (pages - 1 - t * kTilePages)) - 1 : kAll;
    if (holes) bits &= (uint32_t)(__ballot((uint32_t)ids_of(t * kTilePages / kWave) < pool) >> (t * kTilePages % kWave));
    return bits;
  };

  // Loads of a unit: wave w takes the tokens 8 w + ..., eight rows of a plane at a time, whose pieces are permuted where they are read, within a line of memory. Where
  // the pages lie, 64 of them, is in the lanes as well, for the keys and for the values that come behind them.
  const lds_addr_t ring_at = (lds_addr_t)(uintptr_t)(lds_char_t)ring;
  const lds_addr_t load_to = ring_at + wave * 1024, load_end = load_to + L::kRing * L::kBytes;
  const int load_row = 8 * wave + lane / 8;
  uint32_t load_off[L::kPlanes];
#pragma unroll
  for (int j = 0; j < L::kPlanes; ++j) load_off[j] = load_row % S * (D * (int)sizeof(T)) + j * 128 + (lane % 8 ^ swizzle(load_row)) * 16;
  const uint64_t head_at = (uint64_t)hkv * c.kv_head_stride * sizeof(T), k_base = (uint64_t)c.k_cache + head_at;
  const uint64_t v_behind = (uint64_t)c.v_cache - (uint64_t)c.k_cache;
  uint64_t k_page = 0, v_page = 0;              // addresses of 64 pages' keys and values
  int next_k = 0, next_v = 0;                   // tiles to load next,
  int k_lane = 8 * wave / S, v_lane = k_lane;   // their first pages in the lanes
  lds_addr_t to = load_to;                      // and where to
  auto load = [&](uint64_t page, int at) {
#pragma unroll
    for (int r = 0; r < L::kRuns; ++r) {
      const int e = at + r * 8 * kDecWaves / S;
      const uint64_t from = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(page >> 32), e) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)page, e);
#pragma unroll
      for (int j = 0; j < L::kPlanes; ++j)
        load_to_lds<kNT>(reinterpret_cast<const char*>(from), load_off[j], to + j * L::kPlaneBytes + r * kDecWaves * 1024);
    }
    to += L::kBytes;
    to = to == load_end ? load_to : to;
  };
  auto load_keys = [&] {
    if (k_lane < kTilePages) {  // 64 new ones
      const int id = ids_of(next_k / (kWave / kTilePages));
      k_page = k_base + ((uint32_t)id < pool ? (uint64_t)(uint32_t)id * (uint64_t)c.kv_page_stride * sizeof(T) : 0);
    }
    load(k_page, k_lane);
    k_lane = (k_lane + kTilePages) % kWave;
    ++next_k;
  };
  auto load_values = [&] {
    if (v_lane < kTilePages) v_page = k_page + v_behind;  // the keys are at most kLag tiles ahead, and in the same 64 pages as these begin
    load(v_page, v_lane);
    v_lane = (v_lane + kTilePages) % kWave;
    ++next_v;
  };
  // Units go into the ring in the order in which the steps need them (with a lag of two tiles K0 K1 K2 V0 K3 V1 ...): step t takes the keys of tile t and the values of tile t - kLag.
  int loaded = 0;
  for (; loaded < L::kRing - (L::kHalves - 1) && next_v < tiles; ++loaded) {
    if (next_k < tiles && next_k <= next_v + kLag) load_keys();
    else load_values();
  }

  // This lane's query row; one that there is not takes another's query, and nobody reads what becomes of it (a column of the products is for itself).
  const int row = across * 32 + col;
  const bool live = row < item.rows;
  const int place = item.place + (live ? row : 0) / G;
  const int seq = a.groups.members ? a.groups.members[place] : place;
  const bool mine = live && seq >= 0 && seq < c.B;
  const int tokens = mine ? max(c.seq_lens[seq], 0) : 0;  // of this row's sequence
  const T* q = reinterpret_cast<const T*>(a.q) + ((int64_t)(mine ? seq : 0) * c.H + hkv * G + row % G) * D;
  constexpr int kSteps = kBf16 ? D / 16 : D / 8;  // reads of 16 bytes of a key
  u32x4_t qb[kSteps];  // bf16: the pieces 2 s + half; fp32: the pieces of this half
#pragma unroll
  for (int s = 0; s < kSteps; ++s) qb[s] = *reinterpret_cast<const u32x4_t*>(reinterpret_cast<const char*>(q) + (kBf16 ? 2 * s + half : half * kSteps + s) * 16);
  // The queries are waited for here, not in every turn of the loop.
#pragma unroll
  for (int s = 0; s < kSteps; ++s) asm volatile("" : "+v"(qb[s]));
  // tokens that all rows of the wave have
  const int all_have = __builtin_amdgcn_readfirstlane((int)wave_allreduce_minmax<false>((uint32_t)(live ? tokens : INT32_MAX)));
  const bool idle = across * 32 >= item.rows;  // no row of this wave (uniform)
  // tokens that any row of the item has, which are not the wave's alone, and tokens that all rows have that have any here
  int most = 0, least = INT32_MAX;
#pragma unroll
  for (int i = 0; i < kAcross * 32 / kWave; ++i) {
    const int r = i * kWave + lane, at = item.place + min(r, item.rows - 1) / G, s = a.groups.members ? a.groups.members[at] : at;
    const int n = s >= 0 && s < c.B ? c.seq_lens[s] : 0;
    most = max(most, n);
    if (n > item.begin * S) least = min(least, n);
  }
  const int longest = __builtin_amdgcn_readfirstlane((int)wave_allreduce_minmax<true>((uint32_t)most));
  const int shortest = __builtin_amdgcn_readfirstlane((int)wave_allreduce_minmax<false>((uint32_t)least));

  // Where a lane reads, behind a unit's beginning. Keys: token `col`, the pieces of step s, of which four (fp32: eight) are in a plane. Values, bf16: lane i of 16 asks
  // for token i / 4, channels 4 (i % 4) + ..., and gets channel i of the four tokens; two blocks of channels are in a plane. fp32: channel `col` of a block,
  // which is a plane.
  constexpr int kWays = kBf16 ? 4 : 8;
  lds_addr_t k_at[kWays], v_at[kBf16 ? 4 : 8];
#pragma unroll
  for (int s = 0; s < kWays; ++s)
    k_at[s] = ring_at + (kBf16 ? 0 : half * (kSteps / 8) * L::kPlaneBytes) + (along * 32 + col) * 128 + ((kBf16 ? 2 * s + half : s) ^ swizzle(col)) * 16;
#pragma unroll
  for (int i = 0; i < (kBf16 ? 4 : 8); ++i) {
    const int token = 4 * half + (kBf16 ? lane % 16 / 4 + i / 2 * 8 : i % 4 + i / 4 * 8);
    const int off = kBf16 ? i % 2 * 64 + lane % 32 / 16 * 32 + lane % 4 * 8 : col * 4;
    v_at[i] = ring_at + (along * 32 + token) * 128 + ((off / 16) ^ swizzle(token)) * 16 + off % 16;
  }
  struct Keys {
    lds_char_t at[kWays];
    __device__ __forceinline__ u32x4_t read(int s) const {
      return *(__attribute__((address_space(3))) const u32x4_t*)(at[s % kWays] + s / kWays * L::kPlaneBytes);
    }
  };
  auto keys_in = [&](int slot, int h) {
    Keys k;
#pragma unroll
    for (int s = 0; s < kWays; ++s) k.at[s] = (lds_char_t)(uintptr_t)(k_at[s] + slot * L::kBytes) + h * 32 * 128;
    return k;
  };
  struct Values {
    lds_char_t at[kBf16 ? 4 : 8];
    // bf16: of block i % kBlocks, the tokens 4 half + 0..3 and 8 + 4 half + 0..3 of the 16 from 16 (i / kBlocks) on
    __device__ __forceinline__ bf16x8_t read(int i) const {
      const int e = i % kBlocks, n = i / kBlocks;
      s16x4_t part[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) part[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(at[e % 2 + 2 * u] + e / 2 * L::kPlaneBytes + n * 16 * 128));
      return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // fp32: of block e, token 8 (i / 4) + 4 half + i % 4
    __device__ __forceinline__ float read(int i, int e) const {
      return *(__attribute__((address_space(3))) const float*)(at[i % 8] + i / 8 * 16 * 128 + e * L::kPlaneBytes);
    }
  };
  auto values_in = [&](int slot, int h) {
    Values v;
#pragma unroll
    for (int i = 0; i < (kBf16 ? 4 : 8); ++i) v.at[i] = (lds_char_t)(uintptr_t)(v_at[i] + slot * L::kBytes) + h * 32 * 128;
    return v;
  };

  float m = kNegBig, l = 0.f;
  f32x16_t acc[kBlocks];
#pragma unroll
  for (int e = 0; e < kBlocks; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;
  auto zero16 = [] {
    f32x16_t z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
  };

  f32x16_t x;               // logits of a tile: token 8 (i / 4) + 4 half + i % 4 of the wave's 32
  struct Weights {          // probabilities of the tile before
    float f[16];
  } p;
  struct Parts {            // of 8 of them, as operands: three parts of 8 bits, the largest first, whose sum they are
    u32x4_t b[3];
  };
  // Probabilities 2 j and 2 j + 1 of eight.
  auto split = [](const float* f, int j, Parts& to) {
    float r[2] = {f[2 * j], f[2 * j + 1]};
#pragma unroll
    for (int u = 0; u < 3; ++u) {
      to.b[u][j] = pack_hi(__float_as_uint(r[0]), __float_as_uint(r[1]));
#pragma unroll
      for (int i = 0; i < 2; ++i) r[i] -= bf16_part(r[i]);  // exact
    }
  };
  auto product = [&](u32x4_t k, int s, f32x16_t y) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, qb[s]), y, 0, 0, 0);
  };
  // Operands are read a few ahead (left to itself the compiler reads one at a time and waits for it).
  constexpr int kFew = 2;
  auto add = [&](bf16x8_t v, const Parts& w, int e) {
#pragma unroll
    for (int u = 2; u >= 0; --u) acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8_t, w.b[u]), acc[e], 0, 0, 0);
  };
  auto keys = [&](int slot, int h) {
    const Keys k = keys_in(slot, h);
    u32x4_t few[kFew];
#pragma unroll
    for (int s = 0; s < kFew; ++s) few[s] = k.read(s);
    if constexpr (kBf16) {
      x = zero16();
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        x = product(few[s % kFew], s, x);
        if (s + kFew < kSteps) few[s % kFew] = k.read(s + kFew);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      // Several sums of a part of the channels each (two of D = 128, where registers end): one after the other D products would be off by sqrt(D) roundings of the whole logit, more than the
      // exponential is. Output of 2 rows behind 2048 tokens of 64 channels, against 64 bits: 6 to 10e-7 with one sum, 3e-7 with four; 16 rows, 20000 tokens of 128: 13e-7, with two 8e-7.
      constexpr int kSums = D == 64 ? 4 : 2;
      f32x16_t y[kSums];
#pragma unroll
      for (int i = 0; i < kSums; ++i) y[i] = zero16();
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          y[i % kSums] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(few[s % kFew][i]), __uint_as_float(qb[s][i]), y[i % kSums], 0, 0, 0);
        if (s + kFew < kSteps) few[s % kFew] = k.read(s + kFew);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[i] = y[0][i] + y[1][i];
        if constexpr (kSums == 4) x[i] += y[2][i] + y[3][i];
      }
    }
  };
  auto values = [&](int slot, int h) {
    const Values v = values_in(slot, h);
    if constexpr (kBf16) {
      bf16x8_t few[kFew];
#pragma unroll
      for (int i = 0; i < kFew; ++i) few[i] = v.read(i);
      Parts parts;
#pragma unroll
      for (int i = 0; i < 2 * kBlocks; ++i) {
        if (i % kBlocks == 0) {
#pragma unroll
          for (int j = 0; j < 4; ++j) split(p.f + i / kBlocks * 8, j, parts);
        }
        add(few[i % kFew], parts, i % kBlocks);
        if (i + kFew < 2 * kBlocks) few[i % kFew] = v.read(i + kFew);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      float few[kFew][kBlocks];
#pragma unroll
      for (int i = 0; i < kFew; ++i)
#pragma unroll
        for (int e = 0; e < kBlocks; ++e) few[i][e] = v.read(i, e);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int e = 0; e < kBlocks; ++e) {
          acc[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(few[i % kFew][e], p.f[i], acc[e], 0, 0, 0);
          if (i + kFew < 16) few[i % kFew][e] = v.read(i + kFew, e);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  // Before the exponentials of block h of tile t: tokens that do not count, and the reference. -> what earlier sums are to be multiplied by, as soon as the block
  // before, whose probabilities are relative to the old reference, has been added to them.
  const int whole = holes ? 0 : min(pages / kTilePages, (all_have / S - item.begin) / kTilePages);  // tiles of which all tokens count for all rows
  bool moved = false;  // uniform
  auto prepare = [&](int t, int h, f32x16_t& x) {
    if (t >= whole) {
      const uint32_t there = there_at(t);
      const int first = (along + h) * 32, at0 = (item.begin + t * kTilePages) * S + first;
#pragma unroll
      for (int n = 0; n < 4; ++n) {  // pages are whole eights of tokens
        const int end = there >> ((first + 8 * n) / S) & 1 ? tokens : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * n + i] = at0 + 8 * n + 4 * half + i < end ? x[4 * n + i] : -INFINITY;
      }
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
    top *= a.scale_log2;
    float alpha = 1.f;
    moved = __any(top > m);
    if (moved) {
      const float mnew = fmaxf(m, with_lane_xor32(top, OpMax()) + kRoom);
      alpha = fast_exp2(m - mnew);
      m = mnew;
      l *= alpha;
    }
    return alpha;
  };
  auto weight = [&](float logit) {
    const float w = fast_exp2(fmaf(logit, a.scale_log2, -m));
    l += w;
    return w;
  };
  auto rescale = [&](float alpha) {
    if (moved) {
#pragma unroll
      for (int e = 0; e < kBlocks; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[e][i] *= alpha;
    }
  };
  auto weights = [&] {
    if constexpr (kBf16) {
#pragma unroll
      for (int i = 0; i < 16; ++i) p.f[i] = weight(x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) p.f[i] = fast_exp2(fmaf(x[i], a.scale_log2, -m));
      float sum[8];  // fewer roundings of l
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] = p.f[i] + p.f[i + 8];
      l += ((sum[0] + sum[4]) + (sum[1] + sum[5])) + ((sum[2] + sum[6]) + (sum[3] + sum[7]));
    }
  };

  int slot = 0;
  auto next = [&](int s) { return s + 1 == L::kRing ? 0 : s + 1; };
  int taken = 0;  // units, with those of the step
  auto arrive = [&](int units) {
    taken += units;
    const int left = loaded - taken;  // behind them
    wait_units<L::kRing - 4 < 1 ? 1 : L::kRing - 4, L::kLoads>(left);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  // Slots of pages that there are not, and of tokens behind the longest row, may hold anything, and a product with zero is not always zero.
  const int clean = holes ? 0 : min(pages / kTilePages, (longest / S - item.begin) / kTilePages);  // tiles that have none
  auto blank = [&](int t, int s) {
    if (t < clean) return;
    const uint32_t there = there_at(t);
    const int end = longest - (item.begin + t * kTilePages) * S;
    for (int i = threadIdx.x; i < L::kBytes / 16; i += kDecWaves * kWave) {
      const int token = i * 16 % L::kPlaneBytes / 128;
      if (token >= end || !(there >> (token / S) & 1)) *(__attribute__((address_space(3))) u32x4_t*)(uintptr_t)(ring_at + s * L::kBytes + i * 16) = u32x4_t{0, 0, 0, 0};
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };

  // What a step has used, which all waves are done with at the next, takes the next two units, in their order.
  auto load_one = [&](bool keys) {
    if (keys ? next_k < tiles : next_v < tiles) {
      if (keys) load_keys();
      else load_values();
      ++loaded;
    }
  };
  constexpr bool kKeysFirst = L::kRing % 2 == 0;
  // From the logits x of a block (block h of tile t) and the probabilities w of the one before to the logits y of the next and the probabilities v of this one.
  auto block = [&](int t, int h, const Keys& k, const Values& u, f32x16_t& x, f32x16_t& y, Weights& w, Weights& v, auto load_now) {
    const float alpha = prepare(t, h, x);
    constexpr int kEach = 16 / kSteps;  // exponentials between two products
    u32x4_t kf[kFew];
    bf16x8_t vf[kFew];
    y = zero16();
#pragma unroll
    for (int i = 0; i < kFew; ++i) kf[i] = k.read(i);
#pragma unroll
    for (int i = 0; i < kFew; ++i) vf[i] = u.read(i);
    Parts parts;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      y = product(kf[i % kFew], i, y);
      if (i + kFew < kSteps) kf[i % kFew] = k.read(i + kFew);
#pragma unroll
      for (int j = i * kEach; j < (i + 1) * kEach; ++j) v.f[j] = weight(x[j]);
      asm volatile("" : "+v"(l));  // here, and not where they are used
      if (i % kBlocks == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) split(w.f + i / kBlocks * 8, j, parts);
      }
      add(vf[i % kFew], parts, i % kBlocks);
      if (i + kFew < kSteps) vf[i % kFew] = u.read(i + kFew);
      __builtin_amdgcn_sched_barrier(0);
      load_now(i);  // while products are in work
    }
    rescale(alpha);
  };

  arrive(1);
  if (!idle) keys(slot, 0);
  if constexpr (L::kHalves == 2) {
    if (!idle) {
      prepare(0, 0, x);
      weights();
      keys(slot, 1);
    }
    slot = next(slot);
    f32x16_t y;
    Weights w;
    for (int t = 1; t < tiles; ++t) {
      arrive(2);
      const int k_slot = slot, v_slot = next(slot);
      slot = next(v_slot);
      blank(t - 1, v_slot);
      if (idle) {
        load_one(kKeysFirst);
        load_one(!kKeysFirst);
        continue;
      }
      block(t - 1, 1, keys_in(k_slot, 0), values_in(v_slot, 0), x, y, p, w, [&](int i) { if (i == 0) load_one(kKeysFirst); });
      block(t, 0, keys_in(k_slot, 1), values_in(v_slot, 1), y, x, w, p, [&](int i) { if (i == 0) load_one(!kKeysFirst); });
    }
    arrive(1);
    blank(tiles - 1, slot);
    if (!idle) {
      const float alpha = prepare(tiles - 1, 1, x);
      values(slot, 0);
      rescale(alpha);
      weights();
      values(slot, 1);
    }
  } else {
    slot = next(slot);
    if (tiles > 1) {
      arrive(1);
      if (!idle) {
        prepare(0, 0, x);
        weights();
        keys(slot, 0);
      }
      slot = next(slot);
    } else if (!idle) {
      prepare(0, 0, x);
      weights();
    }
    auto step = [&](int t, f32x16_t& x, f32x16_t& y, Weights& w, Weights& v) {
      arrive(2);
      const int k_slot = slot, v_slot = next(slot);
      slot = next(v_slot);
      blank(t - 2, v_slot);
      if (!kBf16 || idle) {
        load_one(kKeysFirst);
        load_one(!kKeysFirst);
        if (idle) return;
      }
      if constexpr (kBf16) {
        block(t - 1, 0, keys_in(k_slot, 0), values_in(v_slot, 0), x, y, w, v, [&](int i) {
          if (i == 0) load_one(kKeysFirst);
          if (i == kSteps / 2) load_one(!kKeysFirst);
        });
      } else {
        const float alpha = prepare(t - 1, 0, x);
        values(v_slot, 0);
        rescale(alpha);
        weights();
        keys(k_slot, 0);
      }
    };
    if constexpr (kBf16) {
      f32x16_t y;
      Weights w;
      int t = 2;
      for (; t + 1 < tiles; t += 2) {  // by twos, so that nothing is copied
        step(t, x, y, p, w);
        step(t + 1, y, x, w, p);
      }
      if (t < tiles) {
        step(t, x, y, p, w);
        x = y;
        p = w;
      }
    } else {
      for (int t = 2; t < tiles; ++t) step(t, x, x, p, p);
    }
    if (tiles > 1) {
      arrive(1);
      load_one(false);  // the keys are all there
      blank(tiles - 2, slot);
      if (!idle) {
        const float alpha = prepare(tiles - 1, 0, x);
        values(slot, 0);
        rescale(alpha);
        weights();
      }
      slot = next(slot);
    }
    arrive(1);
    blank(tiles - 1, slot);
    if (!idle) values(slot, 0);
  }

  if (shortest < min(item.end * S, longest)) {  // (the same in all waves)
    bool odd = false;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd |= !(fabsf(acc[e][i]) < INFINITY);
    int* any = reinterpret_cast<int*>(ring);
    __syncthreads();
    if (threadIdx.x == 0) *any = 0;
    __syncthreads();
    if (__any(odd) && lane == 0) *any = 1;
    __syncthreads();
    const bool alone = __builtin_amdgcn_readfirstlane(*any) != 0;
    __syncthreads();
    if (alone) return true;
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
    if (along == 1) return false;
    const float m2 = o[32 * D + col], l2 = o[32 * D + 32 + col], M = fmaxf(m, m2);
    const float s1 = fast_exp2(m - M), s2 = fast_exp2(m2 - M);
    m = M;
    l = l * s1 + l2 * s2;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[e][i] = acc[e][i] * s1 + o[(e * 16 + i) * 64 + lane] * s2;
  }
  if (!live) return false;
  const int64_t part = (int64_t)hkv * a.shape.max_rows + item.part + row;
  float* out = a.work.part_o + part * D;
#pragma unroll
  for (int e = 0; e < kBlocks; ++e)
#pragma unroll
    for (int n = 0; n < 4; ++n)
      *reinterpret_cast<float4*>(out + e * 32 + 8 * n + 4 * half) =
          make_float4(acc[e][4 * n], acc[e][4 * n + 1], acc[e][4 * n + 2], acc[e][4 * n + 3]);
  if (half == 0) *reinterpret_cast<float2*>(a.work.part_ml + part * 2) = make_float2(m, l);
  return false;
}

__device__ __forceinline__ PrefixItem uniform(const PrefixItem& x) {
  auto of = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  return {of(x.place), of(x.rows), of(x.begin), of(x.end), of(x.seq), of(x.own), of(x.part), 0};
}

// An item: a run of a prefix, or of a member's own pages, which the decode kernels' chunk code takes.
template <typename T, int D, int S, int G, int kAcross, bool kNT>
__global__ __launch_bounds__(kDecWaves* kWave, 2) void prefix_kernel(CacheView c, PrefixArgs a) {
  using L = Unit<T, D, kAcross>;
  constexpr size_t kRingBytes = L::kRing * L::kBytes, kOwnBytes = sizeof(DecodeShared<T, D, G>);
  __shared__ __attribute__((aligned(1024))) char ring[kRingBytes > kOwnBytes ? kRingBytes : kOwnBytes];
  const int hkv = blockIdx.x & (c.Hkv - 1), index = blockIdx.x >> __builtin_ctz(c.Hkv);
  PrefixItem item;
  if (a.shape.plans) {  // a thread for every source
    ItemsPlan<kDecWaves * kWave, true> plan = {c, a, *reinterpret_cast<ItemsShared<kDecWaves * kWave, true>*>(ring)};
    plan.make();
    if (blockIdx.x == 0) {  // for the kernel that joins the results
      if (plan.t < plan.sources) plan.keep(plan.t);
      __syncthreads();
      if (plan.t >= plan.n && plan.t < plan.sources) plan.tell_member(plan.t - plan.n, plan.m);
    }
    if (index >= plan.items()) return;
    int y = index;
    const int k = plan.class_of(y), z = y - plan.at_of(k);
    if (plan.s.kind == k && z >= 0 && z < plan.mine) plan.sh.item = plan.item_of(plan.s, z, plan.leader_of(plan.s));
    __syncthreads();
    item = uniform(plan.sh.item);
    __syncthreads();  // the ring is for keys now
  } else {
    item = a.work.item[index];
    if (index >= *a.work.num_items) return;
  }
  const bool alone = item.own || attend_prefix<T, D, S, kAcross, kNT>(c, a, item, hkv, ring);
  asm volatile("" ::: "memory");  // (one way on; with two, values of the chunk code are formed in front of the products and take their registers)
  if (!alone) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll 1
  for (int i = 0, members = item.own ? 1 : item.rows / G; i < members; ++i) {
    if (i > 0) __syncthreads();  // the LDS is the next one's
    int lane = threadIdx.x % kWave;
    asm volatile("" : "+v"(lane));  // nothing of a turn is formed before the loop, where it would take registers
    int b = item.seq;
    if (!item.own) {
      b = a.groups.members ? a.groups.members[item.place + i] : item.place + i;
      if (b < 0 || b >= c.B) continue;  // (uniform)
    }
    const int N = c.seq_lens[b], end = item.own ? item.end : min(item.end, prefix_pages_of(N, S));
    const int64_t part = (int64_t)hkv * a.shape.max_rows + item.part + i * G;
    const ChunkOut<T> to = {a.work.part_o + part * D, a.work.part_ml + part * 2, reinterpret_cast<T*>(a.out), a.lse_out, 2};
    const Chunk chunk = {hkv, b, item.begin, end, N, 0};
    auto lookup = [&](int e, bool, int& phys, int& ntok) {
      const int ph = c.page_table[(int64_t)b * c.max_pages + e];
      if (ph >= 0 && (int64_t)ph < c.num_phys) {
        phys = ph;
        ntok = min(S, N - e * S);
      }
    };
    decode_chunk<D, S, G, kNT>(c, reinterpret_cast<const T*>(a.q), chunk, wave, lane, lookup, a.scale_log2, to,
                               *reinterpret_cast<DecodeShared<T, D, G>*>(ring));
  }
}

// A chunk of a member's pages, prefix and own: calls with little to read (prefix_plan.hpp). A member's group is the first that ends behind it.
template <typename T, int D, int S, int G>
__global__ __launch_bounds__(kDecWaves* kWave) void prefix_alone_kernel(CacheView c, PrefixArgs a) {
  __shared__ DecodeShared<T, D, G> sh;
  const int hkv = blockIdx.x, z = blockIdx.y, place = blockIdx.z;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, n = a.groups.num_groups;
  const int seq = a.groups.members ? a.groups.members[place] : place;
  const bool valid = seq >= 0 && seq < c.B;
  const int N = valid ? max(c.seq_lens[seq], 0) : 0;
  int group = 0;
  bool down = false;
  for (int i0 = 0; i0 < n; i0 += kWave) {
    const int i = min(i0 + lane, n - 1), from = a.groups.starts[i], to = a.groups.starts[i + 1];
    down |= to < from;
    group += __popcll(__ballot(i0 + lane < n && to <= place));
  }
  const int of = min(group, n - 1), from = a.groups.starts[of], prefix = min(max(a.groups.prefix_pages[of], 0), a.groups.max_prefix_pages);
  const bool listed = valid && !__any(down) && group < n && place >= from && place - from < a.groups.max_members;
  const int end = min(min((N + S - 1) / S, c.max_pages_hint), prefix + a.groups.max_own_pages), chunks = (end + a.shape.chunk_pages - 1) / a.shape.chunk_pages;
  if (hkv == 0 && z == 0 && threadIdx.x == 0) {
    PrefixMember m = {};
    m.seq = listed && chunks > 1 ? seq : -1;  // of one chunk there is nothing to join
    m.own_count = chunks;
    m.own_part = place * a.shape.chunks * G;
    a.work.member[place] = m;
  }
  if (!listed || z >= max(chunks, 1)) return;
  const int64_t part = (int64_t)hkv * a.shape.max_rows + (int64_t)(place * a.shape.chunks + z) * G;
  const ChunkOut<T> to = {a.work.part_o + part * D, a.work.part_ml + part * 2, reinterpret_cast<T*>(a.out), a.lse_out, max(chunks, 1)};
  if (chunks == 0) {
    write_empty<T, D, G>(c, to, seq, hkv);
    return;
  }
  const Chunk chunk = {hkv, seq, z * a.shape.chunk_pages, min((z + 1) * a.shape.chunk_pages, end), N, 0};
  auto lookup = [&](int e, bool, int& phys, int& ntok) {
    const int ph = c.page_table[(int64_t)seq * c.max_pages + e];
    if (ph >= 0 && (int64_t)ph < c.num_phys) {
      phys = ph;
      ntok = min(S, N - e * S);
    }
  };
  decode_chunk<D, S, G, false>(c, reinterpret_cast<const T*>(a.q), chunk, wave, lane, lookup, a.scale_log2, to, sh);
}

// A wave joins the parts of a (member, query head): o = sum of 2^(m_j - M) o_j over sum of 2^(m_j - M) l_j. Lane s takes the pair (m, l) of part s; D / 4 lanes
// read a part's row, so that a load covers 2 or 4 parts, and eight loads are in flight.
template <typename T, int D>
__global__ __launch_bounds__(kMergeWaves* kWave) void prefix_merge_kernel(CacheView c, PrefixArgs a) {
  constexpr int kLanes = D / 4, kParts = kWave / kLanes, kAhead = 8;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int h = blockIdx.y * kMergeWaves + wave, shift = __builtin_ctz(c.H / c.Hkv), G = 1 << shift, hkv = h >> shift;
  const PrefixMember of = a.work.member[blockIdx.x];
  if (h >= c.H || of.seq < 0) return;  // (no barrier below)
  const int n = of.count + of.own_count;
  const int64_t base = (int64_t)hkv * a.shape.max_rows + (h & (G - 1));
  auto row_of = [&](int s) { return base + (s < of.count ? of.part + (int64_t)s * of.step : of.own_part + (int64_t)(s - of.count) * G); };
  const float2* ml = reinterpret_cast<const float2*>(a.work.part_ml);
  const float2 none = make_float2(kNegBig, 0.f);

  const int sub = lane / kLanes, channel = lane % kLanes * 4;
  float4 v[kAhead];
  auto request = [&](int s0) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (s0 + u * kParts < n) v[u] = *reinterpret_cast<const float4*>(a.work.part_o + row_of(min(s0 + u * kParts + sub, n - 1)) * D + channel);  // uniform
  };
  const float2 first = lane < n ? ml[row_of(lane)] : none;
  request(0);
  float M = first.x;
  for (int s0 = kWave; s0 < n; s0 += kWave) M = fmaxf(M, s0 + lane < n ? ml[row_of(s0 + lane)].x : kNegBig);
  M = group_allreduce<kWave>(M, OpMax());
  float L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < n; s0 += kWave) {
    const float2 p = s0 == 0 ? first : (s0 + lane < n ? ml[row_of(s0 + lane)] : none);
    // (a part without tokens that count for this row may have sums that are not finite, from tokens of others)
    const float scale = p.y == 0.f ? -1.f : fast_exp2(p.x - M);
    L = p.y == 0.f ? L : fmaf(p.y, scale, L);
    const int here = min(kWave, n - s0);
    for (int j0 = 0; j0 < here; j0 += kParts * kAhead) {
      if (s0 + j0 > 0) request(s0 + j0);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (j0 + u * kParts >= here) break;  // uniform
        const int j = j0 + u * kParts + sub;
        const float of_j = __shfl(scale, j % kWave, kWave);  // by all lanes, as any may be asked for its own
        if (j >= here || of_j < 0.f) continue;
        o[0] = fmaf(v[u].x, of_j, o[0]);
        o[1] = fmaf(v[u].y, of_j, o[1]);
        o[2] = fmaf(v[u].z, of_j, o[2]);
        o[3] = fmaf(v[u].w, of_j, o[3]);
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

// One translation unit per element type and head dimension: UNIQUE_ELEM, UNIQUE_DIM.
template <int S, int G, int kAcross>
hipError_t launch_items(const CacheView& c, const PrefixArgs& a, hipStream_t st) {
  using T = UNIQUE_ELEM;
  auto go = [&](auto kernel) {
    kernel<<<dim3(c.Hkv * a.shape.max_items), dim3(kDecWaves * kWave), 0, st>>>(c, a);
    return hipGetLastError();
  };
  return a.streams ? go(prefix_kernel<T, UNIQUE_DIM, S, G, kAcross, true>) : go(prefix_kernel<T, UNIQUE_DIM, S, G, kAcross, false>);
}

template <int S, int G>
hipError_t launch_rows(const CacheView& c, const PrefixArgs& a, hipStream_t st) {
  if (a.shape.chunks > 0) {
    prefix_alone_kernel<UNIQUE_ELEM, UNIQUE_DIM, S, G><<<dim3(c.Hkv, a.shape.chunks, c.B), dim3(kDecWaves * kWave), 0, st>>>(c, a);
    return hipGetLastError();
  }
  if constexpr (sizeof(UNIQUE_ELEM) == 2)
    if (a.shape.rows == 64) return launch_items<S, G, 2>(c, a, st);
  return launch_items<S, G, 4>(c, a, st);
}

template <int S>
hipError_t launch_group(const CacheView& c, const PrefixArgs& a, hipStream_t st) {
  switch (c.H / c.Hkv) {
    case 1: return launch_rows<S, 1>(c, a, st);
    case 2: return launch_rows<S, 2>(c, a, st);
    case 4: return launch_rows<S, 4>(c, a, st);
    case 8: return launch_rows<S, 8>(c, a, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

template <>
hipError_t launch_prefix_of<UNIQUE_ELEM, UNIQUE_DIM>(const CacheView& c, const PrefixArgs& a, hipStream_t st) {
  const hipError_t e = c.S == 8 ? launch_group<8>(c, a, st) : (c.S == 16 ? launch_group<16>(c, a, st) : launch_group<32>(c, a, st));
  if (e != hipSuccess || a.shape.chunks == 1) return e;
  prefix_merge_kernel<UNIQUE_ELEM, UNIQUE_DIM><<<dim3(c.B, (c.H + kMergeWaves - 1) / kMergeWaves), dim3(kMergeWaves * kWave), 0, st>>>(c, a);
  return hipGetLastError();
}

}  // namespace unique
