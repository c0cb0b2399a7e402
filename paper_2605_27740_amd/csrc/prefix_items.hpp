// The work items of attention over shared prefixes on the device: what each source has to read, how long items have to be for the chip to be full, where each
// source's items and partial results begin, and the items. The whole workgroup goes through this. Where there are few, every workgroup of the attention kernel makes them for
// itself; else a kernel of one workgroup does, before it.
#pragma once
#include "decode_core.hpp"
#include "serving.hpp"

namespace unique {

constexpr int kClasses = kPrefixKinds;

// kHeld: there is a thread for every source and one more, and what is looked up is in the LDS.
template <int kThreads, bool kHeld>
struct ItemsShared {
  static constexpr int kWaves = kThreads / kWave;
  PrefixSource source[kHeld ? kThreads : 1];
  int first[kClasses][kHeld ? kThreads : 1];  // items of a class before each source's
  int starts[kHeld ? kThreads : 1], prefix[kHeld ? kThreads : 1], full[kHeld ? kThreads : 1];  // full: a member's sequence that is not empty, or -1
  int64_t cost[kWaves];
  int scan[kClasses + 1][kWaves];
  PrefixItem item;
};

template <int kThreads, bool kHeld>
struct ItemsPlan {
  static constexpr int kWaves = kThreads / kWave;
  const CacheView& c;
  const PrefixArgs& a;
  ItemsShared<kThreads, kHeld>& sh;
  const int t = threadIdx.x, lane = t % kWave, wave = t / kWave;
  const int n = a.groups.num_groups, sources = n + c.B, shift = __builtin_ctz(c.H) - __builtin_ctz(c.Hkv), G = 1 << shift;
  int before[kClasses + 1] = {};  // items of each class and rows, in the end all
  PrefixSource s = {};            // of this thread's source (kHeld)
  PrefixMember m = {};            // and its member, if it is one
  int mine = 0, at[kClasses] = {};
  bool ok = true;                 // starts ascend, and groups have no more members than there are rows; else there are no items and no members

  __device__ __forceinline__ int start(int i) const { return kHeld ? sh.starts[i] : a.groups.starts[i]; }
  __device__ __forceinline__ int pages(int i) const {
    return min(max(kHeld ? sh.prefix[i] : a.groups.prefix_pages[i], 0), a.groups.max_prefix_pages);
  }
  __device__ __forceinline__ int bound(int i) const { return min(max(i, 0), c.B); }
  __device__ __forceinline__ int size_of(int from, int to) const { return min(max(bound(to) - bound(from), 0), a.groups.max_members); }
  __device__ __forceinline__ PrefixSource* source() const { return kHeld ? sh.source : a.work.source; }
  __device__ __forceinline__ int& first_of(int k, int i) const { return kHeld ? sh.first[k][i] : a.work.first[(int64_t)k * sources + i]; }

  // What source i has to read; seq: the sequence of a member, and len its length. A member's group is the first that ends behind it.
  __device__ __forceinline__ PrefixSource look_at(int i, int seq, int len, PrefixMember& m) const {
    PrefixSource s = {};
    if (i < n) {
      const int from = start(i), to = start(i + 1), size = size_of(from, to);
      s.place = bound(from);
      s.rows = size * G;
      s.end = size > 1 ? pages(i) : 0;  // (nobody to share it with: all pages are the member's own)
      s.blocks = (s.rows + a.shape.rows - 1) >> __builtin_ctz(a.shape.rows);  // (a power of two)
      return s;
    }
    const int place = i - n;
    int lo = 0, hi = n;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (start(mid + 1) > place) hi = mid;
      else lo = mid + 1;
    }
    m = {};
    m.seq = -1;
    if (lo == n) return s;
    const int from = start(lo), to = start(lo + 1), prefix = pages(lo);
    if (place < from || place - from >= a.groups.max_members || seq < 0 || seq >= c.B) return s;
    m.seq = seq;
    m.step = lo;  // until that is known
    s.place = place;
    s.rows = G;
    s.blocks = 1;
    s.begin = size_of(from, to) > 1 ? prefix : 0;
    s.end = min(min(prefix_pages_of(len, c.S), c.max_pages_hint), prefix + a.groups.max_own_pages);
    return s;
  }
  __device__ __forceinline__ int seq_of(int i) const { return a.groups.members ? a.groups.members[i] : i; }
  __device__ __forceinline__ int len_of(int seq) const { return seq >= 0 && seq < c.B ? c.seq_lens[seq] : 0; }
  // The first sequence of a source that is not empty (one that has ended has lost its pages): its row of the page table is that of the others, as far as their prefix goes.
  __device__ __forceinline__ int leader_of(const PrefixSource& of) const {
    for (int i = of.place, end = of.place + (of.rows >> shift); i < end; ++i) {
      int seq = kHeld ? sh.full[i] : seq_of(i);
      if (!kHeld && len_of(seq) <= 0) seq = -1;
      if (seq >= 0) return seq;
    }
    return -1;
  }

  __device__ __forceinline__ void make() {
    int64_t cost = 0;
    bool down = false;
    if constexpr (kHeld) {
      const int seq = t >= n && t < sources ? seq_of(t - n) : -1;
      if (t <= n) sh.starts[t] = a.groups.starts[t];
      if (t < n) sh.prefix[t] = a.groups.prefix_pages[t];
      const int len = len_of(seq);
      if (t >= n && t < sources) sh.full[t - n] = len > 0 ? seq : -1;
      __syncthreads();
      if (t < sources) s = look_at(t, seq, len, m);
      cost = prefix_cost(s.end - s.begin, s.blocks, t >= n, c.S);
      down = t < n && start(t + 1) < start(t);
    } else {
      for (int i = t; i < sources; i += kThreads) {
        const int seq = i >= n ? seq_of(i - n) : -1;
        s = look_at(i, seq, len_of(seq), m);
        cost += prefix_cost(s.end - s.begin, s.blocks, i >= n, c.S);
        down |= i < n && start(i + 1) < start(i);
        a.work.source[i] = s;
        if (i >= n) a.work.member[i - n] = m;
      }
    }
    // The sum over the workgroup, in two parts of 24 and more bits within a wave.
    const int low = __builtin_amdgcn_readlane(wave_inclusive_scan((int)(cost & 0xffffff)), kWave - 1);
    const int high = __builtin_amdgcn_readlane(wave_inclusive_scan((int)(cost >> 24)), kWave - 1);
    const bool bad = __any(down);
    if (lane == 0) sh.cost[wave] = bad ? -1 : ((int64_t)high << 24) + low;
    __syncthreads();
    cost = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      ok = ok && sh.cost[w] >= 0;
      cost += sh.cost[w];
    }
    if (!ok) return;
    const int item_pages = prefix_item_pages(cost, a.shape.wanted);

    for (int i0 = 0; i0 < sources; i0 += kThreads) {
      const int i = i0 + t;
      if constexpr (!kHeld) s = i < sources ? a.work.source[i] : PrefixSource{};
      const PrefixCut cut = prefix_cut(s.end - s.begin, item_pages, min(s.rows, a.shape.rows), a.shape.row_tokens, c.S, a.shape.tile_pages, i >= n);
      mine = cut.count * s.blocks;
      s.kind = prefix_kind(i >= n, min(cut.pages, s.end - s.begin), item_pages);
      int x[kClasses + 1], upto[kClasses + 1];
#pragma unroll
      for (int k = 0; k < kClasses; ++k) x[k] = s.kind == k ? mine : 0;
      x[kClasses] = mine * (i < n ? a.shape.rows : G);
#pragma unroll
      for (int k = 0; k <= kClasses; ++k) upto[k] = wave_inclusive_scan(x[k]);
      if (!kHeld) __syncthreads();
      if (lane == kWave - 1) {
#pragma unroll
        for (int k = 0; k <= kClasses; ++k) sh.scan[k][wave] = upto[k];
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k <= kClasses; ++k) {
        const int waves = wave_inclusive_scan(lane < kWaves ? sh.scan[k][lane] : 0);
        upto[k] += before[k] + (wave > 0 ? __builtin_amdgcn_readlane(waves, wave - 1) : 0);
        before[k] += __builtin_amdgcn_readlane(waves, kWave - 1);
      }
      s.first_row = upto[kClasses] - x[kClasses];
      s.count = cut.count;
      s.each = cut.pages;
#pragma unroll
      for (int k = 0; k < kClasses; ++k) at[k] = upto[k] - x[k];
      if constexpr (!kHeld) {
        if (i < sources) keep(i);
      }
    }
  }
  __device__ __forceinline__ int at_of(int k) const {
    int x = 0;
#pragma unroll
    for (int j = 0; j < kClasses; ++j) x |= at[j] & -(int)(k == j);  // (a choice becomes an array in memory)
    return x;
  }
  // Source i where others find it.
  __device__ __forceinline__ void keep(int i) const {
    source()[i] = s;
#pragma unroll
    for (int k = 0; k < kClasses; ++k) first_of(k, i) = at[k];
  }
  __device__ __forceinline__ int items() const {
    int sum = 0;
#pragma unroll
    for (int k = 0; k < kClasses; ++k) sum += before[k];
    return sum;
  }
  // The class of item i, which becomes its number within it.
  __device__ __forceinline__ int class_of(int& i) const {
    int k = 0;
#pragma unroll
    for (int j = 0; j < kClasses - 1; ++j)
      if (k == j && i >= before[j]) {
        i -= before[j];
        k = j + 1;
      }
    return k;
  }
  // Item z of a source.
  __device__ __forceinline__ PrefixItem item_of(const PrefixSource& of, int z, int seq) const {
    const int run = z / of.blocks, block = z - run * of.blocks;
    PrefixItem item = {};
    item.own = of.kind != kPrefixRun;
    item.place = of.place + block * (a.shape.rows >> shift);
    item.rows = min(of.rows - block * a.shape.rows, a.shape.rows);
    item.begin = of.begin + run * of.each;
    item.end = min(item.begin + of.each, of.end);
    item.seq = seq;
    item.part = of.first_row + z * (item.own ? G : a.shape.rows);
    return item;
  }
  // Where member i's partial results are. Sources are kept.
  __device__ __forceinline__ void tell_member(int i, PrefixMember m) const {
    if (!ok) m.seq = -1;
    if (m.seq >= 0) {
      const PrefixSource of = source()[m.step], own = source()[n + i];
      m.count = of.count;
      m.part = of.first_row + (i - of.place) * G;  // blocks follow one another
      m.step = of.blocks * a.shape.rows;
      m.own_count = own.count;
      m.own_part = own.first_row;
    }
    a.work.member[i] = m;
  }
};

}  // namespace unique
