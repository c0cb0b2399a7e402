// Eviction of the pages with the smallest accounts.
#include <algorithm>
#include <type_traits>

#include "decode_core.hpp"
#include "dense_plan.hpp"
#include "weigh.hpp"

namespace unique {
namespace {

constexpr int kAccountThreads = 256;

// A row of words behind a buffer descriptor: an access is one instruction with a 32-bit offset, where a pointer makes it a 64-bit
// sum per lane; a load behind the row's end gives 0, and a store there, to kNowhere for instance, is dropped, so that nothing
// branches. With sixteen waves on a compute unit an instruction costs sixteen cycles, and the kernels below are made of little else.
constexpr uint32_t kNowhere = 0xfffffff0u;
struct Row {
  __amdgpu_buffer_rsrc_t at;
  __device__ __forceinline__ Row(const void* p, int words)
      : at(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, words * 4, 0x27000)) {}
  __device__ __forceinline__ uint32_t word(uint32_t off) const { return __builtin_amdgcn_raw_buffer_load_b32(at, (int)off, 0, 0); }
  __device__ __forceinline__ float real(uint32_t off) const { return __uint_as_float(word(off)); }
  __device__ __forceinline__ void put(uint32_t off, uint32_t v) const { __builtin_amdgcn_raw_buffer_store_b32(v, at, (int)off, 0, 0); }
};

// What a page is ranked by: the sum of its accounts over the KV heads in 64 bits, rounded once. kAhead heads are requested at a
// time, whether there are so many or not; w: the last of them.
template <int kPer, int kAhead>
__device__ __forceinline__ void page_ranks(const float* weights, int heads, int weight_stride, int P, const uint32_t (&off)[kPer],
                                           float (&w)[kAhead][kPer], float (&rank)[kPer]) {
  double sum[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) sum[j] = 0.0;
  for (int h0 = 0; h0 < heads; h0 += kAhead) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const Row row(weights + (int64_t)min(h0 + u, heads - 1) * weight_stride, P);
#pragma unroll
      for (int j = 0; j < kPer; ++j) w[u][j] = row.real(off[j]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (h0 + u < heads) {  // uniform
#pragma unroll
        for (int j = 0; j < kPer; ++j) sum[j] += (double)w[u][j];
      }
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) rank[j] = (float)sum[j];
}

// The ranks of all pages, for sequences that a workgroup does not sum up itself; the first pages are kept: +inf.
__global__ __launch_bounds__(kAccountThreads) void rank_kernel(CacheView c, const float* weights, int weight_stride, int sinks, float* rank,
                                                               int rank_stride) {
  const int b = blockIdx.y, p = blockIdx.x * kAccountThreads + threadIdx.x;
  const int P = min((c.seq_lens[b] + c.S - 1) / c.S, c.max_pages_hint);
  if (p >= P) return;
  const uint32_t off[1] = {(uint32_t)p * 4};
  float w[8][1], r[1];
  page_ranks<1, 8>(weights + (int64_t)b * c.Hkv * weight_stride, c.Hkv, weight_stride, P, off, w, r);
  rank[(int64_t)b * rank_stride + p] = p < sinks ? INFINITY : r[0];
}

constexpr int kEvictMost = 16384;       // pages of the longest sequence that a workgroup holds
// Accounts of a sequence up to which its workgroup sums them up and closes their rows, one launch instead of three; above it they are summed up and closed by
// more workgroups. us of the call so / apart, heads x pages of each of 2 sequences, one page too many: 8 x 1000 9.4 / 16.2, 8 x 2900 8.8 / 14.7, 32 x 700
// 10.8 / 15.0, 2 x 8188 8.9 / 15.1; half of the pages evicted: 8 x 2900 12.2 / 15.1, 2 x 8188 14.7 / 18.7, but 8 x 5000 20.6 / 17.0, 8 x 8188 23.5 / 18.6 (32
// sequences 24.7 / 21.9). Rows between would gain by a bound of their own: 8 x 3400, one page too many, 9.6 / 14.6, 4 x 7000 9.5 / 14.9.
constexpr int64_t kSumsHere = 24576;
constexpr int kFew = 4;                 // pages that are sought one by one
constexpr int kGathered = 256;          // keys that one wave searches (16 x 8 x 8188 pages to 1024, us with 64, 128, 256, 512, 1024: 19.7, 19.3, 19.2, 19.3, 20.4)
constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave;

// How many lanes for which pred(j) holds come before each of a wave's kPer rows of 64 lanes, in the order j, wave, lane of the workgroup;
// counts: LDS. -> the rows' masks and what comes before them.
template <int kPer, typename Pred>
__device__ __forceinline__ void rows_before(Pred pred, int* counts, int wave, int lane, unsigned long long (&mask)[kPer], int (&before)[kPer]) {
  int mine = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    mask[j] = __ballot(pred(j));
    mine = lane == j ? __popcll(mask[j]) : mine;
  }
  __syncthreads();  // everyone is done with the previous contents
  if (lane < kPer) counts[lane * kEvictWaves + wave] = mine;
  __syncthreads();
  if (wave == 0) {
    int sum = 0;
#pragma unroll
    for (int i0 = 0; i0 < kPer * kEvictWaves; i0 += kWave) {
      const int i = i0 + lane, n = i < kPer * kEvictWaves ? counts[i] : 0;
      const int upto = wave_inclusive_scan(n);
      if (i < kPer * kEvictWaves) counts[i] = sum + upto - n;
      sum += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
  }
  __syncthreads();
  mine = counts[min(lane, kPer - 1) * kEvictWaves + wave];
#pragma unroll
  for (int j = 0; j < kPer; ++j) before[j] = __builtin_amdgcn_readlane(mine, j);
}
__device__ __forceinline__ int lanes_below(unsigned long long mask, int acc) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, (uint32_t)acc));
}

// Chooses the pages of a sequence that stay and closes its row of the table, a workgroup a sequence with kPer keys a thread. The key
// that separates them is sought between the least and the largest, a fourth of the window at a time from the number of keys above three
// candidates, with comparisons and ballots only (a histogram of exponents would be a few bins; one of equal bins of the window has not been
// tried); done as soon as a candidate has exactly as many above it as stay, or few keys are left, which one wave finishes. A round of eight keys a thread takes 1 us (16 waves issue 110 instructions each). kSums: the pages'
// sums are formed here and the rows of accounts closed, too; else they are in `rank`, and `kept` is for close_kernel.
template <int kPer, bool kSums>
__global__ __launch_bounds__(kEvictThreads) void evict_kernel(CacheView c, EvictArgs a, const float* __restrict__ rank, int rank_stride,
                                                              int32_t* __restrict__ kept, int32_t* __restrict__ pages,
                                                              int32_t* __restrict__ kept_count) {
  constexpr int kAhead = kPer >= 8 ? 4 : 8;
  __shared__ unsigned long long s_least[kFew];
  __shared__ int s_sums[20][4], s_held, s_from;  // (a window is a fourth after a round, rounded up: 17 rounds at most)
  __shared__ uint32_t s_range[2];
  __shared__ uint32_t s_key[kGathered];
  __shared__ int s_counts[kPer * kEvictWaves];
  const int b = blockIdx.x, t = threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave);
  const int N = c.seq_lens[b];
  const int P = max(min((N + c.S - 1) / c.S, c.max_pages_hint), 0), keep = min(P, a.budget);
  uint32_t key[kPer], off[kPer];
  int32_t id[kPer];
  float w[kAhead][kPer];
  const int64_t rows = (int64_t)b * c.Hkv * a.weight_stride;
  {
    const Row table(c.page_table + (int64_t)b * c.max_pages, P);
    float r[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      off[j] = (uint32_t)(j * kEvictThreads + t) * 4;
      id[j] = (int32_t)table.word(off[j]);
    }
    if constexpr (kSums) {
      page_ranks<kPer, kAhead>(a.weights_in + rows, c.Hkv, a.weight_stride, P, off, w, r);
    } else {
      const Row row(rank + (int64_t)b * rank_stride, P);
#pragma unroll
      for (int j = 0; j < kPer; ++j) r[j] = row.real(off[j]);
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int p = j * kEvictThreads + t;
      key[j] = p < a.sinks || p >= P - a.recent ? 0xffffffffu : score_key(r[j]);
      key[j] = p < P ? key[j] : 0u;
    }
  }
  if (t < 80) s_sums[t / 4][t % 4] = 0;
  if (t < 2) s_range[t] = 0;
  if (t < kFew) s_least[t] = 0;
  if (t == 0) s_held = 0;
  __syncthreads();
  // Those above `last` stay, and of those that equal it the first few. One page too many, or a few, as in a decode loop: the smallest
  // keys one after the other, the last page of equal ones, instead of the search.
  uint32_t last = 0;
  bool exact = P - keep <= kFew;  // every key of a page is at least 1
  if (exact) {
    for (int i = 0; i < P - keep; ++i) {
      uint32_t least = ~0u, page = 0;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const uint32_t k = key[j] - 1;  // no page: the largest
        page = k <= least ? j : page;
        least = min(k, least);
      }
      const uint32_t top = wave_allreduce_minmax<false>(least);
      const uint32_t at = wave_allreduce_minmax<true>(least == top ? page * kEvictThreads + t : 0u);
      if (lane == 0) atomicMax(&s_least[i], (unsigned long long)~top << 32 | at);
      __syncthreads();
      const int gone = (int)(uint32_t)s_least[i];
#pragma unroll
      for (int j = 0; j < kPer; ++j) key[j] = j * kEvictThreads + t == gone ? 0u : key[j];
    }
  }
  // The window that holds the key sought: `width` keys' values from `last` on, `here` keys in it and `upper` above; at first all but the pages
  // that stay whatever they are worth.
  uint32_t width = 1;
  int upper = a.sinks + a.recent, here = P - upper;
  if (!exact && upper == keep) {  // nothing else stays
    exact = true;
    last = ~0u;
  }
  if (!exact) {
    uint32_t least = ~0u, most = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      least = min(least, key[j] - 1);  // no page: the largest
      most = max(most, key[j] == ~0u ? 0u : key[j]);
    }
    least = wave_allreduce_minmax<false>(least);
    most = wave_allreduce_minmax<true>(most);
    if (lane == 0) {
      atomicMax(&s_range[0], ~least);
      atomicMax(&s_range[1], most);
    }
    __syncthreads();
    last = ~s_range[0] + 1;
    width = s_range[1] - last + 1;
  }
  for (int round = 0; !exact && width > 1 && here > kGathered; ++round) {
    const uint32_t step = (width - 1) / 4 + 1;
    int m[5] = {upper + here, 0, 0, 0, upper};  // keys from the d-th quarter of the window on
#pragma unroll
    for (int d = 1; d <= 3; ++d) {
      const uint32_t cand = last + min((uint32_t)d * step, width);
#pragma unroll
      for (int j = 0; j < kPer; ++j) m[d] += __popcll(__ballot(key[j] >= cand));
    }
    int* sum = s_sums[round];
    if (lane < 3) atomicAdd(&sum[lane], lane == 0 ? m[1] : (lane == 1 ? m[2] : m[3]));
    __syncthreads();
#pragma unroll
    for (int d = 1; d <= 3; ++d) m[d] = __builtin_amdgcn_readfirstlane(sum[d - 1]);
    const int d = m[3] >= keep ? 3 : (m[2] >= keep ? 2 : (m[1] >= keep ? 1 : 0));
    const int from = d == 3 ? m[3] : (d == 2 ? m[2] : (d == 1 ? m[1] : m[0]));
    upper = d == 3 ? m[4] : (d == 2 ? m[3] : (d == 1 ? m[2] : m[1]));
    here = from - upper;
    last += d * step;
    width = min(step, width - d * step);
    exact = from == keep;
  }
  if (!exact && width > 1) {  // what is left is few enough for one wave
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (key[j] - last < width) s_key[atomicAdd(&s_held, 1)] = key[j];
    __syncthreads();
    if (wave == 0) {
      uint32_t k[kGathered / kWave];
#pragma unroll
      for (int i = 0; i < kGathered / kWave; ++i) k[i] = i * kWave + lane < here ? s_key[i * kWave + lane] : 0u;
      while (width > 1 && !exact) {
        const uint32_t half = width / 2;
        int m = upper;
#pragma unroll
        for (int i = 0; i < kGathered / kWave; ++i) m += __popcll(__ballot(k[i] >= last + half));
        const bool up = m >= keep;
        last = up ? last + half : last;
        width = up ? width - half : half;
        exact = m == keep;
      }
      if (lane == 0) {
        s_key[0] = last;
        s_held = exact;
      }
    }
    __syncthreads();
    last = s_key[0];
    exact = s_held != 0;
  }
  if (P - keep > kFew && exact) last -= 1;  // the smallest that stays
  unsigned long long mask[kPer];
  int before[kPer];
  if (!exact) {  // equal keys: the first few are raised above the others
    rows_before<kPer>([&](int j) { return key[j] > last; }, s_counts, wave, lane, mask, before);
    if (t == kEvictThreads - 1) s_from = before[kPer - 1] + __popcll(mask[kPer - 1]);
    rows_before<kPer>([&](int j) { return key[j] == last; }, s_counts, wave, lane, mask, before);
    const int from_same = keep - s_from;
#pragma unroll
    for (int j = 0; j < kPer; ++j) key[j] = key[j] == last && lanes_below(mask[j], before[j]) < from_same ? ~0u : key[j];
  }
  rows_before<kPer>([&](int j) { return key[j] > last; }, s_counts, wave, lane, mask, before);
  int32_t* freed = a.freed_pages + (int64_t)b * a.freed_stride;
  const Row table_out(a.page_table_out + (int64_t)b * c.max_pages, P), freed_row(freed, P - keep), kept_row(kept + (int64_t)b * a.budget, keep);
  uint32_t to[kPer], vacant[kPer];  // where a page that stays goes; the place, if none will
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int p = j * kEvictThreads + t, at = lanes_below(mask[j], before[j]);  // pages before p that stay
    to[j] = key[j] > last ? (uint32_t)at * 4 : kNowhere;
    vacant[j] = p >= keep ? off[j] : kNowhere;
    table_out.put(to[j], (uint32_t)id[j]);
    table_out.put(vacant[j], ~0u);
    freed_row.put(key[j] > last ? kNowhere : (uint32_t)(p - at) * 4, (uint32_t)id[j]);
    if constexpr (!kSums) kept_row.put(to[j], (uint32_t)p);
  }
  if constexpr (kSums) {  // some heads are read before they are written, as it may be in place; few heads are here already
    for (int h0 = 0; h0 < c.Hkv; h0 += kAhead) {
      if (c.Hkv > kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const Row in(a.weights_in + rows + (int64_t)min(h0 + u, c.Hkv - 1) * a.weight_stride, P);
#pragma unroll
          for (int j = 0; j < kPer; ++j) w[u][j] = in.real(off[j]);
        }
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (h0 + u >= c.Hkv) break;  // uniform
        const Row out(a.weights_out + rows + (int64_t)(h0 + u) * a.weight_stride, P);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          out.put(to[j], __float_as_uint(w[u][j]));
          out.put(vacant[j], 0u);
        }
      }
    }
  }
  for (int i = P - keep + t; i < a.freed_stride; i += kEvictThreads) freed[i] = -1;
  if (t == 0) {
    a.freed_count[b] = P - keep;
    a.seq_lens_out[b] = N - (P - keep) * c.S;
    if constexpr (!kSums) {
      pages[b] = P;
      kept_count[b] = keep;
    }
  }
}

constexpr int kCloseThreads = 512, kCloseBatch = 8;

// Closes rows up to the kept pages, in place or not: kept[] ascends, so that entry i comes from kept[i] >= i and a round of the
// workgroup, which reads before it writes, leaves what later rounds read. blockIdx.x < Hkv: the accounts of a KV head; else the table, and
// the length, which nothing else of this launch reads: it may be written in place.
__global__ __launch_bounds__(kCloseThreads) void close_kernel(CacheView c, EvictArgs a, const int32_t* __restrict__ kept,
                                                              const int32_t* __restrict__ pages, const int32_t* __restrict__ kept_count) {
  const int b = blockIdx.y, t = threadIdx.x;
  const int P = pages[b], n = kept_count[b];
  const Row from(kept + (int64_t)b * a.budget, n);
  const bool accounts = (int)blockIdx.x < c.Hkv;
  const int64_t row = accounts ? ((int64_t)b * c.Hkv + blockIdx.x) * a.weight_stride : (int64_t)b * c.max_pages;
  const Row in(accounts ? (const void*)(a.weights_in + row) : c.page_table + row, P);
  const Row out(accounts ? (void*)(a.weights_out + row) : a.page_table_out + row, P);
  for (int i0 = 0; i0 < n; i0 += kCloseThreads * kCloseBatch) {
    uint32_t v[kCloseBatch];
#pragma unroll
    for (int u = 0; u < kCloseBatch; ++u) v[u] = from.word((uint32_t)(i0 + u * kCloseThreads + t) * 4);  // 0 behind the last
#pragma unroll
    for (int u = 0; u < kCloseBatch; ++u) v[u] = in.word(v[u] * 4);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kCloseBatch; ++u) {
      const int i = i0 + u * kCloseThreads + t;
      out.put(i < n ? (uint32_t)i * 4 : kNowhere, v[u]);
    }
  }
  __syncthreads();
  if (!accounts && t == 0) a.seq_lens_out[b] = c.seq_lens[b] - (P - n) * c.S;
  const uint32_t vacant = accounts ? 0u : ~0u;
  for (int i = n + t; i < P; i += kCloseThreads) out.put((uint32_t)i * 4, vacant);
}

// The freed pages of a part of a sequence whose kept pages launch_select has chosen, for rows that no workgroup holds; the first part also writes
// their number and what lies behind them. Before close_kernel, which may overwrite the table and the lengths: every part reads both.
constexpr int kFreedEach = 4, kFreedPages = kFreedEach * kEvictThreads;
__global__ __launch_bounds__(kEvictThreads) void freed_kernel(CacheView c, EvictArgs a, const int32_t* __restrict__ kept,
                                                              const int32_t* __restrict__ kept_count, int32_t* __restrict__ pages) {
  __shared__ uint32_t s_stays[kFreedPages];
  __shared__ int s_counts[kEvictWaves];
  const int b = blockIdx.y, t = threadIdx.x, lane = t % kWave, wave = t / kWave;
  const int P = max(min((c.seq_lens[b] + c.S - 1) / c.S, c.max_pages_hint), 0), n = kept_count[b], first = blockIdx.x * kFreedPages;
  const int32_t* from = kept + (int64_t)b * a.budget;
  int32_t* freed = a.freed_pages + (int64_t)b * a.freed_stride;
  if (first == 0) {
    for (int i = P - n + t; i < a.freed_stride; i += kEvictThreads) freed[i] = -1;
    if (t == 0) {
      a.freed_count[b] = P - n;
      pages[b] = P;
    }
  }
  if (first >= P) return;
  int lo = 0, hi = n;  // kept pages before `first`
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (from[mid] < first) lo = mid + 1;
    else hi = mid;
  }
#pragma unroll
  for (int u = 0; u < kFreedEach; ++u) s_stays[u * kEvictThreads + t] = 0;
  __syncthreads();
  for (int i = lo + t; i < n; i += kEvictThreads) {
    const int p = from[i] - first;
    if (p >= kFreedPages) break;
    s_stays[p] = 1;
  }
  __syncthreads();
  uint32_t stays[kFreedEach];
  int mine = 0;
#pragma unroll
  for (int u = 0; u < kFreedEach; ++u) mine += stays[u] = s_stays[t * kFreedEach + u];
  const int upto = wave_inclusive_scan(mine);
  if (lane == kWave - 1) s_counts[wave] = upto;
  __syncthreads();
  int before = lo + upto - mine;
  for (int w = 0; w < wave; ++w) before += s_counts[w];
#pragma unroll
  for (int u = 0; u < kFreedEach; ++u) {
    const int p = first + t * kFreedEach + u;
    if (p < P && !stays[u]) freed[p - before] = c.page_table[(int64_t)b * c.max_pages + p];
    before += stays[u];
  }
}

size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }
int rank_stride_of(const CacheView& c) { return (c.max_pages_hint + kScoreStrideAlign - 1) / kScoreStrideAlign * kScoreStrideAlign; }

}  // namespace

// Cut as unique_dense_paged_decode cuts, or not at all where lists would not be; and batches of more rows than it cuts by their lengths are, where
// a row is long, into two chunks to a row or more: with one workgroup to a row the longest row bounds them, and so do rows that are not a multiple of
// the workgroups at a time. us one to a row / so (8 KV heads, G = 4, D = 128, pages of 16): 40 sequences of 1K to 4K tokens 107 / 75, even 138 / 111, 64 of 300 to
// 3100 87 / 68, 40 of 500 to 5000 with eight heads 131 / 66, 33 of 300 to 3000, fp32, 108 / 60, 33 x 2000 69 / 57. About 512 rows that are even and not
// so long fill two workgroups to a compute unit as they are: 64 x 2000 83 / 91, which is why these have to be longer (64 of 200 to 2000 would gain, 55 / 48).
static WeighCut weigh_cut(const CacheView& c) {
  const int rows = c.B * c.Hkv, page_bytes = c.S * c.D * 2 * (c.dtype == 0 ? 4 : 2);
  WeighCut cut = {selection_plan(c, c.max_pages_hint), 0, {}};
  if (cut.plan.num_splits > 1) cut.plan = most_splits(rows, c.max_pages_hint);
  if (dense_balances(c.B, c.Hkv, c.max_pages_hint, page_bytes)) {
    cut.max_chunks = dense_max_chunks(rows, c.max_pages_hint);
  } else if (rows > kDenseSlots / 2 && rows <= 2 * kDenseSlots && c.B <= kDenseMaxBatch && (int64_t)rows * c.max_pages_hint <= INT32_MAX &&
             (int64_t)c.max_pages_hint * page_bytes >= (rows <= 384 ? 512 << 10 : 1024 << 10)) {
    cut.round.slots = (2 * rows + kDenseSlots - 1) / kDenseSlots * kDenseSlots;
    cut.max_chunks = (int)dense_wanted_chunks(rows, c.max_pages_hint, cut.round);
  }
  return cut;
}
static size_t weigh_slots(const CacheView& c, const WeighCut& cut) {
  return cut.max_chunks > 0 ? cut.max_chunks : (size_t)c.B * c.Hkv * cut.plan.num_splits;
}

size_t weigh_floats(const CacheView& c) {
  return weigh_slots(c, weigh_cut(c)) * (c.H / c.Hkv) * (c.D + 2) + (size_t)c.B * c.H * c.max_pages_hint;
}

hipError_t launch_weigh(const CacheView& c, const WeighArgs& a, hipStream_t stream) {
  const WeighCut cut = weigh_cut(c);
  const size_t heads = weigh_slots(c, cut) * (c.H / c.Hkv);
  float* part_ml = a.partials + heads * c.D;
  float* shares = part_ml + heads * 2;
  auto run = [&](auto launch) { return launch(c, a, cut, part_ml, shares, stream); };
  return c.dtype == 0 ? (c.D == 64 ? run(launch_weigh_of<float, 64>) : run(launch_weigh_of<float, 128>))
                      : (c.D == 64 ? run(launch_weigh_of<bf16_t, 64>) : run(launch_weigh_of<bf16_t, 128>));
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
  hipError_t e = hipSuccess;
  const bool sums = (int64_t)c.Hkv * c.max_pages_hint <= kSumsHere && c.max_pages_hint <= 8192;  // (16 keys and accounts a thread spill)
  if (!sums) {
    const dim3 grid((c.max_pages_hint + kAccountThreads - 1) / kAccountThreads, c.B);
    rank_kernel<<<grid, dim3(kAccountThreads), 0, stream>>>(c, a.weights_in, a.weight_stride, a.sinks, rank, rank_stride);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  auto go = [&](auto kernel) {
    kernel<<<dim3(c.B), dim3(kEvictThreads), 0, stream>>>(c, a, rank, rank_stride, kept, pages, kept_count);
    return hipGetLastError();
  };
  auto held = [&](auto per) {
    constexpr int kPer = decltype(per)::value;
    return sums ? go(evict_kernel<kPer, true>) : go(evict_kernel<kPer, false>);
  };
  if (c.max_pages_hint <= 1024) e = held(std::integral_constant<int, 1>());
  else if (c.max_pages_hint <= 4096) e = held(std::integral_constant<int, 4>());
  else if (c.max_pages_hint <= 8192) e = held(std::integral_constant<int, 8>());
  else if (c.max_pages_hint <= kEvictMost) e = go(evict_kernel<16, false>);
  else {
    CacheView one = c;  // a row per sequence
    one.Hkv = one.H = 1;
    one.force_recent = a.recent;
    e = launch_select(one, rank, nullptr, rank_stride, a.budget, kept, kept_count, stream);
    if (e != hipSuccess) return e;
    freed_kernel<<<dim3((c.max_pages_hint + kFreedPages - 1) / kFreedPages, c.B), dim3(kEvictThreads), 0, stream>>>(c, a, kept, kept_count, pages);
    e = hipGetLastError();
  }
  if (e != hipSuccess || sums) return e;
  const bool held_here = c.max_pages_hint <= kEvictMost;  // then the table is closed already
  close_kernel<<<dim3(held_here ? c.Hkv : c.Hkv + 1, c.B), dim3(kCloseThreads), 0, stream>>>(c, a, kept, pages, kept_count);
  return hipGetLastError();
}

}  // namespace unique
