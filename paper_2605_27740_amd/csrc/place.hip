// Places for the new tokens of a step: pages from a stack of free ones, page table, lengths, positions and slots.
//
// Sequence b needs need_b = ceil((n_b + t_b) / S) - ceil(n_b / S) pages; with the sums of need over the sequences before it, its pages are known without
// asking the others: page i of all is entry n - 1 - i of a stack of n. So a workgroup forms four prefix sums over the batch (pages that come back twice,
// tokens, needs), and everything else is per page or per row. Small calls do all of it in one workgroup. In larger ones the rows have a launch of their own, as pages that
// come back must be on the stack before they are given out, and what the outputs may lie over (lengths, positions, the count of pages) is written there too: in the launch
// before it, all workgroups of which make the plan, it is still read.
#include "decode_core.hpp"
#include "place_plan.hpp"
#include "serving.hpp"

namespace unique {
namespace {

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / kWave;
constexpr int kFillThreads = 256;
constexpr int kMostTokens = 1 << 25;              // where sums of tokens saturate, above any number of rows

enum SeatState { kUnplaced = 0, kPlaced = 1, kEnded = 2 };
struct Seat {  // what the rows of a sequence's new tokens need
  int len, first, position, state;  // its length, its first page among all that are given out
};
struct Back {  // what a sequence gives back
  int freed_at, own_at, freed, pages;  // places on the stack; evicted pages, pages of its row if it has ended
};
struct PlaceArrays {
  Seat* seat;   // [B]
  Back* back;   // [B]
  int* starts;  // [B + 1]
  int* size;    // the stack's, with what has come back, and how many pages are given out
};

__device__ __forceinline__ int pages_of(int tokens, int S) { return (tokens + S - 1) / S; }

// Sums over the workgroup of up to 64 Ki values each, whose total fits.
__device__ __forceinline__ int block_sum(int x, int* scratch) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int upto = wave_inclusive_scan(x);
  __syncthreads();
  if (lane == kWave - 1) scratch[wave] = upto;
  __syncthreads();
  return __builtin_amdgcn_readlane(wave_inclusive_scan(lane < kPlanWaves ? scratch[lane] : 0), kWave - 1);
}

// The plan of the whole batch by one workgroup. A thread takes sequences t, t + 1024, ..., so nothing is read that another one writes.
__device__ __forceinline__ void plan_places(const CacheView& c, const unique_placement& p, const PlaceArrays& to) {
  __shared__ int s_scan[4][kPlanWaves], s_sum[kPlanWaves];
  const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, S = c.S;
  const int capacity = p.free_capacity;
  const int64_t most = (int64_t)c.max_pages * S;
  auto freed_of = [&](int b) { return p.freed_count ? min(max(p.freed_count[b], 0), p.freed_stride) : 0; };
  auto length_of = [&](int b) { return (int)min((int64_t)max(c.seq_lens[b], 0), most); };
  auto own_of = [&](int b, int pages) { return pages - (p.shared_pages ? min(max(p.shared_pages[b], 0), pages) : 0); };

  int freed_all = 0, own_all = 0;
  for (int b = t; b < c.B; b += kPlanThreads) {
    freed_all += freed_of(b);
    if (p.new_tokens[b] < 0) own_all += own_of(b, pages_of(length_of(b), S));
  }
  const int before = min(max(*p.free_count, 0), capacity);
  freed_all = block_sum(freed_all, s_sum);
  own_all = block_sum(own_all, s_sum);
  const int size = stack_place(before, (int64_t)freed_all + own_all, capacity);

  int base[4] = {0, 0, 0, 0}, given = 0;  // freed, own, tokens, needs before the strip
  for (int b0 = 0; b0 < c.B; b0 += kPlanThreads) {
    const int b = b0 + t;
    const bool live = b < c.B;
    const int len = live ? length_of(b) : 0, asked = live ? p.new_tokens[b] : 0, pages = pages_of(len, S);
    const bool ended = asked < 0;
    const int tokens = min(max(asked, 0), kMostTokens);
    const bool fits = (int64_t)len + tokens <= most;
    const int freed = live ? freed_of(b) : 0, own = live && ended ? own_of(b, pages) : 0;
    const int need = fits && !ended ? pages_of(len + tokens, S) - pages : 0;
    int x[4] = {freed, own, tokens, need}, upto[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      upto[i] = wave_inclusive_scan(x[i]);
      if (i == 2) upto[i] = (int)min((uint32_t)upto[i], (uint32_t)kMostTokens);
    }
    __syncthreads();
    if (lane == kWave - 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s_scan[i][wave] = upto[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int waves = wave_inclusive_scan(lane < kPlanWaves ? s_scan[i][lane] : 0);
      const int mine = base[i] + upto[i] + (wave > 0 ? __builtin_amdgcn_readlane(waves, wave - 1) : 0);
      upto[i] = i == 2 ? min(mine, kMostTokens) : mine;
      base[i] += __builtin_amdgcn_readlane(waves, kWave - 1);
      if (i == 2) base[i] = min(base[i], kMostTokens);
    }
    if (live) {
      // Sequences whose rows are not there are the last ones, so their needs may count.
      const bool ok = !ended && fits && upto[2] <= p.max_new_tokens && (need == 0 || upto[3] <= size);
      const int position = p.next_positions ? p.next_positions[b] : len;
      to.seat[b] = Seat{len, upto[3] - need, position, ended ? kEnded : (ok ? kPlaced : kUnplaced)};
      to.back[b] = Back{stack_place(before, upto[0] - freed, capacity), stack_place(before, (int64_t)freed_all + (upto[1] - own), capacity), freed, ended ? pages : 0};
      to.starts[b] = upto[2] - tokens;
      if (b == c.B - 1) to.starts[c.B] = upto[2];
      if (ok && need > 0) given = upto[3];  // (the largest is the last)
    }
  }
  __syncthreads();
  // the most of the workgroup: sums of needs only grow
  given = (int)wave_allreduce_minmax<true>((uint32_t)given);
  if (lane == 0) s_sum[wave] = given;
  __syncthreads();
  if (t == 0) {
    for (int w = 0; w < kPlanWaves; ++w) given = max(given, s_sum[w]);
    to.size[0] = size;
    to.size[1] = given;
  }
}

// Pages of sequence b go back, by the threads of a workgroup or wave.
__device__ __forceinline__ void give_back(const CacheView& c, const unique_placement& p, const Back& k, int b, int from, int step) {
  for (int64_t i = from; i < k.freed; i += step)
    if (stack_has(k.freed_at, (int)i, p.free_capacity)) p.free_pages[k.freed_at + i] = p.freed_pages[(int64_t)b * p.freed_stride + i];
  if (k.pages == 0) return;
  const int shared = p.shared_pages ? min(max(p.shared_pages[b], 0), k.pages) : 0;
  const int64_t row = (int64_t)b * c.max_pages;
  constexpr int kFew = 8;  // loads in flight
  for (int i0 = from; i0 < k.pages; i0 += kFew * step) {
    int page[kFew];
#pragma unroll
    for (int u = 0; u < kFew; ++u) page[u] = c.page_table[row + (i0 + u * step < k.pages ? i0 + u * step : i0)];  // this thread's own
#pragma unroll
    for (int u = 0; u < kFew; ++u) {
      const int i = i0 + u * step;
      if (i >= k.pages) break;
      if (i >= shared && stack_has(k.own_at, i - shared, p.free_capacity)) p.free_pages[k.own_at + i - shared] = page[u];
      p.page_table_out[row + i] = -1;
    }
  }
}

// What the caller is told of sequence b, and of the stack.
__device__ __forceinline__ void tell_sequence(const CacheView& c, const unique_placement& p, const PlaceArrays& from, int b) {
  const Seat s = from.seat[b];
  const int start = from.starts[b], end = from.starts[b + 1], placed = s.state == kPlaced ? end - start : 0;
  p.token_starts[b] = start;
  if (b == c.B - 1) p.token_starts[c.B] = end;
  p.placed[b] = placed;
  p.seq_lens_out[b] = s.state == kEnded ? 0 : (placed > 0 ? s.len + placed : c.seq_lens[b]);  // (as it was, also where that is no length of this row)
  if (p.next_positions_out) p.next_positions_out[b] = s.state == kEnded ? 0 : s.position + placed;
  if (b == 0) *p.free_count_out = from.size[0] - from.size[1];
}

// The first sequence from lo on whose rows end behind `row`; there is one.
__device__ __forceinline__ int sequence_of(const int* starts, int lo, int B, int row) {
  int hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (starts[mid + 1] > row) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// The same for 64 rows of a wave, lane after lane, of which the first has a sequence: all lanes look for that one's, in 64 places at a time, and the ends of 64 sequences from there on answer
// the others. Two trips to memory for 4096 sequences and one more, where a search by every lane makes twelve. With one launch fewer: 500 sequences of 1 to 2048 tokens 18.1 / 13.1 us,
// 32 prompts of 8000 to 32768 13.7 / 11.8.
__device__ __forceinline__ int sequence_of_lane(const int* starts, int B, int first, int lane) {
  int lo = 0, hi = B - 1;  // uniform
  while (lo < hi) {
    const int step = (hi - lo + kWave) / kWave, last = lo + (lane + 1) * step - 1;
    const bool behind = last >= hi || starts[last + 1] > first;
    lo += __builtin_ctzll(__ballot(behind)) * step;
    hi = min(lo + step - 1, hi);
  }
  const int end = starts[min(lo + 1 + lane, B)], row = first + lane;
  int at = 0;  // sequences of the 64 that end at or before the row
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) at += __shfl(end, at + d - 1, kWave) <= row ? d : 0;
  if (__builtin_amdgcn_readlane(end, kWave - 1) <= row) return sequence_of(starts, min(lo + kWave, B - 1), B, row);
  return min(lo + at, B - 1);
}

// Position and slot of a row, of sequence b if it has one; the first token of a page also writes the page's entry of the table.
__device__ __forceinline__ void fill_row(const CacheView& c, const unique_placement& p, const PlaceArrays& from, int size, int row, int b) {
  int position = -1;
  int64_t slot = -1;
  if (b >= 0) {
    const Seat s = from.seat[b];
    if (s.state == kPlaced) {
      const int i = row - from.starts[b], at = s.len + i, lp = at / c.S, have = pages_of(s.len, c.S);
      const int64_t entry = (int64_t)b * c.max_pages + lp;
      const int page = lp < have ? c.page_table[entry] : p.free_pages[size - 1 - (s.first + lp - have)];
      position = s.position + i;
      slot = page < 0 ? -1 : (int64_t)page * c.S + at % c.S;
      if (at % c.S == 0) p.page_table_out[entry] = page;
    }
  }
  p.positions[row] = position;
  p.slots[row] = slot;
}

struct PlaceShared {
  Seat seat[kPlanThreads];
  Back back[kPlanThreads];
  int starts[kPlanThreads + 1], size[2];
};

__global__ __launch_bounds__(kPlanThreads) void place_kernel(CacheView c, unique_placement p) {
  __shared__ PlaceShared sh;
  const PlaceArrays at = {sh.seat, sh.back, sh.starts, sh.size};
  plan_places(c, p, at);
  __syncthreads();
  for (int b = threadIdx.x / kWave; b < c.B; b += kPlanWaves) give_back(c, p, sh.back[b], b, threadIdx.x % kWave, kWave);
  for (int b = threadIdx.x; b < c.B; b += kPlanThreads) tell_sequence(c, p, at, b);
  __threadfence_block();  // the stack is read by other waves
  __syncthreads();
  for (int row = threadIdx.x; row < p.max_new_tokens; row += kPlanThreads)
    fill_row(c, p, at, sh.size[0], row, row < sh.starts[c.B] ? sequence_of(sh.starts, 0, c.B, row) : -1);
}

// The plan, by every workgroup, and what its sequences give back.
__global__ __launch_bounds__(kPlanThreads) void place_back_kernel(CacheView c, unique_placement p, PlaceArrays to) {
  __shared__ PlaceShared sh;
  const PlaceArrays at = {sh.seat, sh.back, sh.starts, sh.size};
  plan_places(c, p, at);
  __syncthreads();
  const int t = threadIdx.x;
  if (blockIdx.x == 0) {
    if (t < c.B) to.seat[t] = sh.seat[t];
    for (int b = t; b <= c.B; b += kPlanThreads) to.starts[b] = sh.starts[b];
    if (t < 2) to.size[t] = sh.size[t];
  }
  for (int b = blockIdx.x; b < c.B; b += gridDim.x) give_back(c, p, sh.back[b], b, t, kPlanThreads);
}

// The same in two, where the LDS does not hold the plan.
__global__ __launch_bounds__(kPlanThreads) void place_many_plan_kernel(CacheView c, unique_placement p, PlaceArrays at) { plan_places(c, p, at); }

__global__ __launch_bounds__(kFillThreads) void place_many_back_kernel(CacheView c, unique_placement p, PlaceArrays at) {
  for (int b = blockIdx.x; b < c.B; b += gridDim.x) give_back(c, p, at.back[b], b, threadIdx.x, kFillThreads);
}

// The first workgroups take sequences, the others rows, one a thread (four: 13.1 and 11.8 us where one takes 10.2 and 9.9).
__global__ __launch_bounds__(kFillThreads) void place_fill_kernel(CacheView c, unique_placement p, PlaceArrays at) {
  const int tells = (c.B + kFillThreads - 1) / kFillThreads;
  if ((int)blockIdx.x < tells) {
    const int b = blockIdx.x * kFillThreads + threadIdx.x;
    if (b < c.B) tell_sequence(c, p, at, b);
    return;
  }
  const int size = at.size[0], all = at.starts[c.B];
  const int row = (blockIdx.x - tells) * kFillThreads + threadIdx.x, lane = row % kWave;
  if (row - lane >= p.max_new_tokens) return;  // uniform, as below
  const int b = row - lane < all ? sequence_of_lane(at.starts, c.B, row - lane, lane) : -1;
  if (row < p.max_new_tokens) fill_row(c, p, at, size, row, row < all ? b : -1);
}

// One workgroup takes 5 us, 1 for 1024 rows, 1 for 120 sequences and 1 for 5600 pages that ended sequences give back; two launches take 10 whatever there is: 64 sequences and 2048 rows 7.1 / 10.1, 4096 rows
// 9.4 / 10.5, 8192 rows 13.9 / 10.5; 1000 sequences and 2000 rows 15.4 / 9.7; 360 sequences of up to 13600 pages, 66 of which end, 163 / 11.1. Which sequences end the host does not know:
// rows of the table that hold 2^18 pages in all are 47 us at the very worst.
bool place_is_small(const CacheView& c, int max_new_tokens) {
  return c.B <= kPlanThreads && max_new_tokens + 8ll * c.B <= 5120 && (int64_t)c.B * c.max_pages <= 1 << 18;
}

}  // namespace

size_t place_bytes(const CacheView& c, int max_new_tokens) {
  if (place_is_small(c, max_new_tokens)) return 0;
  return (size_t)c.B * (sizeof(Seat) + sizeof(Back)) + ((size_t)c.B + 3) * sizeof(int);
}

hipError_t launch_place(const CacheView& c, const unique_placement& p, void* workspace, hipStream_t st) {
  if (place_is_small(c, p.max_new_tokens)) {
    place_kernel<<<dim3(1), dim3(kPlanThreads), 0, st>>>(c, p);
    return hipGetLastError();
  }
  PlaceArrays at;
  at.seat = reinterpret_cast<Seat*>(workspace);
  at.back = reinterpret_cast<Back*>(at.seat + c.B);
  at.starts = reinterpret_cast<int*>(at.back + c.B);
  at.size = at.starts + c.B + 1;
  if (c.B <= kPlanThreads) {
    place_back_kernel<<<dim3(c.B < 256 ? c.B : 256), dim3(kPlanThreads), 0, st>>>(c, p, at);
  } else {
    place_many_plan_kernel<<<dim3(1), dim3(kPlanThreads), 0, st>>>(c, p, at);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    place_many_back_kernel<<<dim3(c.B < 2048 ? c.B : 2048), dim3(kFillThreads), 0, st>>>(c, p, at);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int tells = (c.B + kFillThreads - 1) / kFillThreads, rows = (p.max_new_tokens + kFillThreads - 1) / kFillThreads;
  place_fill_kernel<<<dim3(tells + rows), dim3(kFillThreads), 0, st>>>(c, p, at);
  return hipGetLastError();
}

}  // namespace unique
