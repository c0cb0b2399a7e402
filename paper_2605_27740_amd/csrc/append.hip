// Queries, keys and values of new tokens: each query and key head normalised by its root mean square and turned by its position, keys and values
// written to their slots.
//
//   y = x / sqrt(mean(x^2) + eps) * w;  a pair (y_1, y_2) becomes m (y_1 cos a - y_2 sin a, y_1 sin a + y_2 cos a), a = position * f
//
// Memory bounds it: every element is read and written once. A lane holds two 16-byte pieces of a head, those whose channels are paired if the
// pairs are halves of the head, so a pair never leaves its lane; D / (2 * 16 bytes) lanes hold a head and a wave 4 to 16 heads at a time. All heads of a token
// share their angles: lane i of the wave forms those of pair i once, in turns and in 64 bits (a position of 2^20 times a frequency
// leaves 2^-33 of a turn, where 32 bits would leave 2^-4), and the wave takes them from the LDS. Sine and cosine are formed in 64 bits as well, and rounded once: by a
// function of 32 bits fp32 heads were 1.6 times as far from 64 bits as a plain form's. us in 64 / 32 bits: 8192 tokens of 48 bf16 heads 40.1 / 40.4, 65536 of 80 453 / 448.
#include <type_traits>

#include "decode_core.hpp"
#include "serving.hpp"

namespace unique {
namespace {

constexpr int kAppendWaves = 4;

template <typename T>
__device__ __forceinline__ Raw16 pack_vec(const float (&x)[Elem<T>::kVec]) {
  Raw16 r;
  if constexpr (sizeof(T) == 4) {
    r.v = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)float_to_bf16(x[2 * i]) | (uint32_t)float_to_bf16(x[2 * i + 1]) << 16;
    r.v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return r;
}

// m cos and m sin of x turns, |x| <= 1/2, rounded once. Of the nearest quarter turn r is left, pi / 4 at most, for which the series' next terms are 2^-36 of sine and 2^-40 of cosine.
__device__ __forceinline__ float2 cos_sin_of_turns(double x, float m) {
  const double quarter = rint(4.0 * x), r = fma(-0.25, quarter, x) * 6.283185307179586, z = r * r;
  double s = fma(z, -1.0 / 39916800, 1.0 / 362880), c = fma(z, 1.0 / 479001600, -1.0 / 3628800);
  s = fma(z, s, -1.0 / 5040);
  c = fma(z, c, 1.0 / 40320);
  s = fma(z, s, 1.0 / 120);
  c = fma(z, c, -1.0 / 720);
  s = fma(z, s, -1.0 / 6);
  c = fma(z, c, 1.0 / 24);
  s = fma(z * r, s, r);
  c = fma(z, c, -0.5);
  c = fma(z, c, 1.0);
  const int q = (int)quarter & 3;
  const double cs = q & 1 ? s : c, sn = q & 1 ? c : s;
  return make_float2((float)(q == 1 || q == 2 ? -m * cs : m * cs), (float)(q & 2 ? -m * sn : m * sn));
}

// kInterleaved: pairs are neighbours. A wave takes kAhead steps of a token's heads, of which there are `parts`. early: the first heads are asked for before the slot is known.
template <typename T, int D, bool kInterleaved, int kAhead>
__global__ __launch_bounds__(kAppendWaves* kWave) void append_kernel(CacheView c, AppendArgs a, int parts, bool early) {
  constexpr int kVec = Elem<T>::kVec;
  constexpr int kLanes = D / kVec / 2;      // lanes of a head
  constexpr int kHeads = kWave / kLanes;    // heads of a step
  __shared__ float2 s_turn[kAppendWaves][D / 2];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t item = (int64_t)blockIdx.x * kAppendWaves + wave;
  const int64_t row = item / parts;
  if (row >= a.rows) return;  // (no barrier below)
  const int part = (int)(item - row * parts);
  const int64_t slot = a.slots[row];
  const int position = a.positions[row];
  // This lane's two pieces of a head: where halves are paired, one of each half; behind the turned channels neighbours.
  const int R = a.how.rotary_dim, mine = lane % kLanes, pairs = kInterleaved ? 0 : R / (2 * kVec);
  const int c0 = mine < pairs ? mine : 2 * pairs + 2 * (mine - pairs), c1 = mine < pairs ? mine + pairs : c0 + 1;
  const bool norm = a.how.q_weight != nullptr;
  Raw16 wq[2], wk[2];
  if (norm) {
    wq[0] = load_raw(reinterpret_cast<const T*>(a.how.q_weight) + c0 * kVec);
    wq[1] = load_raw(reinterpret_cast<const T*>(a.how.q_weight) + c1 * kVec);
    wk[0] = load_raw(reinterpret_cast<const T*>(a.how.k_weight) + c0 * kVec);
    wk[1] = load_raw(reinterpret_cast<const T*>(a.how.k_weight) + c1 * kVec);
  }
  const int all = c.H + 2 * c.Hkv;
  const T* q = reinterpret_cast<const T*>(a.q) + row * a.q_stride;
  const T* k = reinterpret_cast<const T*>(a.k) + row * a.k_stride;
  const T* v = reinterpret_cast<const T*>(a.v) + row * a.v_stride;

  auto load = [&](int step, Raw16(&x)[2]) {
    const int head = min(step * kHeads + lane / kLanes, all - 1);
    const T* src = head < c.H ? q + head * D : (head < c.H + c.Hkv ? k + (head - c.H) * D : v + (head - c.H - c.Hkv) * D);
    x[0] = load_raw(src + c0 * kVec);
    x[1] = load_raw(src + c1 * kVec);
  };
  const int begin = part * kAhead;
  Raw16 x[kAhead][2];
  auto load_all = [&] {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load(begin + u, x[u]);  // (of a step that there is not: the last head again)
  };
  if (early) load_all();
  if (slot < 0 || slot >= c.num_phys * c.S) return;
  if (lane < R / 2) {
    const double turns = (double)position * (a.how.frequencies[lane] * 0.15915494309189535);
    s_turn[wave][lane] = cos_sin_of_turns(turns - rint(turns), a.how.magnitude);
  }
  __builtin_amdgcn_wave_barrier();  // the LDS serves a wave's accesses in order; the compiler keeps it

  const int shift = __builtin_ctz(c.S), place = (int)slot & (c.S - 1);
  T* q_out = reinterpret_cast<T*>(a.q_out) + row * c.H * D;
  const int64_t token = (slot >> shift) * c.kv_page_stride + (int64_t)place * D;
  T* kc = reinterpret_cast<T*>(const_cast<void*>(c.k_cache)) + token;
  T* vc = reinterpret_cast<T*>(const_cast<void*>(c.v_cache)) + token;

  auto finish = [&](int step, Raw16(&x)[2]) {
    const int head = step * kHeads + lane / kLanes;
    const bool is_q = head < c.H, is_v = head >= c.H + c.Hkv;
    float y[2][kVec];
    unpack_raw(x[0], y[0], (const T*)nullptr);
    unpack_raw(x[1], y[1], (const T*)nullptr);
    if (norm) {  // uniform
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * kVec; ++i) sum = fmaf(y[i / kVec][i % kVec], y[i / kVec][i % kVec], sum);
      sum = group_allreduce<kLanes>(sum, OpSum());
      const float scale = 1.f / sqrtf(sum * (1.f / D) + a.how.eps);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float w[kVec];
        Raw16 raw;
        raw.v.x = is_q ? wq[u].v.x : wk[u].v.x; raw.v.y = is_q ? wq[u].v.y : wk[u].v.y;
        raw.v.z = is_q ? wq[u].v.z : wk[u].v.z; raw.v.w = is_q ? wq[u].v.w : wk[u].v.w;
        unpack_raw(raw, w, (const T*)nullptr);
#pragma unroll
        for (int i = 0; i < kVec; ++i) y[u][i] *= scale * w[i];
      }
    }
    if constexpr (kInterleaved) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int piece = u == 0 ? c0 : c1;
        if (piece * kVec < R) {
#pragma unroll
          for (int i = 0; i < kVec; i += 2) {
            const float2 t = s_turn[wave][piece * (kVec / 2) + i / 2];
            const float y0 = y[u][i], y1 = y[u][i + 1];
            y[u][i] = y0 * t.x - y1 * t.y;
            y[u][i + 1] = y0 * t.y + y1 * t.x;
          }
        }
      }
    } else if (mine < pairs) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float2 t = s_turn[wave][mine * kVec + i];
        const float y0 = y[0][i], y1 = y[1][i];
        y[0][i] = y0 * t.x - y1 * t.y;
        y[1][i] = y0 * t.y + y1 * t.x;
      }
    }
    if (head >= all) return;
    T* dst = is_q ? q_out + head * D
                  : (is_v ? vc + (int64_t)(head - c.H - c.Hkv) * c.kv_head_stride : kc + (int64_t)(head - c.H) * c.kv_head_stride);
    // values go as they are
    Raw16 z0 = pack_vec<T>(y[0]), z1 = pack_vec<T>(y[1]);
    if (is_v) { z0 = x[0]; z1 = x[1]; }
    *reinterpret_cast<uint4*>(dst + c0 * kVec) = z0.v;
    *reinterpret_cast<uint4*>(dst + c1 * kVec) = z1.v;
  };

  if (!early) load_all();
#pragma unroll
  for (int u = 0; u < kAhead; ++u) finish(begin + u, x[u]);
}

}  // namespace

hipError_t launch_append(const CacheView& c, const AppendArgs& a, hipStream_t st) {
  auto with = [&](auto elem, auto dim) {
    using T = decltype(elem);
    constexpr int D = decltype(dim)::value, kHeads = kWave / (D / Elem<T>::kVec / 2);
    const int steps = (c.H + 2 * c.Hkv + kHeads - 1) / kHeads;
    // Two steps a wave, whose angles and weights are formed once, or one where they are little of the time: fp32 heads and calls without norm, in long calls. us, two
    // steps / one, back to back on one set of rows: 8192 bf16 tokens of 48 heads 33.4 / 33.3, 24000 of 80 heads 165 / 177, 65536 445 / 479, without norm 473 / 430; 16384 fp32 tokens of 48 heads
    // 138 / 134. And one where all waves of one step run at once: 32 tokens 5.0 / 4.1 (the kernel).
    const bool one = (int64_t)a.rows * steps <= 8192 || (a.rows >= 16384 && (!a.how.q_weight || c.dtype == 0));
    const int per = one ? 1 : 2, parts = (steps + per - 1) / per;
    const int64_t items = (int64_t)a.rows * parts;
    const bool early = items <= 8192;  // all waves at once: otherwise tokens without a slot would be read in vain
    const int64_t blocks = (items + kAppendWaves - 1) / kAppendWaves;
    if (blocks >= (1ll << 32) / (kAppendWaves * kWave)) return hipErrorInvalidConfiguration;  // threads are counted in 32 bits
    auto go = [&](auto kernel) {
      kernel<<<dim3((unsigned)blocks), dim3(kAppendWaves * kWave), 0, st>>>(c, a, parts, early);
      return hipGetLastError();
    };
    if (one) return a.how.interleaved ? go(append_kernel<T, D, true, 1>) : go(append_kernel<T, D, false, 1>);
    return a.how.interleaved ? go(append_kernel<T, D, true, 2>) : go(append_kernel<T, D, false, 2>);
  };
  auto with_dim = [&](auto elem) {
    return c.D == 64 ? with(elem, std::integral_constant<int, 64>()) : with(elem, std::integral_constant<int, 128>());
  };
  return c.dtype == 0 ? with_dim(float()) : with_dim(bf16_t());
}

}  // namespace unique
