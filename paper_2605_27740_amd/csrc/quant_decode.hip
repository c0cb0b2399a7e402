// Attention of one new token over pages of 4-bit records (the number format: quant.hip, the layout: quant.hpp).
//
// Split-K as over full-precision pages: a workgroup of four waves takes a chunk of a row's list for all G query heads of the KV
// head, a second kernel merges the chunks. A wave takes 32 token slots at a time, two halves of 16. Both products run on the matrix cores in
// bf16: a code times its scale is a bf16 number exactly, and one conversion instruction makes two of them.
// q.k, v_mfma_f32_16x16x32_bf16 per half and 32 channels: A = the keys of 16 slots, lane L supplying slot L % 16 and the channels
// D/4 * (L / 16) + ..., which are consecutive bytes of the record and lie in one block, so that a lane needs one scale per
// half; B = the query heads, repeated over the 16 columns. Lane L ends up with the logits of slots 4 * (L / 16) + i of
// both halves for head L % 16 % G.
// p.V, one v_mfma_f32_16x16x32_bf16 per 16 channels and tile: A = the probabilities, which stay in their lanes -- its eight
// k are the two halves' four slots --, as parts of 8 bits in rows parts times heads; B = the values of those slots, channels
// D/16 * (L % 16) + e: 16 bytes of a half at D = 128, with a scale for each slot.
// fp32 queries are taken as three bf16 numbers (24 bits, exactly), three products instead of one. The probabilities are three parts as well
// (24 bits, exactly): with two an output whose terms cancel was off by 2^-16 of the terms. us with two / three for bf16 (8 KV heads, D = 128):
// 16 x 131072 tokens 353 / 356, eight heads, 12 of 2K to 50K, pages of 32 63.1 / 64.5, the latter's lists of 200 pages 15.7 / 16.8.
#include <type_traits>

#include "dense_cut.hpp"
#include "quant.hpp"

namespace unique {
namespace {

template <typename T, int D, int G>
struct QuantShared {  // the waves' results; output rows are parts times heads
  static constexpr int kSlots = G == 8 ? 16 : 3 * G;
  __attribute__((aligned(16))) float acc[kDecWaves][kSlots][D];
  float m[kDecWaves][G], l[kDecWaves][G];
};

template <bool kNT, typename V>
__device__ __forceinline__ V load_as(const char* p) {
  if constexpr (kNT) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else return *reinterpret_cast<const V*>(p);
}

// Eight codes times a scale (of which the exponent counts) as bf16 numbers.
__device__ __forceinline__ uint32_t two_of(uint32_t codes, float scale, std::integral_constant<int, 0>) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
}
__device__ __forceinline__ uint32_t two_of(uint32_t codes, float scale, std::integral_constant<int, 1>) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
}
__device__ __forceinline__ uint32_t two_of(uint32_t codes, float scale, std::integral_constant<int, 2>) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
}
__device__ __forceinline__ uint32_t two_of(uint32_t codes, float scale, std::integral_constant<int, 3>) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
}
template <int kAt>
using At = std::integral_constant<int, kAt>;

__device__ __forceinline__ bf16x8_t as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8_t, u32x4_t{a, b, c, d});
}
// The byte of a block's scale, at bits 8 * i, moved to a float's exponent; the bits around it do not count.
template <int i>
__device__ __forceinline__ float scale_at(uint32_t bytes) {
  if constexpr (i == 3) return __uint_as_float(bytes >> 1);
  else return __uint_as_float(bytes << (23 - 8 * i));
}

// What a lane holds of a half: 16 slots of keys and values with their scales.
template <int D>
struct QuantHalf {
  uint32_t k[D / 32];      // D/4 channels of slot L % 16
  uint32_t v[4 * D / 128]; // D/16 channels of four slots
  uint32_t ks, vs;         // a byte; four bytes
  int valid;               // how many of the slots 4 * (L / 16) + i hold a token (any value <= 0: none)
  bool full;               // all 16 slots do (uniform)
};

template <int D, int S, int G, bool kNT, typename T, typename Lookup>
__device__ __forceinline__ void quant_chunk(const CacheView& c, const char* __restrict__ records, const T* __restrict__ q, const Chunk& k, int wave,
                                            int lane, Lookup lookup, float scale_log2, const ChunkOut<T>& to, QuantShared<T, D, G>& sh) {
  constexpr QuantTile kT = {S, D};
  constexpr int kSlots32 = 32;                       // token slots of a tile
  constexpr int kSteps = D / 32;                     // q.k steps per half
  constexpr int kVB = D / 16;                        // channels of a value row per lane
  constexpr int kQ = sizeof(T) == 4 ? 3 : 1;         // bf16 numbers of a query element
  constexpr int kSlots = QuantShared<T, D, G>::kSlots;
  constexpr bool kThird = G == 8;                    // the third part of a probability is a product of its own
  constexpr float kRoom = 6.f;                       // log2: how far above the largest logit the reference is put

  const int hkv = k.hkv, b = k.b, begin = k.begin, end = k.end;
  const int kt = lane % 16, kg = lane / 16, part = kt / G;

  // B operand of q.k: query head kt % G, channels D/4 * kg + 8 * s + ...
  const T* q_row = q + ((int64_t)b * c.H + hkv * G + kt % G) * D + kg * (D / 4);
  bf16x8_t qa[kQ][kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    if constexpr (sizeof(T) == 2) {
      qa[0][s] = as_bf16x8(load_raw(q_row + s * 8));
    } else {
      uint32_t w[3][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 x = *reinterpret_cast<const float2*>(q_row + s * 8 + 2 * i);
        const float x1 = x.x - bf16_part(x.x), y1 = x.y - bf16_part(x.y);
        w[0][i] = pack_hi(__float_as_uint(x.x), __float_as_uint(x.y));
        w[1][i] = pack_hi(__float_as_uint(x1), __float_as_uint(y1));
        w[2][i] = pack_hi(__float_as_uint(x1 - bf16_part(x1)), __float_as_uint(y1 - bf16_part(y1)));
      }
#pragma unroll
      for (int j = 0; j < kQ; ++j) qa[j][s] = as_bf16x8(w[j][0], w[j][1], w[j][2], w[j][3]);
    }
  }

  // Softmax state of head kt % G as in decode_core.hpp: the reference m is kRoom above the largest logit and moves when one exceeds it.
  float m = kNegBig, l = 0.f;
  f32x4_t acc[kVB];  // acc[e][i]: output row 4 * kg + i (head row % G), channel kVB * kt + e
#pragma unroll
  for (int e = 0; e < kVB; ++e) acc[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  const int64_t page_bytes = (int64_t)c.Hkv * kT.bytes();
  const char* mine = records + (int64_t)hkv * kT.bytes();
  // where this lane's bytes lie behind the first slot of a half (S = 8: of its page)
  const int kslot = S == 8 ? kt % 8 : kt, vslot = S == 8 ? 4 * kg % 8 : 4 * kg;
  const uint32_t k_off = kT.k_codes() + kslot * (D / 2) + kg * (D / 8), v_off = kT.v_at(vslot, kt);
  const uint32_t ks_off = kT.k_scales() + kg * (D / 4) / kQuantBlock * S + kslot;
  const uint32_t vs_off = kT.v_scales() + kt * kVB / kQuantBlock * S + vslot;
  // bits of a probability that this lane's part of it is without: those of the parts before
  const uint32_t not_first = part >= 1 ? 0xffff0000u : 0u, not_second = part >= 2 ? 0xffff0000u : 0u;

  for (int e0 = begin + wave; e0 < end; e0 += kDecWaves * kWave) {
    int my_phys = 0, my_ntok = 0;
    if (e0 + lane * kDecWaves < end) lookup(e0 + lane * kDecWaves, e0 == begin + wave, my_phys, my_ntok);
    const int n_ent = min(kWave, (end - e0 + kDecWaves - 1) / kDecWaves);
    const int n_tiles = (n_ent * S + kSlots32 - 1) / kSlots32;

    // Loads are unconditional: an entry that is not a page, or none at all, reads the pool's first record, and slots past a sequence's end what
    // the record holds there; their probability is zero and so is, nearly, their scale (below).
    auto issue = [&](int tile, QuantHalf<D>(&half)[2]) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        QuantHalf<D>& x = half[h];
        const char *kp, *vp;  // the records of this lane's key slot and of its value slots
        constexpr int kHalf = S == 32 ? 16 : 0;
        const int first = h * kHalf;  // slot of the page that the half begins with
        if constexpr (S >= 16) {      // one page: scalar
          const int ent = min((tile * kSlots32 + h * 16) / S, kWave - 1);
          const int phys = __builtin_amdgcn_readlane(my_phys, ent);
          const int ntok = tile < n_tiles ? __builtin_amdgcn_readlane(my_ntok, ent) : 0;
          kp = vp = mine + phys * page_bytes;
          x.valid = ntok - first - vslot;
          x.full = ntok >= first + 16;
        } else {  // two pages
          const int e1 = min(tile * 4 + h * 2, kWave - 1), e2 = min(e1 + 1, kWave - 1);
          const int p1 = __builtin_amdgcn_readlane(my_phys, e1), p2 = __builtin_amdgcn_readlane(my_phys, e2);
          const int n1 = __builtin_amdgcn_readlane(my_ntok, e1), n2 = __builtin_amdgcn_readlane(my_ntok, e2);
          kp = mine + (kt < 8 ? p1 : p2) * page_bytes;
          vp = mine + (kg < 2 ? p1 : p2) * page_bytes;
          x.valid = (tile < n_tiles ? (kg < 2 ? n1 : n2) : 0) - vslot;
          x.full = tile < n_tiles && n1 >= 8 && n2 >= 8;
        }
        if constexpr (D == 128) {
          const u32x4_t kw = load_as<kNT, u32x4_t>(kp + first * (D / 2) + k_off);
          const u32x4_t vw = load_as<kNT, u32x4_t>(vp + first * (D / 2) + v_off);
#pragma unroll
          for (int i = 0; i < 4; ++i) { x.k[i] = kw[i]; x.v[i] = vw[i]; }
        } else {
          const u32x2_t kw = load_as<kNT, u32x2_t>(kp + first * (D / 2) + k_off);
          const u32x2_t vw = load_as<kNT, u32x2_t>(vp + first * (D / 2) + v_off);
#pragma unroll
          for (int i = 0; i < 2; ++i) { x.k[i] = kw[i]; x.v[i] = vw[i]; }
        }
        x.ks = load_as<kNT, uint8_t>(kp + first + ks_off);
        x.vs = load_as<kNT, uint32_t>(vp + first + vs_off);
      }
    };
    auto consume = [&](QuantHalf<D>(&half)[2]) {
      f32x4_t logits[2];
      float x[8];
      auto relative = [&] {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaf(logits[i / 4][i % 4], scale_log2, -m);
      };
      const bool full = half[0].full && half[1].full;  // uniform
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float sk = scale_at<0>(half[h].ks);
        f32x4_t sacc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
          const uint32_t w = half[h].k[st];
          const bf16x8_t a = as_bf16x8(two_of(w, sk, At<0>()), two_of(w, sk, At<1>()), two_of(w, sk, At<2>()), two_of(w, sk, At<3>()));
#pragma unroll
          for (int j = 0; j < kQ; ++j) sacc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qa[j][st], sacc, 0, 0, 0);
        }
        logits[h] = sacc;
      }
      if (!full) {  // a slot without a token may hold any scale, also the one that stands for NaN: that of its value becomes the smallest
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int n = half[h].valid;
#pragma unroll
          for (int i = 0; i < 4; ++i) logits[h][i] = i < n ? logits[h][i] : -INFINITY;
          half[h].vs &= n >= 4 ? ~0u : (n <= 0 ? 0u : (1u << (8 * n)) - 1u);
        }
      }
      relative();
      float top = x[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
      if (__any(top > 0.f)) {
        float t = -INFINITY;  // from the logits themselves: m may still be kNegBig
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) t = fmaxf(t, logits[h][i] * scale_log2);
        const float mnew = fmaxf(m, rows_allreduce(t, OpMax()) + kRoom);
        const float alpha = fast_exp2(m - mnew);
        m = mnew;
        l *= alpha;
        relative();
        // output row 4 * kg + i belongs to head (4 * kg + i) % G, whose alpha lane (4 * kg + i) % G holds
        float row_alpha[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          auto lane_alpha = [&](int n) {
            return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(alpha), n));
          };
          row_alpha[i] = lane_alpha(i % G);
          if constexpr (G == 8) row_alpha[i] = kg % 2 ? lane_alpha(4 + i) : row_alpha[i];
        }
#pragma unroll
        for (int e = 0; e < kVB; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[e][i] *= row_alpha[i];
      }
      uint32_t pa[8], pb[8];  // this lane's part of the probabilities; pb: the third part in a product of its own
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = fast_exp2(x[i]);
        l += p;
        float r = p - __uint_as_float(__float_as_uint(p) & not_first);
        if constexpr (kThird) {
          const float r1 = p - bf16_part(p);
          pb[i] = __float_as_uint(r1 - bf16_part(r1)) & ~not_first;
        } else {
          r -= __uint_as_float(__float_as_uint(r) & not_second);
        }
        pa[i] = __float_as_uint(r);
      }
      const bf16x8_t a0 = as_bf16x8(pack_hi(pa[0], pa[1]), pack_hi(pa[2], pa[3]), pack_hi(pa[4], pa[5]), pack_hi(pa[6], pa[7]));
      bf16x8_t a1 = a0;
      if constexpr (kThird) a1 = as_bf16x8(pack_hi(pb[0], pb[1]), pack_hi(pb[2], pb[3]), pack_hi(pb[4], pb[5]), pack_hi(pb[6], pb[7]));
      uint32_t v[8][kVB / 2];  // two channels of a slot
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float s0 = scale_at<0>(half[h].vs), s1 = scale_at<1>(half[h].vs), s2 = scale_at<2>(half[h].vs), s3 = scale_at<3>(half[h].vs);
        const float sv[4] = {s0, s1, s2, s3};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (D == 128) {
            const uint32_t w = half[h].v[i];
            v[4 * h + i][0] = two_of(w, sv[i], At<0>());
            v[4 * h + i][1] = two_of(w, sv[i], At<1>());
            v[4 * h + i][2] = two_of(w, sv[i], At<2>());
            v[4 * h + i][3] = two_of(w, sv[i], At<3>());
          } else {
            const uint32_t w = half[h].v[i / 2];
            v[4 * h + i][0] = i % 2 == 0 ? two_of(w, sv[i], At<0>()) : two_of(w, sv[i], At<2>());
            v[4 * h + i][1] = i % 2 == 0 ? two_of(w, sv[i], At<1>()) : two_of(w, sv[i], At<3>());
          }
        }
      }
#pragma unroll
      for (int e = 0; e < kVB; ++e) {
        const int w = e / 2;
        const bf16x8_t bv = e % 2 == 0 ? as_bf16x8(pack_lo(v[0][w], v[1][w]), pack_lo(v[2][w], v[3][w]), pack_lo(v[4][w], v[5][w]), pack_lo(v[6][w], v[7][w]))
                                       : as_bf16x8(pack_hi(v[0][w], v[1][w]), pack_hi(v[2][w], v[3][w]), pack_hi(v[4][w], v[5][w]), pack_hi(v[6][w], v[7][w]));
        acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, bv, acc[e], 0, 0, 0);
        if constexpr (kThird) acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, bv, acc[e], 0, 0, 0);
      }
    };

    QuantHalf<D> buf[2][2];
    issue(0, buf[0]);
    for (int t0 = 0; t0 < n_tiles; t0 += 2) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        issue(t0 + u + 1, buf[(u + 1) % 2]);
        if (u == 0 || t0 + u < n_tiles) consume(buf[u]);  // uniform
      }
    }
  }

  l = rows_allreduce(l, OpSum());
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (4 * kg + i < kSlots) {
      float* dst = &sh.acc[wave][4 * kg + i][kt * kVB];
#pragma unroll
      for (int e = 0; e < kVB; e += 4)
        *reinterpret_cast<float4*>(dst + e) = make_float4(acc[e][i], acc[e + 1][i], acc[e + 2][i], acc[e + 3][i]);
    }
  }
  if (lane < G) { sh.m[wave][lane] = m; sh.l[wave][lane] = l; }
  __syncthreads();
  finish_chunk<T, D, G>(c, k, to, sh);
}

template <typename T, int D, int S, int G, bool kNT>
__global__ __launch_bounds__(kDecWaves* kWave, sizeof(T) == 4 ? 2 : 3) void quant_partial_kernel(CacheView c, QuantDecodeArgs a, SplitPlan plan) {
  __shared__ QuantShared<T, D, G> sh;
  int split, hkv, b;
  locate_chunk(c, plan, split, hkv, b);
  const int row = b * c.Hkv + hkv;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int begin = split * plan.pages_per_split;
  const int32_t* list = a.sel_pages ? a.sel_pages + (int64_t)row * a.sel_stride : nullptr;
  int first_lp = -1;  // requested together with the lengths
  {
    const int e = begin + wave + lane * kDecWaves;
    if (list && e < min(begin + plan.pages_per_split, a.sel_stride)) first_lp = list[e];
  }
  const int N = c.seq_lens[b];
  const int P = min((N + S - 1) / S, c.max_pages_hint);
  const int cnt = list ? min(a.sel_count[row], a.sel_stride) : P;
  const ChunkOut<T> to = {a.part_o, a.part_ml, reinterpret_cast<T*>(a.out), a.lse_out, plan.num_splits};
  if (begin >= cnt) {
    write_empty<T, D, G>(c, to, b, hkv);
    return;
  }
  const Chunk chunk = {hkv, b, begin, min(begin + plan.pages_per_split, cnt), N, (int64_t)row * plan.num_splits + split};
  auto lookup = [&](int e, bool first, int& phys, int& ntok) {
    const int lp = !list ? e : (first ? first_lp : list[e]);
    if (lp >= 0 && lp < P) {
      const int ph = c.page_table[(int64_t)b * c.max_pages + lp];
      if (ph >= 0 && (int64_t)ph < c.num_phys) {
        phys = ph;
        ntok = min(S, N - lp * S);
      }
    }
  };
  quant_chunk<D, S, G, kNT>(c, a.records, reinterpret_cast<const T*>(a.q), chunk, wave, lane, lookup, a.scale_log2, to, sh);
}

// Every page of sequences that are cut by their lengths.
template <typename T, int D, int S, int G, bool kNT>
__global__ __launch_bounds__(kDecWaves* kWave, sizeof(T) == 4 ? 2 : 3) void quant_dense_kernel(CacheView c, QuantDecodeArgs a, int max_chunks,
                                                                                                  DenseRound round) {
  __shared__ QuantShared<T, D, G> sh;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, w = blockIdx.x;
  BatchChunks bc;
  if (!cut_batch(c, S, max_chunks, w, bc, round)) return;
  const unsigned long long here = sequence_of(c, bc, w);
  if (here == 0) return;
  const Chunk chunk = chunk_of(c, bc, here, w);
  const ChunkOut<T> to = {a.part_o, a.part_ml, nullptr, nullptr, 2};
  auto lookup = [&](int e, bool, int& phys, int& ntok) {
    const int ph = c.page_table[(int64_t)chunk.b * c.max_pages + e];
    if (ph >= 0 && (int64_t)ph < c.num_phys) {
      phys = ph;
      ntok = min(S, chunk.N - e * S);
    }
  };
  quant_chunk<D, S, G, kNT>(c, a.records, reinterpret_cast<const T*>(a.q), chunk, wave, lane, lookup, a.scale_log2, to, sh);
}

template <typename T, int D, int G, int kWaves>
__global__ __launch_bounds__(kWaves* kWave) void quant_merge_kernel(CacheView c, QuantDecodeArgs a, int max_chunks, DenseRound round) {
  __shared__ MergeShared<kWaves, D> sh;
  merge_cut<T, D, G, kWaves>(c, blockIdx.y, blockIdx.x, max_chunks, round, a.part_o, a.part_ml, reinterpret_cast<T*>(a.out), a.lse_out, sh);
}

template <typename T, int D, int S, int G>
hipError_t launch_t(const CacheView& c, const QuantDecodeArgs& a, const SplitPlan& plan, bool stream_nt, hipStream_t st) {
  if (plan.num_splits == 0) {
    const int max_chunks = plan.pages_per_split;
    const DenseRound round = quant_batch(c).round();
    if (stream_nt) quant_dense_kernel<T, D, S, G, true><<<dim3(max_chunks), dim3(kDecWaves * kWave), 0, st>>>(c, a, max_chunks, round);
    else quant_dense_kernel<T, D, S, G, false><<<dim3(max_chunks), dim3(kDecWaves * kWave), 0, st>>>(c, a, max_chunks, round);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (dense_merge_alone(c.B * c.Hkv)) quant_merge_kernel<T, D, G, 1><<<dim3(c.H, c.B), dim3(kWave), 0, st>>>(c, a, max_chunks, round);
    else quant_merge_kernel<T, D, G, kMergeWaves><<<dim3(c.H, c.B), dim3(kMergeWaves * kWave), 0, st>>>(c, a, max_chunks, round);
    return hipGetLastError();
  }
  const dim3 grid = plan.rotate ? dim3(c.Hkv, c.B, plan.num_splits) : dim3(plan.num_splits, c.Hkv, c.B);
  if (stream_nt) quant_partial_kernel<T, D, S, G, true><<<grid, dim3(kDecWaves * kWave), 0, st>>>(c, a, plan);
  else quant_partial_kernel<T, D, S, G, false><<<grid, dim3(kDecWaves * kWave), 0, st>>>(c, a, plan);
  return hipGetLastError();
}

template <typename T, int D, int S>
hipError_t dispatch_g(const CacheView& c, const QuantDecodeArgs& a, const SplitPlan& plan, bool stream_nt, hipStream_t st) {
  switch (c.H / c.Hkv) {
    case 1: return launch_t<T, D, S, 1>(c, a, plan, stream_nt, st);
    case 2: return launch_t<T, D, S, 2>(c, a, plan, stream_nt, st);
    case 4: return launch_t<T, D, S, 4>(c, a, plan, stream_nt, st);
    case 8: return launch_t<T, D, S, 8>(c, a, plan, stream_nt, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

// One translation unit per element type and head dimension: UNIQUE_ELEM, UNIQUE_DIM.
template <>
hipError_t launch_quant_partial<UNIQUE_ELEM, UNIQUE_DIM>(const CacheView& c, const QuantDecodeArgs& a, const SplitPlan& plan, bool stream_nt,
                                                         hipStream_t stream) {
  switch (c.S) {
    case 8: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 8>(c, a, plan, stream_nt, stream);
    case 16: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 16>(c, a, plan, stream_nt, stream);
    case 32: return dispatch_g<UNIQUE_ELEM, UNIQUE_DIM, 32>(c, a, plan, stream_nt, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace unique
