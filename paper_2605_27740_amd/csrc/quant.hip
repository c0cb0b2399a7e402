// Tokens of the cache to 4-bit records and back.
//
// Number format: blocks of 32 channels of a token share a scale 2^e, e = clamp(floor(log2 max|x|) - 2, -126, 125), stored as the byte
// e + 127; a channel is the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} to x / 2^e, ties to the even code, so that what lies
// above 6 (up to 8) becomes 6. A block with an infinity or a NaN gets the byte 255, which stands for NaN. The conversion instructions round so
// and take the scale's exponent bits alone, with 255 as NaN and 0 as 2^-127 (checked lane by lane), so that a byte shifted into
// place is a scale.
//
// A wave takes a (page, KV head): a lane 16 bytes of channels of a few consecutive tokens, whose V codes are consecutive bytes of the record
// (16 of four tokens, D = 128), as are their scales; a load or store of full-precision channels covers whole rows.
#include <type_traits>

#include "device_utils.hpp"
#include "quant.hpp"

namespace unique {
namespace {

constexpr int kQuantWaves = 4;

// kNT: what is read or written in full precision bypasses the caches, of a launch that moves more than they keep (bf16, 8 KV heads, D = 128: 32768 tokens
// restored in 37.2 / 28.3 us, 80000 quantised and restored in 180 / 139). It needs accesses that cover whole lines: with two of 16 bytes for eight fp32
// channels of a lane it took 126 us where plain ones took 79.
template <bool kNT, typename V>
__device__ __forceinline__ V load_as(const void* p) {
  if constexpr (kNT) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else return *reinterpret_cast<const V*>(p);
}
template <bool kNT, typename V>
__device__ __forceinline__ void store_as(void* p, V v) {
  if constexpr (kNT) __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
  else *reinterpret_cast<V*>(p) = v;
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// 16 bytes of channels, eight of bf16 or four of fp32: their largest exponent field, their codes, and the way back. Magnitudes are
// compared as whole numbers, which puts infinity and NaN on top.
__device__ __forceinline__ int top_exponent(u32x4_t x, const bf16_t*) {
  typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
  u16x2_t m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = __builtin_bit_cast(u16x2_t, x[i] & 0x7fff7fffu);
  const u16x2_t top = __builtin_elementwise_max(__builtin_elementwise_max(m[0], m[1]), __builtin_elementwise_max(m[2], m[3]));
  return max(top.x, top.y) >> 7;
}
__device__ __forceinline__ int top_exponent(u32x4_t x, const float*) {
  const u32x4_t m = x & 0x7fffffffu;
  return (int)(max(max(m.x, m.y), max(m.z, m.w)) >> 23);
}
__device__ __forceinline__ uint32_t encode(u32x4_t x, float scale, const bf16_t*) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, (uint32_t)x.x), scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, (uint32_t)x.y), scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, (uint32_t)x.z), scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, (uint32_t)x.w), scale, 3);
  return w;
}
__device__ __forceinline__ uint32_t encode(u32x4_t x, float scale, const float*) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x.x), __uint_as_float(x.y), scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x.z), __uint_as_float(x.w), scale, 1);
  return w;
}
__device__ __forceinline__ u32x4_t decode(uint32_t w, float scale, const bf16_t*) {
  u32x4_t x;
  x.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  x.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  x.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  x.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return x;
}
__device__ __forceinline__ u32x4_t decode(uint32_t w, float scale, const float*) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  return u32x4_t{__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y)};
}

// kBytes bytes as one access.
template <int kBytes>
struct Bytes;
template <> struct Bytes<1> { using type = uint8_t; };
template <> struct Bytes<2> { using type = uint16_t; };
template <> struct Bytes<4> { using type = uint32_t; };
template <> struct Bytes<8> { using type = uint64_t; };
template <> struct Bytes<16> { using type = u32x4_t; };

// How a wave goes over a page's tokens: kRun consecutive ones per lane, kStep at a time.
template <typename T, int D, int S>
struct QuantShape {
  static constexpr int kVec = Elem<T>::kVec, kLanes = D / kVec, kRows = kWave / kLanes;  // channels of a lane, lanes of a token
  static constexpr int kRun = S / kRows < 4 ? S / kRows : 4, kStep = kRun * kRows;
  static constexpr int kBlock = kQuantBlock / kVec;     // lanes of a scale
  static constexpr int kUnit = D / 16;                  // channels of a V unit: half of a lane's, all, or twice as many
  static constexpr int kUnits = kVec > kUnit ? kVec / kUnit : 1;
  static constexpr bool kShared = kVec < kUnit;         // two lanes to a unit
  using Code = typename Bytes<kVec / 2>::type;          // of a lane and token
  using Scales = typename Bytes<kRun>::type;            // of a lane's tokens
  using Unit = typename Bytes<kUnit / 2>::type;         // of a token
  using Units = typename Bytes<kUnit / 2 * kRun>::type; // of a lane's tokens
};

// The scale byte of a block whose kBlock neighbouring lanes hold 16 bytes of channels each; the same in all of them.
template <int kBlock, typename T>
__device__ __forceinline__ uint32_t block_scale(u32x4_t x) {
  int e = top_exponent(x, (const T*)nullptr);  // of 2^e times four
  e = max(e, __builtin_amdgcn_update_dpp(0, e, kDppXor1, 0xf, 0xf, true));
  e = max(e, __builtin_amdgcn_update_dpp(0, e, kDppXor2, 0xf, 0xf, true));
  if constexpr (kBlock == 8) e = max(e, __builtin_amdgcn_update_dpp(0, e, kDppHalfMirror, 0xf, 0xf, true));
  return e == 255 ? 255u : (uint32_t)max(e - 2, 1);
}

// The (page, head) of a wave and the tokens of it that count; false: nothing to do.
struct QuantItem {
  int64_t full;    // element offset of the (page, head) in the cache
  char* tile;      // its part of the record
  int t0, t1;      // slots of the page
};
template <int D, int S>
__device__ __forceinline__ bool quant_item(const CacheView& c, const QuantPool& pool, const int32_t* tok_begin, const int32_t* tok_end,
                                           int pages_per_seq, QuantItem& it) {
  const int b = blockIdx.y;
  const int w = __builtin_amdgcn_readfirstlane(blockIdx.x * kQuantWaves + threadIdx.x / kWave);
  const int hkv = w & (c.Hkv - 1), po = w >> (__ffs(c.Hkv) - 1);
  if (po >= pages_per_seq) return false;
  const int N = c.seq_lens[b];
  const int t0 = tok_begin ? max(tok_begin[b], 0) : 0, t1 = tok_begin ? min(tok_end[b], N) : N;
  if (t0 >= t1) return false;
  const int p = t0 / S + po;
  if (p >= c.max_pages_hint || (int64_t)p * S >= t1) return false;
  const int from = c.page_table[(int64_t)b * c.max_pages + p], to = pool.table[(int64_t)b * c.max_pages + p];
  if (from < 0 || (int64_t)from >= c.num_phys || to < 0 || (int64_t)to >= pool.num) return false;
  it.full = (int64_t)from * c.kv_page_stride + (int64_t)hkv * c.kv_head_stride;
  it.tile = pool.records + ((int64_t)to * c.Hkv + hkv) * QuantTile{S, D}.bytes();
  it.t0 = max(t0 - p * S, 0);
  it.t1 = min(t1 - p * S, S);
  return true;
}

template <typename T, int D, int S, bool kNT>
__global__ __launch_bounds__(kQuantWaves* kWave) void quantise_kernel(CacheView c, QuantPool pool, const int32_t* tok_begin,
                                                                      const int32_t* tok_end, int pages_per_seq) {
  using Sh = QuantShape<T, D, S>;
  constexpr QuantTile kTile = {S, D};
  constexpr int kRun = Sh::kRun, kVec = Sh::kVec;
  QuantItem it;
  if (!quant_item<D, S>(c, pool, tok_begin, tok_end, pages_per_seq, it)) return;
  const int lane = threadIdx.x % kWave, ch = lane % Sh::kLanes;
  const T* kc = reinterpret_cast<const T*>(c.k_cache) + it.full + ch * kVec;
  const T* vc = reinterpret_cast<const T*>(c.v_cache) + it.full + ch * kVec;
  char* codes = it.tile + kTile.k_codes() + ch * (kVec / 2);
  const bool first_of_block = ch % Sh::kBlock == 0, writes_unit = !Sh::kShared || ch % 2 == 0;
  const int unit = ch * kVec / Sh::kUnit;
  for (int first = it.t0 / Sh::kStep * Sh::kStep; first < it.t1; first += Sh::kStep) {
    const int tok0 = first + lane / Sh::kLanes * kRun;
    u32x4_t x[kRun], y[kRun];  // requested together; a slot that does not count reads one that does
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      const int tok = max(it.t0, min(tok0 + j, it.t1 - 1));
      x[j] = load_as<kNT, u32x4_t>(kc + tok * D);
      y[j] = load_as<kNT, u32x4_t>(vc + tok * D);
    }
    typename Sh::Scales ks = 0, vs = 0;
    uint32_t k[kRun], v[kRun];
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      const uint32_t a = block_scale<Sh::kBlock, T>(x[j]), b = block_scale<Sh::kBlock, T>(y[j]);
      k[j] = encode(x[j], scale_of(a), (const T*)nullptr);
      v[j] = encode(y[j], scale_of(b), (const T*)nullptr);
      if constexpr (Sh::kShared) v[j] |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v[j], kDppXor1, 0xf, 0xf, true) << 16;
      ks |= a << (8 * j);
      vs |= b << (8 * j);
    }
    char* k_scale = it.tile + kTile.k_scales() + ch / Sh::kBlock * S + tok0;
    char* v_scale = it.tile + kTile.v_scales() + ch / Sh::kBlock * S + tok0;
    if (tok0 >= it.t0 && tok0 + kRun <= it.t1) {
#pragma unroll
      for (int j = 0; j < kRun; ++j) *reinterpret_cast<typename Sh::Code*>(codes + (tok0 + j) * (D / 2)) = (typename Sh::Code)k[j];
      if (writes_unit) {
#pragma unroll
        for (int u = 0; u < Sh::kUnits; ++u) {
          typename Sh::Units w;
          if constexpr (sizeof(w) == 16) {
            w = u32x4_t{v[0], v[1], v[2], v[3]};
          } else {
            w = 0;
#pragma unroll
            for (int j = 0; j < kRun; ++j)
              w |= (typename Sh::Units)(typename Sh::Unit)(v[j] >> (16 * u)) << (8 * (int)sizeof(typename Sh::Unit) * j);
          }
          *reinterpret_cast<typename Sh::Units*>(it.tile + kTile.v_at(tok0, unit + u)) = w;
        }
      }
      if (first_of_block) {
        *reinterpret_cast<typename Sh::Scales*>(k_scale) = ks;
        *reinterpret_cast<typename Sh::Scales*>(v_scale) = vs;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kRun; ++j) {
        const int tok = tok0 + j;
        if (tok < it.t0 || tok >= it.t1) continue;
        *reinterpret_cast<typename Sh::Code*>(codes + tok * (D / 2)) = (typename Sh::Code)k[j];
        if (writes_unit) {
#pragma unroll
          for (int u = 0; u < Sh::kUnits; ++u)
            *reinterpret_cast<typename Sh::Unit*>(it.tile + kTile.v_at(tok, unit + u)) = (typename Sh::Unit)(v[j] >> (16 * u));
        }
        if (first_of_block) {
          k_scale[j] = (char)(ks >> (8 * j));
          v_scale[j] = (char)(vs >> (8 * j));
        }
      }
    }
  }
}

template <typename T, int D, int S, bool kNT>
__global__ __launch_bounds__(kQuantWaves* kWave) void restore_kernel(CacheView c, QuantPool pool, T* k_out, T* v_out, const int32_t* tok_begin,
                                                                     const int32_t* tok_end, int pages_per_seq) {
  using Sh = QuantShape<T, D, S>;
  constexpr QuantTile kTile = {S, D};
  constexpr int kRun = Sh::kRun, kVec = Sh::kVec;
  QuantItem it;
  if (!quant_item<D, S>(c, pool, tok_begin, tok_end, pages_per_seq, it)) return;
  const int lane = threadIdx.x % kWave, ch = lane % Sh::kLanes, unit = ch * kVec / Sh::kUnit;
  for (int first = it.t0 / Sh::kStep * Sh::kStep; first < it.t1; first += Sh::kStep) {
    const int tok0 = first + lane / Sh::kLanes * kRun;
    uint32_t k[kRun], v[kRun];
#pragma unroll
    for (int j = 0; j < kRun; ++j)
      k[j] = *reinterpret_cast<const typename Sh::Code*>(it.tile + kTile.k_codes() + (tok0 + j) * (D / 2) + ch * (kVec / 2));
    typename Sh::Units w[Sh::kUnits];
#pragma unroll
    for (int u = 0; u < Sh::kUnits; ++u) w[u] = *reinterpret_cast<const typename Sh::Units*>(it.tile + kTile.v_at(tok0, unit + u));
    const uint32_t ks = *reinterpret_cast<const typename Sh::Scales*>(it.tile + kTile.k_scales() + ch / Sh::kBlock * S + tok0);
    const uint32_t vs = *reinterpret_cast<const typename Sh::Scales*>(it.tile + kTile.v_scales() + ch / Sh::kBlock * S + tok0);
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      v[j] = 0;
#pragma unroll
      for (int u = 0; u < Sh::kUnits; ++u) {
        uint32_t of_unit;
        if constexpr (sizeof(typename Sh::Units) == 16) of_unit = w[u][j];
        else of_unit = (typename Sh::Unit)(w[u] >> (8 * (int)sizeof(typename Sh::Unit) * j));
        v[j] |= of_unit << (16 * u);
      }
      if constexpr (Sh::kShared) v[j] >>= 16 * (ch % 2);
    }
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      const int tok = tok0 + j;
      if (tok < it.t0 || tok >= it.t1) continue;
      store_as<kNT>(k_out + it.full + tok * D + ch * kVec, decode(k[j], scale_of(ks >> (8 * j) & 255u), (const T*)nullptr));
      store_as<kNT>(v_out + it.full + tok * D + ch * kVec, decode(v[j], scale_of(vs >> (8 * j) & 255u), (const T*)nullptr));
    }
  }
}

template <typename Launch>
hipError_t with_shape(const CacheView& c, int pages_per_seq, Launch launch) {
  const bool nt = (int64_t)c.B * pages_per_seq * c.Hkv * c.S * c.D * 2 * (c.dtype == 0 ? 4 : 2) > kStreamNtBytes;
  auto streamed = [&](auto elem, auto dim, auto page) {
    if (nt) launch(elem, dim, page, std::true_type());
    else launch(elem, dim, page, std::false_type());
  };
  auto page = [&](auto elem, auto dim) {
    switch (c.S) {
      case 8: streamed(elem, dim, std::integral_constant<int, 8>()); break;
      case 16: streamed(elem, dim, std::integral_constant<int, 16>()); break;
      case 32: streamed(elem, dim, std::integral_constant<int, 32>()); break;
      default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
  };
  auto dim = [&](auto elem) {
    return c.D == 64 ? page(elem, std::integral_constant<int, 64>()) : page(elem, std::integral_constant<int, 128>());
  };
  return c.dtype == 0 ? dim(float()) : dim(bf16_t());
}

dim3 item_grid(const CacheView& c, int pages_per_seq) {
  return dim3((unsigned)(((int64_t)pages_per_seq * c.Hkv + kQuantWaves - 1) / kQuantWaves), c.B);
}

}  // namespace

hipError_t launch_quantise(const CacheView& c, const QuantPool& pool, const int32_t* d_tok_begin, const int32_t* d_tok_end,
                           int max_pages_touched, hipStream_t stream) {
  const int n = d_tok_begin ? max_pages_touched : c.max_pages_hint;
  if (n <= 0) return hipSuccess;
  return with_shape(c, n, [&](auto elem, auto dim, auto page, auto nt) {
    quantise_kernel<decltype(elem), decltype(dim)::value, decltype(page)::value, decltype(nt)::value>
        <<<item_grid(c, n), dim3(kQuantWaves * kWave), 0, stream>>>(c, pool, d_tok_begin, d_tok_end, n);
  });
}

hipError_t launch_restore(const CacheView& c, const QuantPool& pool, void* k_out, void* v_out, const int32_t* d_tok_begin,
                          const int32_t* d_tok_end, int max_pages_touched, hipStream_t stream) {
  const int n = d_tok_begin ? max_pages_touched : c.max_pages_hint;
  if (n <= 0) return hipSuccess;
  return with_shape(c, n, [&](auto elem, auto dim, auto page, auto nt) {
    using T = decltype(elem);
    restore_kernel<T, decltype(dim)::value, decltype(page)::value, decltype(nt)::value><<<item_grid(c, n), dim3(kQuantWaves * kWave), 0, stream>>>(
        c, pool, reinterpret_cast<T*>(k_out), reinterpret_cast<T*>(v_out), d_tok_begin, d_tok_end, n);
  });
}

size_t quant_cut_floats(const CacheView& c) {
  const QuantBatch batch = quant_batch(c);
  return batch.balances() ? (size_t)batch.max_chunks() * (c.H / c.Hkv) * (c.D + 2) : 0;
}

hipError_t launch_quant_decode(const CacheView& c, const void* records, const void* d_q, const int32_t* d_sel_pages, const int32_t* d_sel_count,
                               int sel_stride, int max_list_len, float sm_scale, void* d_out, float* d_lse_out, float* d_partials,
                               size_t partial_floats, hipStream_t stream) {
  // Lists, and every page of sequences that are not cut by their lengths, by the rule for lists as if a page had 2 S D bytes, twice its own: latency and
  // arithmetic are what bounds a short list. us as if it had those of a bf16 page / so / with its own: every page of 1 x 500 tokens 8.3 / 6.2 /
  // 6.3, 2 x 600, eight heads 9.4 / 8.0 / 7.6, the toy model of 2048 tokens 9.0 / 8.9 / 11.5, 4 x 1500 9.6 / 10.0 / 11.2; lists of 16 x 8 rows x 256 18.8 /
  // 18.4 / 18.1, 12 x 8 x 200, eight heads 16.1 / 16.2 / 16.9. (Every page as for full-precision caches, most_splits: 1 x 113 tokens 9.9 / 7.2 so.)
  const int rows = c.B * c.Hkv, page_bytes = QuantTile{c.S, c.D}.bytes();
  SplitPlan plan = plan_splits(c.B, c.Hkv, max_list_len, c.max_pages_hint, c.S * c.D * 2, false);
  size_t slots = (size_t)rows * plan.num_splits;
  const size_t cut_floats = d_sel_pages ? 0 : quant_cut_floats(c);
  if (cut_floats > 0 && partial_floats >= cut_floats) {
    plan = SplitPlan{quant_batch(c).max_chunks(), 0, 0};
    slots = plan.pages_per_split;
  }
  const bool nt = (int64_t)rows * max_list_len * page_bytes > kStreamNtBytes;
  const QuantDecodeArgs a = {reinterpret_cast<const char*>(records), d_q, d_sel_pages, d_sel_count, sel_stride, decode_scale_log2(c, sm_scale),
                             d_partials, d_partials + slots * (c.H / c.Hkv) * c.D, d_out, d_lse_out};
  auto run = [&](auto launch) { return launch(c, a, plan, nt, stream); };
  const hipError_t e = c.dtype == 0 ? (c.D == 64 ? run(launch_quant_partial<float, 64>) : run(launch_quant_partial<float, 128>))
                                    : (c.D == 64 ? run(launch_quant_partial<bf16_t, 64>) : run(launch_quant_partial<bf16_t, 128>));
  if (e != hipSuccess || plan.num_splits <= 1) return e;
  return launch_merge(c, d_sel_pages ? d_sel_count : nullptr, sel_stride, plan, d_partials, d_out, d_lse_out, stream);
}

}  // namespace unique
