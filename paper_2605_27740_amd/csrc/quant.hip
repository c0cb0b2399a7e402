// Tokens of the cache to 4-bit records and back.
//
// Number format: blocks of 32 channels of a token share a scale 2^e, e = clamp(floor(log2 max|x|) - 2, -126, 125), stored as the byte
// e + 127; a channel is the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} to x / 2^e, ties to the even code, so that what lies
// above 6 (up to 8) becomes 6. A block with an infinity or a NaN gets the byte 255, which stands for NaN. The conversion instructions round so
// and take the scale's exponent bits alone, with 255 as NaN and 0 as 2^-127 (checked lane by lane), so that a byte shifted into
// place is a scale.
//
// A wave takes a (page, KV head): a lane eight channels of a token, a load instruction 512 channels of consecutive tokens.
#include <type_traits>

#include "device_utils.hpp"
#include "quant.hpp"

namespace unique {
namespace {

constexpr int kQuantWaves = 4;

__device__ __forceinline__ void load_eight(const bf16_t* p, float (&x)[8]) { load_vec(p, x); }
__device__ __forceinline__ void load_eight(const float* p, float (&x)[8]) {
  float a[4], b[4];
  load_vec(p, a);
  load_vec(p + 4, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}
__device__ __forceinline__ void store_eight(bf16_t* p, const float (&x)[8]) {  // every value is a bf16 number
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xffff0000u);
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_eight(float* p, const float (&x)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

// The scale byte of a block whose lanes (four neighbours) hold eight channels each; the same in all four.
__device__ __forceinline__ uint32_t block_scale(const float (&x)[8]) {
  float top = 0.f;
  uint32_t odd = 0;  // an infinity or NaN here
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    top = fmaxf(top, fabsf(x[i]));
    odd |= (__float_as_uint(x[i]) & 0x7f800000u) == 0x7f800000u;
  }
  top = odd ? INFINITY : top;
  top = group_allreduce<4>(top, OpMax());
  const int exponent = (int)(__float_as_uint(top) >> 23);  // of 2^e times four
  return exponent == 255 ? 255u : (uint32_t)max(exponent - 2, 1);
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

__device__ __forceinline__ uint32_t encode_eight(const float (&x)[8], float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  return w;
}
__device__ __forceinline__ void decode_eight(uint32_t w, float scale, float (&x)[8]) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  const f32x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y; x[4] = c.x; x[5] = c.y; x[6] = d.x; x[7] = d.y;
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

template <typename T, int D, int S>
__global__ __launch_bounds__(kQuantWaves* kWave) void quantise_kernel(CacheView c, QuantPool pool, const int32_t* tok_begin,
                                                                      const int32_t* tok_end, int pages_per_seq) {
  constexpr QuantTile kTile = {S, D};
  constexpr int kLanes = D / 8, kTok = kWave / kLanes;  // lanes of a token, tokens of a load
  QuantItem it;
  if (!quant_item<D, S>(c, pool, tok_begin, tok_end, pages_per_seq, it)) return;
  const int lane = threadIdx.x % kWave, oct = lane % kLanes;
  const T* kc = reinterpret_cast<const T*>(c.k_cache) + it.full;
  const T* vc = reinterpret_cast<const T*>(c.v_cache) + it.full;
  for (int tok = it.t0 / kTok * kTok + lane / kLanes; tok < S; tok += kTok) {
    if (tok >= it.t0 && tok < it.t1) {  // lanes of a block agree
      float x[8], y[8];
      load_eight(kc + tok * D + oct * 8, x);
      load_eight(vc + tok * D + oct * 8, y);
      const uint32_t ks = block_scale(x), vs = block_scale(y);
      *reinterpret_cast<uint32_t*>(it.tile + kTile.k_codes() + tok * (D / 2) + oct * 4) = encode_eight(x, scale_of(ks));
      const uint32_t v = encode_eight(y, scale_of(vs));
      if constexpr (D == 128) {
        *reinterpret_cast<uint32_t*>(it.tile + kTile.v_at(tok, oct)) = v;
      } else {
        *reinterpret_cast<uint16_t*>(it.tile + kTile.v_at(tok, 2 * oct)) = (uint16_t)v;
        *reinterpret_cast<uint16_t*>(it.tile + kTile.v_at(tok, 2 * oct + 1)) = (uint16_t)(v >> 16);
      }
      if (oct % 4 == 0) {
        it.tile[kTile.k_scales() + oct / 4 * S + tok] = (char)ks;
        it.tile[kTile.v_scales() + oct / 4 * S + tok] = (char)vs;
      }
    }
  }
}

template <typename T, int D, int S>
__global__ __launch_bounds__(kQuantWaves* kWave) void restore_kernel(CacheView c, QuantPool pool, T* k_out, T* v_out, const int32_t* tok_begin,
                                                                     const int32_t* tok_end, int pages_per_seq) {
  constexpr QuantTile kTile = {S, D};
  constexpr int kLanes = D / 8, kTok = kWave / kLanes;
  QuantItem it;
  if (!quant_item<D, S>(c, pool, tok_begin, tok_end, pages_per_seq, it)) return;
  const int lane = threadIdx.x % kWave, oct = lane % kLanes;
  for (int tok = it.t0 / kTok * kTok + lane / kLanes; tok < S; tok += kTok) {
    if (tok >= it.t0 && tok < it.t1) {
      const uint32_t kw = *reinterpret_cast<const uint32_t*>(it.tile + kTile.k_codes() + tok * (D / 2) + oct * 4);
      uint32_t vw;
      if constexpr (D == 128) {
        vw = *reinterpret_cast<const uint32_t*>(it.tile + kTile.v_at(tok, oct));
      } else {
        vw = *reinterpret_cast<const uint16_t*>(it.tile + kTile.v_at(tok, 2 * oct)) |
             ((uint32_t)*reinterpret_cast<const uint16_t*>(it.tile + kTile.v_at(tok, 2 * oct + 1)) << 16);
      }
      const uint32_t ks = (uint8_t)it.tile[kTile.k_scales() + oct / 4 * S + tok], vs = (uint8_t)it.tile[kTile.v_scales() + oct / 4 * S + tok];
      float x[8], y[8];
      decode_eight(kw, scale_of(ks), x);
      decode_eight(vw, scale_of(vs), y);
      store_eight(k_out + it.full + tok * D + oct * 8, x);
      store_eight(v_out + it.full + tok * D + oct * 8, y);
    }
  }
}

template <typename Launch>
hipError_t with_shape(const CacheView& c, Launch launch) {
  auto page = [&](auto elem, auto dim) {
    switch (c.S) {
      case 8: launch(elem, dim, std::integral_constant<int, 8>()); break;
      case 16: launch(elem, dim, std::integral_constant<int, 16>()); break;
      case 32: launch(elem, dim, std::integral_constant<int, 32>()); break;
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
  return with_shape(c, [&](auto elem, auto dim, auto page) {
    quantise_kernel<decltype(elem), decltype(dim)::value, decltype(page)::value>
        <<<item_grid(c, n), dim3(kQuantWaves * kWave), 0, stream>>>(c, pool, d_tok_begin, d_tok_end, n);
  });
}

hipError_t launch_restore(const CacheView& c, const QuantPool& pool, void* k_out, void* v_out, const int32_t* d_tok_begin,
                          const int32_t* d_tok_end, int max_pages_touched, hipStream_t stream) {
  const int n = d_tok_begin ? max_pages_touched : c.max_pages_hint;
  if (n <= 0) return hipSuccess;
  return with_shape(c, [&](auto elem, auto dim, auto page) {
    using T = decltype(elem);
    restore_kernel<T, decltype(dim)::value, decltype(page)::value><<<item_grid(c, n), dim3(kQuantWaves * kWave), 0, stream>>>(
        c, pool, reinterpret_cast<T*>(k_out), reinterpret_cast<T*>(v_out), d_tok_begin, d_tok_end, n);
  });
}

hipError_t launch_quant_decode(const CacheView& c, const void* records, const void* d_q, const int32_t* d_sel_pages, const int32_t* d_sel_count,
                               int sel_stride, int max_list_len, float sm_scale, void* d_out, float* d_lse_out, float* d_partials,
                               hipStream_t stream) {
  const int rows = c.B * c.Hkv, page_bytes = QuantTile{c.S, c.D}.bytes();
  SplitPlan plan = d_sel_pages ? plan_splits(c.B, c.Hkv, max_list_len, c.max_pages_hint, page_bytes, false) : most_splits(rows, max_list_len);
  size_t slots = (size_t)rows * plan.num_splits;
  if (!d_sel_pages && dense_balances(c.B, c.Hkv, max_list_len, page_bytes, kQuantLeastBytes)) {
    plan = SplitPlan{dense_max_chunks(rows, max_list_len, kQuantRound), 0, 0};
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
