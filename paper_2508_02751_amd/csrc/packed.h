// Packed caches: rows of 8- or 4-bit codes, with a power of two for every 32 elements.
//
// An element is (-1)^s * 2^(e - bias) * (1 + m / 2^M), or, with e = 0, the same without
// the leading 1 and with e = 1: 4 exponent and 3 mantissa bits (bias 7, all ones but for
// the sign: NaN) or 2 and 1 (bias 1); a scale byte x is 2^(x - 127), 255 NaN.  The
// products have at most 4 significant bits, so bf16 and fp32 hold them exactly, and the
// conversions below, one instruction for two elements, round nothing.
#pragma once

#include "cache.h"

namespace smallkv {

// fp32 queries over rows that bf16 holds exactly (a packed cache's): both products run on bf16
// operands, the queries and the probabilities in three bf16 parts each, which together hold
// what fp32 holds.
struct wide_t {
  float x;
};
template <> struct elem<wide_t> : elem<float> {};
template <int D> struct TileLayout<wide_t, D> : TileLayout<bf16_t, D> {};

constexpr int kBlock = 32;  // elements that share a scale

// The scales of one layer: a row has head_dim / 32 bytes.  Strides in rows' scales.
struct ScaleView {
  const uint8_t *k, *v;
  uint32_t page_stride, head_stride, row_stride;
};

// Host: the codes as a cache whose strides are in elements of the model's dtype, and the
// scales (both of checked descriptors).
inline smallkv_cache_t codes_of(const smallkv_packed_t &p) {
  const int64_t per16 = p.dtype == SMALLKV_F32 ? 4 : 8;
  smallkv_cache_t c{};
  c.k = p.k;
  c.v = p.v;
  c.dtype = p.dtype;
  c.head_dim = p.head_dim;
  c.n_heads = p.n_heads;
  c.page_rows = p.page_rows;
  c.n_pages = p.n_pages;
  c.table_width = p.table_width;
  c.page_stride = p.page_stride / 16 * per16;
  c.head_stride = p.head_stride / 16 * per16;
  c.row_stride = p.row_stride / 16 * per16;
  c.page_table = p.page_table;
  return c;
}
inline ScaleView scale_view(const smallkv_packed_t &p) {
  const int64_t w = p.head_dim / kBlock;
  return ScaleView{p.k_scale, p.v_scale, (uint32_t)(p.scale_page_stride / w), (uint32_t)(p.scale_head_stride / w),
                   (uint32_t)(p.scale_row_stride / w)};
}
inline int format_bits(const smallkv_packed_t &p) { return p.format == SMALLKV_MXFP8 ? 8 : 4; }

// Byte offset of the scales of a row on a page that exists.
template <int D>
__device__ __forceinline__ int64_t scale_offset(const ScaleView &s, const CacheView &c, int page, int row, int head) {
  const uint32_t in = (uint32_t)row & (c.table ? (1u << c.shift) - 1 : ~0u);
  return (int64_t)(((uint64_t)(uint32_t)page * s.page_stride + (uint64_t)in * s.row_stride +
                    (uint64_t)head * s.head_stride) * (D / kBlock));
}

// The scale as the conversions take it: a float of which they use the exponent bits.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// 16 bytes of T (8 bf16 or 4 fp32 elements): elements i * 16 / sizeof(T) on of the codes w.
template <typename T, int F> __device__ __forceinline__ uint4 unpack16(const uint32_t *w, int i, float scale) {
  if constexpr (sizeof(T) == 2 && F == 8) {
    const uint32_t x = w[2 * i], y = w[2 * i + 1];
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, scale, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, scale, true)));
  } else if constexpr (sizeof(T) == 2) {
    const uint32_t x = w[i];
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3)));
  } else {
    f32x2_t a, b;
    if constexpr (F == 8) {
      a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, false);
      b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, true);
    } else {
      const uint32_t x = w[i / 2] >> (i % 2 * 16);
      a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, scale, 0);
      b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, scale, 1);
    }
    return make_uint4(__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1]));
  }
}

// Half of a packed row, its first or last head_dim / 2 elements: codes and scales as they
// are in memory, and as pieces of 16 bytes of T.
template <int D, int F> struct HalfRow {
  static constexpr int kWords = D * F / 64;
  uint32_t w[kWords], scales;  // (the first block's scale in the low byte)
  __device__ __forceinline__ void load(const unsigned char *row, const uint8_t *s, int half) {
#pragma unroll
    for (int i = 0; i < kWords; i += 4) {
      const uint4 x = reinterpret_cast<const uint4 *>(row)[half * (kWords / 4) + i / 4];
      w[i] = x.x;
      w[i + 1] = x.y;
      w[i + 2] = x.z;
      w[i + 3] = x.w;
    }
    if constexpr (D == 128)
      scales = reinterpret_cast<const uint16_t *>(s)[half];
    else
      scales = s[half];
  }
  template <typename T> __device__ __forceinline__ uint4 get(int i) const {
    constexpr int per = kBlock * (int)sizeof(T) / 16;  // pieces of a block
    return unpack16<T, F>(w, i, scale_of(D == 128 ? scales >> (i / per * 8) & 255u : scales));
  }
};

// Element e of a row: of T, or of codes of F bits and their scales.
template <typename T, int F> __device__ __forceinline__ float cached(const unsigned char *row, const uint8_t *scales, int e) {
  if constexpr (F == 0) {
    return elem<T>::load1(row, e);
  } else {
    const float s = scale_of(scales[e / kBlock]);
    if constexpr (F == 8) return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((uint32_t)row[e], s, false)[0];
    return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)row[e / 2] >> (e % 2 * 4), s, 0)[0];
  }
}

}  // namespace smallkv
