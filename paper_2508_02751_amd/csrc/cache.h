// Device views shared by the cache operators: rows of a paged or dense cache,
// the new tokens of a batch, and 16-byte copies from memory straight to LDS.
#pragma once

#include "common.h"

namespace smallkv {

// Rows of one layer's keys and values.  Strides are in units of 16 bytes (the
// host checks that they are whole units below 2^32); `shift` is log2 of the
// rows per page (31 without a table: sequence b is page b).
struct CacheView {
  const unsigned char *k, *v;
  uint32_t page_stride, head_stride, row_stride;
  int32_t n_pages, width, shift, cap;  // cap: rows a sequence can have
  const int32_t *table;
};

// The sequences' new tokens: packed rows start[b] .. start[b+1]-1 are the last
// tokens of sequence b's len[b] cached rows.
struct ChunkView {
  int32_t batch, n_tokens, max_new, max_len;
  const int32_t *start, *len;
};

// Host: the device views of checked descriptors.
inline CacheView cache_view(const smallkv_cache_t &c) {
  const int per16 = c.dtype == SMALLKV_F32 ? 4 : 8;
  CacheView v{};
  v.k = static_cast<const unsigned char *>(c.k);
  v.v = static_cast<const unsigned char *>(c.v);
  v.page_stride = (uint32_t)(c.page_stride / per16);
  v.head_stride = (uint32_t)(c.head_stride / per16);
  v.row_stride = (uint32_t)(c.row_stride / per16);
  v.n_pages = c.n_pages;
  v.table = c.page_table;
  v.width = c.table_width;
  v.shift = 31;
  v.cap = c.page_rows;
  if (c.page_table) {
    v.shift = 0;
    while ((1 << v.shift) < c.page_rows) ++v.shift;
    v.cap = (int32_t)((int64_t)c.page_rows * c.table_width);
  }
  return v;
}
inline ChunkView chunk_view(const smallkv_chunk_t &c) {
  return ChunkView{c.batch, c.n_tokens, c.max_new, c.max_len, c.start, c.len};
}

struct Seq {
  int first, n_new, len;  // first packed row, new tokens, cached rows
};

// Values in device memory are clamped, so that no access leaves its buffer.
__device__ __forceinline__ Seq sequence(const ChunkView &c, int b, int cap) {
  Seq s;
  s.first = clampi(c.start[b], 0, c.n_tokens);
  const int end = clampi(c.start[b + 1], s.first, c.n_tokens);
  s.n_new = min(end - s.first, c.max_new);
  s.len = clampi(c.len[b], 0, min(c.max_len, cap));
  return s;
}

// The page of row `row` (0 <= row < cap) of sequence b.
__device__ __forceinline__ int row_page(const CacheView &c, int b, int row) {
  return c.table ? c.table[(int64_t)b * c.width + (row >> c.shift)] : b;
}
// Byte offset of a row on its page, or -1 where the page is outside the pool.
__device__ __forceinline__ int64_t page_offset(const CacheView &c, int page, int row) {
  const uint32_t in = (uint32_t)row & (c.table ? (1u << c.shift) - 1 : ~0u);
  if ((uint32_t)page >= (uint32_t)c.n_pages) return -1;
  return (int64_t)(((uint64_t)(uint32_t)page * c.page_stride + (uint64_t)in * c.row_stride) << 4);
}
__device__ __forceinline__ int64_t row_offset(const CacheView &c, int b, int row) {
  return page_offset(c, row_page(c, b, row), row);
}

#define SMALLKV_LDS __attribute__((address_space(3)))
#define SMALLKV_GLOBAL __attribute__((address_space(1)))

// 16 bytes per lane from `src` to lds + 16 * lane (lds: the wave's, uniform).
__device__ __forceinline__ void load_to_lds16(const void *src, void *lds) {
  __builtin_amdgcn_global_load_lds((const SMALLKV_GLOBAL void *)src, (SMALLKV_LDS void *)lds, 16, 0, 0);
}

// All of this wave's outstanding memory operations.
__device__ __forceinline__ void wait_memory() {
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("" ::: "memory");
}

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;

// Inclusive sums over the wave (row_shr 1, 2, 4, 8, then across rows of 16 lanes).
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, kWave - 1); }
// The largest value of the wave, the same way (lanes without a source keep theirs).
__device__ __forceinline__ uint32_t wave_umax(uint32_t x) {
  const auto step = [&](uint32_t y) { x = max(x, y); };
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x111, 0xf, 0xf, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x112, 0xf, 0xf, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x114, 0xf, 0xf, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x118, 0xf, 0xf, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x142, 0xa, 0xf, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x143, 0xc, 0xf, false));
  return (uint32_t)last_lane((int)x);
}

// The other half-wave's value (lane ^ 32).
__device__ __forceinline__ float swap_halves_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float swap_halves_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Tiles of cached rows in LDS: row-major, C 16-byte pieces a row, piece c of
// row r at c ^ swizzle(r).  Keys are read a piece per lane, 32 rows at once:
// sixteen neighbouring rows then cover the banks once.  Values are read 64
// bytes (bf16, transposed by the read) or 128 bytes (fp32) of several rows at
// once: rows that are read together go to different parts of the banks.
template <typename T, int D> struct TileLayout {
  static constexpr int C = D * (int)sizeof(T) / 16;
  static constexpr int bytes = D * (int)sizeof(T);
  __device__ __forceinline__ static int swz_k(int r) { return C == 8 ? (r >> 1) & 7 : r & 15; }
  __device__ __forceinline__ static int swz_v(int r) {
    if (sizeof(T) == 4) return ((r >> 2) & 1) << 3;
    return C == 16 ? (r & 3) << 2 : ((r >> 1) & 1) << 2;
  }
};

}  // namespace smallkv
