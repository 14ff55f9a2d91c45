// Rows on their way into a packed cache and back.
//
// append -- queries and keys turned by their rotary positions, keys and values packed: a lane
//           takes 8 neighbouring elements of a head (and, where pairs are halves of the head
//           apart, their 8 partners), four lanes a block of 32.  Keys are turned in 64 bits
//           and rounded once, to their codes: which side of a border between two codes an
//           element falls on does not depend on how the turn rounds.  Their way to fp32 keeps
//           that: rounded to odd (the last bit set where anything was cut off), comparisons
//           with values of fewer bits and the next rounding see what the 64 bits would show.
// read   -- the reverse, without the turn: 16 bytes of output per lane.
#include <algorithm>

#include "launch.h"
#include "packed.h"

namespace smallkv {
namespace {

struct PackArgs {
  ChunkView c;
  CacheView kv;
  ScaleView sc;
  int hq, hk, rot;
  const unsigned char *q, *k, *v;
  unsigned char *q_out, *ck, *cv;
  uint8_t *sk, *sv;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;  // in bytes
  const int32_t *positions;
  const double *freq;
  float amplitude;
  int32_t *row_pos;
  int64_t pos_rows, pos_stride;
};

// cos and sin of an angle, in 64 bits: quarter turns are taken off in two parts of pi / 2
// (the products are exact inside the fused operation), the rest, at most pi / 4, goes into
// the Taylor series (the first terms left out are below 5e-17 there).
__device__ __forceinline__ void cos_sin(double angle, double &co, double &si) {
  const double quarter = rint(angle * 0.63661977236758134308);
  double z = __builtin_fma(-quarter, 1.5707963267948965580, angle);
  z = __builtin_fma(-quarter, 6.1232339957367660359e-17, z);
  const int n = (int)((int64_t)quarter & 3);
  const double z2 = z * z;
  double s = -1.0 / 1307674368000.0;
  s = __builtin_fma(s, z2, 1.0 / 6227020800.0);
  s = __builtin_fma(s, z2, -1.0 / 39916800.0);
  s = __builtin_fma(s, z2, 1.0 / 362880.0);
  s = __builtin_fma(s, z2, -1.0 / 5040.0);
  s = __builtin_fma(s, z2, 1.0 / 120.0);
  s = __builtin_fma(s, z2, -1.0 / 6.0);
  s = __builtin_fma(s * z2, z, z);
  double c = 1.0 / 20922789888000.0;
  c = __builtin_fma(c, z2, -1.0 / 87178291200.0);
  c = __builtin_fma(c, z2, 1.0 / 479001600.0);
  c = __builtin_fma(c, z2, -1.0 / 3628800.0);
  c = __builtin_fma(c, z2, 1.0 / 40320.0);
  c = __builtin_fma(c, z2, -1.0 / 720.0);
  c = __builtin_fma(c, z2, 1.0 / 24.0);
  c = __builtin_fma(c, z2, -0.5);
  c = __builtin_fma(c, z2, 1.0);
  const double x = n & 1 ? s : c, y = n & 1 ? c : s;
  co = n == 1 || n == 2 ? -x : x;
  si = n >= 2 ? -y : y;
}

// fp32, cut off, the last bit set where the rest is not 0 (infinities and NaN as they are).
__device__ __forceinline__ float round_to_odd(double x) {
  const float f = (float)x;
  const double rest = x - (double)f;
  const uint32_t u = __float_as_uint(f);
  if (rest == 0.0 || (u & 1u) || !(fabsf(f) <= 3.402823466e38f)) return f;
  // an even f that is not x: one step towards x is odd
  const bool grow = (rest > 0.0) == (f > 0.0) || f == 0.0f;
  if (f == 0.0f) return __uint_as_float((__double2hiint(x) & 0x80000000u) | 1u);
  return __uint_as_float(grow ? u + 1u : u - 1u);
}

// 8 elements, their block's scale byte (the same in its four lanes) and codes.
template <int F> struct Codes {
  uint32_t scale, w[2];
  __device__ __forceinline__ explicit Codes(const float (&x)[8]) {
    // the block's largest magnitude, by its bits: NaN above infinity above numbers
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp((int)top, (int)top, 0xb1, 0xf, 0xf, false));  // lane ^ 1
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp((int)top, (int)top, 0x4e, 0xf, 0xf, false));  // lane ^ 2
    // exponents of the scale: that of the largest magnitude less 8 (2), one more where its
    // mantissa is past 464 = 1.8125 * 2^8 (7 = 1.75 * 2^2)
    constexpr uint32_t past = F == 8 ? 0x7fffffu - 0x680000u : 0x7fffffu - 0x600000u;
    const int e = clampi((int)((top + past) >> 23) - 127 - (F == 8 ? 8 : 2), -100, F == 8 ? 119 : 125);
    const bool bad = top >= 0x7f800000u;
    scale = bad ? 255u : (uint32_t)(e + 127);
    const float down = __uint_as_float((uint32_t)(127 - e) << 23), most = F == 8 ? 448.0f : 6.0f;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = bad ? 0.0f : fminf(fmaxf(x[i] * down, -most), most);
    w[0] = w[1] = 0;
    if constexpr (F == 8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], p, true);
      }
    } else {
      w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], y[0], y[1], 1.0f, 0);
      w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], y[2], y[3], 1.0f, 1);
      w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], y[4], y[5], 1.0f, 2);
      w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], y[6], y[7], 1.0f, 3);
    }
  }
};

template <typename T> __device__ __forceinline__ void load8(const unsigned char *row, int e, float (&x)[8]) {
  const uint4 *p = reinterpret_cast<const uint4 *>(row + e * (int)sizeof(T));
  elem<T>::unpack(p[0], x);
  if constexpr (sizeof(T) == 4) elem<T>::unpack(p[1], x + 4);
}
template <typename T> __device__ __forceinline__ void store8(unsigned char *row, int e, const float (&x)[8]) {
  uint4 w[sizeof(T) / 2];
  uint32_t *u = reinterpret_cast<uint32_t *>(w);
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) * 2; ++i) {
    if constexpr (sizeof(T) == 4)
      u[i] = __float_as_uint(x[i]);
    else
      u[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{x[2 * i], x[2 * i + 1]}), bf16x2_t));
  }
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(row + e * (int)sizeof(T))[i] = w[i];
}

// HALF pairs (j, j + rot/2) whose halves are whole groups of 8, the same at any rot/2, or
// neighbours.
enum { kHalf = 0, kHalfScalar = 1, kInterleaved = 2 };

// Elements e .. e + 7 of a head (x) turned: cs[j] are cosine and sine of pair j.
template <typename T, int FORM, typename R, typename CS>
__device__ __forceinline__ void turn8(const unsigned char *row, int e, int rot, const CS *cs, const float (&x)[8],
                                      R (&y)[8]) {
  const int half = rot / 2;
  if (FORM == kInterleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const int j = (e + i) / 2;
      const CS r = cs[min(j, half)];
      const R u = x[i], v = x[i + 1];
      y[i] = j < half ? u * r.x - v * r.y : u;
      y[i + 1] = j < half ? u * r.y + v * r.x : v;
    }
    return;
  }
  float other[8];
  if (FORM == kHalf) {
    if (e < rot) load8<T>(row, e < half ? e + half : e - half, other);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = e + i;
    const bool low = at < half, turns = at < rot;
    if (FORM == kHalfScalar) other[i] = turns ? elem<T>::load1(row, low ? at + half : at - half) : 0.0f;
    const CS r = cs[turns ? (low ? at : at - half) : half];
    const R u = x[i], v = FORM == kHalf && e >= rot ? 0.0f : other[i];
    // x' = x cos - y sin of the lower half, y' = y cos + x sin of the upper one
    y[i] = !turns ? u : low ? u * r.x - v * r.y : u * r.x + v * r.y;
  }
}

template <typename T, int D, int F, int FORM, int TOK>
__global__ __launch_bounds__(256) void append_packed(PackArgs a) {
  constexpr int W = D / 8;  // lanes of a head
  __shared__ double2 cs[TOK][D / 2 + 1];
  __shared__ float2 csf[TOK][D / 2 + 1];
  struct Where {
    int64_t row, scale;  // the cache row's offsets for head 0 (row: or -1)
    int token, pos, seq, cached;
  };
  __shared__ Where where[TOK];
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  for (int i = wave; i < TOK; i += 4) {
    const int t = blockIdx.x * TOK + i;
    // the token's sequence: the one that it is in, if any
    int b = -1;
    for (int b0 = 0; b0 < a.c.batch; b0 += kWave) {
      bool in = false;
      if (b0 + lane < a.c.batch) {
        const Seq s = sequence(a.c, b0 + lane, a.kv.cap);
        in = t >= s.first && t < s.first + s.n_new;
      }
      const uint64_t m = __ballot(in);
      if (m) {
        b = b0 + __ffsll((long long)m) - 1;
        break;
      }
    }
    if (lane == 0) {
      Where w{-1, 0, -1, 0, 0, 0};
      if (b >= 0 && t < a.c.n_tokens) {
        const Seq s = sequence(a.c, b, a.kv.cap);
        const int row = s.len - s.n_new + (t - s.first);
        w.token = t;
        w.pos = a.positions ? a.positions[t] : row;
        w.seq = b;
        w.cached = row;
        if (row >= 0) {
          const int page = row_page(a.kv, b, row);
          w.row = page_offset(a.kv, page, row);
          if (w.row >= 0) w.scale = scale_offset<D>(a.sc, a.kv, page, row, 0);
        }
      }
      where[i] = w;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < TOK * (a.rot / 2); i += 256) {
    const int tok = TOK == 1 ? 0 : i / (a.rot / 2), j = i - tok * (a.rot / 2);
    double co, si;
    cos_sin((double)where[tok].pos * a.freq[j], co, si);
    cs[tok][j] = make_double2((double)a.amplitude * co, (double)a.amplitude * si);
    csf[tok][j] = make_float2((float)cs[tok][j].x, (float)cs[tok][j].y);
  }
  __syncthreads();
  const int heads = a.hq + 2 * a.hk, chunks = (heads * W + kWave - 1) / kWave;
  for (int i = wave; i < TOK * chunks; i += 4) {
    const int tok = TOK == 1 ? 0 : i / chunks, item = (i - tok * chunks) * kWave + lane;
    const int h = item / W, e = (item & (W - 1)) * 8;
    const Where at = where[tok];
    if (at.token < 0 || h >= heads) continue;  // (whole heads: four lanes stay or go together)
    if (h < a.hq) {
      const unsigned char *src = a.q + at.token * a.q_token + h * a.q_head;
      float x[8], y[8];
      load8<T>(src, e, x);
      turn8<T, FORM, float>(src, e, a.rot, csf[tok], x, y);
      store8<T>(a.q_out + at.token * a.o_token + h * a.o_head, e, y);
      continue;
    }
    const bool value = h >= a.hq + a.hk;
    const int kh = h - a.hq - (value ? a.hk : 0);
    if (a.row_pos && !value && e == 0 && at.cached >= 0 && at.cached < a.pos_rows)
      a.row_pos[at.seq * a.pos_stride + kh * a.pos_rows + at.cached] = at.pos;
    if (at.row < 0) continue;
    const unsigned char *src = value ? a.v + at.token * a.v_token + kh * a.v_head : a.k + at.token * a.k_token + kh * a.k_head;
    float x[8];
    load8<T>(src, e, x);
    if (!value && a.rot > 0) {
      double y[8];
      turn8<T, FORM, double>(src, e, a.rot, cs[tok], x, y);
#pragma unroll
      for (int n = 0; n < 8; ++n) x[n] = round_to_odd(y[n]);
    }
    const Codes<F> c(x);
    unsigned char *dst = (value ? a.cv : a.ck) + at.row + (((uint64_t)kh * a.kv.head_stride) << 4);
    if (F == 8)
      *reinterpret_cast<uint2 *>(dst + e) = make_uint2(c.w[0], c.w[1]);
    else
      *reinterpret_cast<uint32_t *>(dst + e / 2) = c.w[0];
    if (e % kBlock == 0)
      (value ? a.sv : a.sk)[at.scale + (int64_t)kh * a.sc.head_stride * (D / kBlock) + e / kBlock] = (uint8_t)c.scale;
  }
}

struct ReadArgs {
  int batch, max_len, heads;
  const int32_t *begin, *len;
  CacheView from, to;
  ScaleView sc;
  unsigned char *to_k, *to_v;
};

// blockIdx.x: (sequence, head); blockIdx.y: interleaved shares of the output's pieces; z: K, V.
template <typename T, int D, int F> __global__ __launch_bounds__(256) void read_packed(ReadArgs a) {
  constexpr int E = 16 / (int)sizeof(T), W = D / E, C = E * F / 8;  // elements, pieces a row, bytes of codes
  const int b = blockIdx.x / a.heads, h = blockIdx.x % a.heads;
  const int len = clampi(a.len[b], 0, min(a.max_len, min(a.from.cap, a.to.cap)));
  const int begin = a.begin ? clampi(a.begin[b], 0, len) : 0;
  const unsigned char *from = (blockIdx.z ? a.from.v : a.from.k) + (((uint64_t)h * a.from.head_stride) << 4);
  const uint8_t *scales = blockIdx.z ? a.sc.v : a.sc.k;
  unsigned char *to = (blockIdx.z ? a.to_v : a.to_k) + (((uint64_t)h * a.to.head_stride) << 4);
  const int64_t items = (int64_t)(len - begin) * W;
  for (int64_t i = blockIdx.y * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.y * 256) {
    const int row = begin + (int)(i / W), p = (int)(i & (W - 1));
    const int page = row_page(a.from, b, row);
    const int64_t s = page_offset(a.from, page, row), d = row_offset(a.to, b, row);
    if (s < 0 || d < 0) continue;
    const float scale = scale_of(scales[scale_offset<D>(a.sc, a.from, page, row, h) + p * E / kBlock]);
    uint32_t w[2] = {0, 0};
    if constexpr (C == 8) {
      const uint2 x = *reinterpret_cast<const uint2 *>(from + s + p * C);
      w[0] = x.x;
      w[1] = x.y;
    } else if constexpr (C == 4) {
      w[0] = *reinterpret_cast<const uint32_t *>(from + s + p * C);
    } else {
      w[0] = *reinterpret_cast<const uint16_t *>(from + s + p * C);
    }
    reinterpret_cast<uint4 *>(to + d)[p] = unpack16<T, F>(w, 0, scale);
  }
}

template <typename T, int D, int F, int FORM> void launch_tokens(const PackArgs &a, hipStream_t st) {
  if (a.c.n_tokens < 2048)
    hipLaunchKernelGGL((append_packed<T, D, F, FORM, 1>), dim3(a.c.n_tokens), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((append_packed<T, D, F, FORM, 4>), dim3((a.c.n_tokens + 3) / 4), dim3(256), 0, st, a);
}
template <typename T, int D, int F> void launch_form(const PackArgs &a, int layout, hipStream_t st) {
  (layout == SMALLKV_ROPE_INTERLEAVED ? launch_tokens<T, D, F, kInterleaved>
   : a.rot % 16 == 0 ? launch_tokens<T, D, F, kHalf> : launch_tokens<T, D, F, kHalfScalar>)(a, st);
}
template <typename T, int D, int F> void launch_read(const ReadArgs &a, dim3 grid, hipStream_t st) {
  hipLaunchKernelGGL((read_packed<T, D, F>), grid, dim3(256), 0, st, a);
}

}  // namespace

hipError_t launch_append_packed(const smallkv_chunk_t &c, const smallkv_packed_t &kv, const smallkv_append_t &p,
                                hipStream_t st) {
  if (c.n_tokens == 0) return hipSuccess;
  const int e = kv.dtype == SMALLKV_F32 ? 4 : 2;
  PackArgs a{};
  a.c = chunk_view(c);
  a.kv = cache_view(codes_of(kv));
  a.sc = scale_view(kv);
  a.hq = p.n_q_heads;
  a.hk = kv.n_heads;
  a.rot = p.rot_dim;
  a.q = static_cast<const unsigned char *>(p.q);
  a.k = static_cast<const unsigned char *>(p.k);
  a.v = static_cast<const unsigned char *>(p.v);
  a.q_out = static_cast<unsigned char *>(p.q_out);
  a.ck = static_cast<unsigned char *>(kv.k);
  a.cv = static_cast<unsigned char *>(kv.v);
  a.sk = kv.k_scale;
  a.sv = kv.v_scale;
  a.q_token = p.q_token_stride * e;
  a.q_head = p.q_head_stride * e;
  a.k_token = p.k_token_stride * e;
  a.k_head = p.k_head_stride * e;
  a.v_token = p.v_token_stride * e;
  a.v_head = p.v_head_stride * e;
  a.o_token = p.q_out_token_stride * e;
  a.o_head = p.q_out_head_stride * e;
  a.positions = p.positions;
  a.freq = p.freq;
  a.amplitude = p.amplitude;
  a.row_pos = p.row_pos;
  a.pos_rows = p.pos_rows;
  a.pos_stride = p.pos_seq_stride;
  const bool f8 = format_bits(kv) == 8, d64 = kv.head_dim == 64;
  if (kv.dtype == SMALLKV_F32)
    (f8 ? d64 ? launch_form<float, 64, 8> : launch_form<float, 128, 8>
        : d64 ? launch_form<float, 64, 4> : launch_form<float, 128, 4>)(a, p.layout, st);
  else
    (f8 ? d64 ? launch_form<bf16_t, 64, 8> : launch_form<bf16_t, 128, 8>
        : d64 ? launch_form<bf16_t, 64, 4> : launch_form<bf16_t, 128, 4>)(a, p.layout, st);
  return hipGetLastError();
}

hipError_t launch_read_packed(const smallkv_packed_t &from, const smallkv_cache_t &to, int batch, int max_len,
                              const int32_t *begin, const int32_t *len, hipStream_t st) {
  ReadArgs a{};
  a.batch = batch;
  a.max_len = max_len;
  a.heads = from.n_heads;
  a.begin = begin;
  a.len = len;
  a.from = cache_view(codes_of(from));
  a.sc = scale_view(from);
  a.to = cache_view(to);
  a.to_k = static_cast<unsigned char *>(to.k);
  a.to_v = static_cast<unsigned char *>(to.v);
  const int64_t rows = std::min(max_len, std::min(a.from.cap, a.to.cap));
  const int64_t pieces = rows * (to.head_dim * (to.dtype == SMALLKV_F32 ? 4 : 2) / 16);
  const dim3 grid(batch * from.n_heads, (unsigned)std::min<int64_t>((pieces + 255) / 256, 32), 2);
  const bool f8 = format_bits(from) == 8, d64 = from.head_dim == 64;
  if (to.dtype == SMALLKV_F32)
    (f8 ? d64 ? launch_read<float, 64, 8> : launch_read<float, 128, 8>
        : d64 ? launch_read<float, 64, 4> : launch_read<float, 128, 4>)(a, grid, st);
  else
    (f8 ? d64 ? launch_read<bf16_t, 64, 8> : launch_read<bf16_t, 128, 8>
        : d64 ? launch_read<bf16_t, 64, 4> : launch_read<bf16_t, 128, 4>)(a, grid, st);
  return hipGetLastError();
}

}  // namespace smallkv
