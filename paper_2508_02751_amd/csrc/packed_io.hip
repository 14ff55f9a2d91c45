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
//
// Bound by memory.  Measured (MI355X): 21000 tokens of 32 + 2 x 8 heads of 128 in bf16 (461 MB
// read and written) 88 us, 5.3 TB/s; 8000 of 28 + 2 x 4 heads 33 us; one token each of 64
// sequences 5.6 us, a launch and a chain of dependent loads (sequence, page) beside which the
// rows and angles are on their way.  Read: 4 x 20000 - 32768 rows of 32 heads of 64 from 8 bits
// to bf16 (1.26 GB) 266 us, the rate of a large copy.  Few (sequence, head) pairs make too few
// workgroups for it, at most 32 a pair for K and as many for V: one sequence of 32768 rows of 8
// heads of 128 from 8 bits to bf16 (203 MB) 84 us, 2.4 TB/s, of 2 heads of 64 (25 MB) 23 us, 1.1 TB/s.
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
// Cut off, a finite x past fp32's largest number is that number, whose last bit is set: one step
// back from the infinity that it converts to.
__device__ __forceinline__ float round_to_odd(double x) {
  const float f = (float)x;
  const double rest = x - (double)f;  // NaN of infinities and NaN
  const uint32_t u = __float_as_uint(f);
  if (!(rest < 0.0 || rest > 0.0) || (u & 1u)) return f;
  // an even f that is not x: one step towards x is odd
  const bool grow = (rest > 0.0) == (f > 0.0);
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

// 8 elements of a row as they are in memory.
template <typename T> struct Raw8 {
  u32x4_t w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const unsigned char *row, int e) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const u32x4_t *>(row + e * (int)sizeof(T))[i];
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 4)
        x[i] = __uint_as_float(w[i / 4][i % 4]);
      else
        x[i] = i % 2 ? bf16_hi(w[0][i / 2]) : bf16_lo(w[0][i / 2]);
    }
  }
};
template <typename T> __device__ __forceinline__ void store8(unsigned char *row, int e, const float (&x)[8]) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) * 2; ++i) {
    if constexpr (sizeof(T) == 4)
      r.w[i / 4][i % 4] = __float_as_uint(x[i]);
    else
      r.w[0][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{x[2 * i], x[2 * i + 1]}), bf16x2_t));
  }
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<u32x4_t *>(row + e * (int)sizeof(T))[i] = r.w[i];
}

// HALF pairs (j, j + rot/2) of a head that turns whole, the same where halves are whole groups
// of 8, at any rot/2, or neighbours.
enum { kWhole = 0, kHalf = 1, kHalfScalar = 2, kInterleaved = 3 };

// The elements half a head away: of the lane 8 (128 elements) or 4 (64) further in the head's.
template <typename T, int D> __device__ __forceinline__ Raw8<T> other_half(const Raw8<T> &x) {
  Raw8<T> y;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      int w = (int)x.w[i][j];
      if (D == 128) {
        w = __builtin_amdgcn_update_dpp(w, w, 0x128, 0xf, 0xf, false);  // rotated by 8 of 16 lanes
      } else {
        w = __builtin_amdgcn_update_dpp(w, w, 0x141, 0xf, 0xf, false);  // 8 lanes mirrored,
        w = __builtin_amdgcn_update_dpp(w, w, 0x1b, 0xf, 0xf, false);   // then 4
      }
      y.w[i][j] = (uint32_t)w;
    }
  return y;
}

// Elements e .. e + 7 of a head (x) turned: cs[j] are cosine and sine of pair j, other the
// pairs' other halves (kWhole; kHalf, e < rot).
template <typename T, int D, int FORM, typename R, typename CS>
__device__ __forceinline__ void turn8(const unsigned char *row, int e, int rot, const CS *cs, const float (&x)[8],
                                      const Raw8<T> &partner, R (&y)[8]) {
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
  if (FORM != kHalfScalar) partner.get(other);
  if (FORM == kWhole) {
    const bool low = e < D / 2;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const CS r = cs[(e & (D / 2 - 1)) + i];
      const R u = x[i], v = other[i];
      y[i] = u * r.x + (low ? -v : v) * r.y;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = e + i;
    const bool low = at < half, turns = at < rot;
    if (FORM == kHalfScalar) other[i] = turns ? elem<T>::load1(row, low ? at + half : at - half) : 0.0f;
    const CS r = cs[turns ? (low ? at : at - half) : half];
    const R u = x[i], v = other[i];
    // x' = x cos - y sin of the lower half, y' = y cos + x sin of the upper one
    y[i] = !turns ? u : low ? u * r.x - v * r.y : u * r.x + v * r.y;
  }
}

// A token to a workgroup, NI items (8 elements of a head) to a thread; blockIdx.y: slices of the
// token's items.  The rows are requested first, before anything is known of the token.  A wave's
// items are whole heads, so that queries may be turned in place.
template <typename T, int D, int F, int FORM, int NI> __global__ __launch_bounds__(256) void append_packed(PackArgs a) {
  constexpr int W = D / 8;  // lanes of a head
  __shared__ double2 cs[D / 2 + 1];
  __shared__ float2 csf[D / 2 + 1];
  struct Where {
    int64_t row, scale;  // the cache row's offsets for head 0 (row: or -1)
    int in, pos, seq, cached;
  };
  __shared__ Where where;
  const int lane = threadIdx.x & (kWave - 1), t = blockIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int heads = a.hq + 2 * a.hk;
  // The item's head and first element; four lanes, a block, stay or go together.
  auto item = [&](int n, int &h, int &e) {
    const int i = (blockIdx.y * NI + n) * (int)blockDim.x + (int)threadIdx.x;
    h = i / W;
    e = (i & (W - 1)) * 8;
    return h < heads;
  };
  auto source = [&](int h) {
    if (h < a.hq) return a.q + t * a.q_token + h * a.q_head;
    h -= a.hq;
    return h < a.hk ? a.k + t * a.k_token + h * a.k_head : a.v + t * a.v_token + (h - a.hk) * a.v_head;
  };
  Raw8<T> own[NI], partner[NI];
#pragma unroll
  for (int n = 0; n < NI; ++n) {
    int h, e;
    own[n] = partner[n] = Raw8<T>{};
    if (item(n, h, e)) {
      const unsigned char *src = source(h);
      own[n].load(src, e);
      if (FORM == kHalf && e < a.rot && h < a.hq + a.hk)
        partner[n].load(src, e < a.rot / 2 ? e + a.rot / 2 : e - a.rot / 2);
    }
  }
  // The first wave finds the token's sequence, row and place; a lane turns the angle of a pair, in
  // another wave where positions are given.
  const double freq = lane < a.rot / 2 ? a.freq[lane] : 0.0;
  int pos = a.positions ? a.positions[t] : 0;
  if (wave == 0) {
    int b = -1;
    Seq s{0, 0, 0};
    for (int b0 = 0; b0 < a.c.batch; b0 += kWave) {
      Seq x{0, 0, 0};
      if (b0 + lane < a.c.batch) x = sequence(a.c, b0 + lane, a.kv.cap);
      const uint64_t m = __ballot(t >= x.first && t < x.first + x.n_new);
      if (m) {
        const int l = __builtin_amdgcn_readfirstlane(__ffsll((long long)m) - 1);
        b = b0 + l;
        s = Seq{__builtin_amdgcn_readlane(x.first, l), __builtin_amdgcn_readlane(x.n_new, l),
                __builtin_amdgcn_readlane(x.len, l)};
        break;
      }
    }
    Where w{-1, 0, 0, 0, 0, 0};
    if (b >= 0) {
      const int row = s.len - s.n_new + (t - s.first);
      if (!a.positions) pos = row;
      w.in = 1;
      w.pos = pos;
      w.seq = b;
      w.cached = row;
      if (row >= 0) {
        const int page = row_page(a.kv, b, row);
        w.row = page_offset(a.kv, page, row);
        if (w.row >= 0) w.scale = scale_offset<D>(a.sc, a.kv, page, row, 0);
      }
    }
    if (lane == 0) where = w;
  }
  if (wave == (a.positions ? 1 : 0) && lane < a.rot / 2) {
    double co, si;
    cos_sin((double)pos * freq, co, si);
    co *= (double)a.amplitude;
    si *= (double)a.amplitude;
    cs[lane] = make_double2(co, si);
    csf[lane] = make_float2((float)co, (float)si);
  }
  __syncthreads();
  const Where at = where;
  if (!at.in) return;
#pragma unroll
  for (int n = 0; n < NI; ++n) {
    int h, e;
    if (!item(n, h, e)) continue;
    const unsigned char *src = source(h);
    float x[8];
    own[n].get(x);
    if (FORM == kWhole) partner[n] = other_half<T, D>(own[n]);
    if (h < a.hq) {
      float y[8];
      turn8<T, D, FORM, float>(src, e, a.rot, csf, x, partner[n], y);
      store8<T>(a.q_out + t * a.o_token + h * a.o_head, e, y);
      continue;
    }
    const bool value = h >= a.hq + a.hk;
    const int kh = h - a.hq - (value ? a.hk : 0);
    if (a.row_pos && !value && e == 0 && at.cached >= 0 && at.cached < a.pos_rows)
      a.row_pos[at.seq * a.pos_stride + kh * a.pos_rows + at.cached] = at.pos;
    if (at.row < 0) continue;
    if (!value && a.rot > 0) {
      double y[8];
      turn8<T, D, FORM, double>(src, e, a.rot, cs, x, partner[n], y);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = round_to_odd(y[i]);
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

template <typename T, int D, int F, int FORM, int NI> void launch_items(const PackArgs &a, hipStream_t st) {
  const int items = (a.hq + 2 * a.hk) * (D / 8);
  const int threads = std::max(std::min((items + NI - 1) / NI + 63, 256) / 64 * 64, 128);
  const dim3 grid(a.c.n_tokens, (items + threads * NI - 1) / (threads * NI));
  hipLaunchKernelGGL((append_packed<T, D, F, FORM, NI>), grid, dim3(threads), 0, st, a);
}
template <typename T, int D, int F, int FORM> void launch_tokens(const PackArgs &a, hipStream_t st) {
  // few tokens: an item per thread, the shortest chain; else two or three, for which the sines
  // and cosines are found once (4000 tokens of 36 heads of 128 each of two sequences: 41 us with
  // one, 33 with three; 3000 of 18 heads of 64: 8.1 with one, 7.0 with two)
  if (a.c.n_tokens < 512)
    launch_items<T, D, F, FORM, 1>(a, st);
  else if ((a.hq + 2 * a.hk) * (D / 8) <= 256)
    launch_items<T, D, F, FORM, 2>(a, st);
  else
    launch_items<T, D, F, FORM, 3>(a, st);
}
template <typename T, int D, int F> void launch_form(const PackArgs &a, int layout, hipStream_t st) {
  (layout == SMALLKV_ROPE_INTERLEAVED ? launch_tokens<T, D, F, kInterleaved>
   : a.rot == D ? launch_tokens<T, D, F, kWhole> : a.rot % 16 == 0 ? launch_tokens<T, D, F, kHalf> : launch_tokens<T, D, F, kHalfScalar>)(a, st);
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
