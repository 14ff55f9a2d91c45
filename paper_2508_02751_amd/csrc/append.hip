// Rotary positions of the new tokens and their way into the cache: queries and
// keys turned pair by pair, x' = a (x cos - y sin), y' = a (x sin + y cos), keys
// and values written to the cache rows of their tokens.
//
// Bound by memory: every element is read once and written once, so the pass is
// laid out by 16-byte pieces.  A workgroup takes kTok tokens; each wave finds
// one token's sequence, row and position, the sines and cosines of the tokens'
// angles are computed once (for all heads) into LDS, then the waves walk the
// (token, 64 slots) pairs, a slot being two pieces of one head: the two halves of
// V pairs, or two neighbouring pieces of interleaved pairs, of a head's tail
// that does not turn, or of a value row.
//
// Measured (MI355X): 23380 tokens of 32 + 2 x 8 heads of 128 in bf16 (575 MB) 117 us,
// 4.9 TB/s, the rate of a large copy (4.7); 5003 fp32 tokens of 14 + 2 x 2 heads of 64
// (46 MB) 9.5 us; one token each of 64 sequences 3.8 us, which is the launch and a chain
// of three dependent loads.
#include "cache.h"
#include "launch.h"

namespace smallkv {
namespace {

struct AppendArgs {
  ChunkView c;
  CacheView kv;
  int hq, hk, rot;
  const unsigned char *q, *k, *v;
  unsigned char *q_out, *ck, *cv;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;  // in bytes
  const int32_t *positions;
  const double *freq;
  float amplitude;
  int32_t *row_pos;
  int64_t pos_rows, pos_stride;
};

// cos and sin of `turns` full turns (64 bits): the nearest quarter turn is taken
// off exactly, the rest, at most an eighth of a turn, fits fp32 with an error of
// 2^-28 turns; then the Taylor series of both (the first terms left out are below
// 2e-9 there).
__device__ __forceinline__ void cos_sin(double turns, float &co, float &si) {
  const double quarter = rint(turns * 4.0);
  const float z = (float)(__builtin_fma(quarter, -0.25, turns) * 6.283185307179586476925);
  const int n = (int)((int64_t)quarter & 3);
  const float z2 = z * z;
  float s = 1.0f / 362880.0f;
  s = __builtin_fmaf(s, z2, -1.0f / 5040.0f);
  s = __builtin_fmaf(s, z2, 1.0f / 120.0f);
  s = __builtin_fmaf(s, z2, -1.0f / 6.0f);
  s = __builtin_fmaf(s * z2, z, z);
  float c = -1.0f / 3628800.0f;
  c = __builtin_fmaf(c, z2, 1.0f / 40320.0f);
  c = __builtin_fmaf(c, z2, -1.0f / 720.0f);
  c = __builtin_fmaf(c, z2, 1.0f / 24.0f);
  c = __builtin_fmaf(c, z2, -0.5f);
  c = __builtin_fmaf(c, z2, 1.0f);
  const float x = n & 1 ? s : c, y = n & 1 ? c : s;
  co = n == 1 || n == 2 ? -x : x;
  si = n >= 2 ? -y : y;
}

template <typename T> __device__ __forceinline__ uint4 pack16(const float *x) {
  uint4 w;
  uint32_t *u = reinterpret_cast<uint32_t *>(&w);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      u[i] = __float_as_uint(x[i]);
    } else {
      const bf16x2_t p = __builtin_convertvector((f32x2_t{x[2 * i], x[2 * i + 1]}), bf16x2_t);
      u[i] = __builtin_bit_cast(uint32_t, p);
    }
  }
  return w;
}

// HALF pairs (j, j + rot/2) in whole pieces, the same one by one (rot/2 is not a
// whole number of pieces), or neighbours.
enum { kHalf = 0, kHalfScalar = 1, kInterleaved = 2 };

template <typename T, int D, int FORM, int TOK>
__global__ __launch_bounds__(256) void append(AppendArgs a) {
  constexpr int V = 16 / (int)sizeof(T), kSlots = D / (2 * V);  // elements a piece, slots a head
  __shared__ float2 cs[TOK][D / 2 + 1];
  struct Where {
    int64_t row;  // the cache row's offset for head 0, or -1
    int token, pos, seq, cached;
  };
  __shared__ Where where[TOK];
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  for (int i = wave; i < TOK; i += 4) {
    const int t = blockIdx.x * TOK + i;
    // the token's sequence: the last one that starts at or before it, if it
    // reaches so far
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
      Where w{-1, -1, 0, 0, 0};
      if (b >= 0 && t < a.c.n_tokens) {
        const Seq s = sequence(a.c, b, a.kv.cap);
        const int row = s.len - s.n_new + (t - s.first);
        w.token = t;
        w.pos = a.positions ? a.positions[t] : row;
        w.seq = b;
        w.cached = row;
        if (row >= 0) w.row = row_offset(a.kv, b, row);
      }
      where[i] = w;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < TOK * (a.rot / 2); i += 256) {
    const int tok = TOK == 1 ? 0 : i / (a.rot / 2), j = i - tok * (a.rot / 2);
    float co, si;
    // (1 / 2 pi: the angle in turns)
    cos_sin((double)where[tok].pos * (a.freq[j] * 0.15915494309189533577), co, si);
    cs[tok][j] = make_float2(a.amplitude * co, a.amplitude * si);
  }
  __syncthreads();
  const int heads = a.hq + 2 * a.hk, chunks = (heads * kSlots + kWave - 1) / kWave;
  for (int w = wave; w < TOK * chunks; w += 4) {
    const int tok = TOK == 1 ? 0 : w / chunks, item = (w - tok * chunks) * kWave + lane;
    const int h = item / kSlots, c = item & (kSlots - 1);
    const Where at = where[tok];
    if (at.token < 0 || h >= heads) continue;
    const unsigned char *src;
    unsigned char *dst;
    const bool value = h >= a.hq + a.hk;
    if (h < a.hq) {
      src = a.q + at.token * a.q_token + h * a.q_head;
      dst = a.q_out + at.token * a.o_token + h * a.o_head;
    } else {
      const int kh = h - a.hq - (value ? a.hk : 0);
      src = value ? a.v + at.token * a.v_token + kh * a.v_head : a.k + at.token * a.k_token + kh * a.k_head;
      if (a.row_pos && !value && c == 0 && at.cached >= 0 && at.cached < a.pos_rows)
        a.row_pos[at.seq * a.pos_stride + kh * a.pos_rows + at.cached] = at.pos;
      if (at.row < 0) continue;
      dst = (value ? a.cv : a.ck) + at.row + (((uint64_t)kh * a.kv.head_stride) << 4);
    }
    const int half = a.rot / 2;
    if (FORM == kHalfScalar && !value) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int j = c * V + e;  // pair j, or two elements of the tail
        const int x = j < half ? j : a.rot + 2 * (j - half), y = j < half ? j + half : x + 1;
        const float u = elem<T>::load1(src, x), v = elem<T>::load1(src, y);
        const float2 r = j < half ? cs[tok][j] : make_float2(0.0f, 0.0f);
        elem<T>::store1(dst, x, j < half ? u * r.x - v * r.y : u);
        elem<T>::store1(dst, y, j < half ? u * r.y + v * r.x : v);
      }
      continue;
    }
    const int turning = half / V;  // slots of turning halves
    const bool halves = FORM == kHalf && !value && c < turning;
    const int p0 = halves ? c : 2 * c;
    const int p1 = halves ? c + turning : p0 + 1;
    uint4 x = reinterpret_cast<const uint4 *>(src)[p0], y = reinterpret_cast<const uint4 *>(src)[p1];
    if (halves) {
      float u[V], v[V];
      elem<T>::unpack(x, u);
      elem<T>::unpack(y, v);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float2 r = cs[tok][c * V + e];
        const float m = u[e] * r.x - v[e] * r.y;
        v[e] = u[e] * r.y + v[e] * r.x;
        u[e] = m;
      }
      x = pack16<T>(u);
      y = pack16<T>(v);
    } else if (FORM == kInterleaved && !value && 2 * c * V < a.rot) {
      float u[2 * V];
      elem<T>::unpack(x, u);
      elem<T>::unpack(y, u + V);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int j = c * V + e;
        const float2 r = cs[tok][min(j, half)];
        const float m = u[2 * e] * r.x - u[2 * e + 1] * r.y, n = u[2 * e] * r.y + u[2 * e + 1] * r.x;
        u[2 * e] = j < half ? m : u[2 * e];
        u[2 * e + 1] = j < half ? n : u[2 * e + 1];
      }
      x = pack16<T>(u);
      y = pack16<T>(u + V);
    }
    reinterpret_cast<uint4 *>(dst)[p0] = x;
    reinterpret_cast<uint4 *>(dst)[p1] = y;
  }
}

template <typename T, int D, int FORM> hipError_t launch_form(const AppendArgs &a, hipStream_t st) {
  // few tokens: one per workgroup, the shortest chain; from there on four, whose
  // sequences, sines and cosines are found once (300 tokens of 48 heads of 128: 4.8 us with
  // one, 7.2 with four; 8000 of 18 heads of 64: 12.4, 9.4)
  if (a.c.n_tokens < 2048)
    hipLaunchKernelGGL((append<T, D, FORM, 1>), dim3(a.c.n_tokens), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((append<T, D, FORM, 4>), dim3((a.c.n_tokens + 3) / 4), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <typename T, int D> hipError_t launch_typed(const AppendArgs &a, int layout, hipStream_t st) {
  if (layout == SMALLKV_ROPE_INTERLEAVED) return launch_form<T, D, kInterleaved>(a, st);
  if (a.rot % (2 * (16 / (int)sizeof(T))) == 0) return launch_form<T, D, kHalf>(a, st);
  return launch_form<T, D, kHalfScalar>(a, st);
}

}  // namespace

hipError_t launch_append(const smallkv_chunk_t &c, const smallkv_cache_t &kv, const smallkv_append_t &p,
                         hipStream_t st) {
  if (c.n_tokens == 0) return hipSuccess;
  const int e = kv.dtype == SMALLKV_F32 ? 4 : 2;
  AppendArgs a{};
  a.c = chunk_view(c);
  a.kv = cache_view(kv);
  a.hq = p.n_q_heads;
  a.hk = kv.n_heads;
  a.rot = p.rot_dim;
  a.q = static_cast<const unsigned char *>(p.q);
  a.k = static_cast<const unsigned char *>(p.k);
  a.v = static_cast<const unsigned char *>(p.v);
  a.q_out = static_cast<unsigned char *>(p.q_out);
  a.ck = static_cast<unsigned char *>(kv.k);
  a.cv = static_cast<unsigned char *>(kv.v);
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
  if (kv.dtype == SMALLKV_F32)
    return kv.head_dim == 64 ? launch_typed<float, 64>(a, p.layout, st) : launch_typed<float, 128>(a, p.layout, st);
  return kv.head_dim == 64 ? launch_typed<bf16_t, 64>(a, p.layout, st) : launch_typed<bf16_t, 128>(a, p.layout, st);
}

}  // namespace smallkv
