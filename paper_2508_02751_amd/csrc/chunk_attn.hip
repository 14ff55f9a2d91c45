// Attention of the new tokens of every sequence over a paged or dense cache
// (the last n_b of its len_b rows are the new tokens' own):
//   s_t = scale * <q, K_t> for rows t <= own row,  out = softmax(s) V,
//   lse = ln sum exp(s)
// in one pass over the rows with the running maximum and sum of the softmax.
// The query heads of a kv head share its rows: a row of the left product is a
// (token, query head of the group) pair, row r being token r / g, head r % g.
//
// Both products run on the matrix cores, transposed: S^T = K Q^T leaves each
// lane with one query row (its column) and 16 keys of a 32-key block in
// registers, so the softmax needs one exchange between half-waves, and P^T is
// already laid out as the right operand of O^T = V^T P^T up to the order of
// the keys, which the reads of V follow.  Logits, statistics and the output
// accumulate in fp32; P is rounded to bf16 for the second product of a bf16
// model (its relative error, at most 2^-8, is averaged over the row's keys and stays
// below that of the output's own rounding); fp32 models multiply in fp32.
//
// Two forms:
//   many rows -- NW waves of 32 rows each share every tile of rows in LDS;
//                tiles are double-buffered, copied from memory to LDS directly;
//   few rows  -- sequences of at most 32 rows (a decode step's single tokens):
//                one column of 32 rows, each wave reads its own tiles of keys
//                and the waves' results are joined at the end.
// Where the (tile, kv head) pairs are too few to fill the GPU the rows are cut
// into spans, and chunk_merge joins their records.
#include <algorithm>

#include "cache.h"
#include "launch.h"

namespace smallkv {
namespace {

__device__ __align__(16) unsigned char zero_row[512];  // absent rows are read from here

struct AttnArgs {
  ChunkView c;
  CacheView kv;
  int hq, hkv, g;
  const unsigned char *q;
  unsigned char *out;
  int64_t q_token, q_head, o_token, o_head;  // in elements
  float *lse;     // [n_tokens][hq] or null
  float scale2, scale2_lo;  // scale * log2(e), and what its rounding left
  int few;        // sequences of at most 32 rows go to the few-rows form
  int span;       // cached rows per record; one record: the output is written directly
  int n_split;
  float *rec;     // [split][tile * hkv][rows][D] fp32, then [split][tile * hkv][rows][2]
  int64_t rec_ml; // where the second array starts, in floats
};

constexpr double kLog2e = 1.4426950408889634074;
constexpr float kLn2 = 0.693147180559945309417f;

// The 32-row tile of a sequence or tile number `flat` over all sequences.
struct Tile {
  int b, row0, rows;  // sequence, first row, the sequence's rows
  Seq s;
};

__device__ __forceinline__ bool few_rows(const AttnArgs &a, const Seq &s) {
  return a.few && s.n_new * a.g <= 32;
}

// Tiles of BM rows are numbered sequence by sequence; within one, the last
// rows (which see the most keys) first.
template <int BM> __device__ __forceinline__ bool locate(const AttnArgs &a, int flat, Tile &t) {
  const int lane = threadIdx.x & (kWave - 1);
  for (int b0 = 0; b0 < a.c.batch; b0 += kWave) {
    int n = 0;
    if (b0 + lane < a.c.batch) {
      const Seq s = sequence(a.c, b0 + lane, a.kv.cap);
      if (!few_rows(a, s)) n = (s.n_new * a.g + BM - 1) / BM;
    }
    int x = n;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int y = __shfl_up(x, o, kWave);
      if (lane >= o) x += y;
    }
    const uint64_t m = __ballot(x > flat);
    if (m) {
      const int l = __builtin_amdgcn_readfirstlane(__ffsll((long long)m) - 1);
      t.b = b0 + l;
      const int tiles = __shfl(n, l, kWave), before = __shfl(x, l, kWave) - tiles;
      t.row0 = __builtin_amdgcn_readfirstlane((tiles - 1 - (flat - before)) * BM);
      t.s = sequence(a.c, t.b, a.kv.cap);
      t.rows = t.s.n_new * a.g;
      return true;
    }
    flat -= __builtin_amdgcn_readfirstlane(__shfl(x, kWave - 1, kWave));
  }
  return false;
}

template <bool PRIV, int BM> __device__ __forceinline__ bool find_tile(const AttnArgs &a, int flat, Tile &t) {
  if (!PRIV) return locate<BM>(a, flat, t);
  t.b = flat;
  t.row0 = 0;
  t.s = sequence(a.c, t.b, a.kv.cap);
  t.rows = t.s.n_new * a.g;
  return t.rows > 0 && t.rows <= 32;
}

// A wave's share of the copies of one tile of rows.  The page of the lane's row is
// looked up a tile ahead; the rows' offsets are then passed between lanes.
template <typename T, int D, int BN, int SHARE> struct Loader {
  using L = TileLayout<T, D>;
  static constexpr int kRpi = 64 / L::C;        // rows per instruction
  static constexpr int kInstr = SHARE / kRpi;   // instructions per wave, K or V
  static_assert(SHARE % kRpi == 0 && kInstr >= 1, "a wave copies whole instructions");
  int row, page;  // the lane's row of the looked-up tile, and its page (-1: none)

  __device__ __forceinline__ void lookup(const CacheView &kv, int b, int row0, int len) {
    row = row0 + (int)(threadIdx.x & (BN - 1));
    page = -1;
    if (row < len) page = row_page(kv, b, row);
  }
  // Rows first..first+SHARE-1 of the tile; sk, sv: the tile's start in LDS.
  // Returns which rows exist.
  __device__ __forceinline__ uint64_t issue(const CacheView &kv, const unsigned char *k, const unsigned char *v,
                                            int first, unsigned char *sk, unsigned char *sv) const {
    const int lane = threadIdx.x & (kWave - 1), rr = lane / L::C, p = lane & (L::C - 1);
    const int64_t off = page_offset(kv, page, row);
#pragma unroll
    for (int j = 0; j < kInstr; ++j) {
      const int r = first + j * kRpi + rr;
      const int lo = __shfl((int)off, r, kWave), hi = __shfl((int)(off >> 32), r, kWave);
      const int64_t o = ((int64_t)hi << 32) | (uint32_t)lo;
      const unsigned char *pk = hi < 0 ? zero_row : k + o;
      const unsigned char *pv = hi < 0 ? zero_row : v + o;
      load_to_lds16(pk + ((p ^ L::swz_k(r)) << 4), sk + (first + j * kRpi) * L::bytes);
      load_to_lds16(pv + ((p ^ L::swz_v(r)) << 4), sv + (first + j * kRpi) * L::bytes);
    }
    return __ballot(off >= 0);
  }
};

template <typename T, int D> struct QFrag;
template <int D> struct QFrag<bf16_t, D> {
  bf16x8_t f[D / 16];
  __device__ __forceinline__ void load(const unsigned char *row, int half) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) f[s] = *reinterpret_cast<const bf16x8_t *>(row + s * 32 + half * 16);
  }
};
template <int D> struct QFrag<float, D> {
  f32x4_t f[D / 8];
  __device__ __forceinline__ void load(const unsigned char *row, int half) {
#pragma unroll
    for (int s = 0; s < D / 8; ++s) f[s] = *reinterpret_cast<const f32x4_t *>(row + half * (D * 2) + s * 16);
  }
};

// S^T of 32 keys (rows key0 .. of the tile) and the wave's 32 query rows.
template <typename T, int D>
__device__ __forceinline__ f32x16_t logits32(const unsigned char *sk, int key0, const QFrag<T, D> &q) {
  using L = TileLayout<T, D>;
  const int lane = threadIdx.x & (kWave - 1), r = key0 + (lane & 31), half = lane >> 5;
  const unsigned char *row = sk + r * L::bytes;
  const int z = L::swz_k(r);
  if constexpr (sizeof(T) == 2) {
    f32x16_t s = {};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const bf16x8_t k = *reinterpret_cast<const bf16x8_t *>(row + (((2 * i + half) ^ z) << 4));
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q.f[i], s, 0, 0, 0);
    }
    return s;
  } else {
    // the head dimension in two halves, a half-wave each, and four sums: a chain
    // of D / 8 roundings instead of D / 2, and independent instructions
    f32x16_t s[4] = {};
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const f32x4_t k = *reinterpret_cast<const f32x4_t *>(row + (((half * (D / 8) + i) ^ z) << 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], q.f[i][e], s[e], 0, 0, 0);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
  }
}

// Key of register i of a 32-key block, before the half-wave's 4 * half.
__device__ __forceinline__ constexpr int reg_key(int i) { return 8 * (i / 4) + i % 4; }

// O^T += V^T P^T over 32 keys.
template <typename T, int D>
__device__ __forceinline__ void values32(const unsigned char *sv, int key0, const f32x16_t &p,
                                         f32x16_t (&o)[D / 32]) {
  using L = TileLayout<T, D>;
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8_t pf;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const bf16x2_t w = __builtin_convertvector((f32x2_t{p[8 * s + e], p[8 * s + e + 1]}), bf16x2_t);
        pf[e] = w[0];
        pf[e + 1] = w[1];
      }
      // the transposing read: 16 lanes take 4 rows of 16 elements, lane i of
      // them ends with the 4 rows' element i
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        union { s16x4_t h[2]; bf16x8_t v; } vf;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int r = key0 + 16 * s + 8 * x + 4 * half + ((lane & 15) >> 2);
          const int c = d * 4 + ((lane & 31) >> 4) * 2 + ((lane & 3) >> 1);
          const unsigned char *at = sv + r * L::bytes + ((c ^ L::swz_v(r)) << 4) + (lane & 1) * 8;
          vf.h[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SMALLKV_LDS s16x4_t *)at);
        }
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.v, pf, o[d], 0, 0, 0);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = key0 + reg_key(i) + 4 * half;
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        const int c = d * 8 + ((lane & 31) >> 2);
        const float v = *reinterpret_cast<const float *>(sv + r * L::bytes + ((c ^ L::swz_v(r)) << 4) + (lane & 3) * 4);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[i], o[d], 0, 0, 0);
      }
    }
  }
}

// Sets infinite and NaN elements of 16 bytes to 0; whether there were any.
template <typename T> __device__ __forceinline__ bool drop_not_finite(uint4 &w) {
  uint32_t *x = reinterpret_cast<uint32_t *>(&w);
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool hi = (x[i] & 0x7f800000u) == 0x7f800000u, lo = sizeof(T) == 2 && (x[i] & 0x7f80u) == 0x7f80u;
    any |= hi || lo;
    x[i] &= (hi ? (sizeof(T) == 2 ? 0xffffu : 0u) : ~0u) & (lo ? 0xffff0000u : ~0u);
  }
  return any;
}

template <typename T, int D> struct State {
  float m, l;  // running maximum (log2 units), this half-wave's part of the sum
  f32x16_t o[D / 32];
};

// The running maximum, sum and output of a tile's logits s.
template <typename T, int D, int NB>
__device__ __forceinline__ void softmax_step(State<T, D> &st, f32x16_t (&s)[NB], float c, float c_lo) {
  float mx = s[0][0];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
  mx = swap_halves_max(mx) * c;
  // the reference point moves only when a row's maximum has grown by more than
  // 2^8 since it was set: exponentials up to 2^8 lose nothing in fp32 or bf16
  if (__any(mx > st.m + 8.0f)) {
    const float m = fmaxf(st.m, mx);
    const float f = __builtin_amdgcn_exp2f(st.m - (m == -INFINITY ? 0.0f : m));
    st.m = m;
    st.l *= f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.o[d][i] *= f;
  }
  const float base = st.m == -INFINITY ? 0.0f : st.m;
  float sum = 0.0f;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      // (fp32 models: the factor in two parts; -inf times the second may not be -inf)
      const float x = sizeof(T) == 4 ? __builtin_fmaf(fmaxf(s[b][i], -3.402823466e38f), c_lo, -base) : -base;
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], c, x));
      s[b][i] = p;
      sum += p;
    }
  st.l += sum;
}

// A tile that every row of the wave sees whole.
template <typename T, int D, int BN>
__device__ __forceinline__ void full_tile(State<T, D> &st, const QFrag<T, D> &q, const unsigned char *sk,
                                          const unsigned char *sv, float c, float c_lo) {
  f32x16_t s[BN / 32];
#pragma unroll
  for (int b = 0; b < BN / 32; ++b) s[b] = logits32<T, D>(sk, 32 * b, q);
  softmax_step<T, D>(st, s, c, c_lo);
#pragma unroll
  for (int b = 0; b < BN / 32; ++b) values32<T, D>(sv, 32 * b, s[b], st.o);
}

// Any other, 32 keys at a time.  own: the lane's own row; valid: bit t set iff key
// row0 + t exists.
template <typename T, int D, int BN>
__device__ __forceinline__ void masked_tile(State<T, D> &st, const QFrag<T, D> &q, const unsigned char *sk,
                                            const unsigned char *sv, int row0, int own, uint64_t valid,
                                            float c, float c_lo) {
  const int half = (threadIdx.x & (kWave - 1)) >> 5;
#pragma unroll 1
  for (int k0 = 0; k0 < BN; k0 += 32) {
    f32x16_t s[1] = {logits32<T, D>(sk, k0, q)};
    const uint32_t bits = (uint32_t)(valid >> k0) >> (4 * half);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const bool ok = (bits >> reg_key(i) & 1u) && row0 + k0 + reg_key(i) + 4 * half <= own;
      s[0][i] = ok ? s[0][i] : -INFINITY;
    }
    softmax_step<T, D>(st, s, c, c_lo);
    values32<T, D>(sv, k0, s[0], st.o);
  }
}

// Adds the infinite and NaN values of keys from..to to the lane's own elements of
// an output row that is written already (any weight > 0 leaves them what they are).
template <typename O, typename T, int D>
__device__ __forceinline__ void give_back(const AttnArgs &a, int b, const unsigned char *v, void *out, int from, int to) {
  const int half = (threadIdx.x & (kWave - 1)) >> 5;
#pragma unroll 1
  for (int key = from; key <= to; ++key) {
    const int64_t off = row_offset(a.kv, b, key);
    if (off < 0) continue;
#pragma unroll 1
    for (int i = 0; i < D / 2; ++i) {
      const int e = 8 * (i / 4) + i % 4 + 4 * half;
      const float x = elem<T>::load1(v + off, e);
      if (!(fabsf(x) <= 3.402823466e38f)) elem<O>::store1(out, e, elem<O>::load1(out, e) + x);
    }
  }
}

// PRIV: the few-rows form (waves take turns at the tiles of BN keys).
template <typename T, int D, int NW, bool PRIV, int BN>
__global__ __launch_bounds__(NW * kWave, !PRIV && sizeof(T) == 2 ? 2 : 1) void chunk_attn(AttnArgs a) {
  using L = TileLayout<T, D>;
  constexpr int BM = PRIV ? 32 : NW * 32, kBuf = BN * L::bytes * (PRIV ? NW : 1);
  constexpr int kShare = PRIV ? BN : BN / NW;
  // four arrays: what is copied into one does not hold up the reads of another
  __shared__ __align__(16) unsigned char k0[kBuf], v0[kBuf], k1[kBuf], v1[kBuf];
  __shared__ float ml[2][2][kWave];
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int kvh = blockIdx.x % a.hkv, flat = blockIdx.x / a.hkv;
  Tile t;
  if (!find_tile<PRIV, BM>(a, flat, t)) return;
  const int pos0 = t.s.len - t.s.n_new;  // cached row of the first new token
  const int last = min(t.row0 + BM, t.rows) - 1;
  const int limit = max(pos0 + last / a.g + 1, 0);  // keys the tile's rows see (<= len)
  const int split = blockIdx.y, begin = split * a.span, end = min(limit, begin + a.span);
  if (begin >= limit && split > 0) return;
  // the lane's row
  const int r = t.row0 + (PRIV ? 0 : wave * 32) + (lane & 31);
  const bool live = r < t.rows;
  const int rc = live ? r : t.rows - 1, token = t.s.first + rc / a.g, head = kvh * a.g + rc % a.g;
  const int own = live ? pos0 + rc / a.g : -1;
  const int first_own = pos0 + t.row0 / a.g;  // of the workgroup's first row
  const int highest = pos0 + min(t.row0 + (PRIV ? 0 : wave * 32) + 31, t.rows - 1) / a.g;  // of the wave's last
  const bool idle = !PRIV && t.row0 + wave * 32 >= t.rows;
  QFrag<T, D> q;
  q.load(a.q + (token * a.q_token + head * a.q_head) * (int64_t)sizeof(T), lane >> 5);
  const unsigned char *k = a.kv.k + (((uint64_t)kvh * a.kv.head_stride) << 4);
  const unsigned char *v = a.kv.v + (((uint64_t)kvh * a.kv.head_stride) << 4);

  State<T, D> st;
  st.m = -INFINITY;
  st.l = 0.0f;
#pragma unroll
  for (int d = 0; d < D / 32; ++d) st.o[d] = f32x16_t{};

  constexpr uint64_t kAll = BN == 64 ? ~0ull : (1ull << (BN & 63)) - 1;
  const int step = PRIV ? NW * BN : BN, at = PRIV ? wave * BN * L::bytes : 0;
  const int mine = PRIV ? 0 : wave * kShare;
  int row = begin + (PRIV ? wave * BN : 0);
  Loader<T, D, BN, kShare> ld;
  ld.lookup(a.kv, t.b, row, end);
  uint64_t valid = 0;
  if (row < end) {
    valid = ld.issue(a.kv, k, v, mine, k0 + at, v0 + at);
    ld.lookup(a.kv, t.b, row + step, end);
  }
  // the tile at `row` is in place; the next one goes to (nk, nv)
  auto advance = [&](unsigned char *nk, unsigned char *nv) {
    wait_memory();  // this wave's copies of the tile, and its reads of the other buffer
    if (!PRIV) __syncthreads();
    const uint64_t now = valid;
    if (row + step < end) {
      valid = ld.issue(a.kv, k, v, mine, nk + at, nv + at);
      ld.lookup(a.kv, t.b, row + 2 * step, end);
    }
    return now;
  };
  // tiles that every row sees whole, then the others
  bool odd = false, taken = false;
  uint64_t now = 0;
  bool full = true;
  while (row < end) {
    now = advance(k1, v1);
    if (!(full = row + BN - 1 <= first_own && (now & kAll) == kAll)) break;
    if (!idle) full_tile<T, D, BN>(st, q, k0 + at, v0 + at, a.scale2, a.scale2_lo);
    row += step;
    if (row >= end) break;
    odd = true;
    now = advance(k0, v0);
    if (!(full = row + BN - 1 <= first_own && (now & kAll) == kAll)) break;
    if (!idle) full_tile<T, D, BN>(st, q, k1 + at, v1 + at, a.scale2, a.scale2_lo);
    row += step;
    odd = false;
  }
  while (row < end) {
    unsigned char *sk = (odd ? k1 : k0) + at, *sv = (odd ? v1 : v0) + at;
    if (full) now = advance(odd ? k0 : k1, odd ? v0 : v1);
    full = true;
    if (min(row + BN, end) - 1 > first_own) {
      // some row does not see some key, and 0 * inf or 0 * NaN would reach it
      // through the matrix product: such values are taken out here and given to
      // the rows that see them at the end
      bool found = false;
      for (int i = PRIV ? lane : threadIdx.x; i < BN * L::C; i += PRIV ? kWave : NW * kWave) {
        uint4 w = reinterpret_cast<uint4 *>(sv)[i];
        if (drop_not_finite<T>(w)) {
          reinterpret_cast<uint4 *>(sv)[i] = w;
          found = true;
        }
      }
      taken |= PRIV ? __any(found) : __syncthreads_or(found);
    }
    if (!idle && row <= highest)
      masked_tile<T, D, BN>(st, q, sk, sv, row, own, now, a.scale2, a.scale2_lo);
    row += step;
    odd = !odd;
  }
  if (PRIV) {
    taken = __syncthreads_or(taken);
    // join the waves' results: the upper half hands over to the lower one
    float *x = reinterpret_cast<float *>(k0);
#pragma unroll
    for (int h = NW / 2; h >= 1; h >>= 1) {
      __syncthreads();
      if (wave >= h && wave < 2 * h) {
        float *y = x + (wave - h) * (D / 2) * kWave;
        ml[0][wave - h][lane] = st.m;
        ml[1][wave - h][lane] = st.l;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) y[(d * 16 + i) * kWave + lane] = st.o[d][i];
      }
      __syncthreads();
      if (wave < h) {
        const float *y = x + wave * (D / 2) * kWave;
        const float om = ml[0][wave][lane], ol = ml[1][wave][lane];
        const float m = fmaxf(st.m, om), base = m == -INFINITY ? 0.0f : m;
        const float f = __builtin_amdgcn_exp2f(st.m - base), fo = __builtin_amdgcn_exp2f(om - base);
        st.m = m;
        st.l = st.l * f + ol * fo;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) st.o[d][i] = st.o[d][i] * f + y[(d * 16 + i) * kWave + lane] * fo;
      }
    }
    if (wave > 0) return;
  }
  if (!live) return;
  const float l = swap_halves_sum(st.l);
  const int half = lane >> 5;
  if (a.n_split > 1) {
    const int64_t at_row = ((int64_t)split * gridDim.x + blockIdx.x) * BM + (r - t.row0);
    float *o = a.rec + at_row * D;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4_t *>(o + d * 32 + 2 * i + 4 * half) =
            f32x4_t{st.o[d][i], st.o[d][i + 1], st.o[d][i + 2], st.o[d][i + 3]};
    if (half == 0) {
      a.rec[a.rec_ml + 2 * at_row] = st.m;
      a.rec[a.rec_ml + 2 * at_row + 1] = l;
    }
    if (taken) give_back<float, T, D>(a, t.b, v, o, max(begin, first_own + 2 - BN), min(end - 1, own));
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // (0: the row sees no key)
  unsigned char *o = a.out + (token * a.o_token + head * a.o_head) * (int64_t)sizeof(T);
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const f32x4_t x = f32x4_t{st.o[d][i], st.o[d][i + 1], st.o[d][i + 2], st.o[d][i + 3]} * inv;
      const int e = d * 32 + 2 * i + 4 * half;
      if constexpr (sizeof(T) == 4)
        *reinterpret_cast<f32x4_t *>(o + e * 4) = x;
      else
        *reinterpret_cast<bf16x4_t *>(o + e * 2) = __builtin_convertvector(x, bf16x4_t);
    }
  if (taken) give_back<T, T, D>(a, t.b, v, o, max(begin, first_own + 2 - BN), min(end - 1, own));
  if (a.lse && half == 0)
    a.lse[(int64_t)token * a.hq + head] = l == 0.0f ? -INFINITY : (st.m + __log2f(l)) * kLn2;
}

// Joins the records of a row's spans: a wave per row, D / 64 elements a lane.
template <typename T, int D, bool PRIV, int BM>
__global__ __launch_bounds__(4 * kWave) void chunk_merge(AttnArgs a) {
  constexpr int E = D / kWave;
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int kvh = blockIdx.x % a.hkv, flat = blockIdx.x / a.hkv;
  Tile t;
  if (!find_tile<PRIV, BM>(a, flat, t)) return;
  const int in = blockIdx.y * 4 + wave, r = t.row0 + in;
  if (r >= t.rows) return;
  const int own = t.s.len - t.s.n_new + r / a.g;
  const int token = t.s.first + r / a.g, head = kvh * a.g + r % a.g;
  // spans that hold a row this one sees; the others wrote nothing it needs
  const int n = min(max((own + a.span) / a.span, 0), a.n_split);
  const int64_t stride = (int64_t)gridDim.x * BM, at = (int64_t)blockIdx.x * BM + in;
  float m = -INFINITY;
  for (int s = lane; s < n; s += kWave) m = fmaxf(m, a.rec[a.rec_ml + 2 * (s * stride + at)]);
  m = wave_max(m);
  const float base = m == -INFINITY ? 0.0f : m;
  float l = 0.0f, o[E] = {};
  for (int s = 0; s < n; ++s) {
    const int64_t i = s * stride + at;
    const float w = __builtin_amdgcn_exp2f(a.rec[a.rec_ml + 2 * i] - base);
    l += w * a.rec[a.rec_ml + 2 * i + 1];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += w * a.rec[i * D + lane * E + e];
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  unsigned char *out = a.out + (token * a.o_token + head * a.o_head) * (int64_t)sizeof(T);
#pragma unroll
  for (int e = 0; e < E; ++e) elem<T>::store1(out, lane * E + e, o[e] * inv);
  if (a.lse && lane == 0)
    a.lse[(int64_t)token * a.hq + head] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

template <typename T, int D, int NW, bool PRIV, int BN>
hipError_t launch_form(AttnArgs a, int tiles, int span, int n_split, float *rec, hipStream_t st) {
  constexpr int BM = PRIV ? 32 : NW * 32;
  a.span = span;
  a.n_split = n_split;
  a.rec = rec;
  a.rec_ml = (int64_t)n_split * tiles * a.hkv * BM * D;
  hipLaunchKernelGGL((chunk_attn<T, D, NW, PRIV, BN>), dim3(tiles * a.hkv, n_split), dim3(NW * kWave), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || n_split == 1) return e;
  hipLaunchKernelGGL((chunk_merge<T, D, PRIV, BM>), dim3(tiles * a.hkv, BM / 4), dim3(4 * kWave), 0, st, a);
  return hipGetLastError();
}

template <typename T, int D> hipError_t launch_typed(AttnArgs a, const AttnPlan &p, float *ws, hipStream_t st) {
  constexpr bool h = sizeof(T) == 2;
  if (p.many_tiles) {
    const hipError_t e = launch_form<T, D, kAttnWaves, false, h ? 64 : 32>(a, p.many_tiles, p.many_span, p.many_split, ws, st);
    if (e != hipSuccess) return e;
  }
  if (!p.few_tiles) return hipSuccess;
  return launch_form<T, D, h ? 4 : 2, true, 32>(a, p.few_tiles, p.few_span, p.few_split,
                                                ws + p.many_bytes / sizeof(float), st);
}

int ceil_div(int64_t x, int64_t y) { return (int)((x + y - 1) / y); }

}  // namespace

AttnPlan plan_chunk_attn(const smallkv_chunk_t &c, const smallkv_cache_t &kv, const smallkv_queries_t &q) {
  AttnPlan p{};
  const int g = q.n_heads / kv.n_heads;
  const int64_t rows = (int64_t)c.max_new * g;
  constexpr int kBm = kAttnWaves * 32;
  p.use_few = rows <= 32 || c.batch > 1;
  if (p.use_few) {
    // a workgroup per CU; spans of whole rounds of the waves' tiles
    const int round = kv.dtype == SMALLKV_F32 ? 64 : 128;
    p.few_tiles = c.batch;
    const int64_t units = (int64_t)c.batch * kv.n_heads;
    const int want = units >= 512 ? 1 : ceil_div(512, units);
    p.few_span = ceil_div(ceil_div(c.max_len, want), round) * round;
    p.few_split = ceil_div(c.max_len, p.few_span);
  }
  if (rows > 32) {
    const int64_t per = ceil_div(rows, kBm);
    p.many_tiles = (int)std::min<int64_t>(c.batch * per, (int64_t)c.n_tokens * g / kBm + c.batch);
    const int64_t units = (int64_t)p.many_tiles * kv.n_heads;
    const int want = units >= 384 ? 1 : ceil_div(512, units);
    p.many_span = ceil_div(ceil_div(c.max_len, want), 256) * 256;
    p.many_split = ceil_div(c.max_len, p.many_span);
  }
  const int64_t d2 = (kv.head_dim + 2) * (int64_t)sizeof(float);
  if (p.many_split > 1) p.many_bytes = (size_t)p.many_split * p.many_tiles * kv.n_heads * kBm * d2;
  p.ws_bytes = p.many_bytes;
  if (p.few_split > 1) p.ws_bytes += (size_t)p.few_split * p.few_tiles * kv.n_heads * 32 * d2;
  return p;
}

hipError_t launch_chunk_attn(const smallkv_chunk_t &c, const smallkv_cache_t &kv, const smallkv_queries_t &q,
                             const AttnPlan &p, void *ws, hipStream_t st) {
  if (c.n_tokens == 0) return hipSuccess;
  AttnArgs a{};
  a.c = chunk_view(c);
  a.kv = cache_view(kv);
  a.hq = q.n_heads;
  a.hkv = kv.n_heads;
  a.g = q.n_heads / kv.n_heads;
  a.q = static_cast<const unsigned char *>(q.q);
  a.q_token = q.token_stride;
  a.q_head = q.head_stride;
  a.out = static_cast<unsigned char *>(q.out);
  a.o_token = q.out_token_stride;
  a.o_head = q.out_head_stride;
  a.lse = q.lse;
  a.scale2 = (float)(q.scale * kLog2e);
  a.scale2_lo = (float)(q.scale * kLog2e - a.scale2);
  a.few = p.use_few;
  float *rec = static_cast<float *>(ws);
  if (kv.dtype == SMALLKV_F32)
    return kv.head_dim == 64 ? launch_typed<float, 64>(a, p, rec, st) : launch_typed<float, 128>(a, p, rec, st);
  return kv.head_dim == 64 ? launch_typed<bf16_t, 64>(a, p, rec, st) : launch_typed<bf16_t, 128>(a, p, rec, st);
}

}  // namespace smallkv
