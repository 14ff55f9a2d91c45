// What the attention kernels over plain and packed caches share: the tiles of a batch
// and the spans of its rows, the logits, the running softmax and the product with the
// values from tiles in LDS, the rows' output, and the join of the spans.
#pragma once

#include <algorithm>
#include <type_traits>

#include "launch.h"
#include "packed.h"

namespace smallkv {
namespace {

__device__ __align__(16) unsigned char zero_row[512];  // absent rows are read from here

struct AttnArgs {
  ChunkView c;
  CacheView kv;   // a packed cache's codes
  ScaleView sc;   // and their scales
  int hq, hkv, g;
  const unsigned char *q;
  unsigned char *out;
  int64_t q_token, q_head, o_token, o_head;  // in elements
  float *lse;     // [n_tokens][hq] or null
  float scale2, scale2_lo;  // scale * log2(e), and what its rounding left
  int single;     // no spans, and a tile per sequence
  int splits;     // (tile, span) units that may run at once, per kv head; 0: no spans
  float *rec;     // [unit * hkv][rows][D] fp32, then [unit * hkv][rows][2]
  int64_t rec_ml; // where the second array starts, in floats
  int *span;      // the span, for attn_merge
  int parts;      // of a row's spans in attn_merge, a power of two
};

constexpr double kLog2e = 1.4426950408889634074;
constexpr float kLn2 = 0.693147180559945309417f;

// Steps of the many-rows form's spans (whole tiles), and the shortest in steps.  (179
// tokens over 23719 rows: 86.6 us, 88.9 in steps of 256; 16 over 8192: 25.5 us, 24.1 and
// twice the records with 128 as the shortest.)
constexpr int kManyRound = 64, kManyLeast = 4;
constexpr int kWhole = 1 << 30;  // a span no sequence is longer than

// A tile of rows: its sequence, first row and the sequence's rows; the span's
// number, the spans of its rows and the tile's first unit.
struct Tile {
  int b, row0, rows, split, n_split, unit0;
  Seq s;
};

// Spans of a sequence's rows: at least one, so that rows that see no key are written.
__device__ __forceinline__ int spans_of(int len, int span) {
  return span == kWhole ? 1 : max((len + span - 1) / span, 1);
}

// The sequences of a batch, one per lane: the first 64 stay in registers, the others
// are read again by every pass.
template <int BM> struct Lanes {
  Seq s0;

  __device__ __forceinline__ static Seq read(const AttnArgs &a, int b) {
    return b < a.c.batch ? sequence(a.c, b, a.kv.cap) : Seq{0, 0, 0};
  }
  __device__ __forceinline__ explicit Lanes(const AttnArgs &a) : s0(read(a, threadIdx.x & (kWave - 1))) {}
  __device__ __forceinline__ static int tiles(const AttnArgs &a, const Seq &s) {
    return (s.n_new * a.g + BM - 1) / BM;
  }
  template <typename F> __device__ __forceinline__ void each(const AttnArgs &a, F &&use) const {
    for (int b0 = 0; b0 < a.c.batch; b0 += kWave) {
      const Seq s = b0 ? read(a, b0 + (int)(threadIdx.x & (kWave - 1))) : s0;
      if (use(b0, s, tiles(a, s))) return;
    }
  }
};

// The shortest span, in steps of `round` rows and of at least `least` of them, with
// which all units fit `splits`; kWhole where the tiles alone do not.
template <int BM>
__device__ __forceinline__ int find_span(const AttnArgs &a, const Lanes<BM> &lanes, int round, int least) {
  if (!a.splits) return kWhole;
  int tiles = 0, longest = 0;
  float work = 0.0f;  // cached rows over all tiles, in steps of `round`
  lanes.each(a, [&](int, const Seq &s, int n) {
    tiles += last_lane(wave_scan(n));
    const float steps = n ? (float)((s.len + round - 1) / round) : 0.0f;
    longest = max(longest, (int)wave_max(steps));
    work += wave_sum((float)n * steps);
    return false;
  });
  if (tiles >= a.splits) return kWhole;
  // between work / splits, and work / (splits - tiles): there they fit for sure
  int lo = max((int)(work / (float)a.splits), least), hi = max(min((int)(work / (float)(a.splits - tiles)) + 2, longest), lo);
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    int units = 0;
    lanes.each(a, [&](int, const Seq &s, int n) {
      units += last_lane(wave_scan(n * spans_of(s.len, mid * round)));
      return false;
    });
    if (units <= a.splits)
      hi = mid;
    else
      lo = mid + 1;
  }
  return __builtin_amdgcn_readfirstlane(lo) * round;
}

// Units (or tiles) are numbered sequence by sequence, tile by tile and span by span;
// the last rows of a sequence, which see the most keys, come first.
template <int BM, bool UNITS>
__device__ __forceinline__ bool locate(const AttnArgs &a, const Lanes<BM> &lanes, int span, int flat, Tile &t) {
  int unit = 0;  // of the sequences before
  bool found = false;
  lanes.each(a, [&](int b0, const Seq &s, int n) {
    const int ns = spans_of(s.len, span);
    const int units = wave_scan(n * ns), x = UNITS ? units : wave_scan(n);
    const uint64_t m = __ballot(x > flat);
    if (!m) {
      flat -= last_lane(x);
      unit += last_lane(units);
      return false;
    }
    const int l = __builtin_amdgcn_readfirstlane(__ffsll((long long)m) - 1);
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
    const int tiles = of(n);
    t.b = b0 + l;
    t.s = Seq{of(s.first), of(s.n_new), of(s.len)};
    t.n_split = of(ns);
    const int per = UNITS ? t.n_split : 1, in = flat - (of(x) - tiles * per), tile = in / per;
    t.split = in - tile * per;
    t.unit0 = unit + of(units) - (tiles - tile) * t.n_split;
    t.row0 = (tiles - 1 - tile) * BM;
    t.rows = t.s.n_new * a.g;
    found = true;
    return true;
  });
  return found;
}

// A wave's share of the copies of one tile of rows.  The page of the lane's row is
// looked up a tile ahead (without a branch: the value must not be needed before
// then); the rows' offsets are then passed between lanes.
template <typename L, int BN, int SHARE> struct Loader {
  static constexpr int kRpi = 64 / L::C;        // rows per instruction
  static constexpr int kInstr = SHARE / kRpi;   // instructions per wave, K or V
  static_assert(SHARE % kRpi == 0 && kInstr >= 1, "a wave copies whole instructions");
  const int32_t *pages;  // of the sequence (dense: any readable word)
  int len, page;         // rows from `len` on do not exist; the looked-up page

  __device__ __forceinline__ void init(const AttnArgs &a, int b, int end) {
    pages = a.kv.table ? a.kv.table + (int64_t)b * a.kv.width : a.c.len;
    len = end;
  }
  __device__ __forceinline__ void lookup(const CacheView &kv, int row0) {
    const int row = row0 + (int)(threadIdx.x & (BN - 1));
    page = pages[max(min(row, len - 1), 0) >> kv.shift];  // (dense: shift 31)
  }
  // Offset of the lane's row of the looked-up tile, or -1.
  __device__ __forceinline__ int64_t offset(const CacheView &kv, int b, int row0) const {
    const int row = row0 + (int)(threadIdx.x & (BN - 1));
    const int64_t off = page_offset(kv, kv.table ? page : b, row);
    return row < len ? off : -1;
  }
  __device__ __forceinline__ static int64_t pass(int64_t off, int from) {
    const int lo = __shfl((int)off, from, kWave), hi = __shfl((int)(off >> 32), from, kWave);
    return ((int64_t)hi << 32) | (uint32_t)lo;
  }
  // The lane's row of an instruction and piece of a row; ANEW: computed each time
  // (kept, the addresses of the few-rows form's 16 instructions would take 32 registers).
  template <bool ANEW> __device__ __forceinline__ static void place(int &rr, int &p) {
    int lane = threadIdx.x & (kWave - 1);
    if (ANEW) asm volatile("" : "+v"(lane));
    rr = lane / L::C;
    p = lane & (L::C - 1);
  }
  // Rows first..first+SHARE-1 of the tile; sk, sv: the tile's start in LDS.
  __device__ __forceinline__ static void issue(int64_t off, const unsigned char *k, const unsigned char *v, int first,
                                               unsigned char *sk, unsigned char *sv) {
    int rr, p;
    place<false>(rr, p);
#pragma unroll
    for (int j = 0; j < kInstr; ++j) {
      const int r = first + j * kRpi + rr;
      const int64_t o = pass(off, r);
      load_to_lds16((o < 0 ? zero_row : k + o) + ((p ^ L::swz_k(r)) << 4), sk + (first + j * kRpi) * L::bytes);
      load_to_lds16((o < 0 ? zero_row : v + o) + ((p ^ L::swz_v(r)) << 4), sv + (first + j * kRpi) * L::bytes);
    }
  }
  // The same for all rows, keys or values only.
  template <bool VALUES>
  __device__ __forceinline__ static void issue_one(int64_t off, const unsigned char *base, unsigned char *lds) {
    int rr, p;
    place<true>(rr, p);
#pragma unroll
    for (int j = 0; j < kInstr; ++j) {
      const int r = j * kRpi + rr;
      const int64_t o = pass(off, r);
      load_to_lds16((o < 0 ? zero_row : base + o) + ((p ^ (VALUES ? L::swz_v(r) : L::swz_k(r))) << 4),
                    lds + j * kRpi * L::bytes);
    }
  }
};

// fp32 as a sum of three bf16 numbers (exactly, but for what lies below 2^-133), or as two
// with an error of 2^-17 of it; infinities in the first.  NaN in all (cut off, one that only
// bits below bf16's tell from an infinity is that infinity).
template <int PARTS> __device__ __forceinline__ void split(float x, float (&y)[PARTS]) {
  y[0] = bf16_hi(__float_as_uint(x));
  float rest = fabsf(x) == INFINITY ? 0.0f : x - y[0];
#pragma unroll
  for (int i = 1; i + 1 < PARTS; ++i) {
    y[i] = bf16_hi(__float_as_uint(rest));
    rest -= y[i];
  }
  if (PARTS > 1) y[PARTS - 1] = rest;
}

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

template <int D> struct QFrag<wide_t, D> {
  // (the last part of 128 elements waits in LDS: registers for two waves per SIMD)
  static constexpr int kKept = D == 128 ? 2 : 3, kLds = (3 - kKept) * D / 16;
  bf16x8_t f[kKept][D / 16];
  const bf16x8_t *rest;
  // lds: kLds * 64 pieces of the wave's own
  __device__ __forceinline__ void load(const unsigned char *row, int half, bf16x8_t *lds) {
    rest = lds + (threadIdx.x & (kWave - 1));
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      bf16x8_t x[3];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float y[3];
        split<3>(reinterpret_cast<const float *>(row)[s * 16 + half * 8 + e], y);
#pragma unroll
        for (int p = 0; p < 3; ++p) x[p][e] = (__bf16)y[p];
      }
#pragma unroll
      for (int p = 0; p < kKept; ++p) f[p][s] = x[p];
      if (kKept < 3) lds[s * kWave + (threadIdx.x & (kWave - 1))] = x[2];
    }
  }
  template <int P> __device__ __forceinline__ bf16x8_t part(int i) const {
    if constexpr (P < kKept)
      return f[P][i];
    else
      return rest[i * kWave];
  }
};

// S^T of 32 keys (rows key0 .. of the tile) and the wave's 32 query rows.
template <typename T, int D>
__device__ __forceinline__ f32x16_t logits32(const unsigned char *sk, int key0, const QFrag<T, D> &q) {
  using L = TileLayout<T, D>;
  const int lane = threadIdx.x & (kWave - 1), r = key0 + (lane & 31), half = lane >> 5;
  const unsigned char *row = sk + r * L::bytes;
  const int z = L::swz_k(r);
  if constexpr (std::is_same_v<T, wide_t>) {
    f32x16_t s = {};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const bf16x8_t k = *reinterpret_cast<const bf16x8_t *>(row + (((2 * i + half) ^ z) << 4));
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q.template part<2>(i), s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q.template part<1>(i), s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q.template part<0>(i), s, 0, 0, 0);
    }
    return s;
  } else if constexpr (sizeof(T) == 2) {
    f32x16_t s = {};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const bf16x8_t k = *reinterpret_cast<const bf16x8_t *>(row + (((2 * i + half) ^ z) << 4));
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q.f[i], s, 0, 0, 0);
    }
    return s;
  } else {
    // the head dimension in two halves, a half-wave each, and two sums: a chain
    // of D / 4 roundings instead of D, and independent instructions (four would leave
    // registers for one wave per SIMD: 256 tokens over 4096 rows of 8 kv heads 189 us,
    // with two 166)
    f32x16_t s[2] = {};
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const f32x4_t k = *reinterpret_cast<const f32x4_t *>(row + (((half * (D / 8) + i) ^ z) << 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e & 1] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], q.f[i][e], s[e & 1], 0, 0, 0);
    }
    return s[0] + s[1];
  }
}

// Key of register i of a 32-key block, before the half-wave's 4 * half.
__device__ __forceinline__ constexpr int reg_key(int i) { return 8 * (i / 4) + i % 4; }

template <typename T, int D> struct State {
  float m, l;  // running maximum (log2 units), this half-wave's part of the sum
  float r;     // and of the sum of P as it was rounded (many rows, bf16)
  f32x16_t o[D / 32];
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = r = 0.0f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) o[d] = f32x16_t{};
  }
};

// O^T += V^T P^T over 32 keys.  TWO: a bf16 model's P in two parts, a product each;
// without, one rounded part, whose sum is kept too.
template <typename T, int D, bool TWO, typename L = TileLayout<T, D>>
__device__ __forceinline__ void values32(const unsigned char *sv, int key0, const f32x16_t &p, State<T, D> &st) {
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  if constexpr (std::is_same_v<T, wide_t>) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8_t pf[3];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float y[3];
        split<3>(p[8 * s + e], y);
#pragma unroll
        for (int x = 0; x < 3; ++x) pf[x][e] = (__bf16)y[x];
      }
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        union { s16x4_t h[2]; bf16x8_t v; } vf;
#pragma unroll
        for (int x = 0; x < 2; ++x) {  // (as below)
          const int r = key0 + 16 * s + 8 * x + 4 * half + ((lane & 15) >> 2);
          const int c = d * 4 + ((lane & 31) >> 4) * 2 + ((lane & 3) >> 1);
          const int at = r * L::bytes + ((c ^ L::swz_v(r)) << 4) + (lane & 1) * 8;
          vf.h[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SMALLKV_LDS s16x4_t *)(sv + at));
        }
#pragma unroll
        for (int x = 2; x >= 0; --x) st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.v, pf[x], st.o[d], 0, 0, 0);
      }
    }
  } else if constexpr (sizeof(T) == 2) {
    const bf16x2_t ones = {(__bf16)1.0f, (__bf16)1.0f};
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8_t pf, lo;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        bf16x2_t w, y;
        if constexpr (TWO) {
          // the first part is cut off and the second never 0, so that an infinite value
          // times either is the same infinity
          const uint32_t u0 = __float_as_uint(p[8 * s + e]), u1 = __float_as_uint(p[8 * s + e + 1]);
          w = __builtin_bit_cast(bf16x2_t, __builtin_amdgcn_perm(u1, u0, 0x07060302));
          const float y0 = __builtin_fmaf(p[8 * s + e], 0x1p-24f, p[8 * s + e] - bf16_hi(u0));
          const float y1 = __builtin_fmaf(p[8 * s + e + 1], 0x1p-24f, p[8 * s + e + 1] - bf16_hi(u1));
          y = __builtin_convertvector((f32x2_t{y0, y1}), bf16x2_t);
          lo[e] = y[0];
          lo[e + 1] = y[1];
        } else {
          w = __builtin_convertvector((f32x2_t{p[8 * s + e], p[8 * s + e + 1]}), bf16x2_t);
          sum = __builtin_amdgcn_fdot2_f32_bf16(w, ones, sum, false);
        }
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
          // (one addition: the compiler follows an LDS array through few of them, and
          // does not hold these reads up for copies into other arrays while it does)
          const int at = r * L::bytes + ((c ^ L::swz_v(r)) << 4) + (lane & 1) * 8;
          vf.h[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SMALLKV_LDS s16x4_t *)(sv + at));
        }
        st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.v, pf, st.o[d], 0, 0, 0);
        if constexpr (TWO) st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.v, lo, st.o[d], 0, 0, 0);
      }
    }
    if (!TWO) st.r += sum;
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = key0 + reg_key(i) + 4 * half;
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        const int c = d * 8 + ((lane & 31) >> 2);
        const float v = *reinterpret_cast<const float *>(sv + r * L::bytes + ((c ^ L::swz_v(r)) << 4) + (lane & 3) * 4);
        st.o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[i], st.o[d], 0, 0, 0);
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
    st.r *= f;
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
template <typename T, int D, int BN, typename L = TileLayout<T, D>>
__device__ __forceinline__ void full_tile(State<T, D> &st, const QFrag<T, D> &q, const unsigned char *sk,
                                          const unsigned char *sv, float c, float c_lo) {
  f32x16_t s[BN / 32];
#pragma unroll
  for (int b = 0; b < BN / 32; ++b) s[b] = logits32<T, D>(sk, 32 * b, q);
  softmax_step<T, D>(st, s, c, c_lo);
#pragma unroll
  for (int b = 0; b < BN / 32; ++b) values32<T, D, false, L>(sv, 32 * b, s[b], st);
}

// Any other, 32 keys at a time.  own: the lane's own row; highest: of the wave's; valid:
// bit t set iff key row0 + t exists.
template <typename T, int D, int BN, bool TWO, typename L = TileLayout<T, D>>
__device__ __forceinline__ void masked_tile(State<T, D> &st, const QFrag<T, D> &q, const unsigned char *sk,
                                            const unsigned char *sv, int row0, int own, int highest,
                                            uint64_t valid, float c, float c_lo) {
  const int half = (threadIdx.x & (kWave - 1)) >> 5;
#pragma unroll 1
  for (int k0 = 0; k0 < BN && row0 + k0 <= highest; k0 += 32) {
    f32x16_t s[1] = {logits32<T, D>(sk, k0, q)};
    const uint32_t bits = (uint32_t)(valid >> k0) >> (4 * half);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const bool ok = (bits >> reg_key(i) & 1u) && row0 + k0 + reg_key(i) + 4 * half <= own;
      s[0][i] = ok ? s[0][i] : -INFINITY;
    }
    softmax_step<T, D>(st, s, c, c_lo);
    values32<T, D, TWO, L>(sv, k0, s[0], st);
  }
}

// A workgroup's share of the work, and the lane's row of it.
template <int BM> struct Share {
  Tile t;
  int kvh, unit, begin, end;  // kv head; unit and kv head; the span's cached rows
  int r, token, head, own;    // the lane's row, its cached row (-1: past the last)
  int first_own;              // cached row of the workgroup's first row
  bool live;
  const unsigned char *k, *v; // of the kv head

  // Row `at` of the sequence as the lane's own.
  __device__ __forceinline__ void row(const AttnArgs &a, int at) {
    r = at;
    live = r < t.rows;
    const int rc = live ? r : t.rows - 1;
    token = t.s.first + rc / a.g;
    head = kvh * a.g + rc % a.g;
    own = live ? t.s.len - t.s.n_new + rc / a.g : -1;
  }

  // The share of unit `flat` and a kv head.
  __device__ __forceinline__ bool find(const AttnArgs &a, int flat, int kv_head, int round, int least, int wave_row) {
    kvh = kv_head;
    int span = kWhole;
    if (BM <= 32 && a.single) {
      // no spans and a tile per sequence: many sequences, not searched one by one
      t.b = flat;
      if (flat >= a.c.batch) return false;
      t.s = sequence(a.c, t.b, a.kv.cap);
      t.rows = t.s.n_new * a.g;
      t.row0 = t.split = t.unit0 = 0;
      t.n_split = 1;
      if (t.rows == 0) return false;
    } else {
      const Lanes<BM> lanes(a);
      span = find_span<BM>(a, lanes, round, least);
      if (a.splits && flat == 0 && kvh == 0 && threadIdx.x == 0) *a.span = span;
      if (!locate<BM, true>(a, lanes, span, flat, t)) return false;
    }
    unit = flat * a.hkv + kvh;
    const int pos0 = t.s.len - t.s.n_new;  // cached row of the first new token
    const int last = min(t.row0 + BM, t.rows) - 1;
    const int limit = max(pos0 + last / a.g + 1, 0);  // keys the tile's rows see (<= len)
    begin = t.split * span;  // (one span: 0)
    end = min(limit, begin + span);
    if (begin >= limit && t.split > 0) return false;  // (attn_merge reads no record of it)
    row(a, t.row0 + wave_row + (int)(threadIdx.x & (BM < 32 ? BM - 1 : 31)));
    first_own = pos0 + t.row0 / a.g;
    k = a.kv.k + (((uint64_t)kvh * a.kv.head_stride) << 4);
    v = a.kv.v + (((uint64_t)kvh * a.kv.head_stride) << 4);
    return true;
  }
};

// Adds the infinite and NaN values of keys from..to, times their weights, to the lane's own
// elements (groups of W, `step` apart from `at` on) of an output row that is written
// already: a weight > 0 leaves them what they are, and a logit of -inf, weight 0, makes
// them NaN, as the matrix product does in a tile that nothing is taken out of.
// (F: the bits of a packed cache's codes, 0 for a plain one.)
template <typename O, typename T, int D, int W, int BM, int F>
__device__ __forceinline__ void give_back(const AttnArgs &a, const Share<BM> &w, void *out, int from, int to, int at,
                                          int step) {
#pragma unroll 1
  for (int key = from; key <= to; ++key) {
    const int64_t off = row_offset(a.kv, w.t.b, key);
    if (off < 0) continue;
    const int64_t so = F ? scale_offset<D>(a.sc, a.kv, row_page(a.kv, w.t.b, key), key, w.kvh) : 0;
    bool none = false, known = false;
#pragma unroll 1
    for (int e0 = at; e0 < D; e0 += step)
#pragma unroll 1
      for (int e = e0; e < e0 + W; ++e) {
        const float x = cached<T, F>(w.v + off, a.sc.v + so, e);
        if (fabsf(x) <= 3.402823466e38f) continue;
        if (!known) {
          const unsigned char *q = a.q + (w.token * a.q_token + w.head * a.q_head) * (int64_t)sizeof(T);
          float s = 0.0f;
#pragma unroll 1
          for (int i = 0; i < D; ++i)
            s = __builtin_fmaf(elem<T>::load1(q, i), cached<T, F>(w.k + off, a.sc.k + so, i), s);
          none = s == -INFINITY;
          known = true;
        }
        elem<O>::store1(out, e, none ? NAN : elem<O>::load1(out, e) + x);
      }
  }
}

// The lane's part of a row of the output, or of the span's record: N groups of four
// elements of o, `step` apart from `at` on, l the row's sum.  writes: one lane per row;
// taken: values were taken out of a tile of BN keys.
template <typename T, int D, int BM, int BN, int F = 0, int N>
__device__ __forceinline__ void write_row(const AttnArgs &a, const Share<BM> &w, const f32x4_t (&x)[N], float m, float l,
                                          int at, int step, bool writes, bool taken) {
  const int from = max(w.begin, w.first_own + 2 - BN), to = min(w.end - 1, w.own);
  if (w.t.n_split > 1) {
    const int64_t row = (int64_t)w.unit * BM + (w.r - w.t.row0);
    float *o = a.rec + row * D;
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<f32x4_t *>(o + at + i * step) = x[i];
    if (writes) {
      a.rec[a.rec_ml + 2 * row] = m;
      a.rec[a.rec_ml + 2 * row + 1] = l;
    }
    if (taken) give_back<float, T, D, 4, BM, F>(a, w, o, from, to, at, step);
    return;
  }
  const bool none = l == 0.0f;  // the row sees no key, or only logits of -inf
  const float inv = 1.0f / l;
  unsigned char *o = a.out + (w.token * a.o_token + w.head * a.o_head) * (int64_t)sizeof(T);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const f32x4_t y = none ? f32x4_t{} : x[i] * inv;
    if constexpr (sizeof(T) == 4)
      *reinterpret_cast<f32x4_t *>(o + (at + i * step) * 4) = y;
    else
      *reinterpret_cast<bf16x4_t *>(o + (at + i * step) * 2) = __builtin_convertvector(y, bf16x4_t);
  }
  if (taken && !none) give_back<T, T, D, 4, BM, F>(a, w, o, from, to, at, step);
  if (a.lse && writes)
    a.lse[(int64_t)w.token * a.hq + w.head] = none ? -INFINITY : (m + __log2f(l)) * kLn2;
}

template <typename T, int D, int BM, int BN, bool TWO, int F = 0>
__device__ __forceinline__ void write_row(const AttnArgs &a, const Share<BM> &w, const State<T, D> &st, bool taken) {
  // `rounded`: where one rounded P was multiplied its own sum divides the output, so
  // that the weights add up to 1 (a record holds the output times l / rounded)
  const float l = swap_halves_sum(st.l), rounded = sizeof(T) == 2 && !TWO ? swap_halves_sum(st.r) : l;
  const int half = (threadIdx.x & (kWave - 1)) >> 5;
  if (sizeof(T) == 2 && w.t.n_split == 1) {
    // half-waves exchange four elements of 16, so that each lane writes eight at once
    const bool none = l == 0.0f;
    const float inv = 1.0f / rounded;
    unsigned char *o = a.out + (w.token * a.o_token + w.head * a.o_head) * 2;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      uint32_t y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = j % 2 * 8 + 2 * i;
        const f32x2_t v = none ? f32x2_t{} : f32x2_t{st.o[j / 2][e] * inv, st.o[j / 2][e + 1] * inv};
        y[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
      }
      const auto p = __builtin_amdgcn_permlane32_swap(y[0], y[2], false, false);
      const auto q = __builtin_amdgcn_permlane32_swap(y[1], y[3], false, false);
      if (w.live) *reinterpret_cast<uint4 *>(o + j * 32 + half * 16) = make_uint4(p[0], q[0], p[1], q[1]);
    }
    if (!w.live) return;
    if (taken && !none)
      give_back<T, T, D, 8, BM, F>(a, w, o, max(w.begin, w.first_own + 2 - BN), min(w.end - 1, w.own), 8 * half, 16);
    if (a.lse && half == 0)
      a.lse[(int64_t)w.token * a.hq + w.head] = none ? -INFINITY : (st.m + __log2f(l)) * kLn2;
    return;
  }
  if (!w.live) return;
  const float f = sizeof(T) == 2 && !TWO && l != 0.0f ? l / rounded : 1.0f;
  f32x4_t x[D / 8];
#pragma unroll
  for (int i = 0; i < D / 8; ++i)
    x[i] = f32x4_t{st.o[i / 4][i % 4 * 4], st.o[i / 4][i % 4 * 4 + 1], st.o[i / 4][i % 4 * 4 + 2], st.o[i / 4][i % 4 * 4 + 3]} * f;
  write_row<T, D, BM, BN, F>(a, w, x, st.m, l, 4 * half, 8, half == 0, taken);
}

// Infinite and NaN values of a tile are taken out of it where some row does not see
// some key, since 0 * inf or 0 * NaN would reach that row through the matrix
// product; write_row gives them to the rows that see them.
template <typename T, int N> __device__ __forceinline__ bool take_out(unsigned char *sv, int first, int step) {
  bool found = false;
  for (int i = first; i < N; i += step) {
    uint4 w = reinterpret_cast<uint4 *>(sv)[i];
    if (drop_not_finite<T>(w)) {
      reinterpret_cast<uint4 *>(sv)[i] = w;
      found = true;
    }
  }
  return found;
}

// Waits until at most N of this wave's copies and loads are outstanding.
template <int N> __device__ __forceinline__ void wait_copies() {
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4 | 15 << 8);
  asm volatile("" ::: "memory");
}
// Waits for this wave's LDS reads.
__device__ __forceinline__ void wait_lds() {
  __builtin_amdgcn_s_waitcnt(15 | 3 << 14 | 7 << 4);
  asm volatile("" ::: "memory");
}

constexpr int kFewWaves = 4;

// Joins the states of NW waves in wave 0: the upper half hands over to the lower one.
// x: NW / 2 * (D / 2) * 64 floats, ml: the waves' maxima and sums.
template <typename T, int D, int NW>
__device__ __forceinline__ void join_waves(State<T, D> &st, float *x, float (&ml)[2][NW / 2][kWave]) {
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
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
}

// Joins the records of a tile's spans: four elements of a row per lane, and a row's
// spans dealt to `parts` groups of such lanes, which each take theirs in one pass with
// the running maximum and are joined in LDS.
constexpr int kMaxParts = 32;

template <typename T, int D, int BM>
__global__ __launch_bounds__(kMaxParts * (D / 4)) void attn_merge(AttnArgs a) {
  constexpr int W = D / 4;  // lanes of a row
  __shared__ f32x4_t so[kMaxParts * W];
  __shared__ float2 sml[kMaxParts];
  const int kvh = blockIdx.x % a.hkv, span = *a.span;
  const Lanes<BM> lanes(a);
  Tile t;
  if (span == kWhole || !locate<BM, false>(a, lanes, span, blockIdx.x / a.hkv, t) || t.n_split == 1) return;
  const int group = threadIdx.x / W, e = threadIdx.x % W * 4;
  const int n_rows = blockDim.x / W / a.parts, part = group / n_rows;
  const int in = blockIdx.y * n_rows + group % n_rows, r = t.row0 + in;
  const int own = t.s.len - t.s.n_new + r / a.g;
  const int token = t.s.first + r / a.g, head = kvh * a.g + r % a.g;
  // spans that hold a row this one sees; the others wrote nothing it needs
  const int n = r >= t.rows || own < 0 ? 0 : min(own / span + 1, t.n_split);
  const int64_t stride = (int64_t)a.hkv * BM, at = ((int64_t)t.unit0 * a.hkv + kvh) * BM + in;
  const float *ml = a.rec + a.rec_ml + 2 * at, *rec = a.rec + at * D + e;
  float m = -INFINITY, l = 0.0f;
  f32x4_t o = {};
  auto join = [&](float2 x, const f32x4_t &v) {
    const float top = fmaxf(m, x.x), base = top == -INFINITY ? 0.0f : top;
    const float f = __builtin_amdgcn_exp2f(m - base), w = __builtin_amdgcn_exp2f(x.x - base);
    m = top;
    l = l * f + x.y * w;
    o = o * f + v * w;
  };
  const int count = n > part ? (n - part - 1) / a.parts + 1 : 0;
  const int64_t step = stride * a.parts;
  ml += 2 * part * stride;
  rec += part * stride * D;
#pragma unroll 8
  for (int s = 0; s < count; ++s)
    join(*reinterpret_cast<const float2 *>(ml + 2 * s * step), *reinterpret_cast<const f32x4_t *>(rec + s * step * D));
  if (a.parts > 1) {
    so[threadIdx.x] = o;
    if (e == 0) sml[group] = make_float2(m, l);
    __syncthreads();
    if (part == 0)
      for (int g = group + n_rows; g < n_rows * a.parts; g += n_rows) join(sml[g], so[g * W + threadIdx.x % W]);
  }
  if (part > 0 || r >= t.rows) return;
  const f32x4_t x = l == 0.0f ? f32x4_t{} : o * (1.0f / l);
  unsigned char *out = a.out + (token * a.o_token + head * a.o_head) * (int64_t)sizeof(T);
  if constexpr (sizeof(T) == 4)
    *reinterpret_cast<f32x4_t *>(out + e * 4) = x;
  else
    *reinterpret_cast<bf16x4_t *>(out + e * 2) = __builtin_convertvector(x, bf16x4_t);
  if (a.lse && e == 0)
    a.lse[(int64_t)token * a.hq + head] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// As many parts per row as there can be spans, and all lanes run at once (256 CUs
// of 2048 lanes).  (One token over 32768 rows of 4 kv heads, 128 spans: 39.5 us
// with one part, 7.9 with 32.)  Set before the kernel that writes the records.
struct MergeShape {
  int threads, n_rows;
};
template <int D> MergeShape merge_shape(AttnArgs &a, const AttnPlan &p) {
  const int64_t lanes = (int64_t)p.tiles * a.hkv * p.rows * (D / 4);
  a.parts = 1;
  while (a.parts < kMaxParts && a.parts < p.splits - p.tiles && 2 * a.parts * lanes <= 256 * 2048) a.parts *= 2;
  const int threads = std::max(a.parts * (D / 4), 256);
  a.rec_ml = (int64_t)p.units * a.hkv * p.rows * D;
  return {threads, threads / (D / 4) / a.parts};
}
template <typename T, int D, int BM>
void launch_merge(const AttnArgs &a, const AttnPlan &p, const MergeShape &m, hipStream_t st) {
  hipLaunchKernelGGL((attn_merge<T, D, BM>), dim3(p.tiles * a.hkv, p.rows / m.n_rows), dim3(m.threads), 0, st, a);
}

constexpr size_t kSpanBytes = 256;  // before the records

inline int ceil_div(int64_t x, int64_t y) { return (int)((x + y - 1) / y); }

// Host: a call's arguments, but for the scales of a packed cache.
inline AttnArgs attn_args(const smallkv_chunk_t &c, const smallkv_cache_t &kv, const smallkv_queries_t &q,
                          const AttnPlan &p, void *ws) {
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
  a.splits = p.splits;
  a.single = p.few && !p.splits && p.tiles <= c.batch;
  a.span = static_cast<int *>(ws);
  if (ws) a.rec = reinterpret_cast<float *>(static_cast<char *>(ws) + kSpanBytes);
  return a;
}

}  // namespace
}  // namespace smallkv
