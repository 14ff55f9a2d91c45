// Attention of the new tokens over a packed cache: the sums of smallkv_chunk_attn,
//   s_t = scale * <q, K_t>,  out = softmax(s) V,  lse = ln sum exp(s),
// in one pass over rows of 8- or 4-bit codes.  A code times its block's power of two has few
// enough bits for bf16, so both products run on bf16 operands and lose nothing of K and V; an
// fp32 model's queries and probabilities take three bf16 parts, a product each, which hold all
// 24 bits (on fp32 operands a 4096-token prompt of 32 heads took 1326 us, so 395).
//
// Two forms:
//   many rows -- four or eight waves of 32 rows share tiles of 64 (32) rows in LDS, as
//                smallkv_chunk_attn has them; the threads hold the codes of the tile after
//                next, and convert and write a tile while the one before it is multiplied;
//   few rows  -- (a decode step) columns of 16 rows, each wave walks tiles of 32 keys of its own.
// Where the (tile, kv head) pairs are too few, the cached rows are cut into spans, and
// join_spans joins their records.
//
// Measured (MI355X), and what bounds it:
//   a token each of 64 sequences of 1024 - 4096 rows, 28 and 4 heads of 128, 8 bits (173 MB): 42 us
//     (bf16 rows: 76), 4.1 TB/s: memory at about 5.5 TB/s, the longest sequences' tail, and 6 us
//     before the first rows and after the last; in 4 bits (92 MB) 30 us, where the vector units
//     that unpack are busy half of the time;
//   a token each of 4 sequences of 90001 - 131072 rows, 32 and 8 heads of 128, 8 bits (900 MB):
//     170 us, 5.3 TB/s, memory; in 4 bits (468 MB) 100 us, 4.7 TB/s, 122 where a page holds
//     [row][head], so that a head's 64 bytes lie 512 apart;
//   one token over 512 rows in fp32: 10.3 us, a chain of three dependent loads, two tiles a wave;
//   2 x 2048 tokens over 16384 rows, 32 and 8 heads of 128: 1145 us, 900 TFLOP/s, in 4 bits 1010:
//     products and softmax by turns, as over bf16 rows, and the unpacking;
//   4 x 4096 tokens over 16384 rows, 14 and 2 heads of 64: 1273 us, 660 TFLOP/s, in 4 bits 1285, more
//     than over bf16 rows (1085, workgroups of four waves, three on a CU): a CU has one workgroup.
#include <type_traits>

#include "attn.h"

namespace smallkv {
namespace {

// Values of a tile in LDS as TileLayout has them, and neighbouring pieces exchanged against the
// conflicts of banks in which a piece of codes, which becomes two or four, would be written.  (Of
// the LDS cycles of 2 x 2048 tokens over 16384 rows 16% are lost to conflicts.)
template <int D> struct MixedTile : TileLayout<bf16_t, D> {
  __device__ __forceinline__ static int swz_v(int r) {
    return D == 128 ? (r & 3) << 2 | (r & 3) : (r >> 1 & 1) << 2 | (r >> 1 & 3);
  }
};

// A thread's share of the pieces (16 bytes of codes) of tiles of BN rows of keys and
// values, which go to LDS in bf16.  The page of the lane's row is looked up a tile ahead, as in Loader.
template <int D, int F, int BN, int NT> struct Unpacker {
  using L = MixedTile<D>;
  static constexpr int P = D * F / 128, E = 128 / F;        // pieces of a row, elements of a piece
  static constexpr int kAll = 2 * BN * P, N = (kAll + NT - 1) / NT;
  static constexpr int O = E / 8;                           // 16-byte pieces that it becomes
  const int32_t *pages;
  int len, page;
  uint4 w[N];
  uint32_t s[N];

  __device__ __forceinline__ void init(const AttnArgs &a, int b, int end) {
    pages = a.kv.table ? a.kv.table + (int64_t)b * a.kv.width : a.c.len;
    len = end;
  }
  __device__ __forceinline__ void lookup(const CacheView &kv, int row0) {
    const int row = row0 + (int)(threadIdx.x & (BN - 1));
    page = pages[max(min(row, len - 1), 0) >> kv.shift];  // (dense: shift 31)
  }
  // Requests the looked-up tile; bit t of the result: its row t exists.
  template <int BM> __device__ __forceinline__ uint64_t fetch(const AttnArgs &a, const Share<BM> &x, int row0) {
    const int row = row0 + (int)(threadIdx.x & (BN - 1)), pg = a.kv.table ? page : x.t.b;
    const bool there = row < len && (uint32_t)pg < (uint32_t)a.kv.n_pages;
    const int at = there ? pg : -1;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = j * NT + (int)threadIdx.x, r = i / P & (BN - 1), p = i & (P - 1);
      const bool values = i >= BN * P;
      const int from = __shfl(at, r, kWave);
      const int64_t off = page_offset(a.kv, from, row0 + r);
      w[j] = make_uint4(0, 0, 0, 0);
      s[j] = 0;
      if (off >= 0 && i < kAll) {
        const int64_t so = scale_offset<D>(a.sc, a.kv, from, row0 + r, x.kvh) + p * E / kBlock;
        w[j] = *reinterpret_cast<const uint4 *>((values ? x.v : x.k) + off + p * 16);
        s[j] = (values ? a.sc.v : a.sc.k)[so];
      }
    }
    return __ballot(there);
  }
  // Writes what was requested to LDS.
  __device__ __forceinline__ void store(unsigned char *sk, unsigned char *sv) const {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = j * NT + (int)threadIdx.x, r = i / P & (BN - 1), p = i & (P - 1);
      const bool values = i >= BN * P;
      if (i >= kAll) continue;
      unsigned char *row = (values ? sv : sk) + r * L::bytes;
      const int z = values ? L::swz_v(r) : L::swz_k(r);
#pragma unroll
      for (int o = 0; o < O; ++o)
        *reinterpret_cast<uint4 *>(row + (((p * O + o) ^ z) << 4)) =
            unpack16<bf16_t, F>(reinterpret_cast<const uint32_t *>(&w[j]), o, scale_of(s[j]));
    }
  }
};

template <typename T, int D, int F, int NW, int BN>
__global__ __launch_bounds__(NW * kWave, 2) void packed_many(AttnArgs a) {
  using L = TileLayout<T, D>;
  constexpr int BM = NW * 32, kBuf = BN * L::bytes;
  __shared__ __align__(16) unsigned char k0[kBuf], v0[kBuf], k1[kBuf], v1[kBuf];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Share<BM> w;
  if (!w.find(a, blockIdx.x / a.hkv, blockIdx.x % a.hkv, kManyRound, kManyLeast, wave * 32)) return;
  const int w0 = w.t.row0 + wave * 32;
  const bool idle = w0 >= w.t.rows;
  const int highest = w.t.s.len - w.t.s.n_new + min(w0 + 31, w.t.rows - 1) / a.g;  // of the wave's rows
  QFrag<T, D> q;
  const unsigned char *queries = a.q + (w.token * a.q_token + w.head * a.q_head) * (int64_t)sizeof(T);
  const int half = (threadIdx.x & (kWave - 1)) >> 5;
  if constexpr (sizeof(T) == 4) {
    __shared__ bf16x8_t parts[NW][QFrag<T, D>::kLds ? QFrag<T, D>::kLds : 1][kWave];
    q.load(queries, half, &parts[wave][0][0]);
  } else {
    q.load(queries, half);
  }
  State<T, D> st;
  st.clear();
  constexpr uint64_t kAll = BN == 64 ? ~0ull : (1ull << (BN & 63)) - 1;
  int row = w.begin;
  Unpacker<D, F, BN, NW * kWave> ld;
  ld.init(a, w.t.b, w.end);
  ld.lookup(a.kv, row);
  uint64_t valid = 0, next = 0;  // rows of the tile at `row`, and of the one after it
  if (row < w.end) {
    valid = ld.fetch(a, w, row);
    ld.lookup(a.kv, row + BN);
    ld.store(k0, v0);
    if (row + BN < w.end) next = ld.fetch(a, w, row + BN);
    ld.lookup(a.kv, row + 2 * BN);
  }
  // the tile at `row` is in place; the next one goes to (nk, nv)
  auto advance = [&](unsigned char *nk, unsigned char *nv) {
    __syncthreads();
    const uint64_t now = valid;
    if (row + BN < w.end) {
      ld.store(nk, nv);
      valid = next;
      if (row + 2 * BN < w.end) {
        next = ld.fetch(a, w, row + 2 * BN);
        ld.lookup(a.kv, row + 3 * BN);
      }
    }
    return now;
  };
  // tiles that every row sees whole, then the others
  bool odd = false, taken = false, full = true;
  uint64_t now = 0;
  while (row < w.end) {
    now = advance(k1, v1);
    if (!(full = row + BN - 1 <= w.first_own && (now & kAll) == kAll)) break;
    if (!idle) full_tile<T, D, BN, MixedTile<D>>(st, q, k0, v0, a.scale2, a.scale2_lo);
    row += BN;
    if (row >= w.end) break;
    odd = true;
    now = advance(k0, v0);
    if (!(full = row + BN - 1 <= w.first_own && (now & kAll) == kAll)) break;
    if (!idle) full_tile<T, D, BN, MixedTile<D>>(st, q, k1, v1, a.scale2, a.scale2_lo);
    row += BN;
    odd = false;
  }
  while (row < w.end) {
    unsigned char *sk = odd ? k1 : k0, *sv = odd ? v1 : v0;
    if (full) now = advance(odd ? k0 : k1, odd ? v0 : v1);
    full = true;
    if (min(row + BN, w.end) - 1 > w.first_own)
      taken |= __syncthreads_or(take_out<bf16_t, BN * L::C>(sv, threadIdx.x, NW * kWave));
    if (!idle) masked_tile<T, D, BN, false, MixedTile<D>>(st, q, sk, sv, row, w.own, highest, now, a.scale2, a.scale2_lo);
    row += BN;
    odd = !odd;
  }
  write_row<T, D, BM, BN, false, F>(a, w, st, taken);
}

// 32 packed rows on their way to LDS: neighbouring lanes take neighbouring pieces of a row, so
// that an instruction touches whole lines (a row per lane, as the products want it: 16 lines
// for every 256 bytes, and a third less of the memory's rate).  N pieces a lane.
template <int D, int F> struct RowTile {
  static constexpr int P = D * F / 128, R = kWave / P, N = 32 / R, bytes = D * F / 8;
  u32x4_t w[N];
  uint32_t s[N];
  __device__ __forceinline__ static int row(int j) { return j * R + (int)(threadIdx.x & (kWave - 1)) / P; }
  __device__ __forceinline__ static int piece() { return threadIdx.x & (P - 1); }
  __device__ __forceinline__ void request(const unsigned char *rows, const uint8_t *scales, const int64_t (&off)[N],
                                          const int64_t (&so)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      w[j] = *reinterpret_cast<const u32x4_t *>(rows + off[j]);
      s[j] = scales[so[j]];
    }
  }
};

// Keys of a wave in LDS, as they are: written whole rows at a time, read a piece of 16 rows at a
// time, the pieces of a row exchanged against conflicts of banks.  (Not free of them: of the LDS
// cycles of a decode step, keys and values, 32% are lost to conflicts, of a long one in 4 bits 36%;
// which accesses have them was not found.)
template <int D, int F> struct KeyTile {
  using X = RowTile<D, F>;
  __device__ __forceinline__ static int swz(int r) { return r / (16 / X::P) & (X::P - 1); }
  __device__ __forceinline__ static void store(unsigned char *lds, const X &x) {
#pragma unroll
    for (int j = 0; j < X::N; ++j)
      *reinterpret_cast<u32x4_t *>(lds + X::row(j) * X::bytes + ((X::piece() ^ swz(X::row(j))) << 4)) = x.w[j];
  }
  // A quarter of row r.
  __device__ __forceinline__ static void load(const unsigned char *lds, int r, int quarter, uint32_t (&w)[D * F / 128]) {
    constexpr int kBytes = X::bytes / 4;
    const unsigned char *row = lds + r * X::bytes;
    if constexpr (kBytes == 8) {
      const uint2 x = *reinterpret_cast<const uint2 *>(row + ((quarter / 2 ^ swz(r)) << 4) + quarter % 2 * 8);
      w[0] = x.x;
      w[1] = x.y;
    } else {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t *>(row + (((quarter * (kBytes / 16) + i) ^ swz(r)) << 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * i + e] = x[e];
      }
    }
  }
};

// Values of a wave's 32 keys in LDS, in bf16: written as they come, read 32 bytes of 8 rows at a
// time, their pieces exchanged against conflicts of banks as those of the keys.
template <int D, int F> struct ValueTile {
  using X = RowTile<D, F>;
  static constexpr int bytes = 2 * D, kLow = X::R == 8 ? 0 : X::R == 16 ? 1 : 2;
  __device__ __forceinline__ static int swz(int r) { return (D == 128 ? r & 7 : r >> 1 & 3) << 1 | (r >> kLow & 1); }
};

// Workgroups go to the XCDs, each with an L2 of its own, in turn: the kv heads of a unit, whose
// rows share lines of memory where a page holds [row][head], follow each other on one.
constexpr int kXcds = 8;

// Few rows (a decode step): CB columns of 16, on 16 x 16 tiles; each wave walks tiles of 32
// keys of its own, whose rows it requests a tile ahead.  Keys go through LDS as they are, and
// become operands as they leave it (a quarter-wave holds a quarter of the dimensions: their
// order in the product is free); values become bf16 on their way into it, and the read that
// turns them leaves them as operands.  An fp32 model's queries and probabilities go through
// the products in three bf16 parts, so that they lose nothing that fp32 holds.
template <typename T, int D, int F, int CB, int NW>
__global__ __launch_bounds__(NW * kWave, 2) void packed_few(AttnArgs a) {
  using X = RowTile<D, F>;
  using K = KeyTile<D, F>;
  using L = ValueTile<D, F>;
  constexpr int BN = 32, BM = 16 * CB, QP = sizeof(T) == 4 ? 3 : 1, PP = sizeof(T) == 4 ? 3 : 2;
  constexpr int kKeys = BN * X::bytes, kTile = BN * L::bytes, kSteps = D / 32, kBlocks = D / 16;
  __shared__ __align__(16) unsigned char v0[NW * kTile], k0[NW * kKeys];
  __shared__ float ml[2][NW / 2][CB][kWave];
  const int lane = threadIdx.x & (kWave - 1), quarter = lane >> 4, in = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int flat = blockIdx.x / kXcds / a.hkv * kXcds + blockIdx.x % kXcds;
  int page = 0;  // of row lane % 32 of the tile that is requested next
  if (a.single && a.kv.table && flat < a.c.batch)  // (the first does not wait for the lengths)
    page = a.kv.table[(int64_t)flat * a.kv.width + (min(wave * BN + (lane & 31), a.kv.cap - 1) >> a.kv.shift)];
  Share<BM> w;
  if (!w.find(a, flat, blockIdx.x / kXcds % a.hkv, NW * BN, 1, 0)) return;
  unsigned char *sv = v0 + wave * kTile, *sk = k0 + wave * kKeys;
  constexpr int step = NW * BN;
  const int32_t *pages = a.kv.table ? a.kv.table + (int64_t)w.t.b * a.kv.width : a.c.len;
  X k, v;                        // of the next tile
  int64_t off[X::N], so[X::N];   // of the rows that are requested next, and their blocks' scales
  uint32_t scale[2];             // of the lane's quarters of two keys
  auto lookup = [&](int row) { page = pages[max(min(row + (lane & 31), w.end - 1), 0) >> a.kv.shift]; };
  // Rows that do not exist are read from rows that do, and masked.
  auto place = [&](int row) {
    const int pg = a.kv.table ? page : w.t.b;
    const bool there = (uint32_t)pg < (uint32_t)a.kv.n_pages;
    const uint32_t exist = (uint32_t)__ballot(there && row + (lane & 31) < w.end);
    const int at = there ? pg : 0;
#pragma unroll
    for (int j = 0; j < X::N; ++j) {
      const int r = min(row + X::row(j), w.end - 1), from = __shfl(at, X::row(j), kWave);
      off[j] = page_offset(a.kv, from, r) + X::piece() * 16;
      so[j] = scale_offset<D>(a.sc, a.kv, from, r, w.kvh) + X::piece() * 128 / F / kBlock;
    }
    return exist;
  };
  int row = w.begin + wave * BN;
  if (!a.single) lookup(row);
  bf16x8_t q[CB][QP][kSteps];
  int own[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    w.row(a, w.t.row0 + 16 * c + in);
    own[c] = w.own;
    const unsigned char *x = a.q + (w.token * a.q_token + w.head * a.q_head + quarter * (D / 4)) * (int64_t)sizeof(T);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if constexpr (sizeof(T) == 2) {
        q[c][0][i] = reinterpret_cast<const bf16x8_t *>(x)[i];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float y[QP];
          split<QP>(reinterpret_cast<const float *>(x)[8 * i + e], y);
#pragma unroll
          for (int p = 0; p < QP; ++p) q[c][p][i][e] = (__bf16)y[p];
        }
      }
    }
  }
  float m[CB], l[CB];  // running maximum (log2 units), this quarter-wave's part of the sum
  f32x4_t o[CB][kBlocks];
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    m[c] = -INFINITY;
    l[c] = 0.0f;
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) o[c][d] = f32x4_t{};
  }
  bool taken = false;
  if (row < w.end) {
    uint32_t next = place(row);  // rows of the next tile that exist
    k.request(w.k, a.sc.k, off, so);
    lookup(row + step);
    v.request(w.v, a.sc.v, off, so);
    for (; row < w.end; row += step) {
      const uint32_t rows = next;
      const bool full = row + BN - 1 <= w.first_own && rows == ~0u;
      K::store(sk, k);
      // a quarter's scale: of the lane that brought its (first) piece
      const int from = in % X::R * X::P + quarter * X::P / 4;
      if constexpr (X::R == 8) {
        const int s0 = __shfl((int)k.s[0], from, kWave), s1 = __shfl((int)k.s[1], from, kWave);
        const int s2 = __shfl((int)k.s[2], from, kWave), s3 = __shfl((int)k.s[3], from, kWave);
        scale[0] = in < 8 ? s0 : s1;
        scale[1] = in < 8 ? s2 : s3;
      } else {
        scale[0] = __shfl((int)k.s[0], from, kWave);
        scale[1] = __shfl((int)k.s[X::N - 1], X::R == 32 ? from + 16 * X::P : from, kWave);
      }
      f32x4_t s[CB][2] = {};
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        uint32_t codes[D * F / 128];
        K::load(sk, 16 * n + in, quarter, codes);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const bf16x8_t x = __builtin_bit_cast(bf16x8_t, (unpack16<bf16_t, F>(codes, i, scale_of(scale[n]))));
#pragma unroll
          for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int p = QP - 1; p >= 0; --p) s[c][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[c][p][i], s[c][n], 0, 0, 0);
        }
      }
      next = place(row + step);
      k.request(w.k, a.sc.k, off, so);
      lookup(row + 2 * step);
      if (!full) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool there = rows >> (16 * n + 4 * quarter + i) & 1u;
#pragma unroll
            for (int c = 0; c < CB; ++c)
              if (!there || row + 16 * n + 4 * quarter + i > own[c]) s[c][n][i] = -INFINITY;
          }
      }
      // the running maximum and sum; the reference point moves only when the maximum has
      // grown by more than 2^8 since it was set
      bf16x8_t pf[CB][PP];
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        float mx = s[c][0][0];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[c][n][i]);
        mx = swap_halves_max(swap_rows_max(mx)) * a.scale2;
        if (__any(mx > m[c] + 8.0f)) {
          const float top = fmaxf(m[c], mx), f = __builtin_amdgcn_exp2f(m[c] - (top == -INFINITY ? 0.0f : top));
          m[c] = top;
          l[c] *= f;
#pragma unroll
          for (int d = 0; d < kBlocks; ++d) o[c][d] *= f;
        }
        const float base = m[c] == -INFINITY ? 0.0f : m[c];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = s[c][n][i];
            const float y = sizeof(T) == 4 ? __builtin_fmaf(fmaxf(x, -3.402823466e38f), a.scale2_lo, -base) : -base;
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x, a.scale2, y));
            l[c] += p;
            float parts[PP];
            split<PP>(p, parts);
#pragma unroll
            for (int e = 0; e < PP; ++e) pf[c][e][4 * n + i] = (__bf16)parts[e];
          }
      }
      const bool mixed = min(row + BN, w.end) - 1 > w.first_own;  // rows that some see and some do not
      auto put = [&](auto whole) {
#pragma unroll
        for (int j = 0; j < X::N; ++j) {
          const int r = X::row(j);
          const uint32_t codes[4] = {v.w[j][0], v.w[j][1], v.w[j][2], v.w[j][3]};
#pragma unroll
          for (int i = 0; i < 16 / F; ++i) {
            uint4 x = unpack16<bf16_t, F>(codes, i, scale_of(v.s[j]));
            if (!whole) {
              if (!(rows >> r & 1u)) x = make_uint4(0, 0, 0, 0);
              if (mixed) taken |= drop_not_finite<bf16_t>(x);
            }
            *reinterpret_cast<uint4 *>(sv + r * L::bytes + (((X::piece() * (16 / F) + i) ^ L::swz(r)) << 4)) = x;
          }
        }
      };
      if (full)
        put(std::true_type());
      else
        put(std::false_type());
      v.request(w.v, a.sc.v, off, so);
      // the transposing read: 16 lanes take 4 rows of 16 elements, lane i of them ends with
      // the 4 rows' element i
#pragma unroll
      for (int d = 0; d < kBlocks; ++d) {
        union { s16x4_t h[2]; bf16x8_t v; } x;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int r = 16 * n + 4 * quarter + (in >> 2), c = 2 * d + ((lane & 3) >> 1);
          x.h[n] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (SMALLKV_LDS s16x4_t *)(sv + (r * L::bytes + ((c ^ L::swz(r)) << 4) + (lane & 1) * 8)));
        }
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int e = PP - 1; e >= 0; --e) o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v, pf[c][e], o[c][d], 0, 0, 0);
      }
    }
  }
  taken = __syncthreads_or(taken);
  // join the waves' results: the upper half hands over to the lower one
  float *x = reinterpret_cast<float *>(v0);
#pragma unroll
  for (int h = NW / 2; h >= 1; h >>= 1) {
    __syncthreads();
    float *y = x + (wave & (h - 1)) * CB * (D / 4) * kWave;
    if (wave >= h && wave < 2 * h) {
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        ml[0][wave - h][c][lane] = m[c];
        ml[1][wave - h][c][lane] = l[c];
#pragma unroll
        for (int d = 0; d < kBlocks; ++d) reinterpret_cast<f32x4_t *>(y)[(c * kBlocks + d) * kWave + lane] = o[c][d];
      }
    }
    __syncthreads();
    if (wave < h) {
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        const float om = ml[0][wave][c][lane], ol = ml[1][wave][c][lane];
        const float top = fmaxf(m[c], om), base = top == -INFINITY ? 0.0f : top;
        const float f = __builtin_amdgcn_exp2f(m[c] - base), fo = __builtin_amdgcn_exp2f(om - base);
        m[c] = top;
        l[c] = l[c] * f + ol * fo;
#pragma unroll
        for (int d = 0; d < kBlocks; ++d)
          o[c][d] = o[c][d] * f + reinterpret_cast<const f32x4_t *>(y)[(c * kBlocks + d) * kWave + lane] * fo;
      }
    }
  }
  if (wave > 0) return;
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    w.row(a, w.t.row0 + 16 * c + in);
    const float sum = swap_halves_sum(swap_rows_sum(l[c]));
    if (w.live) write_row<T, D, BM, BN, F>(a, w, o[c], m[c], sum, 4 * quarter, 16, quarter == 0, taken);
  }
}

// Joins the records of a tile's spans: four elements of a row per lane, a row's spans dealt to
// `parts` groups of such lanes, which each take theirs in one pass with the running maximum,
// scale their sums to the row's maximum and add them up in LDS.  Eight parts at most: workgroups
// of 256 threads start sooner than larger ones (128 spans of a token of 28 heads: 5.6 us, with 32
// parts 9.2, with four 7.1; 24 spans of 16 sequences 4.6, 7.5 and 4.2).
constexpr int kJoinParts = 8, kJoinThreads = 256;

template <typename T, int D, int BM> __global__ __launch_bounds__(kJoinThreads) void join_spans(AttnArgs a) {
  constexpr int W = D / 4;  // lanes of a row
  __shared__ f32x4_t so[kJoinThreads];
  __shared__ float2 sml[kJoinThreads / W];
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
  const int64_t step = stride * a.parts;
  const float *ml = a.rec + a.rec_ml + 2 * (at + part * stride), *rec = a.rec + (at + part * stride) * D + e;
  float m = -INFINITY, l = 0.0f;
  f32x4_t o = {};
  const int count = n > part ? (n - part - 1) / a.parts + 1 : 0;
#pragma unroll 4
  for (int s = 0; s < count; ++s) {
    const float2 x = *reinterpret_cast<const float2 *>(ml + 2 * s * step);
    const f32x4_t v = *reinterpret_cast<const f32x4_t *>(rec + s * step * D);
    const float top = fmaxf(m, x.x), base = top == -INFINITY ? 0.0f : top;
    const float f = __builtin_amdgcn_exp2f(m - base), w = __builtin_amdgcn_exp2f(x.x - base);
    m = top;
    l = l * f + x.y * w;
    o = o * f + v * w;
  }
  if (a.parts > 1) {
    if (e == 0) sml[group] = make_float2(m, l);
    __syncthreads();
    float top = -INFINITY;
    for (int g = group % n_rows; g < n_rows * a.parts; g += n_rows) top = fmaxf(top, sml[g].x);
    const float base = top == -INFINITY ? 0.0f : top, f = __builtin_amdgcn_exp2f(m - base);
    so[threadIdx.x] = o * f;
    l = 0.0f;
    for (int g = group % n_rows; g < n_rows * a.parts; g += n_rows)
      l += sml[g].y * __builtin_amdgcn_exp2f(sml[g].x - base);
    m = top;
    __syncthreads();
    if (part > 0) return;
    o = f32x4_t{};
    for (int g = group; g < n_rows * a.parts; g += n_rows) o += so[g * W + threadIdx.x % W];
  }
  if (r >= t.rows) return;
  const f32x4_t x = l == 0.0f ? f32x4_t{} : o * (1.0f / l);
  unsigned char *out = a.out + (token * a.o_token + head * a.o_head) * (int64_t)sizeof(T);
  if constexpr (sizeof(T) == 4)
    *reinterpret_cast<f32x4_t *>(out + e * 4) = x;
  else
    *reinterpret_cast<bf16x4_t *>(out + e * 2) = __builtin_convertvector(x, bf16x4_t);
  if (a.lse && e == 0)
    a.lse[(int64_t)token * a.hq + head] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// rows: of a tile that there can be.
template <typename T, int D, int BM> void launch_join(const AttnArgs &a, const AttnPlan &p, int rows, hipStream_t st) {
  const dim3 grid(p.tiles * a.hkv, ceil_div(rows, kJoinThreads / (D / 4) / a.parts));
  hipLaunchKernelGGL((join_spans<T, D, BM>), grid, dim3(kJoinThreads), 0, st, a);
}

template <typename T, int D, int F> hipError_t launch_typed(AttnArgs a, const AttnPlan &p, hipStream_t st) {
  constexpr bool h = sizeof(T) == 2;
  merge_shape<D>(a, p);
  a.parts = std::min(a.parts, kJoinParts);
  const dim3 grid(p.units * a.hkv), few(p.waves * kWave);
  using M = std::conditional_t<h, bf16_t, wide_t>;
  constexpr int BN = h || D == 64 ? 64 : 32;
  if (!p.few)
    hipLaunchKernelGGL((h && p.rows == 256 ? packed_many<M, D, F, h ? 8 : 4, BN> : packed_many<M, D, F, 4, BN>), grid,
                       dim3(p.rows * 2), 0, st, a);
  else if (p.rows == 16)
    hipLaunchKernelGGL((p.waves == 8 ? packed_few<T, D, F, 1, 8> : packed_few<T, D, F, 1, 4>), grid, few, 0, st, a);
  else if constexpr (h)
    hipLaunchKernelGGL((p.waves == 8 ? packed_few<T, D, F, 2, 8> : packed_few<T, D, F, 2, 4>), grid, few, 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.splits) return e;
  const int rows = (int)std::min<int64_t>(p.rows, (int64_t)a.c.max_new * a.g);
  if (p.rows == 256)
    launch_join<T, D, 256>(a, p, rows, st);
  else if (!p.few)
    launch_join<T, D, 128>(a, p, rows, st);
  else if (p.rows == 16)
    launch_join<T, D, 16>(a, p, rows, st);
  else
    launch_join<T, D, 32>(a, p, rows, st);
  return hipGetLastError();
}

template <typename T> hipError_t launch_format(const AttnArgs &a, const AttnPlan &p, int d, int bits, hipStream_t st) {
  if (bits == 8) return d == 64 ? launch_typed<T, 64, 8>(a, p, st) : launch_typed<T, 128, 8>(a, p, st);
  return d == 64 ? launch_typed<T, 64, 4>(a, p, st) : launch_typed<T, 128, 4>(a, p, st);
}

}  // namespace

AttnPlan plan_packed_attn(const smallkv_chunk_t &c, const smallkv_packed_t &kv, const smallkv_queries_t &q) {
  AttnPlan p{};
  const int g = q.n_heads / kv.n_heads;
  const int64_t rows = (int64_t)c.max_new * g;
  const bool f32 = kv.dtype == SMALLKV_F32;
  // (fp32, up to four tiles of 16: 54 rows over 8 x 4096 and 32 x 2048 cached rows 34 and 48 us,
  // as many rows 38 and 57; bf16, 28 rows: 25 and 27, 23 and 32)
  // Many rows, bf16: tiles of 256 where that leaves little of the last one empty: half as much
  // to unpack (2 x 2048 tokens over 16384 rows of 8 kv heads of 128: 1144 us, 1189 in tiles of
  // 128, in 4 bits 999 and 1109; 1200 rows of 8 sequences 596 and 579; heads of 64 were not
  // compared).
  p.few = rows <= (f32 ? 64 : 32);
  p.rows = !p.few ? (rows >= 1536 && !f32 ? 256 : 128) : f32 || rows <= 16 ? 16 : 32;
  // no more tiles than this, whatever the sequences' lengths
  p.tiles = (int)std::min<int64_t>(c.batch * ceil_div(rows, p.rows), (int64_t)c.n_tokens * g / p.rows + c.batch);
  // Few rows: whole sequences where they are short, or make a workgroup for enough CUs and are
  // not long; else spans, and a join.  (28 query and 4 kv heads of 128 in 8 bits, us: one
  // sequence of 512 rows 9.0, in spans 10.8; of 1024 12.6 and 11.3; 16 of 1024 rows 13.3 and
  // 14.1, 48 13.9 and 19.5; 24 of 2048 20.6 and 19.9, 48 22.5 and 28.4; 32 of 4096 35.9 and
  // 36.0, 48 41.9 and 49.9; 40 of 1024 - 4096 34.7 and 29.6, 48 36.5 and 36.7: with such mixed
  // lengths whole sequences lose at 160 groups, where the rule begins to take them, and no longer
  // at 192.  Heads of 64 in 4 bits: one sequence of 1024 rows 8.0 and 10.1, 32 of 2048 11.9 and
  // 12.0.  Many groups past 4096 rows, and that limit with heads of 64, were not measured.)
  const int64_t groups = (int64_t)p.tiles * kv.n_heads, length = (int64_t)c.max_len * kv.head_dim / 128;
  const bool whole = p.few && p.tiles <= c.batch &&
                     (length <= 512 || (length <= 1024 && groups >= 64) || (c.max_len <= 4096 && groups >= 160));
  // eight waves where that is one workgroup per CU (64 of 1024 - 4096 rows 41.8 us, with four
  // 50.0; 90 of 2048 49.7 and 41.7), from 256 rows on where half the CUs have none (one sequence
  // of 512 rows 9.0 us, with four 9.6; of 300 7.9 and 8.5; 16 of 512 9.5 and 10.0, but 64 of 512
  // 10.9 and 10.6)
  p.waves = whole && c.max_len > (groups <= 128 ? 256 : 512) && groups <= 256 ? 8 : kFewWaves;
  // the workgroups that run at once on 256 CUs, two on each; of 4 bits three (64 of 1024 - 4096
  // rows 32.7 us with two, 28.6 with three; in 8 bits 45.4 and 50.8)
  const bool three = p.rows == 16 && kv.dtype == SMALLKV_BF16 && kv.head_dim == 128 && kv.format == SMALLKV_MXFP4;
  const int slots = std::max((three ? 768 : p.rows == 256 ? 256 : 512) / kv.n_heads, 1);
  const int round = p.few ? 32 * kFewWaves : kManyRound * kManyLeast;
  if (p.tiles < slots && c.max_len > round && !whole)
    p.splits = (int)std::min<int64_t>(slots, (int64_t)p.tiles * ceil_div(c.max_len, round));
  p.units = std::max(p.tiles, p.splits);
  if (p.few) p.units = (p.units + kXcds - 1) / kXcds * kXcds;
  if (p.splits) p.ws_bytes = kSpanBytes + (size_t)p.units * kv.n_heads * p.rows * (kv.head_dim + 2) * sizeof(float);
  return p;
}

hipError_t launch_packed_attn(const smallkv_chunk_t &c, const smallkv_packed_t &kv, const smallkv_queries_t &q,
                              const AttnPlan &p, void *ws, hipStream_t st) {
  if (c.n_tokens == 0) return hipSuccess;
  AttnArgs a = attn_args(c, codes_of(kv), q, p, ws);
  a.sc = scale_view(kv);
  const int d = kv.head_dim, bits = format_bits(kv);
  return kv.dtype == SMALLKV_F32 ? launch_format<float>(a, p, d, bits, st) : launch_format<bf16_t>(a, p, d, bits, st);
}

}  // namespace smallkv
