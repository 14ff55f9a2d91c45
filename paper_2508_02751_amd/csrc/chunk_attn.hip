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
// accumulate in fp32; fp32 models multiply in fp32.  A bf16 model's P for the second
// product:
//   few rows  -- in two bf16 parts, a product each, 2^-16 relative: the rows of K and V
//                bound the pass, not the products (a token each of 64 sequences 62.8 us
//                with two parts, 62.4 with one; heads of 64 19.4 and 19.1);
//   many rows -- in one, each weight off by up to 2^-8 of itself, as much as the output's
//                own rounding: the products bound the pass (4096 tokens over 32768
//                rows 4.45 ms, with two parts 5.75; heads of 64 1.10 and 1.43).  The sum
//                of the rounded P divides the output, so that the weights add up to 1 and a
//                row's error is at most 2^-8 sum w |v - out|: none where one row has all the
//                weight or where values agree.  (Divided by the sum of the unrounded P, which
//                the lse takes: 4.33 and 1.04 ms.  The sum by a matrix product with ones in
//                place of the two-element dot products: 4.54 and 1.13.)
//
// Two forms:
//   many rows -- NW waves of 32 rows each share every tile of rows in LDS;
//                tiles are double-buffered, copied from memory to LDS directly;
//   few rows  -- where no sequence has more than 32 rows (64 in fp32; a decode
//                step): a column of 32 (16) rows, each wave walks its own tiles of 32
//                (16) keys, without a barrier, and the waves' results are joined at
//                the end.
// Where the (tile, kv head) pairs are too few to fill the GPU the cached rows are
// cut into spans, and attn_merge joins their records.  The span is found on the
// device from the sequences' own lengths, as the shortest with which the spans of
// all sequences still run at once: spans of equal length whatever the mixture.
//
// Measured (MI355X, after a hundred calls, when the clock has settled), and what bounds it:
//   2 x 4096 tokens over 32768 rows, 32 query and 8 kv heads of 128, bf16: 4.45 - 4.55 ms,
//     920 TFLOP/s (a bf16 product of 8192^3 by the library: 1218).  The matrix cores are
//     busy 43% and the vector units 48% of the cycles, mostly one after the other, at the
//     1.9 GHz that power leaves; without any softmax the same loops take 3.8 ms.
//     Heads of 64 (4 x 4096 tokens over 16384 rows, 14 heads): 1.10 ms, 765 TFLOP/s, half as
//     many products per exponential (34% and 68%).
//   a token each of 64 sequences of 1024 - 4096 rows, 28 and 4 heads of 128: 63 us for
//     336 MB of keys and values, 5.3 TB/s, + 5 us to join two spans each: memory.
//   one token over 32768 rows of 4 kv heads: 17 + 8 us, 67 MB: latency and two launches.
//   a 4096-token prompt in fp32, 32 and 8 heads of 128: 1.17 ms, 118 TFLOP/s of 153; the
//     matrix cores are busy 75% of the cycles.
#include "attn.h"

namespace smallkv {
namespace {

template <typename T, int D, int NW, int BN>
__global__ __launch_bounds__(NW * kWave, 2) void attn_many(AttnArgs a) {
  using L = TileLayout<T, D>;
  constexpr int BM = NW * 32, kBuf = BN * L::bytes, kRows = BN / NW;
  // four arrays: what is copied into one does not hold up the reads of another
  __shared__ __align__(16) unsigned char k0[kBuf], v0[kBuf], k1[kBuf], v1[kBuf];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Share<BM> w;
  if (!w.find(a, blockIdx.x / a.hkv, blockIdx.x % a.hkv, kManyRound, kManyLeast, wave * 32)) return;
  const int w0 = w.t.row0 + wave * 32;
  const bool idle = w0 >= w.t.rows;
  const int highest = w.t.s.len - w.t.s.n_new + min(w0 + 31, w.t.rows - 1) / a.g;  // of the wave's rows
  QFrag<T, D> q;
  q.load(a.q + (w.token * a.q_token + w.head * a.q_head) * (int64_t)sizeof(T), (threadIdx.x & (kWave - 1)) >> 5);
  State<T, D> st;
  st.clear();
  constexpr uint64_t kAll = BN == 64 ? ~0ull : (1ull << (BN & 63)) - 1;
  int row = w.begin;
  Loader<L, BN, kRows> ld;
  ld.init(a, w.t.b, w.end);
  ld.lookup(a.kv, row);
  uint64_t valid = 0;
  if (row < w.end) {
    const int64_t off = ld.offset(a.kv, w.t.b, row);
    valid = __ballot(off >= 0);
    ld.issue(off, w.k, w.v, wave * kRows, k0, v0);
    ld.lookup(a.kv, row + BN);
  }
  // the tile at `row` is in place; the next one goes to (nk, nv)
  auto advance = [&](unsigned char *nk, unsigned char *nv) {
    wait_memory();  // this wave's copies of the tile, and its reads of the other buffer
    __syncthreads();
    const uint64_t now = valid;
    if (row + BN < w.end) {
      const int64_t off = ld.offset(a.kv, w.t.b, row + BN);
      valid = __ballot(off >= 0);
      ld.issue(off, w.k, w.v, wave * kRows, nk, nv);
      ld.lookup(a.kv, row + 2 * BN);
    }
    return now;
  };
  // tiles that every row sees whole, then the others
  bool odd = false, taken = false, full = true;
  uint64_t now = 0;
  while (row < w.end) {
    now = advance(k1, v1);
    if (!(full = row + BN - 1 <= w.first_own && (now & kAll) == kAll)) break;
    if (!idle) full_tile<T, D, BN>(st, q, k0, v0, a.scale2, a.scale2_lo);
    row += BN;
    if (row >= w.end) break;
    odd = true;
    now = advance(k0, v0);
    if (!(full = row + BN - 1 <= w.first_own && (now & kAll) == kAll)) break;
    if (!idle) full_tile<T, D, BN>(st, q, k1, v1, a.scale2, a.scale2_lo);
    row += BN;
    odd = false;
  }
  while (row < w.end) {
    unsigned char *sk = odd ? k1 : k0, *sv = odd ? v1 : v0;
    if (full) now = advance(odd ? k0 : k1, odd ? v0 : v1);
    full = true;
    if (min(row + BN, w.end) - 1 > w.first_own)
      taken |= __syncthreads_or(take_out<T, BN * L::C>(sv, threadIdx.x, NW * kWave));
    if (!idle) masked_tile<T, D, BN, false>(st, q, sk, sv, row, w.own, highest, now, a.scale2, a.scale2_lo);
    row += BN;
    odd = !odd;
  }
  write_row<T, D, BM, BN, false>(a, w, st, taken);
}

// (three waves per SIMD of 64 elements: the plan counts on them)
template <int D> __global__ __launch_bounds__(kFewWaves * kWave, D == 64 ? 3 : 2) void attn_few_bf16(AttnArgs a) {
  using T = bf16_t;
  using L = TileLayout<T, D>;
  constexpr int NW = kFewWaves, BN = 32, kTile = BN * L::bytes;
  // one tile of keys and one of values per wave: the next keys are requested when
  // this tile's are multiplied, the next values after this tile's
  __shared__ __align__(16) unsigned char k0[NW * kTile], v0[NW * kTile];
  __shared__ float ml[2][NW / 2][kWave];
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Share<32> w;
  if (!w.find(a, blockIdx.x / a.hkv, blockIdx.x % a.hkv, NW * 32, 1, 0)) return;
  unsigned char *sk = k0 + wave * kTile, *sv = v0 + wave * kTile;
  constexpr int step = NW * BN;
  int row = w.begin + wave * BN;
  using Ld = Loader<L, BN, BN>;
  Ld ld;
  ld.init(a, w.t.b, w.end);
  ld.lookup(a.kv, row);
  QFrag<T, D> q;
  q.load(a.q + (w.token * a.q_token + w.head * a.q_head) * (int64_t)sizeof(T), lane >> 5);
  State<T, D> st;
  st.clear();
  wait_copies<0>();  // the queries and the first page number, requested together
  int64_t off = ld.offset(a.kv, w.t.b, row);
  bool taken = false;
  auto masked = [&]() {
    wait_memory();
    if (min(row + BN, w.end) - 1 > w.first_own) {
      taken |= __any(take_out<T, BN * L::C>(sv, lane, kWave));
      wait_lds();
    }
    masked_tile<T, D, BN, true>(st, q, sk, sv, row, w.own, w.end, (uint32_t)__ballot(off >= 0), a.scale2, a.scale2_lo);
  };
  if (row < w.end) {
    Ld::template issue_one<false>(off, w.k, sk);
    ld.lookup(a.kv, row + step);
    Ld::template issue_one<true>(off, w.v, sv);
    // Copies are requested in the order keys, page number, values, and none of them
    // on a condition: a wait for all but the last kInstr leaves the values, or the
    // next keys, on their way.
    for (; row + step < w.end; row += step) {
      if (row + BN - 1 <= w.first_own && __ballot(off >= 0) == ~0ull) {
        wait_copies<Ld::kInstr>();
        f32x16_t s[1] = {logits32<T, D>(sk, 0, q)};
        wait_lds();
        off = ld.offset(a.kv, w.t.b, row + step);
        Ld::template issue_one<false>(off, w.k, sk);
        softmax_step<T, D>(st, s, a.scale2, a.scale2_lo);
        wait_copies<Ld::kInstr>();
        values32<T, D, true>(sv, 0, s[0], st);
      } else {
        masked();
        wait_lds();
        off = ld.offset(a.kv, w.t.b, row + step);
        Ld::template issue_one<false>(off, w.k, sk);
      }
      wait_lds();
      ld.lookup(a.kv, row + 2 * step);
      Ld::template issue_one<true>(off, w.v, sv);
    }
    masked();
  }
  taken = __syncthreads_or(taken);
  join_waves<T, D, NW>(st, reinterpret_cast<float *>(k0), ml);
  if (wave == 0) write_row<T, D, 32, BN, true>(a, w, st, taken);
}

// The same in fp32, on 16 x 16 tiles: a quarter-wave holds a quarter of the head
// dimension of the logits' product, and 4 keys of the 16 in registers.
template <int D> struct FewLayout : TileLayout<float, D> {
  // values are read 64 bytes of rows 4 apart at once
  __device__ __forceinline__ static int swz_v(int r) { return (r >> 2 & 3) << 2; }
};

template <int D> __global__ __launch_bounds__(kFewWaves * kWave, 2) void attn_few_f32(AttnArgs a) {
  using T = float;
  using L = FewLayout<D>;
  constexpr int NW = kFewWaves, BN = 16, kTile = BN * L::bytes, kBlocks = D / 16;
  __shared__ __align__(16) unsigned char k0[NW * kTile], v0[NW * kTile];
  __shared__ float ml[2][NW / 2][kWave];
  const int lane = threadIdx.x & (kWave - 1), quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Share<16> w;
  if (!w.find(a, blockIdx.x / a.hkv, blockIdx.x % a.hkv, NW * BN, 1, 0)) return;
  unsigned char *sk = k0 + wave * kTile, *sv = v0 + wave * kTile;
  constexpr int step = NW * BN;
  int row = w.begin + wave * BN;
  using Ld = Loader<L, BN, BN>;
  Ld ld;
  ld.init(a, w.t.b, w.end);
  ld.lookup(a.kv, row);
  f32x4_t q[kBlocks];
  const float *qrow = reinterpret_cast<const float *>(a.q) + w.token * a.q_token + w.head * a.q_head + quarter * (D / 4);
#pragma unroll
  for (int i = 0; i < kBlocks; ++i) q[i] = reinterpret_cast<const f32x4_t *>(qrow)[i];
  float m = -INFINITY, l = 0.0f;
  f32x4_t o[kBlocks] = {};
  wait_copies<0>();  // the queries and the first page number, requested together
  int64_t off = ld.offset(a.kv, w.t.b, row);
  bool taken = false;
  // the next page number is looked up on the way, and the next keys (while this tile's
  // logits wait for their values) and values requested, if there are any
  auto logits = [&]() {
    f32x4_t s[4] = {};
    const unsigned char *at = sk + (lane & 15) * L::bytes;
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
      const f32x4_t k = *reinterpret_cast<const f32x4_t *>(at + (((quarter * kBlocks + i) ^ L::swz_k(lane & 15)) << 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], q[i][e], s[e], 0, 0, 0);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
  };
  auto weigh = [&](f32x4_t &s) {
    float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    mx = swap_halves_max(fmaxf(mx, __shfl_xor(mx, 16, kWave))) * a.scale2;
    if (__any(mx > m + 8.0f)) {
      const float top = fmaxf(m, mx), f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
      m = top;
      l *= f;
#pragma unroll
      for (int d = 0; d < kBlocks; ++d) o[d] *= f;
    }
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = __builtin_fmaf(fmaxf(s[i], -3.402823466e38f), a.scale2_lo, -base);
      s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale2, x));
      l += s[i];
    }
  };
  auto values = [&](const f32x4_t &p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * quarter + i;
#pragma unroll
      for (int d = 0; d < kBlocks; ++d) {
        const int c = d * 4 + ((lane & 15) >> 2);
        const float v = *reinterpret_cast<const float *>(sv + (r * L::bytes + ((c ^ L::swz_v(r)) << 4) + (lane & 3) * 4));
        o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[i], o[d], 0, 0, 0);
      }
    }
  };
  auto masked = [&]() {
    wait_memory();
    if (min(row + BN, w.end) - 1 > w.first_own) {
      taken |= __any(take_out<T, BN * L::C>(sv, lane, kWave));
      wait_lds();
    }
    f32x4_t s = logits();
    const uint32_t valid = (uint32_t)__ballot(off >= 0) >> (4 * quarter);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = (valid >> i & 1u) && row + 4 * quarter + i <= w.own ? s[i] : -INFINITY;
    weigh(s);
    values(s);
  };
  if (row < w.end) {
    Ld::template issue_one<false>(off, w.k, sk);
    ld.lookup(a.kv, row + step);
    Ld::template issue_one<true>(off, w.v, sv);
    for (; row + step < w.end; row += step) {  // (copies as in attn_few_bf16)
      if (row + BN - 1 <= w.first_own && __ballot(off >= 0) == ~0ull) {
        wait_copies<Ld::kInstr>();
        f32x4_t s = logits();
        wait_lds();
        off = ld.offset(a.kv, w.t.b, row + step);
        Ld::template issue_one<false>(off, w.k, sk);
        weigh(s);
        wait_copies<Ld::kInstr>();
        values(s);
      } else {
        masked();
        wait_lds();
        off = ld.offset(a.kv, w.t.b, row + step);
        Ld::template issue_one<false>(off, w.k, sk);
      }
      wait_lds();
      ld.lookup(a.kv, row + 2 * step);
      Ld::template issue_one<true>(off, w.v, sv);
    }
    masked();
  }
  taken = __syncthreads_or(taken);
  float *x = reinterpret_cast<float *>(k0);
#pragma unroll
  for (int h = NW / 2; h >= 1; h >>= 1) {
    __syncthreads();
    float *y = x + (wave & (h - 1)) * (D / 4) * kWave;
    if (wave >= h && wave < 2 * h) {
      ml[0][wave - h][lane] = m;
      ml[1][wave - h][lane] = l;
#pragma unroll
      for (int d = 0; d < kBlocks; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[(d * 4 + i) * kWave + lane] = o[d][i];
    }
    __syncthreads();
    if (wave < h) {
      const float om = ml[0][wave][lane], ol = ml[1][wave][lane];
      const float top = fmaxf(m, om), base = top == -INFINITY ? 0.0f : top;
      const float f = __builtin_amdgcn_exp2f(m - base), fo = __builtin_amdgcn_exp2f(om - base);
      m = top;
      l = l * f + ol * fo;
#pragma unroll
      for (int d = 0; d < kBlocks; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[d][i] = o[d][i] * f + y[(d * 4 + i) * kWave + lane] * fo;
    }
  }
  if (wave > 0) return;
  l = swap_halves_sum(l + __shfl_xor(l, 16, kWave));
  if (w.live) write_row<T, D, 16, BN>(a, w, o, m, l, 4 * quarter, 16, quarter == 0, taken);
}

template <typename T, int D> hipError_t launch_typed(AttnArgs a, const AttnPlan &p, hipStream_t st) {
  constexpr bool h = sizeof(T) == 2;
  constexpr int BM = kAttnWaves * 32, BF = h ? 32 : 16;
  const dim3 grid(p.units * a.hkv);
  const MergeShape m = merge_shape<D>(a, p);
  if (!p.few)
    hipLaunchKernelGGL((attn_many<T, D, kAttnWaves, h ? 64 : 32>), grid, dim3(kAttnWaves * kWave), 0, st, a);
  else if constexpr (h)
    hipLaunchKernelGGL((attn_few_bf16<D>), grid, dim3(kFewWaves * kWave), 0, st, a);
  else
    hipLaunchKernelGGL((attn_few_f32<D>), grid, dim3(kFewWaves * kWave), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.splits) return e;
  if (p.few)
    launch_merge<T, D, BF>(a, p, m, st);
  else
    launch_merge<T, D, BM>(a, p, m, st);
  return hipGetLastError();
}

}  // namespace

AttnPlan plan_chunk_attn(const smallkv_chunk_t &c, const smallkv_cache_t &kv, const smallkv_queries_t &q) {
  AttnPlan p{};
  const int g = q.n_heads / kv.n_heads;
  const int64_t rows = (int64_t)c.max_new * g;
  const bool f32 = kv.dtype == SMALLKV_F32;
  const int few = f32 ? 16 : 32;
  // (fp32, whose products bound it, up to four tiles: 28 rows over 8 x 4096 and 32 x 2048
  // cached rows 46 us against 96, 56 rows 143 against 180, 112 rows 264 against 200;
  // bf16, 56 rows over 32 x 2048: 38 us against 35)
  p.few = rows <= (f32 ? 64 : 32);
  p.rows = p.few ? few : kAttnWaves * 32;
  // no more tiles than this, whatever the sequences' lengths
  p.tiles = (int)std::min<int64_t>(c.batch * ceil_div(rows, p.rows), (int64_t)c.n_tokens * g / p.rows + c.batch);
  // the workgroups that run at once on 256 CUs: three per CU of bf16 and 64 elements
  // (33 KB of LDS, up to 160 registers), two of 128 elements and of fp32.  (A batch
  // of chunks and tokens of 64 elements: 49 us with 512, 46 with 768, 46 with 1024;
  // a batch-64 decode step of 128 elements: 79 with 256, 70 with 512, 71 with 1024.)
  const int slots = std::max((kv.head_dim == 64 && !f32 ? 768 : 512) / kv.n_heads, 1);
  const int round = p.few ? few * kFewWaves : kManyRound * kManyLeast;
  if (p.tiles < slots && c.max_len > round)
    p.splits = (int)std::min<int64_t>(slots, (int64_t)p.tiles * ceil_div(c.max_len, round));
  p.units = std::max(p.tiles, p.splits);
  if (p.splits) p.ws_bytes = kSpanBytes + (size_t)p.units * kv.n_heads * p.rows * (kv.head_dim + 2) * sizeof(float);
  return p;
}

hipError_t launch_chunk_attn(const smallkv_chunk_t &c, const smallkv_cache_t &kv, const smallkv_queries_t &q,
                             const AttnPlan &p, void *ws, hipStream_t st) {
  if (c.n_tokens == 0) return hipSuccess;
  const AttnArgs a = attn_args(c, kv, q, p, ws);
  if (kv.dtype == SMALLKV_F32)
    return kv.head_dim == 64 ? launch_typed<float, 64>(a, p, st) : launch_typed<float, 128>(a, p, st);
  return kv.head_dim == 64 ? launch_typed<bf16_t, 64>(a, p, st) : launch_typed<bf16_t, 128>(a, p, st);
}

}  // namespace smallkv
