// Attention of the new tokens over a packed cache: the sums of smallkv_chunk_attn with rows
// of 8- or 4-bit codes, which become bf16 or fp32 (exactly) on their way into LDS.
//
// Many rows: a workgroup's threads hold the codes of the tile after next in registers; a tile's are
// converted and written to LDS while the tile before it is multiplied.
#include "attn.h"

namespace smallkv {
namespace {

// A thread's share of the pieces (16 bytes of codes) of tiles of BN rows of keys and
// values.  The page of the lane's row is looked up a tile ahead, as in Loader.
template <typename T, int D, int F, int BN, int NT> struct Unpacker {
  using L = TileLayout<T, D>;
  static constexpr int P = D * F / 128, E = 128 / F;        // pieces of a row, elements of a piece
  static constexpr int kAll = 2 * BN * P, N = (kAll + NT - 1) / NT;
  static constexpr int O = E * (int)sizeof(T) / 16;         // 16-byte pieces that it becomes
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
            unpack16<T, F>(reinterpret_cast<const uint32_t *>(&w[j]), o, scale_of(s[j]));
    }
  }
};

template <typename T, int D, int F, int NW, int BN>
__global__ __launch_bounds__(NW * kWave, sizeof(T) * D == 512 ? 1 : 2) void packed_many(AttnArgs a) {
  using L = TileLayout<T, D>;
  constexpr int BM = NW * 32, kBuf = BN * L::bytes;
  __shared__ __align__(16) unsigned char k0[kBuf], v0[kBuf], k1[kBuf], v1[kBuf];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Share<BM> w;
  if (!w.find(a, blockIdx.x, kManyRound, kManyLeast, wave * 32)) return;
  const int w0 = w.t.row0 + wave * 32;
  const bool idle = w0 >= w.t.rows;
  const int highest = w.t.s.len - w.t.s.n_new + min(w0 + 31, w.t.rows - 1) / a.g;  // of the wave's rows
  QFrag<T, D> q;
  q.load(a.q + (w.token * a.q_token + w.head * a.q_head) * (int64_t)sizeof(T), (threadIdx.x & (kWave - 1)) >> 5);
  State<T, D> st;
  st.clear();
  constexpr uint64_t kAll = BN == 64 ? ~0ull : (1ull << (BN & 63)) - 1;
  int row = w.begin;
  Unpacker<T, D, F, BN, NW * kWave> ld;
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
  write_row<T, D, BM, BN, false, F>(a, w, st, taken);
}

// Values of a wave's 32 keys in LDS, in bf16: written 16 rows of one piece at a time, read 4
// rows of 4 pieces at a time, both without a conflict of banks.
template <int D> struct ValueTile : TileLayout<bf16_t, D> {
  __device__ __forceinline__ static int swz_v(int r) {
    return D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
  }
};

// Few rows (a decode step), bf16: a column of 32, each wave walks tiles of its own.  A lane
// takes half of a key's and of a value's row, as they are, a tile ahead: the keys are
// converted into the operands of their product (whose order of dimensions is free: a
// half-wave holds a half), the values by way of LDS, which turns them.
template <int D, int F> __global__ __launch_bounds__(kFewWaves * kWave, 2) void packed_few(AttnArgs a) {
  using T = bf16_t;
  using L = ValueTile<D>;
  constexpr int NW = kFewWaves, NB = F == 4 || D == 64 ? 2 : 1, BN = 32 * NB, P = D / 16;
  constexpr int kTile = 32 * L::bytes;
  __shared__ __align__(16) unsigned char v0[NW * kTile];
  __shared__ float ml[2][NW / 2][kWave];
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5, in = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Share<32> w;
  if (!w.find(a, blockIdx.x, NW * 32, 1, 0)) return;
  unsigned char *sv = v0 + wave * kTile;
  constexpr int step = NW * BN;
  const int32_t *pages = a.kv.table ? a.kv.table + (int64_t)w.t.b * a.kv.width : a.c.len;
  HalfRow<D, F> k[NB], v[NB];
  int page[NB];     // of the tile that is requested next
  int64_t off[NB];  // of the tile whose values are requested next, or -1, and of its scales
  int64_t so[NB];
  auto lookup = [&](int row) {
#pragma unroll
    for (int n = 0; n < NB; ++n) page[n] = pages[max(min(row + 32 * n + in, w.end - 1), 0) >> a.kv.shift];
  };
  // whether all rows of the tile exist
  auto place = [&](int row) {
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int r = row + 32 * n + in, pg = a.kv.table ? page[n] : w.t.b;
      off[n] = page_offset(a.kv, pg, r);
      if (r >= w.end) off[n] = -1;
      so[n] = scale_offset<D>(a.sc, a.kv, pg, r, w.kvh);
    }
  };
  auto request_keys = [&](int n) {
    k[n].load(off[n] < 0 ? zero_row : w.k + off[n], off[n] < 0 ? zero_row : a.sc.k + so[n], half);
  };
  auto request_values = [&](int n) {
    v[n].load(off[n] < 0 ? zero_row : w.v + off[n], off[n] < 0 ? zero_row : a.sc.v + so[n], half);
  };
  int row = w.begin + wave * BN;
  lookup(row);
  bf16x8_t q[P];
  {
    const unsigned char *x = a.q + (w.token * a.q_token + w.head * a.q_head) * 2 + half * D;
#pragma unroll
    for (int i = 0; i < P; ++i) q[i] = reinterpret_cast<const bf16x8_t *>(x)[i];
  }
  State<T, D> st;
  st.clear();
  bool taken = false;
  if (row < w.end) {
    place(row);
#pragma unroll
    for (int n = 0; n < NB; ++n) request_keys(n);
    lookup(row + step);
#pragma unroll
    for (int n = 0; n < NB; ++n) request_values(n);
    for (; row < w.end; row += step) {
      f32x16_t s[NB];
      uint32_t valid[NB];
      bool full = row + BN - 1 <= w.first_own;
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const uint64_t there = __ballot(off[n] >= 0);
        valid[n] = (uint32_t)there;
        full &= there == ~0ull;
      }
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        s[n] = f32x16_t{};
#pragma unroll
        for (int i = 0; i < P; ++i)
          s[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k[n].template get<T>(i)), q[i],
                                                         s[n], 0, 0, 0);
      }
      place(row + step);
#pragma unroll
      for (int n = 0; n < NB; ++n) request_keys(n);
      lookup(row + 2 * step);
      if (!full) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const uint32_t bits = valid[n] >> (4 * half);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const bool ok = (bits >> reg_key(i) & 1u) && row + 32 * n + reg_key(i) + 4 * half <= w.own;
            s[n][i] = ok ? s[n][i] : -INFINITY;
          }
        }
      }
      softmax_step<T, D, NB>(st, s, a.scale2, a.scale2_lo);
      const bool mixed = min(row + BN, w.end) - 1 > w.first_own;  // rows that some see and some do not
#pragma unroll
      for (int n = 0; n < NB; ++n) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
          uint4 x = v[n].template get<T>(i);
          if (mixed) taken |= drop_not_finite<T>(x);
          *reinterpret_cast<uint4 *>(sv + in * L::bytes + (((half * P + i) ^ L::swz_v(in)) << 4)) = x;
        }
        request_values(n);
        values32<T, D, true, L>(sv, 0, s[n], st);
      }
    }
  }
  taken = __syncthreads_or(taken);
  join_waves<T, D, NW>(st, reinterpret_cast<float *>(v0), ml);
  if (wave == 0) write_row<T, D, 32, BN, true, F>(a, w, st, taken);
}

template <typename T, int D, int F> hipError_t launch_typed(AttnArgs a, const AttnPlan &p, hipStream_t st) {
  constexpr bool h = sizeof(T) == 2;
  const MergeShape m = merge_shape<D>(a, p);
  const dim3 grid(p.units * a.hkv);
  if constexpr (h) {
    if (p.few) hipLaunchKernelGGL((packed_few<D, F>), grid, dim3(kFewWaves * kWave), 0, st, a);
  }
  if (!p.few)
    hipLaunchKernelGGL((packed_many<T, D, F, kAttnWaves, h ? 64 : 32>), grid, dim3(kAttnWaves * kWave), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.splits) return e;
  if (p.few)
    launch_merge<T, D, 32>(a, p, m, st);
  else
    launch_merge<T, D, kAttnWaves * 32>(a, p, m, st);
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
  p.few = rows <= 32 && kv.dtype == SMALLKV_BF16;
  p.rows = p.few ? 32 : kAttnWaves * 32;
  // no more tiles than this, whatever the sequences' lengths
  p.tiles = (int)std::min<int64_t>(c.batch * ceil_div(rows, p.rows), (int64_t)c.n_tokens * g / p.rows + c.batch);
  // the workgroups that run at once on 256 CUs
  const int slots = std::max((p.few ? 512 : 512) / kv.n_heads, 1);
  const int round = p.few ? 32 * kFewWaves : kManyRound * kManyLeast;
  if (p.tiles < slots && c.max_len > round)
    p.splits = (int)std::min<int64_t>(slots, (int64_t)p.tiles * ceil_div(c.max_len, round));
  p.units = std::max(p.tiles, p.splits);
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
