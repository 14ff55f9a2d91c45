// The attention weight that the new tokens give every cached row, added to its
// running score: out[r] = before[r] + sum over (token, head) of exp(s - lse).
//
// No sum leaves its workgroup: no atomics, one order, and the logits are never
// stored.  Three forms:
//   chunk   -- a workgroup owns keys of one kv head (32 per wave, their K rows in
//              registers as the left operand of S^T = K Q^T) and walks the
//              query rows that see them, 64 at a time through LDS.  A lane holds one
//              query row's logits of 16 keys of a block: one fused multiply-add, one
//              exponential and one add each, which bound the pass; the product's
//              matrix instructions run beside them.  Scores per query head: the heads
//              are dealt to workgroups, each walking one head's tokens;
//              per kv head: the rows are (token, head) pairs.  Where that makes too few
//              workgroups (SPLIT), one owns 32 keys, its waves deal the rows among
//              themselves without a barrier, and their sums are added at the end.
//   heads   -- per query head, up to 128 tokens in a sequence: the same with several heads
//              to a workgroup, which reads its keys once for them all.
//   few     -- no sequence has more than 32 (token, head) rows (a decode step): the
//              rows stay in registers as the left operand of S = Q K^T, a lane holds
//              one key's logits, and each wave streams its keys' rows, bound by
//              reading K once.
//
// Measured (MI355X, after a hundred calls, when the clock has settled: the first tens of
// calls, of which the pairs of figures at the rules below are, take up to 15% more): 2048
// tokens of 32 query heads of 64 over 16384 rows, bf16 (1.0e9 exponentials, 129 GFLOP)
// 192 us, the vector units busy 78% of the cycles; 4096 tokens of 32 heads of 128, 93 us,
// 740 TFLOP/s, fp32 596 us, 115 TFLOP/s, the matrix cores busy 74%.  Per kv head, 2048 tokens
// of 14 heads over 8192 rows of 2 kv heads of 64, 74 us (SPLIT): latency, the vector units
// busy 42%, the matrix cores 13%.  A token each of 64 sequences of 1024 - 4096 rows of 4 kv
// heads of 128 (168 MB) 41 us, 4.1 TB/s; of 16 sequences over 82552 rows of 2 kv heads of
// 64 (23 MB) 9.0 us: latency.
#include <algorithm>
#include <type_traits>

#include "cache.h"
#include "launch.h"

namespace smallkv {
namespace {

__device__ __align__(16) unsigned char zero_row[512];

struct ScoreArgs {
  ChunkView c;
  CacheView kv;
  int hq, hkv, g, per_kv;
  const unsigned char *q;
  int64_t q_token, q_head;  // in bytes
  const float *lse;
  const float *before;
  float *out;
  int64_t rows, seq_stride;  // of before and out, in elements
  float scale;    // bf16: scale * log2(e), see weight_of
  int pieces;     // few: workgroups that share a (sequence, kv head)
  int walk;       // heads: tiles of query rows (of one token range) per workgroup
};

constexpr float kLog2e = 1.4426950408889634074f;
constexpr int kNW = 4;

// exp(scale * x - lse).  fp32 models: both as they were given, one rounding of their
// difference, then log2(e): exact to 2^-23 of the difference, not of the logit (with the
// bf16 models' form logits of 1000 gave weights off by 9e-5, most of them one way).
// bf16 models: in log2 units from the start, an instruction less in a pass that the vector
// units bound; the attention that made the lse rounds its factor the same way.
template <typename T> __device__ __forceinline__ float lse_of(float lse) {
  return sizeof(T) == 4 ? lse : lse * kLog2e;
}
template <typename T> __device__ __forceinline__ float weight_of(const ScoreArgs &a, float x, float lse) {
  const float t = __builtin_fmaf(x, a.scale, -lse);
  return __builtin_amdgcn_exp2f(sizeof(T) == 4 ? t * kLog2e : t);
}

// Sums over ROWS (16 or 32) neighbouring lanes' query rows: each exchange halves the keys
// that a lane holds.  The lane ends with key register (lane % ROWS) * 16 / ROWS.
template <int ROWS> __device__ __forceinline__ float sum_rows(float (&acc)[16]) {
  const int lane = threadIdx.x & (kWave - 1);
  auto fold = [&](auto n, int o) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float send = up ? acc[i] : acc[i + n], keep = up ? acc[i + n] : acc[i];
      acc[i] = keep + __shfl_xor(send, o, kWave);
    }
  };
  fold(std::integral_constant<int, 8>(), ROWS / 2);
  fold(std::integral_constant<int, 4>(), ROWS / 4);
  fold(std::integral_constant<int, 2>(), ROWS / 8);
  fold(std::integral_constant<int, 1>(), ROWS / 16);
  return ROWS == 32 ? acc[0] + __shfl_xor(acc[0], 1, kWave) : acc[0];
}

template <typename T, int D, bool PER_KV, bool SPLIT>
__global__ __launch_bounds__(kNW * kWave, SPLIT && sizeof(T) * D == 512 ? 1 : 2) void chunk_scores(ScoreArgs a) {
  using L = TileLayout<T, D>;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kFrag = kBf16 ? D / 16 : D / 8;  // 16-byte pieces of a row per lane
  constexpr int kKeys = SPLIT ? 32 : 32 * kNW, kRows = SPLIT ? 32 * kNW : 64;
  constexpr int kBuf = kRows * L::bytes, kShare = kRows / kNW, kRpi = 64 / L::C, kInstr = kShare / kRpi;
  __shared__ __align__(16) unsigned char q0[kBuf], q1[kBuf];
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  // the first keys, which the most tokens see, come first for all heads (a 4096-token
  // prompt of 32 heads: 96 us, 120 with the heads one after another)
  const int heads = PER_KV ? a.hkv : a.hq, units = a.c.batch * heads, unit = blockIdx.x % units;
  const int b = unit / heads, kvh = PER_KV ? unit % heads : unit % heads / a.g;
  const Seq s = sequence(a.c, b, a.kv.cap);
  const int block0 = (blockIdx.x / units) * kKeys, key0 = block0 + (SPLIT ? 0 : wave * 32);
  if (block0 >= s.len) return;
  const int pos0 = s.len - s.n_new;
  // per query head: this head's tokens; per kv head: (token, head) pairs
  const int g = PER_KV ? a.g : 1, head0 = PER_KV ? kvh * a.g : unit % heads;
  const int first = max(0, block0 - pos0);  // the first token that sees a key of the workgroup
  const int n_tokens = s.n_new - first, n_rows = n_tokens * g;

  uint4 kf[kFrag];
  uint32_t exists;
  {
    const int key = key0 + (lane & 31);
    const int64_t off = key < s.len ? row_offset(a.kv, b, key) : -1;
    const unsigned char *row = off >= 0 ? a.kv.k + off + (((uint64_t)kvh * a.kv.head_stride) << 4) : zero_row;
#pragma unroll
    for (int i = 0; i < kFrag; ++i)
      kf[i] = reinterpret_cast<const uint4 *>(row)[kBf16 ? 2 * i + half : half * kFrag + i];
    exists = (uint32_t)__ballot(off >= 0);
  }

  float acc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.0f;

  // The lane's row of a tile: its token, head and lse, requested a tile ahead and
  // not used before then.  Rows past the last repeat one that exists.
  const int mine = SPLIT ? wave * 32 + (lane & 31) : lane;
  int row_token = PER_KV ? mine / g : mine, row_head = PER_KV ? mine % g : 0;
  const int step_token = PER_KV ? kRows / g : kRows, step_head = PER_KV ? kRows % g : 0;
  int token = 0, head = 0;
  float lse = 0.0f;
  const float *lse0 = a.lse + (int64_t)(s.first + first) * a.hq + head0;
  auto lookup = [&]() {
    token = row_token;
    head = row_head;
    lse = lse0[(int64_t)min(token, n_tokens - 1) * a.hq + head];
    row_token += step_token;
    row_head += step_head;
    if (PER_KV && row_head >= g) {
      row_head -= g;
      ++row_token;
    }
  };
  // own: its cached row; -1, which gives no weight: past the last, or sees no key
  int own = 0, own_now, r0 = 0;
  float lse_x = 0.0f, lse_now;
  const unsigned char *q = a.q + (s.first + first) * a.q_token + head0 * a.q_head;
  auto issue = [&](unsigned char *dst, int row0) {
    const bool dead = token >= n_tokens || lse == -INFINITY;
    own = dead ? -1 : pos0 + first + token;
    lse_x = dead ? 0.0f : lse_of<T>(lse);
    const int rr = lane / L::C, p = lane & (L::C - 1);
#pragma unroll
    for (int j = 0; j < kInstr; ++j) {
      const int r = wave * kShare + j * kRpi + rr;
      uint64_t o;
      if constexpr (PER_KV) {
        const int at = SPLIT ? j * kRpi + rr : r;  // the lane whose row it is
        const int from = __shfl(min(token, n_tokens - 1), at, kWave), h = __shfl(head, at, kWave);
        o = (uint64_t)(uint32_t)from * (uint32_t)a.q_token + (uint64_t)(uint32_t)h * (uint32_t)a.q_head;
      } else {
        o = (uint64_t)(uint32_t)min(row0 + r, n_tokens - 1) * (uint32_t)a.q_token;
      }
      load_to_lds16(q + o + ((p ^ L::swz_k(r)) << 4), dst + (wave * kShare + j * kRpi) * L::bytes);
    }
  };
  if (n_rows > 0) {
    lookup();
    issue(q0, 0);
    lookup();
  }
  auto turn = [&](unsigned char *sq, unsigned char *nq) {
    wait_memory();
    if (!SPLIT) __syncthreads();
    own_now = own;
    lse_now = lse_x;
    if (r0 + kRows < n_rows) {
      issue(nq, r0 + kRows);
      lookup();
    }
#pragma unroll
    for (int blk = 0; blk < (SPLIT ? 1 : kRows / 32); ++blk) {
      const int row = 32 * (SPLIT ? wave : blk) + (lane & 31), z = L::swz_k(row);
      const int o = SPLIT ? own_now : __shfl(own_now, row, kWave);
      const float base = SPLIT ? lse_now : __shfl(lse_now, row, kWave);
      f32x16_t x = {};
#pragma unroll
      for (int i = 0; i < kFrag; ++i) {
        const int c = kBf16 ? 2 * i + half : half * kFrag + i;
        const uint4 w = *reinterpret_cast<const uint4 *>(sq + (row * L::bytes + ((c ^ z) << 4)));
        if constexpr (kBf16) {
          x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[i]),
                                                      __builtin_bit_cast(bf16x8_t, w), x, 0, 0, 0);
        } else {
          const f32x4_t ka = __builtin_bit_cast(f32x4_t, kf[i]), qa = __builtin_bit_cast(f32x4_t, w);
#pragma unroll
          for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(ka[e], qa[e], x, 0, 0, 0);
        }
      }
      if (__any(o < key0 + 31)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key0 + 8 * (i / 4) + i % 4 + 4 * half;
          const float p = weight_of<T>(a, x[i], base);
          acc[i] += key <= o ? p : 0.0f;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] += weight_of<T>(a, x[i], base);
      }
    }
    r0 += kRows;
  };
  while (r0 < n_rows) {
    turn(q0, q1);
    if (r0 >= n_rows) break;
    turn(q1, q0);
  }
  float sum = sum_rows<32>(acc);
  if (SPLIT) {
    float *part = reinterpret_cast<float *>(q0);
    wait_memory();
    __syncthreads();
    part[threadIdx.x] = sum;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 1; w < kNW; ++w) sum += part[w * kWave + lane];
  }
  // bits 4..1 of the lane are the register's bits 3..0
  const int i = (lane & 31) >> 1, in = 8 * (i / 4) + i % 4 + 4 * half, key = key0 + in;
  if (!(lane & 1) && key < s.len) {
    const int64_t at = b * a.seq_stride + (PER_KV ? kvh : head0) * a.rows + key;
    const float old = a.before && key < pos0 ? a.before[at] : 0.0f;
    a.out[at] = old + (exists >> in & 1u ? sum : 0.0f);
  }
}

// Per query head.  A tile of 64 query rows is 64 tokens of a head, or, where no sequence
// has more than P < 64, the tokens of 64 / P heads; a workgroup keeps its keys for up to
// kWalk heads (or such groups of heads), whose sums wait in LDS for the end (a store
// between tiles would be waited for with the next tile's copies).
constexpr int kWalk = 4;

template <typename T, int D, int P>
__global__ __launch_bounds__(kNW * kWave, 2) void head_scores(ScoreArgs a) {
  using L = TileLayout<T, D>;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kFrag = kBf16 ? D / 16 : D / 8;  // 16-byte pieces of a row per lane
  constexpr int kHeads = 64 / P, kShare = 64 / kNW, kRpi = 64 / L::C, kInstr = kShare / kRpi;
  constexpr int kSums = P < 64 ? 2 : 1;  // of a lane per tile
  __shared__ __align__(16) unsigned char q0[64 * L::bytes], q1[64 * L::bytes];
  __shared__ float sums[kWalk * kSums][kNW * kWave];  // the lanes' own
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int per = (a.g + a.walk * kHeads - 1) / (a.walk * kHeads);  // workgroups that share a kv head
  const int units = a.c.batch * a.hkv * per, unit = blockIdx.x % units;
  const int b = unit / (a.hkv * per), kvh = unit / per % a.hkv;
  const Seq s = sequence(a.c, b, a.kv.cap);
  const int block0 = (blockIdx.x / units) * 32 * kNW, key0 = block0 + wave * 32;
  if (block0 >= s.len) return;
  const int pos0 = s.len - s.n_new;
  const int in_group = unit % per * a.walk * kHeads, n_heads = min(a.walk * kHeads, a.g - in_group);
  const int head0 = kvh * a.g + in_group;
  const int first = max(0, block0 - pos0);  // the first token that sees a key of the workgroup
  const int n_tokens = s.n_new - first;

  uint4 kf[kFrag];
  uint32_t exists;
  {
    const int key = key0 + (lane & 31);
    const int64_t off = key < s.len ? row_offset(a.kv, b, key) : -1;
    const unsigned char *row = off >= 0 ? a.kv.k + off + (((uint64_t)kvh * a.kv.head_stride) << 4) : zero_row;
#pragma unroll
    for (int i = 0; i < kFrag; ++i)
      kf[i] = reinterpret_cast<const uint4 *>(row)[kBf16 ? 2 * i + half : half * kFrag + i];
    exists = (uint32_t)__ballot(off >= 0);
  }
  // Row r of tile t of head group h: token 64 t + r % P of head h * kHeads + r / P; past
  // the last, one that exists.
  const int groups = (n_heads + kHeads - 1) / kHeads, tiles = P < 64 ? 1 : (n_tokens + 63) / 64;
  auto head_of = [&](int h, int r) { return min(h * kHeads + r / P, n_heads - 1); };
  auto token_of = [&](int t, int r) { return min(64 * t + (r & (P - 1)), n_tokens - 1); };
  auto issue = [&](int h, int t, unsigned char *dst) {
    const int rr = lane / L::C, p = lane & (L::C - 1);
#pragma unroll
    for (int j = 0; j < kInstr; ++j) {
      const int r = wave * kShare + j * kRpi + rr;
      const unsigned char *row = a.q + (int64_t)(s.first + first + token_of(t, r)) * a.q_token +
                                 (int64_t)(head0 + head_of(h, r)) * a.q_head;
      load_to_lds16(row + ((p ^ L::swz_k(r)) << 4), dst + (wave * kShare + j * kRpi) * L::bytes);
    }
  };
  if (n_tokens > 0) {
    float lse = 0.0f;
    auto lookup = [&](int h, int t) {
      lse = a.lse[(int64_t)(s.first + first + token_of(t, lane)) * a.hq + head0 + head_of(h, lane)];
    };
    float acc[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
    int h = 0, t = 0;  // the tile that is computed
    auto turn = [&](unsigned char *sq, unsigned char *nq) {
      wait_memory();
      __syncthreads();
      // own: the row's cached row; -1, which gives no weight: past the last, or sees no key
      const int token = 64 * t + (lane & (P - 1));
      const bool dead = token >= n_tokens || lse == -INFINITY;
      const int own = dead ? -1 : pos0 + first + token;
      const float lse_x = dead ? 0.0f : lse_of<T>(lse);
      const bool last = t + 1 == tiles;
      const int h_next = last ? h + 1 : h, t_next = last ? 0 : t + 1;
      if (h_next < groups) {
        issue(h_next, t_next, nq);
        lookup(h_next, t_next);
      }
      // the weights of 32 query rows, added to acc
      auto weigh = [&](int blk) {
        const int row = 32 * blk + (lane & 31), z = L::swz_k(row);
        const int o = __shfl(own, row, kWave);
        const float base = __shfl(lse_x, row, kWave);
        f32x16_t x = {};
#pragma unroll
        for (int i = 0; i < kFrag; ++i) {
          const int c = kBf16 ? 2 * i + half : half * kFrag + i;
          const uint4 w = *reinterpret_cast<const uint4 *>(sq + (row * L::bytes + ((c ^ z) << 4)));
          if constexpr (kBf16) {
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[i]),
                                                        __builtin_bit_cast(bf16x8_t, w), x, 0, 0, 0);
          } else {
            const f32x4_t ka = __builtin_bit_cast(f32x4_t, kf[i]), qa = __builtin_bit_cast(f32x4_t, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(ka[e], qa[e], x, 0, 0, 0);
          }
        }
        if (__any(o < key0 + 31)) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = key0 + 8 * (i / 4) + i % 4 + 4 * half;
            const float p = weight_of<T>(a, x[i], base);
            acc[i] += key <= o ? p : 0.0f;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[i] += weight_of<T>(a, x[i], base);
        }
      };
      weigh(0);
      if constexpr (P < 64) {
        sums[2 * h][threadIdx.x] = sum_rows<P>(acc);
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
      }
      weigh(1);
      if (last) {
        sums[P < 64 ? 2 * h + 1 : h][threadIdx.x] = sum_rows<P == 16 ? 16 : 32>(acc);
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
      }
      h = h_next;
      t = t_next;
    };
    issue(0, 0, q0);
    lookup(0, 0);
    while (true) {
      turn(q0, q1);
      if (h >= groups) break;
      turn(q1, q0);
      if (h >= groups) break;
    }
  }
  const int k = P == 16 ? lane & 15 : (lane & 31) >> 1, in = 8 * (k / 4) + k % 4 + 4 * half, key = key0 + in;
  const bool writes = (P == 16 || !(lane & 1)) && key < s.len;
  // all old scores, then all new ones (which may be the same memory)
  float old[kWalk * kSums];
  // the head of a tile's sum of this lane
  auto head = [&](int n) { return n / kSums * kHeads + (P == 64 ? 0 : P == 32 ? n % 2 : n % 2 * 2 + (lane >> 4 & 1)); };
  auto at = [&](int n) { return b * a.seq_stride + (head0 + head(n)) * a.rows + key; };
#pragma unroll
  for (int n = 0; n < kWalk * kSums; ++n)
    old[n] = writes && head(n) < n_heads && a.before && key < pos0 ? a.before[at(n)] : 0.0f;
#pragma unroll
  for (int n = 0; n < kWalk * kSums; ++n)
    if (writes && head(n) < n_heads)
      a.out[at(n)] = old[n] + (n_tokens > 0 && exists >> in & 1u ? sums[n][threadIdx.x] : 0.0f);
}

template <typename T, int D>
__global__ __launch_bounds__(kNW * kWave, 2) void few_scores(ScoreArgs a) {
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kFrag = kBf16 ? D / 16 : D / 8;  // 16-byte pieces of a row per lane
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int units = a.c.batch * a.hkv, unit = blockIdx.x % units;
  const int b = unit / a.hkv, kvh = unit % a.hkv;
  const Seq s = sequence(a.c, b, a.kv.cap);
  // whole rounds of 128 keys, as many to each workgroup as the sequence's own length asks
  // for (16 sequences of 4000 rows in a call for up to 131072: 6.4 us; with a share of
  // max_len each 27.8)
  const int share = ((s.len + 127) / 128 + a.pieces - 1) / a.pieces * 128;
  const int64_t from = (int64_t)(blockIdx.x / units) * share;
  if (from >= s.len) return;
  const int begin = (int)from, end = min(begin + share, s.len);
  const int pos0 = s.len - s.n_new, rows = s.n_new * a.g;
  const unsigned char *k = a.kv.k + (((uint64_t)kvh * a.kv.head_stride) << 4);
  // keys are looked up two blocks ahead and their rows requested one ahead
  const int32_t *pages = a.kv.table ? a.kv.table + (int64_t)b * a.kv.width : a.c.len;
  auto page_of = [&](int key) { return pages[min(key, s.len - 1) >> a.kv.shift]; };  // (dense: any word)
  auto offset_of = [&](int key, int page) {
    const int64_t off = page_offset(a.kv, a.kv.table ? page : b, key);
    return key < end ? off : -1;
  };
  constexpr int step = 32 * kNW;
  int key = begin + wave * 32 + (lane & 31);
  int page = page_of(key), page_next = page_of(key + step);

  // the lane's query row, and the lse (see lse_of) and own cached row of the 16 rows
  // whose logits it will hold
  uint4 qf[kFrag];
  {
    // rows past the last repeat the first, so that no product of theirs is NaN where
    // the others' are not (of keys with infinities)
    const int r = (lane & 31) < rows ? lane & 31 : 0;
    const int64_t t = s.first + r / a.g, h = kvh * a.g + r % a.g;
    const unsigned char *row = rows > 0 ? a.q + t * a.q_token + h * a.q_head : zero_row;
#pragma unroll
    for (int i = 0; i < kFrag; ++i)
      qf[i] = reinterpret_cast<const uint4 *>(row)[kBf16 ? 2 * i + half : half * kFrag + i];
  }
  float lse_x[16];
  int own[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = 8 * (i / 4) + i % 4 + 4 * half;
    lse_x[i] = INFINITY;  // rows past the last, and rows that see no key, give no weight
    own[i] = -1;
    if (r < rows) {
      const float x = a.lse[(int64_t)(s.first + r / a.g) * a.hq + kvh * a.g + r % a.g];
      if (x != -INFINITY) {
        lse_x[i] = lse_of<T>(x);
        own[i] = pos0 + r / a.g;
      }
    }
  }
  int64_t off = offset_of(key, page);
  uint4 kf[kFrag];
  auto load = [&]() {
    const unsigned char *row = off >= 0 ? k + off : zero_row;
#pragma unroll
    for (int i = 0; i < kFrag; ++i)
      kf[i] = reinterpret_cast<const uint4 *>(row)[kBf16 ? 2 * i + half : half * kFrag + i];
  };
  load();
  for (int base = begin + wave * 32; base < end; base += step, key += step) {
    f32x16_t x = {};
#pragma unroll
    for (int i = 0; i < kFrag; ++i) {
      if constexpr (kBf16) {
        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, qf[i]),
                                                    __builtin_bit_cast(bf16x8_t, kf[i]), x, 0, 0, 0);
      } else {
        const f32x4_t qa = __builtin_bit_cast(f32x4_t, qf[i]), ka = __builtin_bit_cast(f32x4_t, kf[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(qa[e], ka[e], x, 0, 0, 0);
      }
    }
    const bool exists = off >= 0, inside = key < end;
    page = page_next;
    off = offset_of(key + step, page);
    load();
    page_next = page_of(key + 2 * step);
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = weight_of<T>(a, x[i], lse_x[i]);
    if (base + 31 > pos0 || rows == 0 || __any(!exists)) {  // some row may not see some key
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = exists && key <= own[i] ? p[i] : 0.0f;
    }
    if (a.per_kv) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum += p[i];
      sum = swap_halves_sum(sum);
      if (half == 0 && inside) {
        const int64_t at = b * a.seq_stride + kvh * a.rows + key;
        a.out[at] = (a.before && key < pos0 ? a.before[at] : 0.0f) + sum;
      }
    } else {
      // rows of head j: j, j + g, j + 2g, ...
      for (int j = 0; j < a.g; ++j) {
        float sum = 0.0f;
        if (s.n_new == 1) {
#pragma unroll
          for (int i = 0; i < 16; ++i) sum = j == 8 * (i / 4) + i % 4 + 4 * half ? p[i] : sum;
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) sum += (8 * (i / 4) + i % 4 + 4 * half) % a.g == j ? p[i] : 0.0f;
        }
        sum = swap_halves_sum(sum);
        if (half == 0 && inside) {
          const int64_t at = b * a.seq_stride + (kvh * a.g + j) * a.rows + key;
          a.out[at] = (a.before && key < pos0 ? a.before[at] : 0.0f) + sum;
        }
      }
    }
  }
}

template <typename T, int D, bool PER_KV, bool SPLIT> void launch_chunk(const ScoreArgs &a, dim3 grid, hipStream_t st) {
  hipLaunchKernelGGL((chunk_scores<T, D, PER_KV, SPLIT>), grid, dim3(kNW * kWave), 0, st, a);
}

template <typename T, int D>
void launch_typed(ScoreArgs a, int max_new, int max_len, hipStream_t st) {
  const int64_t units = (int64_t)a.c.batch * a.hkv;
  const dim3 block(kNW * kWave);
  auto blocks = [&](int keys) { return (unsigned)(((int64_t)max_len + keys - 1) / keys * units); };
  if ((int64_t)max_new * a.g <= 32) {
    // two workgroups per CU, of whole rounds of 128 keys (a batch-16 step over up to
    // 8192 rows: 9.6 us with 512, 11.6 with 1024, 12.1 with 256)
    const int64_t rounds = ((int64_t)max_len + 127) / 128;
    const int64_t each = std::max<int64_t>(1, std::min<int64_t>(rounds, rounds * units / 512));
    a.pieces = (int)((rounds + each - 1) / each);
    hipLaunchKernelGGL((few_scores<T, D>), dim3((unsigned)(a.pieces * units)), block, 0, st, a);
    return;
  }
  const unsigned heads = a.per_kv ? 1 : a.g;
  if (!a.per_kv && max_new <= 128) {
    // (8 sequences of 8192 rows, 32 query heads: 9 tokens 35 us, 120 as a chunk; 64 tokens
    // 73, 119; 128 tokens 114, 155; with 226 tokens and more no faster, 2048 214 against
    // 203.)  More heads to a workgroup while four workgroups per CU are left (30 sequences
    // of 600 rows and 64 heads, 12 tokens: 19 us, 24 with a tile each).
    const int packed = max_new <= 16 ? 4 : max_new <= 32 ? 2 : 1, tiles = ((int)heads + packed - 1) / packed;
    const int64_t pieces = blocks(32 * kNW);
    a.walk = std::min(tiles, kWalk);
    while (a.walk > 1 && pieces * ((tiles + a.walk - 1) / a.walk) < 1024) --a.walk;
    const dim3 grid((unsigned)(pieces * ((tiles + a.walk - 1) / a.walk)));
    auto *kernel = packed == 4 ? head_scores<T, D, 16> : packed == 2 ? head_scores<T, D, 32> : head_scores<T, D, 64>;
    hipLaunchKernelGGL(kernel, grid, block, 0, st, a);
    return;
  }
  // with less than a workgroup per CU (2048 tokens over 8192 rows, two kv heads, 128
  // workgroups: 175 us, split 84; 512 tokens, four, 256 workgroups: 68, split 72)
  const bool split = blocks(32 * kNW) * (int64_t)heads < 256;
  const dim3 grid(blocks(split ? 32 : 32 * kNW) * heads);
  (split ? a.per_kv ? launch_chunk<T, D, true, true> : launch_chunk<T, D, false, true>
   : a.per_kv ? launch_chunk<T, D, true, false> : launch_chunk<T, D, false, false>)(a, grid, st);
}

}  // namespace

hipError_t launch_chunk_scores(const smallkv_chunk_t &c, const smallkv_cache_t &kv, const smallkv_queries_t &q,
                               int n_score_heads, const float *before, float *out, int64_t score_rows,
                               int64_t seq_stride, hipStream_t st) {
  const int e = kv.dtype == SMALLKV_F32 ? 4 : 2;
  ScoreArgs a{};
  a.c = chunk_view(c);
  a.kv = cache_view(kv);
  a.hq = q.n_heads;
  a.hkv = kv.n_heads;
  a.g = q.n_heads / kv.n_heads;
  a.per_kv = n_score_heads != q.n_heads;
  a.q = static_cast<const unsigned char *>(q.q);
  a.q_token = q.token_stride * e;
  a.q_head = q.head_stride * e;
  a.lse = q.lse;
  a.before = before;
  a.out = out;
  a.rows = score_rows;
  a.seq_stride = seq_stride;
  a.scale = e == 4 ? q.scale : q.scale * kLog2e;
  if (kv.dtype == SMALLKV_F32)
    (kv.head_dim == 64 ? launch_typed<float, 64> : launch_typed<float, 128>)(a, c.max_new, c.max_len, st);
  else
    (kv.head_dim == 64 ? launch_typed<bf16_t, 64> : launch_typed<bf16_t, 128>)(a, c.max_new, c.max_len, st);
  return hipGetLastError();
}

}  // namespace smallkv
