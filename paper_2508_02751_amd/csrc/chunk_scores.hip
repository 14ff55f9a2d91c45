// The attention weight that the new tokens give every cached row, added to its
// running score: out[r] = before[r] + sum over (token, head) of exp(s - lse).
//
// A workgroup owns 128 keys of one kv head (32 per wave, their K rows in
// registers as the left operand of S^T = K Q^T) and walks the query rows that
// see them, 64 at a time through LDS, so no sum leaves its workgroup: no
// atomics, one order, and the logits are never stored.  A lane holds one query
// row's logits of 16 keys: one fused multiply-add, one exponential and one add
// each, which bound the pass (an exponential takes four times an add; the
// product's matrix instructions run beside them).
//
// Scores per query head: the heads are dealt to workgroups (blockIdx.y), each
// walking one head's tokens; per kv head: the rows are (token, head) pairs.
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
  int64_t rows;   // of before and out
  float scale2;   // scale * log2(e)
};

constexpr float kLog2e = 1.4426950408889634074f;
constexpr int kNW = 4, kKeys = 32 * kNW, kRows = 64;

template <typename T, int D>
__global__ __launch_bounds__(kNW * kWave) void chunk_scores(ScoreArgs a) {
  using L = TileLayout<T, D>;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kFrag = kBf16 ? D / 16 : D / 8;  // 16-byte pieces of a row per lane
  constexpr int kBuf = kRows * L::bytes, kShare = kRows / kNW, kRpi = 64 / L::C, kInstr = kShare / kRpi;
  __shared__ __align__(16) unsigned char q0[kBuf], q1[kBuf];
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int units = a.c.batch * a.hkv, unit = blockIdx.x % units;
  const int b = unit / a.hkv, kvh = unit % a.hkv;
  const Seq s = sequence(a.c, b, a.kv.cap);
  const int block0 = (blockIdx.x / units) * kKeys, key0 = block0 + wave * 32;
  if (block0 >= s.len) return;
  const int pos0 = s.len - s.n_new;
  // per query head: this head's tokens; per kv head: (token, head) pairs
  const int g = a.per_kv ? a.g : 1, head0 = kvh * a.g + (a.per_kv ? 0 : (int)blockIdx.y);
  const int first = max(0, block0 - pos0);  // the first token that sees a key of the workgroup
  const int n_rows = (s.n_new - first) * g;

  uint4 kf[kFrag];
  bool valid;
  {
    const int key = key0 + (lane & 31);
    const int64_t off = key < s.len ? row_offset(a.kv, b, key) : -1;
    valid = off >= 0;
    const unsigned char *row = valid ? a.kv.k + off + (((uint64_t)kvh * a.kv.head_stride) << 4) : zero_row;
#pragma unroll
    for (int i = 0; i < kFrag; ++i)
      kf[i] = reinterpret_cast<const uint4 *>(row)[kBf16 ? 2 * i + half : half * kFrag + i];
  }
  const uint32_t exists = (uint32_t)__ballot(valid);

  float acc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.0f;

  // the lane's row of the looked-up tile: its queries, own cached row (-1: none)
  // and the lse in log2 units (its rows beyond the last give no weight)
  int64_t off;
  int own;
  float lse2;
  auto lookup = [&](int r0) {
    const int r = r0 + lane;
    off = -1;
    own = -1;
    lse2 = 0.0f;
    if (r < n_rows) {
      const int i = first + (g == 1 ? r : r / g), h = head0 + (g == 1 ? 0 : r % g);
      const int64_t t = s.first + i;
      off = t * a.q_token + h * a.q_head;
      lse2 = a.lse[t * a.hq + h] * kLog2e;
      own = lse2 == -INFINITY ? -1 : pos0 + i;
    }
  };
  auto issue = [&](unsigned char *dst) {
    const int rr = lane / L::C, p = lane & (L::C - 1);
#pragma unroll
    for (int j = 0; j < kInstr; ++j) {
      const int r = wave * kShare + j * kRpi + rr;
      const int lo = __shfl((int)off, r, kWave), hi = __shfl((int)(off >> 32), r, kWave);
      const int64_t o = ((int64_t)hi << 32) | (uint32_t)lo;
      const unsigned char *src = hi < 0 ? zero_row : a.q + o;
      load_to_lds16(src + ((p ^ L::swz_k(r)) << 4), dst + (wave * kShare + j * kRpi) * L::bytes);
    }
  };
  int r0 = 0, own_now, own_next = 0;
  float lse_now, lse_next = 0.0f;
  lookup(0);
  if (n_rows > 0) {
    issue(q0);
    own_next = own;
    lse_next = lse2;
    lookup(kRows);
  }
  auto turn = [&](unsigned char *sq, unsigned char *nq) {
    wait_memory();
    __syncthreads();
    own_now = own_next;
    lse_now = lse_next;
    if (r0 + kRows < n_rows) {
      issue(nq);
      own_next = own;
      lse_next = lse2;
      lookup(r0 + 2 * kRows);
    }
#pragma unroll
    for (int blk = 0; blk < kRows / 32; ++blk) {
      const int row = 32 * blk + (lane & 31), z = L::swz_k(row);
      const int o = __shfl(own_now, row, kWave);
      const float base = __shfl(lse_now, row, kWave);
      f32x16_t x = {};
#pragma unroll
      for (int i = 0; i < kFrag; ++i) {
        const int c = kBf16 ? 2 * i + half : half * kFrag + i;
        const uint4 w = *reinterpret_cast<const uint4 *>(sq + row * L::bytes + ((c ^ z) << 4));
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
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale2, -base));
          acc[i] += key <= o ? p : 0.0f;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale2, -base));
      }
    }
    r0 += kRows;
  };
  while (r0 < n_rows) {
    turn(q0, q1);
    if (r0 >= n_rows) break;
    turn(q1, q0);
  }
  // sums over the 32 query rows: each exchange halves the keys a lane holds
#pragma unroll
  for (int n = 8, o = 16; n >= 1; n >>= 1, o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) {
        const float send = up ? acc[i] : acc[i + n], keep = up ? acc[i + n] : acc[i];
        acc[i] = keep + __shfl_xor(send, o, kWave);
      }
  }
  const float sum = acc[0] + __shfl_xor(acc[0], 1, kWave);
  // bits 4..1 of the lane are the register's bits 3..0
  const int i = (lane & 31) >> 1, in = 8 * (i / 4) + i % 4 + 4 * half, key = key0 + in;
  if (!(lane & 1) && key < s.len) {
    const int64_t at = ((int64_t)b * (a.per_kv ? a.hkv : a.hq) + (a.per_kv ? kvh : head0)) * a.rows + key;
    const float old = a.before && key < pos0 ? a.before[at] : 0.0f;
    a.out[at] = old + (exists >> in & 1u ? sum : 0.0f);
  }
}

}  // namespace

hipError_t launch_chunk_scores(const smallkv_chunk_t &c, const smallkv_cache_t &kv, const smallkv_queries_t &q,
                               int n_score_heads, const float *before, float *out, int64_t score_rows,
                               hipStream_t st) {
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
  a.scale2 = q.scale * kLog2e;
  const dim3 grid((unsigned)((c.max_len + kKeys - 1) / kKeys * c.batch * kv.n_heads), a.per_kv ? 1 : a.g);
  if (kv.dtype == SMALLKV_F32) {
    if (kv.head_dim == 64)
      hipLaunchKernelGGL((chunk_scores<float, 64>), grid, dim3(kNW * kWave), 0, st, a);
    else
      hipLaunchKernelGGL((chunk_scores<float, 128>), grid, dim3(kNW * kWave), 0, st, a);
  } else if (kv.head_dim == 64) {
    hipLaunchKernelGGL((chunk_scores<bf16_t, 64>), grid, dim3(kNW * kWave), 0, st, a);
  } else {
    hipLaunchKernelGGL((chunk_scores<bf16_t, 128>), grid, dim3(kNW * kWave), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace smallkv
