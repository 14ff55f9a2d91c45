// Eviction from a cache by accumulated attention weight.
//
//   evict_select -- one workgroup per (sequence, kv head): the rows' summed
//                   scores as order-preserving 32-bit keys, the exact threshold
//                   of the top ones by a radix descent of 8 bits a pass
//                   (histograms in LDS), then the kept rows in ascending order,
//                   ties to the lowest rows, with their positions and scores;
//   evict_copy   -- the kept rows as a flat array of 16-byte pieces, K and V.
#include <algorithm>

#include "cache.h"
#include "launch.h"

namespace smallkv {
namespace {

constexpr int kST = 1024, kSW = kST / kWave;  // evict_select threads, waves
constexpr int kCT = 256;                      // evict_copy threads

struct EvictArgs {
  int batch, max_len, heads, gs, sinks;
  const int32_t *len, *keep, *recent;
  CacheView from, to;
  unsigned char *to_k, *to_v;
  int row_bytes;
  const float *scores;
  int64_t score_rows;
  const int32_t *row_pos;
  int64_t pos_rows, out_rows;
  float *out_scores;
  int32_t *out_pos, *held;
  int32_t *src;  // [batch * heads][cap]
  int64_t cap;   // rows a sequence can keep
};

struct Budget {
  int n, kept, last, first;
};
__device__ __forceinline__ Budget budget(const EvictArgs &a, int b) {
  Budget x;
  x.n = clampi(a.len[b], 0, min(a.max_len, a.from.cap));
  x.kept = (int)min<int64_t>(clampi(a.keep[b], 0, x.n), a.cap);
  x.last = a.recent ? clampi(a.recent[b], 0, x.kept) : 0;
  x.first = min(a.sinks, x.kept - x.last);
  return x;
}

// Larger key: kept earlier.  NaN below every number.
__device__ __forceinline__ uint32_t score_key(const float *p, int64_t stride, int gs) {
  float f = p[0];
  for (int i = 1; i < gs; ++i) f += p[i * stride];
  return f != f ? 0u : logit_key(f);
}

__global__ __launch_bounds__(kST) void evict_select(EvictArgs a) {
  __shared__ uint32_t hist[kSW][256];
  __shared__ uint32_t total[256];
  __shared__ uint32_t pick[2];  // the digit, and how many are still wanted within it
  __shared__ int cnt[2][kSW];
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int unit = blockIdx.x, b = unit / a.heads, h = unit % a.heads;
  const Budget x = budget(a, b);
  if (h == 0 && threadIdx.x == 0) a.held[b] = x.kept;
  const float *f = a.scores + ((int64_t)b * a.heads + h) * a.gs * a.score_rows;
  const int lo = x.first, hi = x.n - x.last;  // ranked rows
  const uint32_t top = x.kept - x.last - x.first;
  uint32_t prefix = 0, want = top;
  if (top > 0 && top < (uint32_t)(hi - lo)) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = threadIdx.x; i < kSW * 256; i += kST) hist[i / 256][i % 256] = 0;
      __syncthreads();
      for (int r = lo + threadIdx.x; r < hi; r += kST) {
        const uint32_t k = score_key(f + r, a.score_rows, a.gs);
        if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&hist[wave][k >> shift & 255u], 1u);
      }
      __syncthreads();
      if (threadIdx.x < 256) {
        uint32_t t = 0;
        for (int w = 0; w < kSW; ++w) t += hist[w][threadIdx.x];
        total[threadIdx.x] = t;
      }
      __syncthreads();
      if (wave == 0) {
        // bins from the top: lane l holds bins 255-4l .. 252-4l
        uint32_t v[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += v[i] = total[255 - 4 * lane - i];
        uint32_t s = sum;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
          const uint32_t y = __shfl_up(s, o, kWave);
          if (lane >= o) s += y;
        }
        uint32_t above = s - sum;
        if (above < want && s >= want) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (above < want && above + v[i] >= want) {
              pick[0] = 255 - 4 * lane - i;
              pick[1] = want - above;
            }
            above += v[i];
          }
        }
      }
      __syncthreads();
      prefix = prefix << 8 | pick[0];
      want = pick[1];
      __syncthreads();
    }
  } else {
    prefix = top ? 0u : 0xffffffffu;  // every ranked row, or none (no key is all ones)
    want = top;
  }
  // each wave walks its own run of rows; how many the runs before it keep
  const int per = ((x.n + kSW - 1) / kSW + kWave - 1) / kWave * kWave;
  const int r0 = min(wave * per, x.n), r1 = min(r0 + per, x.n);
  int sure = 0, ties = 0;
  for (int r = r0; r < r1; r += kWave) {
    const int row = r + lane;
    bool yes = false, tie = false;
    if (row < r1) {
      yes = row < lo || row >= hi;
      if (!yes) {
        const uint32_t k = score_key(f + row, a.score_rows, a.gs);
        yes = k > prefix;
        tie = k == prefix;
      }
    }
    sure += __popcll(__ballot(yes));
    ties += __popcll(__ballot(tie));
  }
  if (lane == 0) {
    cnt[0][wave] = sure;
    cnt[1][wave] = ties;
  }
  __syncthreads();
  int at = 0, before = 0;  // kept rows and ties of the runs before
  for (int w = 0; w < wave; ++w) {
    at += cnt[0][w];
    before += cnt[1][w];
  }
  at += min(before, (int)want);
  const uint64_t below = (1ull << lane) - 1;
  for (int r = r0; r < r1; r += kWave) {
    const int row = r + lane;
    bool yes = false, tie = false;
    if (row < r1) {
      yes = row < lo || row >= hi;
      if (!yes) {
        const uint32_t k = score_key(f + row, a.score_rows, a.gs);
        yes = k > prefix;
        tie = k == prefix;
      }
    }
    const uint64_t mt = __ballot(tie);
    yes |= tie && before + __popcll(mt & below) < (int)want;
    const uint64_t m = __ballot(yes);
    if (yes) {
      const int64_t to = at + __popcll(m & below);
      a.src[unit * a.cap + to] = row;
      a.out_pos[unit * a.out_rows + to] = a.row_pos ? a.row_pos[unit * a.pos_rows + row] : row;
      if (a.out_scores)
        for (int i = 0; i < a.gs; ++i)
          a.out_scores[((int64_t)unit * a.gs + i) * a.out_rows + to] = f[i * a.score_rows + row];
    }
    at += __popcll(m);
    before += __popcll(mt);
  }
}

// blockIdx.x: (sequence, kv head); blockIdx.y: interleaved shares of the pieces;
// blockIdx.z: K (0) or V (1).
constexpr int kShares = 32;

__global__ __launch_bounds__(kCT) void evict_copy(EvictArgs a) {
  const int unit = blockIdx.x, b = unit / a.heads, h = unit % a.heads;
  const Budget x = budget(a, b);
  const int psh = 31 - __clz(a.row_bytes / 16);
  const int64_t items = (int64_t)x.kept << psh;
  const unsigned char *from = (blockIdx.z ? a.from.v : a.from.k) + (((uint64_t)h * a.from.head_stride) << 4);
  unsigned char *to = (blockIdx.z ? a.to_v : a.to_k) + (((uint64_t)h * a.to.head_stride) << 4);
  for (int64_t q = blockIdx.y * kCT + threadIdx.x; q < items; q += kShares * kCT) {
    const int r = (int)(q >> psh), p = (int)(q & ((1 << psh) - 1));
    const int64_t s = row_offset(a.from, b, a.src[unit * a.cap + r]), d = row_offset(a.to, b, r);
    if (s < 0 || d < 0) continue;
    reinterpret_cast<uint4 *>(to + d)[p] = reinterpret_cast<const uint4 *>(from + s)[p];
  }
}

int64_t kept_cap(const smallkv_evict_t &e) {
  const int64_t cap = cache_view(e.to).cap;
  return std::min(std::min(cap, e.out_rows), (int64_t)e.max_len);
}

}  // namespace

size_t evict_workspace(const smallkv_evict_t &e) {
  return (size_t)e.batch * e.from.n_heads * kept_cap(e) * sizeof(int32_t);
}

hipError_t launch_evict(const smallkv_evict_t &e, void *ws, hipStream_t st) {
  EvictArgs a{};
  a.batch = e.batch;
  a.max_len = e.max_len;
  a.heads = e.from.n_heads;
  a.gs = e.n_score_heads / e.from.n_heads;
  a.sinks = e.sinks;
  a.len = e.len;
  a.keep = e.keep;
  a.recent = e.recent;
  a.from = cache_view(e.from);
  a.to = cache_view(e.to);
  a.to_k = static_cast<unsigned char *>(e.to.k);
  a.to_v = static_cast<unsigned char *>(e.to.v);
  a.row_bytes = e.from.head_dim * (e.from.dtype == SMALLKV_F32 ? 4 : 2);
  a.scores = e.scores;
  a.score_rows = e.score_rows;
  a.row_pos = e.row_pos;
  a.pos_rows = e.pos_rows;
  a.out_rows = e.out_rows;
  a.out_scores = e.out_scores;
  a.out_pos = e.out_pos;
  a.held = e.held;
  a.src = static_cast<int32_t *>(ws);
  a.cap = kept_cap(e);
  const unsigned units = (unsigned)(e.batch * e.from.n_heads);
  hipLaunchKernelGGL(evict_select, dim3(units), dim3(kST), 0, st, a);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL(evict_copy, dim3(units, kShares, 2), dim3(kCT), 0, st, a);
  return hipGetLastError();
}

}  // namespace smallkv
