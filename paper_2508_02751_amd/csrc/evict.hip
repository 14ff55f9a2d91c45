// Eviction from a cache by accumulated attention weight.
//
//   evict_select -- one workgroup of one to sixteen waves per (sequence, kv head):
//                   the rows' summed scores as order-preserving 32-bit keys, read once
//                   and kept in registers (up to 32768 rows; longer rows are read again
//                   by every pass), the exact threshold of the top ones by counting
//                   passes, then the kept rows' numbers in ascending order, ties to
//                   the lowest rows;
//   evict_copy   -- the kept rows as a flat array of 16-byte pieces, K and V, and
//                   their positions and scores.
//
// Measured (MI355X): 4 sequences of 20000 - 32768 rows, 16 layers of 8 kv heads of 64,
// 20% kept (1.4 GB read and written): 57 + 299 us, the copy at the rate of a large copy,
// the selection by its passes over the registers; 24 layers of 8192 rows, 40% kept, the
// scores of 7 query heads added up: 12 + 17 us; one layer of 1237 rows: 6.4 + 2.8 us, two
// launches and the selection's barriers.
#include <algorithm>

#include "cache.h"
#include "launch.h"

namespace smallkv {
namespace {

constexpr int kCT = 256;  // evict_copy threads

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

// Threads of evict_select hold KPT keys each, wave by wave in runs of rows: key j
// of a lane is row (wave * KPT + j) * 64 + lane.  KPT 0: the rows are read anew.
template <int KPT> struct Keys {
  uint32_t k[KPT];
  __device__ __forceinline__ void load(const EvictArgs &a, const float *f, int r0, int lo, int hi) {
    const int lane = threadIdx.x & (kWave - 1);
    float s[KPT];
    for (int i = 0; i < a.gs; ++i, f += a.score_rows) {
      uint32_t row = r0 + lane;
      asm volatile("" : "+v"(row));
#pragma unroll
      for (int j = 0; j < KPT; ++j) {
        const float x = f[min(row + j * kWave, (uint32_t)max(hi - 1, 0))];
        s[j] = i ? s[j] + x : x;
        if (j % 16 == 15) __builtin_amdgcn_sched_barrier(0);  // (loads in flight at a time)
      }
    }
#pragma unroll
    for (int j = 0; j < KPT; ++j) k[j] = s[j] != s[j] ? 0u : logit_key(s[j]);
  }
  template <typename F> __device__ __forceinline__ void each(const EvictArgs &, const float *, int r0, int, F &&use) const {
    int row = r0 + (int)(threadIdx.x & (kWave - 1));
    asm volatile("" : "+v"(row));  // (the rows' numbers are not kept between passes)
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
      use(row + j * kWave, k[j]);
      if (KPT > 8) __builtin_amdgcn_sched_barrier(0);  // (few masks alive at a time)
    }
  }
};
template <> struct Keys<0> {
  __device__ __forceinline__ void load(const EvictArgs &, const float *, int, int, int) {}
  template <typename F>
  __device__ __forceinline__ void each(const EvictArgs &a, const float *f, int r0, int r1, F &&use) const {
    for (int r = r0; r < r1; r += kWave) {
      const int row = r + (int)(threadIdx.x & (kWave - 1));
      use(row, score_key(f + min(row, r1 - 1), a.score_rows, a.gs));
    }
  }
};

// The threshold of the `top` largest keys of rows lo..hi-1, by counting: the
// range between the smallest and the largest key is cut into equal bins
// (keys of floats are spread about evenly in it, where the bits of one digit are
// not: scores share their leading bits, and the counters of a few bins would be
// hit by all lanes at once), the bin that holds the threshold becomes the next
// range, and the descent ends when its keys are equal or all wanted: two or three
// passes instead of four by 8-bit digits.
template <int NT, int KPT>
__global__ __launch_bounds__(NT, KPT <= 16 ? 8 : 4) void evict_select(EvictArgs a) {
  constexpr int kSW = NT / kWave;
  constexpr int kBits = NT == 1024 ? 11 : 9, kBins = 1 << kBits, kOwn = kBins / NT;  // bins per thread
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t part[2][kSW];
  __shared__ uint32_t pick[3];  // the bin, how many of it are wanted, and its count
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int unit = blockIdx.x, b = unit / a.heads;
  const Budget x = budget(a, b);
  if (unit % a.heads == 0 && threadIdx.x == 0) a.held[b] = x.kept;
  if (x.kept == 0) return;
  const float *f = a.scores + (int64_t)unit * a.gs * a.score_rows;
  const int lo = x.first, hi = x.n - x.last;  // ranked rows
  const int per = KPT ? KPT * kWave : ((x.n + kSW - 1) / kSW + kWave - 1) / kWave * kWave;
  const int r0 = min(wave * per, x.n), r1 = min(r0 + per, x.n);
  Keys<KPT> keys;
  keys.load(a, f, r0, lo, x.n);
  const uint32_t top = x.kept - x.last - x.first;
  uint32_t want = top, low = 0u, high = 0xffffffffu;  // the threshold is in [low, high]
  if (top > 0 && top < (uint32_t)(hi - lo)) {
    uint32_t mn = 0xffffffffu, mx = 0u;
    keys.each(a, f, r0, r1, [&](int row, uint32_t k) {
      if (row >= lo && row < hi) {
        mn = min(mn, k);
        mx = max(mx, k);
      }
    });
    mn = ~wave_umax(~mn);
    mx = wave_umax(mx);
    if (lane == 0) {
      part[0][wave] = mn;
      part[1][wave] = mx;
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) hist[threadIdx.x * kOwn + i] = 0u;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSW; ++w) {
      mn = min(mn, part[0][w]);
      mx = max(mx, part[1][w]);
    }
    low = mn;
    high = mx;
    while (low < high) {
      // bins of 2^shift keys, bin 0 the highest keys
      const int bits = 32 - __clz(high - low), shift = max(bits - kBits, 0);
      keys.each(a, f, r0, r1, [&](int row, uint32_t k) {
        if (row >= lo && row < hi && k >= low && k <= high) atomicAdd(&hist[(high - k) >> shift], 1u);
      });
      __syncthreads();
      uint32_t c[kOwn], own = 0;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) own += c[i] = hist[threadIdx.x * kOwn + i];
      const uint32_t s = (uint32_t)wave_scan((int)own);
      if (lane == kWave - 1) part[0][wave] = s;
      __syncthreads();
      uint32_t above = s - own;
#pragma unroll
      for (int w = 0; w < kSW; ++w) above += w < wave ? part[0][w] : 0u;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        if (above < want && above + c[i] >= want) {
          pick[0] = threadIdx.x * kOwn + i;
          pick[1] = want - above;
          pick[2] = c[i];
        }
        above += c[i];
        hist[threadIdx.x * kOwn + i] = 0u;
      }
      __syncthreads();
      const uint32_t from = pick[0] << shift;
      want = pick[1];
      const uint32_t floor = high - from < (1u << shift) - 1 ? low : high - from - ((1u << shift) - 1);
      high -= from;
      low = max(low, floor);
      if (want == pick[2]) {  // the whole bin is kept: its lowest key is a threshold
        high = low;
        want = 0xffffffffu;
      }
    }
  } else if (top == 0) {
    low = 0xffffffffu;  // none (no key is all ones)
  }
  // the ranked rows above `low`, and the first `want` of those equal to it (with a
  // whole bin or all rows kept: all of them)
  if (top > 0 && top == (uint32_t)(hi - lo)) want = 0xffffffffu;
  uint32_t sure = 0, ties = 0;
  keys.each(a, f, r0, r1, [&](int row, uint32_t k) {
    const bool in = row < r1, fixed = row < lo || row >= hi;
    sure += __popcll(__ballot(in && (fixed || k > low)));
    ties += __popcll(__ballot(in && !fixed && k == low));
  });
  __syncthreads();  // (the smallest and largest keys have been read)
  if (lane == 0) {
    part[0][wave] = sure;
    part[1][wave] = ties;
  }
  __syncthreads();
  uint32_t at = 0, before = 0;  // kept rows and ties of the runs before
#pragma unroll
  for (int w = 0; w < kSW; ++w) {
    at += w < wave ? part[0][w] : 0u;
    before += w < wave ? part[1][w] : 0u;
  }
  at += min(before, want);
  const uint64_t below = (1ull << lane) - 1;
  int32_t *src = a.src + unit * a.cap;
  keys.each(a, f, r0, r1, [&](int row, uint32_t k) {
    const bool in = row < r1, fixed = row < lo || row >= hi, tie = in && !fixed && k == low;
    const uint64_t mt = __ballot(tie);
    const bool yes = in && (fixed || k > low || (tie && before + __popcll(mt & below) < want));
    const uint64_t m = __ballot(yes);
    if (yes) src[at + __popcll(m & below)] = row;
    at += __popcll(m);
    before += __popcll(mt);
  });
}

// blockIdx.x: (sequence, kv head); blockIdx.y: interleaved shares of the pieces, as many
// as a piece per thread asks for, up to 32; blockIdx.z: K (0), V (1), or positions and
// scores (2).
__global__ __launch_bounds__(kCT) void evict_copy(EvictArgs a) {
  const int unit = blockIdx.x, b = unit / a.heads, h = unit % a.heads;
  const Budget x = budget(a, b);
  const int32_t *src = a.src + unit * a.cap;
  if (blockIdx.z == 2) {
    for (int r = blockIdx.y * kCT + threadIdx.x; r < x.kept; r += gridDim.y * kCT) {
      const int row = src[r];
      a.out_pos[unit * a.out_rows + r] = a.row_pos ? a.row_pos[unit * a.pos_rows + row] : row;
      if (a.out_scores)
        for (int i = 0; i < a.gs; ++i)
          a.out_scores[((int64_t)unit * a.gs + i) * a.out_rows + r] =
              a.scores[((int64_t)unit * a.gs + i) * a.score_rows + row];
    }
    return;
  }
  const int psh = 31 - __clz(a.row_bytes / 16);
  const int64_t items = (int64_t)x.kept << psh;
  const unsigned char *from = (blockIdx.z ? a.from.v : a.from.k) + (((uint64_t)h * a.from.head_stride) << 4);
  unsigned char *to = (blockIdx.z ? a.to_v : a.to_k) + (((uint64_t)h * a.to.head_stride) << 4);
  for (int64_t q = blockIdx.y * kCT + threadIdx.x; q < items; q += (int64_t)gridDim.y * kCT) {
    const int r = (int)(q >> psh), p = (int)(q & ((1 << psh) - 1));
    const int64_t s = row_offset(a.from, b, src[r]), d = row_offset(a.to, b, r);
    if (s < 0 || d < 0) continue;
    reinterpret_cast<uint4 *>(to + d)[p] = reinterpret_cast<const uint4 *>(from + s)[p];
  }
}

template <int NT, int KPT> void launch_select(const EvictArgs &a, unsigned units, hipStream_t st) {
  hipLaunchKernelGGL((evict_select<NT, KPT>), dim3(units), dim3(NT), 0, st, a);
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
  // eight keys per thread and as few waves as hold the longest sequence (one layer of
  // 1237 rows: 9.8 us with four waves, 11.8 with sixteen; 1088 kv heads of 861: 18, 27)
  const int n = std::min(a.max_len, a.from.cap);
  (n <= 512 ? launch_select<64, 8> : n <= 2048 ? launch_select<256, 8> : n <= 8192 ? launch_select<1024, 8>
   : n <= 16384 ? launch_select<1024, 16> : n <= 32768 ? launch_select<1024, 32> : launch_select<1024, 0>)(a, units, st);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const unsigned shares = (unsigned)std::min<int64_t>((a.cap * (a.row_bytes / 16) + kCT - 1) / kCT, 32);
  hipLaunchKernelGGL(evict_copy, dim3(units, shares, 3), dim3(kCT), 0, st, a);
  return hipGetLastError();
}

}  // namespace smallkv
