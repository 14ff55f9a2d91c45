// Drives the host side of the cache operators (descriptor checks, workspace planning,
// rotary frequencies) with descriptors whose pointers are never dereferenced, so that
// an AddressSanitizer / UBSan build of the library's host code checks them.  Every
// call here returns before anything would be enqueued.  Exits non-zero on an
// unexpected status.
#include <limits.h>
#include <math.h>
#include <stdio.h>

#include "smallkv.h"

static int fails = 0;
#define EXPECT(call, want)                                                      \
  do {                                                                          \
    const int rc_ = (call);                                                     \
    if (rc_ != (want)) {                                                        \
      fprintf(stderr, "%s:%d: %s -> %d, want %d\n", __FILE__, __LINE__, #call, rc_, \
              (int)(want));                                                     \
      ++fails;                                                                  \
    }                                                                           \
  } while (0)

static char *P = reinterpret_cast<char *>(0x1000);
static const int32_t *IP = reinterpret_cast<const int32_t *>(0x1000);
static float *FP = reinterpret_cast<float *>(0x1000);

static smallkv_cache_t cache_of(int dtype, int heads, int d, int page_rows, int width, long long pages) {
  smallkv_cache_t c{};
  c.k = P;
  c.v = P + 4096;
  c.dtype = dtype;
  c.head_dim = d;
  c.n_heads = heads;
  c.page_rows = page_rows;
  c.n_pages = (int32_t)pages;
  c.table_width = width;
  c.row_stride = d;
  c.head_stride = (int64_t)page_rows * d;
  c.page_stride = (int64_t)heads * page_rows * d;
  c.page_table = width ? IP : nullptr;
  return c;
}

int main() {
  const int dtypes[] = {SMALLKV_F32, SMALLKV_BF16}, dims[] = {64, 128};
  const int lens[] = {1, 2, 63, 64, 65, 255, 257, 4096, 131072, 1 << 30};
  const int news[] = {1, 2, 4, 5, 16, 33, 4096, 1 << 20};
  const int groups[] = {1, 3, 7, 16, 64}, batches[] = {1, 3, 64, 1000};
  for (int dtype : dtypes)
    for (int d : dims)
      for (int len : lens)
        for (int nw : news)
          for (int g : groups)
            for (int B : batches) {
              const int heads = 4;
              const int width = (int)(((long long)len + 15) / 16);
              smallkv_cache_t c = cache_of(dtype, heads, d, 16, width, 1 << 20);
              smallkv_chunk_t ch{B, (int)((long long)B * nw > (1 << 30) ? 1 << 30 : B * nw), nw, len, IP, IP};
              smallkv_queries_t q{};
              q.n_heads = heads * g;
              q.scale = 0.125f;
              q.q = q.out = P;
              q.token_stride = q.out_token_stride = (int64_t)q.n_heads * d;
              q.head_stride = q.out_head_stride = d;
              q.lse = FP;
              size_t ws = 1;
              const int rc = smallkv_chunk_attn_workspace_size(&ch, &c, &q, &ws);
              if (rc != SMALLKV_OK && rc != SMALLKV_EUNSUPPORTED) EXPECT(rc, SMALLKV_OK);
              if (rc == SMALLKV_OK && ws) {
                EXPECT(smallkv_chunk_attn(&ch, &c, &q, P, ws - 1, nullptr), SMALLKV_EWORKSPACE);
                EXPECT(smallkv_chunk_attn(&ch, &c, &q, nullptr, ws, nullptr), SMALLKV_EWORKSPACE);
                if (ws > (size_t)256 << 20) {  // records of at most two workgroups per CU and a half
                  fprintf(stderr, "workspace of %zu bytes\n", ws);
                  ++fails;
                }
              }
              EXPECT(smallkv_chunk_scores(&ch, &c, &q, q.n_heads, nullptr, FP, len - 1, LLONG_MAX, nullptr),
                     rc ? rc : SMALLKV_EINVAL);
              EXPECT(smallkv_chunk_scores(&ch, &c, &q, q.n_heads + 1, nullptr, FP, len, LLONG_MAX, nullptr),
                     rc ? rc : SMALLKV_EINVAL);
            }
  smallkv_cache_t c = cache_of(SMALLKV_BF16, 4, 64, 64, 32, 64), to = cache_of(SMALLKV_BF16, 4, 64, 64, 32, 64);
  to.k = P + 8192;
  to.v = P + 12288;
  EXPECT(smallkv_append(nullptr, &c, nullptr, nullptr), SMALLKV_EINVAL);
  EXPECT(smallkv_chunk_attn(nullptr, nullptr, nullptr, nullptr, 0, nullptr), SMALLKV_EINVAL);
  EXPECT(smallkv_chunk_scores(nullptr, &c, nullptr, 4, nullptr, FP, 1, 4, nullptr), SMALLKV_EINVAL);
  EXPECT(smallkv_evict(nullptr, P, 0, nullptr), SMALLKV_EINVAL);
  smallkv_chunk_t none{2, 0, 1, 100, IP, IP};
  smallkv_append_t a{};
  EXPECT(smallkv_append(&none, &c, &a, nullptr), SMALLKV_EINVAL);
  a.q = a.k = a.v = P;
  a.q_out = P + 4096;
  a.n_q_heads = 8;
  a.q_out_token_stride = 512;
  a.q_out_head_stride = 64;
  a.amplitude = 1.0f;
  EXPECT(smallkv_append(&none, &c, &a, nullptr), SMALLKV_OK);  // (no tokens: nothing to enqueue)
  a.row_pos = reinterpret_cast<int32_t *>(P);
  a.pos_rows = INT_MAX;
  a.pos_seq_stride = LLONG_MAX;
  EXPECT(smallkv_append(&none, &c, &a, nullptr), SMALLKV_OK);
  a.pos_rows = (int64_t)INT_MAX + 1;
  EXPECT(smallkv_append(&none, &c, &a, nullptr), SMALLKV_EINVAL);
  smallkv_evict_t e{};
  e.batch = 2;
  e.max_len = 2048;
  e.len = e.keep = IP;
  e.from = c;
  e.to = to;
  e.n_score_heads = 28;
  e.scores = FP;
  e.score_rows = 2048;
  e.out_rows = 1 << 20;
  e.out_pos = e.held = reinterpret_cast<int32_t *>(P);
  size_t ws = 0;
  EXPECT(smallkv_evict_workspace_size(&e, &ws), SMALLKV_OK);
  EXPECT(ws == 2 * 4 * 2048 * 4, 1);  // a row number for every row that may be kept
  EXPECT(smallkv_evict(&e, P, ws - 1, nullptr), SMALLKV_EWORKSPACE);
  e.max_len = (1 << 20) + 1;
  e.score_rows = LLONG_MAX;
  EXPECT(smallkv_evict_workspace_size(&e, &ws), SMALLKV_EUNSUPPORTED);
  double f[64];
  float amp;
  for (int scaling = 0; scaling < 5; ++scaling)
    for (int rot = 2; rot <= 128; rot += 2) {
      EXPECT(smallkv_rope_freqs(rot, 1e4, scaling, 8.0, 1.0, 32.0, 4096, f, &amp), SMALLKV_OK);
      for (int j = 0; j < rot / 2; ++j) EXPECT(isfinite(f[j]) && f[j] > 0.0 && f[j] <= 1.0, 1);
    }
  EXPECT(smallkv_rope_freqs(64, 1e4, 0, 1.0, 0, 0, 0, nullptr, &amp), SMALLKV_EINVAL);
  EXPECT(smallkv_rope_freqs(64, 1e4, 0, 1.0, 0, 0, 0, f, nullptr), SMALLKV_OK);
  EXPECT(smallkv_rope_freqs(INT_MIN, 1e4, 0, 1.0, 0, 0, 0, f, nullptr), SMALLKV_EINVAL);
  if (!fails) printf("cache abi driver ok\n");
  return fails ? 1 : 0;
}
