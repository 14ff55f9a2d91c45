// Drives the host side of the packed cache's calls (descriptor checks, workspace planning)
// with descriptors whose pointers are never dereferenced, so that an AddressSanitizer / UBSan
// build of the library's host code checks them.  Every call here returns before anything
// would be enqueued.  Exits non-zero on an unexpected status.
#include <limits.h>
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
static uint8_t *U = reinterpret_cast<uint8_t *>(0x100000);
static const int32_t *IP = reinterpret_cast<const int32_t *>(0x1000);
static float *FP = reinterpret_cast<float *>(0x1000);

static smallkv_packed_t packed_of(int format, int dtype, int heads, int d, int page_rows, int width) {
  const int bytes = format == SMALLKV_MXFP8 ? d : d / 2;
  smallkv_packed_t p{};
  p.k = P;
  p.v = P + 4096;
  p.k_scale = U;
  p.v_scale = U + 4096;
  p.format = format;
  p.dtype = dtype;
  p.head_dim = d;
  p.n_heads = heads;
  p.page_rows = page_rows;
  p.n_pages = 1 << 20;
  p.table_width = width;
  p.row_stride = bytes;
  p.head_stride = (int64_t)page_rows * bytes;
  p.page_stride = (int64_t)heads * page_rows * bytes;
  p.scale_row_stride = d / 32;
  p.scale_head_stride = (int64_t)page_rows * (d / 32);
  p.scale_page_stride = (int64_t)heads * page_rows * (d / 32);
  p.page_table = width ? IP : nullptr;
  return p;
}

int main() {
  const int formats[] = {SMALLKV_MXFP8, SMALLKV_MXFP4}, dtypes[] = {SMALLKV_F32, SMALLKV_BF16}, dims[] = {64, 128};
  const int lens[] = {1, 2, 127, 129, 512, 513, 1025, 4097, 131072, 1 << 30};
  const int news[] = {1, 2, 5, 16, 33, 4096, 1 << 20};
  const int groups[] = {1, 3, 7, 16, 64}, batches[] = {1, 3, 64, 1000};
  size_t bytes = 0;
  for (int format : formats)
    for (int dtype : dtypes)
      for (int d : dims)
        for (int len : lens)
          for (int nw : news)
            for (int g : groups)
              for (int B : batches) {
                const int heads = 4;
                smallkv_packed_t p = packed_of(format, dtype, heads, d, 16, (int)(((long long)len + 15) / 16));
                smallkv_chunk_t ch{B, (int)((long long)B * nw > (1 << 30) ? 1 << 30 : B * nw), nw, len, IP, IP};
                smallkv_queries_t q{};
                q.n_heads = heads * g;
                q.scale = 0.1f;
                q.q = P;
                q.token_stride = (int64_t)q.n_heads * d;
                q.head_stride = d;
                q.out = P;
                q.out_token_stride = q.token_stride;
                q.out_head_stride = d;
                q.lse = FP;
                const int rc = smallkv_chunk_attn_packed_workspace_size(&ch, &p, &q, &bytes);
                if (rc != SMALLKV_OK && rc != SMALLKV_EUNSUPPORTED) {
                  fprintf(stderr, "workspace size of %d %d %d %d %d %d %d: %d\n", format, dtype, d, len, nw, g, B, rc);
                  ++fails;
                }
                if (rc == SMALLKV_OK && bytes > 0)
                  EXPECT(smallkv_chunk_attn_packed(&ch, &p, &q, P, bytes - 1, nullptr), SMALLKV_EWORKSPACE);
              }
  smallkv_packed_t p = packed_of(SMALLKV_MXFP8, SMALLKV_BF16, 4, 128, 16, 8);
  smallkv_packed_t t = packed_of(SMALLKV_MXFP8, SMALLKV_BF16, 4, 128, 16, 8);
  t.k = P + 65536;
  t.v = P + 131072;
  t.k_scale = U + 65536;
  t.v_scale = U + 131072;
  const int64_t strides[] = {INT64_MIN, -16, 8, 1LL << 40, INT64_MAX, INT64_MAX - 15};
  for (const int64_t s : strides) {
    int64_t smallkv_packed_t::*const fields[] = {
        &smallkv_packed_t::page_stride,       &smallkv_packed_t::head_stride,       &smallkv_packed_t::row_stride,
        &smallkv_packed_t::scale_page_stride, &smallkv_packed_t::scale_head_stride, &smallkv_packed_t::scale_row_stride};
    for (int i = 0; i < 6; ++i) {
      int64_t smallkv_packed_t::*f = fields[i];
      if (i >= 3 && s == 8) continue;  // (whole scales)
      smallkv_packed_t bad = p;
      bad.*f = s;
      smallkv_append_t a{};
      smallkv_chunk_t ch{2, 4, 2, 128, IP, IP};
      const int rc = smallkv_append_packed(&ch, &bad, &a, nullptr);
      if (rc != SMALLKV_EINVAL && rc != SMALLKV_EUNSUPPORTED) {
        fprintf(stderr, "stride %lld: %d\n", (long long)s, rc);
        ++fails;
      }
    }
  }
  smallkv_evict_t e{};
  e.batch = 2;
  e.max_len = 128;
  e.len = e.keep = IP;
  e.n_score_heads = 4;
  e.scores = FP;
  e.score_rows = 128;
  e.out_rows = 64;
  e.out_pos = reinterpret_cast<int32_t *>(0x1000);
  e.held = reinterpret_cast<int32_t *>(0x1000);
  EXPECT(smallkv_evict_packed_workspace_size(&e, &p, &t, &bytes), SMALLKV_OK);
  EXPECT(smallkv_evict_packed(&e, &p, &t, P, bytes - 1, nullptr), SMALLKV_EWORKSPACE);
  EXPECT(smallkv_evict_packed(&e, &p, &p, P, bytes, nullptr), SMALLKV_EINVAL);
  EXPECT(smallkv_evict_packed(nullptr, &p, &t, P, bytes, nullptr), SMALLKV_EINVAL);
  smallkv_cache_t to{};
  to.k = P + (1 << 20);
  to.v = P + (1 << 21);
  to.dtype = SMALLKV_F32;
  to.head_dim = 128;
  to.n_heads = 4;
  to.page_rows = 128;
  to.n_pages = 2;
  to.row_stride = 128;
  to.head_stride = 128 * 128;
  to.page_stride = 4 * 128 * 128;
  EXPECT(smallkv_read_packed(&p, &to, 3, 128, nullptr, IP, nullptr), SMALLKV_EINVAL);  // a page short
  EXPECT(smallkv_read_packed(&p, &to, 2, 0, nullptr, IP, nullptr), SMALLKV_EINVAL);
  EXPECT(smallkv_read_packed(&p, &to, 2, INT_MAX, nullptr, IP, nullptr), SMALLKV_EUNSUPPORTED);
  if (!fails) printf("packed abi driver ok\n");
  return fails ? 1 : 0;
}
