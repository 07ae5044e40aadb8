// Every entry of the rotary positions and the paged cache with rejected
// arguments and empty batches, for a build of the host code with ASan and
// UBSan: validation, layouts and frequencies run, nothing is launched.
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstring>

#include "ckv.h"

static int g_failures = 0;

#define EXPECT(call, want)                                                    \
  do {                                                                        \
    const int got_ = (call);                                                  \
    if (got_ != (want)) {                                                     \
      std::fprintf(stderr, "line %d: %s gave %d (%s)\n", __LINE__, #call, got_, \
                   ckv_last_error_detail());                                  \
      ++g_failures;                                                           \
    }                                                                         \
  } while (0)

int main() {
  alignas(256) static unsigned char mem[16384];
  uint16_t* h = reinterpret_cast<uint16_t*>(mem);
  int32_t* n = reinterpret_cast<int32_t*>(mem);
  float* f = reinterpret_cast<float*>(mem);
  ckv_shape s = {};
  s.batch = 2, s.num_q_heads = 8, s.num_kv_heads = 2, s.head_dim = 128, s.max_ctx = 64;
  s.key_row_stride = s.kv_row_stride = 128;
  ckv_paged_cache c = {};
  c.k_pages = c.v_pages = mem;
  c.page_table = n;
  c.page_stride = 4096, c.head_stride = 2048, c.row_stride = 128;
  c.page_size = 16, c.num_pages = 4, c.table_stride = 4;
  ckv_rope r = {};
  r.inv_freq = reinterpret_cast<double*>(mem);
  r.head_dim = r.rot_dim = 128;
  r.scale = 1.f;
  ckv_rows q = {};
  q.src = mem, q.dst = mem + 2048;
  q.src_token_stride = q.dst_token_stride = 1024;
  q.src_head_stride = q.dst_head_stride = 128;
  q.heads = 8;

  // empty calls run the whole validation
  EXPECT(ckv_rope_rows(&r, 0, n, &q, &q, nullptr), CKV_OK);
  EXPECT(ckv_paged_write(&s, &c, 0, nullptr, n, h, h, 256, &r, &q, nullptr), CKV_OK);
  ckv_shape e = s;
  e.batch = 0;
  EXPECT(ckv_paged_read(&e, &c, n, n, n, 8, h, h, nullptr), CKV_OK);
  EXPECT(ckv_paged_score_keys(&e, &c, h, n, 0.1f, f, nullptr), CKV_OK);
  EXPECT(ckv_paged_decode_attn(&e, &c, 1, h, n, 0.1f, f, f, mem, sizeof mem, nullptr), CKV_OK);

  // extreme sizes and strides meet no overflow
  for (int64_t x : {INT64_MIN, INT64_MIN + 8, (int64_t)-8, (int64_t)0, (int64_t)1 << 36,
                    ((int64_t)1 << 36) + 8, INT64_MAX - 7, INT64_MAX}) {
    ckv_rows b = q;
    b.src_token_stride = x;
    const int rc = ckv_rope_rows(&r, 0, n, &b, nullptr, nullptr);
    if (rc != CKV_OK && rc != CKV_ESHAPE) ++g_failures;
    for (int i = 0; i < 3; ++i) {
      ckv_paged_cache b2 = c;
      (i == 0 ? b2.page_stride : i == 1 ? b2.head_stride : b2.row_stride) = x;
      for (int pages : {1, INT_MAX}) {
        b2.num_pages = pages;
        const int rc2 = ckv_paged_score_keys(&e, &b2, h, n, 0.1f, f, nullptr);
        if (rc2 != CKV_OK && rc2 != CKV_ESHAPE && rc2 != CKV_EUNSUPPORTED) ++g_failures;
      }
    }
    if (x > 0 || x < 0) {
      EXPECT(ckv_paged_write(&s, &c, 0, nullptr, n, h, h, x, nullptr, nullptr, nullptr),
             x == ((int64_t)1 << 36) || x == ((int64_t)1 << 36) + 8 ? CKV_OK : CKV_ESHAPE);
    }
  }
  for (int x : {INT_MIN, -1, 0, INT_MAX}) {
    EXPECT(ckv_rope_rows(&r, x, n, &q, nullptr, nullptr), x == 0 ? CKV_OK : CKV_ESHAPE);
    EXPECT(ckv_paged_read(&e, &c, n, nullptr, nullptr, x, h, h, nullptr), CKV_ESHAPE);
    EXPECT(ckv_paged_decode_attn(&e, &c, x, h, n, 0.1f, f, f, mem, sizeof mem, nullptr),
           CKV_EUNSUPPORTED);
    ckv_paged_cache b = c;
    b.page_size = x;
    EXPECT(ckv_paged_score_keys(&e, &b, h, n, 0.1f, f, nullptr), CKV_EUNSUPPORTED);
    ckv_rope b2 = r;
    b2.rot_dim = x;
    EXPECT(ckv_rope_rows(&b2, 0, n, &q, nullptr, nullptr), CKV_ESHAPE);
  }
  size_t bytes = 0;
  ckv_shape big = s;
  big.batch = 1 << 20, big.max_ctx = 1 << 30;
  EXPECT(ckv_workspace_bytes(&big, 4, CKV_ENTRY_PAGED_DECODE_ATTN, &bytes), CKV_OK);
  if (bytes == 0 || bytes > ((size_t)64 << 20)) ++g_failures;
  EXPECT(ckv_workspace_bytes(&s, 5, CKV_ENTRY_PAGED_DECODE_ATTN, &bytes), CKV_EUNSUPPORTED);

  // frequencies of every kind and size
  static double freq[512];
  for (int kind = CKV_ROPE_PLAIN; kind <= CKV_ROPE_RAMP; ++kind)
    for (int rot : {4, 20, 128, 1024})
      for (int ctx : {1, 4096, INT_MAX})
        for (double factor : {1.0, 32.0, 1e300}) {
          ckv_rope_scaling sc = {kind, ctx, factor, 1.0, 32.0};
          float scale = 0.f;
          const int rc = ckv_rope_frequencies(rot, 10000.0, &sc, freq, &scale);
          if (rc != CKV_OK && !(rc == CKV_EINVAL && kind == CKV_ROPE_BASE && factor > 1e200))
            ++g_failures;
          for (int i = 0; rc == CKV_OK && i < rot / 2; ++i)
            if (!(freq[i] >= 0) || !std::isfinite(freq[i])) ++g_failures;
        }
  EXPECT(ckv_rope_frequencies(64, 10000.0, nullptr, freq, nullptr), CKV_OK);
  EXPECT(ckv_rope_frequencies(64, 10000.0, nullptr, nullptr, nullptr), CKV_EINVAL);
  ckv_kernel_stats st[CKV_K_TOTAL];
  EXPECT(ckv_profile_begin(CKV_K_EVERY), CKV_OK);
  EXPECT(ckv_profile_end_n(st, CKV_K_TOTAL), CKV_OK);
  EXPECT(ckv_profile_end_n(st, CKV_K_TOTAL + 1), CKV_EINVAL);

  if (g_failures) {
    std::fprintf(stderr, "%d failures\n", g_failures);
    return 1;
  }
  std::printf("paged checks ok\n");
  return 0;
}
