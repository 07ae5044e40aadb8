// Every entry of the attention over selected blocks, and the 4-bit cache's, with
// rejected arguments and empty calls, for a build of the host code with ASan and
// UBSan: validation and sizes run, nothing is launched.
#include <climits>
#include <cstdio>

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
  for (int kind = CKV_CACHE_BF16; kind <= CKV_CACHE_E2M1; ++kind) {
    ckv_shape s = {};
    s.batch = 2, s.num_q_heads = 8, s.num_kv_heads = 2, s.head_dim = 128, s.max_ctx = 64;
    s.key_row_stride = s.kv_row_stride = 128;
    ckv_paged_cache c = {};
    c.kind = kind;
    c.k_pages = c.v_pages = mem;
    if (kind != CKV_CACHE_BF16) c.k_exps = c.v_exps = mem;
    c.page_table = n;
    c.page_stride = 4096, c.head_stride = 2048, c.row_stride = 128;
    c.page_size = 16, c.num_pages = 4, c.table_stride = 4;
    ckv_shape e = s;
    e.batch = 0;

    EXPECT(ckv_paged_landmarks(&e, &c, 32, n, n, h, nullptr), CKV_OK);
    EXPECT(ckv_paged_landmarks(&s, &c, 33, n, n, h, nullptr), CKV_EUNSUPPORTED);
    EXPECT(ckv_select_blocks(&s, &c, 32, 4, 0, n, n, h, h, n, nullptr, 0, nullptr), CKV_OK);
    EXPECT(ckv_select_blocks(&s, &c, 32, 4, 2, n, n, h, h, n, mem, 8, nullptr), CKV_EWORKSPACE);
    EXPECT(ckv_paged_block_attn(&s, &c, 32, 4, 0, n, n, h, n, 0.1f, f, f, nullptr, 0, nullptr),
           CKV_OK);
    EXPECT(ckv_paged_block_attn(&s, &c, 32, 4, 2, n, n, h, n, 0.1f, f, f, mem, 8, nullptr),
           CKV_EWORKSPACE);
    EXPECT(ckv_paged_read(&e, &c, n, n, n, 8, h, h, nullptr), CKV_OK);

    // extreme sizes and strides meet no overflow
    for (int64_t x : {INT64_MIN, INT64_MIN + 32, (int64_t)-32, (int64_t)0, (int64_t)1 << 36,
                      ((int64_t)1 << 36) + 32, INT64_MAX - 31, INT64_MAX})
      for (int which = 0; which < 3; ++which) {
        ckv_paged_cache b = c;
        (which == 0 ? b.page_stride : which == 1 ? b.head_stride : b.row_stride) = x;
        b.num_pages = INT_MAX;
        (void)ckv_paged_landmarks(&e, &b, 32, n, n, h, nullptr);
        (void)ckv_select_blocks(&s, &b, 32, 4, 0, n, n, h, h, n, nullptr, 0, nullptr);
        (void)ckv_paged_block_attn(&s, &b, 32, 4, 0, n, n, h, n, 0.1f, f, f, nullptr, 0, nullptr);
      }
    for (int32_t ctx : {1, 31, 33, 65536, 1 << 30})
      for (int32_t tokens : {0, 1, 16, 4095, 1 << 24, INT_MAX, INT_MIN})
        for (int32_t heads : {1, 8, 64})
          for (int32_t group : {1, 4, 16})
            for (int32_t block : {32, 256, INT_MAX, INT_MIN})
              for (int32_t k : {1, 64, INT_MAX, INT_MIN}) {
                ckv_shape b = s;
                b.max_ctx = ctx, b.num_kv_heads = heads, b.num_q_heads = group * heads;
                size_t bytes = 0;
                const int rc = ckv_blocks_workspace_bytes(&b, block, k, tokens, &bytes);
                const int32_t nb = block == 32 || block == 256 ? (ctx - 1) / block + 1 : 1;
                if (rc == CKV_OK && bytes < (size_t)tokens * heads * nb * 4) ++g_failures;
                c.table_stride = INT_MAX;
                if (tokens != 0)  // too small: the sizes are worked out, nothing is launched
                  (void)ckv_select_blocks(&b, &c, block, k, tokens, n, n, h, h, n, mem, 0,
                                          nullptr);
              }
    EXPECT(ckv_blocks_workspace_bytes(&s, 32, 4, 2, nullptr), CKV_EINVAL);
    EXPECT(ckv_blocks_workspace_bytes(nullptr, 32, 4, 2, nullptr), CKV_EINVAL);
  }
  if (g_failures) return 1;
  std::printf("blocks checks ok\n");
  return 0;
}
