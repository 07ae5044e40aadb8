// ckv_blocks.cpp -- the C ABI of the attention over selected blocks: argument
// checks and launches.
#include "ckv_blocks.hpp"

#include "ckv_profile.hpp"

namespace {

using namespace ckv;

int check_block(int32_t block, int32_t* lb) {
  if (block != 32 && block != 64 && block != 128 && block != 256)
    return fail(CKV_EUNSUPPORTED, "block %d not in {32,64,128,256}", block);
  *lb = __builtin_ctz((unsigned)block);
  return CKV_OK;
}

int check_kept(int32_t k) {
  if (k < 1 || k > kMaxKept) return fail(CKV_ESHAPE, "k %d outside [1, %d]", k, kMaxKept);
  return CKV_OK;
}

int check_pages(const PagedPages& pg) {
  if (pg.shift < 4)
    return fail(CKV_EUNSUPPORTED, "page_size %d (blocks take pages of at least 16)",
                1 << pg.shift);
  return CKV_OK;
}

// work-items per dispatch must stay below 2^32
int check_grid(int64_t wgs) {
  if (wgs >= ((int64_t)1 << 24)) return fail(CKV_EUNSUPPORTED, "grid too large for this shape");
  return CKV_OK;
}

// Everything of the tokens but their addresses.
int check_query(const Dims& d, int32_t block, int32_t k, int32_t tokens, BlockTokens* t) {
  CKV_RC(check_block(block, &t->lb));
  CKV_RC(check_kept(k));
  CKV_RC(check_num_tokens(tokens));
  t->n = tokens;
  t->B = d.B;
  t->Hkv = d.Hkv;
  t->Hq = d.Hq;
  t->lg = __builtin_ctz((unsigned)d.G);
  t->max_ctx = d.max_ctx;
  t->nb = (int32_t)(((int64_t)d.max_ctx + block - 1) >> t->lb);
  t->k = k;
  return check_grid((int64_t)tokens * d.Hkv);
}

// Debug mode: the order of the lists (after the tokens' own check).
int debug_check_lists(hipStream_t s, const BlockTokens& t, const int32_t* idx) {
  if (!debug_on()) return CKV_OK;
  BlockListArgs a = {t, idx, nullptr};
  unsigned long long got = 0;
  CKV_RC(debug_run(
      s,
      [&](unsigned long long* flag) {
        a.flag = flag;
        return launch_check_lists(a, s);
      },
      &got));
  if (got == ~0ull) return CKV_OK;
  return fail(CKV_EINVAL, "debug check: the blocks of idx[%lld][%lld] do not ascend",
              (long long)got / t.Hkv, (long long)got % t.Hkv);
}

int check_ws(const void* ws, size_t bytes, size_t need) {
  if (!ws) return fail(CKV_EWORKSPACE, "workspace is NULL (%zu bytes needed)", need);
  if (reinterpret_cast<uintptr_t>(ws) & 255u)
    return fail(CKV_EWORKSPACE, "workspace is not 256-byte aligned");
  if (bytes < need) return fail(CKV_EWORKSPACE, "workspace of %zu bytes, %zu needed", bytes, need);
  return CKV_OK;
}

// How the scoring is cut: four tiles of query rows a workgroup (each landmark loaded
// once for them) while that leaves the device full, and then larger chunks of
// landmarks.
constexpr int64_t kScoreWgs = 1024;

void cut_scores(BlockSelectArgs* a) {
  auto wgs = [&](int tiles, int cols) {
    return tiles_of(a->t, tiles) * a->t.Hkv * ((a->t.nb + cols - 1) / cols);
  };
  // (about a token a request: four requests a tile and more, a wave each)
  const int least = a->t.n <= a->t.B ? 16 : kMarkCols;
  a->row_tiles = wgs(4, kMarkCols) >= kScoreWgs ? 4 : 1;
  a->cols = least;
  while (a->cols < 1024 && wgs(a->row_tiles, 2 * a->cols) >= kScoreWgs) a->cols *= 2;
  a->chunks = (a->t.nb + a->cols - 1) / a->cols;
}

size_t score_bytes(const BlockTokens& t) {
  return align256((size_t)t.n * t.Hkv * t.nb * sizeof(float));
}

size_t norm_bytes(const BlockSelectArgs& a) {
  return align256((size_t)tiles_of(a.t, a.row_tiles) * a.t.Hkv * a.chunks * sizeof(float));
}

// Pieces of a tile's list: as many as fill the device twice over, of two steps a
// wave at least if every token keeps blocks of its own (16 tokens, 32 blocks of 64, 8
// heads: 46 us all three operators; twice as many pieces 53).
constexpr int kBlockWgs = 512;

int cut_pieces(const BlockTokens& t) {
  const int64_t units = std::max<int64_t>(1, tiles_of(t) * t.Hkv);
  const int64_t kept = std::min(t.k, t.nb);
  const int64_t steps = ((16 >> t.lg) * kept) << (t.lb - 5);
  return (int)std::max<int64_t>(
      1, std::min<int64_t>({kBlockWgs / units, steps / 8, (int64_t)kMaxPieces}));
}

// Many tokens of a bf16 cache: four tiles share the staging of a block that one of them
// keeps.  A tile a workgroup against it, us, 16 blocks of 64, 8 KV heads of 4 query
// heads: 512 tokens (256 workgroups of four tiles) 161 / 219, 1024 (512) 267 / 252, 2048
// 487 / 299, 4096 949 / 569; 1024 tokens and 4 heads of 8 (512) 180 / 182, 2048 and 2 of
// 16 (1024) 211 / 158, 1500 and 8 of 1 (192) 187 / 319; 48 blocks, 2048 tokens 1171 / 619.
// Rows of codes are less to read and have to be made bf16: 2048 tokens e4m3 297 / 359,
// e2m1 262 / 337.  With fewer tokens a request than four tiles have a block would be of
// use to one wave.
constexpr int kManyWgs = 512;

bool many_tokens(const BlockTokens& t, Kind kind) {
  return kind == Kind::kBf16 && (int64_t)t.n >= (int64_t)t.B * (kManyTiles * 16 >> t.lg) &&
         tiles_of(t, kManyTiles) * t.Hkv >= kManyWgs;
}

size_t part_bytes(const BlockTokens& t) {
  const int pieces = cut_pieces(t);
  if (pieces == 1) return 0;
  return (size_t)tiles_of(t) * t.Hkv * pieces * 16 * kPartStride * sizeof(float);
}

size_t blocks_ws_bytes(const BlockTokens& t) {
  BlockSelectArgs a = {};
  a.t = t;
  cut_scores(&a);
  return std::max(score_bytes(t) + norm_bytes(a), part_bytes(t));
}

}  // namespace

extern "C" {

int ckv_blocks_workspace_bytes(const ckv_shape* shape, int32_t block, int32_t k,
                               int32_t num_tokens, size_t* bytes) {
  Dims d;
  BlockTokens t = {};
  CKV_RC(check_shape(shape, &d));
  CKV_RC(check_query(d, block, k, num_tokens, &t));
  if (!bytes) return fail(CKV_EINVAL, "bytes is NULL");
  *bytes = blocks_ws_bytes(t);
  return CKV_OK;
}

int ckv_paged_landmarks(const ckv_shape* shape, const ckv_paged_cache* cache, int32_t block,
                        const int32_t* ctx_lens, const int32_t* first, uint16_t* landmarks,
                        void* stream) {
  Dims d;
  MarkArgs a = {};
  CKV_RC(check_shape(shape, &d));
  CKV_RC(check_cache(cache, d, &a.pg));
  CKV_RC(check_pages(a.pg));
  CKV_RC(check_block(block, &a.lb));
  CKV_PTR(ctx_lens);
  if (first) CKV_PTR(first);
  CKV_PTR(landmarks);
  a.ctx_lens = ctx_lens;
  a.first = first;
  a.marks = landmarks;
  a.B = d.B;
  a.max_ctx = d.max_ctx;
  a.nb = (int32_t)(((int64_t)d.max_ctx + block - 1) >> a.lb);
  CKV_RC(check_grid(d.U));
  if (d.U == 0) return CKV_OK;
  // four blocks at once a workgroup; a device's worth of workgroups
  a.slices = (int32_t)std::max<int64_t>(
      1, std::min<int64_t>(4 * device_cus() / d.U, ((int64_t)a.nb + 3) / 4));
  hipStream_t s = (hipStream_t)stream;
  CKV_RC(debug_check(s, ctx_lens, nullptr, nullptr, d.B, d.Hkv, d.max_ctx, 1));
  CKV_RC(debug_check_paged(s, a.pg, ctx_lens, nullptr, nullptr, d.B, d.max_ctx, 0));
  CKV_TRY_HIP(launch_marks(a, (Kind)cache->kind, s), "landmarks launch");
  return CKV_OK;
}

int ckv_select_blocks(const ckv_shape* shape, const ckv_paged_cache* cache, int32_t block,
                      int32_t k, int32_t num_tokens, const int32_t* requests,
                      const int32_t* positions, const uint16_t* q, const uint16_t* landmarks,
                      int32_t* idx, void* ws, size_t ws_bytes, void* stream) {
  Dims d;
  BlockSelectArgs a = {};
  CKV_RC(check_shape(shape, &d));
  CKV_RC(check_cache(cache, d, &a.pg));
  CKV_RC(check_pages(a.pg));
  CKV_RC(check_query(d, block, k, num_tokens, &a.t));
  if (num_tokens == 0) return CKV_OK;  // without tokens their addresses may be NULL
  if (requests) CKV_PTR(requests);
  CKV_PTR(positions);
  CKV_PTR(q);
  CKV_PTR(landmarks);
  CKV_PTR(idx);
  cut_scores(&a);
  CKV_RC(check_grid(tiles_of(a.t, a.row_tiles) * a.chunks * d.Hkv));
  CKV_RC(check_ws(ws, ws_bytes, blocks_ws_bytes(a.t)));
  if (!requests && num_tokens > d.B)
    return fail(CKV_ESHAPE, "%d tokens of %d requests without requests", num_tokens, d.B);
  a.t.req = requests;
  a.t.pos = positions;
  a.t.q = q;
  a.marks = landmarks;
  a.idx = idx;
  a.scores = static_cast<float*>(ws);
  a.norms = reinterpret_cast<float*>(static_cast<char*>(ws) + score_bytes(a.t));
  hipStream_t s = (hipStream_t)stream;
  CKV_RC(debug_check_paged(s, a.pg, nullptr, requests, positions, d.B, d.max_ctx, num_tokens,
                           true));
  CKV_TRY_HIP(launch_select_blocks(a, s), "block selection launch");
  return CKV_OK;
}

int ckv_paged_block_attn(const ckv_shape* shape, const ckv_paged_cache* cache, int32_t block,
                         int32_t k, int32_t num_tokens, const int32_t* requests,
                         const int32_t* positions, const uint16_t* q, const int32_t* idx,
                         float scale, float* out, float* lse, void* ws, size_t ws_bytes,
                         void* stream) {
  Dims d;
  BlockAttnArgs a = {};
  CKV_RC(check_shape(shape, &d));
  CKV_RC(check_cache(cache, d, &a.pg));
  CKV_RC(check_pages(a.pg));
  CKV_RC(check_query(d, block, k, num_tokens, &a.t));
  CKV_RC(check_scale(scale));
  if (scale > 0x1p126f)  // 2 log2(e) times it, a factor of the logits, has to be finite
    return fail(CKV_EINVAL, "scale %g above 2^126", scale);
  if (num_tokens == 0) return CKV_OK;  // without tokens their addresses may be NULL
  if (requests) CKV_PTR(requests);
  CKV_PTR(positions);
  CKV_PTR(q);
  CKV_PTR(idx);
  CKV_PTR(out);
  if (lse) CKV_PTR(lse);
  CKV_RC(check_ws(ws, ws_bytes, blocks_ws_bytes(a.t)));
  if (!requests && num_tokens > d.B)
    return fail(CKV_ESHAPE, "%d tokens of %d requests without requests", num_tokens, d.B);
  a.t.req = requests;
  a.t.pos = positions;
  a.t.q = q;
  a.idx = idx;
  a.out = out;
  a.lse = lse;
  a.part = static_cast<float*>(ws);
  a.scale = scale;
  a.pieces = cut_pieces(a.t);
  a.many = requests && many_tokens(a.t, (Kind)cache->kind);
  hipStream_t s = (hipStream_t)stream;
  CKV_RC(debug_check_paged(s, a.pg, nullptr, requests, positions, d.B, d.max_ctx, num_tokens,
                           true));
  CKV_RC(debug_check_lists(s, a.t, idx));
  CKV_TRY_HIP(launch_block_attn(a, (Kind)cache->kind, s), "block attention launch");
  return CKV_OK;
}

}  // extern "C"
