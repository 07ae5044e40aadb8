// ckv_paged.cpp -- the C ABI of the rotary positions and the paged cache:
// argument checks and launches.
#include "ckv_paged.hpp"

#include <cmath>

#include "ckv_profile.hpp"

namespace {

using namespace ckv;

int check_rope(const ckv_rope* r, RopeSpec* s) {
  if (!r) return fail(CKV_EINVAL, "rope is NULL");
  const double* inv_freq = r->inv_freq;
  CKV_PTR(inv_freq);
  if (r->head_dim < 8 || r->head_dim > 1024 || (r->head_dim & 7))
    return fail(CKV_EUNSUPPORTED, "rope.head_dim %d (8 .. 1024, a multiple of 8)", r->head_dim);
  if (r->rot_dim < 2 || r->rot_dim > r->head_dim || (r->rot_dim & 1))
    return fail(CKV_ESHAPE, "rope.rot_dim %d (even, 2 .. head_dim)", r->rot_dim);
  if (r->layout != CKV_ROPE_HALF && r->layout != CKV_ROPE_INTERLEAVED)
    return fail(CKV_EINVAL, "bad rope.layout %d", r->layout);
  if (r->type != CKV_ROPE_BF16 && r->type != CKV_ROPE_F32)
    return fail(CKV_EINVAL, "bad rope.type %d", r->type);
  if (r->inverse != 0 && r->inverse != 1)
    return fail(CKV_EINVAL, "bad rope.inverse %d", r->inverse);
  if (!std::isfinite(r->scale)) return fail(CKV_EINVAL, "rope.scale must be finite");
  s->inv_freq = inv_freq;
  s->head_dim = r->head_dim;
  s->rot = r->rot_dim;
  s->layout = r->layout;
  s->f32 = r->type == CKV_ROPE_F32;
  s->inverse = r->inverse;
  s->scale = r->scale;
  return CKV_OK;
}

int check_rows(const char* what, const ckv_rows* rows, int32_t tokens, const RopeSpec& r,
               RopeRows* out) {
  if (!rows) return fail(CKV_EINVAL, "%s is NULL", what);
  if (tokens > 0 && (!rows->src || !rows->dst || !aligned16(rows->src) || !aligned16(rows->dst)))
    return fail(CKV_EINVAL, "%s.src and .dst must be 16-byte aligned pointers", what);
  if (rows->reserved != 0) return fail(CKV_EINVAL, "%s.reserved must be 0", what);
  if (rows->heads < 1 || rows->heads > 4096)
    return fail(CKV_ESHAPE, "%s.heads %d outside [1, 4096]", what, rows->heads);
  const int unit = r.f32 ? 4 : 8;  // elements of 16 bytes
  const int64_t strides[4] = {rows->src_token_stride, rows->src_head_stride,
                              rows->dst_token_stride, rows->dst_head_stride};
  for (int64_t x : strides)
    if (x % unit || x < 0 || x > ((int64_t)1 << 38))
      return fail(CKV_ESHAPE, "%s: stride %lld (0 .. 2^38, a multiple of 16 bytes)", what,
                  (long long)x);
  if (rows->src == rows->dst && (strides[0] != strides[2] || strides[1] != strides[3]))
    return fail(CKV_EINVAL, "%s: in place with different strides", what);
  // destination rows apart: heads within a token, or tokens within a head
  const int64_t tok = strides[2], head = strides[3], d = r.head_dim, h = rows->heads;
  const bool many = tokens > 1, by_token = (h == 1 || head >= d) &&
                                           (!many || tok >= (h - 1) * head + d);
  const bool by_head = many && tok >= d && (h == 1 || head >= (tokens - 1) * tok + d);
  if (!by_token && !by_head) return fail(CKV_ESHAPE, "%s: destination rows overlap", what);
  out->src = rows->src;
  out->dst = rows->dst;
  out->src_tok = strides[0];
  out->src_head = strides[1];
  out->dst_tok = strides[2];
  out->dst_head = strides[3];
  out->heads = rows->heads;
  return CKV_OK;
}

int check_num_tokens(int32_t n) {
  if (n < 0 || n > (1 << 24)) return fail(CKV_ESHAPE, "num_tokens %d outside [0, 2^24]", n);
  return CKV_OK;
}

int check_cache(const ckv_paged_cache* c, const Dims& d, PagedPages* p) {
  if (!c) return fail(CKV_EINVAL, "cache is NULL");
  if (c->kind != CKV_CACHE_BF16 && c->kind != CKV_CACHE_E4M3)
    return fail(CKV_EINVAL, "bad cache.kind %d", c->kind);
  const bool e4m3 = c->kind == CKV_CACHE_E4M3;
  void *k_pages = c->k_pages, *v_pages = c->v_pages;
  const int32_t* page_table = c->page_table;
  uint8_t *k_exps = c->k_exps, *v_exps = c->v_exps;
  CKV_PTR(k_pages);
  CKV_PTR(v_pages);
  CKV_PTR(page_table);
  if (e4m3) {
    CKV_PTR(k_exps);
    CKV_PTR(v_exps);
  } else if (k_exps || v_exps) {
    return fail(CKV_EINVAL, "a bf16 cache has no exponents");
  }
  const int ps = c->page_size;
  if (ps < 1 || ps > 65536 || (ps & (ps - 1)))
    return fail(CKV_EUNSUPPORTED, "page_size %d (a power of two up to 65536)", ps);
  if (c->num_pages < 1) return fail(CKV_ESHAPE, "num_pages %d", c->num_pages);
  const int64_t slots = ((int64_t)d.max_ctx + ps - 1) / ps;
  if (c->table_stride < slots)
    return fail(CKV_ESHAPE, "table_stride %d below the %lld pages of max_ctx", c->table_stride,
                (long long)slots);
  const int size = e4m3 ? 1 : 2;
  const int64_t strides[3] = {c->page_stride, c->head_stride, c->row_stride};
  for (int64_t x : strides)
    if (x < kD || x > ((int64_t)1 << 36) || x * size % 16)
      return fail(CKV_ESHAPE, "cache stride %lld (128 .. 2^36 elements, a multiple of 16 bytes)",
                  (long long)x);
  if (c->row_stride * size * ps >= ((int64_t)1 << 31))
    return fail(CKV_EUNSUPPORTED, "page_size %d rows at stride %lld reach 2^31 bytes", ps,
                (long long)c->row_stride);
  int64_t last = 0;
  if (__builtin_mul_overflow((int64_t)c->num_pages, c->page_stride * size, &last) ||
      last > ((int64_t)1 << 61))
    return fail(CKV_ESHAPE, "page_stride %lld times %d pages", (long long)c->page_stride,
                c->num_pages);
  p->k = static_cast<uint8_t*>(k_pages);
  p->v = static_cast<uint8_t*>(v_pages);
  p->k_exps = k_exps;
  p->v_exps = v_exps;
  p->table = page_table;
  p->page_bytes = c->page_stride * size;
  p->head_bytes = c->head_stride * size;
  p->row_bytes = (int32_t)(c->row_stride * size);
  p->shift = __builtin_ctz((unsigned)ps);
  p->num_pages = c->num_pages;
  p->table_stride = c->table_stride;
  p->Hkv = d.Hkv;
  return CKV_OK;
}

// Debug mode: the pages that a reading entry (ctx_lens) or a writing entry
// (req, pos) reaches, checked on the device before its launch.
int debug_check_paged(hipStream_t s, const PagedPages& pg, const int32_t* ctx_lens,
                      const int32_t* req, const int32_t* pos, int B, int max_ctx, int tokens) {
  if (!debug_on()) return CKV_OK;
  PagedCheckArgs a;
  a.pg = pg;
  a.ctx_lens = ctx_lens;
  a.req = req;
  a.pos = pos;
  a.B = B;
  a.max_ctx = max_ctx;
  a.tokens = tokens;
  a.slots = (int32_t)(((int64_t)max_ctx + (1 << pg.shift) - 1) >> pg.shift);
  unsigned long long got = 0;
  const int rc = debug_run(
      s,
      [&](unsigned long long* flag) {
        a.flag = flag;
        return launch_paged_check(a, s);
      },
      &got);
  if (rc) return rc;
  if (got == ~0ull) return CKV_OK;
  const unsigned kind = (unsigned)(got >> 56);
  const long long item = (long long)(got & ((1ull << 56) - 1));
  if (kind == 4)
    return fail(CKV_EINVAL, "debug check: page_table[%lld][%lld] is neither -1 nor below %d",
                item / a.slots, item % a.slots, pg.num_pages);
  if (kind == 5)
    return fail(CKV_EINVAL, "debug check: positions[%lld] is neither -1 nor in [0, %d)", item,
                max_ctx);
  if (kind == 6)
    return fail(CKV_EINVAL, "debug check: requests[%lld] outside [0, %d)", item, B);
  return fail(CKV_EINVAL, "debug check: token %lld has no page to be written to", item);
}

#define CKV_RC(expr)             \
  do {                           \
    const int rc_ = (expr);      \
    if (rc_) return rc_;         \
  } while (0)

}  // namespace

extern "C" {

int ckv_rope_rows(const ckv_rope* rope, int32_t num_tokens, const int32_t* positions,
                  const ckv_rows* q, const ckv_rows* k, void* stream) {
  RopeArgs a = {};
  CKV_RC(check_rope(rope, &a.r));
  CKV_RC(check_num_tokens(num_tokens));
  CKV_RC(check_rows("q", q, num_tokens, a.r, &a.q));
  if (k) CKV_RC(check_rows("k", k, num_tokens, a.r, &a.k));
  if (a.q.heads + a.k.heads > 4096)
    return fail(CKV_ESHAPE, "%d heads in q and k (at most 4096)", a.q.heads + a.k.heads);
  if (num_tokens == 0) return CKV_OK;  // without rows their addresses may be NULL
  CKV_PTR(positions);
  a.pos = positions;
  a.tokens = num_tokens;
  CKV_TRY_HIP(launch_rope(a, (hipStream_t)stream), "rope launch");
  return CKV_OK;
}

int ckv_rope_frequencies(int32_t rot_dim, double base, const ckv_rope_scaling* scaling,
                         double* inv_freq, float* rot_scale) {
  if (rot_dim < 2 || rot_dim > 1024 || (rot_dim & 1))
    return fail(CKV_ESHAPE, "rot_dim %d (even, 2 .. 1024)", rot_dim);
  if (!(base > 1.0) || !std::isfinite(base)) return fail(CKV_EINVAL, "base must be above 1");
  if (!inv_freq) return fail(CKV_EINVAL, "inv_freq is NULL");
  const int kind = scaling ? scaling->kind : CKV_ROPE_PLAIN;
  if (kind < CKV_ROPE_PLAIN || kind > CKV_ROPE_RAMP)
    return fail(CKV_EINVAL, "bad scaling.kind %d", kind);
  const double factor = kind == CKV_ROPE_PLAIN ? 1.0 : scaling->factor;
  if (!(factor >= 1.0) || !std::isfinite(factor))
    return fail(CKV_EINVAL, "scaling.factor must be at least 1");
  const double pi = 3.14159265358979323846;
  double low = 0, high = 0, ctx = 0, b = base, i_high = 0, i_low = 0;
  if (kind == CKV_ROPE_BASE) {
    if (rot_dim <= 2) return fail(CKV_ESHAPE, "CKV_ROPE_BASE needs rot_dim above 2");
    b = base * std::pow(factor, (double)rot_dim / (rot_dim - 2));
    if (!std::isfinite(b)) return fail(CKV_EINVAL, "scaling.factor is too large");
  }
  if (kind == CKV_ROPE_BANDS || kind == CKV_ROPE_RAMP) {
    low = scaling->low;
    high = scaling->high;
    ctx = scaling->orig_ctx;
    if (scaling->orig_ctx < 1) return fail(CKV_EINVAL, "scaling.orig_ctx must be at least 1");
    if (!(low >= 0) || !(high > low) || !std::isfinite(high) || (kind == CKV_ROPE_RAMP && low <= 0))
      return fail(CKV_EINVAL, "scaling needs 0 %s low < high", kind == CKV_ROPE_RAMP ? "<" : "<=");
  }
  if (kind == CKV_ROPE_RAMP) {  // r = ctx * base^(-2i/n) / 2 pi, solved for i
    auto index = [&](double r) {
      return rot_dim * std::log(ctx / (r * 2 * pi)) / (2 * std::log(base));
    };
    i_high = std::max(std::floor(index(high)), 0.0);
    i_low = std::min(std::ceil(index(low)), (double)rot_dim - 1);
    if (i_low <= i_high) i_low = i_high + 0.001;  // a step where both fall on one pair
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    const double f = std::pow(b, -2.0 * i / rot_dim);
    double keep = 1.0;  // share of f, the rest of f / factor
    if (kind == CKV_ROPE_LINEAR) keep = 0.0;
    if (kind == CKV_ROPE_BANDS)
      keep = std::min(std::max((ctx * f / (2 * pi) - low) / (high - low), 0.0), 1.0);
    if (kind == CKV_ROPE_RAMP)
      keep = 1.0 - std::min(std::max((i - i_high) / (i_low - i_high), 0.0), 1.0);
    inv_freq[i] = f * keep + f / factor * (1.0 - keep);
  }
  if (rot_scale)
    *rot_scale = kind == CKV_ROPE_RAMP && factor > 1.0 ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return CKV_OK;
}

int ckv_paged_write(const ckv_shape* shape, const ckv_paged_cache* cache, int32_t num_tokens,
                    const int32_t* requests, const int32_t* positions, const uint16_t* k,
                    const uint16_t* v, int64_t kv_token_stride, const ckv_rope* rope,
                    const ckv_rows* q, void* stream) {
  Dims d;
  PagedWriteArgs a = {};
  CKV_RC(check_shape(shape, &d));
  CKV_RC(check_cache(cache, d, &a.pg));
  CKV_RC(check_num_tokens(num_tokens));
  if ((kv_token_stride & 7) || kv_token_stride < (int64_t)d.Hkv * kD ||
      kv_token_stride > ((int64_t)1 << 38))
    return fail(CKV_ESHAPE, "kv_token_stride %lld (>= Hkv * 128, a multiple of 8)",
                (long long)kv_token_stride);
  if (!requests && num_tokens > d.B)
    return fail(CKV_ESHAPE, "%d tokens of %d requests without requests", num_tokens, d.B);
  if (rope) {
    CKV_RC(check_rope(rope, &a.rope.r));
    if (a.rope.r.head_dim != kD || a.rope.r.f32)
      return fail(CKV_EUNSUPPORTED, "a cache's rope has bf16 rows of %d elements", kD);
    if (q) CKV_RC(check_rows("q", q, num_tokens, a.rope.r, &a.rope.q));
  } else if (q) {
    return fail(CKV_EINVAL, "q without rope");
  }
  if (num_tokens == 0) return CKV_OK;  // without rows their addresses may be NULL
  if (requests) CKV_PTR(requests);
  CKV_PTR(positions);
  CKV_PTR(k);
  CKV_PTR(v);
  if (d.U == 0 && !q) return CKV_OK;  // no requests: all tokens are padding
  hipStream_t s = (hipStream_t)stream;
  CKV_RC(debug_check_paged(s, a.pg, nullptr, requests, positions, d.B, d.max_ctx, num_tokens));
  a.rope.pos = positions;
  a.rope.tokens = num_tokens;
  a.req = requests;
  a.k = k;
  a.v = v;
  a.tok = kv_token_stride;
  a.B = d.B;
  a.max_ctx = d.max_ctx;
  CKV_TRY_HIP(launch_paged_write(a, cache->kind == CKV_CACHE_E4M3, s), "paged write launch");
  return CKV_OK;
}

int ckv_paged_read(const ckv_shape* shape, const ckv_paged_cache* cache,
                   const int32_t* ctx_lens, const int32_t* idx, const int32_t* n_sel, int32_t k,
                   uint16_t* k_dst, uint16_t* v_dst, void* stream) {
  Dims d;
  PagedReadArgs a = {};
  CKV_RC(check_shape(shape, &d));
  CKV_RC(check_cache(cache, d, &a.pg));
  if (idx) {
    CKV_RC(check_k(k));
    CKV_PTR(idx);
    CKV_PTR(n_sel);
  } else {
    if (k < 1 || k > (1 << 30)) return fail(CKV_ESHAPE, "k %d outside [1, 2^30]", k);
    if (n_sel) return fail(CKV_EINVAL, "n_sel without idx");
  }
  CKV_PTR(ctx_lens);
  CKV_PTR(k_dst);
  CKV_PTR(v_dst);
  // work-items per dispatch must stay below 2^32
  if ((int64_t)d.U * ((k + kReadSlots - 1) / kReadSlots) >= ((int64_t)1 << 24))
    return fail(CKV_EUNSUPPORTED, "grid too large for this shape");
  if (d.U == 0) return CKV_OK;
  hipStream_t s = (hipStream_t)stream;
  CKV_RC(debug_check(s, ctx_lens, idx, n_sel, d.B, d.Hkv, d.max_ctx, k));
  CKV_RC(debug_check_paged(s, a.pg, ctx_lens, nullptr, nullptr, d.B, d.max_ctx, 0));
  a.ctx_lens = ctx_lens;
  a.idx = idx;
  a.n_sel = n_sel;
  a.k_dst = k_dst;
  a.v_dst = v_dst;
  a.max_ctx = d.max_ctx;
  a.k = k;
  a.units = d.U;
  CKV_TRY_HIP(launch_paged_read(a, cache->kind == CKV_CACHE_E4M3, s), "paged read launch");
  return CKV_OK;
}

int ckv_paged_score_keys(const ckv_shape* shape, const ckv_paged_cache* cache,
                         const uint16_t* q, const int32_t* ctx_lens, float scale, float* scores,
                         void* stream) {
  Dims d;
  PagedScoreArgs a = {};
  CKV_RC(check_shape(shape, &d));
  CKV_RC(check_cache(cache, d, &a.pg));
  CKV_RC(check_scale(scale));
  CKV_PTR(q);
  CKV_PTR(ctx_lens);
  CKV_PTR(scores);
  if (d.U == 0) return CKV_OK;
  hipStream_t s = (hipStream_t)stream;
  CKV_RC(debug_check(s, ctx_lens, nullptr, nullptr, d.B, d.Hkv, d.max_ctx, 1));
  CKV_RC(debug_check_paged(s, a.pg, ctx_lens, nullptr, nullptr, d.B, d.max_ctx, 0));
  a.q = q;
  a.ctx_lens = ctx_lens;
  a.scores = scores;
  a.scale = scale;
  a.Hq = d.Hq;
  a.B = d.B;
  a.max_ctx = d.max_ctx;
  a.units = d.U;
  const int64_t steps = (int64_t)d.U * ((d.max_ctx + kScoreStep - 1) / kScoreStep);
  const int slots = score_wgs_per_cu(a.pg.shift >= 4) * device_cus();
  a.direct = steps <= slots;
  a.nwg = a.direct ? (int)steps : slots;
  a.piece = a.direct ? kScoreStep : kScorePiece;
  a.chunks = (d.max_ctx + a.piece - 1) / a.piece;
  CKV_TRY_HIP(launch_paged_score(a, cache->kind == CKV_CACHE_E4M3, d.G, s), "paged score launch");
  return CKV_OK;
}

int ckv_paged_decode_attn(const ckv_shape* shape, const ckv_paged_cache* cache,
                          int32_t num_tokens, const uint16_t* q, const int32_t* ctx_lens,
                          float scale, float* out, float* lse, void* ws, size_t ws_bytes,
                          void* stream) {
  Dims d;
  PagedAttnArgs a = {};
  CKV_RC(check_shape(shape, &d));
  CKV_RC(check_cache(cache, d, &a.pg));
  CKV_RC(check_tokens(d, num_tokens));
  CKV_RC(check_scale(scale));
  if (scale > 0x1p126f)  // 2 log2(e) times it, a factor of the logits, has to be finite
    return fail(CKV_EINVAL, "scale %g above 2^126", scale);
  CKV_PTR(q);
  CKV_PTR(ctx_lens);
  CKV_PTR(out);
  if (lse) CKV_PTR(lse);
  const size_t need = paged_attn_ws_bytes(d, num_tokens);
  if (!ws) return fail(CKV_EWORKSPACE, "workspace is NULL (%zu bytes needed)", need);
  if (reinterpret_cast<uintptr_t>(ws) & 255u)
    return fail(CKV_EWORKSPACE, "workspace is not 256-byte aligned");
  if (ws_bytes < need)
    return fail(CKV_EWORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
  if (d.U == 0) return CKV_OK;
  hipStream_t s = (hipStream_t)stream;
  CKV_RC(debug_check(s, ctx_lens, nullptr, nullptr, d.B, d.Hkv, d.max_ctx, 1));
  CKV_RC(debug_check_paged(s, a.pg, ctx_lens, nullptr, nullptr, d.B, d.max_ctx, 0));
  a.q = q;
  a.ctx_lens = ctx_lens;
  a.out = out;
  a.lse = lse;
  a.tail = static_cast<PagedTail*>(ws);
  a.flags = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + paged_tail_bytes(d));
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + paged_tail_bytes(d) +
                                    paged_flag_bytes(d));
  a.scale = scale;
  a.B = d.B;
  a.Hq = d.Hq;
  a.T = num_tokens;
  a.lg = __builtin_ctz((unsigned)d.G);
  a.max_ctx = d.max_ctx;
  // pieces of few steps, a workgroup each and all at once (or whole units), whose
  // last one in a unit joins them: one launch, without a scan over the batch
  const int64_t steps = (d.max_ctx + kPagedStep - 1) / kPagedStep;
  const int cap = paged_wgs_cap(d), held = kPagedWgsPerCu * device_cus();
  const int64_t most = std::min(cap, held);
  auto pieces = [&](int lg) { return ((steps - 1) >> lg) + 1; };
  const int64_t joined = std::min<int64_t>(kMaxDirect, kMaxDirectRows / (num_tokens * d.G));
  auto fits = [&](int64_t n) {
    return n <= joined && (d.U * n <= most || (n == 1 && d.U < (1 << 23)));
  };
  int lg = 0;
  while (!fits(pieces(lg)) && lg < (d.U * pieces(lg) > most ? kMaxPiece : kMaxJoinPiece)) ++lg;
  const bool direct = fits(pieces(lg));
  const int64_t n = pieces(lg), wgs = d.U * n;
  a.nwg = direct ? (int)wgs : std::min(cap, d.U < kFewUnits ? device_cus() : held);
  a.chunks = direct ? (int)n : 0;
  a.piece = lg;
  a.tag = next_fused_tag();
  CKV_TRY_HIP(launch_paged_attn(a, cache->kind == CKV_CACHE_E4M3, s), "paged attention launch");
  return CKV_OK;
}

}  // extern "C"
