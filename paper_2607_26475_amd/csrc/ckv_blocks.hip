// ckv_blocks.hip -- gfx950 kernels of the attention over selected blocks of a paged
// cache, and their host-side launchers.
#include "ckv_blocks.hpp"
#include "ckv_paged_tile.hpp"
#include "ckv_profile.hpp"

namespace ckv {

// Token t of a call: its request and position, or -1, -1 where it has none (padding).
struct Token {
  int32_t req, pos;
};

__device__ __forceinline__ Token token_of(const BlockTokens& a, int64_t t) {
  Token x = {-1, -1};
  if (t >= a.n) return x;
  const int pos = a.pos[t], req = a.req ? a.req[t] : (int)t;
  if ((unsigned)pos < (unsigned)a.max_ctx && (unsigned)req < (unsigned)a.B) x = {req, pos};
  return x;
}

// ---- landmarks -------------------------------------------------------------------
// A wave a block: lane (s, c) adds elements [8c, 8c + 8) of rows s, s + 4, ... in
// fp64, the four sums are added in one order, and the mean is rounded once.  Blocks
// are those from first[b]'s on, `slices` workgroups of four waves a unit over them,
// so that the grid does not grow with max_ctx where only the last block is new.
constexpr int kMarkThreads = 256;

template <Kind KIND>
__global__ __launch_bounds__(kMarkThreads) void k_block_marks(MarkArgs a) {
  const int unit = blockIdx.x / a.slices, slice = blockIdx.x - unit * a.slices;
  const int b = unit / a.pg.Hkv, h = unit - b * a.pg.Hkv;
  const int lane = threadIdx.x & 63, c = lane & 15, s = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = clamp_len(((TablePtr)(uintptr_t)a.ctx_lens)[b], a.max_ctx);
  const int from = a.first ? max(((TablePtr)(uintptr_t)a.first)[b], 0) >> a.lb : 0;
  const TablePtr table = table_of(a.pg, b);
  const int block = 1 << a.lb;
  for (int64_t j = (int64_t)from + 4 * slice + wave; j << a.lb < n; j += 4 * a.slices) {
    const int p0 = (int)(j << a.lb), end = min(p0 + block, n);
    double sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    int rows = 0;  // of this lane
    for (int p = p0; p < end; p += 16) {  // 16 positions of one page
      const int page = table[p >> a.pg.shift];
      if ((unsigned)page >= (unsigned)a.pg.num_pages) continue;
      u32x4 w[4];
      uint32_t e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = min(p + 4 * i + s, end - 1);
        const uint8_t* src = a.pg.k + row_offset(a.pg, page, h, row) + row_part(KIND) * c;
        e[i] = 0;
        if (KIND == Kind::kBf16) {
          w[i] = *reinterpret_cast<const u32x4*>(src);
        } else if (KIND == Kind::kE4M3) {
          const uint2 x = *reinterpret_cast<const uint2*>(src);
          w[i] = u32x4{x.x, x.y, 0u, 0u};
          e[i] = a.pg.k_exps[exp_offset(a.pg, page, h, row)];
        } else {
          w[i] = u32x4{*reinterpret_cast<const uint32_t*>(src), 0u, 0u, 0u};
          e[i] = a.pg.k_exps[4 * exp_offset(a.pg, page, h, row) + (c >> 2)];
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (p + 4 * i + s >= end) break;
        ++rows;
        uint4 y = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
        if (KIND == Kind::kE4M3) y = e4m3_octet(make_uint2(y.x, y.y));
        if (KIND == Kind::kE2M1) y = e2m1_octet(y.x, e[i] << 23);
        float x[8];
        unpack8(y, x);
#pragma unroll
        for (int k = 0; k < 8; ++k)
          sum[k] += KIND == Kind::kE4M3 ? ldexp((double)x[k], (int)e[i] - 127) : (double)x[k];
      }
    }
    rows += __shfl_xor(rows, 16);
    rows += __shfl_xor(rows, 32);
    if (rows == 0) continue;  // for the whole wave
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      sum[k] += __shfl_xor(sum[k], 16);
      sum[k] += __shfl_xor(sum[k], 32);
    }
    if (s != 0) continue;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t bits[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const double mean = sum[2 * k + i] / rows;
        bits[i] = mean - mean == 0.0 ? f64_to_bf16_rne(mean) : 0x7fc0u;
      }
      w[k] = bits[0] | bits[1] << 16;
    }
    uint16_t* dst = a.marks + ((int64_t)unit * a.nb + j) * kD + 8 * c;
    *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// ---- selection: scores -------------------------------------------------------------
// Whether a block has a page (pages of at least 16 positions, blocks of at least 32).
__device__ __forceinline__ bool block_there(const PagedPages& pg, TablePtr table, int j, int lb,
                                            int max_ctx) {
  const int first = j << lb, last = min(first + (1 << lb), max_ctx) - 1;
  for (int s = first >> pg.shift; s <= last >> pg.shift; ++s)
    if ((unsigned)table[s] < (unsigned)pg.num_pages) return true;
  return false;
}

// Scores of earlier blocks, the largest over a group's heads, without the scale:
// query rows x landmarks on 16x16x32 products.  A workgroup has MT tiles of query
// rows and a chunk of landmarks, whose 16-column steps its waves share out; the
// tokens of each request in turn.  Landmarks come from the L2, which holds a
// head's; their largest |.|^2 is left for the selection's error bound.
constexpr int kSelThreads = 256;

template <int G, int MT>
__global__ __launch_bounds__(kSelThreads) void k_block_scores(BlockSelectArgs a) {
  constexpr int kTok = 16 / G, kTokens = kTok * MT;
  __shared__ int32_t req[kTokens], own[kTokens];
  __shared__ float most[4];
  const BlockTokens& t = a.t;
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % t.Hkv, rest = blockIdx.x / t.Hkv;
  const int tile = rest / a.chunks, chunk = rest - tile * a.chunks;
  const int64_t t0 = (int64_t)tile * kTokens;
  if (threadIdx.x < kTokens) {
    const Token x = token_of(t, t0 + threadIdx.x);
    req[threadIdx.x] = x.req;
    own[threadIdx.x] = x.pos >> t.lb;  // -1: none
  }
  __syncthreads();
  const int my_req = lane < kTokens ? req[lane] : -1, my_own = lane < kTokens ? own[lane] : -1;
  bf16x8 q[MT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t tok = min(t0 + m * kTok + r / G, (int64_t)t.n - 1);
    const uint16_t* row = t.q + (tok * t.Hq + h * G + r % G) * kD;
#pragma unroll
    for (int f = 0; f < 4; ++f) q[m][f] = as_bf16x8(ld16(row + 32 * f + 8 * g));
  }
  float norm = 0.f;
  uint64_t left = __ballot(my_req >= 0);
  while (left) {
    const int rq = __builtin_amdgcn_readlane(my_req, __builtin_ctzll(left));
    const bool member = my_req == rq;
    left &= ~__ballot(member);
    int last = member ? my_own : 0;  // blocks that some token of the request has behind it
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) last = max(last, __shfl_xor(last, o));
    const int stop = min((chunk + 1) * a.cols, last);
    const TablePtr table = table_of(a.pg, rq);
    const uint16_t* marks = a.marks + ((int64_t)rq * t.Hkv + h) * t.nb * kD;
    for (int j0 = chunk * a.cols + 16 * wave; j0 < stop; j0 += 64) {
      const int j = j0 + r;
      const uint16_t* mark = marks + (int64_t)min(j, stop - 1) * kD + 8 * g;
      uint4 w[4];
#pragma unroll
      for (int f = 0; f < 4; ++f) w[f] = ld16(mark + 32 * f);
      const bool there = j < stop && block_there(a.pg, table, j, t.lb, t.max_ctx);
      float sq = 0.f;
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        float x[8];
        unpack8(w[f], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) sq = fmaf(x[i], x[i], sq);
      }
      sq += __shfl_xor(sq, 16);
      sq += __shfl_xor(sq, 32);
      if (there) norm = fmaxf(norm, sq);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int f = 0; f < 4; ++f) acc = mfma_16x16x32(q[m][f], as_bf16x8(w[f]), acc);
        // register i of lane (g, r): query row 4g + i, landmark r
        constexpr int kPer = G < 4 ? 4 / G : 1;  // tokens of a lane
        float best[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          best[i] = acc[i * (G < 4 ? G : 4)];
#pragma unroll
          for (int k = 1; k < (G < 4 ? G : 4); ++k)
            best[i] = fmaxf(best[i], acc[i * (G < 4 ? G : 4) + k]);
        }
        if (G >= 8) best[0] = fmaxf(best[0], __shfl_xor(best[0], 16));
        if (G == 16) best[0] = fmaxf(best[0], __shfl_xor(best[0], 32));
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int tok = m * kTok + 4 * g / G + i;
          if ((4 * g) % G == 0 && req[tok] == rq && j < own[tok] && j < stop)
            a.scores[((t0 + tok) * t.Hkv + h) * t.nb + j] =
                there ? fmaxf(best[i], -INFINITY) : -INFINITY;  // of NaN: -inf
        }
      }
    }
  }
  norm = wave_max(norm);
  if (lane == 0) most[wave] = norm;
  __syncthreads();
  if (threadIdx.x == 0)
    a.norms[((int64_t)tile * t.Hkv + h) * a.chunks + chunk] =
        fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
}

// ---- selection: the best -------------------------------------------------------------
// A wave a (token, KV head).  The set is the one of exact scores: fp32 sums of 128
// exact products are off by at most e = 2^-16 |q| |landmark| (2^-15 here, for the
// norms' own rounding), so with the r-th best fp32 score x the blocks above x + 2e
// are in, those below x - 2e are out, and the few between are ranked by their
// scores in fp64, the lower block first where these are equal.
//   The r-th best is found by halving an interval of scores until exactly r lie
// above (8 halvings or so; ties end it at neighbouring floats).  The scores of up
// to 64 V blocks are held in registers, of more read again at each halving.
__device__ __forceinline__ float wave_min(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fminf(x, __shfl_xor(x, o));
  return x;
}

// The group's best score of a block in fp64, the same in every lane: 64 / G lanes
// a head, each 2 G channels in order.
template <int G>
__device__ __forceinline__ double exact_score(const uint16_t* q, const uint16_t* mark) {
  constexpr int kPer = 64 / G;
  const int lane = threadIdx.x & 63, head = lane / kPer, at = 2 * G * (lane % kPer);
  double s = 0.0;
  for (int c = 0; c < 2 * G; c += 2) {
    const uint32_t x = *reinterpret_cast<const uint32_t*>(q + head * kD + at + c);
    const uint32_t y = *reinterpret_cast<const uint32_t*>(mark + at + c);
    s += (double)__uint_as_float(x << 16) * (double)__uint_as_float(y << 16);
    s += (double)__uint_as_float(x & 0xffff0000u) * (double)__uint_as_float(y & 0xffff0000u);
  }
#pragma unroll
  for (int o = 1; o < kPer; o <<= 1) s += __shfl_xor(s, o);
#pragma unroll
  for (int o = kPer; o < 64; o <<= 1) s = fmax(s, __shfl_xor(s, o));
  return s;
}

__device__ __forceinline__ float float_of_key(uint32_t k) {
  return __uint_as_float(key_floor_bits(k));
}

template <int G, int V>
__global__ __launch_bounds__(kSelThreads) void k_select_blocks(BlockSelectArgs a) {
  const BlockTokens& t = a.t;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * (kSelThreads / 64) +
                       __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= (int64_t)t.n * t.Hkv) return;
  const int tok = (int)(unit / t.Hkv), h = (int)(unit - (int64_t)tok * t.Hkv);
  const Token x = token_of(t, tok);
  int32_t* out = a.idx + unit * t.k;
  if (x.req < 0) {
    if (lane < t.k) out[lane] = -1;
    return;
  }
  const int n = x.pos >> t.lb, want = t.k - 1;  // earlier blocks; of them kept
  const float* scores = a.scores + unit * t.nb;
  const int steps = V ? V : (n + 63) / 64;
  float held[V ? V : 1];
#pragma unroll
  for (int i = 0; i < V; ++i)
    held[i] = 64 * i + lane < n ? scores[64 * i + lane] : -INFINITY;
  auto score = [&](int i) {
    if constexpr (V > 0) return held[i];
    else return 64 * i + lane < n ? scores[64 * i + lane] : -INFINITY;
  };
  auto each = [&](auto fn) {
    if constexpr (V > 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) fn(i, score(i));
    } else {
      for (int i = 0; i < steps; ++i) fn(i, score(i));
    }
  };
  auto above = [&](float x) {  // scores of at least x
    int m = 0;
    each([&](int, float s) { m += __popcll(__ballot(s >= x)); });
    return m;
  };
  float lo_s = INFINITY, hi_s = -INFINITY;
  int avail = 0;
  each([&](int, float s) {
    const bool is = s > -INFINITY;
    avail += __popcll(__ballot(is));
    lo_s = fminf(lo_s, is ? s : INFINITY);
    hi_s = fmaxf(hi_s, s);
  });
  // those above `sure` are in; of those from `maybe` on the ones in `mine` (lanes
  // below `few`)
  float sure = -INFINITY, maybe = INFINITY;
  int few = 0, mine = -1;
  if (avail > want) {
    lo_s = wave_min(lo_s);
    hi_s = wave_max(hi_s);
    sure = INFINITY;
    if (want > 0) {
      uint32_t lo = order_key(lo_s), hi = order_key(hi_s) + 1;  // above(lo) > want > above(hi)
      float cut = float_of_key(lo);
      bool even = false;  // exactly `want` of at least `cut`
      for (int round = 0; hi - lo > 1; ++round) {
        uint32_t mid = lo + (hi - lo) / 2;
        if (round < 20) {
          const float m = 0.5f * float_of_key(lo) + 0.5f * float_of_key(hi - 1);
          const uint32_t k = order_key(m);
          if (k > lo && k < hi) mid = k;
        }
        const float f = float_of_key(mid);
        const int m = above(f);
        if (m >= want) lo = mid, cut = f;
        else hi = mid;
        if (m == want) {
          even = true;
          break;
        }
      }
      // the want-th best, the best one less than it, and the error of either
      float in = INFINITY, out_s = -INFINITY;
      each([&](int, float s) {
        if (s >= cut) in = fminf(in, s);
        else out_s = fmaxf(out_s, s);
      });
      in = wave_min(in);
      out_s = wave_max(out_s);
      const uint16_t* q = t.q + ((int64_t)tok * t.Hq + h * G) * kD;
      float qq = 0.f, mm = 0.f;
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(q + i * kD + 2 * lane);
        const float y = __uint_as_float(w << 16), z = __uint_as_float(w & 0xffff0000u);
        qq = fmaf(y, y, fmaf(z, z, qq));
      }
      qq = wave_sum(qq);
      const int per = (16 / G) * a.row_tiles;
      const float* norms = a.norms + ((int64_t)(tok / per) * t.Hkv + h) * a.chunks;
      for (int i = lane; i < (n + a.cols - 1) / a.cols; i += 64) mm = fmaxf(mm, norms[i]);
      mm = wave_max(mm);
      // (squares that vanish are below 2^-126: the bounds of 2^-100 cover them)
      const float e2 = 0x1p-14f * sqrtf(fmaxf(qq, 0x1p-100f)) * sqrtf(fmaxf(mm, 0x1p-100f));
      sure = in + e2;
      if (even && in - out_s > e2) {
        sure = out_s;  // nothing between: all from `cut` on are above it
      } else {
        maybe = in - e2;
        int need = want;
        each([&](int, float s) { need -= __popcll(__ballot(s > sure)); });
        const uint16_t* marks = a.marks + ((int64_t)x.req * t.Hkv + h) * t.nb * kD;
        double best = 0.0;  // lane i: the i-th best of those between
        each([&](int i, float s) {
          uint64_t some = __ballot(s > -INFINITY && !(s > sure) && !(s < maybe));
          while (some) {
            const int j = 64 * i + __builtin_ctzll(some);
            some &= some - 1;
            const double v = exact_score<G>(q, marks + (int64_t)j * kD);
            const int at = __popcll(__ballot(lane < few && best >= v));
            if (at >= need) continue;
            const double up = __shfl_up(best, 1);
            const int j_up = __shfl_up(mine, 1);
            if (lane > at) best = up, mine = j_up;
            if (lane == at) best = v, mine = j;
            few = min(few + 1, need);
          }
        });
      }
    }
  }
  int m = 0;
  each([&](int i, float s) {
    const int j = 64 * i + lane;
    bool in = s > sure;
    const bool between = !in && s > -INFINITY && !(s < maybe);
    if (__any(between))
      for (int k = 0; k < few; ++k)
        if (between && __builtin_amdgcn_readlane(mine, k) == j) in = true;
    const uint64_t all = __ballot(in);
    const int at = m + __popcll(all & ((1ull << lane) - 1));
    if (in && at < want) out[at] = j;
    m += __popcll(all);
  });
  m = min(m, want);
  if (lane >= m && lane < t.k) out[lane] = lane == m ? n : -1;
}

// ---- attention -------------------------------------------------------------------------
// A workgroup has one tile: 16 query rows of 16 / G tokens that follow each other,
// and the blocks that any of them keeps, each with the tokens that keep it.  Blocks
// that several of the tokens keep are loaded and multiplied once, so neighbouring
// tokens, whose lists are mostly alike, share the work; the worst case is a list for
// each.  Steps of 32 positions go to the four waves in turn, as in the decode
// attention; rows whose token does not keep the block, or that lie before the
// position, are masked.  Few tiles: the steps of a list are cut into pieces, a
// workgroup each, and joined by a second launch.
constexpr int kBlockThreads = 256;
constexpr int kStepLg = 5;  // log2 of a wave's positions
static_assert(1 << kStepLg == kPagedTile, "a step");

struct BlockLds {
  float m[4][16], l[4][16];
  float o[4][16][kPartStride];
  int32_t pos[16], req[16], end[16];
  uint32_t list[16 * kMaxKept];   // the tokens' blocks (all ones: none)
  int32_t block[16 * kMaxKept];   // of the tile, each once
  uint32_t who[16 * kMaxKept];    // its tokens' bits, and the first of them << 16
  int32_t count[4];
};

// Whether token i's ascending list holds block v.
__device__ __forceinline__ bool holds(const BlockLds& lds, int i, int k, uint32_t v) {
  int lo = 0, hi = k;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (lds.list[i * k + mid] < v) lo = mid + 1;
    else hi = mid;
  }
  return lo < k && lds.list[i * k + lo] == v;
}

// The tile's tokens and blocks into lds; how many blocks.
__device__ __forceinline__ int gather_blocks(const BlockAttnArgs& a, int64_t t0, int h,
                                             BlockLds& lds) {
  const BlockTokens& t = a.t;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tokens = 16 >> t.lg, n = tokens * t.k;
  if (tid < 16) {
    const Token x = tid < tokens ? token_of(t, t0 + tid) : Token{-1, -1};
    lds.req[tid] = x.req;
    lds.pos[tid] = x.pos;
  }
  __syncthreads();
  for (int e = tid; e < n; e += kBlockThreads) {
    const int i = e / t.k;
    uint32_t v = ~0u;
    if (lds.req[i] >= 0) {
      const int j = a.idx[((t0 + i) * t.Hkv + h) * t.k + (e - i * t.k)];
      if ((unsigned)j <= (unsigned)(lds.pos[i] >> t.lb)) v = (uint32_t)j;
    }
    lds.list[e] = v;
  }
  if (tid < tokens) {  // positions that the request's tokens of this tile see
    int end = 0;
    for (int i = 0; i < tokens; ++i)
      if (lds.req[i] == lds.req[tid]) end = max(end, lds.pos[i] + 1);
    lds.end[tid] = end;
  }
  __syncthreads();
  int total = 0;
  for (int e0 = 0; e0 < n; e0 += kBlockThreads) {
    const int e = e0 + tid, i = e / t.k;
    uint32_t who = 0, v = ~0u;
    if (e < n && (v = lds.list[e]) != ~0u && (e == i * t.k || lds.list[e - 1] != v)) {
      for (int o = 0; o < tokens; ++o) {
        if (lds.req[o] != lds.req[i] || !(o == i || holds(lds, o, t.k, v))) continue;
        if (o < i) {
          who = 0;
          break;
        }
        who |= 1u << o;
      }
    }
    const uint64_t some = __ballot(who != 0);
    if (lane == 0) lds.count[wave] = __popcll(some);
    __syncthreads();
    int at = total + __popcll(some & ((1ull << lane) - 1));
    for (int w = 0; w < 4; ++w) {
      if (w < wave) at += lds.count[w];
      total += lds.count[w];
    }
    if (who) {
      lds.block[at] = (int)v;
      lds.who[at] = who | (uint32_t)i << 16;
    }
    __syncthreads();
  }
  return total;
}

// Where a step of the tile's list lies.
struct BlockStep {
  Ctx x;
  int p0;
  uint32_t who;
  TileAt<true> at;
};

__device__ __forceinline__ BlockStep block_step(const BlockAttnArgs& a, const BlockLds& lds, int h,
                                                int s) {
  const int lg = a.t.lb - kStepLg, e = s >> lg;
  BlockStep b;
  b.who = __builtin_amdgcn_readfirstlane(lds.who[e]);
  const int first = b.who >> 16;
  b.x.b = __builtin_amdgcn_readfirstlane(lds.req[first]);
  b.x.n = __builtin_amdgcn_readfirstlane(lds.end[first]);
  b.x.h = h;
  b.x.table = table_of(a.pg, b.x.b);
  b.p0 = (__builtin_amdgcn_readfirstlane(lds.block[e]) << a.t.lb) +
         ((s - (e << lg)) << kStepLg);
  b.at = tile_at<true>(a.pg, b.x, b.p0);
  return b;
}

__device__ __forceinline__ void store_block_row(const BlockAttnArgs& a, int64_t t0, int h, int row,
                                                int d, const Partial& p) {
  const int64_t tok = t0 + (row >> a.t.lg);
  if (tok >= a.t.n) return;
  const int64_t at = tok * a.t.Hq + (h << a.t.lg) + (row & ((1 << a.t.lg) - 1));
  const float inv = inverse_sum(p.L);
  *reinterpret_cast<float4*>(a.out + at * kD + d) =
      make_float4(p.o.x * inv, p.o.y * inv, p.o.z * inv, p.o.w * inv);
  if (a.lse && d == 0) a.lse[at] = log_sum(p.M, p.L);
}

template <Kind KIND>
__global__ __launch_bounds__(kBlockThreads, 2) void k_block_attn(BlockAttnArgs a) {
  __shared__ BlockLds lds;
  const BlockTokens& bt = a.t;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % bt.Hkv, rest = blockIdx.x / bt.Hkv;
  const int tile = rest / a.pieces, piece = rest - tile * a.pieces;
  const int64_t t0 = (int64_t)tile * (16 >> bt.lg);
  const int blocks = gather_blocks(a, t0, h, lds);
  const int64_t steps = (int64_t)blocks << (bt.lb - kStepLg);
  const int s1 = (int)(steps * (piece + 1) / a.pieces);
  int s = (int)(steps * piece / a.pieces) + wave;
  const int row_tok = r >> bt.lg;
  const int my_end = lds.pos[row_tok] + 1;
  const int64_t tok = min(t0 + row_tok, (int64_t)bt.n - 1);
  const uint16_t* qrow =
      bt.q + (tok * bt.Hq + (h << bt.lg) + (r & ((1 << bt.lg) - 1))) * kD;
  bf16x8 q[4];
#pragma unroll
  for (int f = 0; f < 4; ++f) q[f] = as_bf16x8(ld16(qrow + frag_base<KIND>(f, g)));
  // e4m3 exponents are taken less 128 (as in the decode attention)
  const float c = a.scale * (KIND == Kind::kE4M3 ? 2.f : 1.f) * 1.4426950408889634f;
  WaveState st;
  st.m = -INFINITY;
  st.l = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) st.o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (s < s1) {
    Tile<KIND> t;
    float lg[8];
    BlockStep now = block_step(a, lds, h, s);
    load_k<KIND, true>(a.pg, now.x, now.at, t);
    load_v<KIND, true>(a.pg, now.x, now.at, t);
    s += 4;
    BlockStep next = block_step(a, lds, h, min(s, s1 - 1));
    auto limit = [&] { return now.who >> row_tok & 1u ? my_end : 0; };
    while (s < s1) {
      tile_logits<KIND, true>(t, q, lg);
      load_k<KIND, true>(a.pg, next.x, next.at, t);
      __builtin_amdgcn_sched_barrier(0);
      tile_rest<KIND>(t, true, now.p0, limit(), now.x.n, c, lg, st);
      __builtin_amdgcn_sched_barrier(0);
      load_v<KIND, true>(a.pg, next.x, next.at, t);
      now = next;
      s += 4;
      next = block_step(a, lds, h, min(s, s1 - 1));
    }
    tile_logits<KIND, true>(t, q, lg);
    tile_rest<KIND>(t, true, now.p0, limit(), now.x.n, c, lg, st);
  }
  st.l += __shfl_xor(st.l, 16);
  st.l += __shfl_xor(st.l, 32);
  if (g == 0) {
    lds.m[wave][r] = st.m;
    lds.l[wave][r] = st.l;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float* o = &lds.o[wave][r][8 * (4 * g + j)];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = KIND == Kind::kE4M3 ? 2.f * st.o[e][j] : st.o[e][j];
  }
  __syncthreads();
  for (int i = tid; i < 16 * (kD / 4); i += kBlockThreads) {
    const int row = i >> 5, d = 4 * (i & 31);
    const Partial p = join_waves(lds, row, d);
    if (a.pieces == 1) {
      store_block_row(a, t0, h, row, d, p);
      continue;
    }
    float* part = a.part + ((((int64_t)tile * bt.Hkv + h) * a.pieces + piece) * 16 + row) *
                               kPartStride;
    *reinterpret_cast<float4*>(part + 4 + d) = p.o;
    if (d == 0) {
      part[0] = p.M;
      part[1] = p.L;
    }
  }
}

// Joins a tile's pieces in order: a thread has a row and four channels.
__global__ __launch_bounds__(kBlockThreads) void k_block_merge(BlockAttnArgs a) {
  const int h = blockIdx.x % a.t.Hkv, tile = blockIdx.x / a.t.Hkv;
  const int64_t t0 = (int64_t)tile * (16 >> a.t.lg);
  const float* part = a.part + ((int64_t)tile * a.t.Hkv + h) * a.pieces * 16 * kPartStride;
  for (int i = threadIdx.x; i < 16 * (kD / 4); i += kBlockThreads) {
    const int row = i >> 5, d = 4 * (i & 31);
    const float* p0 = part + (int64_t)row * kPartStride;
    Partial p;
    p.M = -INFINITY;
    p.L = 0.f;
    p.o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < a.pieces; ++k) p.M = fmaxf(p.M, p0[(int64_t)k * 16 * kPartStride]);
    for (int k = 0; k < a.pieces; ++k) {
      const float* x = p0 + (int64_t)k * 16 * kPartStride;
      const float f = x[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[0] - p.M);
      const float4 o = *reinterpret_cast<const float4*>(x + 4 + d);
      p.L = fmaf(f, x[1], p.L);
      p.o.x = fmaf(f, o.x, p.o.x);
      p.o.y = fmaf(f, o.y, p.o.y);
      p.o.z = fmaf(f, o.z, p.o.z);
      p.o.w = fmaf(f, o.w, p.o.w);
    }
    store_block_row(a, t0, h, row, d, p);
  }
}

// ---- launchers ---------------------------------------------------------------------------
hipError_t launch_marks(const MarkArgs& a, Kind kind, hipStream_t s) {
  of_kind(kind, [&](auto k) {
    launch_kernel(CKV_K_BLOCK_MARKS, k_block_marks<k.value>, dim3(a.B * a.pg.Hkv * a.slices),
                  dim3(kMarkThreads), s, a);
  });
  return launch_status();
}

template <class Fn>
static void of_group(int lg, Fn fn) {
  switch (lg) {
    case 0: fn(std::integral_constant<int, 1>{}); break;
    case 1: fn(std::integral_constant<int, 2>{}); break;
    case 2: fn(std::integral_constant<int, 4>{}); break;
    case 3: fn(std::integral_constant<int, 8>{}); break;
    default: fn(std::integral_constant<int, 16>{});
  }
}

hipError_t launch_select_blocks(const BlockSelectArgs& a, hipStream_t s) {
  const dim3 block(kSelThreads);
  of_group(a.t.lg, [&](auto g) {
    constexpr int G = g.value;
    const dim3 grid((unsigned)(tiles_of(a.t, a.row_tiles) * a.chunks * a.t.Hkv));
    if (a.row_tiles == 4)
      launch_kernel(CKV_K_BLOCK_SCORE, k_block_scores<G, 4>, grid, block, s, a);
    else
      launch_kernel(CKV_K_BLOCK_SCORE, k_block_scores<G, 1>, grid, block, s, a);
    const dim3 waves((unsigned)(((int64_t)a.t.n * a.t.Hkv + 3) / 4));
    if (a.t.nb <= 256)
      launch_kernel(CKV_K_BLOCK_SELECT, k_select_blocks<G, 4>, waves, block, s, a);
    else if (a.t.nb <= 1024)
      launch_kernel(CKV_K_BLOCK_SELECT, k_select_blocks<G, 16>, waves, block, s, a);
    else
      launch_kernel(CKV_K_BLOCK_SELECT, k_select_blocks<G, 0>, waves, block, s, a);
  });
  return launch_status();
}

hipError_t launch_block_attn(const BlockAttnArgs& a, Kind kind, hipStream_t s) {
  const int64_t units = tiles_of(a.t) * a.t.Hkv;
  of_kind(kind, [&](auto k) {
    launch_kernel(CKV_K_BLOCK_ATTN, k_block_attn<k.value>, dim3((unsigned)(units * a.pieces)),
                  dim3(kBlockThreads), s, a);
  });
  const hipError_t e = launch_status();
  if (e != hipSuccess || a.pieces == 1) return e;
  launch_kernel(CKV_K_BLOCK_MERGE, k_block_merge, dim3((unsigned)units), dim3(kBlockThreads), s,
                a);
  return launch_status();
}

}  // namespace ckv
