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

// ---- reductions over a wave --------------------------------------------------------
// By lane moves alone (an LDS round trip at each of six steps would be the latency of
// what one wave does here): rows of 16 by rotations, then rows and halves exchanged.
// The result is the same in every lane.
template <class Op>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t x, Op op) {
  x = op(x, dpp_u32<0x128, 0xF, false>(x));  // row_ror
  x = op(x, dpp_u32<0x124, 0xF, false>(x));
  x = op(x, dpp_u32<0x122, 0xF, false>(x));
  x = op(x, dpp_u32<0x121, 0xF, false>(x));
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = op(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return __builtin_amdgcn_readfirstlane(op(b[0], b[1]));
}

__device__ __forceinline__ uint32_t wave_min_u32(uint32_t x) {
  return wave_reduce(x, [](uint32_t a, uint32_t b) { return min(a, b); });
}

template <class Op>
__device__ __forceinline__ float wave_reduce_f32(float x, Op op) {
  return __uint_as_float(wave_reduce(__float_as_uint(x), [op](uint32_t a, uint32_t b) {
    return __float_as_uint(op(__uint_as_float(a), __uint_as_float(b)));
  }));
}

__device__ __forceinline__ float wave_min_f32(float x) {
  return wave_reduce_f32(x, [](float a, float b) { return fminf(a, b); });
}

__device__ __forceinline__ float wave_max_f32(float x) {
  return wave_reduce_f32(x, [](float a, float b) { return fmaxf(a, b); });
}

__device__ __forceinline__ float wave_sum_f32(float x) {
  return wave_reduce_f32(x, [](float a, float b) { return a + b; });
}

// ---- landmarks -------------------------------------------------------------------
// A wave a block: lane (s, c) adds elements [8c, 8c + 8) of rows s, s + 4, ... in
// fp64, the four sums are added in one order, and the mean is rounded once.  Blocks
// are those from first[b]'s on, `slices` workgroups of four waves a unit over them,
// so that the grid does not grow with max_ctx where only the last block is new.  What
// bounds it are dependent loads (length, first, pages, rows) and the fp64 sums' joining:
// pages of 64 rows at once, then all rows, and each lane the join of two channels (128
// new blocks 12.1 -> 5.8 us, those of 2048 new tokens 14.5 -> 9.3).
constexpr int kMarkThreads = 256, kMarkRows = 64;  // rows in flight

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
    for (int p = p0; p < end; p += kMarkRows) {  // 16 positions are of one page
      int page[kMarkRows / 16];
      u32x4 w[kMarkRows / 4];
      uint32_t e[kMarkRows / 4];
#pragma unroll
      for (int i = 0; i < kMarkRows / 16; ++i)
        page[i] = table[min(p + 16 * i, end - 1) >> a.pg.shift];
#pragma unroll
      for (int i = 0; i < kMarkRows / 4; ++i) {
        const int row = min(p + 4 * i + s, end - 1);
        // (rows past the end are of the last one's page)
        const int there = (unsigned)page[i >> 2] < (unsigned)a.pg.num_pages ? page[i >> 2] : 0;
        const uint8_t* src = a.pg.k + row_offset(a.pg, there, h, row) + row_part(KIND) * c;
        e[i] = 0;
        if (KIND == Kind::kBf16) {
          w[i] = *reinterpret_cast<const u32x4*>(src);
        } else if (KIND == Kind::kE4M3) {
          const uint2 x = *reinterpret_cast<const uint2*>(src);
          w[i] = u32x4{x.x, x.y, 0u, 0u};
          e[i] = a.pg.k_exps[exp_offset(a.pg, there, h, row)];
        } else {
          w[i] = u32x4{*reinterpret_cast<const uint32_t*>(src), 0u, 0u, 0u};
          e[i] = a.pg.k_exps[4 * exp_offset(a.pg, there, h, row) + (c >> 2)];
        }
      }
#pragma unroll
      for (int i = 0; i < kMarkRows / 4; ++i) {
        if (p + 4 * i + s >= end || (unsigned)page[i >> 2] >= (unsigned)a.pg.num_pages) continue;
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
    // the four lanes of eight channels add them up, half of them each, then a quarter
    double four[4], two[2];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const double other = __shfl_xor(s & 1 ? sum[k] : sum[4 + k], 16);
      four[k] = (s & 1 ? sum[4 + k] : sum[k]) + other;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const double other = __shfl_xor(s & 2 ? four[k] : four[2 + k], 32);
      two[k] = (s & 2 ? four[2 + k] : four[k]) + other;
    }
    uint32_t bits[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const double mean = two[i] / rows;
      bits[i] = mean - mean == 0.0 ? f64_to_bf16_rne(mean) : 0x7fc0u;
    }
    uint16_t* dst =
        a.marks + ((int64_t)unit * a.nb + j) * kD + 8 * c + 4 * (s & 1) + 2 * (s >> 1);
    *reinterpret_cast<uint32_t*>(dst) = bits[0] | bits[1] << 16;
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
// head's; their largest |.|^2 is left for the selection's error bound.  16 tokens over
// 22 MB of landmarks 10 us; 2048 tokens over 256 landmarks of each of 8 heads 23, of
// which the 17 MB of scores are 4: short chains of loads and products, 1024 workgroups.
constexpr int kSelThreads = 256;

// Sixteen landmarks of a request on their way.
struct ScoreStep {
  uint4 w[4];
  int req, j, stop;  // j: the lane's, below stop
  bool there;
};

template <int G, int MT>
__global__ __launch_bounds__(kSelThreads, 4) void k_block_scores(BlockSelectArgs a) {
  constexpr int kTok = 16 / G, kTokens = kTok * MT;
  __shared__ int32_t req[kTokens], own[kTokens];
  __shared__ int32_t each_req[kTokens], each_last[kTokens];  // requests, once each
  __shared__ float most[4];
  const BlockTokens& t = a.t;
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % t.Hkv, rest = blockIdx.x / t.Hkv;
  const int tile = rest / a.chunks, chunk = rest - tile * a.chunks;
  const int64_t t0 = (int64_t)tile * kTokens;
  const Token x = token_of(t, lane < kTokens ? t0 + lane : (int64_t)t.n);
  const int my_own = x.pos >> t.lb;  // -1: none
  if (threadIdx.x < kTokens) {
    req[lane] = x.req;
    own[lane] = my_own;
  }
  bf16x8 q[MT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t tok = min(t0 + m * kTok + r / G, (int64_t)t.n - 1);
    const uint16_t* row = t.q + (tok * t.Hq + h * G + r % G) * kD;
#pragma unroll
    for (int f = 0; f < 4; ++f) q[m][f] = as_bf16x8(ld16(row + 32 * f + 8 * g));
  }
  int requests = 0;
  uint64_t left = __ballot(x.req >= 0);
  while (left) {
    const int rq = __builtin_amdgcn_readlane(x.req, __builtin_ctzll(left));
    const bool member = x.req == rq;
    left &= ~__ballot(member);
    // blocks that some token of the request has behind it
    const int last = (int)~wave_min_u32(member ? ~(uint32_t)my_own : ~0u);
    if (threadIdx.x == 0) {
      each_req[requests] = rq;
      each_last[requests] = last;
    }
    ++requests;
  }
  __syncthreads();
  // A chunk's steps of 16 landmarks, request by request, go to the waves in turn.
  const int per = a.cols / 16, items = requests * per;
  int item = wave;
  auto ask = [&](ScoreStep& s) {
    for (; item < items; item += 4) {
      const int i = item / per, j0 = chunk * a.cols + 16 * (item - i * per);
      s.stop = min((chunk + 1) * a.cols, __builtin_amdgcn_readfirstlane(each_last[i]));
      if (j0 >= s.stop) continue;
      s.req = __builtin_amdgcn_readfirstlane(each_req[i]);
      s.j = j0 + r;
      const int j = min(s.j, s.stop - 1);
      const uint16_t* mark = a.marks + (((int64_t)s.req * t.Hkv + h) * t.nb + j) * kD + 8 * g;
#pragma unroll
      for (int f = 0; f < 4; ++f) s.w[f] = ld16(mark + 32 * f);
      s.there = block_there(a.pg, table_of(a.pg, s.req), j, t.lb, t.max_ctx) && s.j < s.stop;
      item += 4;
      return true;
    }
    return false;
  };
  float norm = 0.f;
  constexpr bool kAhead = MT == 1;  // (registers for it, and fewer waves to take turns)
  ScoreStep s, next;
  bool more = ask(s);
  while (more) {
    if (kAhead) more = ask(next);
    float sq = 0.f;
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      float y[8];
      unpack8(s.w[f], y);
#pragma unroll
      for (int i = 0; i < 8; ++i) sq = fmaf(y[i], y[i], sq);
    }
    sq += __shfl_xor(sq, 16);
    sq += __shfl_xor(sq, 32);
    if (s.there) norm = fmaxf(norm, sq);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int f = 0; f < 4; ++f) acc = mfma_16x16x32(q[m][f], as_bf16x8(s.w[f]), acc);
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
        // (what is no finite number, +inf here, is summed again by the selection)
        if ((4 * g) % G == 0 && req[tok] == s.req && s.j < own[tok] && s.j < s.stop)
          a.scores[((t0 + tok) * t.Hkv + h) * t.nb + s.j] =
              !s.there ? -INFINITY : fabsf(best[i]) < INFINITY ? best[i] : INFINITY;
      }
    }
    if (kAhead) s = next;
    else more = ask(s);
  }
  norm = wave_max_f32(norm);
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
// to 64 V blocks are held in registers, of more read again at each halving.  A chain of
// about 2000 instructions of one wave: 13 us for 128 (token, KV head) pairs of up to
// 1024 blocks, 26 for 16384 of 256; 64 pairs of 1900 blocks read again 71, held 21.
// Query rows of a group for scores in fp64: 64 / G lanes a head, each 2 G channels.
template <int G>
struct GroupRows {
  static constexpr int kPer = 64 / G;
  uint32_t w[G];
  int at;  // of the lane's channels
  __device__ __forceinline__ void load(const uint16_t* q) {
    const int lane = threadIdx.x & 63;
    at = 2 * G * (lane % kPer);
    const uint32_t* p = reinterpret_cast<const uint32_t*>(q + lane / kPer * kD + at);
#pragma unroll
    for (int i = 0; i < G; ++i) w[i] = p[i];
  }
  // The largest |.|^2 of a head.
  __device__ __forceinline__ float norm() const {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const float y = __uint_as_float(w[i] << 16), z = __uint_as_float(w[i] & 0xffff0000u);
      s = fmaf(y, y, fmaf(z, z, s));
    }
#pragma unroll
    for (int o = 1; o < kPer; o <<= 1) s += __shfl_xor(s, o);
#pragma unroll
    for (int o = kPer; o < 64; o <<= 1) s = fmaxf(s, __shfl_xor(s, o));
    return s;
  }
  // The best scores of four blocks, the same in every lane.
  __device__ __forceinline__ void scores(const uint16_t* marks, const int* j, double* out) const {
    uint32_t m[4][G];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t* p = reinterpret_cast<const uint32_t*>(marks + (int64_t)j[k] * kD + at);
#pragma unroll
      for (int i = 0; i < G; ++i) m[k][i] = p[i];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      double s = 0.0;
#pragma unroll
      for (int i = 0; i < G; ++i) {
        s += (double)__uint_as_float(w[i] << 16) * (double)__uint_as_float(m[k][i] << 16);
        s += (double)__uint_as_float(w[i] & 0xffff0000u) *
             (double)__uint_as_float(m[k][i] & 0xffff0000u);
      }
      out[k] = s;
    }
#pragma unroll
    for (int o = 1; o < kPer; o <<= 1)
#pragma unroll
      for (int k = 0; k < 4; ++k) out[k] += __shfl_xor(out[k], o);
#pragma unroll
    for (int o = kPer; o < 64; o <<= 1)
#pragma unroll
      for (int k = 0; k < 4; ++k) out[k] = fmax(out[k], __shfl_xor(out[k], o));
  }
};

// A score whose fp32 sum is no finite number, summed in fp64: past fp32's range its
// largest, so that what is not there or no number stays below.  (|q|^2 or |landmark|^2
// passes that range too, so the error bound is infinite, and such scores are ranked in
// fp64.)
template <int G>
__device__ __forceinline__ float wide_score(const uint16_t* q, const uint16_t* mark) {
  double best = -INFINITY;
#pragma unroll 1
  for (int k = 0; k < G; ++k) {
    double s = 0.0;
#pragma unroll 1
    for (int i = 0; i < kD; ++i)
      s += (double)__uint_as_float((uint32_t)q[k * kD + i] << 16) *
           (double)__uint_as_float((uint32_t)mark[i] << 16);
    best = fmax(best, s);  // of NaN: -inf
  }
  const double most = 3.4028234663852886e38;
  return (float)(best - best == 0.0 ? fmin(fmax(best, -most), most) : best);
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
  // asked for now, used by the error bound
  GroupRows<G> rows;
  rows.load(t.q + ((int64_t)tok * t.Hq + h * G) * kD);
  const int per = (16 / G) * a.row_tiles;
  const float* norms = a.norms + ((int64_t)(tok / per) * t.Hkv + h) * a.chunks;
  float mm = 0.f;
  for (int i = lane; i < (n + a.cols - 1) / a.cols; i += 64) mm = fmaxf(mm, norms[i]);
  float* scores = a.scores + unit * t.nb;
  const int steps = V ? V : (n + 63) / 64;
  float held[V ? V : 1];
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
  float lo_s, hi_s;
  int avail;
  const uint16_t* marks = a.marks + ((int64_t)x.req * t.Hkv + h) * t.nb * kD;
  for (bool again = false;; again = true) {
    // (addresses and masks that are the same in both rounds would be kept for the second:
    // 512 pairs of 4000 blocks 36.6 us for 34.3, 16384 of 2048 97 for 80)
    int at = lane;
    asm volatile("" : "+v"(at));
#pragma unroll
    for (int i = 0; i < V; ++i) held[i] = 64 * i + at < n ? scores[64 * i + at] : -INFINITY;
    lo_s = INFINITY, hi_s = -INFINITY, avail = 0;
    each([&](int, float s) {
      const bool is = s > -INFINITY;
      avail += __popcll(__ballot(is));
      lo_s = fminf(lo_s, is ? s : INFINITY);
      hi_s = fmaxf(hi_s, s);
    });
    if (again || !__any(hi_s == INFINITY)) break;
    for (int j = lane; j < n; j += 64)
      if (scores[j] == INFINITY)
        scores[j] = wide_score<G>(t.q + ((int64_t)tok * t.Hq + h * G) * kD, marks + (int64_t)j * kD);
  }
  // those above `sure` are in; of those from `maybe` on the ones in `mine` (lanes
  // below `few`)
  float sure = -INFINITY, maybe = INFINITY;
  int few = 0, mine = -1;
  if (avail > want) {
    lo_s = wave_min_f32(lo_s);
    hi_s = wave_max_f32(hi_s);
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
      in = wave_min_f32(in);
      out_s = wave_max_f32(out_s);
      const float qq = rows.norm();
      mm = wave_max_f32(mm);
      // (squares that vanish are below 2^-126: the bounds of 2^-100 cover them)
      const float e2 = 0x1p-14f * sqrtf(fmaxf(qq, 0x1p-100f)) * sqrtf(fmaxf(mm, 0x1p-100f));
      sure = in + e2;
      if (even && in - out_s > e2) {
        sure = out_s;  // nothing between: all from `cut` on are above it
      } else {
        maybe = in - e2;
        int need = want;
        each([&](int, float s) { need -= __popcll(__ballot(s > sure)); });
        auto between = [&](float s) { return s > -INFINITY && !(s > sure) && !(s < maybe); };
        int total = 0;
        each([&](int, float s) { total += __popcll(__ballot(between(s))); });
        double best = 0.0;  // lane i: the i-th best of those between
        for (int base = 0; base < total; base += 64) {
          int cand = -1, seen = -base;  // lane i: the i-th of 64 of them, four at a time
          each([&](int i, float s) {
            for (uint64_t some = __ballot(between(s)); some; some &= some - 1, ++seen)
              if (lane == seen) cand = 64 * i + __builtin_ctzll(some);
          });
          const int count = min(total - base, 64);
          for (int c0 = 0; c0 < count; c0 += 4) {
            int j[4];
            double v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
              j[k] = __builtin_amdgcn_readlane(cand, min(c0 + k, count - 1));
            rows.scores(marks, j, v);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int at = __popcll(__ballot(lane < few && best >= v[k]));
              if (c0 + k >= count || at >= need) continue;
              const double up = __shfl_up(best, 1);
              const int j_up = __shfl_up(mine, 1);
              if (lane > at) best = up, mine = j_up;
              if (lane == at) best = v[k], mine = j[k];
              few = min(few + 1, need);
            }
          }
        }
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
//   Codes have to be made bf16 and V's rows transposed by byte permutes at every step:
// the vector unit bounds it, 370 instructions a step of 32 four-bit positions (2103
// tokens, 8 blocks of 128, groups of 8: 135 us; without masks where a step needs none,
// the maximum raised ahead, three workgroups a CU: 107; blocks in ascending order and
// rows kept in the caches: 104).  16 tokens of as many
// requests, 32 blocks of 64 each: 17 us, and 4 of joining.
constexpr int kBlockThreads = 256;
constexpr int kStepLg = 5;  // log2 of a wave's positions
static_assert(1 << kStepLg == kPagedTile, "a step");

struct BlockLds {
  float m[4][16], l[4][16];
  int32_t pos[16], req[16];
  int32_t count[4];
  union {
    float o[4][16][kPartStride];
    struct {                         // until the last step
      uint32_t list[16 * kMaxKept];  // the tokens' blocks (all ones: none)
      int32_t block[16 * kMaxKept];  // of the tile, each once
      uint32_t who[16 * kMaxKept];   // its tokens' bits, and the first of them << 16
    int32_t end[16 * kMaxKept];    // the positions that these see
    };
  };
};

// Whether token i's list, ascending and then all ones, holds block v.
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
  // A token's blocks together at the front of its list, where a search finds them and
  // finds them ascending: a wave a token, all of its lists asked for at once.
  static_assert(kMaxKept == 64, "a lane an entry");
  uint32_t mine[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int i = 4 * x + wave;
    mine[x] = ~0u;
    if (i < tokens && lds.req[i] >= 0 && lane < t.k)
      mine[x] = (uint32_t)a.idx[((t0 + i) * t.Hkv + h) * t.k + lane];
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int i = 4 * x + wave;
    if (i >= tokens) break;
    const bool counts = (int)mine[x] >= 0 && (int)mine[x] <= lds.pos[i] >> t.lb;
    const uint64_t all = __ballot(counts);
    const int before = __popcll(all & ((1ull << lane) - 1)), count = __popcll(all);
    if (lane < t.k)  // (what does not count, behind what does)
      lds.list[i * t.k + (counts ? before : count + lane - before)] = counts ? mine[x] : ~0u;
  }
  __syncthreads();
  int total = 0;
  for (int e0 = 0; e0 < n; e0 += kBlockThreads) {
    const int e = e0 + tid, i = e / t.k;
    uint32_t who = 0, v = ~0u;
    int end = 0;
    if (e < n && (v = lds.list[e]) != ~0u && (e == i * t.k || lds.list[e - 1] != v)) {
      for (int o = 0; o < tokens; ++o) {
        if (lds.req[o] != lds.req[i] || !(o == i || holds(lds, o, t.k, v))) continue;
        if (o < i) {
          who = 0;
          break;
        }
        who |= 1u << o;
        end = max(end, lds.pos[o] + 1);
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
      lds.end[at] = end;
    }
    __syncthreads();
  }
  // Of many tiles in ascending order, where a thread has one entry to rank (longer lists,
  // more than 256 blocks for 16 rows, share little and stay as they are): their workgroups go through a context together, and
  // find in the L2 what others have read (512 bf16 tokens 200 -> 161 us, 2048 e4m3 ones
  // 360 -> 298; with rows streamed past the caches the order changes nothing).
  if (a.pieces > 1 || total > kBlockThreads) return total;
  uint32_t block = 0, who = 0;
  int rank = 0, end = 0;
  if (tid < total) {
    block = (uint32_t)lds.block[tid];
    who = lds.who[tid];
    end = lds.end[tid];
    for (int e = 0; e < total; ++e) {
      const uint32_t other = (uint32_t)lds.block[e];
      rank += other < block || (other == block && e < tid);
    }
  }
  __syncthreads();
  if (tid < total) {
    lds.block[rank] = (int)block;
    lds.who[rank] = who;
    lds.end[rank] = end;
  }
  __syncthreads();
  return total;
}

// Where a step of the tile's list lies.
struct BlockStep {
  Ctx x;
  int p0;
  uint32_t who;
  TileAt<true> at;
};

// Step s (below s1) or, where none of its block's tokens sees that, the wave's next one
// that is seen: rows behind what they see may not have been written, and bytes of theirs
// that make a NaN would have the sums made again (64 tokens 5 positions into blocks of
// 256, 75 us and 163).  From s1 on the place of the last step, which nobody takes.
__device__ __forceinline__ BlockStep block_step(const BlockAttnArgs& a, const BlockLds& lds, int h,
                                                int& s, int s1) {
  const int lg = a.t.lb - kStepLg;
  BlockStep b;
  for (int e;; s += 4) {
    const int at = min(s, s1 - 1);
    e = at >> lg;
    b.who = __builtin_amdgcn_readfirstlane(lds.who[e]);
    b.x.n = __builtin_amdgcn_readfirstlane(lds.end[e]);
    b.p0 = (__builtin_amdgcn_readfirstlane(lds.block[e]) << a.t.lb) +
           ((at - (e << lg)) << kStepLg);
    if (s >= s1 || b.p0 < b.x.n) break;
  }
  b.x.b = __builtin_amdgcn_readfirstlane(lds.req[b.who >> 16]);
  b.x.h = h;
  b.x.table = table_of(a.pg, b.x.b);
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

// raise_max to HEAD above the largest logit, so that it stays until one passes that:
// sums are scaled at the first steps only, and no weight is above 1 (sums of V next to
// its type's largest would else pass fp32's range).
template <int HEAD>
__device__ __forceinline__ void raise_max_above(float top, float c, WaveState& st) {
  const float m = query_row_max(top) * c;
  const bool more = m > st.m;
  if (__any(more)) {
    const float to = m + HEAD;
    const float f = !more ? 1.f : st.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.m - to);
    st.l *= f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int j = 0; j < 4; ++j) st.o[e][j] *= f;
    if (more) st.m = to;
  }
}

// Powers of two that the maximum is raised above the logits: an e4m3 row's weight takes
// the row's exponent with it, down to 2^-128, where products lose what is below 2^-126
// (8 as for the others: 2048 tokens 300 -> 291 us).
template <Kind KIND>
constexpr int kHead = KIND == Kind::kE4M3 ? 1 : 8;

// The weights of a step and its products with V.  APART: these a token at a time,
// without the rows that it does not see, for V rows whose product with a weight of
// zero is no zero.
template <Kind KIND, bool APART>
__device__ __forceinline__ void block_rest(const BlockAttnArgs& a, Tile<KIND>& t, int p0,
                                           int limit, int n, float c, float* lg, WaveState& st) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  if (KIND == Kind::kE4M3) {
#pragma unroll
    for (int j = 0; j < 8; ++j) lg[j] = scaled(lg[j], t.ke[j >> 2] ^ 0x80808080u, j & 3);
  }
  // Rows whose token does not keep the block get weights of exp2(-inf); single
  // positions are left out only where a step has such.
  const bool kept = limit > p0;
  if (APART || t.there != 255u || __any(kept && limit < p0 + kPagedTile))
    tile_mask<KIND>(t, p0, limit, n, lg);
  raise_max_above<kHead<KIND>>(kept ? top_of(lg) : -INFINITY, c, st);
  uint32_t part[3][8];
  tile_weights<KIND>(t.ve, c, kept ? less_max(st) : -INFINITY, lg, part, st);
  if (!APART) {
    tile_output<KIND>(t, part, st);
    return;
  }
  for (int k = 0; k < 16 >> a.t.lg; ++k) {
    const int end = __builtin_amdgcn_readlane(limit, k << a.t.lg);
    if (end <= p0) continue;
    Tile<KIND> seen = t;
    WaveState one = st;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (p0 + 16 * (j >> 2) + 4 * g + (j & 3) < end) continue;
#pragma unroll
      for (int i = 0; i < Tile<KIND>::kV; ++i) seen.v[j][i] = 0u;
      if (KIND == Kind::kE2M1) seen.ve[j] = 0u;
    }
    tile_output<KIND>(seen, part, one);
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (r >> a.t.lg == k) st.o[e][j] = one.o[e][j];
  }
}

// The waves' sums of a piece of a tile's list, into lds; false: they hold a NaN, and
// nothing is written.
template <Kind KIND, bool APART>
__device__ __forceinline__ bool block_sums(const BlockAttnArgs& a, BlockLds& lds, int h, int tile,
                                           int piece, int blocks) {
  const BlockTokens& bt = a.t;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t t0 = (int64_t)tile * (16 >> bt.lg);
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
  // (as constants the sums would be held twice, and copied at each step)
#pragma unroll
  for (int e = 0; e < 8; ++e) asm("" : "+v"(st.o[e]));
  BlockStep now;
  if (s < s1) now = block_step(a, lds, h, s, s1);
  if (s < s1) {
    Tile<KIND> t;
    float lg[8];
    load_k<KIND, true, false>(a.pg, now.x, now.at, t);
    load_v<KIND, true, false>(a.pg, now.x, now.at, t);
    s += 4;
    BlockStep next = block_step(a, lds, h, s, s1);
    auto limit = [&] { return now.who >> row_tok & 1u ? my_end : 0; };
    for (;;) {  // (the last step asks for K rows that nobody takes)
      tile_logits<KIND, true>(t, q, lg);
      load_k<KIND, true, false>(a.pg, next.x, next.at, t);
      __builtin_amdgcn_sched_barrier(0);
      block_rest<KIND, APART>(a, t, now.p0, limit(), now.x.n, c, lg, st);
      __builtin_amdgcn_sched_barrier(0);
      if (s >= s1) break;
      load_v<KIND, true, false>(a.pg, next.x, next.at, t);
      now = next;
      s += 4;
      next = block_step(a, lds, h, s, s1);
    }
  }
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int j = 0; j < 4; ++j) bad = bad || st.o[e][j] != st.o[e][j];
  // (barriers: the lists have been read)
  if (APART) __syncthreads();
  else if (__builtin_amdgcn_readfirstlane(__syncthreads_or(bad))) return false;
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
  return true;
}

// The rare case out of line, so that it costs the ordinary one no registers: its
// arguments are read again from where the kernel has them.
typedef const __attribute__((address_space(4))) BlockAttnArgs* BlockAttnArgsPtr;
typedef __attribute__((address_space(3))) uint8_t* LdsPtr;

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(LdsPtr)p;
}

__device__ __forceinline__ BlockAttnArgs args_at(uint64_t args) {
  const uint64_t at = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(args >> 32)) << 32 |
                      (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)args);
  return *(const BlockAttnArgs*)(BlockAttnArgsPtr)at;
}

template <Kind KIND>
__device__ __attribute__((noinline)) void block_sums_apart(uint64_t args, uint32_t lds, int h,
                                                           int tile, int piece, int blocks) {
  const BlockAttnArgs a = args_at(args);
  block_sums<KIND, true>(
      a, *(BlockLds*)(LdsPtr)(uintptr_t)__builtin_amdgcn_readfirstlane(lds),
      __builtin_amdgcn_readfirstlane(h), __builtin_amdgcn_readfirstlane(tile),
      __builtin_amdgcn_readfirstlane(piece), __builtin_amdgcn_readfirstlane(blocks));
}

template <Kind KIND>
__global__ __launch_bounds__(kBlockThreads, 3) void k_block_attn(BlockAttnArgs a) {
  __shared__ BlockLds lds;
  const BlockTokens& bt = a.t;
  const int tid = threadIdx.x;
  const int h = blockIdx.x % bt.Hkv, rest = blockIdx.x / bt.Hkv;
  const int tile = rest / a.pieces, piece = rest - tile * a.pieces;
  const int64_t t0 = (int64_t)tile * (16 >> bt.lg);
  const int blocks = gather_blocks(a, t0, h, lds);
  if (!block_sums<KIND, false>(a, lds, h, tile, piece, blocks))
    block_sums_apart<KIND>((uint64_t)__builtin_amdgcn_kernarg_segment_ptr(), lds_address(&lds), h,
                           tile, piece, blocks);
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

// Joins a tile's pieces: a wave has a row, each lane a piece's maximum and sum; then
// half a wave adds the even pieces' channels, four a lane, the other the odd ones'.
__global__ __launch_bounds__(kBlockThreads) void k_block_merge(BlockAttnArgs a) {
  const int lane = threadIdx.x & 63, half = lane >> 5, d = 4 * (lane & 31);
  const int row = (blockIdx.x & 3) * 4 + (threadIdx.x >> 6), unit = blockIdx.x >> 2;
  const int h = unit % a.t.Hkv, tile = unit / a.t.Hkv;
  const int64_t t0 = (int64_t)tile * (16 >> a.t.lg);
  const float* part = a.part + ((int64_t)unit * a.pieces * 16 + row) * kPartStride;
  auto piece = [&](int k) { return part + (int64_t)k * 16 * kPartStride; };
  static_assert(kMaxPieces <= 64, "a lane a piece");
  float m = -INFINITY, l = 0.f;
  if (lane < a.pieces) m = piece(lane)[0], l = piece(lane)[1];
  Partial p;
  p.M = wave_max_f32(m);
  const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - p.M);
  p.L = wave_sum_f32(f * l);
  p.o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = 0; k0 < a.pieces; k0 += 16) {
    float4 o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      o[i] = *reinterpret_cast<const float4*>(piece(min(k0 + 2 * i + half, a.pieces - 1)) + 4 + d);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int k = k0 + 2 * i + half;
      const float w = __shfl(f, k & 63);
      if (k >= a.pieces) continue;
      p.o.x = fmaf(w, o[i].x, p.o.x);
      p.o.y = fmaf(w, o[i].y, p.o.y);
      p.o.z = fmaf(w, o[i].z, p.o.z);
      p.o.w = fmaf(w, o[i].w, p.o.w);
    }
  }
  p.o.x += __shfl_xor(p.o.x, 32);
  p.o.y += __shfl_xor(p.o.y, 32);
  p.o.z += __shfl_xor(p.o.z, 32);
  p.o.w += __shfl_xor(p.o.w, 32);
  if (half == 0) store_block_row(a, t0, h, row, d, p);
}

// ---- attention of many tokens --------------------------------------------------------
// For a bf16 cache, whose rows many tokens would otherwise fetch from the L2 again and
// again: a workgroup has four tiles, a wave each.  The blocks that any of its tokens
// keeps are taken in ascending order, 32 positions at a time, into LDS, the next ones
// while these are multiplied; a wave passes over what none of its tokens keeps.  V's
// operands are made by transposing LDS reads, without byte permutes, and no waves are
// joined.  All workgroups go through the positions alike, so that a head's L2 has what
// they need (2048 tokens, 16 of 256 blocks of 64 each: 0.4 GB of 2.4 from behind it;
// a workgroup a tile reads 5.1, 3.3 of it from behind): 297 us, a workgroup a tile 606.
// What bounds it now is the chain of a step (barrier, the next step's place, products,
// weights, products: 2 us with four workgroups a CU) of which a wave takes part in half.
// Three buffers, loads two steps ahead, leave three workgroups a CU: 422 us.
//   The blocks' order is a merge of the tokens' lists, each lane the cursor of a
// token: the least head of all is next, the lanes that have it are its tokens.
//   Rows are 256 bytes, the 16-byte part p of row i = 8 a + b (a < 2) at p ^ (2 b + a):
// 16 rows of a part, K's operand, and 8 rows of two parts, V's, are in all banks.
constexpr int kManyThreads = 64 * kManyTiles;
constexpr uint32_t kRowBytes = 2 * kD;
constexpr uint32_t kHalfBytes = 16 * kRowBytes, kRowsBytes = 2 * kHalfBytes;
constexpr int kBlockBits = 25;  // max_ctx <= 2^30 in blocks of 32

struct ManyLds {
  alignas(256) uint8_t rows[4 * kPagedTile * kRowBytes];  // [buffer][K, V][row]
  int32_t counts[64];
};

// 32 positions of a block, the same for the workgroup.
struct ManyStep {
  uint64_t who;     // its tokens
  int p0, stop, n;  // stop: where its block ends for the tokens, n: for the request's
  int req;
  int first[2], page[2];
  int pages;        // lane i: page[i & 1]
  __device__ __forceinline__ void take_pages() {
    page[0] = __builtin_amdgcn_readlane(pages, 0);
    page[1] = __builtin_amdgcn_readlane(pages, 1);
  }
  __device__ __forceinline__ bool there(const PagedPages& pg, int i) const {
    return (unsigned)page[i] < (unsigned)pg.num_pages;
  }
};

// A lane's token and its place in its list.
struct ManyCursor {
  int req, end;     // the request's positions that the workgroup's tokens see
  uint32_t rank;
  uint32_t head;    // of the list (unless at == count)
  int at, count;
  const uint32_t* list;
  __device__ __forceinline__ uint32_t key() const {
    return at < count ? rank << kBlockBits | head : ~0u;
  }
};

// The step after s; false: none.
__device__ __forceinline__ bool next_step(const BlockAttnArgs& a, ManyCursor& c, ManyStep& s) {
  s.p0 += kPagedTile;
  if (s.p0 >= s.stop) {
    const uint32_t key = c.key(), least = wave_min_u32(key);
    if (least == ~0u) return false;
    s.who = __ballot(key == least);
    c.at += key == least;
    c.head = c.list[c.at];
    const int l = __builtin_ctzll(s.who);
    s.req = __builtin_amdgcn_readlane(c.req, l);
    s.n = __builtin_amdgcn_readlane(c.end, l);
    s.p0 = (int)(least & ((1u << kBlockBits) - 1)) << a.t.lb;
    s.stop = min(s.p0 + (1 << a.t.lb), s.n);
  }
  // The halves' pages by a vector load, to be looked at a step later: a scalar one
  // would have to be back before the next read of LDS.
#pragma unroll
  for (int i = 0; i < 2; ++i) s.first[i] = half_first(s.p0, i, s.n);
  s.pages = table_of(a.pg, s.req)[(threadIdx.x & 1 ? s.first[1] : s.first[0]) >> a.pg.shift];
  return true;
}

__device__ __forceinline__ uint32_t part_at(int row, int part) {
  return row * kRowBytes + ((part ^ (row << 1 & 14) ^ (row >> 3 & 1)) << 4);
}

// 64 times 16 bytes from base + offset (a lane's) to LDS bytes [to, to + 1024), without
// registers between; there once this wave's vmcnt is 0.  (The builtin makes the
// compiler wait for it at the next read of any LDS, of the other buffer too.)
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t offset, uint32_t to) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2"
      :
      : "s"(to), "v"(offset), "s"(base)
      : "memory", "m0");
}

// (A builtin, which tells the compiler that nothing of its own is in flight either.)
__device__ __forceinline__ void wait_for_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt 0
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ void stage_load(const BlockAttnArgs& a, ManyLds& lds, int buf, int h,
                                           const ManyStep& s) {
  const PagedPages& pg = a.pg;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int v = wave >> 1, half = wave & 1;  // a wave has a half of K or V
  const bool there = half ? s.there(pg, 1) : s.there(pg, 0);
  const int page = there ? half ? s.page[1] : s.page[0] : 0;
  const int first = half ? s.first[1] : s.first[0], last = half_last(first, s.n);
  const uint8_t* rows = (v ? pg.v : pg.k) + row_offset(pg, page, h, first);
  uint8_t* dst = lds.rows + (2 * buf + v) * kRowsBytes + half * kHalfBytes;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 4 * i + (lane >> 4);
    uint8_t* to = dst + 4 * i * kRowBytes;
    if (there)
      load_to_lds(rows, min(row, last) * pg.row_bytes + (part_at(row, lane & 15) & 255u),
                  lds_address(to));
    else
      *reinterpret_cast<uint4*>(to + 16 * lane) = make_uint4(0, 0, 0, 0);
  }
}

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Channels of four rows transposed: lane i of 16 gives the 8 bytes that hold channels
// [4 (i % 4), ...) of row i / 4 and gets channel i of the four rows.
__device__ __forceinline__ uint2 read_transposed(const uint8_t* p) {
  return __builtin_bit_cast(
      uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                 (__attribute__((address_space(3))) s16x4*)(p)));
}

// Rows of four positions from the n-th on as zeros.
__device__ __forceinline__ uint2 first_of(uint2 x, int n) {
  const uint64_t keep = n <= 0 ? 0ull : n >= 4 ? ~0ull : (1ull << 16 * n) - 1;
  return make_uint2(x.x & (uint32_t)keep, x.y & (uint32_t)(keep >> 32));
}

// A wave's 16 query rows over one step.  APART: the products with V a token at a time,
// without the rows that it does not see, for V rows whose product with a weight of
// zero is no zero.
template <bool APART>
__device__ __forceinline__ void many_step(const BlockAttnArgs& a, const ManyLds& lds, int buf,
                                          const ManyStep& s, const bf16x8* q, float c, int tok,
                                          int my_end, WaveState& st) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int limit = s.who >> tok & 1 ? my_end : 0;
  if (!__any(limit > s.p0)) return;
  float lg[8];
  // (offsets from the buffer's on, so that they are not held in registers)
  const uint32_t k = 2 * buf * kRowsBytes + part_at(r, g);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int f = 0; f < 4; ++f)
      x = mfma_16x16x32(as_bf16x8(*static_cast<const uint4*>(__builtin_assume_aligned(
                            lds.rows + (k ^ 64u * f) + i * kHalfBytes, 16))),
                        q[f], x);
#pragma unroll
    for (int j = 0; j < 4; ++j) lg[4 * i + j] = x[j];
  }
  // Rows whose token does not keep the block get weights of exp2(-inf); single
  // positions are left out only where a step has such.
  const bool kept = limit > s.p0;
  if (APART || !s.there(a.pg, 0) || !s.there(a.pg, 1) ||
      __any(kept && limit < s.p0 + kPagedTile)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int end = s.there(a.pg, j >> 2) ? limit : 0;
      if (s.p0 + 16 * (j >> 2) + 4 * g + (j & 3) >= end) lg[j] = -INFINITY;
    }
  }
  const int row = 4 * g + (r >> 2);
  const uint32_t v = (2 * buf + 1) * kRowsBytes + part_at(row, (r >> 1) & 1) + 8 * (r & 1);
  uint4 rows[4];  // of V, for four times 16 channels
  auto read_rows = [&](int part) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint8_t* p = lds.rows + (v ^ 32u * (4 * part + e));
      const uint2 lo = read_transposed(p), hi = read_transposed(p + kHalfBytes);
      rows[e] = make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  };
  read_rows(0);  // on their way while the weights are made
  raise_max_above<kHead<Kind::kBf16>>(kept ? top_of(lg) : -INFINITY, c, st);
  uint32_t part[3][8];
  tile_weights<Kind::kBf16>(nullptr, c, kept ? less_max(st) : -INFINITY, lg, part, st);
  bf16x8 w[3];
  pack_weights(part, w);
  if (!APART) {
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      if (part) read_rows(1);
#pragma unroll
      for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          st.o[4 * part + e] = mfma_16x16x32(as_bf16x8(rows[e]), w[i], st.o[4 * part + e]);
    }
    return;
  }
  for (int t = 0; t < 16 >> a.t.lg; ++t) {
    const int end = __builtin_amdgcn_readlane(limit, t << a.t.lg) - s.p0 - 4 * g;
    if (__builtin_amdgcn_readlane(limit, t << a.t.lg) <= s.p0) continue;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      read_rows(part);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint2 lo = first_of(make_uint2(rows[e].x, rows[e].y), end);
        const uint2 hi = first_of(make_uint2(rows[e].z, rows[e].w), end - 16);
        f32x4 o = st.o[4 * part + e];
#pragma unroll
        for (int i = 0; i < 3; ++i)
          o = mfma_16x16x32(as_bf16x8(make_uint4(lo.x, lo.y, hi.x, hi.y)), w[i], o);
        if (r >> a.t.lg == t) st.o[4 * part + e] = o;
      }
    }
  }
}

template <bool APART>
__device__ __forceinline__ void many_steps(const BlockAttnArgs& a, ManyLds& lds, ManyCursor& cur,
                                           int h, const bf16x8* q, float c, int tok, int my_end,
                                           WaveState& st) {
  st.m = -INFINITY;
  st.l = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) st.o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  cur.at = 0;
  cur.head = cur.list[0];
  // (as constants the sums would be held twice, and copied at each step)
#pragma unroll
  for (int e = 0; e < 8; ++e) asm("" : "+v"(st.o[e]));
  ManyStep now, next;
  next.p0 = next.stop = 0;
  if (!next_step(a, cur, next)) return;  // the same for the workgroup
  next.take_pages();
  stage_load(a, lds, 0, h, next);
  now = next;
  bool more = next_step(a, cur, next);
  for (int buf = 0;; buf ^= 1) {
    // the rows are in LDS, the other buffer's have been used
    wait_for_loads();
    lds_barrier();
    if (more) {
      next.take_pages();
      stage_load(a, lds, buf ^ 1, h, next);
    }
    ManyStep then = next;
    const bool last = !more;
    if (more) more = next_step(a, cur, then);
    many_step<APART>(a, lds, buf, now, q, c, tok, my_end, st);
    if (last) break;
    now = next;
    next = then;
  }
}

// A workgroup's output; false: its sums hold a NaN, and nothing is written but the lists
// and counts, which the call with APART takes as they are.
template <bool APART>
__device__ __forceinline__ bool many_tiles(const BlockAttnArgs& a, ManyLds& lds, uint32_t* lists,
                                           int block) {
  const BlockTokens& bt = a.t;
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = block % bt.Hkv, tile = block / bt.Hkv;
  const int tokens = 64 >> bt.lg;
  const int64_t t0 = (int64_t)tile * tokens;
  const Token x = lane < tokens ? token_of(bt, t0 + lane) : Token{-1, -1};
  ManyCursor cur = {x.req, 0, 0, 0, 0, 0, lists + min(lane, tokens - 1) * bt.k};
  uint64_t left = __ballot(x.req >= 0);
  while (left) {  // each request once
    const int l = __builtin_ctzll(left);
    const bool member = x.req == __builtin_amdgcn_readlane(x.req, l);
    const int end = (int)~wave_min_u32(member ? ~(uint32_t)(x.pos + 1) : ~0u);
    if (member) cur.rank = l, cur.end = end;
    left &= ~__ballot(member);
  }
  // what counts of a list, close together
  for (int i = wave; !APART && i < tokens; i += kManyTiles) {
    const int req = __builtin_amdgcn_readlane(x.req, i);
    const int pos = __builtin_amdgcn_readlane(x.pos, i);
    uint32_t v = ~0u;
    if (req >= 0 && lane < bt.k) {
      const int j = a.idx[((t0 + i) * bt.Hkv + h) * bt.k + lane];
      if ((unsigned)j <= (unsigned)(pos >> bt.lb)) v = (uint32_t)j;
    }
    // once each: the entry before is the last one that counts
    const uint64_t some = __ballot(v != ~0u) & ((1ull << lane) - 1);
    const uint32_t before = __shfl(v, some ? 63 - __builtin_clzll(some) : lane);
    const bool keep = v != ~0u && (some == 0 || before != v);
    const uint64_t all = __ballot(keep);
    if (keep) lists[i * bt.k + __popcll(all & ((1ull << lane) - 1))] = v;
    if (lane == 0) lds.counts[i] = __popcll(all);
  }
  __syncthreads();
  if (lane < tokens) cur.count = lds.counts[lane];
  const int tok = (wave << 4 | r) >> bt.lg;
  const int my_end = __shfl(x.pos, tok) + 1;
  const int64_t token = t0 + tok;
  const int64_t row = min(token, (int64_t)bt.n - 1) * bt.Hq + (h << bt.lg) +
                      (r & ((1 << bt.lg) - 1));
  bf16x8 q[4];
#pragma unroll
  for (int f = 0; f < 4; ++f) q[f] = as_bf16x8(ld16(bt.q + row * kD + 32 * f + 8 * g));
  const float c = a.scale * 1.4426950408889634f;
  WaveState st;
  many_steps<APART>(a, lds, cur, h, q, c, tok, my_end, st);
  if (!APART) {
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int j = 0; j < 4; ++j) bad = bad || st.o[e][j] != st.o[e][j];
    if (__builtin_amdgcn_readfirstlane(__syncthreads_or(bad))) return false;
  }
  st.l += __shfl_xor(st.l, 16);
  st.l += __shfl_xor(st.l, 32);
  const float inv = inverse_sum(st.l);
  float* out = a.out + row * kD + 4 * g;
  if (token < bt.n) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      *reinterpret_cast<float4*>(out + 16 * e) = make_float4(
          st.o[e][0] * inv, st.o[e][1] * inv, st.o[e][2] * inv, st.o[e][3] * inv);
    if (a.lse && g == 0) a.lse[row] = log_sum(st.m, st.l);
  }
  return true;
}

__device__ __attribute__((noinline)) void many_tiles_apart(uint64_t args, uint32_t lds,
                                                           uint32_t lists, int block) {
  const BlockAttnArgs a = args_at(args);
  many_tiles<true>(
      a, *(ManyLds*)(LdsPtr)(uintptr_t)__builtin_amdgcn_readfirstlane(lds),
      (uint32_t*)(LdsPtr)(uintptr_t)__builtin_amdgcn_readfirstlane(lists),
      __builtin_amdgcn_readfirstlane(block));
}

__global__ __launch_bounds__(kManyThreads, 4) void k_block_attn_many(BlockAttnArgs a) {
  __shared__ ManyLds lds;
  extern __shared__ uint32_t lists[];  // [tokens][k], and a word that an ended list reads
  if (!many_tiles<false>(a, lds, lists, blockIdx.x))
    many_tiles_apart((uint64_t)__builtin_amdgcn_kernarg_segment_ptr(), lds_address(&lds),
                     lds_address(lists), blockIdx.x);
}

// ---- debug mode ------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_check_lists(BlockListArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < (int64_t)a.t.n * a.t.Hkv && !block_list_ascends(a, i))
    atomicMin(a.flag, (unsigned long long)i);
}

// ---- launchers ---------------------------------------------------------------------------
hipError_t launch_marks(const MarkArgs& a, Kind kind, hipStream_t s) {
  of_kind(kind, [&](auto k) {
    launch_kernel(CKV_K_BLOCK_MARKS, k_block_marks<k.value>, dim3(a.B * a.pg.Hkv * a.slices),
                  dim3(kMarkThreads), s, a);
  });
  return launch_status();
}

hipError_t launch_check_lists(const BlockListArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.t.n * a.t.Hkv;
  hipLaunchKernelGGL(k_check_lists, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
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
    else if (a.t.nb <= 2048)
      launch_kernel(CKV_K_BLOCK_SELECT, k_select_blocks<G, 32>, waves, block, s, a);
    else if (a.t.nb <= 4096)
      launch_kernel(CKV_K_BLOCK_SELECT, k_select_blocks<G, 64>, waves, block, s, a);
    else
      launch_kernel(CKV_K_BLOCK_SELECT, k_select_blocks<G, 0>, waves, block, s, a);
  });
  return launch_status();
}

hipError_t launch_block_attn(const BlockAttnArgs& a, Kind kind, hipStream_t s) {
  if (a.many) {
    const size_t lists = sizeof(uint32_t) * (a.t.k * (kManyTiles * 16 >> a.t.lg) + 1);
    launch_kernel_lds(CKV_K_BLOCK_MANY, k_block_attn_many,
                      dim3((unsigned)(tiles_of(a.t, kManyTiles) * a.t.Hkv)), dim3(kManyThreads),
                      lists, s, a);
    return launch_status();
  }
  const int64_t units = tiles_of(a.t) * a.t.Hkv;
  of_kind(kind, [&](auto k) {
    launch_kernel(CKV_K_BLOCK_ATTN, k_block_attn<k.value>, dim3((unsigned)(units * a.pieces)),
                  dim3(kBlockThreads), s, a);
  });
  const hipError_t e = launch_status();
  if (e != hipSuccess || a.pieces == 1) return e;
  launch_kernel(CKV_K_BLOCK_MERGE, k_block_merge, dim3((unsigned)(4 * units)), dim3(kBlockThreads), s,
                a);
  return launch_status();
}

}  // namespace ckv
