// ckv_paged_tile.hpp -- device code that the kernels over a paged cache share: rows
// of its three kinds as matrix operands, and one wave's step of an attention.
#pragma once

#include "ckv_paged.hpp"

namespace ckv {

// ---- small helpers -------------------------------------------------------------
// bf16 bits of x, nearest, ties to even; NaN stays NaN.
__device__ __forceinline__ uint32_t bf16_bits(float x) {
  const uint32_t u = __float_as_uint(x);
  return x != x ? (u >> 16) | 0x40u : (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

__device__ __forceinline__ uint4 pack8_bf16(const float* y) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = bf16_bits(y[2 * i]) | (bf16_bits(y[2 * i + 1]) << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// x * 2^(byte - 127).
__device__ __forceinline__ float times_exp(float x, uint32_t byte) {
  return __builtin_amdgcn_ldexpf(x, (int)byte - 127);
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Two e4m3 codes (the low or the high half of w) as two bf16: exact.
template <bool HI>
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
}

// Eight codes as eight bf16.
__device__ __forceinline__ uint4 e4m3_octet(uint2 w) {
  return make_uint4(e4m3_pair<false>(w.x), e4m3_pair<true>(w.x), e4m3_pair<false>(w.y),
                    e4m3_pair<true>(w.y));
}

// Codes 2 i and 2 i + 1 of w as two bf16 times 2^(byte - 127), the byte in bits
// 30 .. 23 of `scale` (its other bits do not matter): exact while |value| < 2^128;
// byte 255 gives NaN.  All 256 bytes and all codes were compared with ldexp.
template <int I>
__device__ __forceinline__ uint32_t e2m1_pair(uint32_t w, uint32_t scale) {
  return __builtin_bit_cast(
      uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, __uint_as_float(scale), I));
}

// (i is a constant of an unrolled loop.)
__device__ __forceinline__ uint32_t e2m1_pair_at(uint32_t w, uint32_t scale, int i) {
  return i == 0   ? e2m1_pair<0>(w, scale)
         : i == 1 ? e2m1_pair<1>(w, scale)
         : i == 2 ? e2m1_pair<2>(w, scale)
                  : e2m1_pair<3>(w, scale);
}

// Eight codes as eight bf16.
__device__ __forceinline__ uint4 e2m1_octet(uint32_t w, uint32_t scale) {
  return make_uint4(e2m1_pair<0>(w, scale), e2m1_pair<1>(w, scale), e2m1_pair<2>(w, scale),
                    e2m1_pair<3>(w, scale));
}

// Byte i of w in bits 30 .. 23.
__device__ __forceinline__ uint32_t scale_of(uint32_t w, int i) {
  return __builtin_amdgcn_alignbit(w, w, 9 + 8 * i);
}

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint2 ld8_nt(const uint8_t* p) {
  const u32x2 v = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
  return make_uint2(v[0], v[1]);
}

__device__ __forceinline__ uint32_t ld4_nt(const uint8_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
}

// N bytes of a row: streamed past the caches, or (STREAM false) kept for others.
template <int N, bool STREAM>
__device__ __forceinline__ auto ld_row(const uint8_t* p) {
  if constexpr (N == 16) {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
    return STREAM ? ld16_nt(q) : ld16(q);
  } else if constexpr (N == 8) {
    return STREAM ? ld8_nt(p) : *reinterpret_cast<const uint2*>(p);
  } else {
    return STREAM ? ld4_nt(p) : *reinterpret_cast<const uint32_t*>(p);
  }
}

// What a kernel only reads, for scalar loads where the index is the wave's.
typedef const __attribute__((address_space(4))) int32_t* TablePtr;

__device__ __forceinline__ int64_t row_offset(const PagedPages& pg, int page, int h, int pos) {
  const int row = pos & ((1 << pg.shift) - 1);
  return page * pg.page_bytes + h * pg.head_bytes + (int64_t)row * pg.row_bytes;
}

__device__ __forceinline__ int64_t exp_offset(const PagedPages& pg, int page, int h, int pos) {
  return (((int64_t)page * pg.Hkv + h) << pg.shift) + (pos & ((1 << pg.shift) - 1));
}

// Codes of 16 bytes of bf16 elements, and exponent bytes a row.
__host__ __device__ constexpr int row_part(Kind k) {
  return k == Kind::kBf16 ? 16 : k == Kind::kE4M3 ? 8 : 4;
}

__host__ __device__ constexpr int exps_of(Kind k) {
  return k == Kind::kBf16 ? 0 : k == Kind::kE4M3 ? 1 : kD / kExpGroup;
}

// ---- keys and values of 16 positions ---------------------------------------------------
// Sixteen consecutive positions from a multiple of 16 on.  With pages of at
// least 16 positions (WIDE) they lie in one page, whose number is the same for
// the whole wave; else every lane looks its rows' pages up.  Rows at or past
// the context's end are read as its last row (rows there may hold anything, and
// a weight of zero times a NaN is a NaN).
__device__ __forceinline__ TablePtr table_of(const PagedPages& pg, int b) {
  return (TablePtr)(uintptr_t)(pg.table + (int64_t)b * pg.table_stride);
}

struct Ctx {
  int b, h, n;            // request, KV head, positions (> 0 where rows are read)
  TablePtr table;         // the request's
};

// Position i of a group in the order that feeds a product's K operand: lane
// (g, r) = (lane / 16, lane % 16) holds row r, in the fragments f = 0 .. 3 the
// elements frag_base(f) + 0 .. 7, 16 bytes a load.  Any order of the 128
// products will do as long as the queries' fragments have the same.
template <Kind KIND>
__device__ __forceinline__ int frag_base(int f, int g) {
  return KIND == Kind::kE4M3   ? 64 * (f >> 1) + 16 * g + 8 * (f & 1)
         : KIND == Kind::kE2M1 ? kExpGroup * g + 8 * f
                               : 32 * f + 8 * g;
}

template <Kind KIND>
struct KRaw {
  static constexpr int kN = row_part(KIND) / 4;  // 16-byte loads
  uint4 w[kN];
  uint32_t e;  // e2m1: the exponent byte of the lane's 32 elements
  __device__ __forceinline__ void load(const uint8_t* row, int g) {
#pragma unroll
    for (int i = 0; i < kN; ++i)
      w[i] = *reinterpret_cast<const uint4*>(row + 64 * i + 16 * g);
  }
  // The same from whole 128-byte lines, streamed past the caches (rows of one
  // page from `base`; read in halves, a line is fetched for the first and has to
  // stay for the second): each load takes both halves of a line of eight rows, the
  // second half through the lanes of r >= 8; lanes r and r ^ 8 then swap what
  // belongs to the other's row.
  template <bool STREAM>
  __device__ __forceinline__ void load_lines(const uint8_t* base, int32_t row_bytes, int32_t cap,
                                             int g, int r) {
    if constexpr (KIND == Kind::kE2M1) {  // rows of 64 bytes: 16 of them a load
      w[0] = ld_row<16, STREAM>(base + (uint32_t)min(r * row_bytes, cap) + 16 * g);
      return;
    }
    const uint8_t* p = base + 8 * (r & 8) + 16 * g;
    const uint32_t at[2] = {(uint32_t)min((r & 7) * row_bytes, cap),
                            (uint32_t)min(((r & 7) + 8) * row_bytes, cap)};
#pragma unroll
    for (int i = 0; i < kN; ++i)
      w[i] = ld_row<16, STREAM>(p + at[i & 1] + 128 * (i >> 1));
  }
  __device__ __forceinline__ void swap_halves(int r) {
    const bool lo = r < 8;
#pragma unroll
    for (int l = 0; l + 1 < kN; l += 2) {
      uint32_t a[4] = {w[l].x, w[l].y, w[l].z, w[l].w};
      uint32_t b[4] = {w[l + 1].x, w[l + 1].y, w[l + 1].z, w[l + 1].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t y = dpp_u32<0x128, 0xF, false>(lo ? b[i] : a[i]);  // row_ror:8
        if (lo) b[i] = y;
        else a[i] = y;
      }
      w[l] = make_uint4(a[0], a[1], a[2], a[3]);
      w[l + 1] = make_uint4(b[0], b[1], b[2], b[3]);
    }
  }
  __device__ __forceinline__ bf16x8 frag(int f) const {
    if constexpr (KIND == Kind::kBf16) return as_bf16x8(w[f]);
    if constexpr (KIND == Kind::kE2M1) {
      const uint32_t c = f & 2 ? (f & 1 ? w[0].w : w[0].z) : (f & 1 ? w[0].y : w[0].x);
      return as_bf16x8(e2m1_octet(c, e << 23));
    }
    const uint4 q = w[f >> 1];
    return as_bf16x8(e4m3_octet(f & 1 ? make_uint2(q.z, q.w) : make_uint2(q.x, q.y)));
  }
};

// ---- a wave's step of an attention ----------------------------------------------------
// One wave's state over the positions it has seen of a unit: lane (g, r) has
// query row r's running maximum m (of logits times log2 e, the same in every
// g), its own positions' sum of weights l, and the weighted V sums
// o[e][j] = O[row r][8 (4g + j) + e].
struct WaveState {
  float m, l;
  f32x4 o[8];
};

// A wave's step: 32 positions from p0 on.
//   logits   S^T = K Q^T: positions in the rows, so lane (g, r) gets query row
//            r at positions 4g + 0 .. 3 of each half
//   weights  exp2 of logits less the running maximum, fp32; split exactly
//            into three bf16 parts (8 + 8 + 8 bits, each the truncation of
//            what the ones before leave), so that the products with V's bf16
//            are exact too and only the fp32 accumulation rounds
//   output   O^T += V^T P^T, 32 positions a product in the order that the
//            weights already have: operand entry (g, j) is position 4g + j of
//            the first half (j < 4) or 4g + j - 4 of the second, and lane (g,
//            r) reads channels [8r, 8r + 8) of those eight rows, 16 bytes a
//            row, and picks its operands out of them by byte permutes
// K of the next step is asked for once this step's logits have taken theirs,
// V once the products have taken its rows: a wave always has one of them in
// flight, and none needs a second set of registers.  Both are streamed past the
// caches by loads of whole lines (4.4 GB of a bf16 batch 745 -> 667 us).
template <Kind KIND>
struct Tile {
  KRaw<KIND> k[2];
  static constexpr int kV = row_part(KIND) / 4;
  uint32_t v[8][kV];                // row j: bf16, or codes
  // exponent bytes: e4m3 of each half's four positions; e2m1 of row j's four groups
  uint32_t ke[KIND == Kind::kE4M3 ? 2 : 1];
  uint32_t ve[KIND == Kind::kE4M3 ? 2 : KIND == Kind::kE2M1 ? 8 : 1];
  uint32_t there;                   // bit j: position j of the lane's rows has a page
};

// Where a step's two halves lie, looked up a step ahead (a lookup between row
// loads would wait for those before it).  Rows past the context's end are read as
// its last row.  With WIDE pages a half's page is the same for every lane, and a
// row's offset from the half's first is the smaller of its own and the last
// row's (cap); else every row has its page.  Pages that are not there are -1.
template <bool WIDE>
struct TileAt {
  int first[2];
  int page[2];      // WIDE: of the halves; else of the lane's K rows
  int v_page[WIDE ? 1 : 8];
  int32_t cap[2];   // WIDE: bytes
};

__device__ __forceinline__ int page_at(const PagedPages& pg, const Ctx& x, int pos) {
  const int page = x.table[pos >> pg.shift];
  return (unsigned)page < (unsigned)pg.num_pages ? page : -1;
}

template <bool WIDE>
__device__ __forceinline__ TileAt<WIDE> tile_at(const PagedPages& pg, const Ctx& x, int p0) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  TileAt<WIDE> t;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    t.first[i] = half_first(p0, i, x.n);
    if (WIDE) {
      t.page[i] = page_at(pg, x, t.first[i]);
      t.cap[i] = half_last(t.first[i], x.n) * pg.row_bytes;
    } else {
      t.page[i] = page_at(pg, x, min(t.first[i] + r, x.n - 1));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        t.v_page[WIDE ? 0 : 4 * i + j] =
            page_at(pg, x, min(t.first[i] + 4 * g + j, x.n - 1));
    }
  }
  return t;
}

// First byte of a half's first row, for the whole wave.
__device__ __forceinline__ int64_t half_base(const PagedPages& pg, const Ctx& x,
                                             const TileAt<true>& at, int i) {
  return row_offset(pg, max(at.page[i], 0), x.h, at.first[i]);
}

template <Kind KIND, bool WIDE, bool STREAM = true>
__device__ __forceinline__ void load_k(const PagedPages& pg, const Ctx& x, const TileAt<WIDE>& at,
                                       Tile<KIND>& t) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int page = max(at.page[i], 0), row = min(at.first[i] + r, x.n - 1);
    if constexpr (WIDE)
      t.k[i].template load_lines<STREAM>(pg.k + half_base(pg, x, at, i), pg.row_bytes, at.cap[i], g, r);
    else
      t.k[i].load(pg.k + row_offset(pg, page, x.h, row), g);
    if (KIND == Kind::kE2M1) t.k[i].e = pg.k_exps[4 * exp_offset(pg, page, x.h, row) + g];
  }
}

template <Kind KIND, bool WIDE, bool STREAM = true>
__device__ __forceinline__ void load_v(const PagedPages& pg, const Ctx& x, const TileAt<WIDE>& at,
                                       Tile<KIND>& t) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  t.there = 0;
  if constexpr (WIDE) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (at.page[i] >= 0) t.there |= 15u << (4 * i);
      if (KIND == Kind::kE2M1) {  // four positions' words at once
        const uint4 e = *reinterpret_cast<const uint4*>(
            pg.v_exps + 4 * (exp_offset(pg, max(at.page[i], 0), x.h, at.first[i]) + 4 * g));
        t.ve[4 * i] = e.x, t.ve[4 * i + 1] = e.y, t.ve[4 * i + 2] = e.z, t.ve[4 * i + 3] = e.w;
      }
      if (KIND == Kind::kE4M3) {  // four positions' bytes at once: rows of one page, a multiple of 4
        const int64_t e = exp_offset(pg, max(at.page[i], 0), x.h, at.first[i]);
        t.ke[i] = *reinterpret_cast<const uint32_t*>(pg.k_exps + e + 4 * g);
        t.ve[i] = *reinterpret_cast<const uint32_t*>(pg.v_exps + e + 4 * g);
      }
    }
  } else {
    uint32_t ke[8], ve[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (at.v_page[j] >= 0) t.there |= 1u << j;
      if (KIND != Kind::kBf16) {
        const int pos = min(at.first[j >> 2] + 4 * g + (j & 3), x.n - 1);
        const int64_t e = exp_offset(pg, max(at.v_page[j], 0), x.h, pos);
        if (KIND == Kind::kE2M1) {
          t.ve[j] = reinterpret_cast<const uint32_t*>(pg.v_exps)[e];
        } else {
          ke[j] = pg.k_exps[e];
          ve[j] = pg.v_exps[e];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (KIND == Kind::kE4M3) {
        t.ke[i] = ke[4 * i] | ke[4 * i + 1] << 8 | ke[4 * i + 2] << 16 | ke[4 * i + 3] << 24;
        t.ve[i] = ve[4 * i] | ve[4 * i + 1] << 8 | ve[4 * i + 2] << 16 | ve[4 * i + 3] << 24;
      }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint8_t* p;
    const int i = j >> 2, row = 4 * g + (j & 3);
    if constexpr (WIDE)
      p = pg.v + half_base(pg, x, at, i) + (uint32_t)min(row * pg.row_bytes, at.cap[i]);
    else
      p = pg.v + row_offset(pg, max(at.v_page[j], 0), x.h, min(at.first[i] + row, x.n - 1));
    uint32_t* v = t.v[j];
    if constexpr (KIND == Kind::kE2M1) {
      v[0] = ld_row<4, STREAM>(p + 4 * r);
    } else if constexpr (KIND == Kind::kE4M3) {
      const uint2 w = ld_row<8, STREAM>(p + 8 * r);
      v[0] = w.x, v[1] = w.y;
    } else {
      const uint4 w = ld_row<16, STREAM>(p + 16 * r);
      v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w;
    }
  }
}

// x * 2^(byte j of w - 128), bytes already taken as signed (w ^ 0x80808080).
__device__ __forceinline__ float scaled(float x, uint32_t w, int j) {
  return __builtin_amdgcn_ldexpf(x, (int)(w << (24 - 8 * j)) >> 24);
}

// Logits of a step for query row r: lg[j] at position p0 + 16 (j / 4) + 4g +
// j % 4, before the scale.
template <Kind KIND, bool WIDE>
__device__ __forceinline__ void tile_logits(Tile<KIND>& t, const bf16x8* q, float* lg) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (WIDE) t.k[i].swap_halves(threadIdx.x & 15);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int f = 0; f < 4; ++f) s = mfma_16x16x32(t.k[i].frag(f), q[f], s);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      lg[4 * i + j] = s[j];
  }
}

// Positions that the query row does not see, or that are not there: logits of
// -inf, V rows of zeros (what was read in their place may be anything).
template <Kind KIND>
__device__ __forceinline__ void tile_mask(Tile<KIND>& t, int p0, int limit, int n, float* lg) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool has = t.there >> j & 1u;
    const int pos = p0 + 16 * (j >> 2) + 4 * g + (j & 3);
    if (!has || pos >= limit) lg[j] = -INFINITY;
#pragma unroll
    for (int i = 0; i < Tile<KIND>::kV; ++i)
      if (!has) t.v[j][i] = 0u;
    // NaN's byte would make zeros NaN, and the words of four positions may be past
    // the context's end
    if (KIND == Kind::kE2M1 && (!has || pos >= n)) t.ve[j] = 0u;
  }
}

// Max over the lanes of a query row, r, r + 16, r + 32, r + 48: rows of lanes
// change places, and then halves (no LDS round trip in the steps' chain).
__device__ __forceinline__ float query_row_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const uint32_t v = __float_as_uint(x);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Logits up to `top` (of this lane) are about to be taken: the running maximum
// follows, and what was summed under the old one is scaled.
__device__ __forceinline__ void raise_max(float top, float c, WaveState& st) {
  top = query_row_max(top);
  const float m = fmaxf(st.m, top * c);
  if (__any(m > st.m)) {
    const float f = st.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.m - m);
    st.l *= f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int j = 0; j < 4; ++j) st.o[e][j] *= f;
    st.m = m;
  }
}

__device__ __forceinline__ float top_of(const float* lg) {
  float top = lg[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) top = fmaxf(top, lg[j]);
  return top;
}

// What logits times c are made less by: the running maximum; nothing seen yet: all
// weights are 0.
__device__ __forceinline__ float less_max(const WaveState& st) {
  return st.m == -INFINITY ? 0.f : -st.m;
}

// ve: e4m3's exponent bytes of the lane's positions of each half.
template <Kind KIND>
__device__ __forceinline__ void tile_weights(const uint32_t* ve, float c, float less,
                                             const float* lg, uint32_t part[3][8],
                                             WaveState& st) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float p = __builtin_amdgcn_exp2f(fmaf(lg[j], c, less));
    st.l += p;
    if (KIND == Kind::kE4M3) p = scaled(p, ve[j >> 2] ^ 0x80808080u, j & 3);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      part[i][j] = __float_as_uint(p);
      p -= __uint_as_float(part[i][j] & 0xffff0000u);
    }
  }
}

// The weights' parts as operands.
__device__ __forceinline__ void pack_weights(const uint32_t part[3][8], bf16x8* w) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    uint32_t y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      y[j] = __builtin_amdgcn_perm(part[i][2 * j + 1], part[i][2 * j], 0x07060302u);
    w[i] = as_bf16x8(make_uint4(y[0], y[1], y[2], y[3]));
  }
}

template <Kind KIND>
__device__ __forceinline__ void tile_output(const Tile<KIND>& t, const uint32_t part[3][8],
                                            WaveState& st) {
  bf16x8 w[3];
  uint32_t scale[8];
#pragma unroll
  for (int j = 0; j < 8; ++j)
    scale[j] = KIND == Kind::kE2M1 ? scale_of(t.ve[j], (threadIdx.x & 15) >> 2) : 0u;
  pack_weights(part, w);
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    uint32_t even[4], odd[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t lo, hi;  // channels e, e + 1 of two rows
      if constexpr (KIND == Kind::kE2M1) {
        lo = e2m1_pair_at(t.v[2 * j][0], scale[2 * j], e >> 1);
        hi = e2m1_pair_at(t.v[2 * j + 1][0], scale[2 * j + 1], e >> 1);
      } else if constexpr (KIND == Kind::kE4M3) {
        lo = e & 2 ? e4m3_pair<true>(t.v[2 * j][e >> 2]) : e4m3_pair<false>(t.v[2 * j][e >> 2]);
        hi = e & 2 ? e4m3_pair<true>(t.v[2 * j + 1][e >> 2])
                   : e4m3_pair<false>(t.v[2 * j + 1][e >> 2]);
      } else {
        lo = t.v[2 * j][e >> 1];
        hi = t.v[2 * j + 1][e >> 1];
      }
      even[j] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
      odd[j] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
    }
    const bf16x8 a = as_bf16x8(make_uint4(even[0], even[1], even[2], even[3]));
    const bf16x8 b = as_bf16x8(make_uint4(odd[0], odd[1], odd[2], odd[3]));
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      st.o[e] = mfma_16x16x32(a, w[i], st.o[e]);
      st.o[e + 1] = mfma_16x16x32(b, w[i], st.o[e + 1]);
    }
  }
}

template <Kind KIND>
__device__ __forceinline__ void tile_rest(Tile<KIND>& t, bool masked, int p, int limit, int n,
                                          float c, float* lg, WaveState& st) {
  if (KIND == Kind::kE4M3) {
#pragma unroll
    for (int j = 0; j < 8; ++j) lg[j] = scaled(lg[j], t.ke[j >> 2] ^ 0x80808080u, j & 3);
  }
  if (masked) tile_mask<KIND>(t, p, limit, n, lg);
  raise_max(top_of(lg), c, st);
  uint32_t part[3][8];
  tile_weights<KIND>(t.ve, c, less_max(st), lg, part, st);
  tile_output<KIND>(t, part, st);
}

// A query row's result from its sums.
__device__ __forceinline__ float inverse_sum(float L) {
  return L > 0.f ? 1.f / L : L;  // nothing seen: 0; NaN stays
}

__device__ __forceinline__ float log_sum(float M, float L) {
  return L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.6931471805599453f;
}

// The four waves' sums for query row `row`, channels [d, d + 4).
struct Partial {
  float M, L;
  float4 o;
};

template <class Lds>  // m, l [4][16], o [4][16][kPartStride]
__device__ __forceinline__ Partial join_waves(const Lds& lds, int row, int d) {
  Partial p;
  p.M = -INFINITY;
#pragma unroll
  for (int k = 0; k < 4; ++k) p.M = fmaxf(p.M, lds.m[k][row]);
  p.L = 0.f;
  p.o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float m = lds.m[k][row];
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - p.M);
    const float4 o = *reinterpret_cast<const float4*>(&lds.o[k][row][d]);
    p.L = fmaf(f, lds.l[k][row], p.L);
    p.o.x = fmaf(f, o.x, p.o.x);
    p.o.y = fmaf(f, o.y, p.o.y);
    p.o.z = fmaf(f, o.z, p.o.z);
    p.o.w = fmaf(f, o.w, p.o.w);
  }
  return p;
}

// fn with the kind as a constant.
template <class Fn>
static void of_kind(Kind kind, Fn fn) {
  if (kind == Kind::kBf16) fn(std::integral_constant<Kind, Kind::kBf16>{});
  else if (kind == Kind::kE4M3) fn(std::integral_constant<Kind, Kind::kE4M3>{});
  else fn(std::integral_constant<Kind, Kind::kE2M1>{});
}

}  // namespace ckv
