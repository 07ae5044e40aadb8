// ckv_paged.hip -- gfx950 kernels of the rotary positions and the paged cache,
// and their host-side launchers.
#include "ckv_paged_tile.hpp"
#include "ckv_profile.hpp"

namespace ckv {

// ---- rotary positions ------------------------------------------------------------
// (cos, sin) of pos * inv_freq.  The angle is formed in quarter turns in fp64
// (an fp32 angle of 2^20 radians is off by up to 1/16), its whole quarters are
// taken off there, and what is left, |x| <= pi/4, goes through the Taylor series
// of sine (to x^9, remainder below 1.8e-9) and cosine (to x^10, below 1.2e-10) in
// fp32.
__device__ __forceinline__ float2 cos_sin(double quarters) {
  const double whole = rint(quarters);
  const float x = (float)(quarters - whole) * 1.5707963267948966f;
  const int n = (int)(whole - 4.0 * floor(whole * 0.25));  // 0 .. 3
  const float x2 = x * x;
  float s = fmaf(x2, 2.7557319e-6f, -1.9841270e-4f);
  s = fmaf(x2, s, 8.3333333e-3f);
  s = fmaf(x2, s, -1.6666667e-1f);
  s = fmaf(x * x2, s, x);
  float c = fmaf(x2, -2.7557319e-7f, 2.4801587e-5f);
  c = fmaf(x2, c, -1.3888889e-3f);
  c = fmaf(x2, c, 4.1666667e-2f);
  c = fmaf(x2, c, -0.5f);
  c = fmaf(x2, c, 1.0f);
  const float a = n & 1 ? s : c, b = n & 1 ? c : s;
  return make_float2(n == 1 || n == 2 ? -a : a, n >= 2 ? -b : b);
}

// The same in fp64 throughout (sine to x^17, remainder below 1e-19; cosine to x^18), for
// keys that are made four bits: a code is decided at the middle between two, where the
// fp32 form's error makes some codes of a prefill their neighbours (steps of up to half
// the value).  22 k tokens written and read back 128 -> 135 us.
__device__ __forceinline__ double2 cos_sin64(double quarters) {
  const double whole = rint(quarters);
  const double x = (quarters - whole) * 1.57079632679489661923;
  const int n = (int)(whole - 4.0 * floor(whole * 0.25));  // 0 .. 3
  const double x2 = x * x;
  double s = 1.0 / 355687428096000.0, c = -1.0 / 6402373705728000.0;  // 17!, 18!
  s = fma(x2, s, -1.0 / 1307674368000.0);
  s = fma(x2, s, 1.0 / 6227020800.0);
  s = fma(x2, s, -1.0 / 39916800.0);
  s = fma(x2, s, 1.0 / 362880.0);
  s = fma(x2, s, -1.0 / 5040.0);
  s = fma(x2, s, 1.0 / 120.0);
  s = fma(x2, s, -1.0 / 6.0);
  s = fma(x * x2, s, x);
  c = fma(x2, c, 1.0 / 20922789888000.0);
  c = fma(x2, c, -1.0 / 87178291200.0);
  c = fma(x2, c, 1.0 / 479001600.0);
  c = fma(x2, c, -1.0 / 3628800.0);
  c = fma(x2, c, 1.0 / 40320.0);
  c = fma(x2, c, -1.0 / 720.0);
  c = fma(x2, c, 1.0 / 24.0);
  c = fma(x2, c, -0.5);
  c = fma(x2, c, 1.0);
  const double a = n & 1 ? s : c, b = n & 1 ? c : s;
  return make_double2(n == 1 || n == 2 ? -a : a, n >= 2 ? -b : b);
}

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 4;       // tokens of a workgroup in a long call
constexpr int kRopeMaxPairs = 512;

// The workgroup's cosines and sines, scale (and direction) included: tab[t *
// pairs + i] for its `tokens` tokens from t0 on.
__device__ __forceinline__ void rope_table(const RopeSpec& r, const int32_t* pos, int t0,
                                           int tokens, float2* tab) {
  const int pairs = r.rot >> 1;
  for (int e = threadIdx.x; e < tokens * pairs; e += kRopeThreads) {
    const int t = e / pairs, i = e - t * pairs;
    // 2 / pi: quarter turns of a radian
    const double q = (double)pos[t0 + t] * (r.inv_freq[i] * 0.63661977236758134308);
    float2 cs = cos_sin(q);
    cs.x *= r.scale;
    cs.y *= r.inverse ? -r.scale : r.scale;
    tab[e] = cs;
  }
}

// The same from fp64 values, which are left in exact[] too.
__device__ __forceinline__ void rope_table64(const RopeSpec& r, const int32_t* pos, int t0,
                                             int tokens, float2* tab, double2* exact) {
  const int pairs = r.rot >> 1;
  for (int e = threadIdx.x; e < tokens * pairs; e += kRopeThreads) {
    const int t = e / pairs, i = e - t * pairs;
    double2 cs = cos_sin64((double)pos[t0 + t] * (r.inv_freq[i] * 0.63661977236758134308));
    cs.x *= r.scale;
    cs.y *= r.inverse ? -r.scale : r.scale;
    exact[e] = cs;
    tab[e] = make_float2((float)cs.x, (float)cs.y);
  }
}

template <typename T>
struct RopeVec;  // 16 bytes of a row
template <>
struct RopeVec<uint16_t> {
  using Bits = uint16_t;
  static constexpr int kN = 8;
  static __device__ __forceinline__ void open(u32x4 v, float* x) {
    unpack8(make_uint4(v[0], v[1], v[2], v[3]), x);
  }
  static __device__ __forceinline__ u32x4 close(const float* y) {
    const uint4 v = pack8_bf16(y);
    return u32x4{v.x, v.y, v.z, v.w};
  }
  static __device__ __forceinline__ float one(const uint16_t* p) {
    return __uint_as_float((uint32_t)*p << 16);
  }
  static __device__ __forceinline__ void put(uint16_t* p, float y) { *p = (uint16_t)bf16_bits(y); }
};
template <>
struct RopeVec<float> {
  using Bits = uint32_t;
  static constexpr int kN = 4;
  static __device__ __forceinline__ void open(u32x4 v, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
  }
  static __device__ __forceinline__ u32x4 close(const float* y) {
    return u32x4{__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]),
                 __float_as_uint(y[3])};
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
  static __device__ __forceinline__ void put(float* p, float y) { *p = y; }
};

// A row's work in items that each own what they read, so that a row may be
// rotated in place.  Where vectors of 16 bytes hold whole pairs or whole runs of
// first elements (rot_dim a multiple of 16 bytes, of 32 for HALF) an item is a
// vector of first elements with the vector of their partners, a vector of
// neighbouring pairs, or (not in place) a vector past rot_dim; else an item is
// one pair.  A thread asks for the rows of kRopeBatch items before it turns the
// first.
constexpr int kRopeBatch = 4;

template <typename T>
__host__ __device__ __forceinline__ bool rope_whole(int rot, int layout) {
  const int n = sizeof(T) == 2 ? 8 : 4;
  return rot % (layout == CKV_ROPE_HALF ? 2 * n : n) == 0;
}

// Rotates `tokens` tokens' rows from token t0 on, in vectors, and copies the
// rest of them; tab as rope_table leaves it.
template <typename T, bool HALF>
__device__ __forceinline__ void rope_vectors(const RopeSpec& r, const RopeRows& rows, int t0,
                                             int tokens, const float2* tab) {
  using V = RopeVec<T>;
  constexpr int N = V::kN;
  const int pairs = r.rot >> 1, turn = (HALF ? pairs : r.rot) / N;
  const int per_row = turn + (rows.src == rows.dst ? 0 : (r.head_dim - r.rot) / N);
  const int n = tokens * rows.heads * per_row;
  for (int e0 = threadIdx.x; e0 < n; e0 += kRopeBatch * kRopeThreads) {
    u32x4 v1[kRopeBatch], v2[kRopeBatch];
    T* dst[kRopeBatch];
    int pair[kRopeBatch];  // the item's first one in the table; -1: copied
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      const int e = min(e0 + i * kRopeThreads, n - 1);  // past the end: loaded, not stored
      const int row = e / per_row, item = e - row * per_row;
      const int t = row / rows.heads, head = row - t * rows.heads;
      const bool turned = item < turn;
      const int first = turned ? N * item : r.rot + N * (item - turn);
      const T* src = static_cast<const T*>(rows.src) + (int64_t)(t0 + t) * rows.src_tok +
                     head * rows.src_head + first;
      dst[i] = static_cast<T*>(rows.dst) + (int64_t)(t0 + t) * rows.dst_tok +
               head * rows.dst_head + first;
      pair[i] = turned ? t * pairs + (HALF ? N : N / 2) * item : -1;
      v1[i] = *reinterpret_cast<const u32x4*>(src);
      if (HALF) v2[i] = *reinterpret_cast<const u32x4*>(src + (turned ? pairs : 0));
    }
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      if (e0 + i * kRopeThreads >= n) break;
      if (pair[i] < 0) {
        *reinterpret_cast<u32x4*>(dst[i]) = v1[i];
        continue;
      }
      const float2* c = tab + pair[i];
      float x1[N], y1[N];
      V::open(v1[i], x1);
      if constexpr (HALF) {
        float x2[N], y2[N];
        V::open(v2[i], x2);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          y1[j] = x1[j] * c[j].x - x2[j] * c[j].y;
          y2[j] = x2[j] * c[j].x + x1[j] * c[j].y;
        }
        *reinterpret_cast<u32x4*>(dst[i] + pairs) = V::close(y2);
      } else {
#pragma unroll
        for (int j = 0; j < N; j += 2) {
          y1[j] = x1[j] * c[j / 2].x - x1[j + 1] * c[j / 2].y;
          y1[j + 1] = x1[j + 1] * c[j / 2].x + x1[j] * c[j / 2].y;
        }
      }
      *reinterpret_cast<u32x4*>(dst[i]) = V::close(y1);
    }
  }
}

// The same pair by pair: 16384 tokens of 40 bf16 rows with 20 of 128 elements
// turned 113 us, where vectors (96 of 128) take 71.
template <typename T, bool HALF>
__device__ __forceinline__ void rope_pairs(const RopeSpec& r, const RopeRows& rows, int t0,
                                           int tokens, const float2* tab) {
  using V = RopeVec<T>;
  const int pairs = r.rot >> 1, n = tokens * rows.heads * pairs;
  for (int e0 = threadIdx.x; e0 < n; e0 += kRopeBatch * kRopeThreads) {
    float x1[kRopeBatch], x2[kRopeBatch];
    T* dst[kRopeBatch];
    int pair[kRopeBatch];
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      const int e = min(e0 + i * kRopeThreads, n - 1);
      const int row = e / pairs, item = e - row * pairs, first = HALF ? item : 2 * item;
      const int t = row / rows.heads, head = row - t * rows.heads;
      const T* src = static_cast<const T*>(rows.src) + (int64_t)(t0 + t) * rows.src_tok +
                     head * rows.src_head + first;
      dst[i] = static_cast<T*>(rows.dst) + (int64_t)(t0 + t) * rows.dst_tok +
               head * rows.dst_head + first;
      pair[i] = t * pairs + item;
      x1[i] = V::one(src);
      x2[i] = V::one(src + (HALF ? pairs : 1));
    }
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      if (e0 + i * kRopeThreads >= n) break;
      const float2 c = tab[pair[i]];
      V::put(dst[i], x1[i] * c.x - x2[i] * c.y);
      V::put(dst[i] + (HALF ? pairs : 1), x2[i] * c.x + x1[i] * c.y);
    }
  }
}

// Copies elements [from, to) of every row, in vectors (both multiples of them)
// or one by one.
template <typename T, bool VECTORS>
__device__ __forceinline__ void copy_part(const RopeRows& rows, int t0, int tokens, int from,
                                          int to) {
  constexpr int N = VECTORS ? RopeVec<T>::kN : 1;
  const int per_row = (to - from) / N, n = tokens * rows.heads * per_row;
  for (int e0 = threadIdx.x; e0 < n; e0 += kRopeBatch * kRopeThreads) {
    u32x4 x[kRopeBatch];
    T* dst[kRopeBatch];
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      const int e = min(e0 + i * kRopeThreads, n - 1);
      const int row = e / per_row, at = from + N * (e - row * per_row);
      const int t = row / rows.heads, head = row - t * rows.heads;
      const T* src = static_cast<const T*>(rows.src) + (int64_t)(t0 + t) * rows.src_tok +
                     head * rows.src_head + at;
      dst[i] = static_cast<T*>(rows.dst) + (int64_t)(t0 + t) * rows.dst_tok +
               head * rows.dst_head + at;
      if constexpr (VECTORS) x[i] = *reinterpret_cast<const u32x4*>(src);
      else x[i][0] = __builtin_bit_cast(typename RopeVec<T>::Bits, *src);
    }
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      if (e0 + i * kRopeThreads >= n) break;
      if constexpr (VECTORS) *reinterpret_cast<u32x4*>(dst[i]) = x[i];
      else *dst[i] = __builtin_bit_cast(T, (typename RopeVec<T>::Bits)x[i][0]);
    }
  }
}

template <typename T, bool HALF, bool WHOLE>
__device__ __forceinline__ void rope_rows(const RopeSpec& r, const RopeRows& rows, int t0,
                                          int tokens, const float2* tab) {
  if constexpr (WHOLE) {
    rope_vectors<T, HALF>(r, rows, t0, tokens, tab);
  } else {
    rope_pairs<T, HALF>(r, rows, t0, tokens, tab);
    if (rows.src == rows.dst) return;
    constexpr int N = RopeVec<T>::kN;
    const int whole = (r.rot + N - 1) / N * N;  // the next vector
    if (whole > r.rot) copy_part<T, false>(rows, t0, tokens, r.rot, whole);
    if (whole < r.head_dim) copy_part<T, true>(rows, t0, tokens, whole, r.head_dim);
  }
}

// Rows in, rows out: the memory bounds it.  16384 tokens of 40 bf16 rows (336 MB
// in and out) 65 us, 5.2 TB/s; 16 tokens 4.7 us, a launch's latency.  A workgroup
// works its tokens' cosines out once, into LDS, and every head takes them there.
template <typename T, bool HALF, bool WHOLE>
__global__ __launch_bounds__(kRopeThreads) void k_rope(RopeArgs a, int per) {
  __shared__ float2 tab[kRopeTokens * kRopeMaxPairs];
  const int t0 = blockIdx.x * per;
  const int tokens = min(per, a.tokens - t0);
  rope_table(a.r, a.pos, t0, tokens, tab);
  __syncthreads();
  rope_rows<T, HALF, WHOLE>(a.r, a.q, t0, tokens, tab);
  if (a.k.heads) rope_rows<T, HALF, WHOLE>(a.r, a.k, t0, tokens, tab);
}

// ---- writing -----------------------------------------------------------------------
// How a written row is turned: not at all; halves or neighbouring pairs in
// whole vectors; one by one.
enum class Turn { kNone, kHalf, kPairs, kEach };

// The vector of a row that holds the partners of its elements [8c, 8c + 8)
// (kHalf).
__device__ __forceinline__ int partner(const RopeSpec& r, int c) {
  const int half = r.rot >> 4;  // vectors
  return c < half ? c + half : c < 2 * half ? c - half : c;
}

// Elements [8c, 8c + 8) of a K row, x with partners o, turned by its position.
template <Turn TURN>
__device__ __forceinline__ void turn8(const RopeSpec& r, const uint16_t* row, int c,
                                      const float2* cs, u32x4 xv, u32x4 ov, float* y) {
  float x[8], o[8];
  unpack8(make_uint4(xv[0], xv[1], xv[2], xv[3]), x);
  unpack8(make_uint4(ov[0], ov[1], ov[2], ov[3]), o);
  const int half = r.rot >> 1;
  if (TURN != Turn::kEach && 8 * c >= r.rot) {
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = x[j];
  } else if (TURN == Turn::kHalf) {
    const bool first = 8 * c < half;
    const float2* k = cs + (first ? 8 * c : 8 * c - half);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = x[j] * k[j].x + (first ? -o[j] : o[j]) * k[j].y;
  } else if (TURN == Turn::kPairs) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float2 k = cs[(8 * c + j) >> 1];
      y[j] = x[j] * k.x - x[j + 1] * k.y;
      y[j + 1] = x[j + 1] * k.x + x[j] * k.y;
    }
  } else {
    for (int j = 0; j < 8; ++j) {
      const int e = 8 * c + j;
      y[j] = x[j];
      if (e >= r.rot) continue;
      const bool halves = r.layout == CKV_ROPE_HALF, first = halves ? e < half : (e & 1) == 0;
      const int other = halves ? (first ? e + half : e - half) : e ^ 1;
      const float2 k = cs[halves ? (first ? e : other) : e >> 1];
      const float p = RopeVec<uint16_t>::one(row + other);
      y[j] = x[j] * k.x + (first ? -p : p) * k.y;
    }
  }
}

// x as fp32 so that a rounding to fewer bits gives what it would give for x: where it
// is not exact, the neighbour with an odd last bit, which is no value of theirs and no
// middle between two.
__device__ __forceinline__ float to_odd(double x) {
  const float f = (float)x;
  const double less = x - (double)f;  // NaN: none, as for infinities
  const uint32_t u = __float_as_uint(f);
  if (!(less != 0.0) || less != less || (u & 1u)) return f;
  if (f == 0.f) return __uint_as_float(less > 0.0 ? 1u : 0x80000001u);
  return __uint_as_float((less > 0.0) == (f > 0.f) ? u + 1 : u - 1);
}

// turn8 in fp64, for rows of four bits.
template <Turn TURN>
__device__ __forceinline__ void turn8_64(const RopeSpec& r, const uint16_t* row, int c,
                                         const double2* cs, u32x4 xv, u32x4 ov, float* y) {
  float x[8], o[8];
  unpack8(make_uint4(xv[0], xv[1], xv[2], xv[3]), x);
  unpack8(make_uint4(ov[0], ov[1], ov[2], ov[3]), o);
  const int half = r.rot >> 1;
  if (TURN != Turn::kEach && 8 * c >= r.rot) {
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = x[j];
    return;
  }
  for (int j = 0; j < 8; ++j) {
    const int e = 8 * c + j;
    const bool halves = TURN == Turn::kHalf || (TURN == Turn::kEach && r.layout == CKV_ROPE_HALF);
    const bool first = halves ? e < half : (e & 1) == 0;
    const int other = halves ? (first ? e + half : e - half) : e ^ 1;
    if (TURN == Turn::kEach && e >= r.rot) {
      y[j] = x[j];
      continue;
    }
    const double2 k = cs[halves ? (first ? e : other) : e >> 1];
    const float p = TURN == Turn::kHalf    ? o[j]
                    : TURN == Turn::kPairs ? x[j ^ 1]
                                           : RopeVec<uint16_t>::one(row + other);
    y[j] = to_odd(fma((double)(first ? -p : p), k.y, (double)x[j] * k.x));
  }
}

// Sixteen lanes write a row: lane c its elements [8c, 8c + 8).
template <Kind KIND>
__device__ __forceinline__ void store_row(uint8_t* row, uint8_t* exp, int c, const float* y) {
  if (KIND == Kind::kBf16) {
    *reinterpret_cast<uint4*>(row + 16 * c) = pack8_bf16(y);
    return;
  }
  if (KIND == Kind::kE2M1) {
    // four lanes hold a group; as bits, magnitudes rank as their values do, and an
    // infinity or NaN above all of them
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(y[j]) & 0x7fffffffu);
    most = max(most, dpp_u32<0xB1, 0xF, false>(most));  // quad_perm [1,0,3,2]
    most = max(most, dpp_u32<0x4E, 0xF, false>(most));  // [2,3,0,1]
    // 6 = 1.5 * 2^2: the byte is the leading power's field less 2, one more where
    // the largest is above 1.5 times it
    const int field = (int)(most >> 23) - 2 + ((most & 0x7fffffu) > 0x400000u ? 1 : 0);
    const uint32_t byte = min(max(field, 2), 252);  // stored values are normal bf16 numbers
    const float scale = __uint_as_float(byte << 23);
    // x / scale, nearest, ties to even, 6 at most
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
    *reinterpret_cast<uint32_t*>(row + 4 * c) = w;
    if ((c & 3) == 0) exp[c >> 2] = most >= 0x7f800000u ? 255 : (uint8_t)byte;
    return;
  }
  float most = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float m = fabsf(y[j]);
    most = fmaxf(most, m < INFINITY ? m : 0.f);
  }
  most = row16_max(most);
  // 448 = 1.75 * 2^8: the byte is the leading power's field less 8, one more
  // where the row's largest is above 1.75 times it; fields below 8 hold rows
  // under 448 * 2^-127
  const uint32_t u = __float_as_uint(most);
  const int byte = max((int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), 0);
  const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);  // 2^(127 - byte)
  float z[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) z[j] = fabsf(y[j]) < INFINITY ? y[j] * inv : NAN;
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], lo, true);
  int hi = __builtin_amdgcn_cvt_pk_fp8_f32(z[4], z[5], 0, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(z[6], z[7], hi, true);
  *reinterpret_cast<uint2*>(row + 8 * c) = make_uint2((uint32_t)lo, (uint32_t)hi);
  if (c == 0) *exp = (uint8_t)byte;
}

// A workgroup writes `per` tokens: their pages and cosines first, into LDS, then
// K and V rows, 16 lanes each, the loads of kRopeBatch rows a thread at once,
// then the queries.  Bound by the memory: 22 k tokens of 32 query rows and 8 keys
// and values each, these to e4m3 (505 MB in and out) 98 us, 5.15 TB/s; to bf16
// (550 MB) 107, 5.15.  With 20 of 128 elements turned, one by one, 169 and 174; 64
// tokens 5.4 us.
template <Kind KIND, Turn TURN>
__global__ __launch_bounds__(kRopeThreads) void k_paged_write(PagedWriteArgs a, int per) {
  __shared__ float2 tab[TURN == Turn::kNone ? 1 : kRopeTokens * (kD / 2)];
  constexpr bool kExact = KIND == Kind::kE2M1 && TURN != Turn::kNone;
  __shared__ double2 exact[kExact ? kRopeTokens * (kD / 2) : 1];
  __shared__ int64_t row_at[kRopeTokens], exp_at[kRopeTokens];  // of head 0; -1: not written
  const int t0 = blockIdx.x * per, tid = threadIdx.x;
  const int tokens = min(per, a.rope.tokens - t0);
  const RopeSpec& r = a.rope.r;
  if (tid < tokens) {
    const int pos = a.rope.pos[t0 + tid], b = a.req ? a.req[t0 + tid] : t0 + tid;
    int page = -1;
    if ((unsigned)pos < (unsigned)a.max_ctx && (unsigned)b < (unsigned)a.B)
      page = page_of(a.pg, b, pos);
    row_at[tid] = page < 0 ? -1 : row_offset(a.pg, page, 0, pos);
    exp_at[tid] = page < 0 ? -1 : exps_of(KIND) * exp_offset(a.pg, page, 0, pos);
  }
  if (kExact) rope_table64(r, a.rope.pos, t0, tokens, tab, exact);
  else if (TURN != Turn::kNone) rope_table(r, a.rope.pos, t0, tokens, tab);
  __syncthreads();
  const int Hkv = a.pg.Hkv, n = tokens * 32 * Hkv;  // (token, head, K | V, 16 lanes)
  for (int e0 = tid; e0 < n; e0 += kRopeBatch * kRopeThreads) {
    u32x4 x[kRopeBatch], o[kRopeBatch];
    const uint16_t* src[kRopeBatch];
    int head[kRopeBatch], tok[kRopeBatch];
    const int c = e0 & 15;
    const bool is_v = e0 & 16;
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      const int row = min(e0 + i * kRopeThreads, n - 1) >> 5;
      tok[i] = row / Hkv;
      head[i] = row - tok[i] * Hkv;
      src[i] = (is_v ? a.v : a.k) + (t0 + tok[i]) * a.tok + head[i] * kD;
      x[i] = *reinterpret_cast<const u32x4*>(src[i] + 8 * c);
      if (TURN == Turn::kHalf)
        o[i] = *reinterpret_cast<const u32x4*>(src[i] + 8 * partner(r, c));
      else
        o[i] = x[i];
    }
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      if (e0 + i * kRopeThreads >= n) break;
      const int64_t at = row_at[tok[i]];
      if (at < 0) continue;
      uint8_t* row = (is_v ? a.pg.v : a.pg.k) + at + head[i] * a.pg.head_bytes;
      if (KIND == Kind::kBf16 && (TURN == Turn::kNone || is_v)) {  // the bits as they are
        *reinterpret_cast<u32x4*>(row + 16 * c) = x[i];
        continue;
      }
      float y[8];
      if (TURN == Turn::kNone || is_v) unpack8(make_uint4(x[i][0], x[i][1], x[i][2], x[i][3]), y);
      else if (kExact) turn8_64<TURN>(r, src[i], c, exact + tok[i] * (r.rot >> 1), x[i], o[i], y);
      else turn8<TURN>(r, src[i], c, tab + tok[i] * (r.rot >> 1), x[i], o[i], y);
      uint8_t* exp = nullptr;
      if (KIND != Kind::kBf16)
        exp = (is_v ? a.pg.v_exps : a.pg.k_exps) + exp_at[tok[i]] +
              exps_of(KIND) * ((int64_t)head[i] << a.pg.shift);
      store_row<KIND>(row, exp, c, y);
    }
  }
  if (TURN == Turn::kNone || a.rope.q.heads == 0) return;
  if (TURN == Turn::kHalf) {
    rope_rows<uint16_t, true, true>(r, a.rope.q, t0, tokens, tab);
  } else if (TURN == Turn::kPairs) {
    rope_rows<uint16_t, false, true>(r, a.rope.q, t0, tokens, tab);
  } else if (r.layout == CKV_ROPE_HALF) {
    rope_rows<uint16_t, true, false>(r, a.rope.q, t0, tokens, tab);
  } else {
    rope_rows<uint16_t, false, false>(r, a.rope.q, t0, tokens, tab);
  }
}

// ---- reading back --------------------------------------------------------------------
// A workgroup moves kReadSlots slots of a unit: thread (s, K | V, c) the 16
// output bytes [16c, 16c + 16) of slots s, s + 8, ..., all of whose positions,
// pages and rows are asked for before the first is used: three dependent
// loads a row.  Rows are streamed past the caches.  2048 selected e4m3 rows of
// each of 128 units (203 MB in and out): 79 us with one row after the other, 49
// with eight at once, 47 streamed, 45.6 with four (4.45 TB/s; 16: 51).
constexpr int kPagedReadThreads = 256;
constexpr int kReadUnroll = kReadSlots * 32 / kPagedReadThreads;

template <Kind KIND>
__global__ __launch_bounds__(kPagedReadThreads) void k_paged_read(PagedReadArgs a) {
  const int c = threadIdx.x & 15;
  const bool is_v = threadIdx.x & 16;
  const int unit = blockIdx.x / a.chunks, first = (blockIdx.x - unit * a.chunks) * kReadSlots;
  const int b = unit / a.pg.Hkv, h = unit - b * a.pg.Hkv;
  const int n = clamp_len(((TablePtr)(uintptr_t)a.ctx_lens)[b], a.max_ctx);
  const int count = a.idx ? clamp_len(((TablePtr)(uintptr_t)a.n_sel)[unit], a.k) : min(a.k, n);
  const int64_t slot0 = (int64_t)unit * a.k;
  const int32_t* table = a.pg.table + (int64_t)b * a.pg.table_stride;
  const uint8_t* pages = (is_v ? a.pg.v : a.pg.k) + h * a.pg.head_bytes + row_part(KIND) * c;
  const uint8_t* exps = is_v ? a.pg.v_exps : a.pg.k_exps;
  uint16_t* dst = (is_v ? a.v_dst : a.k_dst) + slot0 * kD + 8 * c;
  int pos[kReadUnroll], page[kReadUnroll];
#pragma unroll
  for (int i = 0; i < kReadUnroll; ++i) {
    const int s = first + i * (kPagedReadThreads / 32) + (threadIdx.x >> 5);
    pos[i] = s < count ? (a.idx ? a.idx[slot0 + s] : s) : -1;
    if ((unsigned)pos[i] >= (unsigned)n) pos[i] = -1;
  }
#pragma unroll
  for (int i = 0; i < kReadUnroll; ++i) {
    page[i] = pos[i] >= 0 ? table[pos[i] >> a.pg.shift] : -1;
    if ((unsigned)page[i] >= (unsigned)a.pg.num_pages) page[i] = -1;
  }
  // rows that are not there: some row, not stored
  const int mask = (1 << a.pg.shift) - 1;
  u32x4 w[kReadUnroll];
  uint32_t e[kReadUnroll];
#pragma unroll
  for (int i = 0; i < kReadUnroll; ++i) {
    const int row = page[i] >= 0 ? pos[i] & mask : 0;
    const int64_t pg = max(page[i], 0);
    const uint8_t* p = pages + pg * a.pg.page_bytes + row * a.pg.row_bytes;
    if (KIND == Kind::kE4M3) {
      const uint2 x = ld8_nt(p);
      w[i] = u32x4{x.x, x.y, 0u, 0u};
      e[i] = exps[((pg * a.pg.Hkv + h) << a.pg.shift) + row];
    } else if (KIND == Kind::kE2M1) {
      w[i] = u32x4{ld4_nt(p), 0u, 0u, 0u};
      e[i] = exps[4 * (((pg * a.pg.Hkv + h) << a.pg.shift) + row) + (c >> 2)];
    } else {
      w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    }
  }
#pragma unroll
  for (int i = 0; i < kReadUnroll; ++i) {
    if (page[i] < 0) continue;
    const int s = first + i * (kPagedReadThreads / 32) + (threadIdx.x >> 5);
    if (KIND == Kind::kE2M1) {
      *reinterpret_cast<uint4*>(dst + (int64_t)s * kD) = e2m1_octet(w[i][0], e[i] << 23);
    } else if (KIND == Kind::kE4M3) {
      float x[8];
      unpack8(e4m3_octet(make_uint2(w[i][0], w[i][1])), x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = times_exp(x[j], e[i]);
      *reinterpret_cast<uint4*>(dst + (int64_t)s * kD) = pack8_bf16(x);
    } else {
      *reinterpret_cast<u32x4*>(dst + (int64_t)s * kD) = w[i];
    }
  }
}

// ---- ranges of work ------------------------------------------------------------------
// Work is counted in steps of STEP positions of a unit (request, KV head), over
// all units in order: workgroup w of W takes the steps [total * w / W, total *
// (w + 1) / W), whatever requests they belong to, so that a ragged batch, one
// long request and many short ones all fill the device evenly, and the division
// is the device's own (lengths are device data; max_ctx says little about
// them).  Fewer steps than workgroups: one each for the first ones.
__device__ __forceinline__ int64_t range_start(int64_t total, int w, int nwg) {
  return total * w / nwg;
}

struct Lens {
  TablePtr ctx_lens;
  int32_t B, Hkv, max_ctx;
  __device__ __forceinline__ int operator()(int b) const {
    return clamp_len(ctx_lens[b], max_ctx);
  }
};

template <int STEP>
__device__ __forceinline__ int steps_of(const Lens& n, int b) {
  return (n(b) + STEP - 1) / STEP;
}

struct RangeLds {
  int64_t wave_sum[4];
  int64_t off;
  int32_t b;
};

// A workgroup's range and where it begins: step s0's request and head, and its
// number in that unit.
struct Range {
  int64_t s0, s1, total;
  int32_t b, h, step, steps;  // steps: of the unit
};

// Ranges of that many steps (at least `least` each while there are several).
__device__ __forceinline__ int ranges_of(int64_t total, int max_wgs, int least) {
  return (int)min((int64_t)max_wgs, (total + least - 1) / least);
}

template <int STEP>
__device__ __forceinline__ Range find_range(const Lens& n, int max_wgs, int least, RangeLds& lds) {
  constexpr int kThreads = 256;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (n.B + kThreads - 1) / kThreads;
  const int b0 = min(tid * per, n.B), b1 = min(b0 + per, n.B);
  int64_t mine = 0;
  for (int b = b0; b < b1; ++b) mine += (int64_t)steps_of<STEP>(n, b) * n.Hkv;
  int64_t incl = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t up = __shfl_up(incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 63) lds.wave_sum[wave] = incl;
  __syncthreads();
  Range r;
  r.total = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) incl += lds.wave_sum[w];
    r.total += lds.wave_sum[w];
  }
  const int nwg = ranges_of(r.total, max_wgs, least), w = min((int)blockIdx.x, nwg);
  r.s0 = nwg ? range_start(r.total, w, nwg) : 0;
  r.s1 = nwg ? range_start(r.total, min(w + 1, nwg), nwg) : 0;
  int64_t at = incl - mine;
  if (r.s0 < r.s1 && r.s0 >= at && r.s0 < incl) {
    for (int b = b0; b < b1; ++b) {
      const int64_t s = (int64_t)steps_of<STEP>(n, b) * n.Hkv;
      if (r.s0 < at + s) {
        lds.b = b;
        lds.off = r.s0 - at;
        break;
      }
      at += s;
    }
  }
  __syncthreads();
  r.b = r.h = r.step = 0;
  r.steps = 1;
  if (r.s0 < r.s1) {
    r.b = __builtin_amdgcn_readfirstlane(lds.b);
    r.steps = __builtin_amdgcn_readfirstlane(steps_of<STEP>(n, r.b));
    r.h = __builtin_amdgcn_readfirstlane((int)(lds.off / r.steps));
    r.step = __builtin_amdgcn_readfirstlane((int)(lds.off % r.steps));
  }
  return r;
}

// The unit after the range's current one.
template <int STEP>
__device__ __forceinline__ void next_unit(const Lens& n, int64_t at, Range& r) {
  r.step = 0;
  if (++r.h < n.Hkv || at >= r.s1) return;
  r.h = 0;
  do {
    r.steps = __builtin_amdgcn_readfirstlane(steps_of<STEP>(n, ++r.b));
  } while (r.steps == 0);
}

// ---- scores ----------------------------------------------------------------------------
// A workgroup scores a range of steps of kScoreStep positions, 64 a wave, with
// the next step's keys on their way: queries x keys on 16x16x32 products, heads in the
// rows (row m: head m % G, so that for up to four heads every lane row has them
// all) and positions in the columns, so that the largest over a group's heads is
// taken over a lane's registers and, past four heads, over lane rows.  Lane
// row i keeps the results of the step's i-th 16 positions: lane l has position
// p + l.  Scores wait in LDS while keys are loaded: a store between loads would
// be waited for with them (106 -> 92 us for 0.54 GB of e4m3 keys and 17 MB of
// scores, 6.1 TB/s).  128 units of 16384 positions, pages of 64, 16, 8, 4, 2 and 1:
// e4m3 49, 49, 58, 61, 66 and 78 us, bf16 91, 90, 110, 110, 114 and 117.
constexpr int kPagedScoreThreads = 256;
constexpr int kScoreHold = 16;  // steps whose scores a wave holds

template <Kind KIND>
struct ScoreStep {
  KRaw<KIND> k[4];
  uint32_t e;   // of the lane's own position (e4m3)
  bool there;   // likewise
};

// Pages of a step's 64 positions: four halves of one page each (WIDE, for the
// whole wave), or the lane's own positions' and its key rows' (page of row 16 i
// + r in row[i]), looked up a step ahead.
template <bool WIDE>
struct ScorePages {
  int row[4];
  int own;
};

template <bool WIDE>
__device__ __forceinline__ ScorePages<WIDE> score_pages(const PagedPages& pg, const Ctx& x,
                                                        int p) {
  const int lane = threadIdx.x & 63, r = lane & 15;
  ScorePages<WIDE> t;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    t.row[i] = x.table[min(p + 16 * i + (WIDE ? 0 : r), x.n - 1) >> pg.shift];
  if (WIDE) {
    const int g = lane >> 4;
    t.own = g & 2 ? (g & 1 ? t.row[3] : t.row[2]) : (g & 1 ? t.row[1] : t.row[0]);
  } else {
    t.own = x.table[min(p + lane, x.n - 1) >> pg.shift];
  }
  return t;
}

template <Kind KIND, bool WIDE>
__device__ __forceinline__ void load_score_step(const PagedPages& pg, const Ctx& x, int p,
                                                const ScorePages<WIDE>& t, ScoreStep<KIND>& s) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  s.there = (unsigned)t.own < (unsigned)pg.num_pages && p + lane < x.n;
  if (KIND == Kind::kE4M3)
    s.e = pg.k_exps[exp_offset(pg, s.there ? t.own : 0, x.h, min(p + lane, x.n - 1))];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool has = (unsigned)t.row[i] < (unsigned)pg.num_pages;
    if (WIDE) {
      const int first = half_first(p, i, x.n);
      const uint8_t* base = pg.k + row_offset(pg, has ? t.row[i] : 0, x.h, first);
      const int32_t cap = half_last(first, x.n) * pg.row_bytes;
      s.k[i].template load_lines<true>(base, pg.row_bytes, cap, g, r);
      if (KIND == Kind::kE2M1)
        s.k[i].e = pg.k_exps[4 * (exp_offset(pg, has ? t.row[i] : 0, x.h, first) +
                                  min(r, half_last(first, x.n))) + g];
    } else {
      if (KIND == Kind::kE2M1)
        s.k[i].e = pg.k_exps[4 * exp_offset(pg, has ? t.row[i] : 0, x.h,
                                            min(p + 16 * i + r, x.n - 1)) + g];
      s.k[i].load(pg.k + row_offset(pg, has ? t.row[i] : 0, x.h, min(p + 16 * i + r, x.n - 1)),
                  g);
    }
  }
}

// Scores of a step: the largest over the group's heads, of position p + lane.
template <Kind KIND, bool WIDE, int G>
__device__ __forceinline__ float step_scores(ScoreStep<KIND>& s, const bf16x8* q, float scale) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  float best[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if constexpr (WIDE) s.k[i].swap_halves(r);
#pragma unroll
    for (int f = 0; f < 4; ++f) acc = mfma_16x16x32(q[f], s.k[i].frag(f), acc);
    best[i] = acc[0];  // register j of lane (g, r): head (4g + j) % G at position r
#pragma unroll
    for (int j = 1; j < (G < 4 ? G : 4); ++j) best[i] = fmaxf(best[i], acc[j]);
    if (G >= 8) best[i] = fmaxf(best[i], __shfl_xor(best[i], 16));
    if (G == 16) best[i] = fmaxf(best[i], __shfl_xor(best[i], 32));
  }
  float mine = (g & 2 ? (g & 1 ? best[3] : best[2]) : (g & 1 ? best[1] : best[0])) * scale;
  if (KIND == Kind::kE4M3) mine = times_exp(mine, s.e);
  return s.there ? mine : -INFINITY;
}

template <Kind KIND, bool WIDE, int G>
__global__ __launch_bounds__(kPagedScoreThreads, score_wgs_per_cu(WIDE)) void k_paged_score(
    PagedScoreArgs a) {
  __shared__ float hold[4][64 * kScoreHold];  // finished scores, stored some steps later
  __shared__ RangeLds range;
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Lens lens = {(TablePtr)(uintptr_t)a.ctx_lens, a.B, a.pg.Hkv, a.max_ctx};
  Range rg;
  if (a.direct) {  // one step of one unit a workgroup
    const int unit = blockIdx.x / a.chunks;
    rg.step = blockIdx.x - unit * a.chunks;
    rg.b = unit / a.pg.Hkv;
    rg.h = unit - rg.b * a.pg.Hkv;
    rg.steps = steps_of<kScoreStep>(lens, rg.b);
    rg.s0 = 0;
    rg.s1 = rg.step < rg.steps;
  } else {
    rg = find_range<kScoreStep>(lens, a.nwg, 1, range);
  }
  for (int64_t at = rg.s0; at < rg.s1;) {
    const int take = (int)min((int64_t)(rg.steps - rg.step), rg.s1 - at);
    Ctx x;
    x.b = rg.b;
    x.h = rg.h;
    x.n = lens(rg.b);
    x.table = table_of(a.pg, rg.b);
    float* scores = a.scores + ((int64_t)rg.b * a.pg.Hkv + rg.h) * a.max_ctx;
    const int stop = min((rg.step + take) * kScoreStep, x.n);
    int p = rg.step * kScoreStep + 64 * wave;
    if (p < stop) {
      ScoreStep<KIND> s;
      ScorePages<WIDE> pages = score_pages<WIDE>(a.pg, x, p);
      load_score_step<KIND, WIDE>(a.pg, x, p, pages, s);
      pages = score_pages<WIDE>(a.pg, x, lookup_at(p + kScoreStep, stop));
      bf16x8 q[4];
#pragma unroll
      for (int f = 0; f < 4; ++f)
        q[f] = as_bf16x8(ld16(a.q + ((int64_t)x.b * a.Hq + x.h * G + (r & (G - 1))) * kD +
                              frag_base<KIND>(f, g)));
      float* mine = hold[wave] + lane;
      for (int i = 0;;) {
        mine[64 * i++] = step_scores<KIND, WIDE, G>(s, q, a.scale);
        p += kScoreStep;
        const bool more = p < stop;
        if (!more || i == kScoreHold) {
          for (int w = p - i * kScoreStep, k = 0; k < i; ++k, w += kScoreStep)
            if (w + lane < stop) scores[w + lane] = mine[64 * k];
          i = 0;
        }
        if (!more) break;
        load_score_step<KIND, WIDE>(a.pg, x, p, pages, s);
        pages = score_pages<WIDE>(a.pg, x, lookup_at(p + kScoreStep, stop));
      }
    }
    at += take;
    next_unit<kScoreStep>(lens, at, rg);
  }
  if (a.direct) {  // the same step's
    static_assert(kScoreStep == kPagedScoreThreads, "a position a thread");
    const int unit = blockIdx.x / a.chunks;
    const int p = (blockIdx.x - unit * a.chunks) * kScoreStep + threadIdx.x;
    if (p >= lens(unit / a.pg.Hkv) && p < a.max_ctx)
      a.scores[(int64_t)unit * a.max_ctx + p] = -INFINITY;
    return;
  }
  // positions past the contexts' ends, in pieces shared out over the grid
  const int64_t pieces = (int64_t)a.units * a.chunks;
  for (int64_t i = blockIdx.x; i < pieces; i += gridDim.x) {
    const int unit = (int)(i / a.chunks), c = (int)(i - (int64_t)unit * a.chunks);
    const int from = max(lens(unit / a.pg.Hkv), c * a.piece);
    const int to = (int)min((int64_t)(c + 1) * a.piece, (int64_t)a.max_ctx);
    for (int p = from + threadIdx.x; p < to; p += kPagedScoreThreads)
      a.scores[(int64_t)unit * a.max_ctx + p] = -INFINITY;
  }
}

// ---- attention -----------------------------------------------------------------------
constexpr int kPagedAttnThreads = 256;
// Least steps of a range: one step is a chain of latencies and a partial to
// join.  Against ranges of one, us: 8 units of 16 rows and 8192 positions 24.4 ->
// 19.6, 16384 28.7 -> 25.4; one unit of 4 rows and 65536 39.3 -> 22.7 (of 16384
// 16.3 -> 16.5).
constexpr int kLeastSteps = 4;

struct PagedAttnLds {
  float m[4][16], l[4][16];
  float o[4][16][kPartStride];
  float jm[16], jl[16];      // direct: the joining workgroup's own partial (and o[0])
  RangeLds range;
};

// Whether a step has no page at all (for the whole wave).
__device__ __forceinline__ bool no_pages(const TileAt<true>& at) {
  return (at.page[0] & at.page[1]) < 0;
}

__device__ __forceinline__ bool no_pages(const TileAt<false>& at) {
  int all = -1;
#pragma unroll
  for (int j = 0; j < 8; ++j) all &= at.v_page[j];
  return !__any(all >= 0);
}

// The next step from `next` on that has a page, with its lookup.  Steps whose
// pages are all gone are passed over, 64 lookups at a time (of small pages 8
// times 64 positions'), so that a context's time goes by what eviction left of it:
// 150000 to 200001 positions, of which the first page and the last 1024 are kept,
// 98 -> 34 us (e4m3, two sequences), with every page there the same; pages of 4
// and 20000 to 32768 positions 139 -> 46 (bf16, 16 sequences), with every page there
// 283 -> 294.  Called once the step's logits are taken, when the lookup has come.
template <bool WIDE>
__device__ __forceinline__ int with_pages(const PagedPages& pg, const Ctx& x, int next, int end,
                                          TileAt<WIDE>* at) {
  while (next < end && no_pages(*at)) {
    const int lane = threadIdx.x & 63;
    int skip;
    if (WIDE) {
      const int p = next + lane * kPagedStep;
      bool any = false;
      if (p < end) any = page_at(pg, x, p) >= 0 || page_at(pg, x, min(p + 16, x.n - 1)) >= 0;
      const uint64_t mask = __ballot(any) & ~1ull;  // `next` itself has none
      skip = mask ? __builtin_ctzll(mask) : 64;
    } else {
      int page[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {  // steps 2j and 2j + 1, a lane a position
        const int p = next + (2 * j + (lane >> 5)) * kPagedStep + (lane & 31);
        page[j] = page_at(pg, x, min(p, end - 1));
        if (p >= end) page[j] = -1;
      }
      uint32_t mask = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint64_t any = __ballot(page[j] >= 0);
        mask |= (uint32_t)((uint32_t)any != 0) << 2 * j |
                (uint32_t)(any >> 32 != 0) << (2 * j + 1);
      }
      mask &= ~1u;
      skip = mask ? __builtin_ctz(mask) : 16;
    }
    next += skip * kPagedStep;
    *at = tile_at<WIDE>(pg, x, lookup_at(next, end));
  }
  return next;
}

// A wave's steps of a piece: positions [p, end) in strides of kPagedStep.  Only
// the last one can meet the end of a query row's positions (T <= 16 of them are
// not seen by all); the loop's loads are unconditional, so that each wait is
// for the rows it needs and not for all that is in flight.
template <Kind KIND, bool WIDE>
__device__ __forceinline__ void attn_steps(const PagedAttnArgs& a, const Ctx& x, int p, int end,
                                           int limit, float c, const bf16x8* q, WaveState& st) {
  if (p >= end) return;
  const PagedPages& pg = a.pg;
  Tile<KIND> t;
  float lg[8];
  TileAt<WIDE> at = tile_at<WIDE>(pg, x, p);
  p = with_pages<WIDE>(pg, x, p, end, &at);
  if (p >= end) return;
  load_k<KIND, WIDE>(pg, x, at, t);
  load_v<KIND, WIDE>(pg, x, at, t);
  int next = p + kPagedStep;
  at = tile_at<WIDE>(pg, x, lookup_at(next, end));
  while (next < end) {
    tile_logits<KIND, WIDE>(t, q, lg);
    next = with_pages<WIDE>(pg, x, next, end, &at);  // from end on: rows that nobody uses
    load_k<KIND, WIDE>(pg, x, at, t);
    __builtin_amdgcn_sched_barrier(0);
    const bool masked = WIDE ? t.there != 255u : __any(t.there != 255u);
    tile_rest<KIND>(t, masked, p, limit, x.n, c, lg, st);
    __builtin_amdgcn_sched_barrier(0);
    load_v<KIND, WIDE>(pg, x, at, t);
    p = next;
    next += kPagedStep;
    at = tile_at<WIDE>(pg, x, lookup_at(next, end));
  }
  if (p >= end) return;
  tile_logits<KIND, WIDE>(t, q, lg);
  tile_rest<KIND>(t, true, p, limit, x.n, c, lg, st);
}

// The same two steps at a time, for the 4-bit kind: a step's rows are few bytes, and
// loads of one step in flight a wave do not cover the memory's latency (64 sequences
// of 1 k to 32 k positions 262 -> 237 us, two of 150 k to 200 k 100 -> 91; three
// workgroups a CU instead of two: 239 and 98).
template <Kind KIND, bool WIDE>
__device__ __forceinline__ void attn_pairs(const PagedAttnArgs& a, const Ctx& x, int p, int end,
                                           int limit, float c, const bf16x8* q, WaveState& st) {
  if (p >= end) return;
  const PagedPages& pg = a.pg;
  Tile<KIND> t[2];
  TileAt<WIDE> at[2];
  at[0] = tile_at<WIDE>(pg, x, p);
  p = with_pages<WIDE>(pg, x, p, end, &at[0]);
  if (p >= end) return;
  limit = min(limit, end);  // the second step of a pair may lie past the piece
  at[1] = tile_at<WIDE>(pg, x, lookup_at(p + kPagedStep, end));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    load_k<KIND, WIDE>(pg, x, at[i], t[i]);
    load_v<KIND, WIDE>(pg, x, at[i], t[i]);
  }
  int next = p + 2 * kPagedStep;
#pragma unroll
  for (int i = 0; i < 2; ++i) at[i] = tile_at<WIDE>(pg, x, lookup_at(next + i * kPagedStep, end));
  while (p < end) {
    float lg[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) tile_logits<KIND, WIDE>(t[i], q, lg[i]);
    const int to = with_pages<WIDE>(pg, x, next, end, &at[0]);
    if (to != next) at[1] = tile_at<WIDE>(pg, x, lookup_at(to + kPagedStep, end));
    next = to;
#pragma unroll
    for (int i = 0; i < 2; ++i) load_k<KIND, WIDE>(pg, x, at[i], t[i]);
    __builtin_amdgcn_sched_barrier(0);
    const uint32_t all = t[0].there & t[1].there;
    if (next >= end || (WIDE ? all != 255u : __any(all != 255u))) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        tile_mask<KIND>(t[i], p + i * kPagedStep, limit, x.n, lg[i]);
    }
    raise_max(fmaxf(top_of(lg[0]), top_of(lg[1])), c, st);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t part[3][8];
      tile_weights<KIND>(t[i].ve, c, less_max(st), lg[i], part, st);
      tile_output<KIND>(t[i], part, st);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 2; ++i) load_v<KIND, WIDE>(pg, x, at[i], t[i]);
    p = next;
    next += 2 * kPagedStep;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      at[i] = tile_at<WIDE>(pg, x, lookup_at(next + i * kPagedStep, end));
  }
}

__device__ __forceinline__ int64_t out_row(const PagedAttnArgs& a, int b, int h, int row) {
  const int t = row >> a.lg, g = row & ((1 << a.lg) - 1);
  return ((int64_t)b * a.T + t) * a.Hq + (h << a.lg) + g;
}

// One piece: positions [step, step + take) * kPagedStep of unit (b, h), the four
// waves' states left in lds.
template <Kind KIND, bool WIDE, bool LONG>
__device__ __forceinline__ void attn_piece(const PagedAttnArgs& a, int b, int h, int n, int step,
                                           int take, PagedAttnLds& lds) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = a.T << a.lg;
  // e4m3 exponents are taken less 128: one power of two more in the logits'
  // factor and, at the end, in the sums of V
  const float c = a.scale * (KIND == Kind::kE4M3 ? 2.f : 1.f) * 1.4426950408889634f;
  const Ctx x = {b, h, n, table_of(a.pg, b)};
  const int64_t qrow = out_row(a, b, h, r);
  const int limit = r < rows ? n - (a.T - 1 - (r >> a.lg)) : 0;
  bf16x8 q[4];
#pragma unroll
  for (int f = 0; f < 4; ++f)
    q[f] = as_bf16x8(r < rows ? ld16(a.q + qrow * kD + frag_base<KIND>(f, g))
                              : make_uint4(0u, 0u, 0u, 0u));
  WaveState st;
  st.m = -INFINITY;
  st.l = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) st.o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int p = step * kPagedStep + wave * kPagedTile, end = min((step + take) * kPagedStep, n);
  if constexpr (LONG && KIND == Kind::kE2M1)
    attn_pairs<KIND, WIDE>(a, x, p, end, limit, c, q, st);
  else
    attn_steps<KIND, WIDE>(a, x, p, end, limit, c, q, st);
  st.l += __shfl_xor(st.l, 16);
  st.l += __shfl_xor(st.l, 32);
  if (g == 0) {
    lds.m[wave][r] = st.m;
    lds.l[wave][r] = st.l;
  }
  if (r < rows) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float* o = &lds.o[wave][r][8 * (4 * g + j)];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = KIND == Kind::kE4M3 ? 2.f * st.o[e][j] : st.o[e][j];
    }
  }
  __syncthreads();
}

__device__ __forceinline__ void store_result(const PagedAttnArgs& a, int b, int h, int row, int d,
                                             const Partial& p) {
  const int64_t at = out_row(a, b, h, row);
  const float inv = inverse_sum(p.L);
  *reinterpret_cast<float4*>(a.out + at * kD + d) =
      make_float4(p.o.x * inv, p.o.y * inv, p.o.z * inv, p.o.w * inv);
  if (a.lse && d == 0) a.lse[at] = log_sum(p.M, p.L);
}

// A request without any position.
__device__ __forceinline__ void store_empty(const PagedAttnArgs& a, int64_t first_row,
                                            int64_t rows) {
  for (int64_t i = threadIdx.x; i < rows * (kD / 4); i += kPagedAttnThreads)
    reinterpret_cast<float4*>(a.out)[first_row * (kD / 4) + i] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (a.lse)
    for (int64_t i = threadIdx.x; i < rows; i += kPagedAttnThreads)
      a.lse[first_row + i] = -INFINITY;
}

// A workgroup attends over a range of steps, unit by unit; sums of a unit that
// other ranges share go to memory.  Bound by the reading of K and V, whose lines
// are fetched once (4.44 of 4.43 GB, 769 of 762 MB): 4.43 GB of 64 bf16 sequences
// 664 us a call (6.7 TB/s), 0.76 GB of two e4m3 sequences with 16 query rows a unit
// 128 (6.0), of which the join is 6 to 8.  128 units of 16384 positions, pages of
// 64, 16, 8, 4, 2 and 1: e4m3 93, 97, 113, 114, 123 and 148 us, bf16 172, 174, 182,
// 185, 190 and 204.
template <Kind KIND, bool WIDE>
__global__ __launch_bounds__(kPagedAttnThreads, 2) void k_paged_attn(
    PagedAttnArgs a) {
  __shared__ PagedAttnLds lds;
  const int tid = threadIdx.x, w = blockIdx.x, rows = a.T << a.lg;
  const Lens lens = {(TablePtr)(uintptr_t)a.ctx_lens, a.B, a.pg.Hkv, a.max_ctx};
  for (int u = w; u < a.B; u += a.nwg)
    if (lens(u) == 0) store_empty(a, (int64_t)u * a.T * a.Hq, (int64_t)a.T * a.Hq);
  Range rg = find_range<kPagedStep>(lens, a.nwg, kLeastSteps, lds.range);
  PagedTail tail = {0, rg.total, -1, 0};
  int64_t at = rg.s0;
  while (at < rg.s1) {
    const int b = rg.b, h = rg.h, step = rg.step, steps = rg.steps;
    const int take = (int)min((int64_t)(steps - step), rg.s1 - at);
    attn_piece<KIND, WIDE, true>(a, b, h, lens(b), step, take, lds);
    const int slot = at == rg.s0 ? 0 : 1;
    for (int i = tid; i < rows * (kD / 4); i += kPagedAttnThreads) {
      const int row = i >> 5, d = 4 * (i & 31);
      const Partial p = join_waves(lds, row, d);
      if (take == steps) {
        store_result(a, b, h, row, d, p);
        continue;
      }
      float* part = a.part + (((int64_t)w * 2 + slot) * rows + row) * kPartStride;
      *reinterpret_cast<float4*>(part + 4 + d) = p.o;
      if (d == 0) {
        part[0] = p.M;
        part[1] = p.L;
      }
    }
    __syncthreads();
    if (step == 0 && take < steps) {  // begins here and goes on: this range's to join
      tail.unit = b * a.pg.Hkv + h;
      tail.end = at + steps;
      tail.slot = slot;
    }
    at += take;
    next_unit<kPagedStep>(lens, at, rg);
  }
  if (tid == 0) a.tail[w] = tail;
}

// Joins a unit's steps: partials 0 .. steps - 2 handed over in memory, before
// `part` (where the last step's would be), the last one's in lds.  Wave w takes
// query rows w, w + 4, ... (at most ROWS of them; those past the last are the last
// again), all of whose loads are asked for together: lane i weighs step i, then
// lanes take two channels each.
template <int ROWS>
__device__ __forceinline__ void join_steps(const PagedAttnArgs& a, int b, int h, int steps,
                                           const float* part, const PagedAttnLds& lds) {
  const int lane = threadIdx.x & 63, rows = a.T << a.lg;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave >= rows) return;
  const int64_t next = (int64_t)rows * kPartStride;  // in pairs of floats: 2 * rows partial rows
  uint64_t* base = reinterpret_cast<uint64_t*>(const_cast<float*>(part)) - (steps - 1) * next;
  uint64_t* p0[ROWS];
  int row[ROWS];
  float f[ROWS], M[ROWS], L[ROWS];
  float2 o[ROWS];
  uint64_t ml[ROWS];
  constexpr int kAhead = 16 / ROWS;
  uint64_t x[kAhead][ROWS];
  auto load = [&](int i0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int k = 0; k < ROWS; ++k)
        x[i][k] = __hip_atomic_load(p0[k] + min(i0 + i, steps - 2) * next + 2 + lane,
                                    __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    row[k] = min(wave + 4 * k, rows - 1);
    p0[k] = base + row[k] * (kPartStride / 2);
    ml[k] = __hip_atomic_load(p0[k] + min(lane, steps - 2) * next, __ATOMIC_RELAXED,
                              __HIP_MEMORY_SCOPE_AGENT);
  }
  load(0);
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    const bool own = lane == steps - 1, past = lane >= steps;
    const float m = own ? lds.jm[row[k]] : past ? -INFINITY : __uint_as_float((uint32_t)ml[k]);
    const float l = own ? lds.jl[row[k]] : __uint_as_float((uint32_t)(ml[k] >> 32));
    M[k] = wave_max(m);
    f[k] = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M[k]);
    L[k] = wave_sum(f[k] == 0.f && !own ? 0.f : f[k] * l);
    o[k] = make_float2(0.f, 0.f);
  }
  for (int i0 = 0; i0 < steps - 1; i0 += kAhead) {
    if (i0 > 0) load(i0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int k = 0; k < ROWS; ++k) {
        const float fk = i0 + i < steps - 1 ? __shfl(f[k], i0 + i) : 0.f;
        o[k].x = fmaf(fk, __uint_as_float((uint32_t)x[i][k]), o[k].x);
        o[k].y = fmaf(fk, __uint_as_float((uint32_t)(x[i][k] >> 32)), o[k].y);
      }
  }
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    if (wave + 4 * k >= rows) break;
    const float fk = __shfl(f[k], steps - 1);
    const float2 own = *reinterpret_cast<const float2*>(&lds.o[0][row[k]][2 * lane]);
    o[k].x = fmaf(fk, own.x, o[k].x);
    o[k].y = fmaf(fk, own.y, o[k].y);
    const int64_t at = out_row(a, b, h, row[k]);
    const float inv = inverse_sum(L[k]);
    *reinterpret_cast<float2*>(a.out + at * kD + 2 * lane) =
        make_float2(o[k].x * inv, o[k].y * inv);
    if (a.lse && lane == 0) a.lse[at] = log_sum(M[k], L[k]);
  }
}

// The same with a workgroup for every piece of 2^piece steps of every unit
// (workgroup unit * chunks + piece) and the join inside the launch, for few
// steps: each hands its partial over through its flag, once the partial's
// device-coherent stores are done; the workgroup of the unit's last piece waits
// for the flags, which are clear again after the launch, and joins.  Of one
// launch only higher-numbered workgroups wait, for lower-numbered ones that
// never do; should several launches keep each other's off the device, the bound
// ends the wait, and that call's outputs of the unit are NaN.  8 units of 2001
// positions: 7.7 us, against 10.4 with ranges and a second launch; a chain of
// latencies (length, page, rows, hand-over, join), which 8 MB of rows hardly
// lengthen.
constexpr uint32_t kJoinSpinLimit = 1u << 24;  // about 20 s

struct JoinFlag {
  uint64_t* f;
  __device__ __forceinline__ uint64_t load() const {
    return __hip_atomic_load(f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ __forceinline__ void store(uint64_t x) const {
    __hip_atomic_store(f, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ __forceinline__ uint64_t exchange(uint64_t x) const {
    return __hip_atomic_exchange(f, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ __forceinline__ void pause() const { __builtin_amdgcn_s_sleep(2); }
};

template <Kind KIND, bool WIDE>
__global__ __launch_bounds__(kPagedAttnThreads, 2) void k_paged_attn_direct(PagedAttnArgs a) {
  __shared__ PagedAttnLds lds;
  const int tid = threadIdx.x, rows = a.T << a.lg;
  const int unit = blockIdx.x / a.chunks, piece = blockIdx.x - unit * a.chunks;
  const int b = unit / a.pg.Hkv, h = unit - b * a.pg.Hkv;
  const int n = clamp_len(((TablePtr)(uintptr_t)a.ctx_lens)[b], a.max_ctx);
  const int pieces = (n + (kPagedStep << a.piece) - 1) / kPagedStep >> a.piece;
  if (piece >= pieces) {
    if (piece == 0)  // no positions: this unit's query rows
      for (int t = 0; t < a.T; ++t)
        store_empty(a, out_row(a, b, h, t << a.lg), (int64_t)1 << a.lg);
    return;
  }
  attn_piece<KIND, WIDE, false>(a, b, h, n, piece << a.piece, 1 << a.piece, lds);
  const bool last = piece == pieces - 1;
  float* part = a.part + (int64_t)blockIdx.x * 2 * rows * kPartStride;
  for (int i = tid; i < rows * (kD / 4); i += kPagedAttnThreads) {
    const int row = i >> 5, d = 4 * (i & 31);
    const Partial p = join_waves(lds, row, d);
    if (pieces == 1) {
      store_result(a, b, h, row, d, p);
    } else if (last) {  // (row, d) of o[0] is read by this thread alone
      *reinterpret_cast<float4*>(&lds.o[0][row][d]) = p.o;
      if (d == 0) {
        lds.jm[row] = p.M;
        lds.jl[row] = p.L;
      }
    } else {
      uint64_t* o = reinterpret_cast<uint64_t*>(part + row * kPartStride + 4 + d);
      const uint64_t v[2] = {__float_as_uint(p.o.x) | (uint64_t)__float_as_uint(p.o.y) << 32,
                             __float_as_uint(p.o.z) | (uint64_t)__float_as_uint(p.o.w) << 32};
      __hip_atomic_store(o, v[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(o + 1, v[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (d == 0)
        __hip_atomic_store(reinterpret_cast<uint64_t*>(part + row * kPartStride),
                           __float_as_uint(p.M) | (uint64_t)__float_as_uint(p.L) << 32,
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  if (pieces == 1) return;
  if (!last) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) hand_over(JoinFlag{a.flags + blockIdx.x}, a.tag);
    return;
  }
  bool late = false;
  if (tid < pieces - 1)
    late = !take_over(JoinFlag{a.flags + (int64_t)unit * a.chunks + tid}, a.tag, kJoinSpinLimit);
  if (__syncthreads_or(late) && tid < rows) lds.jl[tid] = NAN;  // every output of the unit
  __syncthreads();
  if (rows <= 4) join_steps<1>(a, b, h, pieces, part, lds);
  else if (rows <= 8) join_steps<2>(a, b, h, pieces, part, lds);
  else join_steps<4>(a, b, h, pieces, part, lds);
}

// Joins the unit that workgroup blockIdx.x's range left unfinished: query row
// blockIdx.y over the range's own partial and the first partials of the ranges
// after it, in order.  6 us for a batch's few shared units, 8 for two sequences
// that 512 ranges share (34 partials a unit): latency.
constexpr int kPagedMergeThreads = 256;

__global__ __launch_bounds__(kPagedMergeThreads) void k_paged_merge(PagedAttnArgs a) {
  __shared__ float weight[kMaxPagedWgs];
  __shared__ float4 sums[kPagedMergeThreads / 32][32];
  __shared__ float red[kPagedMergeThreads / 64];
  const int w = blockIdx.x, row = blockIdx.y, rows = a.T << a.lg;
  const PagedTail t = a.tail[w];
  if (t.unit < 0) return;
  // the last range that begins before the unit's end: total * i / nwg < end
  const int64_t nwg = ranges_of(t.total, a.nwg, kLeastSteps);
  const int n = (int)((t.end * nwg - 1) / t.total) - w + 1;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto partial = [&](int i) {
    return a.part + (((int64_t)(w + i) * 2 + (i == 0 ? t.slot : 0)) * rows + row) * kPartStride;
  };
  float M = -INFINITY;
  for (int i = tid; i < n; i += kPagedMergeThreads) M = fmaxf(M, partial(i)[0]);
  M = wave_max(M);
  if (lane == 0) red[wave] = M;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPagedMergeThreads / 64; ++i) M = fmaxf(M, red[i]);
  __syncthreads();
  float L = 0.f;
  for (int i = tid; i < n; i += kPagedMergeThreads) {
    const float m = partial(i)[0];
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
    weight[i] = f;
    L = fmaf(f, partial(i)[1], L);
  }
  L = wave_sum(L);
  if (lane == 0) red[wave] = L;
  __syncthreads();
  L = 0.f;
#pragma unroll
  for (int i = 0; i < kPagedMergeThreads / 64; ++i) L += red[i];
  const int d = tid & 31, part = tid >> 5;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kGroups = kPagedMergeThreads / 32, kAhead = 8;
  for (int i0 = part; i0 < n; i0 += kAhead * kGroups) {
    f32x4 x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      x[k] = *reinterpret_cast<const f32x4*>(partial(min(i0 + k * kGroups, n - 1)) + 4 + 4 * d);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + k * kGroups;
      if (i >= n) break;
      const float f = weight[i];
      o.x = fmaf(f, x[k][0], o.x);
      o.y = fmaf(f, x[k][1], o.y);
      o.z = fmaf(f, x[k][2], o.z);
      o.w = fmaf(f, x[k][3], o.w);
    }
  }
  sums[part][d] = o;
  __syncthreads();
  if (part != 0) return;
  for (int i = 1; i < kPagedMergeThreads / 32; ++i) {
    const float4 x = sums[i][d];
    o.x += x.x, o.y += x.y, o.z += x.z, o.w += x.w;
  }
  const int b = t.unit / a.pg.Hkv, h = t.unit - b * a.pg.Hkv;
  const int64_t at = out_row(a, b, h, row);
  const float inv = inverse_sum(L);
  *reinterpret_cast<float4*>(a.out + at * kD + 4 * d) =
      make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  if (a.lse && d == 0) a.lse[at] = log_sum(M, L);
}

// ---- debug mode ------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_paged_check(PagedCheckArgs a) {
  const int64_t stride = (int64_t)gridDim.x * blockDim.x;
  const int64_t total = paged_check_items(a);
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += stride) {
    const unsigned long long kind = paged_check_item(a, i);
    if (kind) atomicMin(a.flag, kind << 56 | (unsigned long long)i);
  }
}

// ---- launchers ---------------------------------------------------------------------------
static inline int grid_for(int64_t n, int per, int cap) {
  const int64_t b = (n + per - 1) / per;
  return (int)std::max<int64_t>(1, std::min<int64_t>(b, cap));
}

// Tokens of a workgroup: one while that gives at most kRopeFew workgroups.
constexpr int kRopeFew = 2048;
static inline int rope_per(int tokens) { return tokens <= kRopeFew ? 1 : kRopeTokens; }

template <typename T>
static void launch_rope_t(const RopeArgs& a, hipStream_t s) {
  const int per = rope_per(a.tokens);
  const dim3 grid((a.tokens + per - 1) / per), block(kRopeThreads);
  const bool whole = rope_whole<T>(a.r.rot, a.r.layout);
  if (a.r.layout == CKV_ROPE_HALF) {
    if (whole) launch_kernel(CKV_K_ROPE, k_rope<T, true, true>, grid, block, s, a, per);
    else launch_kernel(CKV_K_ROPE, k_rope<T, true, false>, grid, block, s, a, per);
  } else {
    if (whole) launch_kernel(CKV_K_ROPE, k_rope<T, false, true>, grid, block, s, a, per);
    else launch_kernel(CKV_K_ROPE, k_rope<T, false, false>, grid, block, s, a, per);
  }
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t s) {
  a.r.f32 ? launch_rope_t<float>(a, s) : launch_rope_t<uint16_t>(a, s);
  return launch_status();
}

template <Kind KIND, Turn TURN>
static void launch_write_t(const PagedWriteArgs& a, hipStream_t s) {
  const int per = rope_per(a.rope.tokens);
  launch_kernel(CKV_K_PAGED_WRITE, k_paged_write<KIND, TURN>,
                dim3((a.rope.tokens + per - 1) / per), dim3(kRopeThreads), s, a, per);
}

template <Kind KIND>
static void launch_write_e(const PagedWriteArgs& a, hipStream_t s) {
  const RopeSpec& r = a.rope.r;
  if (!r.inv_freq) launch_write_t<KIND, Turn::kNone>(a, s);
  else if (!rope_whole<uint16_t>(r.rot, r.layout)) launch_write_t<KIND, Turn::kEach>(a, s);
  else if (r.layout == CKV_ROPE_HALF) launch_write_t<KIND, Turn::kHalf>(a, s);
  else launch_write_t<KIND, Turn::kPairs>(a, s);
}

hipError_t launch_paged_write(const PagedWriteArgs& a, Kind kind, hipStream_t s) {
  of_kind(kind, [&](auto k) { launch_write_e<k.value>(a, s); });
  return launch_status();
}

hipError_t launch_paged_read(const PagedReadArgs& a, Kind kind, hipStream_t s) {
  PagedReadArgs r = a;
  r.chunks = (a.k + kReadSlots - 1) / kReadSlots;
  const dim3 grid((unsigned)(a.units * r.chunks)), block(kPagedReadThreads);
  of_kind(kind, [&](auto k) {
    launch_kernel(CKV_K_PAGED_READ, k_paged_read<k.value>, grid, block, s, r);
  });
  return launch_status();
}

template <Kind KIND, bool WIDE>
static void launch_score_g(const PagedScoreArgs& a, int G, hipStream_t s) {
  const dim3 grid(a.nwg), block(kPagedScoreThreads);
  switch (G) {
    case 1: launch_kernel(CKV_K_PAGED_SCORE, k_paged_score<KIND, WIDE, 1>, grid, block, s, a); break;
    case 2: launch_kernel(CKV_K_PAGED_SCORE, k_paged_score<KIND, WIDE, 2>, grid, block, s, a); break;
    case 4: launch_kernel(CKV_K_PAGED_SCORE, k_paged_score<KIND, WIDE, 4>, grid, block, s, a); break;
    case 8: launch_kernel(CKV_K_PAGED_SCORE, k_paged_score<KIND, WIDE, 8>, grid, block, s, a); break;
    default: launch_kernel(CKV_K_PAGED_SCORE, k_paged_score<KIND, WIDE, 16>, grid, block, s, a);
  }
}

hipError_t launch_paged_score(const PagedScoreArgs& a, Kind kind, int G, hipStream_t s) {
  of_kind(kind, [&](auto k) {
    if (a.pg.shift >= 4) launch_score_g<k.value, true>(a, G, s);
    else launch_score_g<k.value, false>(a, G, s);
  });
  return launch_status();
}

template <Kind KIND, bool WIDE>
static void launch_attn_t(const PagedAttnArgs& a, hipStream_t s) {
  const dim3 grid(a.nwg), block(kPagedAttnThreads);
  if (a.chunks)
    launch_kernel(CKV_K_PAGED_ATTN, k_paged_attn_direct<KIND, WIDE>, grid, block, s, a);
  else
    launch_kernel(CKV_K_PAGED_ATTN, k_paged_attn<KIND, WIDE>, grid, block, s, a);
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, Kind kind, hipStream_t s) {
  of_kind(kind, [&](auto k) {
    if (a.pg.shift >= 4) launch_attn_t<k.value, true>(a, s);
    else launch_attn_t<k.value, false>(a, s);
  });
  const hipError_t e = launch_status();
  if (e != hipSuccess || a.chunks) return e;
  launch_kernel(CKV_K_PAGED_MERGE, k_paged_merge, dim3(a.nwg, a.T << a.lg),
                dim3(kPagedMergeThreads), s, a);
  return launch_status();
}

hipError_t launch_paged_check(const PagedCheckArgs& a, hipStream_t s) {
  const int64_t total = paged_check_items(a);
  hipLaunchKernelGGL(k_paged_check, dim3(grid_for(total, 256, 4096)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace ckv
