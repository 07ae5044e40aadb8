// ckv_paged.hpp -- launch arguments and launchers of the rotary positions and
// the paged cache (ckv_paged.hip), and what their host side shares.
#pragma once

#include <algorithm>

#include "ckv_check.hpp"

namespace ckv {

// Pages as the kernels see them: byte strides, sizes as shifts.
struct PagedPages {
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_exps;        // [num_pages][Hkv][page_size], e4m3 only
  uint8_t* v_exps;
  const int32_t* table;   // [B][table_stride]
  int64_t page_bytes, head_bytes;
  int32_t row_bytes;      // page_size * row_bytes < 2^31
  int32_t shift;          // log2(page_size)
  int32_t num_pages, table_stride, Hkv;
};

struct RopeSpec {
  const double* inv_freq;
  int32_t head_dim, rot, layout, f32, inverse;
  float scale;
};

struct RopeRows {
  const void* src;
  void* dst;
  int64_t src_tok, src_head, dst_tok, dst_head;  // elements
  int32_t heads;
};

struct RopeArgs {
  RopeSpec r;
  RopeRows q, k;           // k.heads 0: none
  const int32_t* pos;
  int32_t tokens;
};

struct PagedWriteArgs {
  PagedPages pg;
  RopeArgs rope;           // r.inv_freq NULL: rows are stored as they are; q: heads 0, or
                           // rotated too
  const int32_t* req;      // NULL: token t is request t's
  const uint16_t* k;
  const uint16_t* v;
  int64_t tok;             // elements between tokens of k and v
  int32_t B, max_ctx;
};

struct PagedReadArgs {
  PagedPages pg;
  const int32_t* ctx_lens;
  const int32_t* idx;      // [U][k], NULL: position i in slot i
  const int32_t* n_sel;    // [U]
  uint16_t* k_dst;
  uint16_t* v_dst;
  int32_t max_ctx, k, units;
  int32_t chunks;          // workgroups a unit (the launcher's)
};

struct PagedScoreArgs {
  PagedPages pg;
  const uint16_t* q;
  const int32_t* ctx_lens;
  float* scores;
  float scale;
  int32_t B, Hq, max_ctx, units;
  int32_t nwg;
  int32_t direct;          // workgroup (unit, step); else ranges
  int32_t piece, chunks;   // positions of a piece of a unit (direct: a step), pieces of a unit
};

// A unit that begins in a workgroup's range and goes on in the next ones:
// left for the join (unit -1: none).
struct PagedTail {
  int64_t end;             // the unit's last step + 1, over all units
  int64_t total;           // steps of all units
  int32_t unit;
  int32_t slot;            // of the workgroup's own partial
};

constexpr int kPagedTile = 32;              // positions of a wave's step
constexpr int kPagedStep = 4 * kPagedTile;  // and of its workgroup's
constexpr int kMaxPagedWgs = 1024;
// Ranges of the attention: two a CU, which it holds at once; one where few units
// mean that many would have to be joined (1 unit of 262144 bf16 positions 43.9 ->
// 35.4 us, 2 65.9 -> 54.1, 4 98.6 -> 92.3; 16 units of 200 k e4m3 positions would
// go 127 -> 135).
constexpr int kPagedWgsPerCu = 2, kFewUnits = 8;
// The attention in one launch: at most so many pieces a unit (one wave's lanes
// weigh them) and partial rows (its 4 waves load them).  8 units, one launch of
// single steps against ranges and a join, us: 4 rows a unit, 256 positions 7.5 /
// 10.4, 4096 9.6 / 12.5, 8192 14.4 / 17.4; 16 rows, 256 positions 9.9 / 10.9, 2048
// 12.5 / 13.5, 8192 27.5 / 24.1 (of 64 pieces, which the limits leave out).
constexpr int kMaxDirect = 64, kMaxDirectRows = 256;
// Where steps are more than that, or than the workgroups that the device holds,
// pieces of up to 2^3 steps, or whole units that short, however many.  Against
// ranges, us: 64 e4m3 units of 2048 positions 18.1 -> 13.5, 512 bf16 units of 100
// to 1000 38.1 -> 29.8, 78 of 2397 28.1 -> 22.4, 8 of 32768 33.1 -> 29.7.  Pieces
// of 16 would give a batch of even lengths up to 12 % more and cost one of 32 with
// a single long sequence 20.1 -> 28.4.  For the join's sake alone up to 2^2: 8
// units of 8 rows and 8192 positions 17.9 -> 13.6, of 16 rows 20.1 -> 17.3; 2^3
// would leave too much of the device idle (1 unit of 16 rows and 16384 positions
// 18.3 -> 21.6, of 4 rows and 60000 19.0 -> 20.6).
constexpr int kMaxPiece = 3, kMaxJoinPiece = 2;
constexpr int kReadSlots = 32;              // slots of a reading workgroup

// A wave's step is two halves of 16 positions.  First position of half i of the
// step at p0 in a context of n positions: its own, or that of the last 16 where
// the half is past the context's end.  p0 is a multiple of 16, and so is the
// result: a half's rows never leave a page of 16 or more.
__host__ __device__ inline int half_first(int p0, int i, int n) {
  const int own = p0 + 16 * i, last = (n - 1) & ~15;
  return own < last ? own : last;
}

// A half's last row, counted from its first.
__host__ __device__ inline int half_last(int first, int n) {
  return n - 1 - first < 15 ? n - 1 - first : 15;
}

// Where a wave whose next step is at `next` looks and loads: there or, once that
// is past the piece's end, at the piece's last 16 positions (rows that nobody
// uses).  A multiple of 16 whatever `end` is.
__host__ __device__ inline int lookup_at(int next, int end) {
  const int last = (end - 1) & ~15;
  return next < last ? next : last;
}

struct PagedAttnArgs {
  PagedPages pg;
  const uint16_t* q;       // [B][T][Hq][d]
  const int32_t* ctx_lens;
  float* out;              // [B][T][Hq][d]
  float* lse;              // [B][T][Hq] or NULL
  float* part;             // [nwg][2][T*G][kPartStride]
  PagedTail* tail;         // [nwg]
  uint64_t* flags;         // [nwg], direct calls
  uint64_t tag;
  float scale;
  int32_t B, Hq, T, lg;    // lg: log2 G
  int32_t max_ctx, nwg;
  int32_t chunks;          // direct: workgroups (pieces) of a unit; else 0
  int32_t piece;           // direct: a piece has 2^piece steps
};

// The hand-over of a partial in the one-launch attention: a flag (any word at
// first) that the partial's workgroup sets to the launch's tag, and that the
// joining one waits for, `limit` polls at most.  Whoever comes second clears it,
// also where the wait was given up, so it is always zero after the launch: a
// captured launch has the same tag in every replay, and a flag left over would
// pass the replay before's partial off as this one's.  Flag has load, store,
// exchange (relaxed: what is handed over is made visible before) and pause.
template <class Flag>
__host__ __device__ inline void hand_over(Flag f, uint64_t tag) {
  if (f.exchange(tag) == ~tag) f.store(0);  // given up: nobody else looks at it
}

template <class Flag>
__host__ __device__ inline bool take_over(Flag f, uint64_t tag, uint32_t limit) {
  for (uint32_t spin = 0; f.load() != tag; ++spin) {
    if (spin == limit) {
      if (f.exchange(~tag) == tag) break;  // it came after all
      return false;
    }
    f.pause();
  }
  f.store(0);
  return true;
}

// Page of position pos of request b, or -1 where it is not there.
__host__ __device__ inline int page_of(const PagedPages& pg, int b, int pos) {
  const int page = pg.table[(int64_t)b * pg.table_stride + (pos >> pg.shift)];
  return (unsigned)page < (unsigned)pg.num_pages ? page : -1;
}

// Debug mode's checks of paged inputs (CheckArgs' codes go on: 4 page_table
// entry b * slots + s, 5 positions[t], 6 requests[t], 7 the page of a written
// token).
struct PagedCheckArgs {
  PagedPages pg;
  const int32_t* ctx_lens; // reading entries
  const int32_t* req;      // writing entries
  const int32_t* pos;
  unsigned long long* flag;
  int32_t B, max_ctx, tokens;
  int32_t slots;           // table entries of max_ctx positions
};

__host__ __device__ inline int64_t paged_check_items(const PagedCheckArgs& a) {
  return a.ctx_lens ? (int64_t)a.B * a.slots : a.tokens;
}

// What is wrong with item i (0: nothing).  Table entries past a context's end are
// not looked at: a table may be some columns of a wider one, whose last row ends
// before table_stride entries.
__host__ __device__ inline unsigned paged_check_item(const PagedCheckArgs& a, int64_t i) {
  if (a.ctx_lens) {
    const int b = (int)(i / a.slots), s = (int)(i - (int64_t)b * a.slots);
    const int len = a.ctx_lens[b], n = len < a.max_ctx ? len : a.max_ctx;
    if (((int64_t)s << a.pg.shift) >= n) return 0;
    const int page = a.pg.table[(int64_t)b * a.pg.table_stride + s];
    return page != -1 && (unsigned)page >= (unsigned)a.pg.num_pages ? 4 : 0;
  }
  if (a.pos[i] == -1) return 0;
  const int b = a.req ? a.req[i] : (int)i;
  if ((unsigned)a.pos[i] >= (unsigned)a.max_ctx) return 5;
  if ((unsigned)b >= (unsigned)a.B) return 6;
  return page_of(a.pg, b, a.pos[i]) < 0 ? 7 : 0;
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t s);
hipError_t launch_paged_write(const PagedWriteArgs& a, bool e4m3, hipStream_t s);
hipError_t launch_paged_read(const PagedReadArgs& a, bool e4m3, hipStream_t s);
hipError_t launch_paged_score(const PagedScoreArgs& a, bool e4m3, int G, hipStream_t s);
hipError_t launch_paged_attn(const PagedAttnArgs& a, bool e4m3, hipStream_t s);
hipError_t launch_paged_check(const PagedCheckArgs& a, hipStream_t s);

inline int check_tokens(const Dims& d, int32_t tokens) {
  if (tokens < 1 || (int64_t)tokens * d.G > 16)
    return fail(CKV_EUNSUPPORTED, "%d tokens of %d heads a group (1 <= tokens * heads <= 16)",
                tokens, d.G);
  return CKV_OK;
}

// Workgroups that a call can have at most: no more than steps.
inline int paged_wgs_cap(const Dims& d) {
  const int64_t steps = (int64_t)d.U * ((d.max_ctx + kPagedStep - 1) / kPagedStep);
  return (int)std::max<int64_t>(1, std::min<int64_t>(steps, kMaxPagedWgs));
}

// Scoring: steps of kScoreStep positions.  While every step can have a
// workgroup of its own at once they are not cut into ranges (finding a range
// takes a scan over the batch).
constexpr int kScoreStep = 256;
// Workgroups that a CU holds at once (single-row lookups take more registers).
constexpr int score_wgs_per_cu(bool wide) { return wide ? 4 : 3; }
constexpr int kScorePiece = 4096;   // positions past the ends that a workgroup fills in turn

inline size_t paged_tail_bytes(const Dims& d) {
  return align256((size_t)paged_wgs_cap(d) * sizeof(PagedTail));
}

inline size_t paged_flag_bytes(const Dims& d) {
  return align256((size_t)paged_wgs_cap(d) * sizeof(uint64_t));
}

inline size_t paged_attn_ws_bytes(const Dims& d, int32_t tokens) {
  return paged_tail_bytes(d) + paged_flag_bytes(d) +
         align256((size_t)paged_wgs_cap(d) * 2 * tokens * d.G * kPartStride * sizeof(float));
}

}  // namespace ckv
