// ckv_blocks.hpp -- launch arguments and launchers of the attention over selected
// blocks (ckv_blocks.hip), and what their host side shares.
#pragma once

#include "ckv_paged.hpp"

namespace ckv {

constexpr int kMaxKept = 64;      // blocks a query keeps at most
constexpr int kMarkCols = 64;     // landmarks of a scoring workgroup's least chunk
constexpr int kMaxPieces = 64;    // pieces of a tile's list

// Query tokens of a call: token t is position pos[t] of request req[t] (NULL: of
// request t).  A tile is 16 query rows: 16 / G tokens with the G heads of one KV head.
struct BlockTokens {
  const int32_t* req;
  const int32_t* pos;
  const uint16_t* q;       // [N][Hq][d]
  int32_t n, B, Hkv, Hq, lg, max_ctx;
  int32_t lb, nb, k;       // log2 of the block, blocks of max_ctx, blocks kept
};

struct MarkArgs {
  PagedPages pg;
  const int32_t* ctx_lens;
  const int32_t* first;    // [B] or NULL
  uint16_t* marks;         // [B][Hkv][nb][d]
  int32_t B, max_ctx, lb, nb;
  int32_t slices;          // workgroups a unit
};

struct BlockSelectArgs {
  PagedPages pg;
  BlockTokens t;
  const uint16_t* marks;
  int32_t* idx;            // [N][Hkv][k]
  float* scores;           // [N][Hkv][nb], of earlier blocks
  float* norms;            // [tiles][Hkv][chunks]: largest |landmark|^2 of a workgroup
  int32_t row_tiles;       // tiles of a scoring workgroup (1 or 4)
  int32_t cols, chunks;    // its landmarks, workgroups over nb
};

struct BlockAttnArgs {
  PagedPages pg;
  BlockTokens t;
  const int32_t* idx;      // [N][Hkv][k]
  float* out;              // [N][Hq][d]
  float* lse;              // [N][Hq] or NULL
  float* part;             // [tiles][Hkv][pieces][16][kPartStride]
  float scale;
  int32_t pieces;
  int32_t many;            // 64 query rows a workgroup, blocks staged for its waves
};

// Debug mode's check of the lists that an attention is given.
struct BlockListArgs {
  BlockTokens t;
  const int32_t* idx;      // [N][Hkv][k]
  unsigned long long* flag;
};

// Whether the blocks that count of list i (token i / Hkv, head i % Hkv) ascend.
__host__ __device__ inline bool block_list_ascends(const BlockListArgs& a, int64_t i) {
  const int64_t tok = i / a.t.Hkv;
  const int own = a.t.pos[tok] >> a.t.lb;  // -1 (padding): none counts
  int last = -1;
  for (int e = 0; e < a.t.k; ++e) {
    const int j = a.idx[i * a.t.k + e];
    if (j < 0 || j > own) continue;
    if (j < last) return false;
    last = j;
  }
  return true;
}

inline int64_t tiles_of(const BlockTokens& t, int row_tiles = 1) {
  const int per = (16 >> t.lg) * row_tiles;
  return (t.n + per - 1) / per;
}

constexpr int kManyTiles = 4;  // tiles of a workgroup that stages blocks

hipError_t launch_marks(const MarkArgs& a, Kind kind, hipStream_t s);
hipError_t launch_select_blocks(const BlockSelectArgs& a, hipStream_t s);
hipError_t launch_block_attn(const BlockAttnArgs& a, Kind kind, hipStream_t s);
hipError_t launch_check_lists(const BlockListArgs& a, hipStream_t s);

}  // namespace ckv
