// trr_chunk.cuh - what the kernels of attention of chunks share: the plan, the staged tiles and the
// call's arguments and workspace.
#pragma once

#include "trr_span.cuh"

namespace trr {

// Tokens of a staged tile: as many as let the scores (binary32), the weights (binary16) and the sums of two halves
// of 128 rows have TMEM columns of their own: 2 (T + T / 2 + d) <= 512, T a multiple of 16.
__host__ __device__ constexpr int chunk_tile(int d) { return d == 64 ? 96 : 80; }
constexpr int kHalfRows = 128;       // rows of a softmax warpgroup: lanes of TMEM
constexpr int kBlockRows = 2 * kHalfRows;
constexpr int kPlanChunkThreads = 512;
constexpr int kMostChunkTokens = 1 << 20;

// One chunk.  Its stored tokens that any of its queries sees lie on a line of positions: 0 .. sinks-1,
// then lo .. end-1 (sinks 0: one stretch).  They are staged in order of position, as binary16.
struct ChunkPlan {
  int seq, start, len, row0;    // queries row0 .. row0+len-1 at positions start, start+1, ...
  int sinks, lo, end, span;     // span: positions on the line
  int full, local;              // queries of each mode (valid ones); the rest get zero rows
  int tokens, dropped;          // staged tokens; tokens between sinks and lo
  int tile0, tiles;             // tiles of the pool
  int unit0, units;             // units of 64 positions before this chunk, of it
  int block0, blocks;           // blocks of rows before it, of it
  int head;                     // staged tokens below the call's sinks
  int pad[13];
};
static_assert(sizeof(ChunkPlan) == 128, "");

// A block of rows: queries of one mode of a chunk (in order), their heads of one KV head.  It sees
// the chunk's tiles 0 .. head-1 (sinks) and first .. last-1, of which every row sees the whole of
// clean .. clean_end-1.
struct BlockPlan {
  int chunk, row, rows, local;  // rows row .. of (list of queries of the mode) x (heads of a KV head)
  int head, first, last, tiles;
  int clean, clean_end;
  int query0;                   // the mode's first query in the list
  int tile_cost;
  int tile0, sinks;             // of the chunk: its first tile, staged tokens below the call's sinks
  int pad[2];
};
static_assert(sizeof(BlockPlan) == 64, "");

struct ChunkHeader {
  int64_t work, per;            // cost of all segments, a CTA's share
  int bad;                      // error of the whole call: every row is zero
  int blocks, units;
  int splits, flagged;          // shares of the KV heads that staging CTAs take; some flag is set
  int empty;                    // some block has no tiles
  int moved;                    // what is common to some chunk's tokens is taken out of them
  int pad[5];
};

// A segment that a CTA began and the ctas - 1 after it went on with; block < 0: none.
struct PieceInfo {
  int block, kvh, ctas, rows;
  int chunk, query0, row;         // of the block
  int pad;
};

struct ChunkArgs {
  LayerArgs a;
  int n, num_tokens, window_scalar, sinks, ctas, most_tiles;
  int parts;         // CTAs that look for what a chunk's tokens have in common
  float scale_log2;  // softmax scale times log2(e): exponentials are taken in base 2
  const int32_t *seq_ids, *starts, *offsets, *windows;
  const uint8_t* modes;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  // workspace
  ChunkHeader* head;
  ChunkPlan* chunk;   // [n]
  int32_t* list;      // [num_tokens] a chunk's queries: its full ones in order, then its local ones, then the rest
  int2* sight;        // [num_tokens] which of the chunk's staged tokens the query in that place sees: x .. y-1 (a local
                      // one the first `head` as well, as far as y)
  BlockPlan* block;   // [most_blocks]
  int64_t* base;      // [most_blocks + 1] cost before each block (all its KV heads)
  int32_t* flag;      // [n][Hkv] some stored value is not to be had in binary16: its rows are done one by one
  int32_t* moved;     // [n][K, V][Hkv] keys are staged less their offset, values times powers of two
  uint16_t* common;   // [n][K, V][Hkv][D] the offsets (binary16, 0 in channels that have none), the powers (bf16)
  PieceInfo* piece;   // [ctas] the segment that a CTA began and did not finish
  float2* part_ml;    // [2 * ctas][256] (m, l) of a CTA's first piece, or its last
  uint4* part_o;      // [2 * ctas][D / 4][256] four columns of a row (binary32), consecutive rows beside each other
  uint8_t* tile;      // [most_tiles][Hkv][K, V][T x D] binary16, in the tensor core's layout
};

// A tile's row r holds its 16-byte chunk e at (chunks of 64 columns apart) + 128 r + 16 (e ^ r % 8); `rows` of the tile.
__device__ __forceinline__ int tile_at(int rows, int r, int e) { return (e >> 3) * (rows * 128) + r * 128 + (((e ^ r) & 7) << 4); }
template <int D>
__device__ __forceinline__ uint8_t* staged_tile(const ChunkArgs& g, int tile, int h, int which) {
  return g.tile + ((static_cast<int64_t>(tile) * g.a.Hkv + h) * 2 + which) * (chunk_tile(D) * D * 2);
}

// Columns 4 j .. 4 j + 3 of a row of a piece.
template <int D>
__device__ __forceinline__ uint4* part_at(const ChunkArgs& g, int piece, int j, int row) {
  return g.part_o + (static_cast<int64_t>(piece) * (D / 4) + j) * kBlockRows + row;
}

// Where a row of a block comes from.
struct RowSource {
  int query, head;  // head: of all query heads
  int t, lo;        // it sees tokens at positions <= t that are >= lo (or below the call's sinks, where it is local)
};
__device__ __forceinline__ RowSource row_source(const ChunkArgs& g, const ChunkPlan& c, int query0, bool local, int kvh, int row) {
  const int heads = g.a.Hq / g.a.Hkv;
  RowSource r;
  r.query = g.list[query0 + row / heads];
  r.head = kvh * heads + row % heads;
  r.t = c.start + r.query - c.row0;
  r.lo = local ? r.t - (g.windows ? g.windows[r.query] : g.window_scalar) + 1 : 0;
  return r;
}

// Whether something common was taken out of a chunk's K (which 0) or V of a KV head, and what, by channel.
__device__ __forceinline__ bool moved_head(const ChunkArgs& g, int chunk, int kvh, int which) {
  return g.moved[(2ll * chunk + which) * g.a.Hkv + kvh];
}
template <int D>
__device__ __forceinline__ const uint16_t* common_of(const ChunkArgs& g, int chunk, int kvh, int which) {
  return g.common + ((2ll * chunk + which) * g.a.Hkv + kvh) * D;
}
// One over a power of two that is given as a bf16 number.
__device__ __forceinline__ float one_over(uint32_t power) { return __int_as_float((254 << 23) - static_cast<int>(power << 16)); }

// The last of 0 .. n-1 whose value (they ascend) is x or less, 0 if none is, by a whole warp: a chain of one load for 32 of
// them, two for 1024.
template <typename T, typename Value>
__device__ __forceinline__ int last_not_above(int n, T x, int lane, Value value) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, i = lo + lane * step;
    const int k = __popc(__ballot_sync(0xffffffffu, i < hi && value(i) <= x));
    lo += max(0, k - 1) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// The cost of a segment, in sixteenths of a tile (2000 cycles at d 64): its tiles, those with rows hidden a little dearer
// (2250), and a fixed part for its start and end (4500 to 8000; with 30 sixteenths 4096 queries on themselves took 155 us
// against 144 with 60).  Where the halves take turns (blocks of 128 rows or fewer)
// two tiles take 2600 cycles at d 64, but 4300 at d 128, whose three staged tiles leave neither half one ahead.  With a fixed
// part of one tile and all tiles alike, 4096 queries on themselves, 32 heads of 64, took 202 us against 144, as the CTAs with
// the shortest segments came in last; with turns at the price of whole tiles, ragged chunks of d 64 took 402 us against 378;
// at 10 sixteenths of one at d 128 too, local chunks of 256 to 700 queries and windows of 1024 took 151 us against 130.
constexpr int kChunkTileCost = 16, kChunkTurnsCost = 10, kChunkMaskedCost = 2, kChunkSegmentCost = 60;
constexpr int kChunkLeastShare = 48;  // of a CTA: three tiles
__device__ __forceinline__ int64_t chunk_cost(const BlockPlan& b) {
  return b.tiles > 0 ? kChunkSegmentCost + static_cast<int64_t>(b.tile_cost) * b.tiles : 0;
}
// Whether tile 0 and the last tile of the segment that starts at cost `start` are in one CTA's share: its rows are whole then.
__device__ __forceinline__ bool chunk_uncut(int64_t start, int64_t per, const BlockPlan& b) {
  const int64_t first = start + kChunkSegmentCost;
  return first / per == (first + static_cast<int64_t>(b.tile_cost) * (b.tiles - 1)) / per;
}
// Tiles of a segment that lie before cost x (counted from the segment's start).
__device__ __forceinline__ int chunk_tiles_before(int64_t x, const BlockPlan& b) {
  if (x <= kChunkSegmentCost) return 0;
  const int64_t t = (x - kChunkSegmentCost + b.tile_cost - 1) / b.tile_cost;
  return t < b.tiles ? static_cast<int>(t) : b.tiles;
}

}  // namespace trr
