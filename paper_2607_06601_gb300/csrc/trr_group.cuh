// trr_group.cuh - what the kernels of attention over groups and sinks share: jobs, the call's
// arguments and workspace, and how work is cut into equal runs.
#pragma once

#include "trr_tc.cuh"

namespace trr {

constexpr int kRows = 128;       // rows of a segment: lanes of TMEM
constexpr int kTileKeys = 128;   // most tokens of a tile (64 of 16-bit pages: half the ring per copy)
constexpr int kPlanThreads = 128;

// One job, 32 words.
struct Job {
  int seq, lo, t, sinks;                  // tokens in sight: pos <= t and (pos >= lo or pos < sinks)
  int head[kClasses];                     // pages [0, head) hold the sinks
  int first[kClasses], count[kClasses];   // pages [first, first + count)
  int rows, row_blocks, tiles_q, tiles;   // rows = queries x heads of a KV head; tiles of 2-, 4-, 8-bit pages, of all
                                          // (few rows: tiles is the number of blocks)
  int kind;                               // 0: shared, 1: private
  int qbase;                              // shared: its queries in the list; private: the query
  int joined;                             // private: the query has a shared job as well
  int tokens[kClasses];                   // of its sequence
  int pad[5];
};
static_assert(sizeof(Job) == 128, "a warp loads a job one word per lane");

// One query, as the join needs it.
struct QueryPlan {
  int reads;                              // 0: its rows are in place
  int group, rank, shared;                // its group's shared job, its place among that job's queries, whether it is one of them
  int common[kClasses];                   // leading pages that it shares with its group's first full query and sees whole
};
static_assert(sizeof(QueryPlan) == 32, "two 16-byte loads");

struct GroupHeader {
  int64_t work, per;          // cost of the tensor kernel's segments, a CTA's share
  int64_t few_work, few_per;  // cost of the segments of few rows, a warp's share
};

struct GroupArgs {
  LayerArgs a;
  int n, window_scalar, sinks, groups, ctas;
  int few, few_warps;         // most rows of a segment of the kernel for few rows (0: too many even for one query), its warps
  int overlap;                // the kernel for few rows follows the tensor kernel and may run beside it
  float scale_log2;  // softmax scale times log2(e): exponentials are taken in base 2
  const int32_t *seq_ids, *positions, *windows, *offsets;
  const uint8_t* modes;
  const uint16_t* q;
  uint16_t* out;
  // workspace
  GroupHeader* head;
  QueryPlan* plan;
  int32_t* list;      // [n] a group's rows: its full queries in order, from the group's offset on
  Job* jobs;          // [groups] shared, then [n] private
  int32_t* tiles;     // [jobs] tiles of a job of the tensor kernel, else 0; minus the error of a query in error
  int32_t* blocks;    // [jobs] blocks of a job of the kernel for few rows, else 0
  int64_t* base;      // [jobs + 1] cost before each job of the tensor kernel
  float2* home_ml;    // [2][n][Hq] (m, l) of a row of a whole segment, by kind of job
  float* home_o;      // [2][n][Hq][D]
  float2* part_ml;    // [2 * ctas][128] of a piece of a segment, copies of its rows included: a CTA's first one, or its last
  float* part_o;
  int64_t* few_base;  // [jobs + 1] cost before each job of the kernel for few rows
  float2* few_ml;     // [2 * few_warps][8] of a warp's first piece, or its last
  float* few_o;
};

// The cost of a segment: tiles, and a fixed part for its start and end.
constexpr int kTileCost = 2, kSegmentCost = 2;
__device__ __forceinline__ int64_t segment_cost(int tiles) { return kSegmentCost + static_cast<int64_t>(kTileCost) * tiles; }
// Tiles of a segment that lie before cost x (counted from the segment's start).
__device__ __forceinline__ int tiles_before(int64_t x, int tiles) {
  if (x <= kSegmentCost) return 0;
  const int64_t t = (x - kSegmentCost + kTileCost - 1) / kTileCost;
  return t < tiles ? static_cast<int>(t) : tiles;
}

// Copies of a segment's rows that fill the tensor kernel's 128 lanes.
__device__ __forceinline__ int copies_of(int rows) { return rows <= 32 ? 4 : rows <= 64 ? 2 : 1; }

// A CTA's share is two tiles at least: a CTA takes 10 us to its first scores and from its last ones,
// and those left without a tile serve the private segments meanwhile.
constexpr int kLeastShare = kSegmentCost / 2 + 2 * kTileCost;

// Blocks of a warp's run of few rows that are done beside the tensor kernel's shortest share, and beside
// one of kLongShare.  Measured, when the rule came in, on the SMs that the tensor kernel leaves against all
// of them after it: 32 queries on 2048 + 64 tokens of 12 KV heads of 64, 27 us against 33; 16 queries on
// 65536 + 256 tokens of 8 KV heads of 128, 67.7 against 73.0 (eight SMs left to them), on 32768 + 256, 51.9
// against 53.2.  64 such queries would need 32 SMs, and the tensor kernel would lose more than they gain.
// A block is taken for as long as another whatever its width and d, which is rough.
constexpr int kShortShare = 6, kFewShare = 12, kLongShare = 20;

// The same for the kernel for few rows, in blocks.
constexpr int kFewSegmentCost = 1;
__device__ __forceinline__ int64_t few_cost(int blocks) { return kFewSegmentCost + blocks; }
__device__ __forceinline__ int few_before(int64_t x, int blocks) {
  return x <= kFewSegmentCost ? 0 : x - kFewSegmentCost < blocks ? static_cast<int>(x - kFewSegmentCost) : blocks;
}

__device__ __forceinline__ __half2 as_half2(uint32_t w) { return *reinterpret_cast<__half2*>(&w); }
__device__ __forceinline__ uint32_t as_u32(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }

// A whole sector in one store (p aligned to 32 bytes).
__device__ __forceinline__ void st_global8(float* p, const float* v) {
  asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]),
               "f"(v[6]), "f"(v[7])
               : "memory");
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

}  // namespace trr
