// trr_chunk_tc.cuh - attention of blocks of 256 rows over staged tiles, on the tensor cores (tcgen05).
//
//   S = Q K^T,  p = 2^(f S - m),  l += sum p,  O += P V,  and at a row's end O / l or the piece (m, l, O).
//
// One CTA per SM.  A producer warp brings tiles of tokens (K and V) into rings of shared memory, as they were
// staged, with bulk copies.  A block's rows are two halves of 128, a lane of TMEM each; a half has a warp that
// issues its products and a warpgroup that does its softmax, a thread a row.  A block of 128 rows or fewer has its
// rows in both halves, which take its tiles in turn and are joined at the end.  K, V and p are binary16 (11 bits;
// the output has 8), sums and statistics binary32; query rows are scaled by powers of two.
//
// What bounds it.  Per tile of 96 tokens at d 64 the two halves' products take 464 + 384 cycles of the tensor core
// and its shared memory, 24,576 exponentials 768 of the SM's 32 a cycle, and a softmax warp's chain of waits,
// loads from TMEM, weights and stores about 1900, which is what a tile takes: at 4096 queries on themselves, 32
// heads of 64 (four fifths of the tokens stored), 98 to 101 us, 0.55 PFLOP/s, the tensor pipe busy for 25 % of it.  At d 128
// a product of 128 x 80 x 16 from shared memory takes 54 cycles of its bandwidth, 1506 a tile with those of P V;
// measured 1930: 2048 queries of 32 heads at the end of 32,768 tokens, 555 us, 1.54 PFLOP/s, the tensor pipe busy for 65 %.
// (The kernel at d 64 spills 20 bytes a thread of stores and 24 of loads.)
//
// What this layout is for: from a product's end to the issue of one that waits for it pass about 450 cycles
// (completion, barrier, wait, issue).  So no product waits for another: scores, weights and sums have columns of
// their own, and a tile's scores are issued as soon as the last ones have been read.  That gives tiles of 96 and of
// 80 tokens (TMEM has 512 columns).  With 128 tokens at d 128, weights over scores, the call above took 860 us; with
// 128 at d 64, whose scores do not fit a thread's registers, ragged chunks 412 against 397.
#pragma once

#include "trr_chunk.cuh"

namespace trr {

constexpr int kChunkSoftmaxWarps = 8, kChunkProducer = 8, kChunkMma = 9, kChunkFinder = 11;  // products: warps 9 and 10
constexpr int kChunkThreads = 384;
// Registers a thread: 168 at launch; the softmax warpgroups take what the third gives up.
constexpr int kChunkLaunchRegisters = 168, kChunkSoftmaxRegisters = 208, kChunkOtherRegisters = 88;
static_assert(256 * kChunkSoftmaxRegisters + 128 * kChunkOtherRegisters <= kChunkThreads * kChunkLaunchRegisters, "");
constexpr int kRunSlots = 4;

// A run of tiles for one block and KV head, as the softmax warps and the product warps need it.
struct ChunkSegment {
  int tiles;              // 0: no more
  int block, kvh, rows;   // 128 rows or fewer: in both halves, which take the tiles in turn
  int dest;               // -1: the output rows, else the slot of the piece
  int clean, clean_end;   // tiles of the run that every row sees whole
  int from, head, skip;   // the run's first tile of the segment's; the segment's first `head` are the chunk's, the others `skip` further
  int query0, row, local; // of the block
  int sinks;              // staged tokens that a local row sees beside its window
  int pad[2];
};

// A row of a run: its place among all (query, head), and which of the chunk's staged tokens it sees, lo .. hi - 1.
struct ChunkRow {
  int at, lo, hi;  // at < 0: no row
};

template <int D>
struct ChunkSmem {
  static constexpr int kT = chunk_tile(D);
  static constexpr int kQ = kHalfRows * D * 2;      // bytes of Q of a half
  static constexpr int kTile = kT * D * 2;          // bytes of K or V of a tile
  static constexpr int kSlots = D == 64 ? 6 : 3;    // of K, and of V
  static constexpr int kK = 2 * kQ;                 // behind Q
  static constexpr int kV = kK + kSlots * kTile;
  static constexpr int kExchange = kV + kSlots * kTile;  // 32 columns of the second half's rows, and (m, l), for a join
  static constexpr int kMl = kExchange + 32 * kHalfRows * 4;
  static constexpr int kRows = kMl + kHalfRows * 8;
  static constexpr int kSeg = kRows + kRunSlots * kBlockRows * static_cast<int>(sizeof(ChunkRow));
  static constexpr int kBars = kSeg + kRunSlots * static_cast<int>(sizeof(ChunkSegment));
  static constexpr int kNumBars = 2 * kSlots + 3 * kRunSlots + 2 * 6 + 2;
  static constexpr int kAbort = kBars + 8 * kNumBars;
  static constexpr int kTotal = kAbort + 8;
  static_assert(kTotal + 1024 + 64 <= 227 * 1024, "");
  static_assert(kTile % 1024 == 0, "");
};

template <int D>
struct ChunkCtx {
  using L = ChunkSmem<D>;
  static constexpr int kT = L::kT;
  static constexpr int kPartA = D == 64 ? 64 : 48, kPartB = kT - kPartA;  // a thread's scores, as two arrays
  uint8_t* base;  // 1024-byte aligned
  uint32_t tmem;
  const ChunkArgs* args;  // (the kernel's own: read from there, not kept in registers)
  __device__ volatile int* abort_flag() const { return reinterpret_cast<volatile int*>(base + L::kAbort); }
  __device__ volatile int* copied() const { return reinterpret_cast<volatile int*>(base + L::kAbort + 4); }  // tiles that the producer has asked for
  __device__ uint64_t* bar(int i) const { return reinterpret_cast<uint64_t*>(base + L::kBars) + i; }
  __device__ uint64_t* kv_full(int i) const { return bar(i); }
  __device__ uint64_t* kv_empty(int i) const { return bar(L::kSlots + i); }
  __device__ uint64_t* seg_full(int i) const { return bar(2 * L::kSlots + i); }
  __device__ uint64_t* seg_empty(int i) const { return bar(2 * L::kSlots + kRunSlots + i); }
  __device__ uint64_t* rows_full(int i) const { return bar(2 * L::kSlots + 2 * kRunSlots + i); }
  __device__ uint64_t* half_bar(int half, int i) const { return bar(2 * L::kSlots + 3 * kRunSlots + 6 * half + i); }
  __device__ uint64_t* q_full(int half) const { return half_bar(half, 0); }
  __device__ uint64_t* s_full(int half) const { return half_bar(half, 1); }
  __device__ uint64_t* s_read(int half) const { return half_bar(half, 2); }
  __device__ uint64_t* p_full(int half) const { return half_bar(half, 3); }
  __device__ uint64_t* o_done(int half) const { return half_bar(half, 4); }
  __device__ uint64_t* drained(int half) const { return half_bar(half, 5); }
  __device__ uint64_t* join_full() const { return half_bar(2, 0); }
  __device__ uint64_t* join_empty() const { return half_bar(2, 1); }
  __device__ ChunkSegment& seg(int i) const { return reinterpret_cast<ChunkSegment*>(base + L::kSeg)[i]; }
  __device__ ChunkRow* rows(int i) const { return reinterpret_cast<ChunkRow*>(base + L::kRows) + i * kBlockRows; }
  // TMEM columns: scores, weights (two to a column), sums
  __device__ uint32_t col_s(int half) const { return tmem + kT * half; }
  __device__ uint32_t col_p(int half) const { return tmem + (D == 64 ? 192 : 160) + 48 * half; }
  __device__ uint32_t col_o(int half) const { return tmem + 512 - D * (2 - half); }
  __device__ __forceinline__ bool there(uint64_t* b, uint32_t parity) const { return mbar_test_at(smem_u32(b), parity); }
  // A bounded wait by a whole warp; all of its lanes get the same answer.  Once one has given up, none waits any
  // more.  (Short, since a warp among others' code pays for the fetch of every instruction.)
  __device__ __forceinline__ bool wait(uint64_t* b, uint32_t parity) const {
    const uint32_t addr = smem_u32(b);
    for (uint64_t t0 = 0; !__all_sync(0xffffffffu, mbar_poll(addr, parity, args->a.wait_ns));) {
      const uint64_t now = global_ns();
      if (t0 == 0) t0 = now;
      if (__any_sync(0xffffffffu, *abort_flag() || now - t0 >= args->a.wait_ns)) {
        *abort_flag() = 1;
        return false;
      }
    }
    return true;
  }
  // The same for what comes behind the copies of all of a run's tiles, however many: the bound is on the time between two.
  __device__ __forceinline__ bool wait_behind_copies(uint64_t* b, uint32_t parity) const {
    const uint32_t addr = smem_u32(b);
    uint64_t t0 = 0;
    for (int before = -1; !__all_sync(0xffffffffu, mbar_poll(addr, parity, args->a.wait_ns));) {
      const uint64_t now = global_ns();
      const int tiles = *copied();
      if (tiles != before) t0 = now, before = tiles;
      if (__any_sync(0xffffffffu, *abort_flag() || now - t0 >= args->a.wait_ns)) {
        *abort_flag() = 1;
        return false;
      }
    }
    return true;
  }
};

// The producer warp: the runs of this CTA's share, and the copies of their tiles.
template <int D>
__device__ __forceinline__ void chunk_produce(const ChunkArgs& g, const ChunkCtx<D>& x, int lane) {
  using L = ChunkSmem<D>;
  const int64_t per = g.head->per, work = g.head->work;
  const int blocks = g.head->blocks;
  const int64_t b0 = min(work, blockIdx.x * per), b1 = min(work, b0 + per);
  int segs = 0, copies = 0;
  bool ok = true;
  PieceInfo piece = {-1};
  int64_t piece_end = 0;  // cost before its segment's last tile
  auto announce = [&](const ChunkSegment& s) {
    ok = ok && x.wait(x.seg_empty(segs % kRunSlots), ((segs / kRunSlots) & 1) ^ 1);
    if (!ok) return;
    if (lane == 0) {
      x.seg(segs % kRunSlots) = s;
      mbar_arrive(x.seg_full(segs % kRunSlots));
    }
    ++segs;
  };
  // A run is announced before the tiles of the one before it are copied, so that its rows can be fetched in good time.
  ChunkSegment last = {};
  int last_tile0 = 0;
  auto copy = [&]() {
    for (int i = 0; i < last.tiles && ok; ++i, ++copies) {
      const int at = last.from + i, tile = last_tile0 + at + (at < last.head ? 0 : last.skip), slot = copies % L::kSlots;
      ok = x.wait(x.kv_empty(slot), ((copies / L::kSlots) & 1) ^ 1);
      if (!ok) break;
      if (lane == 0) {
        mbar_arrive_expect_tx(x.kv_full(slot), 2 * L::kTile);
        bulk_g2s(x.base + L::kK + slot * L::kTile, staged_tile<D>(g, tile, last.kvh, 0), L::kTile, x.kv_full(slot));
        bulk_g2s(x.base + L::kV + slot * L::kTile, staged_tile<D>(g, tile, last.kvh, 1), L::kTile, x.kv_full(slot));
        *x.copied() = copies + 1;
      }
    }
  };
  if (b0 < b1) {
    fence_proxy_async_global();  // the tiles were staged with ordinary stores
    // the block that holds cost b0: the last one that starts at or before it
    const int lo = last_not_above(blocks, b0, lane, [&](int i) { return g.base[i]; });
    for (int b = lo; b < blocks && ok; ++b) {
      const BlockPlan p = g.block[b];
      const int64_t start = g.base[b];
      if (start >= b1) break;
      if (p.tiles == 0) continue;
      const int64_t cost = chunk_cost(p);
      for (int h = static_cast<int>(max(static_cast<int64_t>(0), (b0 - start) / cost)); h < g.a.Hkv && ok; ++h) {
        const int64_t S = start + h * cost;
        if (S >= b1) break;
        const int t0 = chunk_tiles_before(b0 - S, p), t1 = chunk_tiles_before(b1 - S, p);
        if (t0 >= t1) continue;
        if (t0 == 0 && t1 < p.tiles) {
          piece = PieceInfo{b, h, 0, p.rows, p.chunk, p.query0, p.row};
          piece_end = S + cost - p.tile_cost;
        }
        ChunkSegment s = {};
        s.tiles = t1 - t0; s.block = b; s.kvh = h; s.rows = p.rows;
        s.dest = t0 == 0 && t1 == p.tiles ? -1 : 2 * static_cast<int>(blockIdx.x) + (t0 > 0 ? 0 : 1);
        s.from = t0; s.head = p.head; s.skip = p.first - p.head;
        s.clean = max(p.clean, p.first) - s.skip - t0;
        s.clean_end = p.clean_end - s.skip - t0;
        s.query0 = p.query0; s.row = p.row; s.local = p.local; s.sinks = p.sinks;
        announce(s);
        copy();
        last = s;
        last_tile0 = p.tile0;
      }
    }
  }
  // the last tile is that of the last CTA whose share begins before it or there
  if (piece.block >= 0) piece.ctas = static_cast<int>(min(static_cast<int64_t>(g.ctas), piece_end / per + 1)) - static_cast<int>(blockIdx.x);
  if (lane == 0) g.piece[blockIdx.x] = piece;
  announce(ChunkSegment{});  // no more
  copy();
  // the CTA stays until its copies have landed
  for (int k = max(0, copies - L::kSlots); k < copies; ++k) mbar_wait(x.kv_full(k % L::kSlots), (k / L::kSlots) & 1);
}

// The warp that finds the rows of each run as it is announced, and brings their queries to L1: two chains of loads that
// the softmax warps would wait for.
template <int D>
__device__ __forceinline__ void chunk_find_rows(const ChunkArgs& g, const ChunkCtx<D>& x, int lane) {
  const int heads = g.a.Hq / g.a.Hkv;
  for (int segs = 0;; ++segs) {
    const int slot = segs % kRunSlots;
    if (!x.wait_behind_copies(x.seg_full(slot), (segs / kRunSlots) & 1)) return;  // (a run ahead of the others)
    const ChunkSegment& s = x.seg(slot);
    const int rows = s.rows, tiles = s.tiles, query0 = s.query0, row0 = s.row, head0 = s.kvh * heads;
    if (tiles == 0) return;
#pragma unroll 4
    for (int r = lane; r < kBlockRows; r += 32) {
      ChunkRow row = {-1, 0, INT_MAX};  // (a lane without a row sees every token)
      if (r < rows) {
        const int k = query0 + (row0 + r) / heads;
        const int2 sight = g.sight[k];
        row = ChunkRow{g.list[k] * g.a.Hq + head0 + (row0 + r) % heads, sight.x, sight.y};
        const uint16_t* q = g.q + static_cast<int64_t>(row.at) * D;
        asm volatile("prefetch.global.L1 [%0];" ::"l"(q));
        if (D == 128) asm volatile("prefetch.global.L1 [%0];" ::"l"(q + 64));
      }
      x.rows(slot)[r] = row;
    }
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(x.rows_full(slot));
      mbar_arrive(x.seg_empty(slot));
    }
  }
}

// The warp that issues a half's products (one elected lane does; the whole warp goes along): the next scores
// once these have been read, then O += P V once the weights are there.  Each half has its own: a wait costs 200
// cycles, even for what is there, among warps that move scores and weights.
template <int D>
__device__ __forceinline__ void chunk_mma(const ChunkCtx<D>& x, int half) {
  using L = ChunkSmem<D>;
  constexpr int T = L::kT;
  int segs = 0, done = 0, it = 0, loads = 0;  // done: tiles of the CTA, it: of this half, loads: of Q
  const uint32_t base = smem_u32(x.base), col_s = x.col_s(half), col_p = x.col_p(half), col_o = x.col_o(half);
  const uint32_t id_s = tc_idesc(false, T, false), id_o = tc_idesc(false, D, true);
  const uint64_t q = tc_desc(base + half * L::kQ, 16);
  for (bool ok = true; ok;) {
    if (!x.wait(x.seg_full(segs % kRunSlots), (segs / kRunSlots) & 1)) break;
    const ChunkSegment& sg = x.seg(segs % kRunSlots);
    const int n = __shfl_sync(0xffffffffu, sg.tiles, 0);
    const bool turns = __shfl_sync(0xffffffffu, sg.rows, 0) <= kHalfRows;  // the halves take the tiles in turn
    __syncwarp();
    if (elected()) mbar_arrive(x.seg_empty(segs % kRunSlots));
    ++segs;
    if (n == 0) break;
    const int step = turns ? 2 : 1, first = turns ? half : 0;
    auto tile_there = [&](int i) { return x.there(x.kv_full((done + i) % L::kSlots), ((done + i) / L::kSlots) & 1); };
    auto scores = [&](int i, bool there) -> bool {  // S of the run's tile i
      const int slot = (done + i) % L::kSlots;
      if (!there && !x.wait(x.kv_full(slot), ((done + i) / L::kSlots) & 1)) return false;
      tc_fence_after();
      if (elected()) {
        const uint64_t k = tc_desc(base + L::kK + slot * L::kTile, 16);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          const int at = (j >> 2) * 8, in = 2 * (j & 3);
          tc_mma_ss(col_s, q + (at * kHalfRows + in), k + (at * T + in), id_s, j > 0);
        }
        tc_commit(x.s_full(half));
      }
      __syncwarp();
      return true;
    };
    // A tile of the other half's: seen to come and let go, so that each of a slot's phases has been waited for in order
    // (a parity alone does not tell a phase from the one before the last) and none is over before both have seen it.
    auto pass = [&](int i) -> bool {
      const int slot = (done + i) % L::kSlots;
      if (!x.wait(x.kv_full(slot), ((done + i) / L::kSlots) & 1)) return false;
      if (elected()) mbar_arrive(x.kv_empty(slot));
      __syncwarp();
      return true;
    };
    if (first == 1) ok = pass(0);
    if (first < n) ok = ok && x.wait(x.q_full(half), loads++ & 1) && scores(first, false);
#pragma unroll 1
    for (int i = first; i < n && ok; i += step, ++it) {
      // asked together: three answers take little longer than one
      bool read = x.there(x.s_read(half), it & 1), tile = tile_there(i + step), weights = x.there(x.p_full(half), it & 1);
      read = __all_sync(0xffffffffu, read);
      tile = __all_sync(0xffffffffu, tile);
      weights = __all_sync(0xffffffffu, weights);
      if (turns && i + 1 < n) ok = pass(i + 1);
      if (i + step < n) ok = ok && (read || x.wait(x.s_read(half), it & 1)) && scores(i + step, tile);
      if (!ok || !(ok = weights || x.wait(x.p_full(half), it & 1))) break;
      tc_fence_after();
      if (elected()) {
        const int slot = (done + i) % L::kSlots;
        const uint64_t v = tc_desc(base + L::kV + slot * L::kTile, T * 128);
#pragma unroll
        for (int k = 0; k < T / 16; ++k) tc_mma(col_o, col_p + 8 * k, v + k * (2048 >> 4), id_o, k > 0 || i > first);
        tc_commit(x.kv_empty(slot));
        tc_commit(x.o_done(half));
      }
      __syncwarp();
    }
    done += n;
  }
  if (elected()) tc_commit(x.drained(half));  // nothing is in flight when the CTA ends
  __syncwarp();
  mbar_wait(x.drained(half), 0);
}

// The 32 of bits 0 .. n-1 that lie in word w.
__device__ __forceinline__ uint32_t bits_below(int n, int w) {
  const int k = n - 32 * w;
  return k <= 0 ? 0u : k >= 32 ? 0xffffffffu : (1u << k) - 1;
}

// Scores out of sight become -infinity; s holds tokens FROM .. FROM + N - 1, bit j of the words is token j's.  Sixteen
// at a time, where a row of the warp does not see them all.
template <int FROM, int N, int W>
__device__ __forceinline__ void hide(uint32_t (&s)[N], const uint32_t (&seen)[W]) {
#pragma unroll
  for (int j0 = 0; j0 < N; j0 += 16) {
    const uint32_t bits = seen[(FROM + j0) / 32] >> ((FROM + j0) % 32) & 0xFFFFu;
    if (__all_sync(0xffffffffu, bits == 0xFFFFu)) continue;
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (!(bits >> j & 1)) s[j0 + j] = 0xFF800000u;
  }
}

// Weights 2^(s f + shift) of a thread's scores as binary16, two to a word; returns their sum (in binary32).
template <int N>
__device__ __forceinline__ float weights_of(const uint32_t (&s)[N], uint32_t (&p)[N / 2], float f, float shift) {
  uint64_t sum[2] = {0, 0}, ff, hh;
  asm("mov.b64 %0, {%1, %1};" : "=l"(ff) : "f"(f));
  asm("mov.b64 %0, {%1, %1};" : "=l"(hh) : "f"(shift));
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    uint64_t x;
    float x0, x1;
    asm("{\n .reg .b64 t;\n mov.b64 t, {%1, %2};\n fma.rn.f32x2 %0, t, %3, %4;\n}" : "=l"(x) : "r"(s[i]), "r"(s[i + 1]), "l"(ff), "l"(hh));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x0), "=f"(x1) : "l"(x));
    x0 = exp2_approx(x0);
    x1 = exp2_approx(x1);
    asm("{\n .reg .b64 t;\n mov.b64 t, {%1, %2};\n add.rn.f32x2 %0, %0, t;\n}" : "+l"(sum[i / 2 % 2]) : "f"(x0), "f"(x1));
    p[i / 2] = pack16(false, x0, x1);
  }
  float a, b, c, d;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(sum[0]));
  asm("mov.b64 {%0, %1}, %2;" : "=f"(c), "=f"(d) : "l"(sum[1]));
  return (a + b) + (c + d);
}

// Words into TMEM, in as few stores as may be.
template <int N, int FROM = 0>
__device__ __forceinline__ void put_words(uint32_t col, const uint32_t (&p)[N]) {
  constexpr int W = N - FROM >= 32 ? 32 : N - FROM >= 16 ? 16 : 8;
  uint32_t x[W];
#pragma unroll
  for (int k = 0; k < W; ++k) x[k] = p[FROM + k];
  tmem_st(col + FROM, x);
  if constexpr (FROM + W < N) put_words<N, FROM + W>(col, p);
}

// v[j] of lane 4 g + i becomes v[i] of lane 4 g + j.
__device__ __forceinline__ void turn4(uint32_t (&v)[4][4], int lane) {
#pragma unroll
  for (int s = 1; s < 4; s <<= 1) {
    const bool up = lane & s;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k & s) continue;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t a = v[k][u], b = v[k | s][u], got = __shfl_xor_sync(0xffffffffu, up ? a : b, s);
        v[k][u] = up ? got : a;
        v[k | s][u] = up ? b : got;
      }
    }
  }
}

// The softmax warps of a half, a thread a row.
//
// A row's reference m only has to keep its weights within binary16, and one from its first tile's maximum does for most
// of the tiles that follow: their weights are taken by it at once, without a maximum of their own, and their sum tells
// whether the reference has to move.  Up, where the sum passes binary16's largest value.  Down, where it shows weights that
// binary16, whose steps end at 2^-24, is too coarse for: less than 2^-14 for each token in sight, or for each but the largest
// in the first tile.  (Sums are binary32, so they may grow where the reference falls, by 2^60 at a time and not past 2^100.)
// So a weight is off by 2^-11 of itself or of its tile's mean weight, however much a token elsewhere draws of the row.  With
// the first maximum as the reference for good, a first token of V = 0 left rows 44 % off whose other tokens lay 17 nats below.
//   The first reference stands 2^3 below the maximum, for other tokens of its tile than one that draws most of it.  At 2^8
// below and with no way down references moved more often: ragged chunks took 409 us (384 so, 377 with the maximum for good),
// 2048 queries at the end of 32,768 tokens 685 (654, 645).
template <int D>
__device__ __forceinline__ void chunk_softmax(const ChunkArgs& g, const ChunkCtx<D>& x, int half, int quad, int lane) {
  using L = ChunkSmem<D>;
  using C = ChunkCtx<D>;
  constexpr int T = L::kT, A = C::kPartA, B = C::kPartB;
  constexpr float kMost = 65504.f, kSmall = 0x1p-14f;         // binary16's largest, and smallest of 11 bits
  constexpr float kRoom = 3.f, kFirst = 8.f ;                 // a first reference's distance from the largest weight; that weight
  constexpr float kRoomUp = 8.f, kRoomAlone = 15.f;           // of one moved up; of one whose largest weight stands alone
  constexpr float kDown = 60.f, kGrown = 0x1p40f;             // a reference falls by so much at most, and no more once the row's sum is so large
  static_assert(T * 256 < 65504, "");
  const int row = quad * 32 + lane;
  const uint32_t lanes = static_cast<uint32_t>(quad) << 21;  // the warp's 32 lanes of TMEM
  const uint32_t col_s = x.col_s(half) + lanes, col_p = x.col_p(half) + lanes, col_o = x.col_o(half) + lanes;
  int it = 0, joins = 0;
  float f = 0.f;
  // The rows of run k into shared memory, if the half has a tile of it, as binary16 and scaled by the power of two that
  // brings a row's largest element to [2^14, 2^15), so that elements down to 2^-28 of it keep their bits; the factor from
  // products to base-2 exponents.  Whole lines at a time, as rows are stored: with a row a lane, 32 lines an access, a
  // run's end took 5500 cycles at d 64 and up to 10,000 at 128; now 4500 and 7000.
  auto load_rows = [&](int k) -> bool {
    const int slot = k % kRunSlots;
    if (!x.wait(x.seg_full(slot), (k / kRunSlots) & 1)) return false;
    const bool turns = x.seg(slot).rows <= kHalfRows;
    if (x.seg(slot).tiles <= (turns ? half : 0)) return true;
    if (!x.wait(x.rows_full(slot), (k / kRunSlots) & 1)) return false;
    const int at = x.rows(slot)[(turns ? 0 : half * kHalfRows) + row].at;
    // 16 bytes a lane, consecutive lanes along a row
    constexpr int kLanes = D / 8, kRows = 32 / kLanes;
    const int sub = lane / kLanes, chunk = lane % kLanes;
    uint4 w[kLanes];
#pragma unroll
    for (int i = 0; i < kLanes; ++i) {
      const int from = __shfl_sync(0xffffffffu, at, i * kRows + sub);
      w[i] = from >= 0 ? reinterpret_cast<const uint4*>(g.q + static_cast<int64_t>(from) * D)[chunk] : make_uint4(0, 0, 0, 0);
    }
    int e = 0;
#pragma unroll
    for (int i = 0; i < kLanes; ++i) {
      const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
      uint32_t o[4], top = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) top = __vmaxu2(top, v[k] & 0x7FFF7FFFu);
      top = max(top & 0xFFFFu, top >> 16);
#pragma unroll
      for (int d = 1; d < kLanes; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
      const int of_row = top == 0 || top >= 0x7F80u ? 0 : max(-114, static_cast<int>(top >> 7) - (127 + 14));
      const float down = __int_as_float((127 - of_row) << 23);
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = pack16(false, bf16lo(v[k]) * down, bf16hi(v[k]) * down);
      *reinterpret_cast<uint4*>(x.base + half * L::kQ + tile_at(kHalfRows, quad * 32 + i * kRows + sub, chunk)) = make_uint4(o[0], o[1], o[2], o[3]);
      const int mine = __shfl_sync(0xffffffffu, of_row, lane % kRows * kLanes);
      if (lane / kRows == i) e = mine;
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(x.q_full(half));
    f = fmaxf(g.scale_log2 * __int_as_float((127 + e) << 23), 1.17549435e-38f);
    return true;
  };

  // (from -1: one place in the code brings rows, the first ones too, since what runs for the first time is waited for)
#pragma unroll 1
  for (int segs = -1;; ++segs) {
    const bool begun = segs >= 0;
    const ChunkSegment& sg = x.seg(begun ? segs % kRunSlots : 0);
    const int tiles = begun ? sg.tiles : 0, clean = sg.clean, clean_end = sg.clean_end;
    if (begun && tiles == 0) return;
    const int step = begun && sg.rows <= kHalfRows ? 2 : 1, first = (step - 1) * half;  // 2: the halves have the same rows and take the tiles in turn
    float m = -INFINITY, l = 0.f;
    bool ready = false;    // the next scores are there
    bool settled = false;  // every row of the warp has a reference
    for (int i = first; i < tiles; i += step, ++it) {
      if (!ready && !x.wait(x.s_full(half), it & 1)) return;
      tc_fence_after();
      const bool used = it == 0 || x.there(x.o_done(half), (it - 1) & 1);
      uint32_t a[A], b[B];
      tmem_ld(a, b, col_s);
      tc_fence_before();
      if (lane == 0) mbar_arrive(x.s_read(half));  // the next scores may come (the load was the whole warp's: no need to meet first)
      float least = T * kSmall;  // of the weights' sum
      if (i < clean || i >= clean_end) {  // not every row sees the whole tile
        const int s = sg.from + i, before = (s + (s < sg.head ? 0 : sg.skip)) * T;
        const ChunkRow r = x.rows(segs % kRunSlots)[(2 - step) * half * kHalfRows + row];
        const int hi = min(T, r.hi - before), lo = r.lo - before, sinks = sg.local ? sg.sinks - before : 0;
        uint32_t seen[(T + 31) / 32];
        int any = 0;
#pragma unroll
        for (int w = 0; w < (T + 31) / 32; ++w) {
          seen[w] = bits_below(hi, w) & (~bits_below(lo, w) | bits_below(sinks, w));
          any += __popc(seen[w]);
        }
        if (!__any_sync(0xffffffffu, any)) {  // none of the warp's rows sees any of it
          if (it > 0 && !x.wait(x.o_done(half), (it - 1) & 1)) return;
          const uint32_t none[T / 2] = {};
          put_words(col_p, none);
          tmem_wait_st();
          tc_fence_before();
          if (lane == 0) mbar_arrive(x.p_full(half));
          ready = false;
          continue;
        }
        least = any * kSmall;
        hide<0>(a, seen);
        hide<A>(b, seen);
      }
      // the reference moves, O with it (rows whose own stays are as they were, bit for bit)
      auto move = [&](float to) -> bool {
        const float by = m == to ? 1.f : exp2_approx(m - to);
        l *= by;
        m = to;
        if (i == first) return true;
        if (!x.wait(x.o_done(half), (it - 1) & 1)) return false;
        tc_fence_after();
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
          uint32_t o[16];
          tmem_ld(o, col_o + 16 * c);
#pragma unroll
          for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * by);
          tmem_st(col_o + 16 * c, o);
        }
        return true;
      };
      bool begins = false;  // the row has its first reference from this tile
      if (!settled) {
        const float top = fmaxf(highest(a), highest(b)) * f;
        begins = m == -INFINITY && top != -INFINITY;
        if (!move(begins ? top - kRoom : m)) return;
        settled = __all_sync(0xffffffffu, m != -INFINITY);
      }
      auto shift = [&] { return m == -INFINITY ? 0.f : -m; };
      uint32_t p[A / 2];
      float sum = weights_of(a, p, f, shift());
      // (asked for before the exponentials, which hide how long the answer takes)
      if (!__all_sync(0xffffffffu, used) && !x.wait(x.o_done(half), (it - 1) & 1)) return;  // the last weights have been used
      tc_fence_after();
      put_words(col_p, p);
      {
        uint32_t q[B / 2];
        sum += weights_of(b, q, f, shift());
        put_words(col_p + A / 2, q);
      }
      const bool up = sum > kMost, down = l < kGrown && (begins ? sum - kFirst < least - kSmall : sum < least);
      if (__builtin_expect(__any_sync(0xffffffffu, up || down), 0)) {
        tmem_wait_st();  // the weights stored above are stored again below: the first stores land first
        const float top = fmaxf(highest(a), highest(b)) * f;
        if (!move(up ? fmaxf(m, top - kRoomUp) : !down ? m : begins ? m + (kRoom - kRoomAlone) : fmaxf(top - kRoom, m - kDown))) return;
        sum = weights_of(a, p, f, shift());
        put_words(col_p, p);
        uint32_t q[B / 2];
        sum += weights_of(b, q, f, shift());
        put_words(col_p + A / 2, q);
      }
      l += sum;
      const bool next = x.there(x.s_full(half), (it + 1) & 1);
      tmem_wait_st();
      tc_fence_before();
      if (lane == 0) mbar_arrive(x.p_full(half));
      ready = __all_sync(0xffffffffu, next);
    }
    const bool some = first < tiles;
    const bool turns = step == 2;
    const int first_row = turns ? 0 : half * kHalfRows, dest = sg.dest, at = begun ? x.rows(segs % kRunSlots)[first_row + row].at : -1;
    const bool mine = at >= 0;
    // the next run's rows, while this one's last product runs (its scores are all in: Q's place is free)
    if (!load_rows(segs + 1)) return;
    if (!begun) continue;
    // rows out: the output itself, or (m, l, o) for the join of pieces
    if (some) {
      if (!x.wait(x.o_done(half), (it - 1) & 1)) return;
      tc_fence_after();
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(x.seg_empty(segs % kRunSlots));
    float* const exchange = reinterpret_cast<float*>(x.base + L::kExchange);
    float2* const exchange_ml = reinterpret_cast<float2*>(x.base + L::kMl);
    if (turns && half == 1) {  // to the first half, 32 columns at a time
      if (joins > 0 && !x.wait(x.join_empty(), (joins - 1) & 1)) return;
      exchange_ml[row] = make_float2(m, l);
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c, ++joins) {
        uint32_t o[32];
        if (some) tmem_ld(o, col_o + 32 * c);
        if (c > 0 && !x.wait(x.join_empty(), (joins - 1) & 1)) return;
#pragma unroll
        for (int k = 0; k < 32; ++k) exchange[k * kHalfRows + row] = some ? __uint_as_float(o[k]) : 0.f;
        __syncwarp();
        if (lane == 0) mbar_arrive(x.join_full());
      }
      tc_fence_before();
      continue;
    }
    int to[4];  // rows of the lane and its three neighbours
#pragma unroll
    for (int k = 0; k < 4; ++k) to[k] = __shfl_sync(0xffffffffu, at, (lane & ~3) + k);
    float by = 1.f, other = 0.f, inv = 0.f;  // weights of the halves' sums
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t o[32];
      tmem_ld(o, col_o + 32 * c);
      if (turns) {
        if (!x.wait(x.join_full(), joins & 1)) return;
        if (c == 0) {
          const float2 ml = exchange_ml[row];
          const float high = fmaxf(m, ml.x);
          by = m == -INFINITY ? 0.f : exp2_approx(m - high);
          other = ml.x == -INFINITY ? 0.f : exp2_approx(ml.x - high);
          m = high;
          l = l * by + ml.y * other;
        }
#pragma unroll
        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * by + exchange[k * kHalfRows + row] * other);
        __syncwarp();
        if (lane == 0) mbar_arrive(x.join_empty());
        ++joins;
      }
      if (c == 0) {
        inv = l != 0.f ? 1.f / l : 0.f;
        if (mine && dest >= 0) g.part_ml[static_cast<int64_t>(dest) * kBlockRows + first_row + row] = make_float2(m, l);
        if (mine && dest < 0 && g.lse) g.lse[at] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
      }
      if (dest >= 0) {
#pragma unroll
        for (int k = 0; k < 32; k += 4)
          if (mine) *part_at<D>(g, dest, 8 * c + k / 4, first_row + row) = make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
      } else {
        uint32_t v[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int u = 0; u < 4; ++u) v[k][u] = pack16(true, __uint_as_float(o[8 * k + 2 * u]) * inv, __uint_as_float(o[8 * k + 2 * u + 1]) * inv);
        turn4(v, lane);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (to[k] >= 0) *reinterpret_cast<uint4*>(g.out + static_cast<int64_t>(to[k]) * D + 32 * c + 8 * (lane & 3)) = make_uint4(v[k][0], v[k][1], v[k][2], v[k][3]);
      }
    }
    tc_fence_before();
  }
}

template <int D>
__global__ void __launch_bounds__(kChunkThreads, 1) chunk_attn_kernel(const __grid_constant__ ChunkArgs g) {
  extern __shared__ uint8_t dyn[];
  using L = ChunkSmem<D>;
  __shared__ uint32_t s_tmem;
  ChunkCtx<D> x;
  x.base = dyn + ((1024 - (smem_u32(dyn) & 1023)) & 1023);
  x.args = &g;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    *x.abort_flag() = 0;
    *x.copied() = 0;
    for (int i = 0; i < L::kSlots; ++i) mbar_init(x.kv_full(i), 1), mbar_init(x.kv_empty(i), 2);
    for (int i = 0; i < kRunSlots; ++i) mbar_init(x.seg_full(i), 1), mbar_init(x.seg_empty(i), kChunkSoftmaxWarps + 3), mbar_init(x.rows_full(i), 1);
    for (int h = 0; h < 2; ++h) {
      mbar_init(x.q_full(h), 4), mbar_init(x.s_full(h), 1), mbar_init(x.s_read(h), 4);
      mbar_init(x.p_full(h), 4), mbar_init(x.o_done(h), 1), mbar_init(x.drained(h), 1);
    }
    mbar_init(x.join_full(), 4), mbar_init(x.join_empty(), 4);
    fence_barrier_init();
  }
  pdl_wait();
  pdl_trigger();
  if (g.head->bad || blockIdx.x * g.head->per >= g.head->work) {  // nothing for this CTA
    if (threadIdx.x == 0) g.piece[blockIdx.x].block = -1;
    return;
  }
  if (warp == kChunkMma) tmem_alloc(&s_tmem);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  x.tmem = s_tmem;
  if (warp < kChunkSoftmaxWarps) {
    registers_up<kChunkSoftmaxRegisters>();
    chunk_softmax<D>(g, x, warp >> 2, warp & 3, lane);
  } else {
    registers_down<kChunkOtherRegisters>();
    if (warp == kChunkProducer) chunk_produce<D>(g, x, lane);
    else if (warp == kChunkFinder) chunk_find_rows<D>(g, x, lane);
    else chunk_mma<D>(x, warp - kChunkMma);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kChunkMma) tmem_free(s_tmem);
  if (threadIdx.x == 0 && *x.abort_flag()) set_status(g.a.ctrl, TRR_ERR_TIMEOUT);
}

}  // namespace trr
