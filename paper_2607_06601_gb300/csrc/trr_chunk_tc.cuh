// trr_chunk_tc.cuh - attention of blocks of 256 rows over staged tiles, on the tensor cores (tcgen05).
//
// One CTA per SM.  A producer warp brings tiles of 128 tokens (K, V, positions) into rings of shared
// memory, as they were staged, with bulk copies.  A block's rows are two halves of 128, one to a lane of
// TMEM; one thread issues the products S = Q K^T and O += P V of both, and each half has a warpgroup that
// does its softmax, a thread a row, under the other half's products.  Sums and statistics are binary32.
//
// Tokens of 2, 4 and 8 bits are binary16, and p is rounded to it.  Tokens of 16 bits are bf16, in tiles of
// their own that follow, and p there is a sum of two bf16 numbers (one, of 8 bits, would add as much error
// as the output's own rounding).  Query rows are scaled by powers of two.
#pragma once

#include "trr_chunk.cuh"

namespace trr {

constexpr int kChunkSoftmaxWarps = 8, kChunkProducer = 8, kChunkMma = 9;
constexpr int kChunkThreads = 384;
// Registers a thread: 168 at launch; the softmax warpgroups take what the third gives up.
constexpr int kChunkLaunchRegisters = 168, kChunkSoftmaxRegisters = 208, kChunkOtherRegisters = 88;
static_assert(256 * kChunkSoftmaxRegisters + 128 * kChunkOtherRegisters <= kChunkThreads * kChunkLaunchRegisters, "");
constexpr int kPosSlots = 4, kSpanSlots = 2;

// A run of tiles of one type for one block and KV head, as the softmax and the product warps need it.
struct ChunkSegment {
  int tiles;        // 0: no more
  int wide;         // tiles of 16-bit tokens
  int first, last;  // of the block's runs in this CTA
  int block, kvh, rows;
  int dest;         // -1: the output rows, else the slot of the piece
};

template <int D>
struct ChunkSmem {
  static constexpr int kTile = kChunkTile * D * 2;  // bytes of K or V of a tile, or of Q of a half
  static constexpr int kSlots = D == 64 ? 4 : 2;    // of K, and of V
  static constexpr int kK = 2 * kTile;              // behind Q
  static constexpr int kV = kK + kSlots * kTile;
  static constexpr int kPos = kV + kSlots * kTile;
  static constexpr int kSeg = kPos + kPosSlots * kChunkTile * 4;
  static constexpr int kBars = kSeg + kSpanSlots * static_cast<int>(sizeof(ChunkSegment));
  static constexpr int kNumBars = 4 * kSlots + 2 * kPosSlots + 2 * kSpanSlots + 2 * 7 + 1;
  static constexpr int kTotal = kBars + 8 * kNumBars;
  static_assert(kTotal + 1024 <= 227 * 1024, "");
};

template <int D>
struct ChunkCtx {
  using L = ChunkSmem<D>;
  uint8_t* base;  // 1024-byte aligned
  uint32_t tmem;
  uint64_t wait_ns;
  volatile int* abort_flag;
  __device__ uint64_t* bar(int i) const { return reinterpret_cast<uint64_t*>(base + L::kBars) + i; }
  __device__ uint64_t* k_full(int i) const { return bar(i); }
  __device__ uint64_t* k_empty(int i) const { return bar(L::kSlots + i); }
  __device__ uint64_t* v_full(int i) const { return bar(2 * L::kSlots + i); }
  __device__ uint64_t* v_empty(int i) const { return bar(3 * L::kSlots + i); }
  __device__ uint64_t* pos_full(int i) const { return bar(4 * L::kSlots + i); }
  __device__ uint64_t* pos_empty(int i) const { return bar(4 * L::kSlots + kPosSlots + i); }
  __device__ uint64_t* seg_full(int i) const { return bar(4 * L::kSlots + 2 * kPosSlots + i); }
  __device__ uint64_t* seg_empty(int i) const { return bar(4 * L::kSlots + 2 * kPosSlots + kSpanSlots + i); }
  __device__ uint64_t* half_bar(int half, int i) const { return bar(4 * L::kSlots + 2 * kPosSlots + 2 * kSpanSlots + 7 * half + i); }
  __device__ uint64_t* q_full(int half) const { return half_bar(half, 0); }
  __device__ uint64_t* s_full(int half) const { return half_bar(half, 1); }
  __device__ uint64_t* s_read(int half) const { return half_bar(half, 2); }
  __device__ uint64_t* p_full(int half, int part) const { return half_bar(half, 3 + part); }  // the weights of 64 tokens
  __device__ uint64_t* o_done(int half) const { return half_bar(half, 5); }
  __device__ uint64_t* o_half(int half) const { return half_bar(half, 6); }  // the first 64 tokens of a wide tile (d 64)
  __device__ uint64_t* drained() const { return half_bar(2, 0); }
  __device__ ChunkSegment& seg(int i) const { return reinterpret_cast<ChunkSegment*>(base + L::kSeg)[i]; }
  __device__ const int32_t* pos(int i) const { return reinterpret_cast<const int32_t*>(base + L::kPos) + i * kChunkTile; }
  // TMEM columns.  d 128: S and O of each half, P over S, a wide tile's weights as 64 columns of high parts and
  // 64 of low ones.  d 64: P has columns of its own, so that the next scores can be issued once these have been
  // read; a wide tile's weights take turns in them, 64 tokens at a time.
  __device__ uint32_t col_s(int half) const { return tmem + 128 * half; }
  __device__ uint32_t col_p(int half, int part, int wide) const {
    return D == 128 ? col_s(half) + 32 * part : tmem + 256 + 64 * half + (wide ? 0 : 32 * part);
  }
  __device__ uint32_t col_low(int half, int part) const { return D == 128 ? col_s(half) + 64 + 32 * part : tmem + 256 + 64 * half + 32; }
  __device__ uint32_t col_o(int half) const { return tmem + (D == 128 ? 256 + 128 * half : 384 + 64 * half); }
  // A bounded wait; once one has given up, none waits any more.
  __device__ bool wait(uint64_t* b, uint32_t parity) const {
    if (mbar_poll(smem_u32(b), parity, wait_ns)) return true;
    const uint64_t t0 = global_ns();
    while (!mbar_poll(smem_u32(b), parity, wait_ns)) {
      if (*abort_flag || global_ns() - t0 >= wait_ns) {
        *abort_flag = 1;
        return false;
      }
    }
    return true;
  }
  // The same by a whole warp: all of its lanes get the same answer.
  __device__ bool wait_warp(uint64_t* b, uint32_t parity) const { return __all_sync(0xffffffffu, wait(b, parity)); }
};

// Tiles of a segment that lie before cost x (counted from the segment's start).
__device__ __forceinline__ int chunk_tiles_before(int64_t x, int tiles) {
  if (x <= kChunkSegmentCost) return 0;
  const int64_t t = (x - kChunkSegmentCost + kChunkTileCost - 1) / kChunkTileCost;
  return t < tiles ? static_cast<int>(t) : tiles;
}

// The producer warp: the runs of this CTA's share, and the copies of their tiles.
template <int D>
__device__ __forceinline__ void chunk_produce(const ChunkArgs& g, const ChunkCtx<D>& x, int lane) {
  using L = ChunkSmem<D>;
  const int64_t per = g.head->per, work = g.head->work;
  const int blocks = g.head->blocks;
  const int64_t b0 = min(work, blockIdx.x * per), b1 = min(work, b0 + per);
  int tiles_done = 0, segs = 0, k_copies = 0, pos_copies = 0, v_copies = 0;
  bool ok = true;
  PieceInfo piece = {-1, 0, 0, 0};
  auto push = [&](const ChunkSegment& s, const BlockPlan& p, const ChunkPlan& c, int from) {
    if (!ok || s.tiles == 0) return;
    ok = x.wait_warp(x.seg_empty(segs % kSpanSlots), ((segs / kSpanSlots) & 1) ^ 1);
    if (!ok) return;
    if (lane == 0) {
      x.seg(segs % kSpanSlots) = s;
      mbar_arrive(x.seg_full(segs % kSpanSlots));
    }
    ++segs;
    const int l = s.wide, base = c.tile0 + (l ? c.tiles[0] : 0);
    for (int i = from; i < from + s.tiles; ++i) {
      const int tile = base + (i < p.head[l] ? i : p.first[l] + i - p.head[l]);
      const int slot = tiles_done % L::kSlots, at = tiles_done % kPosSlots;
      ok = x.wait_warp(x.k_empty(slot), ((tiles_done / L::kSlots) & 1) ^ 1);
      if (!ok) return;
      if (lane == 0) {
        mbar_arrive_expect_tx(x.k_full(slot), L::kTile);
        bulk_g2s(x.base + L::kK + slot * L::kTile, staged_tile<D>(g, tile, s.kvh, 0), L::kTile, x.k_full(slot));
      }
      ++k_copies;
      ok = x.wait_warp(x.pos_empty(at), ((tiles_done / kPosSlots) & 1) ^ 1);
      if (!ok) return;
      if (lane == 0) {
        mbar_arrive_expect_tx(x.pos_full(at), 4 * kChunkTile);
        bulk_g2s(x.base + L::kPos + at * 4 * kChunkTile, g.pos + static_cast<int64_t>(tile) * kChunkTile, 4 * kChunkTile, x.pos_full(at));
      }
      ++pos_copies;
      ok = x.wait_warp(x.v_empty(slot), ((tiles_done / L::kSlots) & 1) ^ 1);
      if (!ok) return;
      if (lane == 0) {
        mbar_arrive_expect_tx(x.v_full(slot), L::kTile);
        bulk_g2s(x.base + L::kV + slot * L::kTile, staged_tile<D>(g, tile, s.kvh, 1), L::kTile, x.v_full(slot));
      }
      ++v_copies;
      ++tiles_done;
    }
  };
  if (b0 < b1) {
    fence_proxy_async_global();  // the tiles were staged with ordinary stores
    int lo = 0, hi = blocks - 1;  // the block that holds cost b0: the last one that starts at or before it
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (g.base[mid] <= b0) lo = mid;
      else hi = mid - 1;
    }
    for (int b = lo; b < blocks && ok; ++b) {
      const int64_t start = g.base[b];
      if (start >= b1) break;
      const BlockPlan p = g.block[b];
      if (p.tiles == 0) continue;
      const ChunkPlan& c = g.chunk[p.chunk];
      const int64_t cost = chunk_cost(p.tiles);
      for (int h = static_cast<int>(max(static_cast<int64_t>(0), (b0 - start) / cost)); h < g.a.Hkv && ok; ++h) {
        const int64_t S = start + h * cost;
        if (S >= b1) break;
        const int t0 = chunk_tiles_before(b0 - S, p.tiles), t1 = chunk_tiles_before(b1 - S, p.tiles);
        if (t0 >= t1) continue;
        const int narrow = p.head[0] + p.last[0] - p.first[0];
        if (t0 == 0 && t1 < p.tiles) piece = PieceInfo{b, h, 0, 0};
        ChunkSegment s;
        s.block = b; s.kvh = h; s.rows = p.rows;
        s.dest = t0 == 0 && t1 == p.tiles ? -1 : 2 * static_cast<int>(blockIdx.x) + (t0 > 0 ? 0 : 1);
        s.wide = 0; s.tiles = max(0, min(t1, narrow) - t0); s.first = 1; s.last = t1 <= narrow;
        push(s, p, c, t0);
        s.wide = 1; s.first = t0 >= narrow; s.last = 1; s.tiles = max(0, t1 - max(t0, narrow));
        push(s, p, c, max(t0, narrow) - narrow);
      }
    }
  }
  if (lane == 0) g.piece[blockIdx.x] = piece;
  if (ok) {  // no more
    ok = x.wait_warp(x.seg_empty(segs % kSpanSlots), ((segs / kSpanSlots) & 1) ^ 1);
    if (ok && lane == 0) {
      x.seg(segs % kSpanSlots).tiles = 0;
      mbar_arrive(x.seg_full(segs % kSpanSlots));
    }
  }
  // the CTA stays until its copies have landed
  for (int k = max(0, k_copies - L::kSlots); k < k_copies; ++k) mbar_wait(x.k_full(k % L::kSlots), (k / L::kSlots) & 1);
  for (int k = max(0, v_copies - L::kSlots); k < v_copies; ++k) mbar_wait(x.v_full(k % L::kSlots), (k / L::kSlots) & 1);
  for (int k = max(0, pos_copies - kPosSlots); k < pos_copies; ++k) mbar_wait(x.pos_full(k % kPosSlots), (k / kPosSlots) & 1);
}

// The warp that issues the products (one elected lane does; the whole warp goes along).  The halves take
// turns, O += P V of a tile and S of the next: then one half's softmax runs under the other's products.
// (Left to warps of their own the two fell into step: both waited for the tensor core, then both for the
// exponentials.)  A wait stands before scores that go over weights: nothing orders the two products.
template <int D>
__device__ __forceinline__ void chunk_mma(const ChunkCtx<D>& x) {
  using L = ChunkSmem<D>;
  int segs = 0, tile = 0, it[2] = {0, 0}, loads[2] = {0, 0};  // tile: of the CTA, it: of a half, loads: of its Q
  const uint32_t base = smem_u32(x.base);
  for (bool ok = true; ok;) {
    if (!x.wait_warp(x.seg_full(segs % kSpanSlots), (segs / kSpanSlots) & 1)) break;
    const ChunkSegment& sg = x.seg(segs % kSpanSlots);
    const int n = __shfl_sync(0xffffffffu, sg.tiles, 0), wide = __shfl_sync(0xffffffffu, sg.wide, 0);
    const bool first = __shfl_sync(0xffffffffu, sg.first, 0);
    const int halves = __shfl_sync(0xffffffffu, sg.rows, 0) > kPipeRows ? 2 : 1;
    __syncwarp();
    if (elected()) mbar_arrive(x.seg_empty(segs % kSpanSlots));
    ++segs;
    if (n == 0) break;
    const uint32_t id_s = tc_idesc(wide, kChunkTile, false), id_o = tc_idesc(wide, D, true);
    auto scores = [&](int half, int t) {  // S of tile t (of the CTA), whose K is there
      const int slot = t % L::kSlots;
      tc_fence_after();
      const uint64_t a = tc_desc(base + half * L::kTile, 16), b = tc_desc(base + L::kK + slot * L::kTile, 16);
      if (elected()) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t o = ((k >> 2) * (kChunkTile * 128) + (k & 3) * 32) >> 4;
          tc_mma_ss(x.col_s(half), a + o, b + o, id_s, k > 0);
        }
        tc_commit(x.s_full(half));
        if (half == halves - 1) tc_commit(x.k_empty(slot));
      }
      __syncwarp();
    };
    auto keys = [&](int t) { return x.wait_warp(x.k_full(t % L::kSlots), (t / L::kSlots) & 1); };
    auto values = [&](int half, int i) -> bool {  // O += P V of the segment's tile i
      const int slot = tile % L::kSlots;
      const uint64_t d = tc_desc(base + L::kV + slot * L::kTile, kChunkTile * 128);
#pragma unroll 1
      for (int part = 0; part < 2; ++part) {  // 64 tokens at a time, as their weights come
        if (!x.wait_warp(x.p_full(half, part), it[half] & 1)) return false;
        tc_fence_after();
        if (elected()) {
#pragma unroll
          for (int j = 0; j < kChunkTile / 32; ++j) {
            const int k = part * (kChunkTile / 32) + j;
            tc_mma(x.col_o(half), x.col_p(half, part, wide) + 8 * j, d + k * (2048 >> 4), id_o, k > 0 || i > 0 || !first);
          }
          if (wide) {  // the weights' low parts
#pragma unroll
            for (int j = 0; j < kChunkTile / 32; ++j) {
              const int k = part * (kChunkTile / 32) + j;
              tc_mma(x.col_o(half), x.col_low(half, part) + 8 * j, d + k * (2048 >> 4), id_o, true);
            }
            if (D == 64 && part == 0) tc_commit(x.o_half(half));
          }
          if (part == 1) {
            if (half == halves - 1) tc_commit(x.v_empty(slot));
            tc_commit(x.o_done(half));
          }
        }
        __syncwarp();
      }
      ++it[half];
      return true;
    };
    ok = keys(tile);
    for (int h = 0; h < halves && ok; ++h) {
      if (it[h] > 0) ok = x.wait_warp(x.o_done(h), (it[h] - 1) & 1);
      ok = ok && x.wait_warp(x.q_full(h), loads[h]++ & 1);
      if (ok) scores(h, tile);
    }
    for (int i = 0; i < n && ok; ++i, ++tile) {
      const bool more = i + 1 < n;
      if (D == 64 && more) {  // weights have columns of their own: the next scores as soon as these are read
        ok = keys(tile + 1);
        for (int h = 0; h < halves && ok; ++h) {
          ok = x.wait_warp(x.s_read(h), it[h] & 1);
          if (ok) scores(h, tile + 1);
        }
      }
      ok = ok && x.wait_warp(x.v_full(tile % L::kSlots), (tile / L::kSlots) & 1);
      for (int h = 0; h < halves && ok; ++h) {
        ok = values(h, i);
        if (D == 128 && more && ok) {
          ok = (h > 0 || keys(tile + 1)) && x.wait_warp(x.o_done(h), (it[h] - 1) & 1);
          if (ok) scores(h, tile + 1);
        }
      }
    }
  }
  if (elected()) tc_commit(x.drained());  // nothing is in flight when the CTA ends
  __syncwarp();
  mbar_wait(x.drained(), 0);
}

// How many of 128 ascending positions are below v.
__device__ __forceinline__ int below(const int32_t* pos, int v) {
  int n = 0;
#pragma unroll
  for (int step = 64; step > 0; step >>= 1)
    if (pos[n + step - 1] < v) n += step;
  return n + (pos[n] < v ? 1 : 0);
}

// The 32 of bits 0 .. n-1 that lie in word w.
__device__ __forceinline__ uint32_t bits_below(int n, int w) {
  const int k = n - 32 * w;
  return k <= 0 ? 0u : k >= 32 ? 0xffffffffu : (1u << k) - 1;
}

// The softmax warps of a half, a thread a row.
template <int D>
__device__ __forceinline__ void chunk_softmax(const ChunkArgs& g, const ChunkCtx<D>& x, int half, int quad, int lane) {
  using L = ChunkSmem<D>;
  const int row = quad * 32 + lane;
  const uint32_t lanes = static_cast<uint32_t>(quad) << 21;  // the warp's 32 lanes of TMEM
  const uint32_t col_s = x.col_s(half) + lanes, col_o = x.col_o(half) + lanes;
  int segs = 0, tile = 0, it = 0, wides = 0;
  float m = -INFINITY, l = 0.f, f = 0.f;
  RowSource src = {};
  bool mine = false;
  for (;;) {
    if (!x.wait_warp(x.seg_full(segs % kSpanSlots), (segs / kSpanSlots) & 1)) return;
    const ChunkSegment sg = x.seg(segs % kSpanSlots);
    __syncwarp();
    if (lane == 0) mbar_arrive(x.seg_empty(segs % kSpanSlots));
    ++segs;
    if (sg.tiles == 0) return;
    if (sg.rows <= half * kPipeRows) {
      for (int i = 0; i < sg.tiles; ++i, ++tile) {
        if (!x.wait_warp(x.pos_full(tile % kPosSlots), (tile / kPosSlots) & 1)) return;
        if (lane == 0) mbar_arrive(x.pos_empty(tile % kPosSlots));
      }
      continue;
    }
    // The row's query into shared memory, in the tiles' type, scaled by the power of two that brings its
    // largest element to [1, 2): binary16 then holds what it needs of it.  (The last segment's scores are all in.)
    {
      const BlockPlan& p = g.block[sg.block];
      mine = half * kPipeRows + row < sg.rows;
      uint4 w[D / 8];
      uint32_t top = 0;
      if (mine) {
        src = row_source(g, g.chunk[p.chunk], p.query0, p.local, sg.kvh, p.row + half * kPipeRows + row);
        const uint4* q = reinterpret_cast<const uint4*>(g.q + (static_cast<int64_t>(src.query) * g.a.Hq + src.head) * D);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) w[i] = q[i];
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) top = max(top, max(v[k] & 0x7FFFu, (v[k] >> 16) & 0x7FFFu));
        }
      } else {  // sees every token, so that its warp need not mask for it
        src.t = INT_MAX - 1;
        src.lo = 0;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) w[i] = make_uint4(0, 0, 0, 0);
      }
      int e = top == 0 || top >= 0x7F80u ? 0 : static_cast<int>(top >> 7) - 127;
      e = max(-100, min(120, e));
      const float down = __int_as_float((127 - e) << 23);
      f = fmaxf(g.scale_log2 * __int_as_float((127 + e) << 23), 1.17549435e-38f);
      uint8_t* to = x.base + half * L::kTile;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = pack16(sg.wide, bf16lo(v[k]) * down, bf16hi(v[k]) * down);
        *reinterpret_cast<uint4*>(to + tile_at(row, i)) = make_uint4(o[0], o[1], o[2], o[3]);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(x.q_full(half));
    }
    const bool local = g.block[sg.block].local;
    if (sg.first) m = -INFINITY, l = 0.f;
    for (int i = 0; i < sg.tiles; ++i, ++it, ++tile) {
      const int slot = tile % kPosSlots;
      if (!x.wait_warp(x.pos_full(slot), (tile / kPosSlots) & 1)) return;
      const int32_t* pos = x.pos(slot);
      const bool all = __all_sync(0xffffffffu, pos[kChunkTile - 1] <= src.t && pos[0] >= src.lo);
      if (!x.wait_warp(x.s_full(half), it & 1)) return;
      tc_fence_after();
      uint32_t s[2][64];
      tmem_ld(s, col_s);
      if (D == 64) {  // the next scores may come
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(x.s_read(half));
      }
      if (!all) {
        const int c = below(pos, src.t + 1), from = pos[0] >= src.lo ? 0 : below(pos, src.lo), head = local && from > 0 ? below(pos, g.sinks) : 0;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int word = 2 * h + k;
            const uint32_t seen = bits_below(c, word) & (~bits_below(from, word) | bits_below(head, word));
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (!(seen >> j & 1)) s[h][32 * k + j] = 0xFF800000u;
          }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(x.pos_empty(slot));
      const float top = fmaxf(highest(s[0]), highest(s[1])) * f;
      // m follows the maximum only when that has grown by more than 2^8: p stays within binary16, and O is rarely rescaled
      if (__any_sync(0xffffffffu, top > m + 8.f)) {
        const float next = fmaxf(m, top), by = m == -INFINITY ? 0.f : exp2_approx(m - next);
        l *= by;
        m = next;
        if (i > 0 || !sg.first) {
          if (!x.wait_warp(x.o_done(half), (it - 1) & 1)) return;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            uint32_t o[16];
            tmem_ld(o, col_o + 16 * c);
#pragma unroll
            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * by);
            tmem_st(col_o + 16 * c, o);
          }
        }
      }
      const float shift = m == -INFINITY ? 0.f : -m;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l += weigh(s[h], f, shift);
        if (D == 64 && h == 0 && it > 0 && !x.wait_warp(x.o_done(half), (it - 1) & 1)) return;  // the last weights have been used
        uint32_t p[32];
        if (sg.wide) {  // high parts cut off, low parts what is left, rounded
          uint32_t low[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            const uint32_t a = s[h][2 * k], b = s[h][2 * k + 1];
            p[k] = __byte_perm(a, b, 0x7632);
            low[k] = pack16(true, __uint_as_float(a) - __uint_as_float(a & 0xFFFF0000u), __uint_as_float(b) - __uint_as_float(b & 0xFFFF0000u));
          }
          if (D == 64 && h == 1 && !x.wait_warp(x.o_half(half), wides++ & 1)) return;
          tmem_st(x.col_low(half, h) + lanes, low);
        } else {
#pragma unroll
          for (int k = 0; k < 32; ++k) p[k] = pack16(false, __uint_as_float(s[h][2 * k]), __uint_as_float(s[h][2 * k + 1]));
        }
        tmem_st(x.col_p(half, h, sg.wide) + lanes, p);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(x.p_full(half, h));  // the product of these tokens can start
      }
    }
    if (!sg.last) continue;
    // rows out: the output itself, or (m, l, o) for the join
    if (!x.wait_warp(x.o_done(half), (it - 1) & 1)) return;
    tc_fence_after();
    const int64_t at = static_cast<int64_t>(src.query) * g.a.Hq + src.head;
    if (sg.dest >= 0) {
      const int64_t slot = static_cast<int64_t>(sg.dest) * kBlockRows + half * kPipeRows + row;
      if (mine) g.part_ml[slot] = make_float2(m, l);
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        tmem_ld(o, col_o + 32 * c);
        if (mine) {
#pragma unroll
          for (int k = 0; k < 32; k += 8) st_global8(g.part_o + slot * D + 32 * c + k, reinterpret_cast<const float*>(o + k));
        }
      }
    } else {
      const float inv = l != 0.f ? 1.f / l : 0.f;
      if (mine && g.lse) g.lse[at] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        tmem_ld(o, col_o + 32 * c);
        if (mine) {
#pragma unroll
          for (int k = 0; k < 32; k += 8) {
            uint32_t v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = pack16(true, __uint_as_float(o[k + 2 * u]) * inv, __uint_as_float(o[k + 2 * u + 1]) * inv);
            *reinterpret_cast<uint4*>(g.out + at * D + 32 * c + k) = make_uint4(v[0], v[1], v[2], v[3]);
          }
        }
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
  __shared__ int s_abort;
  ChunkCtx<D> x;
  x.base = dyn + ((1024 - (smem_u32(dyn) & 1023)) & 1023);
  x.wait_ns = g.a.wait_ns;
  x.abort_flag = &s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < L::kSlots; ++i) mbar_init(x.k_full(i), 1), mbar_init(x.k_empty(i), 1), mbar_init(x.v_full(i), 1), mbar_init(x.v_empty(i), 1);
    for (int i = 0; i < kPosSlots; ++i) mbar_init(x.pos_full(i), 1), mbar_init(x.pos_empty(i), kChunkSoftmaxWarps);
    for (int i = 0; i < kSpanSlots; ++i) mbar_init(x.seg_full(i), 1), mbar_init(x.seg_empty(i), kChunkSoftmaxWarps + 1);
    for (int h = 0; h < 2; ++h) {
      mbar_init(x.q_full(h), 4), mbar_init(x.s_full(h), 1), mbar_init(x.s_read(h), 4);
      mbar_init(x.p_full(h, 0), 4), mbar_init(x.p_full(h, 1), 4), mbar_init(x.o_done(h), 1), mbar_init(x.o_half(h), 1);
    }
    mbar_init(x.drained(), 1);
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
    else if (warp == kChunkMma) chunk_mma<D>(x);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kChunkMma) tmem_free(s_tmem);
  if (threadIdx.x == 0 && s_abort) set_status(g.a.ctrl, TRR_ERR_TIMEOUT);
}

}  // namespace trr
