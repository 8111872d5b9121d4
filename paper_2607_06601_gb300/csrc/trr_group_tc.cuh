// trr_group_tc.cuh - attention of segments with many rows on the tensor cores (tcgen05).
//
// One CTA per SM.  A producer warp brings each tile's page slices into a ring of shared memory
// with bulk copies; sixteen warps expand them to 16-bit rows in the tensor core's layout; one
// thread issues the products S = Q K^T and O += P V (sums in TMEM); eight warps do the softmax,
// two threads for each row of TMEM.  Pages of 2, 4 and 8 bits become binary16 (z + c s rounded
// once, 11 bits) and p is rounded to it; pages of 16 bits stay bf16 and p is a sum of two bf16
// numbers there; sums and statistics are binary32.  A segment of 64 or 32 rows or fewer fills the 128 lanes with two or
// four copies of its rows, each of which takes its own part of a tile's tokens, so that all
// warps share the exponentials.
//
// Binary16 keys are the coarsest step: a twelfth bit of a value against the 8 of its code, so at most
// a sixteenth of an 8-bit group's step, unless all of the group's values lie far from zero together.
// Rows of random data come out 1.02 times the output's rounding off (root mean square), with scores
// of standard deviation 16 or single channels 30 times the others 1.2 times, with 50 added to every
// element of K 3.3 to 5.5 times.
//
// What bounds it, for a tile of 128 tokens at d 128: the products take about 1024 cycles, the
// exponentials 1024 (16 a cycle), the expansion's integer instructions about as long; the three
// hand tiles on to one another.  A tile more for every CTA takes 3600 cycles with 2 or 4 bits, 6000
// with 8 (the ring then holds two tiles instead of four and more; whether that is why was not
// tried), and 4800 for the 64 tokens of a tile of 16 bits.
//
// Measured: 64 queries of 32 heads on 32768 shared tokens, 8 KV heads of 128 (27 GFLOP, 36 MB;
// 14.6 us at the measured rate of library products): 65 us, 0.42 PFLOP/s, of which 9 are the start
// to the first scores and 5 the rows out.  16 such queries (two copies of 64 rows): 41 us (both by
// themselves, caches cold).
// With one softmax thread a row and eight expanding warps, 63 queries of 7 prompts took 127 us a
// call against 118 then; softmax warpgroups that take whole tiles in turn, 91 against 87.
#pragma once

#include <type_traits>

#include "trr_group.cuh"

namespace trr {

constexpr int kRawSlots = 8;     // tiles in the ring of raw pages
constexpr int kSegSlots = 4;     // segments announced ahead
constexpr int kMetaSlots = 8;    // tiles whose record the softmax may still need: at least kStages + 2
constexpr int kSoftmaxWarps = 8, kExpandWarps = 16;
constexpr int kMmaWarp = kSoftmaxWarps + kExpandWarps, kProducer = kMmaWarp + 1;
constexpr int kGroupThreads = 32 * (kProducer + 3);  // whole warpgroups: two warps more that do nothing
// Registers a thread: 72 at launch; two softmax warpgroups take what the other five give up
// (256 x 112 + 640 x 56 = 896 x 72).
constexpr int kSoftmaxRegisters = 112, kOtherRegisters = 56;
static_assert(32 * kSoftmaxWarps * kSoftmaxRegisters + (kGroupThreads - 32 * kSoftmaxWarps) * kOtherRegisters <= kGroupThreads * 72, "");

// A segment, or a CTA's piece of one, as the softmax warps need it.
struct Segment {
  int tiles;          // 0: no more
  int row0, rows;     // its rows in the job, at most 128
  int kind, qbase, kvh;
  int dest;           // -2: the output row, -1: the home row, else the piece's slot
  int pad;
};

struct RawPage {
  int off, pos;       // slice and slot positions in the ring; pos < 0: every token in sight
  int valid, cls;     // slots that hold a token
};
struct RawTile {
  int pages, bf16, first, end;
  int lo, t, sinks, all;
  RawPage page[kTileKeys / 16];
};
struct TileMeta {
  int keys, bf16, first, end, all;  // all: 128 tokens, every one in sight
  uint16_t mask[kTileKeys / 16];    // tokens in sight
  int pad[3];
};

template <int D>
struct GroupSmem {
  static constexpr int kStages = D == 64 ? 3 : 2;       // expanded tiles
  static constexpr int kTile = kTileKeys * D * 2;       // bytes of K or V of one
  static constexpr int kScratch = kStages * 2 * kTile;  // merge of row copies: [2 halves][128][17] floats
  static constexpr int kMl = kScratch + 2 * kRows * 17 * 4;  // [2][128] (m, l)
  static constexpr int kTops = kMl + 2 * kRows * 8;          // [2 tiles][2][128] maxima
  static constexpr int kRaw = kTops + 4 * kRows * 4;
  static constexpr int kSeg = kRaw + kRawSlots * static_cast<int>(sizeof(RawTile));
  static constexpr int kMeta = kSeg + kSegSlots * static_cast<int>(sizeof(Segment));
  static constexpr int kBars = kMeta + kMetaSlots * static_cast<int>(sizeof(TileMeta));
  static constexpr int kNumBars = 2 * kRawSlots + 2 * kSegSlots + 4 * kStages + 13;
  static constexpr int kRing = (kBars + kNumBars * 8 + 127) / 128 * 128;
  static constexpr int kTotal = 225 * 1024;  // of the 227 KB a CTA may have; 1 KB aligns the base
  static constexpr int kRingBytes = (kTotal - kRing) / 128 * 128;
  // the widest tile: 8-bit pages with four groups (d 128), or 64 tokens of 16 bits; slot positions of each page
  static_assert(kRingBytes >= kTileKeys * (2 * D + 8 * (D / 32)) + 8 * 256, "a tile must fit the ring");
};

template <int D>
struct Ctx {
  using L = GroupSmem<D>;
  uint8_t* base;  // 1024-byte aligned
  uint32_t tmem;
  uint64_t wait_ns;
  volatile int* abort_flag;
  __device__ uint64_t* bar(int i) const { return reinterpret_cast<uint64_t*>(base + L::kBars) + i; }
  __device__ uint64_t* raw_full(int i) const { return bar(i); }
  __device__ uint64_t* raw_empty(int i) const { return bar(kRawSlots + i); }
  __device__ uint64_t* seg_full(int i) const { return bar(2 * kRawSlots + i); }
  __device__ uint64_t* seg_empty(int i) const { return bar(2 * kRawSlots + kSegSlots + i); }
  // which: 0 K, 1 V
  __device__ uint64_t* kv_full(int which, int i) const { return bar(2 * kRawSlots + 2 * kSegSlots + which * L::kStages + i); }
  __device__ uint64_t* kv_empty(int which, int i) const { return bar(2 * kRawSlots + 2 * kSegSlots + (2 + which) * L::kStages + i); }
  __device__ uint64_t* s_full(int i) const { return bar(2 * kRawSlots + 2 * kSegSlots + 4 * L::kStages + i); }
  __device__ uint64_t* p_full(int i) const { return s_full(2 + i); }
  __device__ uint64_t* o_done(int i) const { return s_full(4 + i); }
  __device__ uint64_t* q_full() const { return s_full(6); }
  __device__ uint64_t* drained() const { return s_full(7); }
  __device__ uint64_t* merged() const { return s_full(8); }
  __device__ uint64_t* pair(int i) const { return s_full(9 + i); }
  __device__ RawTile& raw(int i) const { return reinterpret_cast<RawTile*>(base + L::kRaw)[i]; }
  __device__ Segment& seg(int i) const { return reinterpret_cast<Segment*>(base + L::kSeg)[i]; }
  __device__ TileMeta& meta(int i) const { return reinterpret_cast<TileMeta*>(base + L::kMeta)[i]; }
  __device__ uint32_t tile(int stage, int which) const { return smem_u32(base) + (2 * stage + which) * L::kTile; }
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

// TMEM columns: O, two S (P over S), Q in binary16 and bf16.  A tile of 16-bit pages has 64 tokens at
// most: its weights' low parts take the second half of the columns of its S.
constexpr uint32_t kColO = 0, kColS = 128, kColQ = 384, kColPLow = 64;

// The producer warp: segments and tiles of this CTA's run, and the copies of their pages.
template <int D>
__device__ __forceinline__ void group_produce(const GroupArgs& g, const Ctx<D>& x, int lane) {
  using L = GroupSmem<D>;
  const LayerArgs& a = g.a;
  const int64_t per = g.head->per, work = g.head->work;
  const int64_t b0 = min(work, blockIdx.x * per), b1 = min(work, b0 + per);
  const int jobs = g.few ? g.groups : g.groups + g.n, P = a.P, lg_p = __ffs(P) - 1;
  int it = 0, freed = 0;  // tiles pushed, tiles whose ring bytes are known to be free
  int ring_head = 0, segs = 0;
  bool ok = true;

  // room for `need` bytes and a record; the offset in the ring
  auto book = [&](int need) -> int {
    for (;;) {
      if (it - freed < kRawSlots) {
        if (it == freed) { ring_head = need; return 0; }
        const int tail = x.raw(freed % kRawSlots).page[0].off;
        if (ring_head > tail) {
          if (ring_head + need <= L::kRingBytes) { ring_head += need; return ring_head - need; }
          if (need < tail) { ring_head = need; return 0; }
        } else if (ring_head + need < tail) {
          ring_head += need;
          return ring_head - need;
        }
      }
      if (!x.wait_warp(x.raw_empty(freed % kRawSlots), (freed / kRawSlots) & 1)) return -1;
      ++freed;
    }
  };

  if (b0 < b1) {
    // the job that holds cost b0: the last one that starts at or before it
    int lo = 0, hi = jobs;
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, i = lo + lane * step;
      const int k = __popc(__ballot_sync(0xffffffffu, i < hi && g.base[i] <= b0));
      const int last = lo + (k - 1) * step;
      hi = min(hi, last + step);
      lo = last;
      if (step == 1) break;
    }
    for (int j = lo; j < jobs && ok; ++j) {
      const int64_t jbase = g.base[j];  // (all loads of a job before the first branch on one)
      const int w = reinterpret_cast<const int*>(g.jobs + j)[lane], tiles = g.tiles[j];
      if (jbase >= b1) break;
      auto field = [&](int i) { return __shfl_sync(0xffffffffu, w, i); };
      if (tiles <= 0) continue;
      const int seq = field(0), jlo = field(1), jt = field(2), sinks = field(3);
      int head[kClasses], first[kClasses], upto[kClasses + 1];
      upto[0] = 0;
      for (int c = 0; c < kClasses; ++c) {
        head[c] = field(4 + c);
        first[c] = field(8 + c);
        upto[c + 1] = upto[c] + head[c] + field(12 + c);
      }
      const int rows = field(16), row_blocks = field(17), tiles_q = field(18), kind = field(20), qbase = field(21), joined = field(22);
      const int64_t cost = segment_cost(tiles);
      const int nsegs = a.Hkv * row_blocks;
      // a batch of 32 pages, one per lane, of the 2-, 4- and 8-bit pages or of the others
      int batch = -1, slice = 0, room = 0, bytes = 0, valid = 0, cls = 0;
      bool whole = true;
      const uint8_t* src = nullptr;  // the page
      for (int s = static_cast<int>(max(static_cast<int64_t>(0), (b0 - jbase) / cost)); s < nsegs && ok; ++s) {
        const int64_t S = jbase + s * cost;
        if (S >= b1) break;
        const int t0 = tiles_before(b0 - S, tiles), t1 = tiles_before(b1 - S, tiles);
        if (t0 >= t1) continue;
        const int kvh = s / row_blocks, rb = s % row_blocks;
        ok = x.wait_warp(x.seg_empty(segs % kSegSlots), ((segs / kSegSlots) & 1) ^ 1);
        if (!ok) break;
        if (lane == 0) {
          Segment& sg = x.seg(segs % kSegSlots);
          sg.tiles = t1 - t0;
          sg.row0 = rb * kRows;
          sg.rows = min(kRows, rows - rb * kRows);
          sg.kind = kind; sg.qbase = qbase; sg.kvh = kvh;
          sg.dest = t1 - t0 == tiles ? (joined ? -1 : -2) : 2 * blockIdx.x + (t0 > 0 ? 0 : 1);
          mbar_arrive(x.seg_full(segs % kSegSlots));
        }
        ++segs;
        for (int tile = t0; tile < t1; ++tile) {
          const bool wide = tile >= tiles_q;
          const int lg = wide ? 6 - lg_p : 7 - lg_p;  // log2 of a tile's pages
          const int i0 = (wide ? tile - tiles_q : tile) << lg, end = wide ? upto[4] - upto[3] : upto[3];
          const int b = (i0 >> 5) + (wide ? 1 << 28 : 0);
          if (b != batch) {
            batch = b;
            const int i = (i0 & ~31) + lane;
            cls = wide ? 3 : i >= upto[2] ? 2 : i >= upto[1] ? 1 : 0;
            const int in = wide ? i : i - (cls == 2 ? upto[2] : cls == 1 ? upto[1] : 0);
            int h = head[0], f = first[0], n = field(23);
#pragma unroll
            for (int c = 1; c < kClasses; ++c) {
              const int m = field(23 + c);
              if (cls == c) h = head[c], f = first[c], n = m;
            }
            if (i < end) {
              const int k = in < h ? in : f + in - h;
              const int64_t at = (static_cast<int64_t>(seq) * kClasses + cls) * a.MP + k;
              const int page = a.pt[at], pf = a.pfirst[at], pl = a.plast[at];
              valid = min(P, n - k * P);
              whole = valid == P && pl <= jt && (pf >= jlo || pl < sinks);
              slice = a.slice[cls];
              src = a.pool[cls] + page * a.page_bytes[cls];
              room = (slice + 127) / 128 * 128 + (whole ? 0 : (4 * P + 127) / 128 * 128);
              bytes = slice + (whole ? 0 : 4 * P);
              // the ring holds a few tiles; the rest of the batch comes as far as L2 meanwhile
              if (i - i0 >= 2 << lg && i < (wide ? t1 - tiles_q : min(t1, tiles_q)) << lg)
                prefetch_l2(src + a.hdr + static_cast<int64_t>(kvh) * slice, slice);
            }
            __syncwarp();
          }
          const int pages = min(1 << lg, end - i0), l0 = i0 & 31, r = lane - l0;
          const bool mine = r >= 0 && r < pages;
          int off = mine ? room : 0;
#pragma unroll
          for (int o = 1; o < kTileKeys / 16; o <<= 1) {  // at most eight pages
            const int y = __shfl_up_sync(0xffffffffu, off, o);
            if (lane >= o) off += y;
          }
          const int need = __shfl_sync(0xffffffffu, off, l0 + pages - 1);
          const bool all_in = __all_sync(0xffffffffu, !mine || whole);
          const int total = __reduce_add_sync(0xffffffffu, mine ? bytes : 0);
          const int at = book(need);
          if (at < 0) { ok = false; break; }
          const int slot = it % kRawSlots;
          RawTile& rec = x.raw(slot);
          if (mine) {
            off += at - room;
            rec.page[r] = RawPage{off, whole ? -1 : off + (slice + 127) / 128 * 128, valid, cls};
          }
          if (lane == 0) {
            rec.pages = pages; rec.bf16 = wide; rec.first = tile == t0; rec.end = 0;
            rec.lo = jlo; rec.t = jt; rec.sinks = sinks; rec.all = all_in && pages << lg_p == kTileKeys;
          }
          __syncwarp();
          if (lane == 0) mbar_arrive_expect_tx(x.raw_full(slot), total);
          __syncwarp();
          if (mine) {
            uint8_t* to = x.base + L::kRing + off;
            bulk_g2s(to, src + a.hdr + static_cast<int64_t>(kvh) * slice, slice, x.raw_full(slot));
            if (!whole) bulk_g2s(to + (slice + 127) / 128 * 128, src, 4 * P, x.raw_full(slot));
          }
          ++it;
        }
      }
    }
  }
  if (ok) {  // no more tiles, no more segments
    ok = x.wait_warp(x.seg_empty(segs % kSegSlots), ((segs / kSegSlots) & 1) ^ 1);
    if (ok && lane == 0) {
      x.seg(segs % kSegSlots).tiles = 0;
      mbar_arrive(x.seg_full(segs % kSegSlots));
    }
    if (ok && book(0) >= 0) {
      if (lane == 0) {
        x.raw(it % kRawSlots).end = 1;
        mbar_arrive(x.raw_full(it % kRawSlots));
      }
      ++it;
    }
  }
  // the CTA stays until its copies have landed
  for (int k = max(0, it - kRawSlots); k < it; ++k) mbar_wait(x.raw_full(k % kRawSlots), (k / kRawSlots) & 1);
}

// Chunk e (8 elements) of row `key` of an expanded tile.
__device__ __forceinline__ uint8_t* tile_chunk(uint8_t* tile, int key, int e) {
  return tile + (e >> 3) * (kTileKeys * 128) + key * 128 + (((e ^ key) & 7) << 4);
}

// z + c s of eight codes, given as four words of two binary16 values 1024 + c, rounded once.
__device__ __forceinline__ uint4 expand8(uint32_t p0, uint32_t p1, uint32_t p2, uint32_t p3, __half2 s, __half2 z) {
  const __half2 k = as_half2(0x64006400u);  // 1024: the difference is exact
  return make_uint4(as_u32(__hfma2(__hsub2(as_half2(p0), k), s, z)), as_u32(__hfma2(__hsub2(as_half2(p1), k), s, z)),
                    as_u32(__hfma2(__hsub2(as_half2(p2), k), s, z)), as_u32(__hfma2(__hsub2(as_half2(p3), k), s, z)));
}

__device__ __forceinline__ void store16(uint32_t smem, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(smem), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// 32 elements of one group into the four chunks at `to`, which differ in the two lowest bits of
// their place in a line only.  codes: chunk i of an 8-bit row lies at 16 i ^ flip.
template <int B>
__device__ __forceinline__ void expand32(const uint8_t* codes, int flip, __half2 s, __half2 z, uint32_t to) {
  if (B == 8) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 raw = *reinterpret_cast<const uint4*>(codes + (16 * i ^ flip));
      const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
      for (int q = 0; q < 2; ++q)
        store16(to ^ (32 * i + 16 * q),
                expand8(__byte_perm(w[2 * q], 0x64646464u, 0x4140), __byte_perm(w[2 * q], 0x64646464u, 0x4342),
                        __byte_perm(w[2 * q + 1], 0x64646464u, 0x4140), __byte_perm(w[2 * q + 1], 0x64646464u, 0x4342), s, z));
    }
  } else if (B == 4) {
    const uint4 raw = *reinterpret_cast<const uint4*>(codes);
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t t[4];  // elements k and k + 4
#pragma unroll
      for (int k = 0; k < 4; ++k) t[k] = ((w[q] >> (4 * k)) & 0x000F000Fu) | 0x64006400u;
      store16(to ^ 16 * q, expand8(__byte_perm(t[0], t[1], 0x5410), __byte_perm(t[2], t[3], 0x5410), __byte_perm(t[0], t[1], 0x7632),
                                   __byte_perm(t[2], t[3], 0x7632), s, z));
    }
  } else {
    const uint2 raw = *reinterpret_cast<const uint2*>(codes);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const uint32_t w = q ? raw.y : raw.x;
      uint32_t t[8];  // elements k and k + 8
#pragma unroll
      for (int k = 0; k < 8; ++k) t[k] = ((w >> (2 * k)) & 0x00030003u) | 0x64006400u;
      store16(to ^ 32 * q, expand8(__byte_perm(t[0], t[1], 0x5410), __byte_perm(t[2], t[3], 0x5410), __byte_perm(t[4], t[5], 0x5410),
                                   __byte_perm(t[6], t[7], 0x5410), s, z));
      store16(to ^ (32 * q + 16), expand8(__byte_perm(t[0], t[1], 0x7632), __byte_perm(t[2], t[3], 0x7632), __byte_perm(t[4], t[5], 0x7632),
                                          __byte_perm(t[6], t[7], 0x7632), s, z));
    }
  }
}

// The same one element at a time, for a group whose largest level rounds past binary16's
// largest value: such a value stays at it.
__device__ __noinline__ void expand32_capped(const uint8_t* codes, int flip, int b, uint32_t sz, uint32_t to) {
  const float s = __low2float(as_half2(sz)), z = __high2float(as_half2(sz));
#pragma unroll 1
  for (int i = 0; i < 32; ++i) {
    const int bit = i * b, at = bit >> 3;
    const int code = (codes[b == 8 ? at ^ flip : at] >> (bit & 7)) & ((1 << b) - 1);
    const float v = fminf(fmaxf(z + code * s, -65504.f), 65504.f);
    asm volatile("st.shared.b16 [%0], %1;" ::"r"((to ^ (i >> 3) * 16) + 2 * (i & 7)), "h"(__half_as_ushort(__float2half_rn(v))) : "memory");
  }
}

// A lane's units of a token's row: every other 32 of its dimensions.
template <int D, int B>
__device__ __forceinline__ void expand_row(const uint8_t* sl, const uint32_t* sz, int o, bool swz, int lg_units, bool zero, int odd, uint32_t to) {
#pragma unroll 1
  for (int i = 0; i < D / 64; ++i, to += kTileKeys * 128) {
    const int u = 2 * i + odd, ou = o + u * 4 * B;
    if (zero) {
      for (int q = 0; q < 4; ++q) store16(to ^ 16 * q, make_uint4(0, 0, 0, 0));
      continue;
    }
    const uint32_t w = sz[u >> lg_units];
    // permuted rows of 8 bits: the bits that the chunks' order in their line of 128 bytes flips
    const int flip = B == 8 && swz ? (ou >> 3) & 0x70 : 0;
    const uint8_t* codes = sl + (ou ^ (flip & 0x60));
    const __half2 s = as_half2(__byte_perm(w, 0, 0x1010)), z = as_half2(__byte_perm(w, 0, 0x3232));
    const __half2 top = __hfma2(__float2half2_rn(static_cast<float>((1 << B) - 1)), s, z);
    if ((as_u32(top) & 0x7C00u) == 0x7C00u) expand32_capped(codes, flip & 0x10, B, w, to);
    else expand32<B>(codes, flip & 0x10, s, z, to);
  }
}

// The expanding warps: warps 0-7 write K, 8-15 V, each of 16 tokens.  Two lanes share a token
// and 64 dimensions of its row, so that eight lanes' chunks of a store lie in eight banks.
template <int D>
__device__ __forceinline__ void group_expand(const GroupArgs& g, const Ctx<D>& x, int warp, int lane) {
  using L = GroupSmem<D>;
  const LayerArgs& a = g.a;
  const int which = warp >> 3, key0 = (warp & 7) * 16, key = key0 + (lane >> 1), P = a.P, lg_p = __ffs(P) - 1, ng = D / a.G;
  const int lg_units = __ffs(a.G) - 6;  // log2 of a group's units of 32 dimensions
  const uint8_t* ring = x.base + L::kRing;
  for (int it = 0;; ++it) {
    const int slot = it % kRawSlots, stage = it % L::kStages;
    if (!x.wait_warp(x.raw_full(slot), (it / kRawSlots) & 1)) return;
    if (!x.wait_warp(x.kv_empty(which, stage), ((it / L::kStages) & 1) ^ 1)) return;
    const RawTile& r = x.raw(slot);
    TileMeta& m = x.meta(it % kMetaSlots);
    const bool end = r.end;
    if (!end) {
      const int keys = r.pages << lg_p;
      if (warp == 0 && lane == 0) m.keys = keys, m.bf16 = r.bf16, m.first = r.first, m.end = 0, m.all = r.all;
      if (key0 < keys) {  // a page holds 16 tokens or more: all 16 of the warp are in one
        const RawPage pg = r.page[key0 >> lg_p];
        bool seen = true;
        if (pg.pos >= 0) {
          const int at = (key0 & (P - 1)) + (lane & 15), pos = reinterpret_cast<const int32_t*>(ring + pg.pos)[at];
          seen = at < pg.valid && pos <= r.t && (pos >= r.lo || pos < r.sinks);
        }
        const uint32_t mask = __ballot_sync(0xffffffffu, seen) & 0xFFFFu;
        if (which == 0 && lane == 0) m.mask[warp] = static_cast<uint16_t>(mask);
        uint8_t* tile = x.base + (2 * stage + which) * L::kTile;
        const uint8_t* sl = ring + pg.off;
        if (r.bf16) {  // rows copied 16 bytes at a time, consecutive lanes along a row
          const int flip = a.swz ? 0x70 : 0;
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            constexpr int kN = D / 8;
            const int row = (i * 32 + lane) / kN, e = (i * 32 + lane) % kN, k = key0 + row;
            uint4 v = make_uint4(0, 0, 0, 0);  // a V row out of sight is zero: its weight of 0 times infinity would not be
            if (which == 0 || (mask >> row & 1)) {
              const int o = (which * P + (k & (P - 1))) * D * 2 + 16 * e;
              v = *reinterpret_cast<const uint4*>(sl + (o ^ ((o >> 3) & flip)));
            }
            *reinterpret_cast<uint4*>(tile_chunk(tile, k, e)) = v;
          }
        } else {
          const int row = (D / 8) << (pg.cls + 1), at = which * P + (key & (P - 1)), odd = lane & 1;
          const uint32_t* sz = reinterpret_cast<const uint32_t*>(sl + 2 * P * row) + at * ng;
          const bool zero = which == 1 && !(mask >> (lane >> 1) & 1);
          const uint32_t to = x.tile(stage, which) + key * 128 + (((4 * odd ^ key) & 7) << 4);
          if (pg.cls == 0) expand_row<D, 2>(sl, sz, at * row, false, lg_units, zero, odd, to);
          else if (pg.cls == 1) expand_row<D, 4>(sl, sz, at * row, false, lg_units, zero, odd, to);
          else expand_row<D, 8>(sl, sz, at * row, a.swz, lg_units, zero, odd, to);
        }
      } else if (which == 0 && lane == 0) {
        m.mask[warp] = 0;
      }
      fence_proxy_async_smem();
    } else if (warp == 0 && lane == 0) {
      m.end = 1;
    }
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(x.raw_empty(slot));
      mbar_arrive(x.kv_full(which, stage));
    }
    if (end) return;
  }
}

// The warp that issues the products (one elected lane does; the whole warp goes along, so that
// addresses and descriptors stay in uniform registers).  Tile it's scores are issued before tile
// it-1's P V, so that the tensor core works while the softmax does; K's place is free again once
// its scores are, V's once its product is.
template <int D>
__device__ __forceinline__ void group_mma(const Ctx<D>& x) {
  using L = GroupSmem<D>;
  int segs = 0, keys_before = 0;
  bool bf16_before = false, first_before = false, pending = false;
  auto pv = [&](int it) -> bool {  // O += P V of tile it
    const int stage = it % L::kStages;
    if (!x.wait_warp(x.kv_full(1, stage), (it / L::kStages) & 1) || !x.wait_warp(x.p_full(it & 1), (it >> 1) & 1)) return false;
    tc_fence_after();
    const uint32_t id = tc_idesc(bf16_before, D, true);
    const uint64_t d = tc_desc(x.tile(stage, 1), kTileKeys * 128);
    const uint32_t p = x.tmem + kColS + 128 * (it & 1);  // 16 weights in 8 columns
    if (elected()) {
#pragma unroll
      for (int k = 0; k < kTileKeys / 16; ++k)
        if (16 * k < keys_before) tc_mma(x.tmem + kColO, p + 8 * k, d + k * (2048 >> 4), id, k > 0 || !first_before);
      if (bf16_before) {  // the weights' low parts
#pragma unroll
        for (int k = 0; k < kTileKeys / 32; ++k)
          if (16 * k < keys_before) tc_mma(x.tmem + kColO, p + kColPLow + 8 * k, d + k * (2048 >> 4), id, true);
      }
      tc_commit(x.kv_empty(1, stage));
      tc_commit(x.o_done(it & 1));
    }
    __syncwarp();
    pending = false;
    return true;
  };
  for (int it = 0;; ++it) {
    const int stage = it % L::kStages;
    if (!x.wait_warp(x.kv_full(0, stage), (it / L::kStages) & 1)) break;
    const TileMeta& m = x.meta(it % kMetaSlots);
    if (__shfl_sync(0xffffffffu, m.end, 0)) {
      if (pending) pv(it - 1);
      break;
    }
    const int keys = __shfl_sync(0xffffffffu, m.keys, 0);
    const bool bf16 = __shfl_sync(0xffffffffu, m.bf16, 0), first = __shfl_sync(0xffffffffu, m.first, 0);
    if (it >= 2 && !x.wait_warp(x.o_done(it & 1), ((it - 2) >> 1) & 1)) break;  // tile it-2's weights, under the new scores, have been used
    if (first) {
      if (pending && !pv(it - 1)) break;
      if (!x.wait_warp(x.q_full(), segs & 1)) break;
      ++segs;
    }
    tc_fence_after();
    const uint32_t id = tc_idesc(bf16, keys, false);
    const uint32_t qcol = x.tmem + kColQ + (bf16 ? 64 : 0);
    const uint64_t d = tc_desc(x.tile(stage, 0), 16);
    if (elected()) {
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
        tc_mma(x.tmem + kColS + 128 * (it & 1), qcol + 8 * k, d + (((k >> 2) * (kTileKeys * 128) + (k & 3) * 32) >> 4), id, k > 0);
      tc_commit(x.s_full(it & 1));
      tc_commit(x.kv_empty(0, stage));
    }
    __syncwarp();
    if (pending && !pv(it - 1)) break;
    pending = true;
    keys_before = keys; bf16_before = bf16; first_before = first;
  }
  if (elected()) tc_commit(x.drained());  // nothing is in flight when the CTA ends
  __syncwarp();
  mbar_wait(x.drained(), 0);
}

// Scores out of sight become -infinity: their weight is 0 and they are no maximum.
template <int N>
__device__ __forceinline__ void mask_scores(uint32_t (&s)[N], const uint16_t* masks) {
#pragma unroll
  for (int k = 0; k < N / 16; ++k) {
    const uint32_t mask = masks[k];
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!(mask >> i & 1)) s[16 * k + i] = 0xFF800000u;
  }
}

// The softmax warps.  Warps w and w + 4 share 32 rows (lanes of TMEM); of the tokens of a tile
// that their copy of the rows takes, the first has the first half, the second the other.
template <int D>
__device__ __forceinline__ void group_softmax(const GroupArgs& g, const Ctx<D>& x, int warp, int lane) {
  using L = GroupSmem<D>;
  const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane, heads = g.a.Hq / g.a.Hkv;
  const uint32_t lanes = x.tmem + (static_cast<uint32_t>(quad) << 21);  // the warp's 32 lanes
  float* scratch = reinterpret_cast<float*>(x.base + L::kScratch) + half * kRows * 17;
  float2* ml = reinterpret_cast<float2*>(x.base + L::kMl);
  float* tops = reinterpret_cast<float*>(x.base + L::kTops);
  uint32_t meets = 0;
  auto meet = [&]() -> bool {  // the softmax warps wait for one another (bounded, unlike a CTA barrier)
    __syncwarp();
    if (lane == 0) mbar_arrive(x.merged());
    return x.wait_warp(x.merged(), meets++ & 1);
  };

  // (query, head) of row r of a segment
  auto row_of = [&](const Segment& sg, int r, int* query, int* head) {
    const int rr = sg.row0 + r;
    *query = sg.kind == 0 ? g.list[sg.qbase + rr / heads] : sg.qbase;
    *head = sg.kvh * heads + rr % heads;
  };
  // Half of the row's dimensions of Q into TMEM; the row's factor from products to base-2
  // exponents.  Each row is scaled by a power of two that brings its largest element to [1, 2):
  // binary16 then holds what it needs of it.
  float factor = 0.f;
  auto load_q = [&](const Segment& sg, int copies) {
    const int r = row & (kRows / copies - 1);
    uint32_t w[D / 4];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < D / 4; ++i) w[i] = 0;
    if (r < sg.rows) {
      int query, head;
      row_of(sg, r, &query, &head);
      const uint4* src = reinterpret_cast<const uint4*>(g.q + (static_cast<int64_t>(query) * g.a.Hq + head) * D);
      uint4 other[D / 16];
#pragma unroll
      for (int i = 0; i < D / 16; ++i) other[i] = src[(half ^ 1) * (D / 16) + i];
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const uint4 u = src[half * (D / 16) + i];
        w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
      }
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const uint32_t v[4] = {other[i].x, other[i].y, other[i].z, other[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          top = max(top, max(v[k] & 0x7FFFu, (v[k] >> 16) & 0x7FFFu));
          top = max(top, max(w[4 * i + k] & 0x7FFFu, (w[4 * i + k] >> 16) & 0x7FFFu));
        }
      }
    }
    int e = top == 0 || top >= 0x7F80u ? 0 : static_cast<int>(top >> 7) - 127;
    e = max(-100, min(120, e));
    const float down = __int_as_float((127 - e) << 23);
    factor = fmaxf(g.scale_log2 * __int_as_float((127 + e) << 23), 1.17549435e-38f);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      uint32_t o[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) o[k] = pack16(false, bf16lo(w[16 * i + k]) * down, bf16hi(w[16 * i + k]) * down);
      tmem_st(lanes + kColQ + half * (D / 4) + 16 * i, o);
#pragma unroll
      for (int k = 0; k < 16; ++k) o[k] = pack16(true, bf16lo(w[16 * i + k]) * down, bf16hi(w[16 * i + k]) * down);
      tmem_st(lanes + kColQ + 64 + half * (D / 4) + 16 * i, o);
    }
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(x.q_full());
  };

  int it = 0, segs = 0;
  if (!x.wait_warp(x.seg_full(0), 0)) return;
  Segment sg = x.seg(0);
  int copies = copies_of(sg.rows);
  if (sg.tiles > 0) load_q(sg, copies);
  while (sg.tiles > 0) {
    const float f = factor;
    float m = -INFINITY, l = 0.f;
    // One tile; N: the scores of this thread (64, 32 or 16 with 1, 2 or 4 copies of the rows).
    auto one_tile = [&](auto n, int tile) -> bool {
      constexpr int N = decltype(n)::value, kCopies = 64 / N;
      if (!x.wait_warp(x.s_full(it & 1), (it >> 1) & 1)) return false;
      tc_fence_after();
      const TileMeta& meta = x.meta(it % kMetaSlots);
      const uint32_t scol = lanes + kColS + 128 * (it & 1);
      const int copy = quad * kCopies / 4, c0 = copy * 2 * N + half * N;  // this thread's first token
      uint32_t s[N];
      tmem_ld(s, scol + c0);
      if (!meta.all) mask_scores(s, meta.mask + c0 / 16);
      float top = highest(s);
      // the row's maximum over both warps; behind it, all scores have been read
      float* xch = tops + (it & 1) * 2 * kRows;
      xch[half * kRows + row] = top;
      __syncwarp();
      if (lane == 0) mbar_arrive(x.pair(quad));
      if (!x.wait_warp(x.pair(quad), it & 1)) return false;
      top = fmaxf(top, xch[(half ^ 1) * kRows + row]) * f;
      // m follows the maximum only when that has grown by more than 2^8: p stays within binary16, and O is rarely rescaled
      if (__any_sync(0xffffffffu, top > m + 8.f)) {
        const float next = fmaxf(m, top), by = m == -INFINITY ? 0.f : exp2_approx(m - next);
        l *= by;
        m = next;
        if (tile > 0) {  // half of O's columns each
          if (!x.wait_warp(x.o_done((it - 1) & 1), ((it - 1) >> 1) & 1)) return false;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[16];
            const uint32_t at = lanes + kColO + half * (D / 2) + 16 * c;
            tmem_ld(o, at);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * by);
            tmem_st(at, o);
          }
        }
      }
      l += weigh(s, f, m == -INFINITY ? 0.f : -m);
      // weights over the scores, two to a column; none on the tokens of the other copies.  Of 16-bit
      // pages, whose values are exact, a weight is a sum of two bf16 numbers (16 bits, where one has 8).
      auto rest = [&](uint32_t col) {
        if (kCopies > 1) {
          const uint32_t none[N / 2] = {};
#pragma unroll
          for (int k = 1; k < kCopies; ++k) tmem_st(col + ((copy + k) % kCopies * 2 * N + half * N) / 2, none);
        }
      };
      if (meta.bf16) {
#pragma unroll
        for (int c = 0; c < N / 2; c += 8) {
          uint32_t high[8], low[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float a = __uint_as_float(s[2 * (c + i)]), b = __uint_as_float(s[2 * (c + i) + 1]);
            high[i] = pack16(true, a, b);
            low[i] = pack16(true, a - bf16lo(high[i]), b - bf16hi(high[i]));
          }
          tmem_st(scol + c0 / 2 + c, high);
          tmem_st(scol + kColPLow + c0 / 2 + c, low);
        }
        rest(scol + kColPLow);
      } else {
        uint32_t p[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) p[i] = pack16(false, __uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1]));
        tmem_st(scol + c0 / 2, p);
      }
      rest(scol);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(x.p_full(it & 1));
      return true;
    };
    for (int tile = 0; tile < sg.tiles; ++tile, ++it) {
      const bool ok = copies == 1 ? one_tile(std::integral_constant<int, 64>(), tile)
                                  : copies == 2 ? one_tile(std::integral_constant<int, 32>(), tile) : one_tile(std::integral_constant<int, 16>(), tile);
      if (!ok) return;
    }
    // the next segment's rows go in while this one's last product runs
    const Segment done = sg;
    const int done_copies = copies;
    ++segs;
    if (!x.wait_warp(x.seg_full(segs % kSegSlots), (segs / kSegSlots) & 1)) return;
    sg = x.seg(segs % kSegSlots);
    copies = copies_of(sg.rows);
    if (sg.tiles > 0) load_q(sg, copies);
    if (!x.wait_warp(x.o_done((it - 1) & 1), ((it - 1) >> 1) & 1)) return;
    tc_fence_after();

    // rows out: the output itself, or (m, l, o) for the join.  Both warps of a row have its m and
    // half of its l; copies have their own of both.
    ml[half * kRows + row] = make_float2(m, l);
    if (!meet()) return;
    if (done.dest >= 0) {  // a piece: the join takes the copies' rows one by one
      const int64_t slot = static_cast<int64_t>(done.dest) * kRows + row;
      if (half == 0) g.part_ml[slot] = make_float2(m, l + ml[kRows + row].y);
      float* to = g.part_o + slot * D + half * (D / 2);
      const bool live = (row & (kRows / done_copies - 1)) < done.rows;
#pragma unroll 1
      for (int c = 0; c < D / 64; ++c) {
        uint32_t o[32];
        tmem_ld(o, lanes + kColO + half * (D / 2) + 32 * c);
        if (live) {
#pragma unroll
          for (int i = 0; i < 32; i += 8)  // a lane's row: whole sectors
            st_global8(to + 32 * c + i, reinterpret_cast<const float*>(o + i));
        }
      }
    } else {
    const int width = kRows / done_copies;
    const int r = row / done_copies, cols = 16 / done_copies, c0 = (row % done_copies) * cols;  // what this thread writes of 16 columns
    float high = -INFINITY, sum = 0.f;
    for (int k = 0; k < done_copies; ++k) high = fmaxf(high, ml[r + k * width].x);
    for (int k = 0; k < done_copies; ++k) {
      const float2 v = ml[r + k * width];
      if (v.x != -INFINITY) sum += (v.y + ml[kRows + r + k * width].y) * exp2_approx(v.x - high);
    }
    float own_high = -INFINITY;  // of the row whose columns of O this thread reads
    for (int k = 0; k < done_copies; ++k) own_high = fmaxf(own_high, ml[(row & (width - 1)) + k * width].x);
    const float weight = m == -INFINITY ? 0.f : exp2_approx(m - own_high);
    int query = 0, head = 0;
    const bool live = r < done.rows;
    if (live) row_of(done, r, &query, &head);
    const int64_t at = static_cast<int64_t>(query) * g.a.Hq + head, home = static_cast<int64_t>(done.kind) * g.n * g.a.Hq + at;
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    if (live && c0 == 0 && half == 0 && done.dest == -1) g.home_ml[home] = make_float2(high, sum);
    auto put = [&](int col, const float4 v) {
      if (done.dest == -2)
        *reinterpret_cast<uint2*>(g.out + at * D + col) = make_uint2(pack16(true, v.x * inv, v.y * inv), pack16(true, v.z * inv, v.w * inv));
      else *reinterpret_cast<float4*>(g.home_o + home * D + col) = v;
    };
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t o[16];
      const int col = half * (D / 2) + 16 * c;
      tmem_ld(o, lanes + kColO + col);
      if (done_copies == 1) {
        if (live) {
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            put(col + i, make_float4(__uint_as_float(o[i]), __uint_as_float(o[i + 1]), __uint_as_float(o[i + 2]), __uint_as_float(o[i + 3])));
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) scratch[row * 17 + i] = m == -INFINITY ? 0.f : __uint_as_float(o[i]) * weight;
        if (!meet()) return;
        if (live)
          for (int i = 0; i < cols; i += 4) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            for (int k = 0; k < done_copies; ++k)
#pragma unroll
              for (int u = 0; u < 4; ++u) v[u] += scratch[(r + k * width) * 17 + c0 + i + u];
            put(col + c0 + i, make_float4(v[0], v[1], v[2], v[3]));
          }
        if (!meet()) return;
      }
    }
    }
    if (!meet()) return;  // (m, l) and O have been read
    tc_fence_before();
    if (lane == 0) mbar_arrive(x.seg_empty((segs - 1) % kSegSlots));
  }
}

template <int D>
__global__ void __launch_bounds__(kGroupThreads, 1) group_attn_kernel(const __grid_constant__ GroupArgs g) {
  extern __shared__ uint8_t dyn[];
  using L = GroupSmem<D>;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  Ctx<D> x;
  x.base = dyn + ((1024 - (smem_u32(dyn) & 1023)) & 1023);
  x.wait_ns = g.a.wait_ns;
  x.abort_flag = &s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < kRawSlots; ++i) mbar_init(x.raw_full(i), 1), mbar_init(x.raw_empty(i), kExpandWarps);
    for (int i = 0; i < kSegSlots; ++i) mbar_init(x.seg_full(i), 1), mbar_init(x.seg_empty(i), kSoftmaxWarps);
    for (int i = 0; i < 2 * L::kStages; ++i) mbar_init(x.kv_full(0, i), kExpandWarps / 2), mbar_init(x.kv_empty(0, i), 1);  // K, V
    for (int i = 0; i < 2; ++i) mbar_init(x.s_full(i), 1), mbar_init(x.p_full(i), kSoftmaxWarps), mbar_init(x.o_done(i), 1);
    mbar_init(x.q_full(), kSoftmaxWarps);
    mbar_init(x.drained(), 1);
    mbar_init(x.merged(), kSoftmaxWarps);
    for (int i = 0; i < 4; ++i) mbar_init(x.pair(i), 2);
    fence_barrier_init();
  }
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x * g.head->per >= g.head->work) return;  // nothing for this CTA
  if (warp == kMmaWarp) tmem_alloc(&s_tmem);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  x.tmem = s_tmem;
  if (warp < kSoftmaxWarps) {
    registers_up<kSoftmaxRegisters>();
    group_softmax<D>(g, x, warp, lane);
  } else {
    registers_down<kOtherRegisters>();
    if (warp < kMmaWarp) group_expand<D>(g, x, warp - kSoftmaxWarps, lane);
    else if (warp == kProducer) group_produce<D>(g, x, lane);
    else if (warp == kMmaWarp) group_mma<D>(x);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_free(s_tmem);
  if (threadIdx.x == 0 && s_abort) set_status(g.a.ctrl, TRR_ERR_TIMEOUT);
}

}  // namespace trr
