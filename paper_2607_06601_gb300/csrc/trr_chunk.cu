// trr_chunk.cu - trr_chunk_attn: attention of chunks of new tokens over the paged cache.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(s_ij - m_i) / sum_j exp(s_ij - m_i),  s_ij = scale q_i k_j
// over the stored tokens j that query i sees: j <= t_i and (full, or j >= t_i-w_i+1, or j < sinks).
//
// A chunk's many queries read the same tokens, so those are brought back from their codes once, not
// once for each block of rows:
//   chunk_plan_kernel    a CTA per chunk: its queries sorted by mode (a block of rows then has one mode and
//                        reads no more than that mode sees), the positions that any of them sees, how
//                        many tokens are stored there.  Some more per chunk: what its tokens have in
//                        common (see there).  The CTA that ends last lays chunks end to end.
//   chunk_stage_kernel   the stored tokens in sight, in order of position, as tiles in the layout that the tensor
//                        core reads, in binary16: z + c s rounded once (11 bits against the 8 of the output), 16-bit
//                        values as they are, less what is common.  And each block's tiles.
//   chunk_attn_kernel    one CTA per SM; all blocks' tiles, for every KV head, laid end to end are cut into
//                        equal runs, so that a long segment is spread over CTAs and a CTA takes many short ones.
//   chunk_join_kernel    joins the parts of rows that were cut, (m, l, o) by m' = max m,
//                        l' = sum l 2^(m - m'), and so for o; puts back what was taken out of K and V.
//
// Alone, from cold caches, in us (plan, stage, attention, join): one chunk of 512 queries of 12 heads on 2048 tokens
// 11, 12, 19, 9; 32 chunks of 8 on 2048 tokens of 12 heads 11, 57, 45, 6; 4096 queries on themselves, 32 heads of 64,
// 14, 21, 98 to 101, 11; 2048 at the end of 32,768 tokens, 8 KV heads of 128, 11, 37, 555, 17.  Plan and join are chains
// of dependent loads and of code that is read for the first time; a launch's start hides behind its forerunner's end.
//   Staging is bound by the memory: 4.5 bits a value in and 16 out.  The 32 chunks above write 201 MB in 57 us, 4 TB/s
// with what is read, as reading back does, and the attention reads it at 4.6 TB/s.  Four CTAs an SM, a head's loads
// ahead: with two or three heads ahead that call, which took 130 us then, took 151 and 163, with 3 CTAs an SM 145, with 5
// no less.  At 64 registers 52 bytes a thread are spilled (80 loaded); the loop that takes out what is common spills
// 472 (692), and the 32 chunks above take 50 us more where keys have an offset.
//
// Tokens of which binary16 holds too little flag their chunk and KV head: a 16-bit value of 65536 and more, an infinity or
// NaN; a key further than 65504 from its offset; bits lost below 2^-24 in a 16-bit row of K or V that has nothing above 2^-14
// (of V: as it is scaled).  Rows of a flagged head are done one by one in binary32, from the pages, by the join kernel, since
// 0 times infinity would reach rows that do not see the token.  That takes 20 to 700 times as long (the header has figures).
#include <algorithm>
#include <climits>

#include "trr_chunk_tc.cuh"

namespace trr {

constexpr int kStageCtas = 4;  // CTAs of the staging kernel on an SM

// ------------------------------------------------------------------------------ plan --

// Errors of a call: the lowest failing query's, kept as INT_MAX - (16 query + error) so that 0 means none.
__device__ __forceinline__ void chunk_fail(const ChunkArgs& g, int query, int err) {
  atomicMax(g.a.ctrl + kChunkBad, INT_MAX - (16 * query + err));
}

// Sum over the CTA's threads before this one (and over all, in *total).  Every thread calls it.
__device__ __forceinline__ int64_t scan_before(int64_t x, int64_t* warp_sums, int64_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x / 32;
  int64_t s = x;
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = s;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int w = 0; w < warps; ++w) {
    if (w < warp) before += warp_sums[w];
    all += warp_sums[w];
  }
  *total = all;
  return before + s - x;
}

// What is common to the tokens of a channel, taken from eight of them that are spread over all that the sequence stores.  Any
// choice gives the same rows but for rounding.
//   Keys: binary16 rounds one by 2^-11 of itself, so where an offset is common to all keys of a channel, scores are off by 2^-11
// of what it adds to them, though it adds the same to all and changes no weight: with 50 added to keys of standard deviation
// 1, rows were up to 3 % off.  Keys are staged less an offset where the eight lie within a third of their middle; it is that middle.
// (Of normal numbers around 0 one channel in ten million passes for one with an offset.)
//   Values: binary16's steps end at 2^-24, so where a channel's are that small, its sums have few bits left or none, beside
// channels that are none the worse.  Where the eight are below 2^-12, values are staged times the power of two that brings
// their largest to 2^-8 (so that a value may be 2^23 times as large and be in binary16's range), and rows are divided by it as
// they are written.
// (With 16, and half as many channels a CTA, 32 chunks of 12 heads took 126.5 us against 125.)
constexpr int kSamples = 8;
// CTAs that share a chunk's channels out: a pass each, but no more than the GPU holds at once.
constexpr int kMostParts = 8, kMostCommonCtas = 512;
// By one of the CTAs that share a chunk's channels out; `part` of them.
__device__ __forceinline__ void find_common(const ChunkArgs& g, int chunk, int part) {
  __shared__ const uint8_t* s_page[kSamples];
  __shared__ int s_class[kSamples], s_slot[kSamples], s_total, s_moved[kPlanChunkThreads / 64];
  const LayerArgs& a = g.a;
  const int tid = threadIdx.x, lg_group = __ffs(a.G) - 1, lg_d = __ffs(a.d) - 1, heads = kPlanChunkThreads >> lg_d;
  const int64_t head0 = static_cast<int64_t>(chunk) * 2 * a.Hkv;
  const int both = 2 * a.Hkv;  // K of each KV head, then V of each
  if (tid < kSamples) {
    const int seq = g.seq_ids[chunk];
    const bool none = g.offsets[chunk + 1] <= g.offsets[chunk] || seq < 0 || seq >= a.S;  // (or refused: nothing is staged then)
    const int64_t list = static_cast<int64_t>(none ? 0 : seq) * kClasses;
    int nt[kClasses], total = 0;
#pragma unroll
    for (int c = 0; c < kClasses; ++c) total += nt[c] = none ? 0 : a.ntok[list + c];
    int at = total > 0 ? static_cast<int>(static_cast<int64_t>(tid) * (total - 1) / (kSamples - 1)) : 0, cls = 0;
#pragma unroll
    for (int c = 0; c < kClasses - 1; ++c)
      if (cls == c && at >= nt[c]) at -= nt[c], cls = c + 1;
    if (total > 0) s_page[tid] = a.pool[cls] + a.pt[(list + cls) * a.MP + at / a.P] * a.page_bytes[cls] + a.hdr;
    s_class[tid] = cls;
    s_slot[tid] = at % a.P;
    if (tid == 0) s_total = total;
  }
  for (int x0 = part * kPlanChunkThreads; x0 < both * a.d; x0 += g.parts * kPlanChunkThreads) {
    const int x = x0 + tid, which = x >> lg_d >= a.Hkv, h = (x >> lg_d) - which * a.Hkv, j = x & (a.d - 1);
    if (tid < heads) s_moved[tid] = 0;
    __syncthreads();
    float lo = INFINITY, hi = -INFINITY;
    bool number = s_total > 0 && h < a.Hkv;
    if (number) {
      uint32_t w[kSamples], sz[kSamples];
#pragma unroll
      for (int s = 0; s < kSamples; ++s) {  // all loads first, of one form for every class
        const int c = s_class[s], row = a.d << (c + 1) >> 3, at = which * a.P + s_slot[s];
        const uint8_t* slice = s_page[s] + static_cast<int64_t>(h) * a.slice[c];
        int o = at * row + (j << (c + 1) >> 3);
        if (c >= 2 && a.swz) o = static_cast<int>(swz_off(o));
        w[s] = *reinterpret_cast<const uint16_t*>(slice + (o & ~1)) >> 8 * (o & 1);
        sz[s] = *reinterpret_cast<const uint32_t*>(slice + (c == 3 ? 0 : 2 * a.P * row + ((at << lg_d >> lg_group) + (j >> lg_group)) * 4));
      }
#pragma unroll
      for (int s = 0; s < kSamples; ++s) {
        const int lg = s_class[s] + 1, code = w[s] >> ((j << lg) & 7) & ((1 << (1 << lg)) - 1);
        const float k = lg == 4 ? __uint_as_float(w[s] << 16) : __fmaf_rn(static_cast<float>(code), __low2float(as_half2(sz[s])), __high2float(as_half2(sz[s])));
        number = number && fabsf(k) < 32768.f;
        lo = fminf(lo, k);
        hi = fmaxf(hi, k);
      }
    }
    const float middle = 0.5f * (lo + hi), top = fmaxf(hi, -lo);
    const bool moved = number && (which ? top > 0.f && top < 0x1p-12f : 3.f * (hi - lo) < fabsf(middle));
    float common = which ? 1.f : 0.f;
    if (moved) common = which ? __int_as_float((246 - static_cast<int>(__float_as_uint(top) >> 23)) << 23) : middle;
    // (an offset is rounded to binary16, a power of two is a bf16 number)
    if (h < a.Hkv) g.common[(head0 << lg_d) + x] = which ? __float_as_uint(common) >> 16 : __half_as_ushort(__float2half_rn(common));
    if (moved) s_moved[tid >> lg_d] = 1;
    __syncthreads();
    if (tid < heads && (x0 >> lg_d) + tid < both) {
      g.moved[head0 + (x0 >> lg_d) + tid] = s_moved[tid];
      if (s_moved[tid]) a.ctrl[kChunkMoved] = 1;
    }
  }
}

// One chunk: its queries in their places, what they see, how much is stored there.
__device__ __forceinline__ void plan_chunk(const ChunkArgs& g, int i, int seq, int start, int row0, int len, int err, int64_t* s_sums, int& s_lo,
                                           int (&s_before)[4][kClasses]) {
  const LayerArgs& a = g.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int h = tid; h < a.Hkv; h += kPlanChunkThreads) g.flag[static_cast<int64_t>(i) * a.Hkv + h] = 0;
  // a query's place: 0 full, 1 local, 2 a zero row
  auto kind_of = [&](int k, int* window) -> int {
    const int q = row0 + k, mode = g.modes[q];
    if (err) return 2;
    if (mode > TRR_MODE_FULL) {
      chunk_fail(g, q, TRR_ERR_INVALID_ARG);
      return 2;
    }
    if (mode == TRR_MODE_SKIP) return 2;
    if (mode == TRR_MODE_FULL) return 0;
    *window = g.windows ? g.windows[q] : g.window_scalar;
    if (*window >= 1) return 1;
    chunk_fail(g, q, TRR_ERR_INVALID_ARG);
    return 2;
  };
  // A thread takes some queries in a row, twice: to count each kind, and to put them in their places, queries of one kind
  // behind another, each kind in order.  (Short code: in a small call each first pass of an instruction costs.)
  const int share = (len + kPlanChunkThreads - 1) / kPlanChunkThreads, first = min(len, tid * share), last = min(len, first + share);
  constexpr int kCount = 21;  // bits of a count
  static_assert(kMostChunkTokens < 1 << kCount, "");
  int64_t kinds = 0, all = 0;
  int lo = INT_MAX;
#pragma unroll 1
  for (int k = first; k < last; ++k) {
    int w = 0;
    const int kind = kind_of(k, &w);
    kinds += 1ll << (kCount * kind);
    if (kind == 1) lo = min(lo, max(0, start + k - w + 1));
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  if (lane == 0) atomicMin(&s_lo, lo);
  const int64_t before = scan_before(kinds, s_sums, &all);
  auto count = [](int64_t x, int kind) { return static_cast<int>(x >> (kCount * kind) & ((1 << kCount) - 1)); };
  const int full = count(all, 0), local = count(all, 1);
  int place[3] = {row0 + count(before, 0), row0 + full + count(before, 1), row0 + full + local + count(before, 2)};
#pragma unroll 1
  for (int k = first; k < last; ++k) {
    int w = 0;
    const int kind = kind_of(k, &w);
    g.list[kind == 0 ? place[0] : kind == 1 ? place[1] : place[2]] = row0 + k;
    place[0] += kind == 0;
    place[1] += kind == 1;
    place[2] += kind == 2;
  }
  // the positions in sight of any query, and the tokens stored there
  const bool reads = full + local > 0;
  lo = full > 0 ? 0 : s_lo;
  const int end = start + len, sinks = reads ? min(g.sinks, lo) : 0;
  static_assert(kPlanChunkThreads / 32 == 4 * kClasses, "a warp for each class of four positions");
  if (reads) {
    const int which = warp / kClasses, before = tokens_before(a, seq, warp % kClasses, which == 0 ? sinks : which == 1 ? lo : which == 2 ? end : min(g.sinks, end), lane);
    if (lane == 0) s_before[which][warp % kClasses] = before;
  }
  __syncthreads();
  const int heads = a.Hq / a.Hkv;
  if (tid == 0) {
    ChunkPlan c = {};
    c.seq = seq; c.start = start; c.len = len; c.row0 = row0;
    c.full = full; c.local = local;
    if (reads) {
      c.sinks = sinks; c.lo = lo; c.end = end; c.span = sinks + end - lo;
      for (int k = 0; k < kClasses; ++k) {
        c.dropped += s_before[1][k] - s_before[0][k];
        c.tokens += s_before[2][k] - s_before[1][k] + s_before[0][k];
        c.head += s_before[3][k];
      }
      c.tiles = (c.tokens + chunk_tile(a.d) - 1) / chunk_tile(a.d);
      c.units = (c.span + kSpan - 1) / kSpan;
      c.blocks = (full * heads + kBlockRows - 1) / kBlockRows + (local * heads + kBlockRows - 1) / kBlockRows;
    }
    g.chunk[i] = c;
  }
}

__global__ void __launch_bounds__(kPlanChunkThreads) chunk_plan_kernel(const __grid_constant__ ChunkArgs g) {
  __shared__ int s_bad, s_lo, s_before[4][kClasses], s_last;
  __shared__ int64_t s_sums[kPlanChunkThreads / 32];
  const LayerArgs& a = g.a;
  const int tid = threadIdx.x, i = blockIdx.x;
  if (tid == 0) s_bad = 0, s_lo = INT_MAX;
  pdl_wait();
  pdl_trigger();
  if (i >= g.n) {  // the CTAs behind the chunks' look for what their tokens have in common
    find_common(g, (i - g.n) / g.parts, (i - g.n) % g.parts);
  } else {
    __syncthreads();
    for (int x = tid; x <= g.n; x += kPlanChunkThreads) {
      const int o = g.offsets[x], next = x < g.n ? g.offsets[x + 1] : o;
      if (o < 0 || o > g.num_tokens || next < o) s_bad = 1;
    }
    const int begin = g.offsets[i], upto = g.offsets[i + 1], seq = g.seq_ids[i], start = g.starts[i];
    __syncthreads();
    const bool bad = s_bad;
    const int row0 = bad ? 0 : begin, len = bad ? 0 : upto - begin;
    const int err = bad ? TRR_ERR_INVALID_ARG : seq < 0 || seq >= a.S ? TRR_ERR_INVALID_ARG : start < 0 || start > a.maxctx - len ? TRR_ERR_BAD_POSITION : 0;
    if (tid == 0 && err && (bad || len > 0)) chunk_fail(g, row0, err);
    plan_chunk(g, i, seq, start, row0, len, err, s_sums, s_lo, s_before);
    if (tid == 0 && bad) a.ctrl[kChunkRefused] = 1;
  }
  __syncthreads();
  if (tid == 0) s_last = atom_add_acq_rel(a.ctrl + kChunkDone, 1) == g.n * (1 + g.parts) - 1;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  // the last CTA: chunks end to end
  int64_t tiles = 0, units = 0, blocks = 0;
  for (int x0 = 0; x0 < g.n; x0 += kPlanChunkThreads) {
    const int x = x0 + tid;
    int t = 0, u = 0, b = 0;
    if (x < g.n) {
      const volatile ChunkPlan* c = g.chunk + x;
      t = c->tiles; u = c->units; b = c->blocks;
    }
    int64_t all;
    const int64_t t0 = tiles + scan_before(t, s_sums, &all);
    tiles += all;
    const int64_t u0 = units + scan_before(u, s_sums, &all);
    units += all;
    const int64_t b0 = blocks + scan_before(b, s_sums, &all);
    blocks += all;
    if (x < g.n) {
      ChunkPlan* c = g.chunk + x;
      c->tile0 = static_cast<int>(min(t0, static_cast<int64_t>(INT_MAX)));
      c->unit0 = static_cast<int>(min(u0, static_cast<int64_t>(INT_MAX)));
      c->block0 = static_cast<int>(b0);
    }
  }
  if (tid == 0) {
    int whole = atomicExch(a.ctrl + kChunkRefused, 0) ? TRR_ERR_INVALID_ARG : 0;
    if (!whole && tiles > g.most_tiles) {  // the workspace is too small for what is stored
      whole = TRR_ERR_OUT_OF_MEMORY;
      chunk_fail(g, 0, whole);
    }
    ChunkHeader h = {};
    h.bad = whole;
    if (!whole) {
      h.blocks = static_cast<int>(blocks); h.units = static_cast<int>(units);
      const int stagers = kStageCtas * g.ctas;
      h.splits = units > 0 ? shares_of_heads(units, (a.Hkv + 1) / 2, stagers, copy_ns(5ll * a.Hkv * a.d, stagers)) : 1;
    }
    h.moved = atomicExch(a.ctrl + kChunkMoved, 0);
    *g.head = h;
    const int e = atomicExch(a.ctrl + kChunkBad, 0);
    if (e) set_status(a.ctrl, (INT_MAX - e) & 15);
    a.ctrl[kChunkDone] = 0;
  }
}

// ----------------------------------------------------------------------------- stage --

// z + c s of sixteen elements of class C as binary16, rounded once; a value past binary16's largest stays at it
// (a group's largest level may round past the largest value that the append takes).
template <int C>
__device__ __forceinline__ void expand_f16(const Codes16& x, uint4 (&v)[2]) {
  constexpr int B = 2 << C;
  const __half2 s = as_half2(__byte_perm(x.sz, 0, 0x1010)), z = as_half2(__byte_perm(x.sz, 0, 0x3232));
  const __half2 k = as_half2(0x64006400u), top = as_half2(0x7BFF7BFFu);  // 1024 (1024 + c is exact), 65504
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const uint32_t w0 = B == 8 ? (half ? x.w[0].z : x.w[0].x) : B == 4 ? (half ? x.w[0].y : x.w[0].x) : (half ? x.w[0].x >> 16 : x.w[0].x);
    uint32_t p[4];
    if (B == 8) {
      const uint32_t w1 = half ? x.w[0].w : x.w[0].y;
      p[0] = __byte_perm(w0, 0x64646464u, 0x4140); p[1] = __byte_perm(w0, 0x64646464u, 0x4342);
      p[2] = __byte_perm(w1, 0x64646464u, 0x4140); p[3] = __byte_perm(w1, 0x64646464u, 0x4342);
    } else if (B == 4) {
      uint32_t t[4];  // elements i and i + 4
#pragma unroll
      for (int i = 0; i < 4; ++i) t[i] = ((w0 >> (4 * i)) & 0x000F000Fu) | 0x64006400u;
      p[0] = __byte_perm(t[0], t[1], 0x5410); p[1] = __byte_perm(t[2], t[3], 0x5410);
      p[2] = __byte_perm(t[0], t[1], 0x7632); p[3] = __byte_perm(t[2], t[3], 0x7632);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = ((w0 >> (4 * i)) & 3u) | ((w0 << (14 - 4 * i)) & 0x30000u) | 0x64006400u;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = as_u32(__hmin2(__hfma2(__hsub2(as_half2(p[i]), k), s, z), top));
    v[half] = make_uint4(p[0], p[1], p[2], p[3]);
  }
}

// Eight bf16 values as binary16; their largest magnitude, and whether binary16 lacks bits of one.
__device__ __forceinline__ uint4 convert_f16(uint4 v, uint32_t* top, bool* lost) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = bf16lo(w[i]), b = bf16hi(w[i]);
    *top = max(*top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
    const uint32_t h = pack16(false, a, b);
    *lost |= __low2float(as_half2(h)) != a || __high2float(as_half2(h)) != b;
    w[i] = h;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The tiles that block b's rows see.
__device__ __forceinline__ void plan_block(const ChunkArgs& g, int b, int lane) {
  const LayerArgs& a = g.a;
  // its chunk: the last one whose first block is b or before it
  const int lo = last_not_above(g.n, b, lane, [&](int i) { return g.chunk[i].block0; });
  const ChunkPlan c = g.chunk[lo];
  const int heads = a.Hq / a.Hkv, full_blocks = (c.full * heads + kBlockRows - 1) / kBlockRows, T = chunk_tile(a.d);
  const bool local = b - c.block0 >= full_blocks;
  BlockPlan p = {};
  p.chunk = lo; p.local = local;
  p.tile0 = c.tile0; p.sinks = c.head;
  p.row = (b - c.block0 - (local ? full_blocks : 0)) * kBlockRows;
  p.rows = min(kBlockRows, (local ? c.local : c.full) * heads - p.row);
  p.query0 = c.row0 + (local ? c.full : 0);
  // its queries' first and last positions, and the first that any of them, and all of them, see past the sinks
  const int k0 = p.row / heads, k1 = (p.row + p.rows - 1) / heads;
  const int t0 = c.start + g.list[p.query0 + k0] - c.row0, t1 = c.start + g.list[p.query0 + k1] - c.row0;
  int from = 0, from_all = 0;
  if (local) {
    from = INT_MAX;
    for (int k = k0 + lane; k <= k1; k += 32) {
      const int q = g.list[p.query0 + k], lo_q = max(0, c.start + q - c.row0 - (g.windows ? g.windows[q] : g.window_scalar) + 1);
      from = min(from, lo_q);
      from_all = max(from_all, lo_q);
    }
    from = __reduce_min_sync(0xffffffffu, from);
    from_all = __reduce_max_sync(0xffffffffu, from_all);
  }
  const int head = local ? min(g.sinks, from) : 0;
  // ranks of five positions: lanes 0 .. 19, a class of a position each
  const int which = lane >> 2, x = which == 0 ? head : which == 1 ? from : which == 2 ? t1 + 1 : which == 3 ? from_all : t0 + 1;
  int r = lane < 20 ? place_of(a, c.seq, lane & 3, x).before : 0;
  r += __shfl_xor_sync(0xffffffffu, r, 1);
  r += __shfl_xor_sync(0xffffffffu, r, 2);
  if (x >= c.lo) r -= c.dropped;
  const int rank0 = __shfl_sync(0xffffffffu, r, 0), rank1 = __shfl_sync(0xffffffffu, r, 4), rank2 = __shfl_sync(0xffffffffu, r, 8);
  p.clean = (__shfl_sync(0xffffffffu, r, 12) + T - 1) / T;
  p.clean_end = __shfl_sync(0xffffffffu, r, 16) / T;
  p.head = (rank0 + T - 1) / T;
  p.first = rank1 / T;
  p.last = max(p.first, (rank2 + T - 1) / T);
  if (p.head >= p.first) p.head = p.first = 0;  // one stretch from the start
  p.tiles = p.head + p.last - p.first;
  if (p.tiles > 0) {
    const int whole = max(0, min(p.clean_end, p.last) - max(p.clean, p.first));
    p.tile_cost = (p.rows <= kHalfRows && a.d == 64 ? kChunkTurnsCost : kChunkTileCost) +
                  (kChunkMaskedCost * (p.tiles - whole) + p.tiles / 2) / p.tiles;
  }
  if (lane == 0) g.block[b] = p;
}

// Zero rows of heads h0 .. h1 - 1 of a query, by a warp.
__device__ __forceinline__ void zero_rows(const ChunkArgs& g, int q, int h0, int h1, int lane) {
  const int64_t at = static_cast<int64_t>(q) * g.a.Hq + h0;
  uint4* out = reinterpret_cast<uint4*>(g.out + at * g.a.d);
  for (int i = lane; i < (h1 - h0) * g.a.d / 8; i += 32) out[i] = make_uint4(0, 0, 0, 0);
  if (g.lse)
    for (int h = lane; h < h1 - h0; h += 32) g.lse[at + h] = -INFINITY;
}

// Sixteen elements of a token's K less their offset, or of its V times their powers of two, from binary32 rounded once to
// binary16; their largest magnitude's bits, and whether binary16 lacks bits of one.
template <int C, int D>
__device__ __forceinline__ void expand_moved(const Codes16& x, int which, const uint16_t* common, uint4 (&v)[2], uint32_t* top, bool* lost) {
  float y[16];
  expand_f32<C>(x, y);
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const uint4 c = reinterpret_cast<const uint4*>(common)[half];
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a = y[8 * half + 2 * i], b = y[8 * half + 2 * i + 1];
      a = which ? a * bf16lo(w[i]) : a - __low2float(as_half2(w[i]));
      b = which ? b * bf16hi(w[i]) : b - __high2float(as_half2(w[i]));
      o[i] = pack16(false, a, b);
      *top = max(*top, max(__float_as_uint(a) & 0x7FFFFFFFu, __float_as_uint(b) & 0x7FFFFFFFu));
      if (C == 3) *lost |= __low2float(as_half2(o[i])) != a || __high2float(as_half2(o[i])) != b;
    }
    v[half] = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// A token's rows of every step-th head into its tile: 16 elements a lane of K and of V.  All lanes of the warp call it.
// (MOVED: what is common to some chunk's tokens is taken out.)
template <int C, int D, bool MOVED>
__device__ __forceinline__ void stage_token(const ChunkArgs& g, int chunk, const uint8_t* page, int slot, int row, bool live, int h0, int h1, int step, int e) {
  constexpr int T = chunk_tile(D), kLanes = D / 16;
  const CodesAt<C, D> at(g.a, slot, e);
  const int tile = row / T, r = row - tile * T;
  uint8_t* to = g.tile + static_cast<int64_t>(tile) * g.a.Hkv * (4 * T * D) + (tile_at(T, r, 2 * e) & ~31);
  const bool odd = r & 1;  // two chunks of a sector lie in the order of the row's place in its line
  const int64_t slice_bytes = g.a.slice[C];
  const uint8_t* slice = page + g.a.hdr + h0 * slice_bytes;
  // a head's codes are asked for before the last head's are written: nothing moves a load over a store by itself
  Codes16 next[2];
  if (h0 < h1) next[0] = at.load(slice, 0), next[1] = at.load(slice, 1);
#pragma unroll 1
  for (int h = h0; h < h1; h += step) {
    const Codes16 x[2] = {next[0], next[1]};
    slice += step * slice_bytes;
    if (h + step < h1) next[0] = at.load(slice, 0), next[1] = at.load(slice, 1);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      uint4 v[2];
      if (C == 3 || MOVED) {
        // beyond 65504 as binary32, 65536 as bf16; 2^-14
        constexpr uint32_t kPast = MOVED ? 0x477FE001u : 0x4780u, kNear = MOVED ? 0x38800000u : 0x3880u;
        uint32_t top = 0;
        bool lost = false;
        if (MOVED) {
          expand_moved<C, D>(x[which], which, common_of<D>(g, chunk, h, which) + 16 * e, v, &top, &lost);
        } else {
          v[0] = convert_f16(x[which].w[0], &top, &lost);
          v[1] = convert_f16(x[which].w[1], &top, &lost);
        }
        if (C == 3) {
#pragma unroll
          for (int o = 1; o < kLanes; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        }
        if (live && (top >= kPast || (lost && top < kNear))) {
          g.flag[static_cast<int64_t>(chunk) * g.a.Hkv + h] = 1;
          g.head->flagged = 1;
        }
      } else {
        expand_f16<C == 3 ? 0 : C>(x[which], v);
      }
      if (live) store_sector(to + (2 * h + which) * (2 * T * D), odd ? v[1] : v[0], odd ? v[0] : v[1]);
    }
  }
}

// The tokens that a CTA has found, of KV heads h0 .. h1 - 1.
template <int D, bool MOVED>
__device__ __forceinline__ void stage_unit(const ChunkArgs& g, const Found<32 / (D / 16)>& f, int chunk, int h0, int h1, int lg) {
  for_groups(f, lg, h0, [&](int k, const auto& tok, bool live, int h, int step) {
    const int e = threadIdx.x % (D / 16);
    if (k == 0) stage_token<0, D, MOVED>(g, chunk, tok.page, tok.slot, tok.row, live, h, h1, step, e);
    else if (k == 1) stage_token<1, D, MOVED>(g, chunk, tok.page, tok.slot, tok.row, live, h, h1, step, e);
    else if (k == 2) stage_token<2, D, MOVED>(g, chunk, tok.page, tok.slot, tok.row, live, h, h1, step, e);
    else stage_token<3, D, MOVED>(g, chunk, tok.page, tok.slot, tok.row, live, h, h1, step, e);
  });
}
// A CTA's units: 64 positions of a chunk's line, some of the KV heads.
template <int D, bool MOVED>
__device__ __forceinline__ void stage_units(const ChunkArgs& g, Found<32 / (D / 16)>& f, int units, int splits) {
  constexpr int T = chunk_tile(D);
  const LayerArgs& a = g.a;
  const int tid = threadIdx.x, lane = tid & 31;
  const int per = (a.Hkv + splits - 1) / splits;
  int chunk = -1;
  ChunkPlan c;
  for (int u = gridDim.x - 1 - blockIdx.x; u < units * splits; u += gridDim.x) {
    const int unit = u / splits, h0 = u % splits * per, h1 = min(a.Hkv, h0 + per);
    if (chunk < 0 || unit >= c.unit0 + c.units) {
      chunk = last_not_above(g.n, unit, lane, [&](int i) { return g.chunk[i].unit0; });
      c = g.chunk[chunk];
    }
    const int x = (unit - c.unit0) * kSpan + (tid >> 2), cls = tid & 3;
    const int pos = x < c.sinks ? x : x - c.sinks + c.lo;
    Place p{0, -1, 0};
    if (x < c.span) p = place_of(a, c.seq, cls, pos);
    // rank among the staged tokens: the sum over the classes
    int rank = p.before;
    rank += __shfl_xor_sync(0xffffffffu, rank, 1);
    rank += __shfl_xor_sync(0xffffffffu, rank, 2);
    const int row = c.tile0 * T + rank - (pos >= c.lo ? c.dropped : 0);
    f.gather(a, p, cls, p.page >= 0 ? row : -1, tid);
    stage_unit<D, MOVED>(g, f, chunk, h0, h1, lg_parts(per));
  }
}
// (Out of line, and called where nothing else is live, so that the loop without is as fast as if this were not there.)
template <int D>
__device__ __noinline__ void stage_moved_units(const ChunkArgs& g, Found<32 / (D / 16)>& f, int units, int splits) {
  stage_units<D, true>(g, f, units, splits);
}

template <int D>
__global__ void __launch_bounds__(kSpanThreads, kStageCtas) chunk_stage_kernel(const __grid_constant__ ChunkArgs g) {
  constexpr int T = chunk_tile(D);
  constexpr int kLanes = D / 16;
  __shared__ Found<32 / kLanes> f;
  __shared__ int64_t s_sums[kSpanThreads / 32];
  __shared__ int s_last;
  const LayerArgs& a = g.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_trigger();
  const ChunkHeader head = *g.head;
  if (head.bad) {
    for (int q = blockIdx.x * (kSpanThreads / 32) + warp; q < g.num_tokens; q += gridDim.x * (kSpanThreads / 32)) zero_rows(g, q, 0, a.Hq, lane);
    return;
  }
  // Three kinds of work, dealt out from the first CTA up, from the middle and from the last one down, so that in a small
  // call each CTA has one of them.  Blocks of rows first: the CTA that is done last lays them end to end.
  for (int b = blockIdx.x * (kSpanThreads / 32) + warp; b < head.blocks; b += gridDim.x * (kSpanThreads / 32)) plan_block(g, b, lane);
  __syncthreads();
  if (tid == 0) s_last = atom_add_acq_rel(a.ctrl + kChunkPlanned, 1) == static_cast<int>(gridDim.x) - 1;
  __syncthreads();
  if (s_last) {
    __threadfence();
    int64_t work = 0;
    bool empty = false;
    for (int x0 = 0; x0 < head.blocks; x0 += kSpanThreads) {
      const int x = x0 + tid;
      BlockPlan b = {};
      if (x < head.blocks) {
        b.tiles = reinterpret_cast<const volatile BlockPlan*>(g.block)[x].tiles;
        b.tile_cost = reinterpret_cast<const volatile BlockPlan*>(g.block)[x].tile_cost;
      }
      int64_t all;
      const int64_t before = work + scan_before(a.Hkv * chunk_cost(b), s_sums, &all);
      work += all;
      if (x < head.blocks) g.base[x] = before;
      empty |= x < head.blocks && b.tiles == 0;
    }
    empty = __syncthreads_or(empty);
    if (tid == 0) {
      g.head->empty = empty;
      g.base[head.blocks] = work;
      g.head->work = work;
      g.head->per = max((work + g.ctas - 1) / g.ctas, static_cast<int64_t>(kChunkLeastShare));
      a.ctrl[kChunkPlanned] = 0;
    }
  }
  // which staged tokens each query sees, by eight lanes: the classes of two positions; queries that read nothing have zero rows
  for (int k0 = ((blockIdx.x + gridDim.x / 2) % gridDim.x * (kSpanThreads / 32) + warp) * 4; k0 < g.num_tokens; k0 += gridDim.x * (kSpanThreads / 32) * 4) {
    const int k = k0 + lane / 8;
    int lo = 0, hi = g.n - 1;  // a place of the list: of the last chunk that starts at k or before it
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (g.chunk[mid].row0 <= k) lo = mid;
      else hi = mid - 1;
    }
    const ChunkPlan& p = g.chunk[lo];
    const bool mine = k < g.num_tokens && k >= p.row0 && k < p.row0 + p.len, reads = mine && k < p.row0 + p.full + p.local;
    const int q = mine ? g.list[k] : 0;
    int rank = 0;
    if (reads) {
      const int t = p.start + q - p.row0;
      const int from = k >= p.row0 + p.full ? max(0, t - (g.windows ? g.windows[q] : g.window_scalar) + 1) : 0, x = lane & 4 ? t + 1 : from;
      rank = place_of(a, p.seq, lane & 3, x).before - ((lane & 3) == 0 && x >= p.lo ? p.dropped : 0);
    }
    rank += __shfl_xor_sync(0xffffffffu, rank, 1);
    rank += __shfl_xor_sync(0xffffffffu, rank, 2);
    const int upto = __shfl_xor_sync(0xffffffffu, rank, 4);
    if (reads && (lane & 7) == 0) g.sight[k] = make_int2(rank, upto);
    for (uint32_t left = __ballot_sync(0xffffffffu, mine && !reads && (lane & 7) == 0); left; left &= left - 1)
      zero_rows(g, __shfl_sync(0xffffffffu, q, __ffs(left) - 1), 0, a.Hq, lane);
  }
  if (head.moved) stage_moved_units<D>(g, f, head.units, head.splits);
  else stage_units<D, false>(g, f, head.units, head.splits);
  // rows of a chunk's last tile past its tokens are zero (their weights are)
  for (int k = blockIdx.x; k < g.n; k += gridDim.x) {
    const ChunkPlan& p = g.chunk[k];
    const int at = p.tokens % T, tile = p.tile0 + p.tiles - 1;
    if (at == 0) continue;
    for (int j = 0; j < 2 * a.Hkv; ++j)
      for (int x = tid; x < (T - at) * (D / 8); x += kSpanThreads)
        *reinterpret_cast<uint4*>(staged_tile<D>(g, tile, j >> 1, j & 1) + tile_at(T, at + x / (D / 8), x % (D / 8))) = make_uint4(0, 0, 0, 0);
  }
}

// ------------------------------------------------------------------------------ rows --

// Element j of K (which 0) or V (1) of KV head h of a stored token, in binary32.
template <int D>
__device__ __forceinline__ float stored_value(const LayerArgs& a, int c, const uint8_t* page, int slot, int h, int which, int j, int lg_group) {
  const uint8_t* slice = page + a.hdr + static_cast<int64_t>(h) * a.slice[c];
  const int lg = c + 1, row = D << lg >> 3;  // 2^lg bits an element
  int64_t o = (static_cast<int64_t>(which) * a.P + slot) * row + (j << lg >> 3);
  if (c >= 2 && a.swz) o = swz_off(o);
  if (c == 3) return __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(slice + o)) << 16);
  const int code = slice[o] >> ((j << lg) & 7) & ((1 << (1 << lg)) - 1);
  const __half2 sz = as_half2(reinterpret_cast<const uint32_t*>(slice + 2 * a.P * row)[(which * a.P + slot) * (D >> lg_group) + (j >> lg_group)]);
  return __fmaf_rn(static_cast<float>(code), __low2float(sz), __high2float(sz));
}

// One row from the pages, by a warp: 32 tokens at a time, the statistics of the softmax running along.
template <int D>
__device__ __forceinline__ void one_row(const ChunkArgs& g, const ChunkPlan& ch, const RowSource& s, bool local, int kvh, int lane) {
  constexpr int E = D / 32;
  const LayerArgs& a = g.a;
  const int64_t at = static_cast<int64_t>(s.query) * a.Hq + s.head;
  const uint16_t* q = g.q + at * D;
  const int lg_group = __ffs(a.G) - 1;
  float o[E] = {}, m = -INFINITY, l = 0.f;
  for (int c = 0; c < kClasses; ++c) {
    const int64_t list = static_cast<int64_t>(ch.seq) * kClasses + c;
    const int nt = a.ntok[list];
    for (int k = 0; k * a.P < nt; ++k) {
      if (a.pfirst[list * a.MP + k] > s.t) break;
      const uint8_t* page = a.pool[c] + a.pt[list * a.MP + k] * a.page_bytes[c];
      for (int s0 = 0; s0 < min(a.P, nt - k * a.P); s0 += 32) {
        const int slot = s0 + lane;
        const int pos = slot < min(a.P, nt - k * a.P) ? reinterpret_cast<const int32_t*>(page)[slot] : INT_MAX;
        const bool see = pos <= s.t && (pos >= s.lo || (local && pos < g.sinks));
        uint32_t left = __ballot_sync(0xffffffffu, see);
        if (left == 0) continue;
        float d = -INFINITY;
        if (see) {
          d = 0.f;
          for (int j = 0; j < D; ++j) d += __uint_as_float(static_cast<uint32_t>(q[j]) << 16) * stored_value<D>(a, c, page, slot, kvh, 0, j, lg_group);
          d *= g.scale_log2;
        }
        float next = fmaxf(m, d);
        for (int x = 16; x > 0; x >>= 1) next = fmaxf(next, __shfl_xor_sync(0xffffffffu, next, x));
        const float by = m == next ? 1.f : exp2f(m - next), p = d == -INFINITY ? 0.f : exp2f(d - next);
        m = next;
        float sum = p;
        for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
        l = l * by + sum;
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] *= by;
        for (; left; left &= left - 1) {
          const int from = __ffs(left) - 1;
          const float w = __shfl_sync(0xffffffffu, p, from);
#pragma unroll
          for (int i = 0; i < E; ++i) o[i] += w * stored_value<D>(a, c, page, s0 + from, kvh, 1, lane * E + i, lg_group);
        }
      }
    }
  }
  const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int i = 0; i < E; i += 2) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(o[i] * inv, o[i + 1] * inv);
    *reinterpret_cast<__nv_bfloat162*>(g.out + at * D + lane * E + i) = x;
  }
  if (g.lse && lane == 0) g.lse[at] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// What the keys' offset adds to the scores of row `at` (query and head), in units of the natural logarithm, summed over elements
// first, first + step, ...: staged keys are less by it, which moves all of a row's scores by as much, no weight, and the
// logarithm of their sum.
template <int D>
__device__ __forceinline__ float moved_score(const ChunkArgs& g, int chunk, int kvh, int64_t at, int first, int step) {
  const uint16_t *q = g.q + at * D, *offset = common_of<D>(g, chunk, kvh, 0);
  float sum = 0.f;
#pragma unroll 1
  for (int j = first; j < D; j += step) sum += __uint_as_float(static_cast<uint32_t>(q[j]) << 16) * __half2float(__ushort_as_half(offset[j]));
  return sum * g.scale_log2 * 0.6931471805599453f;
}

// What was taken out of a row's K and V put back, by a warp.  V was staged times powers of two, by which a bf16 number is
// divided without a rounding.
template <int D>
__device__ __forceinline__ void put_back(const ChunkArgs& g, int chunk, int kvh, int64_t at, int lane) {
  if (g.lse && moved_head(g, chunk, kvh, 0)) {
    float sum = moved_score<D>(g, chunk, kvh, at, lane, 32);
    for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
    if (lane == 0 && g.lse[at] != -INFINITY) g.lse[at] += sum;
  }
  if (moved_head(g, chunk, kvh, 1)) {
    const uint16_t* power = common_of<D>(g, chunk, kvh, 1);
    for (int j = lane; j < D; j += 32) {
      uint16_t* o = g.out + at * D + j;
      *o = __bfloat16_as_ushort(__float2bfloat16_rn(__uint_as_float(static_cast<uint32_t>(*o) << 16) * one_over(power[j])));
    }
  }
}

// One row of a cut segment, by eight lanes: D / 8 values each.
template <int D>
__device__ __forceinline__ void join_row(const ChunkArgs& g, int cta, const PieceInfo& piece, int r, int lane, bool moved) {
  constexpr int E = D / 8;
  const int heads = g.a.Hq / g.a.Hkv, query = g.list[piece.query0 + (piece.row + r) / heads];
  // parts: the last one of CTA `cta`, the first ones of those that follow
  auto piece_of = [&](int j) { return 2 * j + (j == cta); };
  auto slot = [&](int j) { return static_cast<int64_t>(piece_of(j)) * kBlockRows + r; };
  const int end = cta + piece.ctas;
  float m = -INFINITY, l = 0.f, o[E] = {};
#pragma unroll 4
  for (int j = cta; j < end; ++j) m = fmaxf(m, g.part_ml[slot(j)].x);
#pragma unroll 2
  for (int j = cta; j < end; ++j) {
    const float2 ml = g.part_ml[slot(j)];
    const float w = ml.x == -INFINITY ? 0.f : exp2_approx(ml.x - m);
    float4 v[E / 4];
#pragma unroll
    for (int i = 0; i < E / 4; ++i) v[i] = *reinterpret_cast<const float4*>(part_at<D>(g, piece_of(j), lane + 8 * i, r));
    l += ml.y * w;
    if (w == 0.f) continue;  // (a part in which nothing was seen may hold anything)
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      o[4 * i] += v[i].x * w;
      o[4 * i + 1] += v[i].y * w;
      o[4 * i + 2] += v[i].z * w;
      o[4 * i + 3] += v[i].w * w;
    }
  }
  const int64_t at = static_cast<int64_t>(query) * g.a.Hq + piece.kvh * heads + (piece.row + r) % heads;
  const float inv = l != 0.f ? 1.f / l : 0.f;
  float score = 0.f;
  if (moved) {
    if (g.lse && moved_head(g, piece.chunk, piece.kvh, 0)) score = moved_score<D>(g, piece.chunk, piece.kvh, at, 0, 1);
    if (moved_head(g, piece.chunk, piece.kvh, 1)) {
      const uint16_t* power = common_of<D>(g, piece.chunk, piece.kvh, 1) + 4 * lane;
#pragma unroll
      for (int i = 0; i < E; ++i) o[i] *= one_over(power[i / 4 * 32 + i % 4]);
    }
  }
#pragma unroll
  for (int i = 0; i < E / 4; ++i)
    *reinterpret_cast<uint2*>(g.out + at * D + 32 * i + 4 * lane) =
        make_uint2(pack16(true, o[4 * i] * inv, o[4 * i + 1] * inv), pack16(true, o[4 * i + 2] * inv, o[4 * i + 3] * inv));
  if (g.lse && lane == 0) g.lse[at] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f + score : -INFINITY;
}

constexpr int kJoinCtas = 4;

template <int D>
__global__ void __launch_bounds__(256, kJoinCtas) chunk_join_kernel(const __grid_constant__ ChunkArgs g) {
  constexpr int kJoinRows = 256 / 8;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, bad = g.head->bad, blocks = g.head->blocks;
  const bool flagged = g.head->flagged, empty = g.head->empty, moved = g.head->moved;
  auto careful = [&](int chunk, int kvh) { return flagged && g.flag[static_cast<int64_t>(chunk) * g.a.Hkv + kvh]; };
  for (int x = blockIdx.x; x < g.ctas * (kBlockRows / kJoinRows); x += gridDim.x) {
    const int cta = x / (kBlockRows / kJoinRows), r = x % (kBlockRows / kJoinRows) * kJoinRows + threadIdx.x / 8;
    const PieceInfo piece = g.piece[cta];  // (none where the call is refused)
    if (piece.block >= 0 && r < piece.rows && !careful(piece.chunk, piece.kvh)) join_row<D>(g, cta, piece, r, threadIdx.x & 7, moved);
  }
  if (bad || !(flagged || empty || moved)) return;
  // rows with nothing stored in sight, those that are done one by one, and whole ones of which something was taken out
  for (int64_t x = blockIdx.x; x < static_cast<int64_t>(blocks) * g.a.Hkv * (kBlockRows / kJoinRows); x += gridDim.x) {
    const int64_t y = x / (kBlockRows / kJoinRows);
    const BlockPlan& b = g.block[y / g.a.Hkv];
    const int kvh = static_cast<int>(y % g.a.Hkv), r0 = static_cast<int>(x % (kBlockRows / kJoinRows)) * kJoinRows;
    const bool by_one = b.tiles > 0 && careful(b.chunk, kvh);
    if (b.tiles > 0 && !by_one && !(moved && chunk_uncut(g.base[y / g.a.Hkv] + kvh * chunk_cost(b), g.head->per, b))) continue;
    const ChunkPlan& c = g.chunk[b.chunk];
    for (int r = r0 + warp; r < min(b.rows, r0 + kJoinRows); r += 8) {
      const RowSource s = row_source(g, c, b.query0, b.local, kvh, b.row + r);
      if (b.tiles == 0) zero_rows(g, s.query, s.head, s.head + 1, lane);
      else if (by_one) one_row<D>(g, c, s, b.local, kvh, lane);
      else put_back<D>(g, b.chunk, kvh, static_cast<int64_t>(s.query) * g.a.Hq + s.head, lane);
    }
  }
}

// ----------------------------------------------------------------------------- calls --

static int64_t most_blocks(const Layout& l, int n, int num_tokens) {
  return static_cast<int64_t>(num_tokens) * (l.Hq / l.Hkv) / kBlockRows + 2 * static_cast<int64_t>(n);
}

// Lays the workspace out (b == nullptr: counts its bytes); the tiles take what is left of `bytes`.
static int64_t lay_workspace(ChunkArgs* g, uint8_t* b, const Layout& l, int n, int num_tokens, int ctas, int64_t most_tiles) {
  int64_t off = 0;
  auto take = [&](int64_t bytes) {
    uint8_t* p = b + off;
    off += (bytes + 255) / 256 * 256;
    return p;
  };
  const int64_t blocks = most_blocks(l, n, num_tokens);
  g->head = reinterpret_cast<ChunkHeader*>(take(sizeof(ChunkHeader)));
  g->chunk = reinterpret_cast<ChunkPlan*>(take(static_cast<int64_t>(sizeof(ChunkPlan)) * n));
  g->list = reinterpret_cast<int32_t*>(take(4ll * num_tokens));
  g->sight = reinterpret_cast<int2*>(take(8ll * num_tokens));
  g->block = reinterpret_cast<BlockPlan*>(take(static_cast<int64_t>(sizeof(BlockPlan)) * blocks));
  g->base = reinterpret_cast<int64_t*>(take(8 * (blocks + 1)));
  g->flag = reinterpret_cast<int32_t*>(take(4ll * n * l.Hkv));
  g->moved = reinterpret_cast<int32_t*>(take(8ll * n * l.Hkv));
  g->common = reinterpret_cast<uint16_t*>(take(4ll * n * l.Hkv * l.d));
  g->piece = reinterpret_cast<PieceInfo*>(take(static_cast<int64_t>(sizeof(PieceInfo)) * ctas));
  g->part_ml = reinterpret_cast<float2*>(take(8ll * 2 * ctas * kBlockRows));
  g->part_o = reinterpret_cast<uint4*>(take(4ll * 2 * ctas * kBlockRows * l.d));
  const int64_t fixed = off, T = chunk_tile(l.d);
  g->tile = take((most_tiles * l.Hkv * 2 * T * l.d * 2 + 1023) / 1024 * 1024);
  return most_tiles ? off : fixed;
}

cudaError_t configure_chunk() {
  auto one = [](void (*k)(ChunkArgs), int bytes) {
    // its warpgroups share out the registers of the launch: no fewer than they were counted on
    cudaFuncAttributes at;
    const cudaError_t e = cudaFuncGetAttributes(&at, k);
    if (e != cudaSuccess) return e;
    if (at.numRegs * kChunkThreads < 256 * kChunkSoftmaxRegisters + 128 * kChunkOtherRegisters) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  const cudaError_t e = one(chunk_attn_kernel<64>, ChunkSmem<64>::kTotal + 1024);
  return e != cudaSuccess ? e : one(chunk_attn_kernel<128>, ChunkSmem<128>::kTotal + 1024);
}

}  // namespace trr

using namespace trr;

static trr_status check_sizes(const Layout& l, int32_t n, int32_t num_tokens) {
  if (n < 0 || n > kMostSpans || num_tokens < 0 || num_tokens > kMostChunkTokens) return TRR_ERR_INVALID_ARG;
  if (l.head_modes) return TRR_ERR_UNSUPPORTED;  // one mode per token
  return static_cast<int64_t>(num_tokens) * l.Hq > INT_MAX - kBlockRows ? TRR_ERR_UNSUPPORTED : TRR_OK;  // (rows are counted in 32 bits)
}

extern "C" trr_status trr_chunk_workspace_bytes(const trr_cache* cache, int32_t num_chunks, int32_t num_tokens, int64_t max_keys, uint64_t* bytes) {
  if (!cache || !bytes || max_keys < 0) return TRR_ERR_INVALID_ARG;
  const Layout& l = cache_layout(cache);
  const trr_status st = check_sizes(l, num_chunks, num_tokens);
  if (st != TRR_OK) return st;
  // a sequence stores no more tokens than it has positions, or the pools have slots; a chunk ends in a partly filled tile
  int64_t slots = 0;
  for (int c = 0; c < kClasses; ++c) slots += static_cast<int64_t>(l.cap[c]) * l.P;
  const int64_t keys = std::min(max_keys, num_chunks * std::min<int64_t>(l.maxctx, slots)), tiles = keys / chunk_tile(l.d) + num_chunks;
  if (tiles > INT_MAX / chunk_tile(l.d)) return TRR_ERR_UNSUPPORTED;
  ChunkArgs g;
  *bytes = static_cast<uint64_t>(lay_workspace(&g, nullptr, l, num_chunks, num_tokens, cache_num_sms(cache), tiles));
  return TRR_OK;
}

extern "C" trr_status trr_chunk_attn(trr_cache* cache, int32_t layer, int32_t num_chunks, const int32_t* seq_ids, const int32_t* starts,
                                     const int32_t* offsets, int32_t num_tokens, const void* q_bf16, const uint8_t* modes,
                                     const int32_t* windows, int32_t window_scalar, int32_t sinks, float softmax_scale,
                                     void* out_bf16, float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!cache) return TRR_ERR_INVALID_ARG;
  const Layout& l = cache_layout(cache);
  if (layer < 0 || layer >= l.L || sinks < 0) return TRR_ERR_INVALID_ARG;
  trr_status st = check_sizes(l, num_chunks, num_tokens);
  if (st != TRR_OK) return st;
  cache_set_launches(cache, 0);
  if (num_chunks == 0 || num_tokens == 0) return TRR_OK;
  if (!seq_ids || !starts || !offsets || !q_bf16 || !modes || !out_bf16) return TRR_ERR_INVALID_ARG;
  const uintptr_t q0 = reinterpret_cast<uintptr_t>(q_bf16), out0 = reinterpret_cast<uintptr_t>(out_bf16), row_bytes = 2ull * num_tokens * l.Hq * l.d;
  if (((q0 | out0) & 15) || (reinterpret_cast<uintptr_t>(lse) & 3)) return TRR_ERR_INVALID_ARG;
  if (q0 < out0 + row_bytes && out0 < q0 + row_bytes) return TRR_ERR_INVALID_ARG;  // (queries are read again where a row is done one by one)
  uint64_t least = 0;
  st = trr_chunk_workspace_bytes(cache, num_chunks, num_tokens, 0, &least);
  if (st != TRR_OK) return st;
  if (!workspace || workspace_bytes < least || (reinterpret_cast<uintptr_t>(workspace) & 255)) return TRR_ERR_OUT_OF_MEMORY;
  ChunkArgs g;
  g.a = layer_args(l, cache_views(cache), layer);
  g.a.wait_ns = cache_wait_ns(cache);
  g.n = num_chunks; g.num_tokens = num_tokens; g.window_scalar = window_scalar; g.sinks = sinks;
  g.ctas = cache_num_sms(cache);
  g.parts = std::max(1, std::min({kMostParts, kMostCommonCtas / num_chunks, (2 * l.Hkv * l.d + kPlanChunkThreads - 1) / kPlanChunkThreads}));
  g.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.f / sqrtf(static_cast<float>(l.d))) * 1.4426950408889634f;
  g.seq_ids = seq_ids; g.starts = starts; g.offsets = offsets; g.windows = windows; g.modes = modes;
  g.q = static_cast<const uint16_t*>(q_bf16);
  g.out = static_cast<uint16_t*>(out_bf16);
  g.lse = lse;
  const int64_t fixed = lay_workspace(&g, nullptr, l, num_chunks, num_tokens, g.ctas, 0), T = chunk_tile(l.d), per_tile = 4 * l.Hkv * T * l.d;
  const int64_t bytes = static_cast<int64_t>(std::min<uint64_t>(workspace_bytes, 1ull << 60));
  int64_t room = std::min<int64_t>((bytes - fixed) / per_tile, INT_MAX / T);
  if (lay_workspace(&g, nullptr, l, num_chunks, num_tokens, g.ctas, room) > bytes) --room;  // (its parts are rounded up)
  g.most_tiles = static_cast<int>(room);
  lay_workspace(&g, static_cast<uint8_t*>(workspace), l, num_chunks, num_tokens, g.ctas, g.most_tiles);
  cache_note_call(cache, layer);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int launches = 0;
  cudaError_t e = launch_pdl(chunk_plan_kernel, dim3(num_chunks * (1 + g.parts)), dim3(kPlanChunkThreads), 0, s, g);
  if (e == cudaSuccess) {
    ++launches;
    e = launch_pdl(l.d == 64 ? chunk_stage_kernel<64> : chunk_stage_kernel<128>, dim3(kStageCtas * g.ctas), dim3(kSpanThreads), 0, s, g);
  }
  if (e == cudaSuccess) {
    ++launches;
    e = l.d == 64 ? launch_pdl(chunk_attn_kernel<64>, dim3(g.ctas), dim3(kChunkThreads), ChunkSmem<64>::kTotal + 1024, s, g)
                  : launch_pdl(chunk_attn_kernel<128>, dim3(g.ctas), dim3(kChunkThreads), ChunkSmem<128>::kTotal + 1024, s, g);
  }
  if (e == cudaSuccess) {
    ++launches;
    e = launch_pdl(l.d == 64 ? chunk_join_kernel<64> : chunk_join_kernel<128>, dim3(8 * g.ctas), dim3(256), 0, s, g);
  }
  if (e == cudaSuccess) ++launches;
  cache_set_launches(cache, launches);
  return e == cudaSuccess ? TRR_OK : TRR_ERR_CUDA;
}
