// trr_pages.cu - page operations over every layer of a cache: trr_fork, trr_evict,
// trr_free_seqs and trr_compact.
//
// Sequences may name the same full pages.  No count of users is kept: a full page is never
// written again, a partly filled one has one user (a fork copies it), and which pages are in
// use is read off the page tables when trr_compact asks.  So the append and decode kernels,
// which hand out ids from next_page upwards, know nothing of sharing.
//
// What bounds them: page copies are HBM traffic (each byte read and written once); the
// tables are a few kilobytes per sequence, so everything else is launch and load latency.
// Two forks of 32 sequences of 4096 tokens over 24 layers of 32 KV heads, with eviction, releases
// and two compactions between (3.33 GB): 595 us, 5.6 TB/s of the 6.8 that a copy reaches; the same
// over 12 layers of 12 heads and 2048 tokens (0.63 GB): 140 us, 4.5 TB/s.
#include <algorithm>

#include "trr_internal.cuh"

namespace trr {

constexpr int kMaxPageOp = 4096;      // most entries of a fork, eviction or release
constexpr int kPieceBytes = 32768;    // one CTA's share of a page copy: 8 loads of 16 bytes in flight per thread
constexpr int kCopyThreads = 256;

struct PageArgs {
  int L, S, Hkv, P, MP, W32, hdr, maskb, ctas;
  int cap[kClasses], slice[kClasses], pieces[kClasses], pieces_before[kClasses + 1];
  int64_t page_bytes[kClasses];
  int32_t *ctrl, *last_pos, *ntok, *pt, *pfirst, *plast, *lastpg;
  uint32_t* presence;
  uint8_t* pool[kClasses];
};

static PageArgs page_args(const trr_cache* cache) {
  const Layout& l = cache_layout(cache);
  const Views& v = cache_views(cache);
  PageArgs a;
  a.L = l.L; a.S = l.S; a.Hkv = l.Hkv; a.P = l.P; a.MP = l.MP; a.W32 = l.W32;
  a.hdr = static_cast<int>(l.hdr); a.maskb = static_cast<int>(l.maskb);
  a.ctas = cache_num_sms(cache);
  a.pieces_before[0] = 0;
  for (int c = 0; c < kClasses; ++c) {
    a.cap[c] = l.cap[c];
    a.slice[c] = static_cast<int>(l.slice[c]);
    a.page_bytes[c] = l.page_bytes[c];
    a.pieces[c] = static_cast<int>((l.page_bytes[c] + kPieceBytes - 1) / kPieceBytes);
    a.pieces_before[c + 1] = a.pieces_before[c] + a.pieces[c];
    a.pool[c] = v.pool[c];
  }
  a.ctrl = v.ctrl; a.last_pos = v.last_pos; a.ntok = v.ntok; a.presence = v.presence;
  a.pt = v.pt; a.pfirst = v.pfirst; a.plast = v.plast; a.lastpg = v.lastpg;
  return a;
}

// How many of x[0..n) (ascending) are below v, by one warp: 32 probes narrow the range to
// its 32nd part, so two or three rounds of loads.
__device__ __forceinline__ int warp_below(const int32_t* x, int n, int v, int lane) {
  int lo = 0, hi = n;  // x[i] < v for i < lo, x[i] >= v for i >= hi
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32;
    const int i = lo + lane * step;
    const unsigned m = __ballot_sync(0xffffffffu, i < hi && x[i] < v);
    const int k = __popc(m);  // probes are ascending: the first k are below
    if (k == 0) return lo;
    const int last = lo + (k - 1) * step;
    hi = min(hi, last + step);
    lo = last + 1;
  }
  return lo;
}

// Copies piece `piece` of a page of class c.  With keep >= 0 and per-head modes, the
// presence bits of the slots from `keep` up are cleared in the copy: an append sets a
// slot's bits and expects them clear.
__device__ __forceinline__ void copy_piece(const PageArgs& a, int c, int from, int to, int piece, int keep) {
  const int64_t off = static_cast<int64_t>(piece) * kPieceBytes;
  const int n = static_cast<int>(min(static_cast<int64_t>(kPieceBytes), a.page_bytes[c] - off)) / 16;
  const uint4* src = reinterpret_cast<const uint4*>(a.pool[c] + from * a.page_bytes[c] + off);
  uint4* dst = reinterpret_cast<uint4*>(a.pool[c] + to * a.page_bytes[c] + off);
  constexpr int kPer = kPieceBytes / 16 / kCopyThreads;
  uint4 w[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int k = threadIdx.x + i * kCopyThreads;
    if (k < n) w[i] = __ldcs(src + k);
  }
  if (a.maskb && keep >= 0) {
    const unsigned long long m = keep >= 64 ? ~0ull : (1ull << keep) - 1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int64_t o = off + (threadIdx.x + i * kCopyThreads) * 16 - a.hdr;
      if (o >= 0 && o < static_cast<int64_t>(a.Hkv) * a.slice[c] && o % a.slice[c] == a.slice[c] - a.maskb) {
        w[i].x &= static_cast<uint32_t>(m);
        w[i].y &= static_cast<uint32_t>(m >> 32);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int k = threadIdx.x + i * kCopyThreads;
    if (k < n) dst[k] = w[i];
  }
}

// ------------------------------------------------------------------------------ fork --

// One (layer, entry, class) of a fork.
struct ForkPlan {
  int take;  // pages of the source that the fork keeps, the last one perhaps cut or partly filled
  int kept;  // tokens it keeps of the last of them
  int from;  // that page, when it has to be copied, else -1
  int last;  // position of the last token kept
};

// CTA (layer, entry), warp c plans class c; the CTA that finishes last checks the pools and
// hands out the copies' ids in order of (layer, entry).
__global__ void __launch_bounds__(128) fork_plan_kernel(PageArgs a, int n, const int32_t* __restrict__ src,
                                                        const int32_t* __restrict__ dst,
                                                        const int32_t* __restrict__ lengths, ForkPlan* plan, int32_t* to) {
  __shared__ int s_bad, s_last, s_count[kClasses][4];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, c = threadIdx.x >> 5;
  const int layer = blockIdx.x / n, i = blockIdx.x % n;
  const int s = src[i], d = dst[i], length = lengths[i];
  if (threadIdx.x == 0) s_bad = s < 0 || s >= a.S || d < 0 || d >= a.S || length < 0;
  __syncthreads();
  bool clash = false;
  for (int j = threadIdx.x; j < n; j += blockDim.x) clash |= j != i && (dst[j] == d || src[j] == d);
  if (clash) s_bad = 1;
  __syncthreads();
  ForkPlan p{0, 0, -1, -1};
  if (!s_bad) {
    const int64_t row = (static_cast<int64_t>(layer) * a.S + s) * kClasses + c;
    const int nt = a.ntok[row], np = (nt + a.P - 1) / a.P;
    p.take = warp_below(a.pfirst + row * a.MP, np, length, lane);
    if (p.take > 0) {
      const int k = p.take - 1, page = a.pt[row * a.MP + k], fill = min(a.P, nt - k * a.P);
      const int32_t* pos = reinterpret_cast<const int32_t*>(a.pool[c] + page * a.page_bytes[c]);
      int last = -1;
      for (int x = lane; x < fill; x += 32) {
        const int q = pos[x];
        if (q < length) { ++p.kept; last = q; }
      }
      p.kept = __reduce_add_sync(0xffffffffu, p.kept);
      p.last = __reduce_max_sync(0xffffffffu, last);
      if (p.kept < a.P) p.from = page;
    }
  }
  if (lane == 0) plan[static_cast<int64_t>(blockIdx.x) * kClasses + c] = p;
  __syncthreads();
  if (threadIdx.x == 0) {
    if (s_bad) atomicExch(a.ctrl + kForkError, TRR_ERR_INVALID_ARG);
    s_last = atom_add_acq_rel(a.ctrl + kForkDone, 1) == static_cast<int>(gridDim.x) - 1;
  }
  __syncthreads();
  if (!s_last) return;

  // every thread counts a run of entries, then numbers it
  const int64_t rows = gridDim.x, per = (rows + blockDim.x - 1) / blockDim.x;
  const int64_t r0 = min(rows, threadIdx.x * per), r1 = min(rows, r0 + per);
  int mine[kClasses] = {0, 0, 0, 0};
  for (int64_t r = r0; r < r1; ++r)
#pragma unroll
    for (int k = 0; k < kClasses; ++k) mine[k] += __ldcg(&plan[r * kClasses + k].from) >= 0;
  int before[kClasses];
#pragma unroll
  for (int k = 0; k < kClasses; ++k) {
    int x = mine[k];
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    before[k] = x - mine[k];
    if (lane == 31) s_count[k][c] = x;
  }
  __syncthreads();
  int err = a.ctrl[kForkError];
#pragma unroll
  for (int k = 0; k < kClasses; ++k) {
    int total = 0;
    for (int w = 0; w < 4; ++w) {
      if (w < c) before[k] += s_count[k][w];
      total += s_count[k][w];
    }
    before[k] += a.ctrl[kNextPage + k];
    if (!err && a.ctrl[kNextPage + k] + total > a.cap[k]) err = TRR_ERR_OUT_OF_PAGES;
  }
  for (int64_t r = r0; r < r1; ++r)
#pragma unroll
    for (int k = 0; k < kClasses; ++k)
      if (__ldcg(&plan[r * kClasses + k].from) >= 0) to[r * kClasses + k] = before[k]++;
  __syncthreads();
  if (threadIdx.x == 0) {
    if (err) set_status(a.ctrl, err);
    else
      for (int k = 0; k < kClasses; ++k)
        a.ctrl[kNextPage + k] += s_count[k][0] + s_count[k][1] + s_count[k][2] + s_count[k][3];
    a.ctrl[kForkOk] = err == 0;
    a.ctrl[kForkDone] = 0;
    a.ctrl[kForkError] = 0;
  }
}

// CTAs 0 .. rows-1 write the tables of one (layer, entry), the others copy one piece of one
// copied page.
__global__ void __launch_bounds__(kCopyThreads) fork_write_kernel(PageArgs a, int n, const int32_t* __restrict__ src,
                                                                  const int32_t* __restrict__ dst,
                                                                  const int32_t* __restrict__ lengths,
                                                                  const ForkPlan* plan, const int32_t* to) {
  pdl_wait();
  pdl_trigger();
  if (!a.ctrl[kForkOk]) return;
  const int rows = a.L * n;
  if (static_cast<int>(blockIdx.x) >= rows) {
    const int x = blockIdx.x - rows, pieces = a.pieces_before[kClasses];
    const int64_t r = x / pieces;
    const int k = x % pieces;
    int c = 0;
    while (k >= a.pieces_before[c + 1]) ++c;
    const ForkPlan p = plan[r * kClasses + c];
    if (p.from >= 0) copy_piece(a, c, p.from, to[r * kClasses + c], k - a.pieces_before[c], p.kept);
    return;
  }
  __shared__ int s_old[kClasses];
  const int layer = blockIdx.x / n, i = blockIdx.x % n, length = lengths[i];
  const int64_t s = static_cast<int64_t>(layer) * a.S + src[i], d = static_cast<int64_t>(layer) * a.S + dst[i];
  if (threadIdx.x < kClasses) s_old[threadIdx.x] = (a.ntok[d * kClasses + threadIdx.x] + a.P - 1) / a.P;
  __syncthreads();
  for (int c = 0; c < kClasses; ++c) {
    const int64_t r = static_cast<int64_t>(blockIdx.x) * kClasses + c;
    const ForkPlan p = plan[r];
    const int64_t from = (s * kClasses + c) * a.MP, at = (d * kClasses + c) * a.MP;
    const int copied = p.from >= 0 ? to[r] : -1;
    for (int k = threadIdx.x; k < max(p.take, s_old[c]); k += blockDim.x) {
      const bool in = k < p.take, end = k == p.take - 1 && copied >= 0;
      const int page = in ? a.pt[from + k] : -1, first = in ? a.pfirst[from + k] : -1, last = in ? a.plast[from + k] : -1;
      a.pt[at + k] = end ? copied : page;
      a.pfirst[at + k] = first;
      a.plast[at + k] = end ? p.last : last;
      if (k == p.take - 1) a.lastpg[d * kClasses + c] = end ? copied : page;
    }
    if (threadIdx.x == 0) {
      a.ntok[d * kClasses + c] = p.take > 0 ? (p.take - 1) * a.P + p.kept : 0;
      if (p.take == 0) a.lastpg[d * kClasses + c] = -1;
    }
  }
  for (int w = threadIdx.x; w < a.W32; w += blockDim.x) {
    const int64_t left = static_cast<int64_t>(length) - 32ll * w;
    const uint32_t m = left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1;
    a.presence[d * a.W32 + w] = a.presence[s * a.W32 + w] & m;
  }
  if (threadIdx.x == 0) a.last_pos[d] = min(a.last_pos[s], length - 1);
}

// ------------------------------------------------------------------- evict and free --

// CTA (layer, entry).  Pages are in position order, so the pages to forget of a class are
// one run [k0, k1): those behind it move up by its length.
__global__ void __launch_bounds__(256) evict_kernel(PageArgs a, int n, const int32_t* __restrict__ seqs,
                                                    const int32_t* __restrict__ keep_from, int sinks) {
  __shared__ int s_k0[kClasses], s_k1[kClasses], s_bad;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, c = threadIdx.x >> 5;
  const int layer = blockIdx.x / n, i = blockIdx.x % n, q = seqs[i];
  if (threadIdx.x == 0) s_bad = q < 0 || q >= a.S;
  __syncthreads();
  bool named = false;
  for (int j = threadIdx.x; j < i; j += blockDim.x) named |= seqs[j] == q;
  if (named) s_bad = 1;
  __syncthreads();
  if (s_bad) {
    if (threadIdx.x == 0) set_status(a.ctrl, TRR_ERR_INVALID_ARG);
    return;
  }
  const int64_t s = static_cast<int64_t>(layer) * a.S + q;
  if (c < kClasses) {
    const int64_t row = s * kClasses + c;
    const int full = a.ntok[row] / a.P;
    const int k0 = warp_below(a.pfirst + row * a.MP, full, sinks, lane);
    const int k1 = warp_below(a.plast + row * a.MP, full, keep_from[i], lane);
    if (lane == 0) s_k0[c] = k0, s_k1[c] = max(k0, k1);
  }
  __syncthreads();
  for (int k = 0; k < kClasses; ++k) {  // the tokens of the forgotten pages are no longer present
    const int32_t* table = a.pt + (s * kClasses + k) * a.MP;
    const int slots = (s_k1[k] - s_k0[k]) * a.P;
#pragma unroll 4
    for (int x = threadIdx.x; x < slots; x += blockDim.x) {
      const int page = table[s_k0[k] + x / a.P];
      const int pos = reinterpret_cast<const int32_t*>(a.pool[k] + page * a.page_bytes[k])[x % a.P];
      atomicAnd(a.presence + s * a.W32 + pos / 32, ~(1u << (pos % 32)));
    }
  }
  __syncthreads();
  if (c >= kClasses) return;
  const int gone = s_k1[c] - s_k0[c];
  if (gone == 0) return;
  const int64_t row = s * kClasses + c;
  const int nt = a.ntok[row], np = (nt + a.P - 1) / a.P;
  int32_t* const lists[3] = {a.pt + row * a.MP, a.pfirst + row * a.MP, a.plast + row * a.MP};
  for (int k = s_k0[c] + lane; k - lane < np; k += 32) {  // in place: a warp reads its 32 entries before any is written
    int v[3];
    for (int x = 0; x < 3; ++x) v[x] = k + gone < np ? lists[x][k + gone] : -1;
    __syncwarp();
    if (k < np)
      for (int x = 0; x < 3; ++x) lists[x][k] = v[x];
    __syncwarp();
  }
  if (lane == 0) {
    a.ntok[row] = nt - gone * a.P;
    a.lastpg[row] = np > gone ? lists[0][np - gone - 1] : -1;
  }
}

__global__ void __launch_bounds__(128) free_kernel(PageArgs a, int n, const int32_t* __restrict__ seqs) {
  __shared__ int s_pages[kClasses];
  pdl_wait();
  pdl_trigger();
  const int layer = blockIdx.x / n, q = seqs[blockIdx.x % n];
  if (q < 0 || q >= a.S) {
    if (threadIdx.x == 0) set_status(a.ctrl, TRR_ERR_INVALID_ARG);
    return;
  }
  const int64_t s = static_cast<int64_t>(layer) * a.S + q;
  if (threadIdx.x < kClasses) s_pages[threadIdx.x] = (a.ntok[s * kClasses + threadIdx.x] + a.P - 1) / a.P;
  __syncthreads();
  for (int c = 0; c < kClasses; ++c) {
    const int64_t row = s * kClasses + c;
    for (int k = threadIdx.x; k < s_pages[c]; k += blockDim.x)
      a.pt[row * a.MP + k] = a.pfirst[row * a.MP + k] = a.plast[row * a.MP + k] = -1;
  }
  for (int w = threadIdx.x; w < a.W32; w += blockDim.x) a.presence[s * a.W32 + w] = 0;
  if (threadIdx.x < kClasses) a.ntok[s * kClasses + threadIdx.x] = 0, a.lastpg[s * kClasses + threadIdx.x] = -1;
  if (threadIdx.x == 0) a.last_pos[s] = -1;
}

// --------------------------------------------------------------------------- compact --

// Workspace of a compaction, per class.
struct CompactArgs {
  uint32_t* used[kClasses];   // a bit per page id
  int32_t* holes[kClasses];   // unused ids below the pages in use
  int32_t* movers[kClasses];  // used ids above
  int32_t* moved[kClasses];   // new id of a mover
  int32_t* count;             // [kClasses] pages that move, [kClasses] pages in use
  int words;                  // of all `used`, which lie side by side
};

__global__ void __launch_bounds__(256) compact_clear_kernel(CompactArgs w) {
  pdl_wait();
  pdl_trigger();
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < w.words; i += gridDim.x * blockDim.x) w.used[0][i] = 0;
}

// One warp per page table row: a bit for every page it names.
__global__ void __launch_bounds__(256) compact_mark_kernel(PageArgs a, CompactArgs w) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int64_t rows = static_cast<int64_t>(a.L) * a.S * kClasses;
  for (int64_t r = blockIdx.x * 8ll + (threadIdx.x >> 5); r < rows; r += gridDim.x * 8ll) {
    const int c = static_cast<int>(r % kClasses), np = (a.ntok[r] + a.P - 1) / a.P;
    for (int k = lane; k < np; k += 32) {
      const int page = a.pt[r * a.MP + k];
      const uint32_t bit = 1u << (page % 32);
      // shared pages: most find their bit set and need no atomic
      if (!(__ldcg(w.used[c] + page / 32) & bit)) atomicOr(w.used[c] + page / 32, bit);
    }
  }
}

__device__ __forceinline__ int block_exclusive(int x, int* s_warp, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  int y = x;
  for (int o = 1; o < 32; o <<= 1) {
    const int z = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) y += z;
  }
  if (lane == 31) s_warp[warp] = y;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < warps; ++i) {
    if (i < warp) before += s_warp[i];
    all += s_warp[i];
  }
  __syncthreads();
  *total = all;
  return before + y - x;
}

// CTA c pairs class c's movers with its holes, both ascending.
__global__ void __launch_bounds__(1024) compact_plan_kernel(PageArgs a, CompactArgs w) {
  __shared__ int s_warp[32];
  pdl_wait();
  pdl_trigger();
  const int c = blockIdx.x, next = a.ctrl[kNextPage + c], words = (next + 31) / 32;
  const int per = (words + blockDim.x - 1) / blockDim.x;
  const int w0 = min(words, static_cast<int>(threadIdx.x) * per), w1 = min(words, w0 + per);
  int used = 0, live;
  for (int i = w0; i < w1; ++i) used += __popc(w.used[c][i]);
  block_exclusive(used, s_warp, &live);
  int nh = 0, nm = 0;
  auto split = [&](int i, uint32_t* holes, uint32_t* movers) {  // of the 32 ids of word i
    const int below = min(32, max(0, live - 32 * i));
    const uint32_t low = below == 32 ? 0xffffffffu : (1u << below) - 1, u = w.used[c][i];
    *holes = ~u & low;
    *movers = u & ~low;
  };
  uint32_t h, m;
  for (int i = w0; i < w1; ++i) {
    split(i, &h, &m);
    nh += __popc(h);
    nm += __popc(m);
  }
  int total;
  int kh = block_exclusive(nh, s_warp, &total), km = block_exclusive(nm, s_warp, &total);
  for (int i = w0; i < w1; ++i) {
    split(i, &h, &m);
    for (; h; h &= h - 1) w.holes[c][kh++] = 32 * i + __ffs(h) - 1;
    for (; m; m &= m - 1) w.movers[c][km++] = 32 * i + __ffs(m) - 1;
  }
  __syncthreads();
  for (int k = threadIdx.x; k < total; k += blockDim.x) w.moved[c][w.movers[c][k]] = w.holes[c][k];
  if (threadIdx.x == 0) {
    w.count[c] = total;
    w.count[kClasses + c] = live;
    a.ctrl[kNextPage + c] = live;
  }
}

// Page copies in pieces, then the tables' new ids.  A mover's id is above every hole's, so
// no copy reads what another writes.
__global__ void __launch_bounds__(kCopyThreads) compact_move_kernel(PageArgs a, CompactArgs w) {
  pdl_wait();
  pdl_trigger();
  int64_t before[kClasses + 1] = {0};
  for (int c = 0; c < kClasses; ++c) before[c + 1] = before[c] + static_cast<int64_t>(w.count[c]) * a.pieces[c];
  if (before[kClasses] == 0) return;
  for (int64_t x = blockIdx.x; x < before[kClasses]; x += gridDim.x) {
    int c = 0;
    while (x >= before[c + 1]) ++c;
    const int k = static_cast<int>((x - before[c]) / a.pieces[c]);
    copy_piece(a, c, w.movers[c][k], w.holes[c][k], static_cast<int>((x - before[c]) % a.pieces[c]), -1);
  }
  const int lane = threadIdx.x & 31;
  const int64_t rows = static_cast<int64_t>(a.L) * a.S * kClasses;
  for (int64_t r = blockIdx.x * 8ll + (threadIdx.x >> 5); r < rows; r += gridDim.x * 8ll) {
    const int c = static_cast<int>(r % kClasses), live = w.count[kClasses + c], np = (a.ntok[r] + a.P - 1) / a.P;
    if (w.count[c] == 0) continue;
    for (int k = lane; k < np; k += 32) {
      const int page = a.pt[r * a.MP + k];
      if (page >= live) a.pt[r * a.MP + k] = w.moved[c][page];
    }
    if (lane == 0 && a.lastpg[r] >= live) a.lastpg[r] = w.moved[c][a.lastpg[r]];
  }
}

static int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

static int64_t fork_bytes(const Layout& l) {
  const int64_t rows = static_cast<int64_t>(l.L) * std::min(l.S, kMaxPageOp) * kClasses;
  return up256(rows * sizeof(ForkPlan)) + up256(rows * 4);
}
static int64_t compact_bytes(const Layout& l) {
  int64_t words = 0, ids = 0;
  for (int c = 0; c < kClasses; ++c) words += (l.cap[c] + 31) / 32, ids += up256(4ll * l.cap[c]);
  return 256 + up256(4 * words) + 3 * ids;
}
int64_t pages_workspace_bytes(const Layout& l) { return std::max(fork_bytes(l), compact_bytes(l)); }

static bool entries_ok(const trr_cache* cache, int n) {
  return n >= 0 && n <= std::min(cache_layout(cache).S, kMaxPageOp);
}

}  // namespace trr

using namespace trr;

extern "C" trr_status trr_workspace_bytes(const trr_cache* cache, uint64_t* bytes) {
  if (!cache || !bytes) return TRR_ERR_INVALID_ARG;
  const Layout& l = cache_layout(cache);
  *bytes = static_cast<uint64_t>(std::max(pages_workspace_bytes(l), group_workspace_bytes(l, cache_num_sms(cache))));
  return TRR_OK;
}

extern "C" trr_status trr_fork(trr_cache* cache, int32_t n, const int32_t* src_seqs, const int32_t* dst_seqs,
                               const int32_t* lengths, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!cache || !entries_ok(cache, n)) return TRR_ERR_INVALID_ARG;
  cache_set_launches(cache, 0);
  if (n == 0) return TRR_OK;
  if (!src_seqs || !dst_seqs || !lengths) return TRR_ERR_INVALID_ARG;
  const trr_status st = check_workspace(cache, workspace, workspace_bytes);
  if (st != TRR_OK) return st;
  const PageArgs a = page_args(cache);
  const int64_t rows = static_cast<int64_t>(a.L) * n;
  ForkPlan* plan = static_cast<ForkPlan*>(workspace);
  int32_t* to = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + up256(rows * kClasses * sizeof(ForkPlan)));
  const int64_t ctas = rows * (1 + a.pieces_before[kClasses]);
  if (ctas > 0x7fffffff) return TRR_ERR_UNSUPPORTED;
  cache_note_every_layer(cache);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (launch_pdl(fork_plan_kernel, dim3(static_cast<unsigned>(rows)), dim3(128), 0, s, a, static_cast<int>(n), src_seqs, dst_seqs,
                 lengths, plan, to) != cudaSuccess)
    return TRR_ERR_CUDA;
  if (launch_pdl(fork_write_kernel, dim3(static_cast<unsigned>(ctas)), dim3(kCopyThreads), 0, s, a, static_cast<int>(n), src_seqs,
                 dst_seqs, lengths, static_cast<const ForkPlan*>(plan), static_cast<const int32_t*>(to)) != cudaSuccess)
    return TRR_ERR_CUDA;
  cache_set_launches(cache, 2);
  return TRR_OK;
}

extern "C" trr_status trr_evict(trr_cache* cache, int32_t n, const int32_t* seq_ids, const int32_t* keep_from, int32_t sinks,
                                void* stream) {
  if (!cache || !entries_ok(cache, n) || sinks < 0) return TRR_ERR_INVALID_ARG;
  cache_set_launches(cache, 0);
  if (n == 0) return TRR_OK;
  if (!seq_ids || !keep_from) return TRR_ERR_INVALID_ARG;
  const PageArgs a = page_args(cache);
  if (static_cast<int64_t>(a.L) * n > 0x7fffffff) return TRR_ERR_UNSUPPORTED;
  cache_note_every_layer(cache);
  if (launch_pdl(evict_kernel, dim3(a.L * n), dim3(256), 0, static_cast<cudaStream_t>(stream), a, static_cast<int>(n), seq_ids,
                 keep_from, static_cast<int>(sinks)) != cudaSuccess)
    return TRR_ERR_CUDA;
  cache_set_launches(cache, 1);
  return TRR_OK;
}

extern "C" trr_status trr_free_seqs(trr_cache* cache, int32_t n, const int32_t* seq_ids, void* stream) {
  if (!cache || !entries_ok(cache, n)) return TRR_ERR_INVALID_ARG;
  cache_set_launches(cache, 0);
  if (n == 0) return TRR_OK;
  if (!seq_ids) return TRR_ERR_INVALID_ARG;
  const PageArgs a = page_args(cache);
  if (static_cast<int64_t>(a.L) * n > 0x7fffffff) return TRR_ERR_UNSUPPORTED;
  cache_note_every_layer(cache);
  if (launch_pdl(free_kernel, dim3(a.L * n), dim3(128), 0, static_cast<cudaStream_t>(stream), a, static_cast<int>(n), seq_ids) !=
      cudaSuccess)
    return TRR_ERR_CUDA;
  cache_set_launches(cache, 1);
  return TRR_OK;
}

extern "C" trr_status trr_compact(trr_cache* cache, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!cache) return TRR_ERR_INVALID_ARG;
  cache_set_launches(cache, 0);
  const trr_status st = check_workspace(cache, workspace, workspace_bytes);
  if (st != TRR_OK) return st;
  const PageArgs a = page_args(cache);
  CompactArgs w;
  uint8_t* b = static_cast<uint8_t*>(workspace);
  w.count = reinterpret_cast<int32_t*>(b);
  uint32_t* used = reinterpret_cast<uint32_t*>(b + 256);
  w.words = 0;
  for (int c = 0; c < kClasses; ++c) {
    w.used[c] = used + w.words;
    w.words += (a.cap[c] + 31) / 32;
  }
  b += 256 + up256(4ll * w.words);
  for (int c = 0; c < kClasses; ++c) {
    const int64_t ids = up256(4ll * a.cap[c]);
    w.holes[c] = reinterpret_cast<int32_t*>(b);
    w.movers[c] = reinterpret_cast<int32_t*>(b + ids);
    w.moved[c] = reinterpret_cast<int32_t*>(b + 2 * ids);
    b += 3 * ids;
  }
  cache_note_every_layer(cache);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int64_t rows = static_cast<int64_t>(a.L) * a.S * kClasses;
  const int row_ctas = static_cast<int>(std::min<int64_t>((rows + 7) / 8, 8ll * a.ctas));
  bool ok = launch_pdl(compact_clear_kernel, dim3(std::max(1, std::min((w.words + 255) / 256, a.ctas))), dim3(256), 0, s, w) ==
            cudaSuccess;
  ok = ok && launch_pdl(compact_mark_kernel, dim3(row_ctas), dim3(256), 0, s, a, w) == cudaSuccess;
  ok = ok && launch_pdl(compact_plan_kernel, dim3(kClasses), dim3(1024), 0, s, a, w) == cudaSuccess;
  ok = ok && launch_pdl(compact_move_kernel, dim3(4 * a.ctas), dim3(kCopyThreads), 0, s, a, w) == cudaSuccess;
  if (!ok) return TRR_ERR_CUDA;
  cache_set_launches(cache, 4);
  return TRR_OK;
}
