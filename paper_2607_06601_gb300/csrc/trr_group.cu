// trr_group.cu - trr_decode_attn_sinks and trr_decode_attn_shared: decode attention whose
// local queries keep the first tokens in sight, and whose queries may share pages.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(s_ij - m_i) / sum_j exp(s_ij - m_i),  s_ij = scale q_i k_j
// over the stored tokens j that query i sees: j <= t_i and (full, or j >= t_i-w_i+1, or
// j < sinks).  Any split of the tokens can be joined again: parts (m, l, o) with
// l = sum exp(s - m), o = sum exp(s - m) v give m' = max m, l' = sum l exp(m - m'), and so for o.
//
// Three kernels:
//   group_plan_kernel     cuts the call into jobs.  A shared job is the pages that all full
//                         queries of a group have in common, with all their rows; a private
//                         job is what is left for one query.  A job is one segment per KV head
//                         and block of 128 rows; all rows of a segment see the same tokens.
//   group_attn_kernel     one CTA per SM; the segments' tiles (up to 128 tokens), laid end to
//                         end, are cut into one equal run for each CTA, so that a long segment
//                         is spread over many CTAs and a CTA takes many short ones.
//   group_combine_kernel  joins the parts of every row.
//
// In the attention kernel a producer warp brings each tile's page slices into a ring of shared
// memory with bulk copies; eight warps expand them to 16-bit rows in the tensor core's layout;
// one thread issues the products S = Q K^T and O += P V (tcgen05, sums in TMEM); four warps do
// the softmax, one row of TMEM per thread.  Pages of 2, 4 and 8 bits become binary16 (z + c s
// rounded once, 11 bits), pages of 16 bits stay bf16; p is rounded to the same type, sums and
// statistics are binary32.  A segment of 64 or 32 rows or fewer fills the 128 lanes with two or
// four copies of its rows, each of which takes its own part of a tile's tokens, so that all
// four warps share the exponentials.
#include <algorithm>
#include <climits>

#include "trr_few.cuh"

namespace trr {

// ------------------------------------------------------------------------------ plan --

// Error of query i, 0 when it is valid.
__device__ __forceinline__ int query_error(const GroupArgs& g, int i) {
  const int seq = g.seq_ids[i], t = g.positions[i], mode = g.modes[i];
  const int w = g.windows ? g.windows[i] : g.window_scalar;
  if (seq < 0 || seq >= g.a.S || mode > TRR_MODE_FULL || (mode == TRR_MODE_LOCAL && w < 1)) return TRR_ERR_INVALID_ARG;
  return t < 0 || t >= g.a.maxctx ? TRR_ERR_BAD_POSITION : 0;
}

// How many of x[0..n) (ascending) are below v, by one warp: 32 probes a round.
__device__ __forceinline__ int count_below(const int32_t* x, int n, int v, int lane) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32, i = lo + lane * step;
    const int k = __popc(__ballot_sync(0xffffffffu, i < hi && x[i] < v));
    if (k == 0) return lo;
    const int last = lo + (k - 1) * step;
    hi = min(hi, last + step);
    lo = last + 1;
  }
  return lo;
}

// Tiles (or blocks) of a job of nq pages of 2, 4 and 8 bits and n16 of 16.
__device__ __forceinline__ int job_tiles(const GroupArgs& g, bool few, int nq, int n16, int* tiles_q) {
  const int P = g.a.P, ppt = kTileKeys / P, ppt16 = kTileKeys / 2 / P;
  *tiles_q = (nq + ppt - 1) / ppt;
  return few ? nq * (P > 32 ? P / 32 : 1) + n16 * (P / 16) : *tiles_q + (n16 + ppt16 - 1) / ppt16;
}

// CTA i plans query i, warp c its class c; the CTA that finishes last plans the groups and lays
// the jobs end to end.  All of it is chains of dependent loads, so what a query's CTA can settle
// alone (its private job unless it is a full query of a group, the zero rows of a query that reads
// nothing) does not wait for the last one.
__global__ void __launch_bounds__(kPlanThreads) group_plan_kernel(const __grid_constant__ GroupArgs g) {
  __shared__ int s_bad, s_group, s_leader, s_last, s_first_err, s_there;
  __shared__ int64_t s_sum[kPlanThreads / 32];
  __shared__ Job s_job;
  const LayerArgs& a = g.a;
  const int lane = threadIdx.x & 31, c = threadIdx.x >> 5, i = blockIdx.x, heads = a.Hq / a.Hkv;
  if (threadIdx.x == 0) s_bad = 0, s_group = -1, s_leader = INT_MAX, s_first_err = INT_MAX;
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  for (int x = threadIdx.x; x <= g.groups && g.groups > 0; x += kPlanThreads) {
    const int o = g.offsets[x], next = x < g.groups ? g.offsets[x + 1] : o;
    if (o < 0 || o > g.n || next < o) s_bad = 1;
    if (o <= i && i < next) s_group = x;
  }
  int err = query_error(g, i);
  const int mode = g.modes[i], t = g.positions[i], seq = g.seq_ids[i];
  __syncthreads();
  if (s_bad) err = TRR_ERR_INVALID_ARG;
  const bool reads = !err && mode != TRR_MODE_SKIP;
  const bool member = reads && mode == TRR_MODE_FULL && s_group >= 0;
  if (member) {  // the group's first full query, whose pages the others' are compared with
    for (int j = g.offsets[s_group] + threadIdx.x; j <= i; j += kPlanThreads)
      if (g.modes[j] == TRR_MODE_FULL && !query_error(g, j)) {
        atomicMin(&s_leader, j);
        break;
      }
    __syncthreads();
  }
  const int lo = mode == TRR_MODE_LOCAL ? t - (g.windows ? g.windows[i] : g.window_scalar) + 1 : INT_MIN;
  int head = 0, first = 0, end = 0, common = 0;
  if (reads) {
    const int64_t row = static_cast<int64_t>(seq) * kClasses + c;
    const int nt = a.ntok[row], np = (nt + a.P - 1) / a.P;
    const int32_t *pf = a.pfirst + row * a.MP, *pl = a.plast + row * a.MP;
    if (np > 0) {
      const bool all = pl[np - 1] <= t;  // the usual case: no token after the query
      end = all ? np : count_below(pf, np, t + 1, lane);
      if (mode == TRR_MODE_LOCAL) {
        // page k starts at position k P or later: the sinks lie in the first ceil(sinks / P) pages
        const int most = static_cast<int>(min(static_cast<int64_t>(end), (static_cast<int64_t>(g.sinks) + a.P - 1) / a.P));
        head = count_below(pf, most, g.sinks, lane);
        first = max(head, count_below(pl, end, lo, lane));
      }
      if (member) {  // whole pages in sight, then those that the leader names too
        const int full = nt / a.P;
        const int whole = all ? full : count_below(pl, min(full, end), t + 1, lane);
        const int32_t* mine = a.pt + row * a.MP;
        const int64_t lead_row = static_cast<int64_t>(g.seq_ids[s_leader]) * kClasses + c;
        const int32_t* theirs = a.pt + lead_row * a.MP;
        const int most = min(whole, a.ntok[lead_row] / a.P);
        common = most;
        for (int k0 = 0; k0 < most && common == most; k0 += 256) {
          bool differs[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int k = k0 + 32 * u + lane;
            differs[u] = k < most && mine[k] != theirs[k];
          }
#pragma unroll
          for (int u = 7; u >= 0; --u) {
            const unsigned m = __ballot_sync(0xffffffffu, differs[u]);
            if (m) common = k0 + 32 * u + __ffs(m) - 1;
          }
        }
      }
    }
  }
  QueryPlan& p = g.plan[i];
  if (lane == 0) {
    p.common[c] = common;
    s_job.head[c] = head;
    s_job.first[c] = first;
    s_job.count[c] = max(0, end - first);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    int nq = 0;
    for (int k = 0; k < 3; ++k) nq += s_job.head[k] + s_job.count[k];
    s_job.seq = seq; s_job.lo = lo; s_job.t = t; s_job.sinks = mode == TRR_MODE_LOCAL ? g.sinks : 0;
    s_job.rows = heads;
    s_job.row_blocks = (heads + kRows - 1) / kRows;
    s_job.tiles = job_tiles(g, g.few, nq, s_job.head[3] + s_job.count[3], &s_job.tiles_q);
    s_job.kind = 1; s_job.qbase = i; s_job.joined = 0;
    const int there = reads && (member || s_job.tiles > 0);
    p.reads = there; p.group = member ? s_group : -1; p.rank = 0; p.shared = 0;
    g.tiles[g.groups + i] = err ? -err : there ? s_job.tiles : 0;
    s_there = there;
  }
  __syncthreads();
  if (threadIdx.x < 32) reinterpret_cast<int*>(g.jobs + g.groups + i)[threadIdx.x] = reinterpret_cast<const int*>(&s_job)[threadIdx.x];
  if (!s_there) {  // nothing in sight
    uint4* out = reinterpret_cast<uint4*>(g.out + static_cast<int64_t>(i) * a.Hq * a.d);
    for (int x = threadIdx.x; x < a.Hq * a.d / 8; x += kPlanThreads) out[x] = make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  if (threadIdx.x == 0) s_last = atom_add_acq_rel(a.ctrl + kGroupDone, 1) == static_cast<int>(gridDim.x) - 1;
  __syncthreads();
  if (!s_last) return;
  if (threadIdx.x == 0) a.ctrl[kGroupDone] = 0;

  for (int x = c; x < g.groups; x += kPlanThreads / 32) {  // groups: a warp each
    Job* job = g.jobs + x;
    int members = 0, least[kClasses] = {INT_MAX, INT_MAX, INT_MAX, INT_MAX};
    const int q0 = s_bad ? 0 : g.offsets[x], q1 = s_bad ? 0 : g.offsets[x + 1];
    for (int j0 = q0; j0 < q1; j0 += 32) {
      const int j = j0 + lane;
      const bool in = j < q1 && __ldcg(&g.plan[j].group) >= 0;
      const unsigned m = __ballot_sync(0xffffffffu, in);
      if (in) {
        const int rank = members + __popc(m & ((1u << lane) - 1));
        const int4 common = __ldcg(reinterpret_cast<const int4*>(g.plan[j].common));
        g.list[q0 + rank] = j;
        g.plan[j].rank = rank;
        least[0] = min(least[0], common.x);
        least[1] = min(least[1], common.y);
        least[2] = min(least[2], common.z);
        least[3] = min(least[3], common.w);
      }
      members += __popc(m);
    }
    int pages = 0;
    for (int k = 0; k < kClasses; ++k) {
      least[k] = __reduce_min_sync(0xffffffffu, least[k]);
      if (members < 2) least[k] = 0;  // nobody to share with
      pages += least[k];
    }
    __syncwarp();
    if (pages > 0)  // the members' private jobs start behind the shared pages
      for (int j = q0 + lane; j < q1; j += 32)
        if (__ldcg(&g.plan[j].group) >= 0) {
          Job* own = g.jobs + g.groups + j;
          int nq = 0, n16 = 0, tiles_q;
          for (int k = 0; k < kClasses; ++k) {
            const int left = max(0, __ldcg(&own->count[k]) - least[k]);
            own->first[k] = least[k];
            own->count[k] = left;
            (k < 3 ? nq : n16) += left;
          }
          const int tiles = job_tiles(g, g.few, nq, n16, &tiles_q);
          own->tiles_q = tiles_q;
          own->tiles = tiles;
          own->joined = 1;
          g.tiles[g.groups + j] = tiles;
          g.plan[j].shared = 1;
        }
    if (lane == 0) {
      job->seq = pages > 0 ? __ldcg(&g.jobs[g.groups + g.list[q0]].seq) : 0;
      job->lo = INT_MIN; job->t = INT_MAX; job->sinks = 0;
      for (int k = 0; k < kClasses; ++k) job->head[k] = 0, job->first[k] = 0, job->count[k] = least[k];
      job->rows = members * heads;
      job->row_blocks = (job->rows + kRows - 1) / kRows;
      int tiles_q = 0;
      const int tiles = pages > 0 ? job_tiles(g, false, least[0] + least[1] + least[2], least[3], &tiles_q) : 0;
      job->tiles_q = tiles_q;
      job->tiles = tiles;
      job->kind = 0; job->qbase = q0; job->joined = 1;
      g.tiles[x] = tiles;
    }
  }
  __syncthreads();
  // cost before each job
  const int private_blocks = (heads + kRows - 1) / kRows;
  auto prefix = [&](int from, int jobs, bool few, int64_t* base) -> int64_t {
    int64_t before = 0;
    for (int j0 = 0; j0 < jobs; j0 += kPlanThreads) {
      const int j = j0 + threadIdx.x, at = from + j, tiles = j < jobs ? __ldcg(g.tiles + at) : 0;
      int64_t x = 0;
      if (tiles > 0)
        x = few ? few_cost(tiles) * a.Hkv
                : segment_cost(tiles) * a.Hkv * (at < g.groups ? __ldcg(&g.jobs[at].row_blocks) : private_blocks);
      if (tiles < 0) atomicMin(&s_first_err, (at - g.groups) * 16 - tiles);
      int64_t y = x;
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t z = __shfl_up_sync(0xffffffffu, y, o);
        if (lane >= o) y += z;
      }
      if (lane == 31) s_sum[c] = y;
      __syncthreads();
      int64_t all = 0;
      for (int k = 0; k < kPlanThreads / 32; ++k) {
        if (k < c) y += s_sum[k];
        all += s_sum[k];
      }
      if (j < jobs) base[j] = before + y - x;
      before += all;
      __syncthreads();
    }
    if (threadIdx.x == 0) base[jobs] = before;
    return before;
  };
  const int jobs = g.few ? g.groups : g.groups + g.n;
  const int64_t work = prefix(0, jobs, false, g.base);
  const int64_t few_work = g.few ? prefix(g.groups, g.n, true, g.few_base) : 0;
  if (threadIdx.x == 0) {
    g.head->work = work;
    g.head->per = (work + g.ctas - 1) / g.ctas;
    g.head->few_work = few_work;
    g.head->few_per = (few_work + g.few_warps - 1) / g.few_warps;
    g.head->jobs = jobs;
    if (s_first_err != INT_MAX) set_status(a.ctrl, s_first_err % 16);
  }
}

// ------------------------------------------------------------------------- attention --

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
  int lo, t, sinks, pad;
  RawPage page[kTileKeys / 16];
};
struct TileMeta {
  int keys, bf16, first, end;
  uint32_t mask[4];   // tokens in sight
};

template <int D>
struct GroupSmem {
  static constexpr int kStages = D == 64 ? 3 : 2;      // expanded tiles
  static constexpr int kTile = kTileKeys * D * 2;      // bytes of K or V of one
  static constexpr int kScratch = kStages * 2 * kTile; // merge of row copies: [128][33] floats, then (m, l)
  static constexpr int kMl = kScratch + kRows * 33 * 4;
  static constexpr int kRaw = kMl + kRows * 8;
  static constexpr int kSeg = kRaw + kRawSlots * static_cast<int>(sizeof(RawTile));
  static constexpr int kMeta = kSeg + kSegSlots * static_cast<int>(sizeof(Segment));
  static constexpr int kBars = kMeta + kStages * static_cast<int>(sizeof(TileMeta));
  static constexpr int kNumBars = 2 * kRawSlots + 2 * kSegSlots + 2 * kStages + 2 + 2 + 5;
  static constexpr int kRing = (kBars + kNumBars * 8 + 16 + 127) / 128 * 128;
  static constexpr int kTotal = 225 * 1024;  // of the 227 KB a CTA may have; 1 KB aligns the base
  static constexpr int kRingBytes = (kTotal - kRing) / 128 * 128;
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
  __device__ uint64_t* kv_full(int i) const { return bar(2 * kRawSlots + 2 * kSegSlots + i); }
  __device__ uint64_t* kv_empty(int i) const { return bar(2 * kRawSlots + 2 * kSegSlots + L::kStages + i); }
  __device__ uint64_t* s_full(int i) const { return bar(2 * kRawSlots + 2 * kSegSlots + 2 * L::kStages + i); }
  __device__ uint64_t* p_full(int i) const { return s_full(2 + i); }
  __device__ uint64_t* o_done(int i) const { return s_full(4 + i); }
  __device__ uint64_t* q_full() const { return s_full(6); }
  __device__ uint64_t* drained() const { return s_full(7); }
  __device__ uint64_t* merged() const { return s_full(8); }
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

constexpr uint32_t kColO = 0, kColS = 128, kColQ = 384;  // TMEM columns: O, two S (P over S), Q in binary16 and bf16

// The producer warp: segments and tiles of this CTA's run, and the copies of their pages.
template <int D>
__device__ void group_produce(const GroupArgs& g, const Ctx<D>& x, int lane) {
  using L = GroupSmem<D>;
  const LayerArgs& a = g.a;
  const int64_t per = g.head->per, work = g.head->work;
  const int64_t b0 = min(work, blockIdx.x * per), b1 = min(work, b0 + per);
  const int jobs = g.head->jobs, P = a.P;
  int it = 0, freed = 0;           // tiles pushed, tiles whose ring bytes are known to be free
  int ring_head = 0, my_start = 0; // lane s: where slot s's tile starts
  int segs = 0;
  bool ok = true;

  // room for `need` bytes and a record; the offset in the ring
  auto book = [&](int need) -> int {
    for (;;) {
      if (it - freed < kRawSlots) {
        if (it == freed) { ring_head = need; return 0; }
        const int tail = __shfl_sync(0xffffffffu, my_start, freed % kRawSlots);
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
      const int64_t jbase = g.base[j];
      if (jbase >= b1) break;
      const int w = reinterpret_cast<const int*>(g.jobs + j)[lane];
      auto field = [&](int i) { return __shfl_sync(0xffffffffu, w, i); };
      const int tiles = field(19);
      if (tiles == 0) continue;
      const int seq = field(0), jlo = field(1), jt = field(2), sinks = field(3);
      int head[kClasses], first[kClasses], upto[kClasses + 1];
      upto[0] = 0;
      for (int c = 0; c < kClasses; ++c) {
        head[c] = field(4 + c);
        first[c] = field(8 + c);
        upto[c + 1] = upto[c] + head[c] + field(12 + c);
      }
      const int rows = field(16), row_blocks = field(17), tiles_q = field(18), kind = field(20), qbase = field(21), joined = field(22);
      const int nt = lane < kClasses ? a.ntok[static_cast<int64_t>(seq) * kClasses + lane] : 0;
      const int64_t cost = segment_cost(tiles);
      const int nsegs = a.Hkv * row_blocks;
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
        // batches of 32 pages, one per lane, of the 2-, 4- and 8-bit pages, then of the others
        int batch = -1, page = 0, cls = 0, valid = 0;
        bool whole = true;
        for (int tile = t0; tile < t1 && ok; ++tile) {
          const bool wide = tile >= tiles_q;
          const int ppt = (wide ? kTileKeys / 2 : kTileKeys) / P;
          const int i0 = (wide ? tile - tiles_q : tile) * ppt, end = wide ? upto[4] - upto[3] : upto[3];
          const int b = (wide ? 1 << 28 : 0) + i0 / 32;
          if (b != batch) {
            batch = b;
            const int i = i0 / 32 * 32 + lane;
            cls = wide ? 3 : i >= upto[2] ? 2 : i >= upto[1] ? 1 : 0;
            const int in = wide ? i : i - upto[cls];
            int h = head[0], f = first[0], n = __shfl_sync(0xffffffffu, nt, 0);
#pragma unroll
            for (int c = 1; c < kClasses; ++c) {
              const int m = __shfl_sync(0xffffffffu, nt, c);
              if (cls == c) h = head[c], f = first[c], n = m;
            }
            if (i < end) {
              const int k = in < h ? in : f + in - h;
              const int64_t at = (static_cast<int64_t>(seq) * kClasses + cls) * a.MP + k;
              page = a.pt[at];
              const int pf = a.pfirst[at], pl = a.plast[at];
              valid = min(P, n - k * P);
              whole = valid == P && pl <= jt && (pf >= jlo || pl < sinks);
            }
          }
          const int pages = min(ppt, end - i0), l0 = i0 % 32;
          const bool mine = lane >= l0 && lane < l0 + pages;
          const int slice = cls == 0 ? a.slice[0] : cls == 1 ? a.slice[1] : cls == 2 ? a.slice[2] : a.slice[3];
          const int room = mine ? (slice + 127) / 128 * 128 + (whole ? 0 : (4 * P + 127) / 128 * 128) : 0;
          int off = room;
          for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, off, o);
            if (lane >= o) off += y;
          }
          const int need = __shfl_sync(0xffffffffu, off, 31);
          const int bytes = __reduce_add_sync(0xffffffffu, mine ? slice + (whole ? 0 : 4 * P) : 0);
          const int at = book(need);
          if (at < 0) { ok = false; break; }
          const int slot = it % kRawSlots;
          if (lane == slot) my_start = at;
          off += at - room;
          RawTile& r = x.raw(slot);
          if (mine) r.page[lane - l0] = RawPage{off, whole ? -1 : off + (slice + 127) / 128 * 128, valid, cls};
          if (lane == 0) {
            r.pages = pages; r.bf16 = wide; r.first = tile == t0; r.end = 0;
            r.lo = jlo; r.t = jt; r.sinks = sinks;
          }
          __syncwarp();
          if (lane == 0) mbar_arrive_expect_tx(x.raw_full(slot), bytes);
          __syncwarp();
          if (mine) {
            const uint8_t* pool = cls == 0 ? a.pool[0] : cls == 1 ? a.pool[1] : cls == 2 ? a.pool[2] : a.pool[3];
            const int64_t pb = cls == 0 ? a.page_bytes[0] : cls == 1 ? a.page_bytes[1] : cls == 2 ? a.page_bytes[2] : a.page_bytes[3];
            const uint8_t* src = pool + page * pb;
            bulk_g2s(x.base + L::kRing + off, src + a.hdr + static_cast<int64_t>(kvh) * slice, slice, x.raw_full(slot));
            if (!whole) bulk_g2s(x.base + L::kRing + off + (slice + 127) / 128 * 128, src, 4 * P, x.raw_full(slot));
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

// z + c s of eight codes, given as four words of two binary16 values 1024 + c, rounded once.
template <bool CLAMP>
__device__ __forceinline__ uint4 expand8(uint32_t p0, uint32_t p1, uint32_t p2, uint32_t p3, __half2 s, __half2 z) {
  const __half2 k = as_half2(0x64006400u);  // 1024: the difference is exact
  __half2 v[4] = {__hfma2(__hsub2(as_half2(p0), k), s, z), __hfma2(__hsub2(as_half2(p1), k), s, z),
                  __hfma2(__hsub2(as_half2(p2), k), s, z), __hfma2(__hsub2(as_half2(p3), k), s, z)};
  if (CLAMP) {  // a value that rounds past 65504 stays finite
    const __half2 top = as_half2(0x7BFF7BFFu), low = as_half2(0xFBFFFBFFu);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __hmax2(__hmin2(v[i], top), low);
  }
  return make_uint4(as_u32(v[0]), as_u32(v[1]), as_u32(v[2]), as_u32(v[3]));
}

// Chunk e (8 elements) of row `key` of an expanded tile.
template <int D>
__device__ __forceinline__ uint8_t* tile_chunk(uint8_t* tile, int key, int e) {
  return tile + (e >> 3) * (kTileKeys * 128) + key * 128 + (((e ^ key) & 7) << 4);
}

// Expands one row of a 2-, 4- or 8-bit page: K or V (which) of slot `slot` of the slice at sl.
template <int D, int B, bool CLAMP>
__device__ __forceinline__ void expand_row(const uint8_t* sl, int which, int slot, int P, int lg_group, bool swz, int lane,
                                           uint8_t* tile, int key) {
  constexpr int kRow = D * B / 8, kN = kRow / 16;  // bytes and 16-byte chunks of a row
  constexpr int kPer = 128 / B;                    // elements of a chunk
  const int ng = D >> lg_group;
  const uint32_t* sz = reinterpret_cast<const uint32_t*>(sl + 2 * P * kRow) + (which * P + slot) * ng;
  const int row = (which * P + slot) * kRow;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    // rows of 128 bytes in a plain order: each lane starts at its own chunk, so that eight lanes read eight banks
    const int j = kN == 8 && !swz ? (i + lane) & 7 : i;
    const int o = row + 16 * j;
    const uint4 raw = *reinterpret_cast<const uint4*>(sl + (B == 8 && swz ? static_cast<int>(swz_off(o)) : o));
    const uint32_t word[4] = {raw.x, raw.y, raw.z, raw.w};
    uint32_t szw = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int el = j * kPer + q * (kPer / 4);  // the word's first element
      if (q == 0 || (kPer == 64 && q == 2)) szw = sz[el >> lg_group];  // a group holds 32 elements or more
      const __half2 s = as_half2(__byte_perm(szw, 0, 0x1010)), z = as_half2(__byte_perm(szw, 0, 0x3232));
      const uint32_t w = word[q];
      if (B == 8) {
        if (q & 1) continue;
        const uint32_t w2 = word[q | 1];
        *reinterpret_cast<uint4*>(tile_chunk<D>(tile, key, el >> 3)) =
            expand8<CLAMP>(__byte_perm(w, 0x64646464u, 0x4140), __byte_perm(w, 0x64646464u, 0x4342),
                           __byte_perm(w2, 0x64646464u, 0x4140), __byte_perm(w2, 0x64646464u, 0x4342), s, z);
      } else if (B == 4) {
        uint32_t t[4];  // elements k and k + 4
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = ((w >> (4 * k)) & 0x000F000Fu) | 0x64006400u;
        *reinterpret_cast<uint4*>(tile_chunk<D>(tile, key, el >> 3)) =
            expand8<CLAMP>(__byte_perm(t[0], t[1], 0x5410), __byte_perm(t[2], t[3], 0x5410), __byte_perm(t[0], t[1], 0x7632),
                           __byte_perm(t[2], t[3], 0x7632), s, z);
      } else {
        uint32_t t[8];  // elements k and k + 8
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = ((w >> (2 * k)) & 0x00030003u) | 0x64006400u;
        *reinterpret_cast<uint4*>(tile_chunk<D>(tile, key, el >> 3)) =
            expand8<CLAMP>(__byte_perm(t[0], t[1], 0x5410), __byte_perm(t[2], t[3], 0x5410), __byte_perm(t[4], t[5], 0x5410),
                           __byte_perm(t[6], t[7], 0x5410), s, z);
        *reinterpret_cast<uint4*>(tile_chunk<D>(tile, key, (el >> 3) + 1)) =
            expand8<CLAMP>(__byte_perm(t[0], t[1], 0x7632), __byte_perm(t[2], t[3], 0x7632), __byte_perm(t[4], t[5], 0x7632),
                           __byte_perm(t[6], t[7], 0x7632), s, z);
      }
    }
  }
}

// Whether a group's largest level rounds past binary16's largest value.
template <int D, int B>
__device__ __forceinline__ bool level_overflows(const uint8_t* sl, int which, int slot, int P, int lg_group) {
  const int ng = D >> lg_group;
  const uint32_t* sz = reinterpret_cast<const uint32_t*>(sl + 2 * P * (D * B / 8)) + (which * P + slot) * ng;
  bool over = false;
  for (int i = 0; i < ng; ++i) {
    const __half2 h = as_half2(sz[i]);
    const float top = static_cast<float>((1 << B) - 1) * __low2float(h) + __high2float(h);
    over |= !(fabsf(top) < 65504.f);
  }
  return over;
}

template <int D, int B>
__device__ __forceinline__ void expand(const uint8_t* sl, int which, int slot, int P, int lg_group, bool swz, int lane, uint8_t* tile,
                                       int key) {
  if (level_overflows<D, B>(sl, which, slot, P, lg_group)) expand_row<D, B, true>(sl, which, slot, P, lg_group, swz, lane, tile, key);
  else expand_row<D, B, false>(sl, which, slot, P, lg_group, swz, lane, tile, key);
}

// The expanding warps: warps 0-3 write K, 4-7 V; a thread has one token of the tile.
template <int D>
__device__ void group_expand(const GroupArgs& g, const Ctx<D>& x, int warp, int lane) {
  using L = GroupSmem<D>;
  const LayerArgs& a = g.a;
  const int which = warp >> 2, key = (warp & 3) * 32 + lane, P = a.P, lg_p = __ffs(P) - 1, lg_group = __ffs(a.G) - 1;
  const bool swz = a.swz;
  for (int it = 0;; ++it) {
    const int slot = it % kRawSlots, stage = it % L::kStages;
    if (!x.wait_warp(x.raw_full(slot), (it / kRawSlots) & 1)) return;
    if (!x.wait_warp(x.kv_empty(stage), ((it / L::kStages) & 1) ^ 1)) return;
    const RawTile& r = x.raw(slot);
    TileMeta& m = x.meta(stage);
    const bool end = r.end;
    if (!end) {
      const int keys = r.pages << lg_p;
      const bool in = key < keys;
      const RawPage pg = r.page[in ? key >> lg_p : 0];
      const int at = key & (P - 1);
      const uint8_t* ring = x.base + L::kRing;
      bool seen = in;
      if (in && pg.pos >= 0) {
        const int pos = reinterpret_cast<const int32_t*>(ring + pg.pos)[at];
        seen = at < pg.valid && pos <= r.t && (pos >= r.lo || pos < r.sinks);
      }
      const unsigned mask = __ballot_sync(0xffffffffu, seen);
      if (which == 0 && lane == 0) m.mask[warp & 3] = mask;
      if (warp == 0 && lane == 0) m.keys = keys, m.bf16 = r.bf16, m.first = r.first, m.end = 0;
      uint8_t* tile = x.base + (2 * stage + which) * L::kTile;
      if (r.bf16) {  // rows copied 16 bytes at a time, consecutive lanes along a row
        constexpr int kN = D / 8;
#pragma unroll 4
        for (int i = 0; i < kN; ++i) {
          const int row = (i * 32 + lane) / kN, e = (i * 32 + lane) % kN, k = (warp & 3) * 32 + row;
          if (k < keys) {
            uint4 v = make_uint4(0, 0, 0, 0);  // a V row out of sight is zero: its weight of 0 times infinity would not be
            if (which == 0 || (mask >> row & 1)) {
              const int o = (which * P + (k & (P - 1))) * D * 2 + 16 * e;
              v = *reinterpret_cast<const uint4*>(ring + r.page[k >> lg_p].off + (swz ? static_cast<int>(swz_off(o)) : o));
            }
            *reinterpret_cast<uint4*>(tile_chunk<D>(tile, k, e)) = v;
          }
        }
      } else if (in) {
        if (which == 1 && !seen) {
          for (int e = 0; e < D / 8; ++e) *reinterpret_cast<uint4*>(tile_chunk<D>(tile, key, e)) = make_uint4(0, 0, 0, 0);
        } else {
          const uint8_t* sl = ring + pg.off;
          if (pg.cls == 0) expand<D, 2>(sl, which, at, P, lg_group, swz, lane, tile, key);
          else if (pg.cls == 1) expand<D, 4>(sl, which, at, P, lg_group, swz, lane, tile, key);
          else expand<D, 8>(sl, which, at, P, lg_group, swz, lane, tile, key);
        }
      }
      fence_proxy_async_smem();
    } else if (warp == 0 && lane == 0) {
      m.end = 1;
    }
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(x.raw_empty(slot));
      mbar_arrive(x.kv_full(stage));
    }
    if (end) return;
  }
}

// The thread that issues the products.  Tile it's scores are issued before tile it-1's P V, so
// that the tensor core works while the softmax does.
template <int D>
__device__ void group_mma(const Ctx<D>& x) {
  using L = GroupSmem<D>;
  int segs = 0, keys_before = 0;
  bool bf16_before = false, first_before = false, pending = false;
  auto pv = [&](int it) -> bool {  // O += P V of tile it
    if (!x.wait(x.p_full(it & 1), (it >> 1) & 1)) return false;
    tc_fence_after();
    const uint32_t id = tc_idesc(bf16_before, D, true);
    const uint64_t d = tc_desc(x.tile(it % L::kStages, 1), kTileKeys * 128);
    for (int k = 0; k < keys_before / 16; ++k)
      tc_mma(x.tmem + kColO, x.tmem + kColS + 128 * (it & 1) + 8 * k, d + k * (2048 >> 4), id, !(first_before && k == 0));
    tc_commit(x.kv_empty(it % L::kStages));
    tc_commit(x.o_done(it & 1));
    pending = false;
    return true;
  };
  for (int it = 0;; ++it) {
    const int stage = it % L::kStages;
    if (!x.wait(x.kv_full(stage), (it / L::kStages) & 1)) break;
    const TileMeta& m = x.meta(stage);
    if (m.end) {
      if (pending) pv(it - 1);
      break;
    }
    const int keys = m.keys;
    const bool bf16 = m.bf16, first = m.first;
    if (it >= 2 && !x.wait(x.o_done(it & 1), ((it - 2) >> 1) & 1)) break;  // tile it-2's weights, under the new scores, have been used
    if (first) {
      if (pending && !pv(it - 1)) break;
      if (!x.wait(x.q_full(), segs & 1)) break;
      ++segs;
    }
    tc_fence_after();
    const uint32_t id = tc_idesc(bf16, keys, false);
    const uint32_t qcol = x.tmem + kColQ + (bf16 ? 64 : 0);
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
      tc_mma(x.tmem + kColS + 128 * (it & 1), qcol + 8 * k,
             tc_desc(x.tile(stage, 0) + (k >> 2) * (kTileKeys * 128) + (k & 3) * 32, 16), id, k > 0);
    tc_commit(x.s_full(it & 1));
    if (pending && !pv(it - 1)) break;
    pending = true;
    keys_before = keys; bf16_before = bf16; first_before = first;
  }
  tc_commit(x.drained());  // nothing is in flight when the CTA ends
  mbar_wait(x.drained(), 0);
}

template <int D>
__device__ void group_softmax(const GroupArgs& g, const Ctx<D>& x, int warp, int lane) {
  using L = GroupSmem<D>;
  const int tid = warp * 32 + lane, heads = g.a.Hq / g.a.Hkv;
  const uint32_t lanes = x.tmem + (static_cast<uint32_t>(warp) << 21);  // this warp's 32 lanes
  float* scratch = reinterpret_cast<float*>(x.base + L::kScratch);
  float2* ml = reinterpret_cast<float2*>(x.base + L::kMl);
  uint32_t meets = 0;
  auto meet = [&]() -> bool {  // the softmax warps wait for one another (bounded, unlike a CTA barrier)
    mbar_arrive(x.merged());
    return x.wait_warp(x.merged(), meets++ & 1);
  };

  // (query, head) of row r of a segment
  auto row_of = [&](const Segment& sg, int r, int* query, int* head) {
    const int rr = sg.row0 + r;
    *query = sg.kind == 0 ? g.list[sg.qbase + rr / heads] : sg.qbase;
    *head = sg.kvh * heads + rr % heads;
  };
  // Q of a segment into TMEM; the row's factor from products to base-2 exponents.  Each row is
  // scaled by a power of two that brings its largest element to [1, 2): binary16 then holds
  // what it needs of it.
  float factor = 0.f;
  auto load_q = [&](const Segment& sg, int copies) {
    const int r = tid & (kRows / copies - 1);
    uint32_t w[D / 2];
    uint32_t top = 0;
    if (r < sg.rows) {
      int query, head;
      row_of(sg, r, &query, &head);
      const uint4* src = reinterpret_cast<const uint4*>(g.q + (static_cast<int64_t>(query) * g.a.Hq + head) * D);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const uint4 u = src[i];
        w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
      }
#pragma unroll
      for (int i = 0; i < D / 2; ++i) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
    } else {
#pragma unroll
      for (int i = 0; i < D / 2; ++i) w[i] = 0;
    }
    int e = top == 0 || top >= 0x7F80u ? 0 : static_cast<int>(top >> 7) - 127;
    e = max(-100, min(120, e));
    const float down = __int_as_float((127 - e) << 23);
    factor = fmaxf(g.scale_log2 * __int_as_float((127 + e) << 23), 1.17549435e-38f);
#pragma unroll
    for (int half = 0; half < D / 64; ++half) {
      uint32_t o[32];
#pragma unroll
      for (int i = 0; i < 32; ++i)
        o[i] = as_u32(__floats2half2_rn(bf16lo(w[32 * half + i]) * down, bf16hi(w[32 * half + i]) * down));
      tmem_st32(lanes + kColQ + 32 * half, o);
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(bf16lo(w[32 * half + i]) * down, bf16hi(w[32 * half + i]) * down);
        o[i] = *reinterpret_cast<const uint32_t*>(&b);
      }
      tmem_st32(lanes + kColQ + 64 + 32 * half, o);
    }
    tmem_wait_st();
    tc_fence_before();
    mbar_arrive(x.q_full());
  };
  auto copies_of = [](int rows) { return rows <= 32 ? 4 : rows <= 64 ? 2 : 1; };

  int it = 0, segs = 0;
  if (!x.wait_warp(x.seg_full(0), 0)) return;
  Segment sg = x.seg(0);
  int copies = copies_of(sg.rows);
  if (sg.tiles > 0) load_q(sg, copies);
  while (sg.tiles > 0) {
    const int chunks = 4 / copies, chunk0 = copies == 1 ? 0 : copies == 2 ? (warp >> 1) * 2 : warp;  // this warp's 32-token chunks
    const float f = factor;
    float m = -INFINITY, l = 0.f;
    for (int tile = 0; tile < sg.tiles; ++tile, ++it) {
      const int stage = it % L::kStages;
      if (!x.wait_warp(x.kv_full(stage), (it / L::kStages) & 1)) return;
      const TileMeta& meta = x.meta(stage);
      const int keys = meta.keys;
      const bool bf16 = meta.bf16;
      if (!x.wait_warp(x.s_full(it & 1), (it >> 1) & 1)) return;
      tc_fence_after();
      const uint32_t scol = lanes + kColS + 128 * (it & 1);
      float top = -INFINITY;
      for (int c = chunk0; c < chunk0 + chunks; ++c) {
        const uint32_t mask = 32 * c < keys ? meta.mask[c] : 0;
        if (mask == 0) continue;
        uint32_t s[32];
        tmem_ld32(s, scol + 32 * c);
        if (mask == 0xffffffffu) {
#pragma unroll
          for (int i = 0; i < 32; ++i) top = fmaxf(top, __uint_as_float(s[i]));
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (mask >> i & 1) top = fmaxf(top, __uint_as_float(s[i]));
        }
      }
      top *= f;
      // m follows the maximum only when that has grown by more than 2^8: p stays within binary16, and O is rarely rescaled
      if (__any_sync(0xffffffffu, top > m + 8.f)) {
        const float next = fmaxf(m, top), by = m == -INFINITY ? 0.f : exp2_approx(m - next);
        l *= by;
        m = next;
        if (tile > 0) {
          if (!x.wait_warp(x.o_done((it - 1) & 1), ((it - 1) >> 1) & 1)) return;
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tmem_ld32(o, lanes + kColO + 32 * c);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * by);
            tmem_st32(lanes + kColO + 32 * c, o);
          }
        }
      }
      const float shift = m == -INFINITY ? 0.f : -m;
      for (int c = 0; c < 4 && 32 * c < keys; ++c) {
        uint32_t p[16];
        const uint32_t mask = c >= chunk0 && c < chunk0 + chunks ? meta.mask[c] : 0;
        if (mask == 0) {
#pragma unroll
          for (int i = 0; i < 16; ++i) p[i] = 0;
        } else {
          uint32_t s[32];
          tmem_ld32(s, scol + 32 * c);
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            float p0 = exp2_approx(fmaf(__uint_as_float(s[i]), f, shift)), p1 = exp2_approx(fmaf(__uint_as_float(s[i + 1]), f, shift));
            if (mask != 0xffffffffu) {
              if (!(mask >> i & 1)) p0 = 0.f;
              if (!(mask >> (i + 1) & 1)) p1 = 0.f;
            }
            l += p0 + p1;
            if (bf16) {
              const __nv_bfloat162 b = __floats2bfloat162_rn(p0, p1);
              p[i / 2] = *reinterpret_cast<const uint32_t*>(&b);
            } else {
              p[i / 2] = as_u32(__floats2half2_rn(p0, p1));
            }
          }
        }
        tmem_st16(scol + 16 * c, p);  // over scores that have been read
      }
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(x.p_full(it & 1));
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

    // rows out: the output itself, or (m, l, o) for the join
    const int width = kRows / done_copies;
    float weight = 1.f, sum = l, high = m;
    if (done_copies > 1) {
      ml[tid] = make_float2(m, l);
      if (!meet()) return;
      high = -INFINITY;
      for (int k = 0; k < done_copies; ++k) high = fmaxf(high, ml[(tid & (width - 1)) + k * width].x);
      sum = 0.f;
      for (int k = 0; k < done_copies; ++k) {
        const float2 v = ml[(tid & (width - 1)) + k * width];
        if (v.x != -INFINITY) sum += v.y * exp2_approx(v.x - high);
      }
      weight = m == -INFINITY ? 0.f : exp2_approx(m - high);
      if (!meet()) return;
      if (tid < width) ml[tid] = make_float2(high, sum);
      if (!meet()) return;
    }
    // thread -> row and columns of each 32 that it writes
    const int r = tid / done_copies, cols = 32 / done_copies, c0 = (tid % done_copies) * cols;
    int query = 0, head = 0;
    float2 mine = make_float2(high, sum);
    if (done_copies > 1) mine = ml[r];
    const bool live = r < done.rows;
    if (live) row_of(done, r, &query, &head);
    const int64_t home = (static_cast<int64_t>(done.kind) * g.n + query) * g.a.Hq + head;
    float* to = done.dest >= 0 ? g.part_o + (static_cast<int64_t>(done.dest) * kRows + r) * D : g.home_o + home * D;
    uint16_t* out = g.out + (static_cast<int64_t>(query) * g.a.Hq + head) * D;
    const float inv = mine.y != 0.f ? 1.f / mine.y : 0.f;
    if (live && c0 == 0 && done.dest > -2)
      (done.dest >= 0 ? g.part_ml[static_cast<int64_t>(done.dest) * kRows + r] : g.home_ml[home]) = mine;
    auto put = [&](int col, const float4 v) {
      if (done.dest == -2) {
        const __nv_bfloat162 b0 = __floats2bfloat162_rn(v.x * inv, v.y * inv), b1 = __floats2bfloat162_rn(v.z * inv, v.w * inv);
        *reinterpret_cast<uint2*>(out + col) = make_uint2(*reinterpret_cast<const uint32_t*>(&b0), *reinterpret_cast<const uint32_t*>(&b1));
      } else {
        *reinterpret_cast<float4*>(to + col) = v;
      }
    };
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t o[32];
      tmem_ld32(o, lanes + kColO + 32 * c);
      if (done_copies == 1) {
        if (live)
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            put(32 * c + i, make_float4(__uint_as_float(o[i]), __uint_as_float(o[i + 1]), __uint_as_float(o[i + 2]), __uint_as_float(o[i + 3])));
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) scratch[tid * 33 + i] = m == -INFINITY ? 0.f : __uint_as_float(o[i]) * weight;
        if (!meet()) return;
        if (live)
          for (int i = 0; i < cols; i += 4) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            for (int k = 0; k < done_copies; ++k)
#pragma unroll
              for (int u = 0; u < 4; ++u) v[u] += scratch[(r + k * width) * 33 + c0 + i + u];
            put(32 * c + c0 + i, make_float4(v[0], v[1], v[2], v[3]));
          }
        if (!meet()) return;
      }
    }
    tc_fence_before();
    __syncwarp();
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
  constexpr int kMmaWarp = kSoftmaxWarps + kExpandWarps, kProducer = kMmaWarp + 1;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < kRawSlots; ++i) mbar_init(x.raw_full(i), 1), mbar_init(x.raw_empty(i), kExpandWarps);
    for (int i = 0; i < kSegSlots; ++i) mbar_init(x.seg_full(i), 1), mbar_init(x.seg_empty(i), kSoftmaxWarps);
    for (int i = 0; i < L::kStages; ++i) mbar_init(x.kv_full(i), kExpandWarps), mbar_init(x.kv_empty(i), 1);
    for (int i = 0; i < 2; ++i) mbar_init(x.s_full(i), 1), mbar_init(x.p_full(i), 32 * kSoftmaxWarps), mbar_init(x.o_done(i), 1);
    mbar_init(x.q_full(), 32 * kSoftmaxWarps);
    mbar_init(x.drained(), 1);
    mbar_init(x.merged(), 32 * kSoftmaxWarps);
    fence_barrier_init();
  }
  if (warp == kMmaWarp) tmem_alloc(&s_tmem);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  x.tmem = s_tmem;
  pdl_wait();
  pdl_trigger();
  if (warp < kSoftmaxWarps) group_softmax<D>(g, x, warp, lane);
  else if (warp < kMmaWarp) group_expand<D>(g, x, warp - kSoftmaxWarps, lane);
  else if (warp == kProducer) group_produce<D>(g, x, lane);
  else if (lane == 0) group_mma<D>(x);
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_free(s_tmem);
  if (threadIdx.x == 0 && s_abort) set_status(g.a.ctrl, TRR_ERR_TIMEOUT);
}

// ----------------------------------------------------------------------------- join --

// One warp per (query, head): the parts of its row, at most one shared and one private
// segment, each whole or in one piece per CTA (or warp).  A lane looks up one part; the parts'
// rows are then read four at a time.
template <int D>
__global__ void __launch_bounds__(128) group_combine_kernel(const __grid_constant__ GroupArgs g) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31, heads = g.a.Hq / g.a.Hkv;
  const int64_t at = blockIdx.x * 4ll + (threadIdx.x >> 5);
  if (at >= static_cast<int64_t>(g.n) * g.a.Hq) return;
  const int query = static_cast<int>(at / g.a.Hq), head = static_cast<int>(at % g.a.Hq), kvh = head / heads;
  pdl_wait();
  pdl_trigger();
  const int4 p = *reinterpret_cast<const int4*>(g.plan + query);  // reads, group, rank, shared
  if (!p.x) return;
  float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 1
  for (int kind = p.w ? 0 : 1; kind < 2; ++kind) {
    const int j = kind == 0 ? p.y : g.groups + query, tiles = g.tiles[j];
    if (tiles <= 0) continue;
    const bool few = kind == 1 && g.few;
    const int rr = (kind == 0 ? p.z * heads : 0) + head % heads;
    const int64_t cost = few ? few_cost(tiles) : segment_cost(tiles), share = few ? g.head->few_per : g.head->per;
    const int64_t S = few ? g.few_base[query] + kvh * cost
                          : g.base[j] + (static_cast<int64_t>(kvh) * (kind == 0 ? g.jobs[j].row_blocks : (heads + kRows - 1) / kRows) + rr / kRows) * cost;
    const int64_t last = S + cost - 1;
    int64_t c0, c1;
    if (last < 0x7fffffff) c0 = static_cast<uint32_t>(S) / static_cast<uint32_t>(share), c1 = static_cast<uint32_t>(last) / static_cast<uint32_t>(share);
    else c0 = S / share, c1 = last / share;
    const float2* mls = few ? g.few_ml : g.part_ml;
    const float* rows = few ? g.few_o : g.part_o;
    const int pitch = few ? kFewRows : kRows, sub = few ? rr : rr % kRows;
    for (int64_t b = c0; b <= c1; b += 32) {
      const int64_t x0 = (b + lane) * share - S, x1 = x0 + share;
      const int t0 = few ? few_before(x0, tiles) : tiles_before(x0, tiles), t1 = few ? few_before(x1, tiles) : tiles_before(x1, tiles);
      const bool there = b + lane <= c1 && t0 < t1;
      int64_t slot = (2 * (b + lane) + (t0 > 0 ? 0 : 1)) * pitch + sub;
      if (__any_sync(0xffffffffu, there && t1 - t0 == tiles)) {  // all of it in one part
        if (!p.w) return;                                        // which is the row, in place
        slot = (static_cast<int64_t>(kind) * g.n + query) * g.a.Hq + head;
        mls = g.home_ml;
        rows = g.home_o;
      }
      const float2 v = there ? mls[slot] : make_float2(-INFINITY, 0.f);
      float top = v.x;
      for (int k = 16; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
      const float next = fmaxf(m, top);
      if (next == -INFINITY) continue;
      const float w = v.x == -INFINITY ? 0.f : exp2_approx(v.x - next), by = m == -INFINITY ? 0.f : exp2_approx(m - next);
      float sum = v.x == -INFINITY ? 0.f : v.y * w;
      for (int k = 16; k; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
      l = l * by + sum;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= by;
      m = next;
      unsigned parts = __ballot_sync(0xffffffffu, v.x != -INFINITY);
      while (parts) {
        float row[4][E], f[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int from = parts ? __ffs(parts) - 1 : 0;
          const int64_t s = __shfl_sync(0xffffffffu, slot, from);
          f[u] = __shfl_sync(0xffffffffu, w, from);
          if (!parts) f[u] = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) row[u][e] = parts ? rows[s * D + lane * E + e] : 0.f;
          parts &= parts - 1;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] += row[u][e] * f[u];
      }
    }
  }
  const float inv = l != 0.f ? 1.f / l : 0.f;
  uint16_t* out = g.out + at * D + lane * E;
  const __nv_bfloat162 b0 = __floats2bfloat162_rn(o[0] * inv, o[1] * inv);
  if (E == 2) {
    *reinterpret_cast<uint32_t*>(out) = *reinterpret_cast<const uint32_t*>(&b0);
  } else {
    const __nv_bfloat162 b1 = __floats2bfloat162_rn(o[E - 2] * inv, o[E - 1] * inv);
    *reinterpret_cast<uint2*>(out) = make_uint2(*reinterpret_cast<const uint32_t*>(&b0), *reinterpret_cast<const uint32_t*>(&b1));
  }
}

// ----------------------------------------------------------------------------- calls --

// Lays the workspace out for n queries (b == nullptr: counts its bytes).
static int64_t lay_workspace(GroupArgs* g, uint8_t* b, const Layout& l, int n, int ctas, int few_warps) {
  int64_t off = 0;
  auto take = [&](int64_t bytes) {
    uint8_t* p = b + off;
    off += (bytes + 255) / 256 * 256;
    return p;
  };
  const int64_t rows = static_cast<int64_t>(n) * l.Hq, parts = 2ll * ctas * kRows;
  g->head = reinterpret_cast<GroupHeader*>(take(sizeof(GroupHeader)));
  g->plan = reinterpret_cast<QueryPlan*>(take(static_cast<int64_t>(sizeof(QueryPlan)) * n));
  g->list = reinterpret_cast<int32_t*>(take(4ll * n));
  g->jobs = reinterpret_cast<Job*>(take(static_cast<int64_t>(sizeof(Job)) * 2 * n));
  g->tiles = reinterpret_cast<int32_t*>(take(4ll * 2 * n));
  g->base = reinterpret_cast<int64_t*>(take(8ll * (2 * n + 1)));
  g->home_ml = reinterpret_cast<float2*>(take(8 * 2 * rows));
  g->home_o = reinterpret_cast<float*>(take(4 * 2 * rows * l.d));
  g->part_ml = reinterpret_cast<float2*>(take(8 * parts));
  g->part_o = reinterpret_cast<float*>(take(4 * parts * l.d));
  g->few_base = reinterpret_cast<int64_t*>(take(8ll * (n + 1)));
  g->few_ml = reinterpret_cast<float2*>(take(8ll * 2 * few_warps * kFewRows));
  g->few_o = reinterpret_cast<float*>(take(4ll * 2 * few_warps * kFewRows * l.d));
  return off;
}

int64_t group_workspace_bytes(const Layout& l, int ctas) {
  GroupArgs g;
  return lay_workspace(&g, nullptr, l, l.max_queries, ctas, ctas * kFewCtas * kFewWarps);
}

// The kernel for few rows of a layout, nullptr where its columns (query heads of a KV head x
// groups) are more than a product's eight.
static void (*few_kernel(const Layout& l))(GroupArgs) {
  const int ng = l.d / l.G;
  if (l.Hq / l.Hkv * ng > 8) return nullptr;
  if (l.d == 64) return ng == 1 ? group_few_kernel<64, 1> : group_few_kernel<64, 2>;
  return ng == 1 ? group_few_kernel<128, 1> : ng == 2 ? group_few_kernel<128, 2> : group_few_kernel<128, 4>;
}

cudaError_t configure_group() {
  for (auto k : {group_few_kernel<64, 1>, group_few_kernel<64, 2>}) {
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
    if (e != cudaSuccess) return e;
  }
  for (auto k : {group_few_kernel<128, 1>, group_few_kernel<128, 2>, group_few_kernel<128, 4>}) {
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
    if (e != cudaSuccess) return e;
  }
  cudaError_t e = cudaFuncSetAttribute(group_attn_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, GroupSmem<64>::kTotal + 1024);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(group_attn_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, GroupSmem<128>::kTotal + 1024);
}

template <int D>
static cudaError_t launch_kernels(const GroupArgs& g, void (*few)(GroupArgs), cudaStream_t s, int* launches) {
  *launches = 0;
  cudaError_t e = launch_pdl(group_plan_kernel, dim3(g.n), dim3(kPlanThreads), 0, s, g);
  if (e != cudaSuccess) return e;
  ++*launches;
  if (few) {
    e = launch_pdl(few, dim3(g.few_warps / kFewWarps), dim3(32 * kFewWarps), kFewSmem, s, g);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  if (!few || g.groups > 0) {
    e = launch_pdl(group_attn_kernel<D>, dim3(g.ctas), dim3(kGroupThreads), GroupSmem<D>::kTotal + 1024, s, g);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  const int64_t rows = static_cast<int64_t>(g.n) * g.a.Hq;
  e = launch_pdl(group_combine_kernel<D>, dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(128), 0, s, g);
  if (e == cudaSuccess) ++*launches;
  return e;
}

static trr_status launch_group(trr_cache* cache, int layer, int n, const int32_t* seq_ids, const int32_t* positions,
                               const void* q, const uint8_t* modes, const int32_t* windows, int window_scalar, int sinks,
                               int groups, const int32_t* offsets, float softmax_scale, void* out, void* workspace,
                               uint64_t workspace_bytes, void* stream) {
  if (!cache) return TRR_ERR_INVALID_ARG;
  const Layout& l = cache_layout(cache);
  if (layer < 0 || layer >= l.L || n < 0 || n > l.max_queries || sinks < 0 || groups < 0 || groups > n) return TRR_ERR_INVALID_ARG;
  cache_set_launches(cache, 0);
  if (n == 0) return TRR_OK;
  if (!seq_ids || !positions || !q || !modes || !out || (groups > 0 && !offsets)) return TRR_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) return TRR_ERR_INVALID_ARG;
  if (l.head_modes) return TRR_ERR_UNSUPPORTED;  // one mode per token
  const trr_status st = check_workspace(cache, workspace, workspace_bytes);
  if (st != TRR_OK) return st;
  GroupArgs g;
  g.a = layer_args(l, cache_views(cache), layer);
  g.n = n; g.window_scalar = window_scalar; g.sinks = sinks; g.groups = groups;
  g.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.f / sqrtf(static_cast<float>(l.d))) * 1.4426950408889634f;
  g.seq_ids = seq_ids; g.positions = positions; g.windows = windows; g.offsets = offsets; g.modes = modes;
  g.q = static_cast<const uint16_t*>(q);
  g.out = static_cast<uint16_t*>(out);
  g.a.wait_ns = cache_wait_ns(cache);
  g.ctas = cache_num_sms(cache);
  const auto few = few_kernel(l);
  g.few = few != nullptr;
  g.few_warps = g.ctas * kFewCtas * kFewWarps;
  lay_workspace(&g, static_cast<uint8_t*>(workspace), l, n, g.ctas, g.few_warps);
  cache_note_call(cache, layer);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int launches = 0;
  const cudaError_t e = l.d == 64 ? launch_kernels<64>(g, few, s, &launches) : launch_kernels<128>(g, few, s, &launches);
  cache_set_launches(cache, launches);
  return e == cudaSuccess ? TRR_OK : TRR_ERR_CUDA;
}

}  // namespace trr

using namespace trr;

extern "C" trr_status trr_decode_attn_sinks(trr_cache* cache, int32_t layer, int32_t n, const int32_t* seq_ids,
                                            const int32_t* q_positions, const void* q_bf16, const uint8_t* modes,
                                            const int32_t* windows, int32_t window_scalar, int32_t sinks,
                                            float softmax_scale, void* out_bf16, void* workspace, uint64_t workspace_bytes,
                                            void* stream) {
  return launch_group(cache, layer, n, seq_ids, q_positions, q_bf16, modes, windows, window_scalar, sinks, 0, nullptr,
                      softmax_scale, out_bf16, workspace, workspace_bytes, stream);
}

extern "C" trr_status trr_decode_attn_shared(trr_cache* cache, int32_t layer, int32_t n, const int32_t* seq_ids,
                                             const int32_t* q_positions, const void* q_bf16, const uint8_t* modes,
                                             const int32_t* windows, int32_t window_scalar, int32_t sinks, int32_t num_groups,
                                             const int32_t* group_offsets, float softmax_scale, void* out_bf16,
                                             void* workspace, uint64_t workspace_bytes, void* stream) {
  return launch_group(cache, layer, n, seq_ids, q_positions, q_bf16, modes, windows, window_scalar, sinks, num_groups,
                      group_offsets, softmax_scale, out_bf16, workspace, workspace_bytes, stream);
}
