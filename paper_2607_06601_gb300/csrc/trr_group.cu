// trr_group.cu - trr_decode_attn_sinks and trr_decode_attn_shared: decode attention whose
// local queries keep the first tokens in sight, and whose queries may share pages.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(s_ij - m_i) / sum_j exp(s_ij - m_i),  s_ij = scale q_i k_j
// over the stored tokens j that query i sees: j <= t_i and (full, or j >= t_i-w_i+1, or
// j < sinks).  Any split of the tokens can be joined again: parts (m, l, o) with
// l = sum exp(s - m), o = sum exp(s - m) v give m' = max m, l' = sum l exp(m - m'), and so for o.
//
// Four kernels:
//   group_plan_kernel     cuts the call into jobs.  A shared job is the pages that all full
//                         queries of a group have in common, with all their rows; a private
//                         job is what is left for one query.  A job is one segment per KV head
//                         and block of 128 rows; all rows of a segment see the same tokens.
//   group_attn_kernel     one CTA per SM; the segments' tiles (up to 128 tokens), laid end to
//                         end, are cut into one equal run for each CTA, so that a long segment
//                         is spread over many CTAs and a CTA takes many short ones.
//   group_few_kernel      the segments of few rows (rows x groups of a row at most 8: a product's
//                         columns), codes as they are stored.  64 queries of 32 heads with windows
//                         of 511: 97 us when it came in, 221 on the tensor cores.
//   group_combine_kernel  joins the parts of every row.
//
// The plan and the join are chains of dependent loads: 6 to 9 us and 4 to 9 us of a call with up to
// eight groups.  The CTA that finishes last plans the groups, four at a time, and so the plan grows
// with their number: 10 us for one group of 4 queries, 19 for 32, 52 for 128, 96 for 256, 184 for 512
// (by itself, caches cold).
//
#include <algorithm>
#include <climits>

#include "trr_few.cuh"
#include "trr_group_tc.cuh"

namespace trr {

// ------------------------------------------------------------------------------ plan --

// Error of query i, 0 when it is valid.
__device__ __forceinline__ int query_error(const GroupArgs& g, int i) {
  const int seq = g.seq_ids[i], t = g.positions[i], mode = g.modes[i];
  const int w = g.windows ? g.windows[i] : g.window_scalar;
  if (seq < 0 || seq >= g.a.S || mode > TRR_MODE_FULL || (mode == TRR_MODE_LOCAL && w < 1)) return TRR_ERR_INVALID_ARG;
  return t < 0 || t >= g.a.maxctx ? TRR_ERR_BAD_POSITION : 0;
}

// How many of x[0..n) (ascending) are below v.  The whole warp calls it; its lanes may search in
// groups of `width` from lane `from` on, each its own list, with that many probes a round.
__device__ __forceinline__ int count_below(const int32_t* x, int n, int v, int lane, int width, int from) {
  const unsigned group = width == 32 ? 0xffffffffu : (1u << width) - 1;
  int lo = 0, hi = n;
  while (__any_sync(0xffffffffu, lo < hi)) {
    const int step = (hi - lo + width - 1) / width, i = lo + lane * step;
    const int k = __popc(__ballot_sync(0xffffffffu, i < hi && x[i] < v) >> from & group);
    if (lo >= hi) continue;
    const int last = lo + (k - 1) * step;
    if (k > 0) hi = min(hi, last + step), lo = last + 1;
    else hi = lo;
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
  __shared__ int64_t s_sum[2][kPlanThreads / 32];
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
  int head = 0, first = 0, end = 0, common = 0, tokens = 0;
  if (reads) {
    const int64_t row = static_cast<int64_t>(seq) * kClasses + c;
    const int nt = a.ntok[row], np = (nt + a.P - 1) / a.P;
    tokens = nt;
    const int32_t *pf = a.pfirst + row * a.MP, *pl = a.plast + row * a.MP;
    if (np > 0) {
      // three searches at once, by 16, 8 and 8 lanes: pages before the window, pages with a sink
      // (page k starts at position k P or later: they lie in the first ceil(sinks / P)), pages up to t
      const int sinks = mode == TRR_MODE_LOCAL ? static_cast<int>(min(static_cast<int64_t>(np), (static_cast<int64_t>(g.sinks) + a.P - 1) / a.P)) : 0;
      const bool all = pl[np - 1] <= t;  // the usual case: no token after the query
      const bool near = lane < 16, third = lane >= 24;
      const int found = count_below(near ? pl : pf, near ? (mode == TRR_MODE_LOCAL ? np : 0) : third ? (all ? 0 : np) : sinks,
                                    near ? lo : third ? t + 1 : g.sinks, near ? lane : lane & 7, near ? 16 : 8, near ? 0 : lane & ~7);
      end = all ? np : __shfl_sync(0xffffffffu, found, 24);
      if (mode == TRR_MODE_LOCAL) {
        head = min(__shfl_sync(0xffffffffu, found, 16), end);
        first = max(head, min(__shfl_sync(0xffffffffu, found, 0), end));
      }
      if (member) {  // whole pages in sight, then those that the leader names too
        const int full = nt / a.P;
        const int whole = all ? full : count_below(pl, min(full, end), t + 1, lane, 32, 0);
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
    s_job.tokens[c] = tokens;
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
    s_job.tiles = job_tiles(g, g.few > 0, nq, s_job.head[3] + s_job.count[3], &s_job.tiles_q);
    s_job.kind = 1; s_job.qbase = i; s_job.joined = 0;
    const int there = reads && (member || s_job.tiles > 0);
    p.reads = there; p.group = member ? s_group : -1; p.rank = 0; p.shared = 0;
    const int tiles = there ? s_job.tiles : 0;
    g.tiles[g.groups + i] = err ? -err : g.few ? 0 : tiles;
    g.blocks[g.groups + i] = g.few ? tiles : 0;
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
    int members = 0, least[kClasses] = {INT_MAX, INT_MAX, INT_MAX, INT_MAX}, seq = 0;
    const int q0 = s_bad ? 0 : g.offsets[x], q1 = s_bad ? 0 : g.offsets[x + 1];
    bool in = false;          // of the last 32 queries: whether the lane's is a member, its private pages
    int4 mine = make_int4(0, 0, 0, 0);
    for (int j0 = q0; j0 < q1; j0 += 32) {
      const int j = j0 + lane, at = min(j, q1 - 1);
      const int4 common = __ldcg(reinterpret_cast<const int4*>(g.plan[at].common));
      mine = __ldcg(reinterpret_cast<const int4*>(g.jobs[g.groups + at].count));
      const int own_seq = __ldcg(&g.jobs[g.groups + at].seq);
      in = j < q1 && __ldcg(&g.plan[at].group) >= 0;
      const unsigned m = __ballot_sync(0xffffffffu, in);
      if (members == 0 && m) seq = __shfl_sync(0xffffffffu, own_seq, __ffs(m) - 1);
      if (in) {
        const int rank = members + __popc(m & ((1u << lane) - 1));
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
    if (pages > 0)  // the members' private jobs start behind the shared pages
      for (int j = q0 + lane; j < q1; j += 32) {
        Job* own = g.jobs + g.groups + j;
        if (q1 - q0 > 32) {  // (a larger group's are read again)
          in = __ldcg(&g.plan[j].group) >= 0;
          mine = __ldcg(reinterpret_cast<const int4*>(own->count));
        }
        if (!in) continue;
        const int left[kClasses] = {max(0, mine.x - least[0]), max(0, mine.y - least[1]), max(0, mine.z - least[2]), max(0, mine.w - least[3])};
        int tiles_q;
        const int tiles = job_tiles(g, g.few > 0, left[0] + left[1] + left[2], left[3], &tiles_q);
        for (int k = 0; k < kClasses; ++k) own->first[k] = least[k], own->count[k] = left[k];
        own->tiles_q = tiles_q;
        own->tiles = tiles;
        own->joined = 1;
        (g.few ? g.blocks : g.tiles)[g.groups + j] = tiles;
        g.plan[j].shared = 1;
      }
    if (lane == 0) {
      job->seq = seq;
      job->lo = INT_MIN; job->t = INT_MAX; job->sinks = 0;
      for (int k = 0; k < kClasses; ++k) job->tokens[k] = least[k] * a.P, job->head[k] = 0, job->first[k] = 0, job->count[k] = least[k];
      job->rows = members * heads;
      job->row_blocks = (job->rows + kRows - 1) / kRows;
      int tiles_q = 0;
      const bool few = job->rows <= g.few;  // a small group's rows are few, too
      const int tiles = pages > 0 ? job_tiles(g, few, least[0] + least[1] + least[2], least[3], &tiles_q) : 0;
      job->tiles_q = tiles_q;
      job->tiles = tiles;
      job->kind = 0; job->qbase = q0; job->joined = 1;
      g.tiles[x] = few ? 0 : tiles;
      g.blocks[x] = few ? tiles : 0;
    }
  }
  __syncthreads();
  // cost before each job
  const int private_blocks = (heads + kRows - 1) / kRows;
  const int jobs = g.groups + g.n;
  int64_t work = 0, few_work = 0;  // of the jobs so far, for the tensor kernel and the one for few rows
  for (int j0 = 0; j0 < jobs; j0 += kPlanThreads) {
    const int j = j0 + threadIdx.x, tiles = j < jobs ? __ldcg(g.tiles + j) : 0, blocks = j < jobs ? __ldcg(g.blocks + j) : 0;
    const int row_blocks = j < g.groups ? __ldcg(&g.jobs[j].row_blocks) : private_blocks;
    if (tiles < 0) atomicMin(&s_first_err, (j - g.groups) * 16 - tiles);
    const int64_t x = tiles > 0 ? segment_cost(tiles) * a.Hkv * row_blocks : 0;
    const int64_t z = blocks > 0 ? few_cost(blocks) * a.Hkv : 0;
    int64_t x1 = x, z1 = z;
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t u = __shfl_up_sync(0xffffffffu, x1, o), v = __shfl_up_sync(0xffffffffu, z1, o);
      if (lane >= o) x1 += u, z1 += v;
    }
    if (lane == 31) s_sum[0][c] = x1, s_sum[1][c] = z1;
    __syncthreads();
    int64_t all_x = 0, all_z = 0;
    for (int k = 0; k < kPlanThreads / 32; ++k) {
      if (k < c) x1 += s_sum[0][k], z1 += s_sum[1][k];
      all_x += s_sum[0][k];
      all_z += s_sum[1][k];
    }
    if (j < jobs) g.base[j] = work + x1 - x, g.few_base[j] = few_work + z1 - z;
    work += all_x;
    few_work += all_z;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    g.base[jobs] = work;
    g.few_base[jobs] = few_work;
    g.head->work = work;
    // The few rows' runs: one for each warp of the SMs that the tensor kernel leaves, if that brings
    // them home beside it, else one for each warp of all SMs, after it.
    const int warps = kFewCtas * kFewWarps;
    auto split = [](int64_t x, int64_t n) -> int64_t {  // rounded up (in 32 bits where they do: half a microsecond less)
      x += n - 1;
      return x <= 0xffffffffll && n <= 0xffffffffll ? static_cast<uint32_t>(x) / static_cast<uint32_t>(n) : x / n;
    };
    auto share = [&](int64_t sms) { return max(static_cast<int64_t>(kLeastShare), split(work, sms)); };
    int64_t per = share(g.ctas), left = g.ctas - split(work, per);
    if (few_work > left * warps * kShortShare && per >= kLongShare) {
      const int64_t few_sms = split(few_work, warps * kFewShare);
      if (few_sms * 16 <= g.ctas) per = share(g.ctas - few_sms), left = max(few_sms, g.ctas - split(work, per));
    }
    const bool beside = left > 0 && few_work <= left * warps * (per >= kLongShare ? kFewShare : kShortShare);
    g.head->per = per;
    g.head->few_work = few_work;
    st_release(&g.head->few_per, split(few_work, beside ? left * warps : g.few_warps));  // last: see group_few_kernel
    if (s_first_err != INT_MAX) set_status(a.ctrl, s_first_err % 16);
  }
}

// ----------------------------------------------------------------------------- join --

// One warp per (query, head): the parts of its row, at most one shared and one private
// segment, each whole or in one piece per CTA (or warp).  A lane looks up one part; the parts'
// rows are then read eight at a time.
template <int D>
__global__ void __launch_bounds__(128) group_combine_kernel(const __grid_constant__ GroupArgs g) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31, heads = g.a.Hq / g.a.Hkv;
  const int64_t at = blockIdx.x * 4ll + (threadIdx.x >> 5);
  if (at >= static_cast<int64_t>(g.n) * g.a.Hq) return;
  const int query = static_cast<int>(at / g.a.Hq), head = static_cast<int>(at % g.a.Hq), kvh = head / heads;
  pdl_wait();
  pdl_trigger();
  // what the search for the parts needs, in two rounds of loads: this, then both jobs' sizes and places
  const int4 p = *reinterpret_cast<const int4*>(g.plan + query);  // reads, group, rank, shared
  const int64_t per = g.head->per, few_per = g.head->few_per;
  if (!p.x) return;
  struct Place {
    int tiles, blocks, row_blocks, rows;
    int64_t base, few_base;
  } place[2];
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    const int j = kind == 0 ? (p.w ? p.y : 0) : g.groups + query;
    const bool any = kind == 1 || p.w;
    place[kind] = Place{any ? g.tiles[j] : 0, any ? g.blocks[j] : 0, kind == 0 && any ? g.jobs[j].row_blocks : (heads + kRows - 1) / kRows,
                        kind == 0 && any ? g.jobs[j].rows : heads, g.base[j], g.few_base[j]};
  }
  float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 1
  for (int kind = 0; kind < 2; ++kind) {
    const Place at_job = kind == 0 ? place[0] : place[1];
    const bool few = at_job.blocks > 0;
    const int tiles = few ? at_job.blocks : at_job.tiles;
    if (tiles <= 0) continue;
    const int rr = (kind == 0 ? p.z * heads : 0) + head % heads;
    const int64_t cost = few ? few_cost(tiles) : segment_cost(tiles), share = few ? few_per : per;
    const int64_t S = few ? at_job.few_base + kvh * cost : at_job.base + (static_cast<int64_t>(kvh) * at_job.row_blocks + rr / kRows) * cost;
    const int64_t last = S + cost - 1;
    int64_t c0, c1;
    if (last < 0x7fffffff) c0 = static_cast<uint32_t>(S) / static_cast<uint32_t>(share), c1 = static_cast<uint32_t>(last) / static_cast<uint32_t>(share);
    else c0 = S / share, c1 = last / share;
    const float2* mls = few ? g.few_ml : g.part_ml;
    const float* rows = few ? g.few_o : g.part_o;
    // a piece of the tensor kernel has a row for each of the copies that filled its lanes
    const int copies = few ? 1 : copies_of(min(kRows, at_job.rows - rr / kRows * kRows)), lg = copies >> 1;
    const int pitch = few ? kFewRows : kRows, sub = (few ? rr : rr % kRows) + (lane & (copies - 1)) * (kRows / copies);
    for (int64_t b = c0; b <= c1; b += 32 >> lg) {
      const int64_t c = b + (lane >> lg), x0 = c * share - S, x1 = x0 + share;
      const int t0 = few ? few_before(x0, tiles) : tiles_before(x0, tiles), t1 = few ? few_before(x1, tiles) : tiles_before(x1, tiles);
      bool there = c <= c1 && t0 < t1;
      int64_t slot = (2 * c + (t0 > 0 ? 0 : 1)) * pitch + sub;
      if (__any_sync(0xffffffffu, there && t1 - t0 == tiles)) {  // all of it in one part, its copies joined
        if (!p.w) return;                                        // which is the row, in place
        slot = (static_cast<int64_t>(kind) * g.n + query) * g.a.Hq + head;
        mls = g.home_ml;
        rows = g.home_o;
        there = there && (lane & (copies - 1)) == 0;
      }
      const float2 v = there ? mls[slot] : make_float2(-INFINITY, 0.f);
      unsigned parts = __ballot_sync(0xffffffffu, there);
      float top = v.x;
      for (int k = 16; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
      const float next = fmaxf(m, top);
      const float w = v.x == -INFINITY ? 0.f : exp2_approx(v.x - next), by = m == -INFINITY ? 0.f : exp2_approx(m - next);
      float sum = v.x == -INFINITY ? 0.f : v.y * w;
      for (int k = 16; k; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
      l = l * by + sum;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= by;
      m = next;
      constexpr int kAhead = 8;
      while (parts) {
        float row[kAhead][E], f[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int from = parts ? __ffs(parts) - 1 : 0;
          const float* src = rows + __shfl_sync(0xffffffffu, slot, from) * D + lane * E;
          f[u] = __shfl_sync(0xffffffffu, w, from);
          if (parts) {
            if (E == 4) {
              const float4 x = *reinterpret_cast<const float4*>(src);
              row[u][0] = x.x; row[u][1] = x.y; row[u][E - 2] = x.z; row[u][E - 1] = x.w;
            } else {
              const float2 x = *reinterpret_cast<const float2*>(src);
              row[u][0] = x.x; row[u][1] = x.y;
            }
          } else {
            f[u] = 0.f;
          }
          parts &= parts - 1;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (f[u] != 0.f)  // (a part in which nothing was seen may hold anything)
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
  g->blocks = reinterpret_cast<int32_t*>(take(4ll * 2 * n));
  g->base = reinterpret_cast<int64_t*>(take(8ll * (2 * n + 1)));
  g->home_ml = reinterpret_cast<float2*>(take(8 * 2 * rows));
  g->home_o = reinterpret_cast<float*>(take(4 * 2 * rows * l.d));
  g->part_ml = reinterpret_cast<float2*>(take(8 * parts));
  g->part_o = reinterpret_cast<float*>(take(4 * parts * l.d));
  g->few_base = reinterpret_cast<int64_t*>(take(8ll * (2 * n + 1)));
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
  auto tensor_kernel = [](void (*k)(GroupArgs), int bytes) {
    // its warpgroups share out the registers of the launch: no fewer than they were counted on
    cudaFuncAttributes at;
    cudaError_t e = cudaFuncGetAttributes(&at, k);
    if (e != cudaSuccess) return e;
    if (at.numRegs * kGroupThreads < 32 * kSoftmaxWarps * kSoftmaxRegisters + (kGroupThreads - 32 * kSoftmaxWarps) * kOtherRegisters)
      return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  const cudaError_t e = tensor_kernel(group_attn_kernel<64>, GroupSmem<64>::kTotal + 1024);
  return e != cudaSuccess ? e : tensor_kernel(group_attn_kernel<128>, GroupSmem<128>::kTotal + 1024);
}

template <int D>
static cudaError_t launch_kernels(const GroupArgs& g, void (*few)(GroupArgs), cudaStream_t s, int* launches) {
  *launches = 0;
  cudaError_t e = launch_pdl(group_plan_kernel, dim3(g.n), dim3(kPlanThreads), 0, s, g);
  if (e != cudaSuccess) return e;
  ++*launches;
  if (!few || g.groups > 0) {
    e = launch_pdl(group_attn_kernel<D>, dim3(g.ctas), dim3(kGroupThreads), GroupSmem<D>::kTotal + 1024, s, g);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  if (few) {
    e = launch_pdl(few, dim3(g.few_warps / kFewWarps), dim3(32 * kFewWarps), kFewSmem, s, g);
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
  g.few = few ? kFewRows / (l.d / l.G) : 0;
  g.overlap = groups > 0;
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
