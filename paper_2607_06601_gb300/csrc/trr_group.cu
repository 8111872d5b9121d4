// trr_group.cu - trr_decode_attn_sinks and trr_decode_attn_shared: decode attention whose
// local queries keep the first tokens in sight, and whose queries may share pages.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(s_ij - m_i) / sum_j exp(s_ij - m_i),  s_ij = scale q_i k_j
// over the stored tokens j that query i sees: j <= t_i and (full, or j >= t_i-w_i+1, or
// j < sinks).
//
// One CTA per (query, head): its warps take the pages in turn, lanes hold the dimensions, and
// each warp keeps a running maximum, sum and row in binary32 that are merged at the end.
#include <climits>

#include "trr_internal.cuh"

namespace trr {

struct GroupArgs {
  LayerArgs a;
  int n, window_scalar, sinks, groups;
  float scale_log2;  // softmax scale times log2(e): exponentials are taken in base 2
  const int32_t *seq_ids, *positions, *windows, *offsets;
  const uint8_t* modes;
  const uint16_t* q;
  uint16_t* out;
};

// Error of query i, 0 when it is valid.
__device__ __forceinline__ int query_error(const GroupArgs& g, int i) {
  const int seq = g.seq_ids[i], t = g.positions[i], mode = g.modes[i];
  const int w = g.windows ? g.windows[i] : g.window_scalar;
  if (seq < 0 || seq >= g.a.S || mode > TRR_MODE_FULL || (mode == TRR_MODE_LOCAL && w < 1)) return TRR_ERR_INVALID_ARG;
  return t < 0 || t >= g.a.maxctx ? TRR_ERR_BAD_POSITION : 0;
}

// Whether the offsets of the groups ascend within [0, n]; every thread of the CTA calls it.
__device__ __forceinline__ bool offsets_ok(const GroupArgs& g) {
  bool bad = false;
  if (g.groups > 0)
    for (int i = threadIdx.x; i <= g.groups; i += blockDim.x) {
      const int x = g.offsets[i];
      bad |= x < 0 || x > g.n || (i > 0 && x < g.offsets[i - 1]);
    }
  return !__syncthreads_or(bad);
}

__global__ void __launch_bounds__(1024) group_check_kernel(GroupArgs g) {
  __shared__ int s_first;
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x == 0) s_first = INT_MAX;
  const bool ok = offsets_ok(g);
  for (int i = threadIdx.x; i < g.n; i += blockDim.x) {
    const int err = ok ? query_error(g, i) : TRR_ERR_INVALID_ARG;
    if (err) atomicMin(&s_first, i * 16 + err);
  }
  __syncthreads();
  if (threadIdx.x == 0 && s_first != INT_MAX) set_status(g.a.ctrl, s_first % 16);
}

template <int D>
__global__ void __launch_bounds__(128) group_attn_kernel(GroupArgs g) {
  constexpr int E = D / 32;
  __shared__ float s_row[4][D], s_m[4], s_l[4];
  pdl_wait();
  pdl_trigger();
  const LayerArgs& a = g.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int i = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, kvh = h / (a.Hq / a.Hkv), ng = D / a.G;
  const bool ok = offsets_ok(g);
  uint16_t* out = g.out + (static_cast<int64_t>(i) * a.Hq + h) * D;
  float m = -INFINITY, l = 0.f, o[E], q[E];
  for (int e = 0; e < E; ++e) {
    o[e] = 0.f;
    q[e] = __uint_as_float(static_cast<uint32_t>(g.q[(static_cast<int64_t>(i) * a.Hq + h) * D + lane * E + e]) << 16) * g.scale_log2;
  }
  const int mode = g.modes[i], t = g.positions[i];
  if (ok && mode != TRR_MODE_SKIP && !query_error(g, i)) {
    const int lo = mode == TRR_MODE_FULL ? 0 : t - (g.windows ? g.windows[i] : g.window_scalar) + 1;
    for (int c = 0; c < kClasses; ++c) {
      const int b = bits_of_class(c), rowb = D * b / 8;
      const int64_t row = static_cast<int64_t>(g.seq_ids[i]) * kClasses + c;
      const int nt = a.ntok[row], np = (nt + a.P - 1) / a.P;
      for (int k = warp; k < np; k += 4) {
        const int first = a.pfirst[row * a.MP + k], last = a.plast[row * a.MP + k];
        if (first > t || (last < lo && first >= g.sinks)) continue;
        const uint8_t* page = a.pool[c] + a.pt[row * a.MP + k] * a.page_bytes[c];
        const uint8_t* sl = page + a.hdr + static_cast<int64_t>(kvh) * a.slice[c];
        for (int x = 0; x < min(a.P, nt - k * a.P); ++x) {
          const int pos = reinterpret_cast<const int32_t*>(page)[x];
          if (pos > t || (pos < lo && pos >= g.sinks)) continue;
          float kv[2][E];
          for (int w = 0; w < 2; ++w)
            for (int e = 0; e < E; ++e) {
              const int j = lane * E + e;
              const int64_t at = static_cast<int64_t>(w) * a.P * rowb + x * rowb + j * b / 8;
              const int64_t off = a.swz && b >= 8 ? swz_off(at) : at;
              if (b == 16) {
                kv[w][e] = __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(sl + off)) << 16);
              } else {
                const int code = (sl[off] >> (j * b % 8)) & ((1 << b) - 1);
                const __half* sz = reinterpret_cast<const __half*>(sl + 2 * a.P * rowb + ((w * a.P + x) * ng + j / a.G) * 4);
                kv[w][e] = __half2float(sz[1]) + code * __half2float(sz[0]);
              }
            }
          float s = 0.f;
          for (int e = 0; e < E; ++e) s += q[e] * kv[0][e];
          for (int z = 16; z; z >>= 1) s += __shfl_xor_sync(0xffffffffu, s, z);
          const float m2 = fmaxf(m, s), f = m == -INFINITY ? 0.f : exp2f(m - m2), p = exp2f(s - m2);
          l = l * f + p;
          for (int e = 0; e < E; ++e) o[e] = o[e] * f + p * kv[1][e];
          m = m2;
        }
      }
    }
  }
  for (int e = 0; e < E; ++e) s_row[warp][lane * E + e] = o[e];
  if (lane == 0) s_m[warp] = m, s_l[warp] = l;
  __syncthreads();
  if (threadIdx.x < D) {
    const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    float sum = 0.f, x = 0.f;
    for (int w = 0; w < 4; ++w) {
      const float f = s_l[w] != 0.f ? exp2f(s_m[w] - top) : 0.f;
      sum += f * s_l[w];
      x += f * s_row[w][threadIdx.x];
    }
    out[threadIdx.x] = __bfloat16_as_ushort(__float2bfloat16_rn(sum != 0.f ? x / sum : 0.f));
  }
}

int64_t group_workspace_bytes(const Layout&) { return 256; }

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
  cache_note_call(cache, layer);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (launch_pdl(group_check_kernel, dim3(1), dim3(1024), 0, s, g) != cudaSuccess ||
      launch_pdl(l.d == 64 ? group_attn_kernel<64> : group_attn_kernel<128>, dim3(n * l.Hq), dim3(128), 0, s, g) != cudaSuccess)
    return TRR_ERR_CUDA;
  cache_set_launches(cache, 2);
  return TRR_OK;
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
