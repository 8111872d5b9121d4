// trr_read.cu - trr_kv_read: stretches of a cache read back, dequantised, in order of position.
//
//   k_out[r][h][j] = z + c_j s (2, 4 and 8 bits) or the stored bf16 (16 bits) of the token at row r's
//   position, 0 where none is stored; so for V; bits_out[r][h] its width, or 0.
//
// c s is exact in binary32 (8 bits times 11) and the sum is rounded once there; a bf16 output is
// rounded once more, to 8 bits.
//
// Bound by the memory: a token of 64 dimensions comes in as 90 bytes (K and V, 4.5 bits a value on
// average) and leaves as 256.  A warp takes one head's K or V rows of a class at a time, 16 bytes of
// bf16 a lane, consecutive lanes along a row, so that whole lines are written.
#include <algorithm>
#include <climits>

#include "trr_span.cuh"

namespace trr {

constexpr int kMostRows = 1 << 30;

struct ReadArgs {
  LayerArgs a;
  int n, rows, splits;  // stretches, rows of the outputs, shares of the KV heads that CTAs take
  const int32_t *seq_ids, *starts, *offsets;
  void *k, *v;
  uint8_t* bits;
  int64_t k_stride, v_stride;  // elements from a row to the next
};

// z + c s of eight elements, in binary32.
template <int B>
__device__ __forceinline__ void expand_f32(const Codes& x, float (&v)[8]) {
  if (B == 16) {
    const uint32_t w[4] = {x.w.x, x.w.y, x.w.z, x.w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16lo(w[i]), v[2 * i + 1] = bf16hi(w[i]);
    return;
  }
  const float s = __low2float(as_half2(x.sz)), z = __high2float(as_half2(x.sz));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t w = B == 8 && i >= 4 ? x.w.y : x.w.x;
    const uint32_t c = B == 8 ? __byte_perm(w, 0x4B000000u, 0x7540 + (i & 3)) : ((w >> (B * i)) & ((1u << B) - 1)) | 0x4B000000u;
    v[i] = __fmaf_rn(__uint_as_float(c) - 8388608.f, s, z);  // 2^23 + c as binary32: the difference is exact
  }
}

__device__ __forceinline__ void store8(float* to, const float (&v)[8]) {
  reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(uint16_t* to, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&x);
  }
  *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Rows of one class (B 0: rows of zeros), heads h0 .. h1 - 1; a warp takes a head's K or V.
template <int B, int D, typename T>
__device__ __forceinline__ void copy_rows(const ReadArgs& g, const Found& f, int h0, int h1) {
  constexpr int c = B == 0 ? kClasses : B == 2 ? 0 : B == 4 ? 1 : B == 8 ? 2 : 3, kLanes = D / 8, kStep = 32 / kLanes, kAhead = 4;
  const int n = f.count[c], lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = lane % kLanes, lg_group = __ffs(g.a.G) - 1;
  if (n == 0) return;
  for (int j = 2 * h0 + warp; j < 2 * h1; j += kSpanThreads / 32) {
    const int h = j >> 1, which = j & 1;
    T* out = static_cast<T*>(which ? g.v : g.k) + h * D + 8 * e;
    const int64_t stride = which ? g.v_stride : g.k_stride;
    for (int t0 = lane / kLanes; t0 < n; t0 += kAhead * kStep) {
      Codes x[kAhead];
      bool there[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int t = t0 + u * kStep;
        there[u] = t < n;
        if (B != 0 && there[u]) {
          const Found::Token& tok = f.token[c][t];
          if (g.a.maskb) {  // per-head modes: the token may not store this head
            const uint8_t* slice = tok.page + g.a.hdr + static_cast<int64_t>(h) * g.a.slice[c];
            there[u] = *reinterpret_cast<const uint64_t*>(slice + g.a.slice[c] - g.a.maskb) >> tok.slot & 1;
          }
          if (there[u]) x[u] = load_codes<B == 0 ? 2 : B, D>(g.a, tok.page, tok.slot, h, which, e, lg_group);
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int t = t0 + u * kStep;
        if (t >= n) continue;
        const int row = f.token[c][t].row;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (B != 0 && there[u]) expand_f32<B == 0 ? 2 : B>(x[u], v);
        store8(out + row * stride, v);
        if (g.bits && which == 0 && e == 0) g.bits[static_cast<int64_t>(row) * g.a.Hkv + h] = B != 0 && there[u] ? B : 0;
      }
    }
  }
}

template <int D, typename T>
__global__ void __launch_bounds__(kSpanThreads) read_kernel(const __grid_constant__ ReadArgs g) {
  __shared__ Found f;
  __shared__ int s_bad;
  const LayerArgs& a = g.a;
  const int i = threadIdx.x >> 2, c = threadIdx.x & 3, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) s_bad = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  for (int x = threadIdx.x; x <= g.n; x += kSpanThreads) {
    const int o = g.offsets[x], next = x < g.n ? g.offsets[x + 1] : o;
    if (o < 0 || o > g.rows || next < o) s_bad = 1;
  }
  __syncthreads();
  const bool bad = s_bad;
  // errors: the lowest failing stretch's, kept as INT_MAX - (16 stretch + error) so that 0 means none
  auto fail = [&](int at, int err) { atomicMax(a.ctrl + kReadBad, INT_MAX - (16 * at + err)); };
  if (bad) {
    if (blockIdx.x == 0 && threadIdx.x == 0) fail(0, TRR_ERR_INVALID_ARG);
  } else if (blockIdx.x == 0) {
    for (int x = threadIdx.x; x < g.n; x += kSpanThreads) {
      const int seq = g.seq_ids[x], start = g.starts[x], len = g.offsets[x + 1] - g.offsets[x];
      if (len == 0) continue;
      if (seq < 0 || seq >= a.S) fail(x, TRR_ERR_INVALID_ARG);
      else if (start < 0 || start > a.maxctx - len) fail(x, TRR_ERR_BAD_POSITION);
    }
  }
  const int units = (g.rows + kSpan - 1) / kSpan * g.splits, per = (a.Hkv + g.splits - 1) / g.splits;
  const int row_end = bad ? g.rows : g.offsets[g.n], row_begin = bad ? 0 : g.offsets[0];
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    const int row = u / g.splits * kSpan + i, h0 = u % g.splits * per, h1 = min(a.Hkv, h0 + per);
    __syncthreads();  // the last unit's tokens have been read
    if (threadIdx.x <= kClasses) f.count[threadIdx.x] = 0;
    __syncthreads();
    const bool mine = row >= row_begin && row < row_end;
    Place p{0, -1, 0};
    if (mine && !bad) {
      int lo = 0, hi = g.n - 1;  // the last stretch that starts at the row or before it
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (g.offsets[mid] <= row) lo = mid;
        else hi = mid - 1;
      }
      const int seq = g.seq_ids[lo], start = g.starts[lo], len = g.offsets[lo + 1] - g.offsets[lo];
      if (seq >= 0 && seq < a.S && start >= 0 && start <= a.maxctx - len) p = place_of(a, seq, c, start + row - g.offsets[lo]);
    }
    const bool here = p.page >= 0;
    const bool any = __ballot_sync(0xffffffffu, here) >> (lane & ~3) & 15;
    if (here) f.token[c][atomicAdd(&f.count[c], 1)] = Found::Token{a.pool[c] + p.page * a.page_bytes[c], p.slot, row};
    if (mine && !any && c == 0) f.token[kClasses][atomicAdd(&f.count[kClasses], 1)] = Found::Token{nullptr, 0, row};
    __syncthreads();
    copy_rows<16, D, T>(g, f, h0, h1);
    copy_rows<8, D, T>(g, f, h0, h1);
    copy_rows<4, D, T>(g, f, h0, h1);
    copy_rows<2, D, T>(g, f, h0, h1);
    copy_rows<0, D, T>(g, f, h0, h1);
  }
  __syncthreads();
  if (threadIdx.x == 0 && atom_add_acq_rel(a.ctrl + kReadDone, 1) == static_cast<int>(gridDim.x) - 1) {
    const int e = atomicExch(a.ctrl + kReadBad, 0);
    if (e) set_status(a.ctrl, (INT_MAX - e) & 15);
    a.ctrl[kReadDone] = 0;
  }
}

}  // namespace trr

using namespace trr;

extern "C" trr_status trr_kv_read(trr_cache* cache, int32_t layer, int32_t n, const int32_t* seq_ids, const int32_t* starts,
                                  const int32_t* offsets, int32_t num_rows, int32_t type, void* k_out, int64_t k_stride,
                                  void* v_out, int64_t v_stride, uint8_t* bits_out, void* stream) {
  if (!cache) return TRR_ERR_INVALID_ARG;
  const Layout& l = cache_layout(cache);
  if (layer < 0 || layer >= l.L || n < 0 || n > kMostSpans || num_rows < 0 || num_rows > kMostRows || (type != TRR_BF16 && type != TRR_F32)) return TRR_ERR_INVALID_ARG;
  cache_set_launches(cache, 0);
  if (n == 0 || num_rows == 0) return TRR_OK;
  if (!seq_ids || !starts || !offsets || !k_out || !v_out) return TRR_ERR_INVALID_ARG;
  const int64_t row = static_cast<int64_t>(l.Hkv) * l.d, unit = type == TRR_BF16 ? 8 : 4;
  if (k_stride < row || v_stride < row || k_stride % unit || v_stride % unit) return TRR_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) & 15) return TRR_ERR_INVALID_ARG;
  ReadArgs g;
  g.a = layer_args(l, cache_views(cache), layer);
  g.n = n; g.rows = num_rows;
  g.seq_ids = seq_ids; g.starts = starts; g.offsets = offsets;
  g.k = k_out; g.v = v_out; g.bits = bits_out;
  g.k_stride = k_stride; g.v_stride = v_stride;
  const int sms = cache_num_sms(cache), spans = (num_rows - 1) / kSpan + 1;
  // a small call's heads are shared out among CTAs, so that it fills the GPU too
  const int most = (2 * l.Hkv + kSpanThreads / 32 - 1) / (kSpanThreads / 32);
  g.splits = std::max(1, std::min(most, 8 * sms / spans));
  const int64_t units = static_cast<int64_t>(spans) * g.splits;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(units, 8 * sms)));
  auto kernel = l.d == 64 ? (type == TRR_BF16 ? read_kernel<64, uint16_t> : read_kernel<64, float>)
                          : (type == TRR_BF16 ? read_kernel<128, uint16_t> : read_kernel<128, float>);
  cache_note_call(cache, layer);
  const cudaError_t e = launch_pdl(kernel, grid, dim3(kSpanThreads), 0, static_cast<cudaStream_t>(stream), g);
  cache_set_launches(cache, e == cudaSuccess ? 1 : 0);
  return e == cudaSuccess ? TRR_OK : TRR_ERR_CUDA;
}
