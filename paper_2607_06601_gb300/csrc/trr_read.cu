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
constexpr int kReadCtas = 3;  // CTAs on an SM

struct ReadArgs {
  LayerArgs a;
  int n, rows, splits;  // stretches, rows of the outputs, shares of the KV heads that CTAs take
  const int32_t *seq_ids, *starts, *offsets;
  void *k, *v;
  uint8_t* bits;
  int64_t k_stride, v_stride;  // elements from a row to the next
  int sectors;                 // every row starts at 32 bytes
};

// z + c s of eight elements of b bits, in binary32.
template <int B>
__device__ __forceinline__ void expand_f32(uint32_t w0, uint32_t w1, uint32_t sz, float (&v)[8]) {
  const float s = __low2float(as_half2(sz)), z = __high2float(as_half2(sz));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t w = B == 8 && i >= 4 ? w1 : w0;
    const uint32_t c = B == 8 ? __byte_perm(w, 0x4B000000u, 0x7540 + (i & 3)) : ((w >> (B * i)) & ((1u << B) - 1)) | 0x4B000000u;
    v[i] = __fmaf_rn(__uint_as_float(c) - 8388608.f, s, z);  // 2^23 + c as binary32: the difference is exact
  }
}

// Eight elements of half `k` of a lane's sixteen.
__device__ __forceinline__ void expand(const Codes16& x, int cls, int k, float (&v)[8]) {
  const uint4 w = x.w[0];
  if (cls == 3) {
    const uint4 y = x.w[k];
    const uint32_t u[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16lo(u[i]), v[2 * i + 1] = bf16hi(u[i]);
  } else if (cls == 2) {
    expand_f32<8>(k ? w.z : w.x, k ? w.w : w.y, x.sz, v);
  } else if (cls == 1) {
    expand_f32<4>(k ? w.y : w.x, 0, x.sz, v);
  } else if (cls == 0) {
    expand_f32<2>(k ? w.x >> 16 : w.x, 0, x.sz, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
  }
}

__device__ __forceinline__ uint4 as_bf16(const float (&v)[8]) {
  return make_uint4(pack16(true, v[0], v[1]), pack16(true, v[2], v[3]), pack16(true, v[4], v[5]), pack16(true, v[6], v[7]));
}
__device__ __forceinline__ uint4 bits_of(const float* v) {
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}

// The tokens that the CTA has found, of heads h0 .. h1 - 1: a warp takes eight (d 64) or four rows of a head's K or V
// of one class at a time, 16 elements a lane.  Sector: rows start at 32 bytes.
template <int D, typename T>
__device__ __forceinline__ void copy_rows(const ReadArgs& g, const Found& f, int h0, int h1) {
  constexpr int kLanes = D / 16, kRows = 32 / kLanes, kAhead = 4;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = lane % kLanes, lg_group = __ffs(g.a.G) - 1;
  const int groups = f.groups(kRows), items = 2 * (h1 - h0) * groups;
  for (int x0 = warp; x0 < items; x0 += kAhead * (kSpanThreads / 32)) {
    Codes16 x[kAhead];
    int cls[kAhead], row[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int item = x0 + u * (kSpanThreads / 32), j = item / groups, h = h0 + (j >> 1);
      cls[u] = kClasses;
      row[u] = -1;
      if (item >= items) continue;
      int first, n;
      cls[u] = f.group(item - j * groups, kRows, &first, &n);
      const int t = first + lane / kLanes;
      if (t >= n) continue;
      const Found::Token& tok = f.token[cls[u]][t];
      row[u] = tok.row;
      if (g.a.maskb && cls[u] < kClasses) {  // per-head modes: the token may not store this head
        const uint8_t* slice = tok.page + g.a.hdr + static_cast<int64_t>(h) * g.a.slice[cls[u]];
        if (!(*reinterpret_cast<const uint64_t*>(slice + g.a.slice[cls[u]] - g.a.maskb) >> tok.slot & 1)) cls[u] = kClasses;
      }
      if (cls[u] < kClasses) x[u] = load_codes16<D>(g.a, cls[u], tok.page, tok.slot, h, j & 1, e, lg_group);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (row[u] < 0) continue;
      const int j = (x0 + u * (kSpanThreads / 32)) / groups, h = h0 + (j >> 1);
      T* to = static_cast<T*>(j & 1 ? g.v : g.k) + row[u] * (j & 1 ? g.v_stride : g.k_stride) + h * D + 16 * e;
      float v[8];
      uint4 o[4];
      expand(x[u], cls[u], 0, v);
      if (sizeof(T) == 2) o[0] = as_bf16(v);
      else o[0] = bits_of(v), o[1] = bits_of(v + 4);
      expand(x[u], cls[u], 1, v);
      if (sizeof(T) == 2) o[1] = as_bf16(v);
      else o[2] = bits_of(v), o[3] = bits_of(v + 4);
      if (g.sectors) {
        store_sector(to, o[0], o[1]);
        if (sizeof(T) == 4) store_sector(to + 8, o[2], o[3]);
      } else {
#pragma unroll
        for (int k = 0; k < static_cast<int>(sizeof(T)); ++k) reinterpret_cast<uint4*>(to)[k] = o[k];
      }
      if (g.bits && (j & 1) == 0 && e == 0) g.bits[static_cast<int64_t>(row[u]) * g.a.Hkv + h] = cls[u] < kClasses ? 2 << cls[u] : 0;
    }
  }
}

template <int D, typename T>
__global__ void __launch_bounds__(kSpanThreads, kReadCtas) read_kernel(const __grid_constant__ ReadArgs g) {
  __shared__ Found f;
  __shared__ int s_bad;
  const LayerArgs& a = g.a;
  const int i = threadIdx.x >> 2, c = threadIdx.x & 3;
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
    f.gather(a, p, c, mine ? row : -1, threadIdx.x);
    copy_rows<D, T>(g, f, h0, h1);
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
  const int64_t size = type == TRR_BF16 ? 2 : 4;
  g.sectors = ((reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out) | static_cast<uint64_t>(k_stride * size) |
                static_cast<uint64_t>(v_stride * size)) & 31) == 0;
  const int sms = cache_num_sms(cache), spans = (num_rows - 1) / kSpan + 1;
  // a small call's heads are shared out among CTAs, so that it fills the GPU too
  const int most = (2 * l.Hkv + kSpanThreads / 32 - 1) / (kSpanThreads / 32);
  g.splits = std::max(1, std::min(most, kReadCtas * sms / spans));
  const int64_t units = static_cast<int64_t>(spans) * g.splits;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(units, kReadCtas * sms)));
  auto kernel = l.d == 64 ? (type == TRR_BF16 ? read_kernel<64, uint16_t> : read_kernel<64, float>)
                          : (type == TRR_BF16 ? read_kernel<128, uint16_t> : read_kernel<128, float>);
  cache_note_call(cache, layer);
  const cudaError_t e = launch_pdl(kernel, grid, dim3(kSpanThreads), 0, static_cast<cudaStream_t>(stream), g);
  cache_set_launches(cache, e == cudaSuccess ? 1 : 0);
  return e == cudaSuccess ? TRR_OK : TRR_ERR_CUDA;
}
