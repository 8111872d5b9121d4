// trr_read.cu - trr_kv_read: stretches of a cache read back, dequantised, in order of position.
//
//   k_out[r][h][j] = z + c_j s (2, 4 and 8 bits) or the stored bf16 (16 bits) of the token at row r's
//   position, 0 where none is stored; so for V; bits_out[r][h] its width, or 0.
//
// c s is exact in binary32 (8 bits times 11) and the sum is rounded once there; a bf16 output is
// rounded once more, to 8 bits.
//
// Bound by the memory: a token of 64 dimensions comes in as 90 bytes (K and V, 4.5 bits a value on
// average) and leaves as 256.  A warp takes one head's K and V rows of a class at a time, 16 values a
// lane, consecutive lanes along a row, so that whole lines are written.
//
// Alone, from cold caches, 65,536 rows of 12 heads of 64 in bf16 take 58 us, 40,000 of 32 heads in binary32 141 us (DRAM
// 5.2 TB/s, 112 MB read and 623 written), 131,072 of 8 heads of 128 in bf16 122 us; a copy of as many
// bytes 40, 114 and 96.  What is left are the searches before a CTA's first rows (5 us in which
// nothing is written) and the loads' latency under so many stores.  Two heads' loads ahead at 80 registers
// and three CTAs an SM were no gain: 71, 149 and 132 us a whole call where one head's at four CTAs then took 69, 153
// and 138.  At 64 registers 32 to 44 bytes a thread are spilled.
#include <algorithm>
#include <climits>
#include <cstdint>

#include "trr_span.cuh"

namespace trr {

constexpr int kMostRows = 1 << 30;
constexpr int kReadCtas = 4;  // CTAs on an SM

struct ReadArgs {
  LayerArgs a;
  int n, rows, span, splits;  // stretches, rows of the outputs; how many of them, and shares of the KV heads, CTAs take
  const int32_t *seq_ids, *starts, *offsets;
  void *k, *v;
  uint8_t* bits;
  int64_t k_stride, v_stride;  // elements from a row to the next
  int sectors;                 // every row starts at 32 bytes
  int lg_parts;                // a CTA's warps share a group's heads out in 2^lg_parts parts
};

__device__ __forceinline__ uint4 as_bf16(const float* v) {
  return make_uint4(pack16(true, v[0], v[1]), pack16(true, v[2], v[3]), pack16(true, v[4], v[5]), pack16(true, v[6], v[7]));
}
__device__ __forceinline__ uint4 bits_of(const float* v) {
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}

__device__ __forceinline__ void store16(const ReadArgs& g, uint16_t* to, const float (&v)[16]) {
  const uint4 a = as_bf16(v), b = as_bf16(v + 8);
  if (g.sectors) {
    store_sector(to, a, b);
  } else {
    reinterpret_cast<uint4*>(to)[0] = a;
    reinterpret_cast<uint4*>(to)[1] = b;
  }
}
__device__ __forceinline__ void store16(const ReadArgs& g, float* to, const float (&v)[16]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint4 a = bits_of(v + 8 * k), b = bits_of(v + 8 * k + 4);
    if (g.sectors) {
      store_sector(to + 8 * k, a, b);
    } else {
      reinterpret_cast<uint4*>(to + 8 * k)[0] = a;
      reinterpret_cast<uint4*>(to + 8 * k)[1] = b;
    }
  }
}

// A token's rows of every step-th head: 16 elements a lane of K and of V.
template <int C, int D, typename T>
__device__ __forceinline__ void copy_token(const ReadArgs& g, const uint8_t* page, int slot, int row, bool live, int h0, int h1, int step, int e) {
  const CodesAt<C == kClasses ? 0 : C, D> at(g.a, slot, e);
  T* k = static_cast<T*>(g.k) + row * g.k_stride + 16 * e;
  T* v = static_cast<T*>(g.v) + row * g.v_stride + 16 * e;
  if (!live) return;
  const int64_t slice_bytes = g.a.slice[C == kClasses ? 0 : C];
  const uint8_t* slice = page + g.a.hdr + h0 * slice_bytes;
  // a head's codes are asked for before the last head's are written: nothing moves a load over a store by itself
  Codes16 ck = {}, cv = {};
  bool there = false;
  auto load = [&](int h) {
    there = C != kClasses && h < h1;
    if (there && g.a.maskb)  // per-head modes: the token may not store this head
      there = *reinterpret_cast<const uint64_t*>(slice + slice_bytes - g.a.maskb) >> slot & 1;
    if (there) ck = at.load(slice, 0), cv = at.load(slice, 1);
    slice += step * slice_bytes;
  };
  load(h0);
#pragma unroll 1
  for (int h = h0; h < h1; h += step) {
    const Codes16 k0 = ck, v0 = cv;
    const bool now = there;
    load(h + step);
    float x[16];
    if (now) expand_f32<C>(k0, x);
    else expand_f32<kClasses>(k0, x);
    store16(g, k + h * D, x);
    if (now) expand_f32<C>(v0, x);
    else expand_f32<kClasses>(v0, x);
    store16(g, v + h * D, x);
    if (g.bits && e == 0) g.bits[static_cast<int64_t>(row) * g.a.Hkv + h] = now ? 2 << C : 0;
  }
}

template <int D, typename T>
__global__ void __launch_bounds__(kSpanThreads, kReadCtas) read_kernel(const __grid_constant__ ReadArgs g) {
  constexpr int kLanes = D / 16;
  __shared__ Found<32 / kLanes> f;
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
  const int units = (g.rows + g.span - 1) / g.span * g.splits, per = (a.Hkv + g.splits - 1) / g.splits;
  const int row_end = bad ? g.rows : g.offsets[g.n], row_begin = bad ? 0 : g.offsets[0];
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    const int row = u / g.splits * g.span + i, h0 = u % g.splits * per, h1 = min(a.Hkv, h0 + per);
    const bool mine = i < g.span && row >= row_begin && row < row_end;
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
    for_groups(f, g.lg_parts, h0, [&](int cls, const auto& tok, bool live, int h, int step) {
      const int e = threadIdx.x % kLanes;
      if (cls == 0) copy_token<0, D, T>(g, tok.page, tok.slot, tok.row, live, h, h1, step, e);
      else if (cls == 1) copy_token<1, D, T>(g, tok.page, tok.slot, tok.row, live, h, h1, step, e);
      else if (cls == 2) copy_token<2, D, T>(g, tok.page, tok.slot, tok.row, live, h, h1, step, e);
      else if (cls == 3) copy_token<3, D, T>(g, tok.page, tok.slot, tok.row, live, h, h1, step, e);
      else copy_token<kClasses, D, T>(g, nullptr, 0, tok.row, live, h, h1, step, e);
    });
  }
  __syncthreads();
  if (threadIdx.x == 0 && atom_add_acq_rel(a.ctrl + kReadDone, 1) == static_cast<int>(gridDim.x) - 1) {
    const int e = atomicExch(a.ctrl + kReadBad, 0);
    if (e) set_status(a.ctrl, (INT_MAX - e) & 15);
    a.ctrl[kReadDone] = 0;
  }
}

// How the rows are cut into units: some of them (48 to 64) of a share of the heads.  With the heads in s shares a unit has
// as many rows as fill the fewest rounds of `ctas` CTAs evenly; of all s the one that takes least, where 64 rows of all
// heads take `whole` ns among as many others and a unit 5 us more to find its tokens.  Whole calls with cold caches, against units of 64
// rows always: 65,536 rows of 12 heads of 64 in bf16 65 us against 69 (2 rounds of 54 rows, the second one was 0.7 full),
// 131,072 of 8 heads of 128 130 against 138; with 32 rows as the least, 40,000 of 32 heads in binary32 157 against 153.
struct Shares {
  int span, splits;  // rows; shares of the heads
};
static Shares shares_of(int64_t rows, int heads, int ctas, int64_t whole) {
  constexpr int64_t kLeastSpan = 48;
  Shares best = {kSpan, 1};
  int64_t least = INT64_MAX;
  for (int s = 1; s <= (heads + 1) / 2; ++s) {
    const int64_t units = (rows + kSpan - 1) / kSpan, rounds = (units * s + ctas - 1) / ctas, room = rounds * ctas / s;
    const int64_t span = std::max(kLeastSpan, (rows + room - 1) / room), per = (heads + s - 1) / s;
    const int64_t t = rounds * (whole * span * per / (kSpan * heads) + 5000);
    if (t < least) best = Shares{static_cast<int>(span), s}, least = t;
  }
  return best;
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
  const int64_t row = static_cast<int64_t>(l.Hkv) * l.d, unit_bytes = type == TRR_BF16 ? 2 : 4, unit = 16 / unit_bytes;
  if (k_stride < row || v_stride < row || k_stride % unit || v_stride % unit) return TRR_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) & 15) return TRR_ERR_INVALID_ARG;
  ReadArgs g;
  g.a = layer_args(l, cache_views(cache), layer);
  g.n = n; g.rows = num_rows;
  g.seq_ids = seq_ids; g.starts = starts; g.offsets = offsets;
  g.k = k_out; g.v = v_out; g.bits = bits_out;
  g.k_stride = k_stride; g.v_stride = v_stride;
  g.sectors = ((reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out) | static_cast<uint64_t>(k_stride * unit_bytes) |
                static_cast<uint64_t>(v_stride * unit_bytes)) & 31) == 0;
  const int sms = cache_num_sms(cache);
  // (half a byte a value in, on average)
  const int64_t bytes = 2 * row * unit_bytes + row;
  const Shares shares = shares_of(num_rows, l.Hkv, kReadCtas * sms, copy_ns(bytes, kReadCtas * sms));
  g.span = shares.span;
  g.splits = shares.splits;
  const int64_t units = static_cast<int64_t>((num_rows - 1) / g.span + 1) * g.splits;
  g.lg_parts = lg_parts((l.Hkv + g.splits - 1) / g.splits);
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(units, kReadCtas * sms)));
  auto kernel = l.d == 64 ? (type == TRR_BF16 ? read_kernel<64, uint16_t> : read_kernel<64, float>)
                          : (type == TRR_BF16 ? read_kernel<128, uint16_t> : read_kernel<128, float>);
  cache_note_call(cache, layer);
  const cudaError_t e = launch_pdl(kernel, grid, dim3(kSpanThreads), 0, static_cast<cudaStream_t>(stream), g);
  cache_set_launches(cache, e == cudaSuccess ? 1 : 0);
  return e == cudaSuccess ? TRR_OK : TRR_ERR_CUDA;
}
