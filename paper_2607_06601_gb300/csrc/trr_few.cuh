// trr_few.cuh - attention of a segment with few rows (the query heads of one KV head, for one
// query or for a small group): warps that work alone, on codes as they are stored.
//
// Every warp takes one equal run of blocks (up to 32 tokens of a page, for one KV head) of the
// call's private segments, laid end to end.  It brings the blocks into its own ring of shared
// memory with bulk copies issued several blocks ahead, and multiplies with warp-wide products
// of 16 x 8 x 16 (binary32 sums):
//   scores   S^T = K Q^T: 16 tokens x 8 columns.  A column is a (query head, group) pair: the
//            query row restricted to one quantiser group, so that sum_g s_g (q c)_g + z_g sum(q)_g
//            needs only the codes.  Rows are 16 tokens; a quad of lanes holds a token's row, a
//            lane a quarter of it in a run, so codes come in whole words.
//   output   O^T += V^T W: 16 dimensions x 8 columns, W = p s.  A lane holds an eighth of the
//            dimensions of two pairs of tokens; byte permutes pair the tokens' codes.
// A code is used as the binary16 number `offset + code` made by setting its bits under an
// exponent (16 + c, 4 + c, 1024 + c for 4, 2, 8 bits: no conversion, no subtraction).  The offset's
// part of a score is taken off in binary32; that of the output, and half the codes' range with it,
// by a product of the same weights with a constant, block by block, so that the running sums hold
// centred values: z + s (middle of the range), the rest of a value, is added up apart.
//
// The softmax reference m follows the largest score plus log2 of the token's V scale, so that
// W = p s stays below 2^9 in binary16 whatever the size of the values; 16-bit pages keep p as a
// sum of two bf16 numbers.  Groups of a row share the reference: one whose scale is a thousand times
// below the other's keeps fewer bits of its own dimensions (an error 11 times the output's rounding
// there, and none that the row's largest values would show).
//
// What bounds it: instructions and their latency (four warps a scheduler keep it half busy): about
// 230 for 16 tokens of a KV head and as many for each block, whatever the width.  The partial
// pages at a window's edge and the sinks' add half as many bytes again.
//
// Measured by itself, caches cold, on 64 queries of 32 heads of 64 with windows of 511 and 16 sinks
// (67.5 MB, 10 us at the copy rate): 41 us, 1.6 TB/s; 128 queries on 8 KV heads of 128 with windows
// of 1024 (95.4 MB): 53 us, 1.8 TB/s.  The product that centres the codes costs 0 to 2 % of that.
#pragma once

#include "trr_group.cuh"

namespace trr {

constexpr int kFewWarps = 8;      // warps of a CTA
constexpr int kFewCtas = 2;       // CTAs of an SM (three of 80 registers a thread are slower: 56 us against 44 then, on those 64 queries)
constexpr int kFewStages = 8;     // blocks in a warp's ring
constexpr int kFewRows = 8;       // most rows of a segment
constexpr int kFewSmem = 112 * 1024;  // of a CTA

// Where a warp's copies stand; in shared memory, since few instructions of a block need it.
struct FewCursor {
  int64_t b0, b1, base;         // the warp's run of cost, the job's start
  int j, seg, tile0, pad0;      // job, segment, its first block for this warp
  int tiles, pages_q;           // the job's blocks, its pages of 2, 4 and 8 bits
};

// A block in the ring.
struct FewBlock {
  int cls, keys, off, pos;      // pos < 0: all its tokens are in sight
  int valid, lo, t, sinks;
  int kind, qbase, kvh, rows;   // the segment, as in its job
  int dest, state, pad[2];      // state: 1 first block of a segment's piece, 2 last one
};

template <int D, int NG>
struct FewSmem {
  static constexpr int kQ = kFewRows / NG * D * 2;                          // query rows in binary16, then in bf16, scaled
  static constexpr int kFactor = 2 * kQ;                               // a factor for each row, sums of its groups
  static constexpr int kRowIds = kFactor + 4 * kFewRows + 4 * kFewRows * 4;  // query * Hq + head of each row
  static constexpr int kBlocks = kRowIds + 4 * kFewRows;
  static constexpr int kJob = kBlocks + kFewStages * static_cast<int>(sizeof(FewBlock));  // the cursor's job
  static constexpr int kCursor = kJob + static_cast<int>(sizeof(Job));
  static constexpr int kBars = kCursor + static_cast<int>(sizeof(FewCursor));
  static constexpr int kRing = (kBars + 8 * kFewStages + 127) / 128 * 128;
  static constexpr int kWarp = kFewSmem / kFewWarps / 128 * 128;  // a warp's share
  static constexpr int kRingBytes = kWarp - kRing;
};
static_assert(FewSmem<64, 1>::kRingBytes >= 32 * 136 + 128 && FewSmem<64, 2>::kRingBytes >= 32 * 144 + 128 &&
                  FewSmem<128, 1>::kRingBytes >= 32 * 264 + 128 && FewSmem<128, 4>::kRingBytes >= 32 * 288 + 128,
              "the widest blocks");

// A code as a binary16 number has kOffset added to it; kMiddle lies halfway between a class's least
// and largest code, and kMinus is -(kOffset + kMiddle) twice.
template <int B>
struct Codes;
template <>
struct Codes<2> { static constexpr float kOffset = 4.f, kMiddle = 1.5f; static constexpr uint32_t kMinus = 0xC580C580u; };
template <>
struct Codes<4> { static constexpr float kOffset = 16.f, kMiddle = 7.5f; static constexpr uint32_t kMinus = 0xCDE0CDE0u; };
template <>
struct Codes<8> { static constexpr float kOffset = 1024.f, kMiddle = 128.f; static constexpr uint32_t kMinus = 0xE480E480u; };
template <>
struct Codes<16> { static constexpr float kOffset = 0.f, kMiddle = 0.f; static constexpr uint32_t kMinus = 0; };

// Codes i of both 16-bit halves of x as binary16 numbers offset + code.
__device__ __forceinline__ uint32_t codes4(uint32_t x, int i) {
  const uint32_t y = i == 0 ? x << 6 : i == 1 ? x << 2 : i == 2 ? x >> 2 : x >> 6;
  return (y & 0x03C003C0u) | 0x4C004C00u;
}
__device__ __forceinline__ uint32_t codes2(uint32_t x, int i) {
  const uint32_t y = i < 4 ? x << (8 - 2 * i) : x >> (2 * i - 8);
  return (y & 0x03000300u) | 0x44004400u;
}

template <bool BF16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// One warp's running state of a segment.
template <int D, int NG>
struct FewState {
  static constexpr int kSteps = D / 16;          // products over the dimensions
  static constexpr int kHeads = NG == 1 ? 2 : 1; // query heads of the lane's two columns
  float acc[kSteps][4];                          // O^T: dimensions 2 i, 2 i + 1 of the lane's run x its two columns
  float m[kHeads], l[kHeads], f[kHeads];         // reference, sum, factor from products to base-2 exponents
  float corr[2];                                 // sum p (z + s kMiddle) of the lane's columns
  float qsum[2];
  uint32_t q[kSteps][2];                         // the columns' query rows, in the order of q_class's codes
  int q_class;
};

// The query rows as the second operand, in the order in which class B's codes come out of their
// words (4 bits: elements i and i + 4 together, 2 bits: i and i + 8).
template <int D, int NG, int B>
__device__ __forceinline__ void few_load_q(FewState<D, NG>& s, const uint8_t* smem, int rows, int lane) {
  const int n = lane >> 2, part = lane & 3, head = n / NG;
  const bool live = head < rows && part * NG / 4 == n % NG;  // the lane's dimensions lie in the column's group
  const uint4* row = reinterpret_cast<const uint4*>(smem + (B == 16 ? FewSmem<D, NG>::kQ : 0) + ((live ? head : 0) * D + part * (D / 4)) * 2);
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {  // 16 elements
    uint4 u = row[2 * i], v = row[2 * i + 1];
    if (!live) u = v = make_uint4(0, 0, 0, 0);
    const uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (B == 2) {
        s.q[4 * i + t][0] = __byte_perm(w[t], w[t + 4], 0x5410);
        s.q[4 * i + t][1] = __byte_perm(w[t], w[t + 4], 0x7632);
      } else if (B == 4) {
        const int k = t / 2 * 4 + t % 2;
        s.q[4 * i + t][0] = __byte_perm(w[k], w[k + 2], 0x5410);
        s.q[4 * i + t][1] = __byte_perm(w[k], w[k + 2], 0x7632);
      } else {
        s.q[4 * i + t][0] = w[2 * t];
        s.q[4 * i + t][1] = w[2 * t + 1];
      }
    }
  }
  s.q_class = B;
}

// 16 tokens of a block of `keys`, from token b on: K codes, V codes, K scales, V scales side by
// side at blk; bit k of mask: token b + k is in sight.
template <int D, int NG, int B>
__device__ __forceinline__ void few_tokens(FewState<D, NG>& s, const uint8_t* blk, int keys, int b, uint32_t mask, bool swz, int lane) {
  using S = FewState<D, NG>;
  constexpr int kRow = D * B / 8;
  constexpr float kOff = Codes<B>::kOffset;
  const int quad = lane >> 2, part = lane & 3;
  const int flip = swz ? 0x70 : 0;  // permuted rows: chunk ^ line % 8 (swz_off)
  auto at = [&](int o) { return blk + (B >= 8 ? o ^ ((o >> 3) & flip) : o); };
  const uint32_t* ksz = reinterpret_cast<const uint32_t*>(blk + 2 * keys * kRow);
  const uint32_t* vsz = ksz + keys * NG;
  const int g0 = NG == 1 ? 0 : (2 * part) % NG;  // the group of the lane's first column; the second's is the next
  auto scales = [&](const uint32_t* sz, int key, uint32_t (&to)[2]) {
    if (NG == 1) {
      to[0] = to[1] = sz[key];
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(sz + key * NG + g0);
      to[0] = u.x;
      to[1] = u.y;
    }
  };

  float x[2][S::kHeads];      // scores in base-2 exponents of tokens b + quad and + 8
  uint32_t vs[2][2];          // V's (scale, zero) of the lane's tokens and columns
  float top[S::kHeads];
#pragma unroll
  for (int h = 0; h < S::kHeads; ++h) top[h] = -INFINITY;
  {
    float c[4] = {0.f, 0.f, 0.f, 0.f};
    const int k0 = (b + quad) * kRow + part * (kRow / 4), k1 = k0 + 8 * kRow;
    if (B == 2) {
#pragma unroll
      for (int w = 0; w < D / 64; ++w) {
        const uint32_t u = *reinterpret_cast<const uint32_t*>(blk + k0 + 4 * w), v = *reinterpret_cast<const uint32_t*>(blk + k1 + 4 * w);
#pragma unroll
        for (int t = 0; t < 4; ++t)
          mma16816<false>(c, codes2(u, 2 * t), codes2(v, 2 * t), codes2(u, 2 * t + 1), codes2(v, 2 * t + 1), s.q[4 * w + t][0], s.q[4 * w + t][1]);
      }
    } else if (B == 4) {
#pragma unroll
      for (int w = 0; w < D / 64; ++w) {
        const uint2 u2 = *reinterpret_cast<const uint2*>(blk + k0 + 8 * w), v2 = *reinterpret_cast<const uint2*>(blk + k1 + 8 * w);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t u = t < 2 ? u2.x : u2.y, v = t < 2 ? v2.x : v2.y;
          mma16816<false>(c, codes4(u, 2 * (t & 1)), codes4(v, 2 * (t & 1)), codes4(u, 2 * (t & 1) + 1), codes4(v, 2 * (t & 1) + 1), s.q[4 * w + t][0],
                          s.q[4 * w + t][1]);
        }
      }
    } else if (B == 8) {
#pragma unroll
      for (int w = 0; w < D / 64; ++w) {
        const uint4 u4 = *reinterpret_cast<const uint4*>(at(k0 + 16 * w)), v4 = *reinterpret_cast<const uint4*>(at(k1 + 16 * w));
        const uint32_t u[4] = {u4.x, u4.y, u4.z, u4.w}, v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
        for (int t = 0; t < 4; ++t)
          mma16816<false>(c, __byte_perm(u[t], 0x64646464u, 0x4140), __byte_perm(v[t], 0x64646464u, 0x4140), __byte_perm(u[t], 0x64646464u, 0x4342),
                          __byte_perm(v[t], 0x64646464u, 0x4342), s.q[4 * w + t][0], s.q[4 * w + t][1]);
      }
    } else {
#pragma unroll
      for (int w = 0; w < D / 32; ++w) {
        const uint4 u = *reinterpret_cast<const uint4*>(at(k0 + 16 * w)), v = *reinterpret_cast<const uint4*>(at(k1 + 16 * w));
        mma16816<true>(c, u.x, v.x, u.y, v.y, s.q[2 * w][0], s.q[2 * w][1]);
        mma16816<true>(c, u.z, v.z, u.w, v.w, s.q[2 * w + 1][0], s.q[2 * w + 1][1]);
      }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int key = b + 8 * r + quad;
      const bool seen = mask >> (8 * r + quad) & 1;
      float y[S::kHeads], grow = 0.f;
      if (B == 16) {
        if (NG == 1) { y[0] = c[2 * r]; y[S::kHeads - 1] = c[2 * r + 1]; }
        else y[0] = c[2 * r] + c[2 * r + 1];
      } else {
        uint32_t ks[2];
        scales(ksz, key, ks);
        scales(vsz, key, vs[r]);
        const __half2 k0s = as_half2(ks[0]), k1s = as_half2(ks[1]);
        const float y0 = __low2float(k0s) * (c[2 * r] - kOff * s.qsum[0]) + __high2float(k0s) * s.qsum[0];
        const float y1 = __low2float(k1s) * (c[2 * r + 1] - kOff * s.qsum[1]) + __high2float(k1s) * s.qsum[1];
        if (NG == 1) { y[0] = y0; y[S::kHeads - 1] = y1; }
        else y[0] = y0 + y1;
        uint32_t e = max(vs[r][0] & 0x7C00u, vs[r][1] & 0x7C00u);  // the larger scale's exponent
        if (NG == 4) e = max(e, __shfl_xor_sync(0xffffffffu, e, 1));
        grow = static_cast<float>(static_cast<int>(e >> 10) - 15);
      }
      if (NG == 4) y[0] += __shfl_xor_sync(0xffffffffu, y[0], 1);
#pragma unroll
      for (int h = 0; h < S::kHeads; ++h) {
        x[r][h] = seen ? y[h] * s.f[h] : -INFINITY;
        if (seen) top[h] = fmaxf(top[h], x[r][h] + grow);
      }
    }
  }
  bool far = top[0] > s.m[0] + 8.f;
  if (S::kHeads == 2) far |= top[S::kHeads - 1] > s.m[S::kHeads - 1] + 8.f;
  if (__any_sync(0xffffffffu, far)) {  // a new reference, the same for all lanes of a column
#pragma unroll
    for (int h = 0; h < S::kHeads; ++h) {
      float t = top[h];
      for (int o = 4; o < 32; o <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
      const float next = fmaxf(s.m[h], t), by = s.m[h] == -INFINITY ? 0.f : exp2_approx(s.m[h] - next);
      s.m[h] = next;
      s.l[h] *= by;
#pragma unroll
      for (int col = 0; col < 2; ++col)
        if (S::kHeads == 1 || col == h) {
          s.corr[col] *= by;
#pragma unroll
          for (int i = 0; i < S::kSteps; ++i) s.acc[i][col] *= by, s.acc[i][2 + col] *= by;
        }
    }
  }
  {
    uint32_t w[2][2];  // weights of token rows quad, quad + 8: binary16, or bf16 high and low parts
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const bool seen = mask >> (8 * r + quad) & 1;
      float p[S::kHeads];
#pragma unroll
      for (int h = 0; h < S::kHeads; ++h) {
        p[h] = seen ? exp2_approx(x[r][h] - s.m[h]) : 0.f;
        s.l[h] += p[h];
      }
      const float p0 = p[0], p1 = p[S::kHeads - 1];
      if (B == 16) {
        const __nv_bfloat162 hi = __floats2bfloat162_rn(p0, p1);
        const __nv_bfloat162 lo = __floats2bfloat162_rn(p0 - __low2float(hi), p1 - __high2float(hi));
        w[r][0] = *reinterpret_cast<const uint32_t*>(&hi);
        w[r][1] = *reinterpret_cast<const uint32_t*>(&lo);
      } else {
        const __half2 v0 = as_half2(vs[r][0]), v1 = as_half2(vs[r][1]);
        __half2 wv = __floats2half2_rn(p0 * __low2float(v0), p1 * __low2float(v1));
        if (!seen) wv = as_half2(0u);  // the scale of a slot that holds nothing may be anything
        w[r][0] = as_u32(wv);
        if (seen) {
          s.corr[0] += p0 * fmaf(Codes<B>::kMiddle, __low2float(v0), __high2float(v0));
          s.corr[1] += p1 * fmaf(Codes<B>::kMiddle, __low2float(v1), __high2float(v1));
        }
      }
    }
    const uint32_t b0 = transpose8(w[0][0]), b1 = transpose8(w[1][0]);
    uint32_t l0 = 0, l1 = 0;
    if (B == 16) l0 = transpose8(w[0][1]), l1 = transpose8(w[1][1]);
    // The sums run over all of a warp's tokens of a segment: they take in V's distance from the middle
    // of its range alone.  The offset, ten times and more the size of a value, would cost them their
    // last bits with every product (rows over 30,000 tokens of 8 bits came out 9 % off).
    if (B != 16) {
#pragma unroll
      for (int i = 0; i < S::kSteps; ++i) mma16816<false>(s.acc[i], Codes<B>::kMinus, Codes<B>::kMinus, Codes<B>::kMinus, Codes<B>::kMinus, b0, b1);
    }
    // tokens 2 part, 2 part + 1 (and 8 further on): an eighth of the dimensions, from quad * D / 8
    const int kp = b + 2 * part;
    const int v0 = (keys + kp) * kRow + quad * (kRow / 8);
    if (B == 2) {
      uint32_t lo, hi;  // pairs of tokens: 8 codes of each of two
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint8_t* p = blk + v0 + 2 * i;
        lo = *reinterpret_cast<const uint16_t*>(p) | static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(p + kRow)) << 16;
        hi = *reinterpret_cast<const uint16_t*>(p + 8 * kRow) | static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(p + 9 * kRow)) << 16;
#pragma unroll
        for (int t = 0; t < 4; ++t)
          mma16816<false>(s.acc[4 * i + t], codes2(lo, 2 * t), codes2(lo, 2 * t + 1), codes2(hi, 2 * t), codes2(hi, 2 * t + 1), b0, b1);
      }
    } else if (B == 4) {
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint8_t* p = blk + v0 + 4 * i;
        const uint32_t w0 = *reinterpret_cast<const uint32_t*>(p), w1 = *reinterpret_cast<const uint32_t*>(p + kRow);
        const uint32_t w8 = *reinterpret_cast<const uint32_t*>(p + 8 * kRow), w9 = *reinterpret_cast<const uint32_t*>(p + 9 * kRow);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint32_t lo = __byte_perm(w0, w1, u ? 0x7632 : 0x5410), hi = __byte_perm(w8, w9, u ? 0x7632 : 0x5410);
#pragma unroll
          for (int t = 0; t < 2; ++t)
            mma16816<false>(s.acc[4 * i + 2 * u + t], codes4(lo, 2 * t), codes4(lo, 2 * t + 1), codes4(hi, 2 * t), codes4(hi, 2 * t + 1), b0, b1);
        }
      }
    } else if (B == 8) {
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint2 w0 = *reinterpret_cast<const uint2*>(at(v0 + 8 * i)), w1 = *reinterpret_cast<const uint2*>(at(v0 + kRow + 8 * i));
        const uint2 w8 = *reinterpret_cast<const uint2*>(at(v0 + 8 * kRow + 8 * i)), w9 = *reinterpret_cast<const uint2*>(at(v0 + 9 * kRow + 8 * i));
#pragma unroll
        for (int u = 0; u < 4; ++u) {  // dimensions 2 u, 2 u + 1
          const uint32_t sel = u & 1 ? 0x7362 : 0x5140;
          const uint32_t lo = __byte_perm(u < 2 ? w0.x : w0.y, u < 2 ? w1.x : w1.y, sel), hi = __byte_perm(u < 2 ? w8.x : w8.y, u < 2 ? w9.x : w9.y, sel);
          mma16816<false>(s.acc[4 * i + u], __byte_perm(lo, 0x64646464u, 0x4140), __byte_perm(lo, 0x64646464u, 0x4342),
                          __byte_perm(hi, 0x64646464u, 0x4140), __byte_perm(hi, 0x64646464u, 0x4342), b0, b1);
        }
      }
    } else {
      // rows out of sight become zero: their weight of 0 times infinity would not be
      const uint32_t seen = mask >> (2 * part);
      const uint32_t ma = (seen & 1 ? 0x0000FFFFu : 0u) | (seen & 2 ? 0xFFFF0000u : 0u);
      const uint32_t mb = (seen & 0x100 ? 0x0000FFFFu : 0u) | (seen & 0x200 ? 0xFFFF0000u : 0u);
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint4 q0 = *reinterpret_cast<const uint4*>(at(v0 + 16 * i)), q1 = *reinterpret_cast<const uint4*>(at(v0 + kRow + 16 * i));
        const uint4 q8 = *reinterpret_cast<const uint4*>(at(v0 + 8 * kRow + 16 * i)), q9 = *reinterpret_cast<const uint4*>(at(v0 + 9 * kRow + 16 * i));
        const uint32_t a0[4] = {q0.x, q0.y, q0.z, q0.w}, a1[4] = {q1.x, q1.y, q1.z, q1.w}, a8[4] = {q8.x, q8.y, q8.z, q8.w},
                       a9[4] = {q9.x, q9.y, q9.z, q9.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t e0 = __byte_perm(a0[u], a1[u], 0x5410) & ma, e1 = __byte_perm(a0[u], a1[u], 0x7632) & ma;
          const uint32_t e2 = __byte_perm(a8[u], a9[u], 0x5410) & mb, e3 = __byte_perm(a8[u], a9[u], 0x7632) & mb;
          mma16816<true>(s.acc[4 * i + u], e0, e1, e2, e3, b0, b1);
          mma16816<true>(s.acc[4 * i + u], e0, e1, e2, e3, l0, l1);
        }
      }
    }
  }
}

template <int D, int NG, int B>
__device__ __forceinline__ void few_class(FewState<D, NG>& s, const uint8_t* smem, const FewBlock& b, uint32_t mask, bool swz, int lane) {
  if (s.q_class != B) few_load_q<D, NG, B>(s, smem, b.rows, lane);
  const uint8_t* blk = smem + FewSmem<D, NG>::kRing + b.off;
  const int keys = b.keys;
  // one copy of the code for both halves of a block: the warps' instructions have to fit the cache together
#pragma unroll 1
  for (int k = 0; k < keys; k += 16)
    if (mask >> k & 0xFFFFu) few_tokens<D, NG, B>(s, blk, keys, k, mask >> k & 0xFFFFu, swz, lane);
}

// A segment's piece begins: its query rows, each with the power of two that brings its largest
// element to [1, 2), and an empty state.
template <int D, int NG>
__device__ __forceinline__ void few_begin(FewState<D, NG>& s, const GroupArgs& g, uint8_t* smem, const FewBlock& b, int lane) {
  const int rows = b.rows;
  int* ids = reinterpret_cast<int*>(smem + FewSmem<D, NG>::kRowIds);
  __syncwarp();
  if (lane < rows) {
    const int heads = g.a.Hq / g.a.Hkv;
    const int query = b.kind == 1 ? b.qbase : g.list[b.qbase + lane / heads];
    ids[lane] = query * g.a.Hq + b.kvh * heads + (b.kind == 1 ? lane : lane % heads);
  }
  float* factor = reinterpret_cast<float*>(smem + FewSmem<D, NG>::kFactor);
  float* sums = factor + kFewRows;  // [row][group] of the binary16 elements
  __syncwarp();
  constexpr int kLanes = D / 8, kGroupLanes = kLanes / NG;  // lanes of a row, of a group
  for (int i = lane; i < (rows * kLanes + 31) / 32 * 32; i += 32) {
    const bool live = i < rows * kLanes;
    uint4 u = make_uint4(0, 0, 0, 0);
    if (live) u = reinterpret_cast<const uint4*>(g.q + static_cast<int64_t>(ids[i / kLanes]) * D)[i % kLanes];
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = max(top, max(w[k] & 0x7FFFu, (w[k] >> 16) & 0x7FFFu));
    for (int o = 1; o < kLanes; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    int e = top == 0 || top >= 0x7F80u ? 0 : static_cast<int>(top >> 7) - 127;
    e = max(-100, min(120, e));
    const float down = __int_as_float((127 - e) << 23);
    uint32_t h[4], b16[4];
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float lo = bf16lo(w[k]) * down, hi = bf16hi(w[k]) * down;
      const __half2 x = __floats2half2_rn(lo, hi);
      const __nv_bfloat162 y = __floats2bfloat162_rn(lo, hi);
      h[k] = as_u32(x);
      b16[k] = *reinterpret_cast<const uint32_t*>(&y);
      sum += __low2float(x) + __high2float(x);
    }
    for (int o = 1; o < kGroupLanes; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (live) {
      reinterpret_cast<uint4*>(smem)[i] = make_uint4(h[0], h[1], h[2], h[3]);
      reinterpret_cast<uint4*>(smem + FewSmem<D, NG>::kQ)[i] = make_uint4(b16[0], b16[1], b16[2], b16[3]);
      if (i % kLanes == 0) factor[i / kLanes] = fmaxf(g.scale_log2 * __int_as_float((127 + e) << 23), 1.17549435e-38f);
      if (i % kGroupLanes == 0) sums[i / kGroupLanes] = sum;
    }
  }
  __syncwarp();
#pragma unroll
  for (int col = 0; col < 2; ++col) {
    const int n = 2 * (lane & 3) + col;
    s.qsum[col] = n / NG < rows ? sums[n] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) s.acc[i][k] = 0.f;
#pragma unroll
  for (int h = 0; h < FewState<D, NG>::kHeads; ++h) {
    const int head = NG == 1 ? 2 * (lane & 3) + h : 2 * (lane & 3) / NG;
    s.m[h] = -INFINITY;
    s.l[h] = 0.f;
    s.f[h] = head < rows ? factor[head] : 1.f;
  }
  s.corr[0] = s.corr[1] = 0.f;
  s.q_class = 0;
}

// It ends: the row, or its part.
template <int D, int NG>
__device__ __forceinline__ void few_end(FewState<D, NG>& s, const GroupArgs& g, const uint8_t* smem, const FewBlock& b, int lane) {
  using S = FewState<D, NG>;
  constexpr int kRun = D / 8;
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) {
#pragma unroll
    for (int h = 0; h < S::kHeads; ++h) s.l[h] += __shfl_xor_sync(0xffffffffu, s.l[h], o);
    s.corr[0] += __shfl_xor_sync(0xffffffffu, s.corr[0], o);
    s.corr[1] += __shfl_xor_sync(0xffffffffu, s.corr[1], o);
  }
  const int quad = lane >> 2, part = lane & 3, group = quad * NG / 8;  // the group of the lane's dimensions
#pragma unroll
  for (int col = 0; col < 2; ++col) {
    const int n = 2 * part + col, r = n / NG, h = NG == 1 ? col : 0;
    if (r >= b.rows || n % NG != group) continue;
    const int id = reinterpret_cast<const int*>(smem + FewSmem<D, NG>::kRowIds)[r];
    const int64_t home = static_cast<int64_t>(b.kind) * g.n * g.a.Hq + id;
    float v[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) v[i] = s.acc[i / 2][i % 2 * 2 + col] + s.corr[col];
    if (b.dest == -2) {
      const float inv = s.l[h] != 0.f ? 1.f / s.l[h] : 0.f;
      uint16_t* out = g.out + static_cast<int64_t>(id) * D + quad * kRun;
#pragma unroll
      for (int i = 0; i < kRun; i += 8) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const __nv_bfloat162 x = __floats2bfloat162_rn(v[i + 2 * k] * inv, v[i + 2 * k + 1] * inv);
          w[k] = *reinterpret_cast<const uint32_t*>(&x);
        }
        *reinterpret_cast<uint4*>(out + i) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else {
      const int64_t row = static_cast<int64_t>(b.dest) * kFewRows + r;
      float* to = (b.dest >= 0 ? g.few_o + row * D : g.home_o + home * D) + quad * kRun;
      if (quad == 0) (b.dest >= 0 ? g.few_ml[row] : g.home_ml[home]) = make_float2(s.m[h], s.l[h]);
#pragma unroll
      for (int i = 0; i < kRun; i += 8) st_global8(to + i, v + i);
    }
  }
}

template <int D, int NG>
__global__ void __launch_bounds__(32 * kFewWarps, kFewCtas) group_few_kernel(const __grid_constant__ GroupArgs g) {
  extern __shared__ __align__(128) uint8_t dyn[];
  using L = FewSmem<D, NG>;
  const LayerArgs& a = g.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* smem = dyn + warp * L::kWarp;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kBars);
  FewBlock* blocks = reinterpret_cast<FewBlock*>(smem + L::kBlocks);
  if (lane == 0) {
    for (int i = 0; i < kFewStages; ++i) mbar_init(bars + i, 1);
    fence_barrier_init();
  }
  __syncwarp();
  // After the tensor kernel this one starts beside it, to fill the SMs that run out of tiles: it reads
  // nothing that kernel writes, and waits for it at its end instead.  The tensor kernel's CTAs let it
  // start only after their own wait for the plan, so the plan has ended; but that orders nothing for
  // this kernel's memory.  So each thread's first load acquires the plan's last store, which released
  // the whole plan and, through the plan's own wait, what the kernels before it wrote: page tables,
  // pages, query rows.  Loads and copies behind it find all of that.
  if (!g.overlap) pdl_wait();
  pdl_trigger();
  const int64_t per = ld_acquire(&g.head->few_per);
  fence_proxy_async_global();
  FewCursor& cur = *reinterpret_cast<FewCursor*>(smem + L::kCursor);
  Job& job = *reinterpret_cast<Job*>(smem + L::kJob);
  const int me = blockIdx.x * kFewWarps + warp, P = a.P, jobs = g.groups + g.n;
  const int lg_p = __ffs(P) - 1, lg_q = max(0, lg_p - 5), lg_w = lg_p - 4;  // log2 of the blocks of a page: 32 tokens, 16 of 16 bits
  int tile = 0, tile1 = 0, batch = -1;       // the segment's next block, its end for this warp; batch of 32 blocks that the lanes hold
  // the lane's block of the batch: its K codes in KV head 0, and class | all in sight << 2 |
  // tokens << 3 | 16 slots instead of 32 << 9 | bytes / 16 << 10
  const uint8_t* mine = nullptr;
  uint32_t info = 0;
  {
    const int64_t work = g.head->few_work, b0 = min(work, me * per), b1 = min(work, b0 + per);
    if (b0 >= b1) {
      if (g.overlap) pdl_wait();
      return;
    }
    int lo = 0, hi = jobs;  // the job that holds cost b0: the last one that starts at or before it
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, i = lo + lane * step;
      const int k = __popc(__ballot_sync(0xffffffffu, i < hi && g.few_base[i] <= b0));
      const int last = lo + (k - 1) * step;
      hi = min(hi, last + step);
      lo = last;
      if (step == 1) break;
    }
    if (lane == 0) cur.b0 = b0, cur.b1 = b1, cur.j = lo;
    __syncwarp();
  }

  // The copies' cursor.  Every lane reads and works out the same; lane 0 writes.
  auto open_segment = [&](int seg) -> bool {  // the job's first segment from `seg` on with blocks for this warp
    const int64_t b0 = cur.b0, b1 = cur.b1, base = cur.base;
    const int tiles = cur.tiles;
    for (; seg < a.Hkv; ++seg) {
      const int64_t S = base + seg * few_cost(tiles);
      if (S >= b1) return false;
      const int t0 = few_before(b0 - S, tiles), t1 = few_before(b1 - S, tiles);
      if (t0 < t1) {
        tile = t0;
        tile1 = t1;
        __syncwarp();
        if (lane == 0) cur.seg = seg, cur.tile0 = t0;
        __syncwarp();
        return true;
      }
    }
    return false;
  };
  auto open_job = [&](int j) -> bool {        // the first job from `j` on with blocks for this warp
    for (; j < jobs; ++j) {
      const int64_t base = g.few_base[j];  // (all loads of a job before the first branch on one)
      const int tiles = g.blocks[j], word = reinterpret_cast<const int*>(g.jobs + j)[lane];
      if (base >= cur.b1) return false;
      if (tiles == 0) continue;
      __syncwarp();
      reinterpret_cast<int*>(&job)[lane] = word;
      __syncwarp();
      if (lane == 0) {
        int q = 0;
        for (int c = 0; c < 3; ++c) q += job.head[c] + job.count[c];
        cur.pages_q = q;
        cur.tiles = tiles;
        cur.base = base;
        cur.j = j;
      }
      __syncwarp();
      batch = -1;
      if (open_segment(static_cast<int>(max(static_cast<int64_t>(0), (cur.b0 - base) / few_cost(tiles))))) return true;
    }
    return false;
  };
  bool more = open_job(cur.j);

  auto load_batch = [&]() {
    batch = tile >> 5;
    const int i = (batch << 5) + lane;
    if (i < cur.tiles) {
      const int nq = cur.pages_q << lg_q;
      const bool wide = i >= nq;
      const int lg = wide ? lg_w : lg_q, n = wide ? i - nq : i, sub = n & ((1 << lg) - 1);
      int in = n >> lg, c = wide ? 3 : 0;
      if (!wide) {
#pragma unroll 1
        for (; c < 2; ++c) {
          const int m = job.head[c] + job.count[c];
          if (in < m) break;
          in -= m;
        }
      }
      const int h = job.head[c], k = in < h ? in : job.first[c] + in - h;
      const int64_t at = (static_cast<int64_t>(job.seq) * kClasses + c) * a.MP + k;
      const int page = a.pt[at], pf = a.pfirst[at], pl = a.plast[at], valid = min(P, job.tokens[c] - k * P);
      const bool whole = valid == P && pl <= job.t && (pf >= job.lo || pl < job.sinks);
      // no more slots than hold a token, or, of a page that ends before the window, than can be sinks
      // (slot x of page k holds position k P + x or a later one)
      const int slot0 = sub << (wide ? 4 : 5), fill = max(0, valid - slot0);
      const int most = pl < job.lo ? min(fill, max(1, job.sinks - k * P - slot0)) : fill;
      const int keys = min(P, wide || most <= 16 ? 16 : 32), row = (D / 8) << (c + 1), block = min(P, wide ? 16 : 32);
      const int bytes = 2 * keys * (row + (wide ? 0 : NG * 4));
      mine = a.pool[c] + page * a.page_bytes[c] + a.hdr + sub * block * row;
      info = c | (whole ? 4 : 0) | min(keys, fill) << 3 | (keys == 16 ? 1 << 9 : 0) | bytes / 16 << 10;
    }
    __syncwarp();
  };

  int issued = 0, taken = 0;                 // blocks brought, blocks used
  int ring_head = 0, low = 0;                // where the next one goes; the ring is filled up when no more than `low` are left
  // Brings as many of the segment's next blocks as the batch holds and the ring has room for, one per lane.
  auto bring = [&]() {
    if (tile >> 5 != batch) load_batch();
    const int l0 = tile & 31, want = min(min(32 - l0, tile1 - tile), kFewStages - (issued - taken));
    const int r = lane - l0;
    const bool cand = r >= 0 && r < want;
    const bool all_in = info & 4;
    const int bytes = (info >> 10) * 16, body = (bytes + 127) & ~127, need = cand ? body + (all_in ? 0 : 128) : 0;
    int upto = need;
#pragma unroll
    for (int o = 1; o < kFewStages; o <<= 1) {  // lanes outside the candidates add nothing
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    int start = ring_head, space = L::kRingBytes;
    if (issued == taken) {
      start = 0;
    } else {
      const int tail = blocks[taken % kFewStages].off;
      if (ring_head <= tail) {
        space = tail - ring_head - 1;
      } else {
        space = L::kRingBytes - ring_head;
        if (__shfl_sync(0xffffffffu, need, l0) > space) start = 0, space = tail - 1;
      }
    }
    const int k = __popc(__ballot_sync(0xffffffffu, cand && upto <= space));
    if (k == 0) return;
    const int seg = cur.seg, tile0 = cur.tile0, tiles = cur.tiles;
    if (cand && r < k) {
      const int slot = (issued + r) % kFewStages, c = info & 3, keys = info & 512 ? 16 : 32, off = start + upto - need;
      FewBlock& b = blocks[slot];
      b.cls = c; b.keys = keys; b.off = off; b.pos = all_in ? -1 : off + body;
      b.valid = info >> 3 & 63; b.lo = job.lo; b.t = job.t; b.sinks = job.sinks;
      b.kind = job.kind; b.qbase = job.qbase; b.kvh = seg; b.rows = job.rows; b.state = (tile + r == tile0 ? 1 : 0) | (tile + r == tile1 - 1 ? 2 : 0);
      b.dest = tile1 - tile0 < tiles ? 2 * me + (tile0 > 0 ? 0 : 1) : job.joined ? -1 : -2;
      mbar_arrive_expect_tx(bars + slot, bytes + (all_in ? 0 : 4 * keys));
      const uint8_t* src = mine + static_cast<int64_t>(seg) * a.slice[c];
      uint8_t* to = smem + L::kRing + off;
      const int row = (D / 8) << (c + 1);  // `sub`: the block's first slot in its page
      const int sub = ((tile + r - (c == 3 ? cur.pages_q << lg_q : 0)) & ((1 << (c == 3 ? lg_w : lg_q)) - 1)) * min(P, c == 3 ? 16 : 32);
      if (keys == P) {  // the block is the whole slice
        bulk_g2s(to, src, bytes, bars + slot);
      } else {          // K codes, V codes, K scales, V scales
        const uint8_t* sz = src - sub * row + 2 * P * row + sub * NG * 4;
        bulk_g2s(to, src, keys * row, bars + slot);
        bulk_g2s(to + keys * row, src + P * row, keys * row, bars + slot);
        if (c < 3) {
          bulk_g2s(to + 2 * keys * row, sz, keys * NG * 4, bars + slot);
          bulk_g2s(to + keys * (2 * row + NG * 4), sz + P * NG * 4, keys * NG * 4, bars + slot);
        }
      }
      if (!all_in) bulk_g2s(to + body, mine - sub * row - a.hdr + 4 * sub, 4 * keys, bars + slot);
    }
    __syncwarp();
    ring_head = start + __shfl_sync(0xffffffffu, upto, l0 + k - 1);
    issued += k;
    tile += k;
    low = (issued - taken) / 2;
    if (tile == tile1 && !open_segment(seg + 1)) more = open_job(cur.j + 1);  // on to the next segment, or job
  };

  FewState<D, NG> s;
  bool late = false;
  while (more || taken < issued) {
    if (more && issued - taken <= low) bring();
    if (issued == taken) continue;  // the segment's end left the ring empty
    const int slot = taken % kFewStages;
    late = !__all_sync(0xffffffffu, mbar_wait(bars + slot, (taken / kFewStages) & 1, a.wait_ns));
    if (late) break;
    const FewBlock& b = blocks[slot];
    if (b.state & 1) few_begin<D, NG>(s, g, smem, b, lane);
    bool seen = lane < b.keys;
    if (b.pos >= 0 && seen) {
      const int pos = reinterpret_cast<const int32_t*>(smem + L::kRing + b.pos)[lane];
      seen = lane < b.valid && pos <= b.t && (pos >= b.lo || pos < b.sinks);
    }
    const uint32_t mask = __ballot_sync(0xffffffffu, seen);
    if (mask) {
      if (b.cls == 0) few_class<D, NG, 2>(s, smem, b, mask, a.swz, lane);
      else if (b.cls == 1) few_class<D, NG, 4>(s, smem, b, mask, a.swz, lane);
      else if (b.cls == 2) few_class<D, NG, 8>(s, smem, b, mask, a.swz, lane);
      else few_class<D, NG, 16>(s, smem, b, mask, a.swz, lane);
    }
    if (b.state & 2) few_end<D, NG>(s, g, smem, b, lane);
    __syncwarp();
    ++taken;
  }
  if (late) {  // the warp stays until its copies have landed
    for (int k = taken; k < issued; ++k) mbar_wait(bars + k % kFewStages, (k / kFewStages) & 1);
    if (lane == 0) set_status(a.ctrl, TRR_ERR_TIMEOUT);
  }
  if (g.overlap) pdl_wait();  // so that its end is the tensor kernel's, too
}

}  // namespace trr
