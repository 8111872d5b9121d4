// trr_span.cuh - stretches of positions of sequences: which tokens are stored there, in which pages,
// and their rows brought back from codes.  trr_kv_read and trr_chunk_attn are built on it.
//
// A call names its stretches by seq_ids[n], starts[n] and offsets[n + 1]: rows offsets[i] ..
// offsets[i+1]-1 are positions starts[i], starts[i] + 1, ... of sequence seq_ids[i].
//
// A CTA takes 64 positions at a time.  Four threads share a position, one for each width class: each
// counts, by two binary searches (the first positions of the class's pages, then the slots of one
// page), how many tokens of its class lie before the position, and whether one lies at it.  The four
// counts also are the position's rank among the stored tokens, so that rows of all classes can be laid
// down in order of position without a sort.  The searches are a chain of about log2(pages) +
// log2(P) loads, most of them the same for all positions; several CTAs per SM hide them.
#pragma once

#include "trr_group.cuh"

namespace trr {

constexpr int kSpan = 64;            // positions that a CTA takes at a time (reading back: at most)
constexpr int kSpanThreads = 4 * kSpan;
constexpr int kMostSpans = 4096;     // stretches of a call

// Tokens of class c of sequence seq that lie before position p; whether one lies at p, and where.
struct Place {
  int before;
  int page, slot;  // of the token at p; page < 0: none
};
__device__ __forceinline__ Place place_of(const LayerArgs& a, int seq, int c, int p) {
  const int64_t row = static_cast<int64_t>(seq) * kClasses + c;
  const int nt = a.ntok[row];
  const int32_t* first = a.pfirst + row * a.MP;
  int lo = 0, hi = (nt + a.P - 1) / a.P;
  while (lo < hi) {  // pages whose first token is at p or before
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= p) lo = mid + 1;
    else hi = mid;
  }
  if (lo == 0) return Place{0, -1, 0};
  const int k = lo - 1, page = a.pt[row * a.MP + k], n = min(a.P, nt - k * a.P);
  const int32_t* pos = reinterpret_cast<const int32_t*>(a.pool[c] + page * a.page_bytes[c]);
  int l = 0, h = n;
  while (l < h) {
    const int mid = (l + h) >> 1;
    if (pos[mid] < p) l = mid + 1;
    else h = mid;
  }
  return Place{k * a.P + l, l < n && pos[l] == p ? page : -1, l};
}

// The same count by a whole warp, 32 probes at a time: for a position that others wait for.
__device__ __forceinline__ int tokens_before(const LayerArgs& a, int seq, int c, int p, int lane) {
  const int64_t row = static_cast<int64_t>(seq) * kClasses + c;
  const int nt = a.ntok[row];
  const int32_t* first = a.pfirst + row * a.MP;
  int lo = 0, hi = (nt + a.P - 1) / a.P;
  while (lo < hi) {  // pages whose first token is before p
    const int step = (hi - lo + 31) / 32, i = lo + lane * step;
    const int k = __popc(__ballot_sync(0xffffffffu, i < hi && first[i] < p));
    if (k == 0) break;
    const int last = lo + (k - 1) * step;
    hi = min(hi, last + step);
    lo = last + 1;
  }
  if (lo == 0) return 0;
  const int k = lo - 1, n = min(a.P, nt - k * a.P);
  const int32_t* pos = reinterpret_cast<const int32_t*>(a.pool[c] + a.pt[row * a.MP + k] * a.page_bytes[c]);
  int below = 0;
  for (int s = 0; s < n; s += 32) below += __popc(__ballot_sync(0xffffffffu, s + lane < n && pos[s + lane] < p));
  return k * a.P + below;
}

// Tokens that a CTA has found, class by class, in order; class kClasses: positions that store nothing.  ROWS of a
// class's, at most, form a group, which a warp takes together.
template <int ROWS>
struct Found {
  struct Token {
    const uint8_t* page;
    int slot, row;  // row: where its values go
  };
  static constexpr int kMostGroups = kSpan / ROWS + kClasses + 1;
  Token token[kClasses + 1][kSpan];
  int warp_count[kSpanThreads / 32][kClasses + 1];
  int count[kClasses + 1], groups;
  int16_t group_class[kMostGroups], group_first[kMostGroups];

  // Thread 4 i + c brings class c's place of position i and the row that its values go to (row < 0: the position is
  // not asked for).  Every thread of the CTA calls it; what was found before has then been read by all.
  __device__ __forceinline__ void gather(const LayerArgs& a, const Place& p, int c, int row, int tid) {
    const int lane = tid & 31, warp = tid >> 5;
    const uint32_t here = __ballot_sync(0xffffffffu, p.page >= 0), mine = 0x11111111u << c;
    const uint32_t any = (here | here >> 1 | here >> 2 | here >> 3) & 0x11111111u;  // positions that store a token
    const uint32_t none = __ballot_sync(0xffffffffu, row >= 0) & ~any & 0x11111111u;
    __syncthreads();
    if (lane < 4) warp_count[warp][lane] = __popc(here & 0x11111111u << lane);
    if (lane == 4) warp_count[warp][kClasses] = __popc(none);
    __syncthreads();
    auto before = [&](int k) {
      int n = 0;
      for (int w = 0; w < warp; ++w) n += warp_count[w][k];
      return n;
    };
    const uint32_t below = (1u << lane) - 1;
    if (p.page >= 0) token[c][before(c) + __popc(here & mine & below)] = Token{a.pool[c] + p.page * a.page_bytes[c], p.slot, row};
    if (none >> lane & 1) token[kClasses][before(kClasses) + __popc(none & below)] = Token{nullptr, 0, row};
    if (warp == 0) {
      int n = 0;
      if (lane <= kClasses)
        for (int w = 0; w < kSpanThreads / 32; ++w) n += warp_count[w][lane];
      int mine_groups = (n + ROWS - 1) / ROWS, first = mine_groups;
      for (int o = 1; o < 8; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, first, o);
        if (lane >= o) first += y;
      }
      first -= mine_groups;
      if (lane <= kClasses) {
        count[lane] = n;
        for (int k = 0; k < mine_groups; ++k) group_class[first + k] = lane, group_first[first + k] = k * ROWS;
        if (lane == kClasses) groups = first + mine_groups;
      }
    }
    __syncthreads();
  }
};

// Sixteen consecutive elements of a row, as they are stored.
struct Codes16 {
  uint4 w[2];   // 2, 4 and 8 bits: the codes in the first 4, 8 or 16 bytes; 16 bits: the values
  uint32_t sz;  // scale and zero (binary16) of their group
};

// Where elements 16 e .. 16 e + 15 of a token's K and V lie in its slices, the same in every KV head's.
template <int C, int D>
struct CodesAt {
  static constexpr int kRow = (D << (C + 1)) >> 3;  // bytes of a row
  int code[2][2], sz[2];                            // [K, V], of 16 bits [first, second half]
  __device__ __forceinline__ CodesAt(const LayerArgs& a, int slot, int e) {
    const int lg_group = __ffs(a.G) - 1;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const int o = (which * a.P + slot) * kRow + (e << (C + 2));
      code[which][0] = C >= 2 && a.swz ? static_cast<int>(swz_off(o)) : o;
      code[which][1] = C == 3 ? (a.swz ? static_cast<int>(swz_off(o + 16)) : o + 16) : 0;
      sz[which] = 2 * a.P * kRow + ((which * a.P + slot) * (D >> lg_group) + (16 * e >> lg_group)) * 4;
    }
  }
  __device__ __forceinline__ Codes16 load(const uint8_t* slice, int which) const {
    Codes16 r;
    const uint8_t* p = slice + code[which][0];
    if (C == 3) {
      r.w[0] = *reinterpret_cast<const uint4*>(p);
      r.w[1] = *reinterpret_cast<const uint4*>(slice + code[which][1]);
      return r;
    }
    if (C == 2) {
      r.w[0] = *reinterpret_cast<const uint4*>(p);
    } else if (C == 1) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      r.w[0].x = x.x;
      r.w[0].y = x.y;
    } else {
      r.w[0].x = *reinterpret_cast<const uint32_t*>(p);
    }
    r.sz = *reinterpret_cast<const uint32_t*>(slice + sz[which]);
    return r;
  }
};

// (a, b) x (f, f) and (a, b) x (f, f) + (z, z).
__device__ __forceinline__ void scale_pair(float& a, float& b, float f) {
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %2};\n mul.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}" : "+f"(a), "+f"(b) : "f"(f));
}
__device__ __forceinline__ void affine_pair(float& a, float& b, float f, float z) {
  asm("{\n .reg .b64 x, y, w;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %2};\n mov.b64 w, {%3, %3};\n fma.rn.f32x2 x, x, y, w;\n mov.b64 {%0, %1}, x;\n}"
      : "+f"(a), "+f"(b)
      : "f"(f), "f"(z));
}

// z + c s of sixteen elements of class C (kClasses: zeros), in binary32.  A code stays where it is in its word, which
// is read as a binary32 subnormal, c 2^(p - 149) at bit p: with s 2^(100 - p) and z 2^-49 the sum has the roundings of
// z + c s (nothing is subnormal: s and z are binary16), 2^-49 times.
template <int C>
__device__ __forceinline__ void expand_f32(const Codes16& x, float (&v)[16]) {
  if constexpr (C == kClasses) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = 0.f;
  } else if constexpr (C == 3) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t w[4] = {x.w[k].x, x.w[k].y, x.w[k].z, x.w[k].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) v[8 * k + 2 * i] = bf16lo(w[i]), v[8 * k + 2 * i + 1] = bf16hi(w[i]);
    }
  } else {
    constexpr int B = 2 << C, kWords = B / 2, kHalf = 16 / B;  // elements in half a word
    const uint32_t w[4] = {x.w[0].x, x.w[0].y, x.w[0].z, x.w[0].w};
    const float s = __low2float(as_half2(x.sz)), z = __high2float(as_half2(x.sz)) * 0x1p-49f;
#pragma unroll
    for (int i = 0; i < kHalf; ++i) {
      const uint32_t mask = ((1u << B) - 1) << (B * i);
      const float f = s * __int_as_float((127 + 100 - B * i) << 23);
#pragma unroll
      for (int k = 0; k < kWords; ++k) {
        float& a = v[2 * kHalf * k + i];
        float& b = v[2 * kHalf * k + kHalf + i];
        a = __uint_as_float(w[k] & mask);
        b = __uint_as_float((w[k] >> 16) & mask);
        affine_pair(a, b, f, z);
        scale_pair(a, b, 0x1p49f);
      }
    }
  }
}

// A CTA's groups, shared out with `parts` shares of the heads (a power of two) among its warps: body(class, token,
// whether the lane has one, first head, step).
template <int ROWS, typename Body>
__device__ __forceinline__ void for_groups(const Found<ROWS>& f, int lg_parts, int h0, Body body) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int x = warp; x < f.groups << lg_parts; x += kSpanThreads / 32) {
    const int g = x >> lg_parts, c = f.group_class[g], t = f.group_first[g] + lane / (32 / ROWS);
    const bool live = t < f.count[c];
    body(c, f.token[c][live ? t : 0], live, h0 + (x & ((1 << lg_parts) - 1)), 1 << lg_parts);
  }
}

// Parts that a group's heads are shared out in: enough that eight warps come out nearly even, two heads each at least.
__host__ __device__ inline int lg_parts(int heads) { return heads >= 8 ? 2 : heads >= 4 ? 1 : 0; }

// Shares of the heads that a unit (64 positions) is cut into: as many as make the rounds of `ctas` CTAs shortest, where
// a unit whole takes `whole` ns among as many others, and each share 5 us more to find its tokens.  For staging: reading
// back took this rule over with units of fewer positions besides (there, with what both measured), which were no gain for
// staging, as the longer plan took what they gave.
__device__ __forceinline__ int shares_of_heads(int64_t units, int most, int ctas, int64_t whole) {
  int best = 1;
  float least = 0.f;
#pragma unroll 1
  for (int s = 1; s <= most; ++s) {  // (a choice only: no more than binary32)
    const float t = ceilf(static_cast<float>(units) * s / ctas) * (static_cast<float>(whole) / s + 5000.f);
    if (s == 1 || t < least) best = s, least = t;
  }
  return best;
}
// The time that 64 positions of `bytes` each take when every CTA copies as much, at 6.5 bytes a ps.
__host__ __device__ inline int64_t copy_ns(int64_t bytes, int ctas) { return bytes * kSpan * ctas / 6500; }

// 32 bytes in one store (p aligned to them).
__device__ __forceinline__ void store_sector(void* p, uint4 a, uint4 b) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z),
               "r"(b.w)
               : "memory");
}

}  // namespace trr
