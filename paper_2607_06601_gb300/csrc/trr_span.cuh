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

constexpr int kSpan = 64;            // positions that a CTA takes at a time
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

// Tokens that a CTA has found, class by class, in order; class kClasses: positions that store nothing.
struct Found {
  struct Token {
    const uint8_t* page;
    int slot, row;  // row: where its values go
  };
  Token token[kClasses + 1][kSpan];
  int count[kClasses + 1];
  int warp_count[kSpanThreads / 32][kClasses + 1];

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
    if (tid <= kClasses) {
      int n = 0;
      for (int w = 0; w < kSpanThreads / 32; ++w) n += warp_count[w][tid];
      count[tid] = n;
    }
    __syncthreads();
  }
  // Groups of `rows` tokens of one class: how many, and the class, first token and number of tokens of one.
  __device__ __forceinline__ int groups(int rows) const {
    int n = 0;
    for (int c = 0; c <= kClasses; ++c) n += (count[c] + rows - 1) / rows;
    return n;
  }
  __device__ __forceinline__ int group(int i, int rows, int* first, int* n) const {
    int c = 0;
    for (; c < kClasses; ++c) {
      const int k = (count[c] + rows - 1) / rows;
      if (i < k) break;
      i -= k;
    }
    *first = i * rows;
    *n = count[c];
    return c;
  }
};

// Sixteen consecutive elements of a row, as they are stored.
struct Codes16 {
  uint4 w[2];   // 2, 4 and 8 bits: the codes in the first 4, 8 or 16 bytes; 16 bits: the values
  uint32_t sz;  // scale and zero (binary16) of their group
};

// Elements 16 e .. 16 e + 15 of K (which 0) or V (1) of KV head h.
template <int D>
__device__ __forceinline__ Codes16 load_codes16(const LayerArgs& a, int c, const uint8_t* page, int slot, int h, int which, int e, int lg_group) {
  const uint8_t* slice = page + a.hdr + static_cast<int64_t>(h) * a.slice[c];
  const int lg = c + 1, row = D << lg >> 3, o = (which * a.P + slot) * row + (e << (lg + 1));
  Codes16 r = {};
  if (c == 3) {
    r.w[0] = *reinterpret_cast<const uint4*>(slice + (a.swz ? swz_off(o) : o));
    r.w[1] = *reinterpret_cast<const uint4*>(slice + (a.swz ? swz_off(o + 16) : o + 16));
    return r;
  }
  if (c == 2) {
    r.w[0] = *reinterpret_cast<const uint4*>(slice + (a.swz ? swz_off(o) : o));
  } else if (c == 1) {
    const uint2 x = *reinterpret_cast<const uint2*>(slice + o);
    r.w[0].x = x.x;
    r.w[0].y = x.y;
  } else {
    r.w[0].x = *reinterpret_cast<const uint32_t*>(slice + o);
  }
  r.sz = reinterpret_cast<const uint32_t*>(slice + 2 * a.P * row)[(which * a.P + slot) * (D >> lg_group) + (16 * e >> lg_group)];
  return r;
}

// 32 bytes in one store (p aligned to them).
__device__ __forceinline__ void store_sector(void* p, uint4 a, uint4 b) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z),
               "r"(b.w)
               : "memory");
}

}  // namespace trr
