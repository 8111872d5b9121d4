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

// Tokens that a CTA has found, class by class; class kClasses: positions that store nothing.
struct Found {
  struct Token {
    const uint8_t* page;
    int slot, row;  // row: where its values go
  };
  Token token[kClasses + 1][kSpan];
  int count[kClasses + 1];
};

// Eight consecutive elements of a row, as they are stored.
struct Codes {
  uint4 w;      // 2, 4 and 8 bits: the codes in w.x (and w.y); 16 bits: the values
  uint32_t sz;  // scale and zero (binary16) of their group
};

// Elements 8 e .. 8 e + 7 of K (which 0) or V (1) of KV head h.
template <int B, int D>
__device__ __forceinline__ Codes load_codes(const LayerArgs& a, const uint8_t* page, int slot, int h, int which, int e, int lg_group) {
  constexpr int c = B == 2 ? 0 : B == 4 ? 1 : B == 8 ? 2 : 3, kRow = D * B / 8;
  const uint8_t* slice = page + a.hdr + static_cast<int64_t>(h) * a.slice[c];
  int o = (which * a.P + slot) * kRow + e * B;
  if (B >= 8 && a.swz) o = static_cast<int>(swz_off(o));
  Codes r;
  r.w = make_uint4(0, 0, 0, 0);
  r.sz = 0;
  if (B == 16) {
    r.w = *reinterpret_cast<const uint4*>(slice + o);
    return r;
  }
  if (B == 8) {
    const uint2 x = *reinterpret_cast<const uint2*>(slice + o);
    r.w.x = x.x;
    r.w.y = x.y;
  } else if (B == 4) {
    r.w.x = *reinterpret_cast<const uint32_t*>(slice + o);
  } else {
    r.w.x = *reinterpret_cast<const uint16_t*>(slice + o);
  }
  const int ng = D >> lg_group;
  r.sz = reinterpret_cast<const uint32_t*>(slice + 2 * a.P * kRow)[(which * a.P + slot) * ng + (8 * e >> lg_group)];
  return r;
}

}  // namespace trr
