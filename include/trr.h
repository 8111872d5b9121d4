/*
 * trr.h - C ABI of the TriRoute serving hot path on GB300 (sm_103a).
 *
 * TriRoute (arxiv 2607.06601) routes every token, at every layer, with a policy
 * pi_t = (a_t, e_t, b_t) (Sec. 3.1).  This library implements the inference-time
 * consumer of two of its axes:
 *   - a_t in {skip, local, full}: how much of the past the query reads
 *     (Sec. 3.2(A), Eq. 2);
 *   - b_t in {2, 4, 8, 16}: the bit-width at which the token's own K/V are written
 *     to the cache for later queries (Sec. 3.2(C), Eq. 4; 16 = native bf16).
 * At inference the decisions are hard (argmax), only the selected computation runs,
 * and each token's KV is stored at its chosen width in a paged cache (Sec. 3.8).
 * Sec. 7 names the two kernels a production system needs: mode-aware attention over
 * ragged skip/local/full work, and a mixed-precision paged KV cache that groups tokens
 * by precision.  Those are trr_decode_attn and trr_kv_append below.  The hard
 * decisions themselves (arg max of the router's logits) and their cost under the
 * model of Sec. 3.5 are trr_route_decisions; trr_kv_append_routed and
 * trr_decode_attn_routed take the same decisions inside their own kernels.
 *
 * Conventions shared by every entry point
 *   - Pointers marked "device" are CUDA device pointers on the current device; the
 *     library never takes ownership of them.  "host" pointers are read before return.
 *   - Every call is asynchronous and stream-ordered on `stream` (a cudaStream_t passed
 *     as void*; NULL = legacy default stream).  No call synchronises the device except
 *     trr_get_status and trr_destroy.
 *   - Host-detectable errors (NULL pointers, sizes out of range, layer out of range)
 *     return an error immediately and enqueue nothing.
 *   - Device-detectable errors (see trr_kv_append / trr_decode_attn) are recorded in a
 *     sticky device status word that keeps the FIRST error since it was last read;
 *     trr_get_status reads and clears it.  No kernel traps or asserts.
 *   - One stream at a time per cache: calls on the same cache must not overlap.
 *   - Kernels are launched with programmatic dependent launch.  The index arrays of a
 *     call (sequence ids, positions, bit-widths, modes, windows, router logits of the
 *     *_routed calls) are read while the previous kernel of the stream may still be
 *     running, so they must not be outputs of that kernel (produce them one kernel
 *     earlier, or copy them in from the host).  Query, K and V rows are read after it
 *     has finished.  A decode step (trr_decode_step) whose layer was not touched by the
 *     two calls enqueued before it on the cache also reads the layer's cache state early
 *     (see there); the other calls read the cache only after the previous kernel.
 *
 * Cache memory layout (fixed; the CPU oracle re-derives it independently)
 *   class index c = 0,1,2,3 <-> b = 2,4,8,16.   P = page_size, d = head_dim,
 *   G = group_size, Hkv = num_kv_heads, MP = ceil(max_context / P),
 *   W32 = ceil(max_context / 32).
 *   Metadata (int32 unless noted), all indexed [layer][seq]...:
 *     last_pos  [L][S]          last position appended to (layer, seq), -1 if none
 *     ntok      [L][S][4]       tokens of class c stored for (layer, seq)
 *     presence  [L][S][W32] u32 bit (p % 32) of word p / 32 set <=> token p is stored
 *     page_table[L][S][4][MP]   page ids of class c, in position order
 *     page_first[L][S][4][MP]   position of the first token of each page
 *     page_last [L][S][4][MP]   position of the last token of each page
 *     next_page [4]             pages handed out so far per class (bump allocator)
 *   Pools: class c holds pages_per_class[c] pages of PAGE_BYTES(b) bytes each:
 *     HDR        = roundup(4 * P, 128)           header: int32 positions[P]
 *     TOKB(b)    = 2*(d*b/8) + 2*(d/G)*4   (b < 16)  |  4*d   (b = 16)
 *     SLICE(b)   = P * TOKB(b) + MASKB          one KV head of one page
 *     MASKB      = 16 with head_modes, else 0
 *     PAGE_BYTES = roundup(HDR + Hkv * SLICE(b), 128)
 *     head h starts at HDR + h * SLICE(b); inside it, for b < 16:
 *       K codes [P][d*b/8] | V codes [P][d*b/8] | K sz [P][d/G][2] | V sz [P][d/G][2]
 *     where sz = (scale, zero) as IEEE binary16, and for b = 16:
 *       K [P][d] bf16 | V [P][d] bf16.
 *   Code packing: element j of a head vector sits at byte floor(j*b/8), bit (j*b) % 8,
 *   least significant bits first (2-bit codes 1,2,3,0 -> byte 0x39).
 *   Chunk order of 8- and 16-bit rows: in every cache except those of query groups
 *   g = Hq/Hkv >= 2 with g * (d/G) <= 8 and head_modes = 0, the K and V code regions of
 *   b = 8 and b = 16 slices store byte x of the slice (x counted from the slice's start,
 *   x < 2*P*d*b/8) at x' = 128*n + 16*(k XOR (n % 8)) + x % 16, where n = x / 128 and
 *   k = (x / 16) % 8: each 128-byte line keeps its 16-byte chunks in a permuted order
 *   (the order the attention's lanes read them without shared-memory bank conflicts).
 *   Everything else (b = 2 and 4, scales, positions, masks) is stored as above.
 *   Page allocation: entries are taken in array order; an entry of class c whose
 *   (layer, seq) has ntok % P == 0 opens page next_page[c]++ .
 *   Shared pages: after trr_fork several sequences of a layer may name the same full page;
 *   a partly filled page always belongs to one sequence.  After trr_evict a sequence's
 *   ntok counts the tokens still stored.  Entries of page_table, page_first and page_last
 *   past a class's ceil(ntok / P) are -1 in the rows that trr_fork, trr_evict and
 *   trr_free_seqs write.
 *   Per-head modes (head_modes = 1): the last 16 bytes of KV head h's slice hold a
 *   little-endian uint64 (then 8 zero bytes): bit `slot` set <=> the token in that slot
 *   stores KV head h.  A page starts with every bit clear when its slot 0 is written.
 */
#ifndef TRR_H
#define TRR_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define TRR_API __attribute__((visibility("default")))
#else
#define TRR_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  TRR_OK = 0,
  TRR_ERR_INVALID_ARG = 1,   /* bad pointer, size, enum value (bits, mode) or window */
  TRR_ERR_OUT_OF_MEMORY = 2, /* cudaMalloc failed or caller pool too small */
  TRR_ERR_OUT_OF_PAGES = 3,  /* a class pool is exhausted */
  TRR_ERR_BAD_POSITION = 4,  /* position outside [0, max_context) or not increasing */
  TRR_ERR_CUDA = 5,          /* a CUDA runtime call failed */
  TRR_ERR_UNSUPPORTED = 6,   /* configuration outside the supported set */
  TRR_ERR_BAD_VALUE = 7,     /* non-finite or |x| > 65504 value in a quantised group */
  TRR_ERR_TIMEOUT = 8        /* a bounded wait inside a kernel gave up */
} trr_status;

enum { TRR_F32 = 0, TRR_BF16 = 1 }; /* types of trr_kv_read's outputs */

enum { TRR_MODE_SKIP = 0, TRR_MODE_LOCAL = 1, TRR_MODE_FULL = 2 }; /* a_t, Eq. 2 */

typedef struct trr_cache_config {
  int32_t num_layers;      /* L >= 1 */
  int32_t max_seqs;        /* S >= 1: sequence ids are 0 .. S-1 */
  int32_t num_q_heads;     /* Hq, a multiple of num_kv_heads */
  int32_t num_kv_heads;    /* Hkv >= 1 */
  int32_t head_dim;        /* d: 64 or 128 */
  int32_t group_size;      /* G: 32, 64 or 128 with G <= d (quantiser group along d) */
  int32_t page_size;       /* P: 16, 32 or 64 tokens */
  int32_t max_context;     /* positions are 0 .. max_context-1 */
  int32_t pages_per_class[4]; /* pool capacity for b = 2, 4, 8, 16 */
  int32_t max_append;      /* largest n accepted by trr_kv_append */
  int32_t max_queries;     /* largest n accepted by trr_decode_attn */
  int32_t split_bytes;     /* least KV bytes (of 8-bit tokens) per split-K work item; 0 = 24576 */
  int32_t skip_writes_kv;  /* 0: a skip token stores no KV (default); 1: it stores KV */
  int32_t head_modes;      /* 0: one mode per token, modes[n] (default); 1: one mode per
                              query head, modes[n][Hq] (Sec. 3.2(A): per head by default),
                              with a presence mask per KV head in every page */
  void* pool;              /* device memory of >= trr_cache_required_bytes, or NULL */
  uint64_t pool_bytes;     /* size of `pool` (ignored when pool is NULL) */
} trr_cache_config;

typedef struct trr_cache trr_cache; /* opaque */

/* Bytes of device memory a cache with this configuration needs (metadata, scratch
 * and the four page pools).  Returns TRR_ERR_UNSUPPORTED / TRR_ERR_INVALID_ARG for a
 * configuration outside the supported set. */
TRR_API trr_status trr_cache_required_bytes(const trr_cache_config* cfg, uint64_t* bytes);

/* Create a cache on the current device.  With cfg->pool == NULL the library
 * cudaMallocs the memory and frees it in trr_destroy; otherwise it carves everything
 * out of the caller's buffer (>= trr_cache_required_bytes, 256-byte aligned), which
 * must outlive the cache.  All metadata starts empty.  Synchronous. */
TRR_API trr_status trr_create_cache(const trr_cache_config* cfg, trr_cache** out);

/* Quantise-on-write append (Sec. 3.2(C), Eq. 4; Sec. 3.8).
 *   n entries, taken in array order; entry i is token positions[i] of sequence
 *   seq_ids[i] at `layer`, with K/V rows k[i][Hkv][d], v[i][Hkv][d] (bf16, device,
 *   contiguous), bit-width bits[i] in {2,4,8,16} and attention mode modes[i].
 *   A skip token (modes[i] == 0) stores nothing unless skip_writes_kv == 1.
 *   With head_modes, modes is [n][Hq] (uint8, device): KV head j of entry i is stored
 *   when a query head reading it (h / (Hq / Hkv) == j) has a mode other than skip, or
 *   always with skip_writes_kv == 1; an entry none of whose KV heads is stored takes no
 *   slot.  An entry that takes a slot has every KV head's row written, and its slot's
 *   bit set in the presence mask of each KV head it stores.
 *   For b < 16 each group of G consecutive elements of a head vector is stored as
 *     z = fp16(min x),  s = fp16(fl32(fl32(max x - min x) / (2^b - 1))),
 *     c_j = clamp(rne((x_j - z) / s), 0, 2^b - 1)   (c_j = 0 when s == 0)
 *   with fl32 = IEEE binary32 round-to-nearest-even and rne taken on the EXACT quotient
 *   (c_j is the nearest level z + c*s, ties to the even c); b = 16 stores the bf16 bits.
 *   seq_ids, positions, k, v, bits, modes: device arrays; 0 <= n <= max_append.  They may
 *   be read while the previous kernel of the stream (a trr_* call) is still running:
 *   they must not be outputs of that call.
 *   Device-detected errors: seq id out of range or bits/mode not allowed
 *   (INVALID_ARG), a position outside [0, max_context) or not above the sequence's
 *   last one (BAD_POSITION), a pool running out (OUT_OF_PAGES).  Any of these makes
 *   the whole call a no-op and records the error of the lowest failing index.
 *   A quantised group holding a non-finite value or |x| > 65504 is stored as zeros
 *   and records BAD_VALUE; the rest of the call takes effect. */
TRR_API trr_status trr_kv_append(trr_cache* cache, int32_t layer, int32_t n,
                         const int32_t* seq_ids, const int32_t* positions,
                         const void* k_bf16, const void* v_bf16,
                         const uint8_t* bits, const uint8_t* modes, void* stream);

/* Mode-routed split-K decode attention over the mixed-precision cache (Eq. 2).
 *   n queries; query i belongs to sequence seq_ids[i] at position t = q_positions[i],
 *   has rows q[i][Hq][d] (bf16, device) and mode modes[i]:
 *     skip : out row = 0
 *     local: softmax attention over the stored tokens j with t-w+1 <= j <= t,
 *            w = windows[i] (or window_scalar when windows == NULL), w >= 1
 *     full : softmax attention over the stored tokens j <= t.
 *   With head_modes, modes is [n][Hq] and each query head h runs its own mode over the
 *   tokens that store its KV head (presence bit set); the window check applies when any
 *   head is local, and a mode value outside {0, 1, 2} in any head fails the query.
 *   Query head h reads KV head h / (Hq / Hkv).  Scores are softmax_scale * q.k
 *   (softmax_scale <= 0 means 1/sqrt(d)) with K/V dequantised as z + c*s; fp32
 *   accumulation, bf16 (round-to-nearest-even) output out[i][Hq][d] (device).
 *   A query with no stored token in range gets a zero row.
 *   Device-detected errors (seq id, mode or window invalid: INVALID_ARG; position
 *   outside [0, max_context): BAD_POSITION) zero that query's row and record the
 *   error of the lowest failing index; other queries are computed.
 *   seq_ids, q_positions, q, modes, windows, out: device; 0 <= n <= max_queries.
 *   seq_ids, q_positions, modes and windows may be read while the previous kernel of the
 *   stream (a trr_* call) is still running: they must not be outputs of that call. */
TRR_API trr_status trr_decode_attn(trr_cache* cache, int32_t layer, int32_t n,
                           const int32_t* seq_ids, const int32_t* q_positions,
                           const void* q_bf16, const uint8_t* modes,
                           const int32_t* windows, int32_t window_scalar,
                           float softmax_scale, void* out_bf16, void* stream);

/* One decode step of one layer in one kernel: trr_kv_append of the n entries followed by
 * trr_decode_attn of their queries at the same positions and modes (Sec. 3.8: at
 * inference each token's KV is stored at its chosen width b_t, Sec. 3.2(C) Eq. 4, and its
 * query attends in its mode a_t, Sec. 3.2(A) Eq. 2, over the cache including its own new
 * token).
 *   Entry i is token positions[i] of sequence seq_ids[i] (all distinct: one token per
 *   sequence) with K/V rows k[i][Hkv][d], v[i][Hkv][d] (bf16), bit-width bits[i] and mode
 *   modes[i], as trr_kv_append takes them; its query q[i][Hq][d] (bf16) attends at
 *   t = positions[i] in mode modes[i] with window windows[i] (or window_scalar) and
 *   writes out[i][Hq][d] (bf16), as trr_decode_attn does.  The results are those of the
 *   two calls in that order: the same page bytes and metadata, and attention over every
 *   stored token up to t in range, the entry's own token included.
 *   seq_ids, positions, k, v, bits, modes, q, windows, out: device arrays;
 *   0 <= n <= min(256, max_append, max_queries); k, v, q, out 16-byte aligned.  A cache
 *   with head_modes returns TRR_ERR_UNSUPPORTED.
 *   Errors are those of both calls, checked for the whole call before anything is
 *   stored: sequence id, bit-width or mode not allowed, a sequence named twice, or a
 *   local query with a window below 1 (INVALID_ARG); a position outside
 *   [0, max_context) or not above the sequence's last one (BAD_POSITION); a pool running
 *   out (OUT_OF_PAGES).  Any of these makes the call store nothing and write zero rows
 *   for every query, and records the error of the lowest failing entry.  A group that
 *   cannot be quantised (BAD_VALUE) is handled as trr_kv_append handles it.
 *   The index arrays (seq_ids, positions, bits, modes, windows) may be read while the
 *   previous kernel of the stream is still running: they must not be outputs of that
 *   kernel.  k, v and q are read after it has finished.  When neither of the two calls
 *   enqueued before this one on the cache was for the same layer, the kernel also reads
 *   the layer's cache state and starts its page copies before the previous kernel has
 *   finished; this relies on every kernel of the stream (the caller's included) not
 *   letting its successor start before its own predecessor has finished, which holds
 *   for kernels launched without programmatic dependent launch. */
TRR_API trr_status trr_decode_step(trr_cache* cache, int32_t layer, int32_t n, const int32_t* seq_ids,
                                   const int32_t* positions, const void* k_bf16, const void* v_bf16,
                                   const uint8_t* bits, const uint8_t* modes, const void* q_bf16,
                                   const int32_t* windows, int32_t window_scalar, float softmax_scale,
                                   void* out_bf16, void* stream);

/* trr_decode_attn without any per-call scratch in the cache's memory (this entry point
 * has no counterpart in the paper; it serves callers that cannot allocate).
 *   Same arguments, results and error contract as trr_decode_attn, but its scratch
 *   (control words, split arrival counters, fp32 partials) lives in one
 *   32 MiB array that the library declares as a static device variable: every GPU that
 *   loads the library holds it until the process exits, and no call allocates device
 *   memory.  This is for callers that must not call cudaMalloc at the point of the
 *   call, such as an engine running inside a fixed, fully reserved memory budget, and
 *   that need more queries per call than the cache's max_queries scratch was sized
 *   for: n is bounded by the array instead of by max_queries.
 *   The call needs 256 + n * Hq * (4 * (1 + ceil(S_cap / 16)) + S_cap * (4*d + 16))
 *   bytes (plus 256-byte rounding per region), with S_cap the most splits per query of
 *   this cache; a call above 32 MiB returns TRR_ERR_OUT_OF_MEMORY and launches nothing.
 *   The first call on a device looks up the array's device address (once per device,
 *   with that device current); make that first call before any stream capture.
 *   Every call clears what must start at zero and then overwrites the array, so calls
 *   that overlap on the GPU (on different streams, or from different caches) race;
 *   serialise them. */
TRR_API trr_status trr_decode_attn_static(trr_cache* cache, int32_t layer, int32_t n,
                                          const int32_t* seq_ids, const int32_t* q_positions,
                                          const void* q_bf16, const uint8_t* modes,
                                          const int32_t* windows, int32_t window_scalar,
                                          float softmax_scale, void* out_bf16, void* stream);

/* The router's hard decisions at inference and their cost (Sec. 3.8: the router takes
 * the arg max of its logits and only the selected computation runs; Sec. 3.5 cost
 * model, evaluated at the one-hot policy as Appendix C's expected_cost does).
 *   mode_logits[n][3] (options skip, local, full) and bit_logits[n][4] (options
 *   b = 2, 4, 8, 16): fp32, device.  Decision = index of the largest logit, the first
 *   of equal ones; a NaN logit is never chosen; a row of NaN gives option 0.
 *   Outputs (device, each may be NULL): modes[n], bits[n] (uint8, the values
 *   trr_kv_append / trr_decode_attn take); attn_flops[n] = Hq * 2 * d * kappa with
 *   kappa the key positions the query reads at 0-indexed position p = positions[i]:
 *   full p + 1, local min(p + 1, window), skip 0 (p < 0 is charged as p = 0);
 *   kv_bits[n] = 2 * Hkv * d * b bits (the cost model's 2 d_kv b), 0 for a skip token
 *   when skip_writes_kv == 0 (it stores nothing).
 *   totals[4] (int64, device, ADDED to, so that calls over layers and steps
 *   accumulate): sum of attn_flops, sum of kv_bits, the dense attention cost
 *   sum Hq * 2 * d * (p + 1) and the dense memory cost n * 2 * Hkv * d * 16, the
 *   normalisers of the budget fractions (Appendix C).
 *   positions, window >= 1 and the head shape are needed only when attn_flops,
 *   kv_bits or totals is given.  Float arrays 4-byte aligned, int64 arrays 8-byte.
 *   The logits and positions are read after the previous kernel of the stream has
 *   finished.  The outputs must not be passed to the very next trr_* call on the
 *   stream (trr_kv_append and trr_decode_attn read their index arrays while the
 *   previous kernel still runs): pass the logits to the *_routed calls instead, which
 *   decide the same way. */
TRR_API trr_status trr_route_decisions(int32_t n, const float* mode_logits, const float* bit_logits,
                                       const int32_t* positions, int32_t window, int32_t num_q_heads,
                                       int32_t head_dim, int32_t num_kv_heads, int32_t skip_writes_kv,
                                       uint8_t* modes, uint8_t* bits, int64_t* attn_flops,
                                       int64_t* kv_bits, int64_t* totals, void* stream);

/* trr_kv_append with each entry's mode and bit-width decided in the append's own
 * planning step from the router's logits, exactly as trr_route_decisions decides:
 * bit_logits[n][4] (b = 2, 4, 8, 16) and mode_logits[n][3] (skip, local, full), fp32,
 * device, 4-byte aligned.  Otherwise the same arguments, results and error contract as
 * trr_kv_append (the logits, like the other inputs, may be read while the previous
 * kernel of the stream is still running).  Decisions are per token: a cache with
 * head_modes returns TRR_ERR_UNSUPPORTED. */
TRR_API trr_status trr_kv_append_routed(trr_cache* cache, int32_t layer, int32_t n,
                                        const int32_t* seq_ids, const int32_t* positions,
                                        const void* k_bf16, const void* v_bf16,
                                        const float* bit_logits, const float* mode_logits,
                                        void* stream);

/* trr_decode_attn with each query's mode decided in the attention's planning step from
 * mode_logits[n][3] (skip, local, full; fp32, device, 4-byte aligned), exactly as
 * trr_route_decisions decides.  Otherwise the same as trr_decode_attn.  Decisions are
 * per token: a cache with head_modes returns TRR_ERR_UNSUPPORTED. */
TRR_API trr_status trr_decode_attn_routed(trr_cache* cache, int32_t layer, int32_t n,
                                          const int32_t* seq_ids, const int32_t* q_positions,
                                          const void* q_bf16, const float* mode_logits,
                                          const int32_t* windows, int32_t window_scalar,
                                          float softmax_scale, void* out_bf16, void* stream);

/* ---------------------------------------------------------------- shared prompts --
 *
 * Sequences that share a past (samples of one prompt, beams), sequences that stream past
 * their window, and the pages behind them.  The paper stores every token once per
 * sequence (Sec. 3.8); these calls keep its cache and its modes, and let sequences name
 * the same pages.
 *
 * Calls that take a workspace use `workspace_bytes` bytes of device memory at `workspace`
 * (256-byte aligned), at least trr_workspace_bytes(cache), only while they run: one
 * workspace serves every call on the cache, and caches whose calls do not overlap may use
 * one between them.  A smaller or misaligned one returns TRR_ERR_OUT_OF_MEMORY and
 * enqueues nothing. */
TRR_API trr_status trr_workspace_bytes(const trr_cache* cache, uint64_t* bytes);

/* Fork: for each entry i and every layer, sequence dst_seqs[i] becomes a copy of sequence
 * src_seqs[i] as it was after its position lengths[i] - 1: the same stored tokens, the
 * same last position (or lengths[i] - 1 where that is less).  What dst_seqs[i] held is
 * forgotten.  Pages whose P slots are all below lengths[i] are shared; the one page per
 * layer and class that is not is copied to a page of its own, so that either sequence
 * can be appended to.  dst_seqs[i] == src_seqs[i] cuts the sequence back to lengths[i]
 * positions.  Page ids of the copies: next_page upwards, in order of (layer, entry).
 *   src_seqs, dst_seqs, lengths: int32, device; 0 <= n <= min(max_seqs, 4096).
 *   Device-detected errors: a sequence id out of range, a negative length, a dst_seqs
 *   value that appears twice or is another entry's source (INVALID_ARG), a pool running
 *   out (OUT_OF_PAGES).  Any of these makes the whole call a no-op. */
TRR_API trr_status trr_fork(trr_cache* cache, int32_t n, const int32_t* src_seqs, const int32_t* dst_seqs,
                            const int32_t* lengths, void* workspace, uint64_t workspace_bytes, void* stream);

/* Evict: for each entry i and every layer, forget the full pages of sequence seq_ids[i]
 * whose tokens all lie in [sinks, keep_from[i]): what attention with `sinks` first tokens
 * and a window that starts at keep_from[i] does not read.  Their tokens count as not
 * stored from then on, in every mode; pages that hold a token to keep stay whole.
 *   seq_ids, keep_from: int32, device; 0 <= n <= min(max_seqs, 4096); sinks >= 0.
 *   Device-detected errors: a sequence id out of range or named before in the call
 *   (INVALID_ARG); that entry does nothing, the others take effect. */
TRR_API trr_status trr_evict(trr_cache* cache, int32_t n, const int32_t* seq_ids, const int32_t* keep_from,
                             int32_t sinks, void* stream);

/* Free: forget sequences seq_ids[0..n) in every layer (as new, any position may come
 * next).  Pages go back to the pools with the next trr_compact.
 *   seq_ids: int32, device; 0 <= n <= min(max_seqs, 4096).  An id out of range records
 *   INVALID_ARG; the others take effect. */
TRR_API trr_status trr_free_seqs(trr_cache* cache, int32_t n, const int32_t* seq_ids, void* stream);

/* Compact: give the pages that no sequence names back to the pools.  In each class, with
 * m pages in use, the pages with ids m and above move, in ascending order, to the unused
 * ids below m in ascending order; page tables follow, and next_page becomes m.  Stored
 * tokens, and so every attention result, stay as they were. */
TRR_API trr_status trr_compact(trr_cache* cache, void* workspace, uint64_t workspace_bytes, void* stream);

/* Decode attention with sinks: trr_decode_attn, but a local query also sees the first
 * `sinks` positions: local: the stored tokens j <= t with j >= t-w+1 or j < sinks.
 *   sinks >= 0 (0: trr_decode_attn's results, but for rounding; that call is one launch and
 *   the faster one where no sinks are kept: see trr_decode_attn_shared).  seq_ids,
 *   q_positions, modes, windows: device, read after the previous kernel of the stream has
 *   finished; q, out 16-byte aligned.  Otherwise the arguments, results and error contract of trr_decode_attn; a
 *   cache with head_modes returns TRR_ERR_UNSUPPORTED. */
TRR_API trr_status trr_decode_attn_sinks(trr_cache* cache, int32_t layer, int32_t n, const int32_t* seq_ids,
                                         const int32_t* q_positions, const void* q_bf16, const uint8_t* modes,
                                         const int32_t* windows, int32_t window_scalar, int32_t sinks,
                                         float softmax_scale, void* out_bf16, void* workspace,
                                         uint64_t workspace_bytes, void* stream);

/* Decode attention of queries whose sequences share pages: trr_decode_attn_sinks with the
 * queries given in groups, queries group_offsets[i] .. group_offsets[i+1]-1 forming group
 * i (queries outside every group stand alone).  Groups change no result but for rounding.
 * In each class, the leading pages that all full queries of a group name and see whole
 * are read once for the group; so put sequences forked from one prompt in one group, and
 * a sequence that shares nothing in none.
 *   Which call: this one pays where many rows share a long past.  GPU time of a call, this
 *   one against trr_decode_attn, no sinks: 64 queries of 32 heads on 32,768 shared tokens
 *   of 8 KV heads of 128, 93 and 526 us; 16 of them, 60 and 165; 8 of one sequence (a
 *   chunk), 62 and 139, on 8,192 tokens 44 and 48.  A KV head for each query head: 32
 *   queries of 12 heads on 2,048 tokens, 32 and 30; 63 routed queries on 7 prompts of
 *   4,099, 71 and 63.  Short prompts of a few samples each are better left to
 *   trr_decode_attn (4 queries of 12 heads on each of 128 prompts of 512: 123 and 73), and
 *   so are windows without sinks (64 queries of 32 heads, window 511: 47 and 29; 128
 *   queries on 8 KV heads of 128, window 1024: 59 and 57).
 *   group_offsets: int32[num_groups + 1], device, ascending from >= 0 to <= n;
 *   0 <= num_groups <= n.  Offsets that are not make every row zero and record
 *   INVALID_ARG.  Otherwise as trr_decode_attn_sinks. */
TRR_API trr_status trr_decode_attn_shared(trr_cache* cache, int32_t layer, int32_t n, const int32_t* seq_ids,
                                          const int32_t* q_positions, const void* q_bf16, const uint8_t* modes,
                                          const int32_t* windows, int32_t window_scalar, int32_t sinks,
                                          int32_t num_groups, const int32_t* group_offsets, float softmax_scale,
                                          void* out_bf16, void* workspace, uint64_t workspace_bytes, void* stream);

/* ------------------------------------------------------------- prompts by chunks --
 *
 * Calls on stretches of consecutive positions: stretch i is positions starts[i],
 * starts[i] + 1, ... of sequence seq_ids[i], and its rows in the call's other arrays are
 * offsets[i] .. offsets[i+1]-1.  seq_ids[n], starts[n], offsets[n + 1]: int32, device, read
 * after the previous kernel of the stream has finished (so they may be its outputs);
 * 0 <= n <= 4096.  A stretch may be empty (its sequence and start are then not looked at),
 * a sequence may be named more than once.  Rows in no stretch are left as they are.
 * Device-detected errors: offsets that do not ascend from >= 0 to <= the call's rows make
 * every row zero and record INVALID_ARG; a sequence id out of range (INVALID_ARG) or a
 * stretch that leaves [0, max_context) (BAD_POSITION) makes the stretch's rows zero; the
 * error of the lowest failing row is recorded. */

/* Bytes of workspace for trr_chunk_attn of num_chunks chunks with num_tokens queries whose
 * positions, and all before them, number at most max_keys: the sum of starts[i] + length
 * of chunk i (counting what is stored is enough, and chunks of local queries count their
 * windows and sinks only).  A chunk counts max_context, or what the four pools hold, at most;
 * a token takes 4 * num_kv_heads * head_dim bytes.  UNSUPPORTED where num_tokens *
 * num_q_heads or the workspace's tokens come to 2^31 - 256 or more, or the cache has head_modes. */
TRR_API trr_status trr_chunk_workspace_bytes(const trr_cache* cache, int32_t num_chunks, int32_t num_tokens,
                                             int64_t max_keys, uint64_t* bytes);

/* Attention of chunks of new tokens: the queries of a prompt's chunk, or of a few drafted
 * tokens, over everything that their sequences have stored up to them.  Append the
 * chunk's tokens first (trr_kv_append): a query sees its own token and the chunk's earlier
 * ones as they are stored.
 *   Chunks are stretches (above) of num_tokens rows: query r of chunk i stands at
 *   t = starts[i] + r - offsets[i], has rows q[r][Hq][d] (bf16) and mode modes[r]:
 *     skip : out row = 0
 *     local: softmax attention over the stored tokens j <= t with j >= t-w+1 or
 *            j < sinks, w = windows[r] (or window_scalar when windows == NULL), w >= 1
 *     full : softmax attention over the stored tokens j <= t,
 *   as trr_decode_attn_sinks has it for the same queries (but for rounding, see below):
 *   out[r][Hq][d] (bf16), a zero row where nothing is in sight.  lse (may be NULL): lse[r][Hq] float32, the natural
 *   logarithm of the sum of exp(softmax_scale * q.k) over the tokens in sight, -infinity
 *   for a zero row; with it, rows over parts of a past can be joined.
 *   seq_ids, starts, offsets, q, modes, windows, out, lse: device; q and out 16-byte
 *   aligned and not overlapping, lse 4-byte aligned; 0 <= num_tokens <= 2^20; sinks >= 0.
 *   workspace: device memory, 256-byte aligned, trr_chunk_workspace_bytes of it, used only
 *   while the call runs.  One that is smaller than that of max_keys 0 or misaligned returns
 *   TRR_ERR_OUT_OF_MEMORY and enqueues nothing; one that turns out too small for what is
 *   stored makes every row zero and records OUT_OF_MEMORY.
 *   Device-detected errors: those of stretches; a mode not allowed or a local query with a
 *   window below 1 (INVALID_ARG) makes that query's rows zero.  A cache with head_modes
 *   returns TRR_ERR_UNSUPPORTED.
 *   How near: K, V and the softmax weights are rounded to binary16 (11 bits, in steps of 2^-24
 *   below 2^-14), sums are binary32.
 *     A score is off by up to 2^-11 of the sum over channels of |softmax_scale q_j (k_j - c_j)|,
 *     c_j being what the channel's keys have in common (the middle of eight of them that lie
 *     within a third of it, else 0); 16-bit keys below 2^-14 by 2^-25 |softmax_scale q_j| each.
 *     That moves the token's weight by as large a part of it, and lse by no more.
 *     Beside that an element of out is off by its rounding to bf16, and by its weights' and
 *     values' roundings: a weight's by 2^-11 of it, or of the mean weight of its neighbours
 *     (blocks of 96 tokens in order of position at head_dim 64, of 80 at 128), a value's by
 *     2^-11 of it, or 2^-13 of the largest of eight values of its channel (2^-25, were those 0).
 *   Tokens of which binary16 holds too little make all rows of their chunk's KV head be done one
 *   by one in binary32: 16-bit values of 65536 and more, infinities, NaN, keys further than 65504
 *   from c, a 16-bit K or V row all of which lies below 2^-14 (of V: of what its channels are
 *   scaled to) and loses bits.  One such token in every head took 512 queries on 16,384 tokens
 *   (32 heads on 8 of 128) from 0.17 to 114 ms, 4096 on themselves (32 heads of 64) from 0.16 to
 *   33 ms, 32 chunks of 8 on 2,048 (12 heads of 64) from 0.16 to 3.5 ms.
 *   Which call: everything in sight is brought back to binary16 in the workspace, once for all
 *   queries of a chunk, and that costs the same for one query and for 64; trr_decode_attn reads
 *   the past once for each query, trr_decode_attn_shared (full queries, chunks as its groups)
 *   about once for each chunk and 128 rows.  From how many queries a chunk this call is the
 *   fastest depends on how many chunks fill the GPU and on the heads.  GPU time of full queries
 *   with cold caches, in us, this call / trr_decode_attn / trr_decode_attn_shared:
 *     32 chunks on 2,048 tokens, 12 heads of 64, of 1 query each: 132 / 40 / 58, of 4:
 *       131 / 83 / 73, of 8: 131 / 136 / 132, of 16: 133 / 246 / 155, of 64: 135 / 961 / 318;
 *     32 chunks on 4,096, 32 heads on 8 of 128, of 1: 292 / 86 / 79, of 8: 296 / 301 / 176,
 *       of 16: 298 / 573 / 223, of 32: 303 / 1080 / 318;
 *     1 chunk on 2,048, 12 heads of 64, of 8: 44 / 28 / 40, of 32: 44 / 37 / 41,
 *       of 128: 48 / 81 / 61;
 *     1 chunk on 32,768, 32 heads on 8 of 128, of 8: 119 / 118 / 69, of 32: 145 / 297 / 71,
 *       of 128: 138 / 1006 / 150. */
TRR_API trr_status trr_chunk_attn(trr_cache* cache, int32_t layer, int32_t num_chunks, const int32_t* seq_ids,
                                  const int32_t* starts, const int32_t* offsets, int32_t num_tokens, const void* q_bf16,
                                  const uint8_t* modes, const int32_t* windows, int32_t window_scalar, int32_t sinks,
                                  float softmax_scale, void* out_bf16, float* lse, void* workspace,
                                  uint64_t workspace_bytes, void* stream);

/* Read back: K and V of stretches (above), dequantised, one row a position.
 *   Row r: k_out[r * k_stride + h*d + j] = z + c*s (rounded once to binary32) or the stored
 *   bf16 value of the token at the row's position, for KV head h < Hkv; so for v_out; zeros
 *   where the sequence stores no token (or, with head_modes, the token not that head).
 *   type: TRR_F32, or TRR_BF16 (that value rounded to bf16).  Strides in elements, at least
 *   Hkv * d, rows and both arrays 16-byte aligned.  bits_out (may be NULL): [num_rows][Hkv]
 *   uint8, the width (2, 4, 8 or 16) that the row's token is stored at, 0 for zeros.
 *   Appending the rows again at their widths stores values as near to these as Eq. 4
 *   comes; it does not always give the same codes (scale and zero are taken anew).
 *   0 <= num_rows <= 2^30.  Device-detected errors: those of stretches. */
TRR_API trr_status trr_kv_read(trr_cache* cache, int32_t layer, int32_t n, const int32_t* seq_ids, const int32_t* starts,
                               const int32_t* offsets, int32_t num_rows, int32_t type, void* k_out, int64_t k_stride,
                               void* v_out, int64_t v_stride, uint8_t* bits_out, void* stream);

/* Free library-owned memory (waits for the device first).  A caller pool is not
 * freed.  NULL is accepted. */
TRR_API trr_status trr_destroy(trr_cache* cache);

/* Read and clear the sticky device status (synchronises `stream`).  After
 * TRR_ERR_TIMEOUT it also returns the cache's per-call counters to their start values
 * (on `stream`, before returning), so that later calls on the cache run normally. */
TRR_API trr_status trr_get_status(trr_cache* cache, void* stream);

/* Bound of every wait inside this cache's attention and decode-step kernels, in
 * nanoseconds of the GPU's global timer (0 = the default, 2 s; below 20000 the waiting
 * warps poll instead of suspending, so that the limit is kept).  A wait that runs out
 * makes its CTA stop, lets its copies in flight land, records TRR_ERR_TIMEOUT and
 * returns; the call's rows are then undefined and a decode step stores nothing.  No
 * kernel waits without a bound.  Host-side setting, read at each later call. */
TRR_API trr_status trr_set_wait_limit(trr_cache* cache, uint64_t nanoseconds);

/* Forget every sequence of every layer and return all pages to the pools
 * (stream-ordered; metadata only, page bytes are not cleared). */
TRR_API trr_status trr_reset(trr_cache* cache, void* stream);

/* Location of one layout region inside the cache's device memory, for inspection:
 * 0 last_pos, 1 ntok, 2 presence, 3 page_table, 4 page_first, 5 page_last,
 * 6 next_page, 7..10 pools of b = 2, 4, 8, 16.  *ptr is a device pointer. */
TRR_API trr_status trr_get_region(const trr_cache* cache, int32_t region, void** ptr,
                          uint64_t* bytes);

/* Number of SMs and kernels the last trr_decode_attn / trr_kv_append launched
 * (host-side bookkeeping, no synchronisation). */
TRR_API int32_t trr_last_launch_count(const trr_cache* cache);

#ifdef __cplusplus
}
#endif
#endif /* TRR_H */
