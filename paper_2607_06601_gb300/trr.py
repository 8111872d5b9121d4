"""Python binding of the C ABI in include/trr.h (argument marshalling only).

Every step of the serving path runs in the CUDA library ``_build/libtrr.so``; this
module only checks tensor dtypes / devices / shapes, passes raw device pointers and the
current CUDA stream, and turns status codes into exceptions.  There is no fallback: if
the library is missing, loading it raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

from . import build as _build

STATUS = {0: "OK", 1: "INVALID_ARG", 2: "OUT_OF_MEMORY", 3: "OUT_OF_PAGES", 4: "BAD_POSITION",
          5: "CUDA", 6: "UNSUPPORTED", 7: "BAD_VALUE", 8: "TIMEOUT"}
MODE_SKIP, MODE_LOCAL, MODE_FULL = 0, 1, 2
REGIONS = {"last_pos": 0, "ntok": 1, "presence": 2, "page_table": 3, "page_first": 4,
           "page_last": 5, "next_page": 6, "pool2": 7, "pool4": 8, "pool8": 9, "pool16": 10}


class TrrError(RuntimeError):
    def __init__(self, where: str, code: int):
        super().__init__(f"{where}: {STATUS.get(code, code)}")
        self.code = code


class trr_cache_config(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("max_seqs", ctypes.c_int32),
                ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("group_size", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("max_context", ctypes.c_int32),
                ("pages_per_class", ctypes.c_int32 * 4), ("max_append", ctypes.c_int32),
                ("max_queries", ctypes.c_int32), ("split_bytes", ctypes.c_int32),
                ("skip_writes_kv", ctypes.c_int32), ("head_modes", ctypes.c_int32),
                ("pool", ctypes.c_void_p),
                ("pool_bytes", ctypes.c_uint64)]


EXPORTS = ("trr_cache_required_bytes", "trr_create_cache", "trr_kv_append", "trr_decode_attn",
           "trr_decode_step", "trr_decode_attn_static", "trr_route_decisions", "trr_kv_append_routed",
           "trr_decode_attn_routed", "trr_destroy", "trr_get_status", "trr_set_wait_limit", "trr_reset",
           "trr_get_region", "trr_workspace_bytes", "trr_fork", "trr_evict", "trr_free_seqs", "trr_compact",
           "trr_decode_attn_sinks", "trr_decode_attn_shared", "trr_chunk_workspace_bytes", "trr_chunk_attn", "trr_kv_read",
           "trr_last_launch_count")

_lib = None


def library_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = False) -> ctypes.CDLL:
    """Load libtrr.so (built by __graft_entry__.build()); raise if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB
    if not os.path.exists(path):
        if not build_if_missing:
            raise RuntimeError(f"CUDA library {path} is missing: run __graft_entry__.build() first")
        _build.build()
    L = ctypes.CDLL(path)
    P, I32, U64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64
    L.trr_cache_required_bytes.argtypes = [ctypes.POINTER(trr_cache_config), ctypes.POINTER(U64)]
    L.trr_create_cache.argtypes = [ctypes.POINTER(trr_cache_config), ctypes.POINTER(P)]
    L.trr_kv_append.argtypes = [P, I32, I32, P, P, P, P, P, P, P]
    L.trr_decode_attn.argtypes = [P, I32, I32, P, P, P, P, P, I32, ctypes.c_float, P, P]
    L.trr_decode_attn_static.argtypes = [P, I32, I32, P, P, P, P, P, I32, ctypes.c_float, P, P]
    L.trr_decode_step.argtypes = [P, I32, I32, P, P, P, P, P, P, P, P, I32, ctypes.c_float, P, P]
    L.trr_route_decisions.argtypes = [I32, P, P, P, I32, I32, I32, I32, I32, P, P, P, P, P, P]
    L.trr_kv_append_routed.argtypes = [P, I32, I32, P, P, P, P, P, P, P]
    L.trr_decode_attn_routed.argtypes = [P, I32, I32, P, P, P, P, P, I32, ctypes.c_float, P, P]
    L.trr_destroy.argtypes = [P]
    L.trr_get_status.argtypes = [P, P]
    L.trr_set_wait_limit.argtypes = [P, U64]
    L.trr_reset.argtypes = [P, P]
    L.trr_get_region.argtypes = [P, I32, ctypes.POINTER(P), ctypes.POINTER(U64)]
    L.trr_last_launch_count.argtypes = [P]
    L.trr_workspace_bytes.argtypes = [P, ctypes.POINTER(U64)]
    L.trr_fork.argtypes = [P, I32, P, P, P, P, U64, P]
    L.trr_evict.argtypes = [P, I32, P, P, I32, P]
    L.trr_free_seqs.argtypes = [P, I32, P, P]
    L.trr_compact.argtypes = [P, P, U64, P]
    L.trr_decode_attn_sinks.argtypes = [P, I32, I32, P, P, P, P, P, I32, I32, ctypes.c_float, P, P, U64, P]
    L.trr_decode_attn_shared.argtypes = [P, I32, I32, P, P, P, P, P, I32, I32, I32, P, ctypes.c_float, P, P, U64, P]
    I64 = ctypes.c_int64
    L.trr_chunk_workspace_bytes.argtypes = [P, I32, I32, I64, ctypes.POINTER(U64)]
    L.trr_chunk_attn.argtypes = [P, I32, I32, P, P, P, I32, P, P, P, I32, I32, ctypes.c_float, P, P, P, U64, P]
    L.trr_kv_read.argtypes = [P, I32, I32, P, P, P, I32, I32, P, I64, P, I64, P, P]
    for name in EXPORTS:
        getattr(L, name).restype = I32
    _lib = L
    return L


def _check(where, code):
    if code != 0:
        raise TrrError(where, code)


def _stream(stream):
    """The cudaStream_t of `stream`, or of the current stream (asked for as a number: building the
    Stream object of torch.cuda.current_stream takes 3 us of a call's host time)."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _dev(t: torch.Tensor, dtype, name):
    """The address of a contiguous CUDA tensor of that dtype (ctypes turns it into a pointer)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _new(shape, dtype, device, stream):
    """Memory for a call on `stream`: the allocator takes it from that stream's own, whose last users are
    behind it there, and hands it out again only after what the current stream does with it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    current = torch.cuda.current_stream()
    if current != stream:
        t.record_stream(current)
    return t


def make_config(num_layers, max_seqs, num_q_heads, num_kv_heads, head_dim, group_size,
                page_size, max_context, pages_per_class, max_append=1024, max_queries=1024,
                split_bytes=0, skip_writes_kv=0, head_modes=0) -> trr_cache_config:
    cfg = trr_cache_config()
    cfg.num_layers, cfg.max_seqs = num_layers, max_seqs
    cfg.num_q_heads, cfg.num_kv_heads = num_q_heads, num_kv_heads
    cfg.head_dim, cfg.group_size, cfg.page_size = head_dim, group_size, page_size
    cfg.max_context = max_context
    for i in range(4):
        cfg.pages_per_class[i] = int(pages_per_class[i])
    cfg.max_append, cfg.max_queries = max_append, max_queries
    cfg.split_bytes, cfg.skip_writes_kv = split_bytes, skip_writes_kv
    cfg.head_modes = head_modes
    return cfg


def trr_cache_required_bytes(cfg: trr_cache_config) -> int:
    out = ctypes.c_uint64()
    _check("trr_cache_required_bytes", load().trr_cache_required_bytes(ctypes.byref(cfg), ctypes.byref(out)))
    return int(out.value)


def trr_create_cache(cfg: trr_cache_config, pool: torch.Tensor | None = None) -> ctypes.c_void_p:
    if pool is not None:
        cfg.pool = ctypes.c_void_p(pool.data_ptr())
        cfg.pool_bytes = pool.numel() * pool.element_size()
    h = ctypes.c_void_p()
    _check("trr_create_cache", load().trr_create_cache(ctypes.byref(cfg), ctypes.byref(h)))
    return h


def trr_kv_append(cache, layer, seq_ids, positions, k, v, bits, modes, stream=None):
    n = seq_ids.numel()
    _check("trr_kv_append", load().trr_kv_append(
        cache, layer, n, _dev(seq_ids, torch.int32, "seq_ids"), _dev(positions, torch.int32, "positions"),
        _dev(k, torch.bfloat16, "k"), _dev(v, torch.bfloat16, "v"), _dev(bits, torch.uint8, "bits"),
        _dev(modes, torch.uint8, "modes"), _stream(stream)))


def trr_decode_attn(cache, layer, seq_ids, q_positions, q, modes, windows, window_scalar,
                    softmax_scale, out, stream=None):
    n = seq_ids.numel()
    win = None if windows is None else _dev(windows, torch.int32, "windows")
    _check("trr_decode_attn", load().trr_decode_attn(
        cache, layer, n, _dev(seq_ids, torch.int32, "seq_ids"),
        _dev(q_positions, torch.int32, "q_positions"), _dev(q, torch.bfloat16, "q"),
        _dev(modes, torch.uint8, "modes"), win, int(window_scalar), float(softmax_scale),
        _dev(out, torch.bfloat16, "out"), _stream(stream)))


def trr_decode_step(cache, layer, seq_ids, positions, k, v, bits, modes, q, windows, window_scalar,
                    softmax_scale, out, stream=None):
    """One decode step of one layer in one kernel: the append of every entry's token, then
    every entry's query at the same position and mode (see include/trr.h)."""
    n = seq_ids.numel()
    win = None if windows is None else _dev(windows, torch.int32, "windows")
    _check("trr_decode_step", load().trr_decode_step(
        cache, layer, n, _dev(seq_ids, torch.int32, "seq_ids"), _dev(positions, torch.int32, "positions"),
        _dev(k, torch.bfloat16, "k"), _dev(v, torch.bfloat16, "v"), _dev(bits, torch.uint8, "bits"),
        _dev(modes, torch.uint8, "modes"), _dev(q, torch.bfloat16, "q"), win, int(window_scalar),
        float(softmax_scale), _dev(out, torch.bfloat16, "out"), _stream(stream)))


def trr_decode_attn_static(cache, layer, seq_ids, q_positions, q, modes, windows, window_scalar,
                           softmax_scale, out, stream=None):
    """trr_decode_attn with its scratch in the library's static device array: no
    allocation anywhere on the way (see include/trr.h)."""
    n = seq_ids.numel()
    win = None if windows is None else _dev(windows, torch.int32, "windows")
    _check("trr_decode_attn_static", load().trr_decode_attn_static(
        cache, layer, n, _dev(seq_ids, torch.int32, "seq_ids"),
        _dev(q_positions, torch.int32, "q_positions"), _dev(q, torch.bfloat16, "q"),
        _dev(modes, torch.uint8, "modes"), win, int(window_scalar), float(softmax_scale),
        _dev(out, torch.bfloat16, "out"), _stream(stream)))


def _opt(t, dtype, name):
    return None if t is None else _dev(t, dtype, name)


def trr_route_decisions(mode_logits, bit_logits, positions=None, window=1, num_q_heads=1, head_dim=1,
                        num_kv_heads=1, skip_writes_kv=0, modes=None, bits=None, attn_flops=None,
                        kv_bits=None, totals=None, stream=None):
    """Hard decisions of n tokens (and, with positions, their cost) into the given
    device tensors; ``totals`` (int64[4]) is added to."""
    n = mode_logits.shape[0] if mode_logits.dim() else 0
    if mode_logits.numel() != 3 * n or bit_logits.numel() != 4 * n:
        raise ValueError("mode_logits must be [n][3] and bit_logits [n][4]")
    for t, k, name in ((modes, n, "modes"), (bits, n, "bits"), (attn_flops, n, "attn_flops"),
                       (kv_bits, n, "kv_bits"), (positions, n, "positions"), (totals, 4, "totals")):
        if t is not None and t.numel() != k:
            raise ValueError(f"{name} must have {k} elements")
    _check("trr_route_decisions", load().trr_route_decisions(
        n, _dev(mode_logits, torch.float32, "mode_logits"), _dev(bit_logits, torch.float32, "bit_logits"),
        _opt(positions, torch.int32, "positions"), int(window), int(num_q_heads), int(head_dim),
        int(num_kv_heads), int(skip_writes_kv), _opt(modes, torch.uint8, "modes"),
        _opt(bits, torch.uint8, "bits"), _opt(attn_flops, torch.int64, "attn_flops"),
        _opt(kv_bits, torch.int64, "kv_bits"), _opt(totals, torch.int64, "totals"), _stream(stream)))


def trr_kv_append_routed(cache, layer, seq_ids, positions, k, v, bit_logits, mode_logits, stream=None):
    n = seq_ids.numel()
    if bit_logits.numel() != 4 * n or mode_logits.numel() != 3 * n:
        raise ValueError("bit_logits must be [n][4] and mode_logits [n][3]")
    _check("trr_kv_append_routed", load().trr_kv_append_routed(
        cache, layer, n, _dev(seq_ids, torch.int32, "seq_ids"), _dev(positions, torch.int32, "positions"),
        _dev(k, torch.bfloat16, "k"), _dev(v, torch.bfloat16, "v"),
        _dev(bit_logits, torch.float32, "bit_logits"), _dev(mode_logits, torch.float32, "mode_logits"),
        _stream(stream)))


def trr_decode_attn_routed(cache, layer, seq_ids, q_positions, q, mode_logits, windows, window_scalar,
                           softmax_scale, out, stream=None):
    n = seq_ids.numel()
    if mode_logits.numel() != 3 * n:
        raise ValueError("mode_logits must be [n][3]")
    win = None if windows is None else _dev(windows, torch.int32, "windows")
    _check("trr_decode_attn_routed", load().trr_decode_attn_routed(
        cache, layer, n, _dev(seq_ids, torch.int32, "seq_ids"),
        _dev(q_positions, torch.int32, "q_positions"), _dev(q, torch.bfloat16, "q"),
        _dev(mode_logits, torch.float32, "mode_logits"), win, int(window_scalar), float(softmax_scale),
        _dev(out, torch.bfloat16, "out"), _stream(stream)))


def trr_workspace_bytes(cache) -> int:
    out = ctypes.c_uint64()
    _check("trr_workspace_bytes", load().trr_workspace_bytes(cache, ctypes.byref(out)))
    return int(out.value)


def _same_length(n, t, name):
    if t.numel() != n:
        raise ValueError(f"{name} must have {n} elements, got {t.numel()}")


def trr_fork(cache, src_seqs, dst_seqs, lengths, workspace, stream=None):
    """dst_seqs[i] becomes src_seqs[i] up to position lengths[i] - 1, sharing its full pages."""
    n = src_seqs.numel()
    _same_length(n, dst_seqs, "dst_seqs")
    _same_length(n, lengths, "lengths")
    _check("trr_fork", load().trr_fork(
        cache, n, _dev(src_seqs, torch.int32, "src_seqs"), _dev(dst_seqs, torch.int32, "dst_seqs"),
        _dev(lengths, torch.int32, "lengths"), _dev(workspace, torch.uint8, "workspace"), workspace.numel(),
        _stream(stream)))


def trr_evict(cache, seq_ids, keep_from, sinks, stream=None):
    """Forget the full pages of each sequence that lie in [sinks, keep_from[i])."""
    n = seq_ids.numel()
    _same_length(n, keep_from, "keep_from")
    _check("trr_evict", load().trr_evict(cache, n, _dev(seq_ids, torch.int32, "seq_ids"),
                                         _dev(keep_from, torch.int32, "keep_from"), int(sinks), _stream(stream)))


def trr_free_seqs(cache, seq_ids, stream=None):
    _check("trr_free_seqs", load().trr_free_seqs(cache, seq_ids.numel(), _dev(seq_ids, torch.int32, "seq_ids"),
                                                 _stream(stream)))


def trr_compact(cache, workspace, stream=None):
    _check("trr_compact", load().trr_compact(cache, _dev(workspace, torch.uint8, "workspace"), workspace.numel(),
                                             _stream(stream)))


def _check_queries(n, q_positions, modes, windows):
    _same_length(n, q_positions, "q_positions")
    _same_length(n, modes, "modes")
    if windows is not None:
        _same_length(n, windows, "windows")


def trr_decode_attn_sinks(cache, layer, seq_ids, q_positions, q, modes, windows, window_scalar, sinks,
                          softmax_scale, out, workspace, stream=None):
    """trr_decode_attn whose local queries also see the first `sinks` positions."""
    n = seq_ids.numel()
    _check_queries(n, q_positions, modes, windows)
    _check("trr_decode_attn_sinks", load().trr_decode_attn_sinks(
        cache, layer, n, _dev(seq_ids, torch.int32, "seq_ids"), _dev(q_positions, torch.int32, "q_positions"),
        _dev(q, torch.bfloat16, "q"), _dev(modes, torch.uint8, "modes"), _opt(windows, torch.int32, "windows"),
        int(window_scalar), int(sinks), float(softmax_scale), _dev(out, torch.bfloat16, "out"),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)))


def trr_decode_attn_shared(cache, layer, seq_ids, q_positions, q, modes, windows, window_scalar, sinks,
                           group_offsets, softmax_scale, out, workspace, stream=None):
    """trr_decode_attn_sinks with the pages that a group's full queries share read once."""
    n = seq_ids.numel()
    _check_queries(n, q_positions, modes, windows)
    if group_offsets.numel() < 1:
        raise ValueError("group_offsets must have an element more than there are groups")
    _check("trr_decode_attn_shared", load().trr_decode_attn_shared(
        cache, layer, n, _dev(seq_ids, torch.int32, "seq_ids"), _dev(q_positions, torch.int32, "q_positions"),
        _dev(q, torch.bfloat16, "q"), _dev(modes, torch.uint8, "modes"), _opt(windows, torch.int32, "windows"),
        int(window_scalar), int(sinks), group_offsets.numel() - 1,
        _dev(group_offsets, torch.int32, "group_offsets"), float(softmax_scale), _dev(out, torch.bfloat16, "out"),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)))


def _check_stretches(seq_ids, starts, offsets):
    n = seq_ids.numel()
    _same_length(n, starts, "starts")
    _same_length(n + 1, offsets, "offsets")
    return n


def trr_chunk_workspace_bytes(cache, num_chunks, num_tokens, max_keys) -> int:
    out = ctypes.c_uint64()
    _check("trr_chunk_workspace_bytes", load().trr_chunk_workspace_bytes(cache, num_chunks, num_tokens, int(max_keys), ctypes.byref(out)))
    return int(out.value)


def trr_chunk_attn(cache, layer, seq_ids, starts, offsets, q, modes, windows, window_scalar, sinks, softmax_scale, out, lse,
                   workspace, stream=None):
    """Attention of chunks of new tokens (see include/trr.h); lse may be None."""
    n, tokens = _check_stretches(seq_ids, starts, offsets), modes.numel()
    if windows is not None:
        _same_length(tokens, windows, "windows")
    _check("trr_chunk_attn", load().trr_chunk_attn(
        cache, layer, n, _dev(seq_ids, torch.int32, "seq_ids"), _dev(starts, torch.int32, "starts"),
        _dev(offsets, torch.int32, "offsets"), tokens, _dev(q, torch.bfloat16, "q"), _dev(modes, torch.uint8, "modes"),
        _opt(windows, torch.int32, "windows"), int(window_scalar), int(sinks), float(softmax_scale),
        _dev(out, torch.bfloat16, "out"), _opt(lse, torch.float32, "lse"), _dev(workspace, torch.uint8, "workspace"),
        workspace.numel(), _stream(stream)))


TYPES = {torch.float32: 0, torch.bfloat16: 1}


def _rows_at(t, rows, name):
    """Address and row stride (elements) of a CUDA tensor of `rows` rows, each of them contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in TYPES:
        raise ValueError(f"{name} must be a CUDA tensor of float32 or bfloat16")
    if t.dim() < 2 or t.shape[0] != rows:
        raise ValueError(f"{name} must have {rows} rows, each contiguous")
    if t.is_contiguous():  # (a row of it, t[0], takes 2 us of a call's host time)
        return t.data_ptr(), t.numel() // rows if rows else 0
    if not t[0].is_contiguous():
        raise ValueError(f"{name} must have {rows} rows, each contiguous")
    return t.data_ptr(), t.stride(0)


def trr_kv_read(cache, layer, seq_ids, starts, offsets, k, v, bits, stream=None):
    """K and V of stretches read back into k and v, [rows][Hkv][d] (see include/trr.h); bits may be None."""
    n, rows = _check_stretches(seq_ids, starts, offsets), k.shape[0]
    if k.dtype != v.dtype:
        raise ValueError("k and v must have one type")
    (k_at, k_stride), (v_at, v_stride) = _rows_at(k, rows, "k"), _rows_at(v, rows, "v")
    _check("trr_kv_read", load().trr_kv_read(
        cache, layer, n, _dev(seq_ids, torch.int32, "seq_ids"), _dev(starts, torch.int32, "starts"),
        _dev(offsets, torch.int32, "offsets"), rows, TYPES[k.dtype], k_at, k_stride, v_at, v_stride,
        _opt(bits, torch.uint8, "bits"), _stream(stream)))


def trr_destroy(cache):
    _check("trr_destroy", load().trr_destroy(cache))


def trr_get_status(cache, stream=None) -> int:
    return int(load().trr_get_status(cache, _stream(stream)))


def trr_reset(cache, stream=None):
    _check("trr_reset", load().trr_reset(cache, _stream(stream)))


def trr_get_region(cache, region) -> tuple[int, int]:
    p, nb = ctypes.c_void_p(), ctypes.c_uint64()
    _check("trr_get_region", load().trr_get_region(cache, REGIONS.get(region, region),
                                                   ctypes.byref(p), ctypes.byref(nb)))
    return int(p.value or 0), int(nb.value)


def trr_last_launch_count(cache) -> int:
    return int(load().trr_last_launch_count(cache))


class Cache:
    """A cache on the current CUDA device whose memory is one caller-owned uint8 tensor."""

    def __init__(self, num_layers, max_seqs, num_q_heads, num_kv_heads, head_dim, group_size,
                 page_size, max_context, pages_per_class, max_append=1024, max_queries=1024,
                 split_bytes=0, skip_writes_kv=0, device=None, zero_pool=False, head_modes=0):
        self.cfg = make_config(num_layers, max_seqs, num_q_heads, num_kv_heads, head_dim,
                               group_size, page_size, max_context, pages_per_class, max_append,
                               max_queries, split_bytes, skip_writes_kv, head_modes)
        self.head_modes = int(head_modes)
        self.nbytes = trr_cache_required_bytes(self.cfg)
        alloc = torch.zeros if zero_pool else torch.empty
        self.pool = alloc(self.nbytes, dtype=torch.uint8, device=device or torch.cuda.current_device())
        self.handle = trr_create_cache(self.cfg, self.pool)
        self.L, self.S, self.Hq, self.Hkv = num_layers, max_seqs, num_q_heads, num_kv_heads
        self.d, self.G, self.P, self.max_context = head_dim, group_size, page_size, max_context
        self._workspace = None

    def _check_modes(self, modes, n):
        want = n * (self.Hq if self.head_modes else 1)
        if modes.numel() != want:
            raise ValueError(f"modes must have {want} elements "
                             f"({'[n][Hq]' if self.head_modes else '[n]'}), got {modes.numel()}")

    def append(self, layer, seq_ids, positions, k, v, bits, modes, stream=None):
        self._check_modes(modes, seq_ids.numel())
        trr_kv_append(self.handle, layer, seq_ids, positions, k, v, bits, modes, stream)

    def decode_attn(self, layer, seq_ids, q_positions, q, modes, windows=None, window_scalar=0,
                    softmax_scale=0.0, out=None, stream=None):
        self._check_modes(modes, seq_ids.numel())
        if out is None:
            out = _new((seq_ids.numel(), self.Hq, self.d), torch.bfloat16, q.device, stream)
        trr_decode_attn(self.handle, layer, seq_ids, q_positions, q, modes, windows, window_scalar,
                        softmax_scale, out, stream)
        return out

    def decode_step(self, layer, seq_ids, positions, k, v, bits, modes, q, windows=None, window_scalar=0,
                    softmax_scale=0.0, out=None, stream=None):
        self._check_modes(modes, seq_ids.numel())
        if out is None:
            out = _new((seq_ids.numel(), self.Hq, self.d), torch.bfloat16, q.device, stream)
        trr_decode_step(self.handle, layer, seq_ids, positions, k, v, bits, modes, q, windows, window_scalar,
                        softmax_scale, out, stream)
        return out

    def append_routed(self, layer, seq_ids, positions, k, v, bit_logits, mode_logits, stream=None):
        trr_kv_append_routed(self.handle, layer, seq_ids, positions, k, v, bit_logits, mode_logits, stream)

    def decode_attn_routed(self, layer, seq_ids, q_positions, q, mode_logits, windows=None,
                           window_scalar=0, softmax_scale=0.0, out=None, stream=None):
        if out is None:
            out = _new((seq_ids.numel(), self.Hq, self.d), torch.bfloat16, q.device, stream)
        trr_decode_attn_routed(self.handle, layer, seq_ids, q_positions, q, mode_logits, windows,
                               window_scalar, softmax_scale, out, stream)
        return out

    def workspace(self, stream=None) -> torch.Tensor:
        """Device memory of the calls below, allocated once for the cache, on the stream of the first
        of them: call it before capturing them in a CUDA graph."""
        if self._workspace is None:
            self._workspace = _new(trr_workspace_bytes(self.handle), torch.uint8, self.pool.device, stream)
        return self._workspace

    def fork(self, src_seqs, dst_seqs, lengths, stream=None):
        """Sequence dst_seqs[i] becomes a copy of src_seqs[i] up to position lengths[i] - 1, in every
        layer, sharing its full pages."""
        trr_fork(self.handle, src_seqs, dst_seqs, lengths, self.workspace(stream), stream)

    def evict(self, seq_ids, keep_from, sinks=0, stream=None):
        """Forget the full pages of each sequence that lie in [sinks, keep_from[i]), in every layer."""
        trr_evict(self.handle, seq_ids, keep_from, sinks, stream)

    def free(self, seq_ids, stream=None):
        """Forget the sequences, in every layer; compact() gives their pages back."""
        trr_free_seqs(self.handle, seq_ids, stream)

    def compact(self, stream=None):
        """Give the pages that no sequence names back to the pools."""
        trr_compact(self.handle, self.workspace(stream), stream)

    def _rows(self, seq_ids, q, out, stream):
        """The output of an attention call: q and out are [n][Hq][d]."""
        n = seq_ids.numel()
        size = n * self.Hq * self.d
        if q.numel() != size or (out is not None and out.numel() != size):
            raise ValueError(f"q and out must have {size} elements ([n][Hq][d])")
        return _new((n, self.Hq, self.d), torch.bfloat16, q.device, stream) if out is None else out

    def decode_attn_sinks(self, layer, seq_ids, q_positions, q, modes, sinks, windows=None, window_scalar=0,
                          softmax_scale=0.0, out=None, stream=None):
        """decode_attn whose local queries also see the first `sinks` positions."""
        out = self._rows(seq_ids, q, out, stream)
        trr_decode_attn_sinks(self.handle, layer, seq_ids, q_positions, q, modes, windows, window_scalar, sinks,
                              softmax_scale, out, self.workspace(stream), stream)
        return out

    def decode_attn_shared(self, layer, seq_ids, q_positions, q, modes, group_offsets, windows=None, window_scalar=0,
                           sinks=0, softmax_scale=0.0, out=None, stream=None):
        """decode_attn_sinks of queries in groups (group_offsets, int32, one more than there are groups):
        the pages that a group's full queries share are read once for the group."""
        out = self._rows(seq_ids, q, out, stream)
        trr_decode_attn_shared(self.handle, layer, seq_ids, q_positions, q, modes, windows, window_scalar, sinks,
                               group_offsets, softmax_scale, out, self.workspace(stream), stream)
        return out

    def chunk_workspace(self, num_chunks, num_tokens, max_keys=None, stream=None) -> torch.Tensor:
        """Device memory of a chunk_attn call on chunks of at most these sizes (see there)."""
        keys = num_chunks * self.max_context if max_keys is None else max_keys
        return _new(trr_chunk_workspace_bytes(self.handle, num_chunks, num_tokens, keys), torch.uint8, self.pool.device, stream)

    def chunk_attn(self, layer, seq_ids, starts, offsets, q, modes, windows=None, window_scalar=0, sinks=0, softmax_scale=0.0,
                   out=None, with_lse=False, lse=None, max_keys=None, workspace=None, stream=None):
        """Attention of chunks of new tokens, which have been appended before: rows offsets[i] .. offsets[i+1]-1 of q
        ([n][Hq][d]) are queries of sequence seq_ids[i] at positions starts[i], starts[i] + 1, ...; modes[n] and windows[n]
        are theirs.  Returns the rows, and with `with_lse` (or an `lse` to write to) the logarithms of their softmax sums,
        [n][Hq] float32.  Rows of a new `out` that no chunk names are not set.

        max_keys: at most how many positions the chunks reach over, the sum of starts[i] + length; by default every
        chunk's whole context, or all that the pools hold where that is less.  It sizes the workspace, 4 * Hkv * d bytes
        a position, which is allocated for the call unless one of `chunk_workspace` is given: a cache of many long
        contexts should give one of the two (32 chunks of 131,072 positions of 32 heads of 64 come to 34 GB)."""
        n = modes.numel()
        size = n * self.Hq * self.d
        if q.numel() != size or (out is not None and out.numel() != size):
            raise ValueError(f"q and out must have {size} elements ([n][Hq][d])")
        if lse is None and with_lse:
            lse = _new((n, self.Hq), torch.float32, q.device, stream)
        if lse is not None and lse.numel() != n * self.Hq:
            raise ValueError(f"lse must have {n * self.Hq} elements ([n][Hq])")
        if out is None:
            out = _new((n, self.Hq, self.d), torch.bfloat16, q.device, stream)
        if workspace is None:
            workspace = self.chunk_workspace(seq_ids.numel(), n, max_keys, stream)
        trr_chunk_attn(self.handle, layer, seq_ids, starts, offsets, q, modes, windows, window_scalar, sinks, softmax_scale,
                       out, lse, workspace, stream)
        return out if lse is None else (out, lse)

    def read(self, layer, seq_ids, starts, offsets, rows, dtype=torch.bfloat16, k=None, v=None, bits=None, stream=None):
        """K, V ([rows][Hkv][d], bfloat16 or float32) and widths ([rows][Hkv] uint8, 0: not stored) of what the cache
        holds: rows offsets[i] .. offsets[i+1]-1 are positions starts[i], starts[i] + 1, ... of sequence seq_ids[i].
        k and v may be given (their rows contiguous, at any stride).  Rows of new tensors that no stretch names are
        not set."""
        shape = (rows, self.Hkv, self.d)
        device = self.pool.device
        k = _new(shape, dtype, device, stream) if k is None else k
        v = _new(shape, k.dtype, device, stream) if v is None else v
        bits = _new(shape[:2], torch.uint8, device, stream) if bits is None else bits
        for t, name in ((k, "k"), (v, "v")):
            if t.shape[0] != rows or t.numel() != rows * self.Hkv * self.d:
                raise ValueError(f"{name} must have {rows} rows of {self.Hkv * self.d} elements ([rows][Hkv][d])")
        if bits.numel() != rows * self.Hkv:
            raise ValueError(f"bits must have {rows * self.Hkv} elements ([rows][Hkv])")
        trr_kv_read(self.handle, layer, seq_ids, starts, offsets, k, v, bits, stream)
        return k, v, bits

    def status(self, stream=None) -> int:
        return trr_get_status(self.handle, stream)

    def set_wait_limit(self, nanoseconds: int):
        """Bound of every in-kernel wait of this cache's calls (0: the default, 2 s)."""
        _check("trr_set_wait_limit", load().trr_set_wait_limit(self.handle, int(nanoseconds)))

    def reset(self, stream=None):
        trr_reset(self.handle, stream)

    def region(self, name) -> torch.Tensor:
        """A uint8 view (no copy) of one layout region inside the cache memory."""
        ptr, nb = trr_get_region(self.handle, name)
        off = ptr - self.pool.data_ptr()
        return self.pool[off:off + nb]

    def launches(self) -> int:
        return trr_last_launch_count(self.handle)

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            trr_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
