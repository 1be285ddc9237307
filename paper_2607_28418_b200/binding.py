"""ctypes binding of libwide.so: the same entry points as include/wide.h, taking torch tensors.

Argument marshalling only -- every step of the path runs in the library's CUDA kernels.  Torch
is used for device memory and streams.  There is no fallback: if the shared library is missing
or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Dict, Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libwide.so")

OK = 0
BF16, F32 = 0, 1
ROUTE_TOPK, ROUTE_PAIR_ARGMAX = 0, 1
OP_ROUTE, OP_REORDER, OP_FFN, OP_OPROJ, OP_UNPERMUTE = 0, 1, 2, 3, 4
FLAG_NONE, FLAG_SIMT, FLAG_FORCE_PREFILL, FLAG_FORCE_DECODE, FLAG_INPUT_MASKED = 0, 1, 2, 4, 8
FLAG_KAXIS_GROUP, FLAG_KAXIS_OWNER, FLAG_REDUCE_BF16 = 16, 32, 64
FLAG_DECODE_TC = 128
FLAG_ROPE_INTERLEAVED, FLAG_ROPE_INVERSE = 256, 512
DECODE_MAX_TOKENS = 64
DECODE_GEMV_MAX_TOKENS = 2
MAX_GROUPS = 256
MAX_SEQS = 4096
ERR_INVALID_ARG, ERR_UNSUPPORTED_SHAPE, ERR_ALIGNMENT, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = -1, -2, -3, -4, -5, -6
ERR_BAD_INDEX = -7

EXPORTS = ["wide_create", "wide_destroy", "wide_status", "wide_set_wait_limit_ns", "wide_profile_begin",
           "wide_profile_end", "wide_launch_count", "wide_selftest_wait", "wide_strerror",
           "wide_version", "wide_workspace_bytes", "wide_route", "wide_route_static", "wide_route_pair_prepared_bytes",
           "wide_route_pair_norm_workspace_bytes", "wide_route_pair_prepare", "wide_route_pair_norm", "wide_reorder",
           "wide_mask_slice", "wide_ffn_tp",
           "wide_ffn",
           "wide_oproj", "wide_attn", "wide_qproj", "wide_unpermute",
           "wide_rope", "wide_cache_page_bytes", "wide_cache_write", "wide_cache_read", "wide_attn_cache_workspace_bytes",
           "wide_attn_cache"]

_c_void_p, _c_int, _c_size_t, _c_uint = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_uint
_c_ll = ctypes.c_longlong


class _CacheStruct(ctypes.Structure):   # wide_cache
    _fields_ = [("pages", _c_void_p), ("n_pages", _c_int), ("page_size", _c_int), ("n_kv_heads", _c_int),
                ("head_dim", _c_int), ("quant_group", _c_int)]


class _SeqsStruct(ctypes.Structure):    # wide_seqs
    _fields_ = [("page_table", _c_void_p), ("kv_lens", _c_void_p), ("row_start", _c_void_p), ("n_seqs", _c_int),
                ("max_pages", _c_int)]


class WideError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where} failed: {code} ({strerror(code)})")


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libwide.so (built by ``python -m paper_2607_28418_b200.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_28418_b200.build`; "
                           "there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    lib.wide_create.argtypes = [ctypes.POINTER(_c_void_p), _c_int]
    lib.wide_destroy.argtypes = [_c_void_p]
    lib.wide_status.argtypes = [_c_void_p, _c_void_p, ctypes.POINTER(_c_int)]
    lib.wide_set_wait_limit_ns.argtypes = [_c_void_p, ctypes.c_uint64]
    lib.wide_selftest_wait.argtypes = [_c_void_p, _c_void_p]
    lib.wide_profile_begin.argtypes = [_c_void_p, _c_int]
    lib.wide_profile_end.argtypes = [_c_void_p, _c_void_p, ctypes.c_char_p, _c_size_t]
    lib.wide_launch_count.argtypes = [_c_void_p, ctypes.POINTER(ctypes.c_ulonglong)]
    lib.wide_strerror.argtypes = [_c_int]
    lib.wide_strerror.restype = ctypes.c_char_p
    lib.wide_version.argtypes = []
    lib.wide_workspace_bytes.argtypes = [_c_int] * 7
    lib.wide_workspace_bytes.restype = _c_size_t
    lib.wide_route.argtypes = [_c_void_p, _c_void_p, _c_void_p, _c_int, _c_int, _c_int, _c_void_p, _c_void_p,
                               _c_int, _c_int, _c_int, _c_int, _c_void_p, _c_void_p, _c_void_p, _c_void_p,
                               _c_size_t, _c_uint]
    lib.wide_route_static.argtypes = lib.wide_route.argtypes[:15] + [_c_uint]
    lib.wide_route_pair_prepared_bytes.argtypes = [_c_int] * 3
    lib.wide_route_pair_prepared_bytes.restype = _c_size_t
    lib.wide_route_pair_norm_workspace_bytes.argtypes = [_c_int] * 2
    lib.wide_route_pair_norm_workspace_bytes.restype = _c_size_t
    lib.wide_route_pair_prepare.argtypes = [_c_void_p] * 5 + [_c_int] * 3 + [_c_void_p, _c_size_t]
    lib.wide_route_pair_norm.argtypes = [_c_void_p, _c_void_p, _c_void_p, _c_int, _c_int, _c_void_p, _c_void_p, _c_int, _c_int,
                                         _c_void_p, ctypes.c_float, _c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_size_t]
    lib.wide_reorder.argtypes = [_c_void_p, _c_void_p, _c_void_p, _c_int, _c_int, _c_int] + [_c_void_p] * 10
    lib.wide_mask_slice.argtypes = [_c_void_p, _c_void_p, _c_void_p, _c_int, _c_int, _c_int, _c_int, _c_void_p]
    lib.wide_ffn.argtypes = [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_int, _c_int,
                             _c_int, _c_int, _c_int, _c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_void_p,
                             _c_void_p, _c_int, _c_void_p, _c_size_t, _c_uint]
    lib.wide_ffn_tp.argtypes = [_c_void_p] * 6 + [_c_int] * 5 + [_c_void_p] * 6 + [_c_int, _c_int, _c_void_p, _c_size_t]
    lib.wide_oproj.argtypes = [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_int, _c_int, _c_int, _c_int, _c_int,
                               _c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_int,
                               _c_void_p, _c_size_t, _c_uint]
    lib.wide_attn.argtypes = [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_int, _c_int, _c_int, _c_int,
                              _c_int, _c_int, _c_int, _c_void_p, _c_void_p, _c_void_p, _c_int, ctypes.c_float,
                              _c_void_p, _c_uint]
    lib.wide_qproj.argtypes = [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_int, _c_int, _c_int, _c_int, _c_int,
                               _c_void_p, _c_void_p, _c_void_p, _c_uint]
    lib.wide_unpermute.argtypes = [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_int,
                                   _c_int, _c_int, _c_int, _c_void_p]
    lib.wide_rope.argtypes = [_c_void_p] * 4 + [_c_int] * 6 + [_c_ll] * 2 + [_c_void_p, _c_int] + [_c_void_p] * 4 + [_c_ll] * 2 + [_c_uint]
    lib.wide_cache_page_bytes.argtypes = [_c_int] * 4
    lib.wide_cache_page_bytes.restype = _c_size_t
    for fn in (lib.wide_cache_write, lib.wide_cache_read):
        fn.argtypes = [_c_void_p] * 6 + [_c_int] * 2 + [_c_ll] * 2
    lib.wide_attn_cache_workspace_bytes.argtypes = [_c_int] * 4
    lib.wide_attn_cache_workspace_bytes.restype = _c_size_t
    lib.wide_attn_cache.argtypes = [_c_void_p] * 5 + [_c_int, _c_int, _c_ll, _c_int, _c_int, _c_void_p, _c_int,
                                                      ctypes.c_float, _c_void_p, _c_void_p, _c_size_t, _c_uint]
    for name in EXPORTS:
        if name not in ("wide_strerror", "wide_workspace_bytes", "wide_route_pair_prepared_bytes",
                        "wide_route_pair_norm_workspace_bytes", "wide_cache_page_bytes", "wide_attn_cache_workspace_bytes"):
            getattr(lib, name).restype = _c_int
    _lib = lib
    return lib


def strerror(code: int) -> str:
    return load_library().wide_strerror(code).decode()


def version() -> int:
    return load_library().wide_version()


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous CUDA tensor")
    return _c_void_p(t.data_ptr())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise ValueError(f"unsupported dtype {t.dtype}")


def _stream() -> _c_void_p:
    return _c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(code: int, where: str):
    if code != OK:
        raise WideError(code, where)


class Context:
    """Owns a wide_ctx for one device.  Scratch buffers are torch tensors cached per size."""

    def __init__(self, device: int = 0):
        self.lib = load_library()
        self.device = torch.device("cuda", device)
        h = _c_void_p()
        with torch.cuda.device(self.device):
            _check(self.lib.wide_create(ctypes.byref(h), device), "wide_create")
        self.handle = h
        self._ws: Dict[int, torch.Tensor] = {}

    def close(self):
        if self.handle:
            self.lib.wide_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace(self, nbytes: int, slot: int = 0) -> torch.Tensor:
        cur = self._ws.get(slot)
        if cur is None or cur.numel() < nbytes:
            cur = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
            self._ws[slot] = cur
        return cur

    def status(self) -> int:
        v = _c_int(0)
        _check(self.lib.wide_status(self.handle, _stream(), ctypes.byref(v)), "wide_status")
        return v.value

    def set_wait_limit_ns(self, ns: int):
        _check(self.lib.wide_set_wait_limit_ns(self.handle, int(ns)), "wide_set_wait_limit_ns")

    def selftest_wait(self):
        """Enqueue the kernel whose only wait can never be satisfied (see wide_selftest_wait)."""
        _check(self.lib.wide_selftest_wait(self.handle, _stream()), "wide_selftest_wait")

    def profile_begin(self, max_records: int = 4096):
        _check(self.lib.wide_profile_begin(self.handle, max_records), "wide_profile_begin")

    def profile_end(self) -> Dict[str, Dict[str, float]]:
        """{kernel name: {"launches": n, "total_ms": t}} for everything launched since profile_begin."""
        buf = ctypes.create_string_buffer(8192)
        _check(self.lib.wide_profile_end(self.handle, _stream(), buf, len(buf)), "wide_profile_end")
        out = {}
        for line in buf.value.decode().splitlines():
            name, n, ms = line.split(",")
            out[name] = {"launches": int(n), "total_ms": float(ms)}
        return out

    def launch_count(self) -> int:
        v = ctypes.c_ulonglong(0)
        _check(self.lib.wide_launch_count(self.handle, ctypes.byref(v)), "wide_launch_count")
        return int(v.value)


def upload(a, dtype: str, device: Optional[torch.device] = None) -> torch.Tensor:
    """Host float32 array -> CUDA tensor of the workload dtype ("bf16": the values must already be
    bf16-representable, the upload is then exact; "fp32": as is)."""
    import numpy as np

    from . import synth
    device = device or torch.device("cuda", torch.cuda.current_device())
    if dtype == "bf16":
        bits = synth.to_bf16_bits(a)
        return torch.from_numpy(bits.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device)


def workspace_bytes(op: int, dtype: int, tokens: int, hidden: int, inner: int, group: int, n_groups: int) -> int:
    return int(load_library().wide_workspace_bytes(op, dtype, tokens, hidden, inner, group, n_groups))


def wide_route(ctx: Context, x: torch.Tensor, w_router: torch.Tensor, n_groups: int, k: int = 0,
               mode: int = ROUTE_TOPK, w2: Optional[torch.Tensor] = None, rank: int = 0,
               k_per_token: Optional[torch.Tensor] = None, want_scores: bool = False,
               mask_bits: Optional[torch.Tensor] = None, flags: int = 0):
    """Returns (mask_bits int32 [T, W] holding the uint32 words, scores or None)."""
    T, D = x.shape
    W = (n_groups + 31) // 32
    if mask_bits is None:
        mask_bits = torch.empty((T, W), dtype=torch.int32, device=x.device)
    ncol = n_groups if mode == ROUTE_TOPK else 2 * n_groups
    scores = torch.empty((T, ncol), dtype=torch.float32, device=x.device) if want_scores else None
    nbytes = workspace_bytes(OP_ROUTE, _dtype_code(x), T, D, 0, 0, n_groups)
    ws = ctx.workspace(nbytes, slot=1)
    rc = ctx.lib.wide_route(ctx.handle, _stream(), _ptr(x), _dtype_code(x), T, D, _ptr(w_router), _ptr(w2), rank,
                            n_groups, mode, k, _ptr(k_per_token), _ptr(mask_bits), _ptr(scores), _ptr(ws),
                            ws.numel(), flags)
    _check(rc, "wide_route")
    return mask_bits, scores


def wide_route_pair_prepare(ctx: Context, w1: torch.Tensor, w2: torch.Tensor, norm_weight: Optional[torch.Tensor],
                            n_groups: int) -> torch.Tensor:
    """Once per weight set: the prepared buffer wide_route_pair_norm reads."""
    D, rank = w1.shape
    nbytes = int(ctx.lib.wide_route_pair_prepared_bytes(D, rank, n_groups))
    prepared = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=w1.device)
    rc = ctx.lib.wide_route_pair_prepare(ctx.handle, _stream(), _ptr(w1), _ptr(w2), _ptr(norm_weight), D, rank, n_groups,
                                         _ptr(prepared), prepared.numel())
    _check(rc, "wide_route_pair_prepare")
    return prepared


def wide_route_pair_norm(ctx: Context, x: torch.Tensor, w1: torch.Tensor, w2: torch.Tensor, norm_weight: Optional[torch.Tensor],
                         eps: float, prepared: torch.Tensor, n_groups: int, want_scores: bool = False,
                         mask_bits: Optional[torch.Tensor] = None):
    """Eq. 4 on RMSNorm(x): returns (mask_bits, logits of the normalised input or None)."""
    T, D = x.shape
    rank = w1.shape[1]
    if mask_bits is None:
        mask_bits = torch.empty((T, (n_groups + 31) // 32), dtype=torch.int32, device=x.device)
    scores = torch.empty((T, 2 * n_groups), dtype=torch.float32, device=x.device) if want_scores else None
    ws = ctx.workspace(int(ctx.lib.wide_route_pair_norm_workspace_bytes(T, rank)), slot=1)
    rc = ctx.lib.wide_route_pair_norm(ctx.handle, _stream(), _ptr(x), T, D, _ptr(w1), _ptr(w2), rank, n_groups,
                                      _ptr(norm_weight), float(eps), _ptr(prepared), _ptr(mask_bits), _ptr(scores), _ptr(ws),
                                      ws.numel())
    _check(rc, "wide_route_pair_norm")
    return mask_bits, scores


ROUTE_STATIC_BYTES = 2 << 20


def wide_route_static(ctx: Context, x: torch.Tensor, w_router: torch.Tensor, n_groups: int, k: int = 0,
                      mode: int = ROUTE_TOPK, w2: Optional[torch.Tensor] = None, rank: int = 0,
                      k_per_token: Optional[torch.Tensor] = None, scores: Optional[torch.Tensor] = None,
                      mask_bits: Optional[torch.Tensor] = None, flags: int = 0):
    """wide_route for callers that may not allocate: scratch is the library's fixed device array
    (problems beyond ROUTE_STATIC_BYTES of scratch are refused with ERR_WORKSPACE).  Pass
    preallocated ``mask_bits`` (and ``scores``) to keep the whole call allocation-free; calls that
    overlap on the GPU share the array and must be serialised by the caller."""
    T, D = x.shape
    if mask_bits is None:
        mask_bits = torch.empty((T, (n_groups + 31) // 32), dtype=torch.int32, device=x.device)
    rc = ctx.lib.wide_route_static(ctx.handle, _stream(), _ptr(x), _dtype_code(x), T, D, _ptr(w_router), _ptr(w2),
                                   rank, n_groups, mode, k, _ptr(k_per_token), _ptr(mask_bits), _ptr(scores), flags)
    _check(rc, "wide_route_static")
    return mask_bits, scores


def wide_reorder(ctx: Context, mask_bits: torch.Tensor, n_groups: int, tile_m: int = 128,
                 out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    T = mask_bits.shape[0]
    n_tiles = (T + tile_m - 1) // tile_m
    dev = mask_bits.device
    if out is None:
        i32 = dict(dtype=torch.int32, device=dev)
        out = {
            "perm": torch.empty((n_groups, T), **i32),
            "counts": torch.empty((n_groups,), **i32),
            "tile_map": torch.empty((n_tiles, n_groups), dtype=torch.uint8, device=dev),
            "work_list": torch.empty((max(n_tiles * n_groups, 1), 2), **i32),
            "n_work": torch.empty((1,), **i32),
            "union_list": torch.empty((n_groups,), **i32),
            "n_union": torch.empty((1,), **i32),
            "offsets": torch.empty((n_groups + 1,), **i32),
            "token_order": torch.empty((T,), **i32),
            "token_rank": torch.empty((T,), **i32),
        }
    rc = ctx.lib.wide_reorder(ctx.handle, _stream(), _ptr(mask_bits), T, n_groups, tile_m, _ptr(out["perm"]),
                              _ptr(out["counts"]), _ptr(out["tile_map"]), _ptr(out["work_list"]),
                              _ptr(out["n_work"]), _ptr(out["union_list"]), _ptr(out["n_union"]),
                              _ptr(out["offsets"]), _ptr(out.get("token_order")), _ptr(out.get("token_rank")))
    _check(rc, "wide_reorder")
    return out


def group_range(n_groups: int, world: int, rank: int):
    """Groups [begin, end) owned by `rank` when n_groups are dealt to `world` ranks in contiguous,
    balanced ranges (the first n_groups % world ranks hold one group more)."""
    base, rem = divmod(n_groups, world)
    begin = rank * base + min(rank, rem)
    return begin, begin + base + (1 if rank < rem else 0)


def wide_mask_slice(ctx: Context, mask_bits: torch.Tensor, n_groups: int, group_begin: int, group_end: int,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
    T = mask_bits.shape[0]
    if out is None:
        out = torch.empty((T, max(1, (group_end - group_begin + 31) // 32)), dtype=torch.int32, device=mask_bits.device)
    rc = ctx.lib.wide_mask_slice(ctx.handle, _stream(), _ptr(mask_bits), T, n_groups, group_begin, group_end, _ptr(out))
    _check(rc, "wide_mask_slice")
    return out


def wide_ffn_tp(ctx: Context, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, group: int,
                mask_bits_local: torch.Tensor, meta: Dict[str, torch.Tensor], shard_ptrs, rows_per_rank: int):
    """One rank's group-sharded FFN part, added straight into the fp32 shards of the ranks that own
    the token rows.  ``shard_ptrs``: one device address per rank (ints), e.g. ``t.data_ptr()`` of a
    local tensor for this rank and the peer-mapped addresses of the others."""
    T, D = x.shape
    d_ff = w_gate.shape[0]
    world = len(shard_ptrs)
    table = (ctypes.c_void_p * world)(*[ctypes.c_void_p(int(p)) for p in shard_ptrs])
    nbytes = workspace_bytes(OP_FFN, BF16, T, D, d_ff, group, d_ff // group)
    ws = ctx.workspace(nbytes, slot=0)
    rc = ctx.lib.wide_ffn_tp(ctx.handle, _stream(), _ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down), _dtype_code(x), T, D,
                             d_ff, group, _ptr(mask_bits_local), _ptr(meta["perm"]), _ptr(meta["counts"]),
                             _ptr(meta.get("token_order")), _ptr(meta.get("token_rank")),
                             ctypes.cast(table, ctypes.c_void_p), world, rows_per_rank, _ptr(ws), ws.numel())
    _check(rc, "wide_ffn_tp")


def wide_ffn(ctx: Context, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
             group: int, mask_bits: torch.Tensor, meta: Optional[Dict[str, torch.Tensor]] = None,
             out_dtype: Optional[torch.dtype] = None, flags: int = 0, y: Optional[torch.Tensor] = None) -> torch.Tensor:
    T, D = x.shape
    d_ff = w_gate.shape[0]
    out_dtype = out_dtype or x.dtype
    if y is None:
        y = torch.empty((T, D), dtype=out_dtype, device=x.device)
    dt = _dtype_code(x)
    nbytes = workspace_bytes(OP_FFN, dt, T, D, d_ff, group, d_ff // group)
    ws = ctx.workspace(nbytes, slot=0)
    m = meta or {}
    rc = ctx.lib.wide_ffn(ctx.handle, _stream(), _ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down), dt, T, D, d_ff,
                          group, _ptr(mask_bits), _ptr(m.get("perm")), _ptr(m.get("counts")),
                          _ptr(m.get("token_order")), _ptr(m.get("token_rank")), _ptr(y), _dtype_code(y), _ptr(ws),
                          ws.numel(), flags)
    _check(rc, "wide_ffn")
    return y


def wide_oproj(ctx: Context, attn_out: torch.Tensor, w_o: torch.Tensor, group: int, mask_bits: torch.Tensor,
               meta: Optional[Dict[str, torch.Tensor]] = None, out_dtype: Optional[torch.dtype] = None,
               flags: int = 0, y: Optional[torch.Tensor] = None) -> torch.Tensor:
    T, K = attn_out.shape
    D = w_o.shape[0]
    out_dtype = out_dtype or attn_out.dtype
    if y is None:
        y = torch.empty((T, D), dtype=out_dtype, device=attn_out.device)
    dt = _dtype_code(attn_out)
    nbytes = workspace_bytes(OP_OPROJ, dt, T, D, K, group, K // group)
    ws = ctx.workspace(nbytes, slot=0)
    m = meta or {}
    rc = ctx.lib.wide_oproj(ctx.handle, _stream(), _ptr(attn_out), _ptr(w_o), dt, T, D, K, group, _ptr(mask_bits),
                            _ptr(m.get("perm")), _ptr(m.get("counts")), _ptr(m.get("token_order")),
                            _ptr(m.get("token_rank")), _ptr(y), _dtype_code(y), _ptr(ws), ws.numel(), flags)
    _check(rc, "wide_oproj")
    return y


def wide_attn(ctx: Context, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, n_q_heads: int, n_kv_heads: int,
              heads_per_group: int, meta: Optional[Dict[str, torch.Tensor]], causal: bool = True, scale: float = 0.0,
              flags: int = 0, o: Optional[torch.Tensor] = None, mask_bits: Optional[torch.Tensor] = None) -> torch.Tensor:
    """q [T_q, H_q*d], k/v [T_k, H_kv*d] bf16; meta = wide_reorder outputs of the attention mask
    (prefill form), mask_bits = the mask itself (decode form, a handful of query tokens)."""
    Tq, Tk = q.shape[0], k.shape[0]
    head_dim = q.shape[1] // n_q_heads
    if o is None:
        o = torch.empty_like(q)
    m = meta or {}
    rc = ctx.lib.wide_attn(ctx.handle, _stream(), _ptr(q), _ptr(k), _ptr(v), _dtype_code(q), Tq, Tk, n_q_heads,
                           n_kv_heads, head_dim, heads_per_group, _ptr(mask_bits), _ptr(m.get("perm")),
                           _ptr(m.get("counts")), 1 if causal else 0, float(scale), _ptr(o), flags)
    _check(rc, "wide_attn")
    return o


def wide_qproj(ctx: Context, x: torch.Tensor, w: torch.Tensor, group: int, meta: Dict[str, torch.Tensor],
               flags: int = 0, y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [T, D], w [n_out, D] bf16; meta = wide_reorder outputs of the [T, n_out/group] mask."""
    T, D = x.shape
    n_out = w.shape[0]
    if y is None:
        y = torch.empty((T, n_out), dtype=x.dtype, device=x.device)
    rc = ctx.lib.wide_qproj(ctx.handle, _stream(), _ptr(x), _ptr(w), _dtype_code(x), T, D, n_out, group,
                            _ptr(meta["perm"]), _ptr(meta["counts"]), _ptr(y), flags)
    _check(rc, "wide_qproj")
    return y


def wide_unpermute(ctx: Context, src_packed: torch.Tensor, meta: Dict[str, torch.Tensor], tokens: int,
                   n_groups: int, group: int, dst: Optional[torch.Tensor] = None) -> torch.Tensor:
    if dst is None:
        dst = torch.empty((tokens, n_groups * group), dtype=src_packed.dtype, device=src_packed.device)
    rc = ctx.lib.wide_unpermute(ctx.handle, _stream(), _ptr(src_packed), _ptr(meta["perm"]), _ptr(meta["counts"]),
                                _ptr(meta["offsets"]), tokens, n_groups, group, src_packed.element_size(),
                                _ptr(dst))
    _check(rc, "wide_unpermute")
    return dst


# ------------------------------------------------------------------------------ rotary positions, the 4-bit cache
# A decode step makes these calls for a few microseconds of GPU work, so they ask torch as little as they can.
def _rows(t: torch.Tensor, width: int, what: str):
    """Address and row stride of a [rows, width] matrix whose rows may lie apart (a slice of a fused projection)."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or shape[1] != width or stride[1] != 1:
        raise ValueError(f"{what}: expected [rows, {width}] with contiguous rows")
    return t.data_ptr(), (stride[0] if shape[0] > 1 else width)     # one row may claim any stride


def _same_device(index: int, *tensors: Optional[torch.Tensor]):
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError(f"expected tensors on cuda:{index}, got one on {t.device}")


def _int32(t: Optional[torch.Tensor], what: str):
    if t is None:
        return None
    if t.dtype != torch.int32 or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous int32 tensor")
    return t.data_ptr()


def _on_device(call):
    """The context's device as the current one for the length of a call."""
    @functools.wraps(call)
    def wrapped(ctx, *args, **kw):
        if torch._C._cuda_getDevice() == ctx.device.index:
            return call(ctx, *args, **kw)
        with torch.cuda.device(ctx.device):
            return call(ctx, *args, **kw)
    return wrapped


@functools.lru_cache(maxsize=None)
def cache_page_bytes(page_size: int, n_kv_heads: int, head_dim: int, quant_group: int) -> int:
    """Bytes of one page of the 4-bit cache (0: the shape is not supported)."""
    return int(load_library().wide_cache_page_bytes(page_size, n_kv_heads, head_dim, quant_group))


class _Fixed:
    """A handle whose C structure holds the addresses of its tensors: the tensors' contents may change, the tensors may not."""

    __slots__ = ()
    _fixed = ()

    def __setattr__(self, name, value):
        if name in self._fixed:
            raise AttributeError(f"{type(self).__name__}.{name} is fixed: change the tensor in place, or make another {type(self).__name__}")
        object.__setattr__(self, name, value)

    def __delattr__(self, name):
        if name in self._fixed:
            raise AttributeError(f"{type(self).__name__}.{name} is fixed")
        object.__delattr__(self, name)

    def __setstate__(self, state):      # a copy: its attributes and its slots
        for part in state:
            for name, value in (part or {}).items():
                object.__setattr__(self, name, value)


class Cache(_Fixed):
    """The 4-bit cache of a layer: ``pages`` is any contiguous uint8 CUDA tensor of n_pages *
    cache_page_bytes(...) bytes, first dimension n_pages (see wide_cache in include/wide.h)."""

    __slots__ = _fixed = ("pages", "n_kv_heads", "head_dim", "quant_group", "page_size", "struct")

    def __init__(self, pages: torch.Tensor, n_kv_heads: int, head_dim: int, quant_group: int = 64, page_size: int = 64):
        if pages.dtype != torch.uint8 or not pages.is_contiguous() or pages.dim() < 2:
            raise ValueError("pages: expected a contiguous uint8 tensor, one page in the first dimension")
        size = cache_page_bytes(page_size, n_kv_heads, head_dim, quant_group)
        if size == 0:
            raise WideError(ERR_UNSUPPORTED_SHAPE, "Cache")
        n_pages = pages.shape[0]
        if pages.numel() != n_pages * size:
            raise ValueError(f"pages: expected {size} bytes a page, got {pages.numel() // max(1, n_pages)}")
        put = object.__setattr__
        put(self, "pages", pages)
        put(self, "n_kv_heads", n_kv_heads)
        put(self, "head_dim", head_dim)
        put(self, "quant_group", quant_group)
        put(self, "page_size", page_size)
        put(self, "struct", _CacheStruct(pages.data_ptr(), n_pages, page_size, n_kv_heads, head_dim, quant_group))

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, quant_group: int = 64, page_size: int = 64, device="cuda") -> "Cache":
        size = cache_page_bytes(page_size, n_kv_heads, head_dim, quant_group)
        if size == 0:
            raise WideError(ERR_UNSUPPORTED_SHAPE, "Cache.empty")
        return cls(torch.empty((n_pages, size), dtype=torch.uint8, device=device), n_kv_heads, head_dim, quant_group, page_size)


class Sequences(_Fixed):
    """Where the sequences of a call lie (see wide_seqs): page_table int32 [n_seqs, max_pages], kv_lens
    int32 [n_seqs] (the new tokens included), row_start int32 [n_seqs + 1] or None (one new row each).  The tensors' contents may
    change between calls, the tensors themselves may not."""

    __slots__ = _fixed = ("page_table", "kv_lens", "row_start", "n_seqs", "struct")

    def __init__(self, page_table: torch.Tensor, kv_lens: torch.Tensor, row_start: Optional[torch.Tensor] = None):
        shape = page_table.shape
        if len(shape) != 2 or kv_lens.shape != shape[:1]:
            raise ValueError("expected page_table [n_seqs, max_pages] and kv_lens [n_seqs]")
        if row_start is not None and row_start.shape != (shape[0] + 1,):
            raise ValueError("expected row_start [n_seqs + 1]")
        put = object.__setattr__
        put(self, "page_table", page_table)
        put(self, "kv_lens", kv_lens)
        put(self, "row_start", row_start)
        put(self, "n_seqs", shape[0])
        put(self, "struct", _SeqsStruct(_int32(page_table, "page_table"), _int32(kv_lens, "kv_lens"), _int32(row_start, "row_start"), shape[0], shape[1]))


@_on_device
def wide_rope(ctx: Context, q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor, inv_freq: torch.Tensor,
              axis: Optional[torch.Tensor] = None, head_dim: int = 128, interleaved: bool = False, inverse: bool = False,
              q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """Rotary positions of q [T, n_q_heads * head_dim] and k (or None): returns (q_out, k_out).  positions
    int32 [T] or [n_axes, T]; inv_freq float64 [rot_dim / 2]; axis int32 [rot_dim / 2], the axis a pair
    follows.  q_out = q / k_out = k rotate in place.  ``inverse`` rotates back, which is the gradient."""
    if q.dim() != 2 or (k is not None and (k.dim() != 2 or k.shape[0] != q.shape[0] or k.dtype != q.dtype)):
        raise ValueError("expected q [T, n_q_heads * head_dim] and k [T, n_kv_heads * head_dim] of one dtype")
    (T, wq), wk = q.shape, 0 if k is None else k.shape[1]
    if head_dim <= 0 or wq % head_dim or wk % head_dim:
        raise ValueError("q and k must hold whole heads")
    where = positions.shape
    if len(where) not in (1, 2) or where[-1] != T:
        raise ValueError("expected positions [T] or [n_axes, T]")
    if inv_freq.dtype != torch.float64 or not inv_freq.is_contiguous() or (axis is not None and axis.shape != inv_freq.shape):
        raise ValueError("expected inv_freq float64 [rot_dim / 2] and axis of its shape")
    if q_out is None:
        q_out = q.new_empty((T, wq))
    elif q_out.shape != q.shape or q_out.dtype != q.dtype:
        raise ValueError("q_out: expected q's shape and dtype")
    if k is None:
        if k_out is not None:
            raise ValueError("k_out without k")
    elif k_out is None:
        k_out = k.new_empty((T, wk))
    elif k_out.shape != k.shape or k_out.dtype != k.dtype:
        raise ValueError("k_out: expected k's shape and dtype")
    index = ctx.device.index
    _same_device(index, q, k, positions, inv_freq, axis, q_out, k_out)
    (qp, qs), (qo, oqs) = _rows(q, wq, "q"), _rows(q_out, wq, "q_out")
    (kp, ks), (ko, oks) = ((None, 0), (None, 0)) if k is None else (_rows(k, wk, "k"), _rows(k_out, wk, "k_out"))
    flags = (FLAG_ROPE_INTERLEAVED if interleaved else 0) | (FLAG_ROPE_INVERSE if inverse else 0)
    pos, ax = _int32(positions, "positions"), _int32(axis, "axis")
    if T == 0:
        return q_out, k_out
    rc = ctx.lib.wide_rope(ctx.handle, torch._C._cuda_getCurrentRawStream(index), qp, kp, _dtype_code(q), T, wq // head_dim,
                           wk // head_dim, head_dim, 2 * inv_freq.numel(), qs, ks, pos, where[0] if len(where) == 2 else 1,
                           inv_freq.data_ptr(), ax, qo, ko, oqs, oks, flags)
    if rc != OK:
        raise WideError(rc, "wide_rope")
    return q_out, k_out


def _move(ctx: Context, what: str, call, cache: Cache, seqs: Sequences, k: torch.Tensor, v: torch.Tensor):
    if k.dtype != v.dtype or k.shape != v.shape:
        raise ValueError("k and v must have one shape and dtype")
    index = ctx.device.index
    _same_device(index, cache.pages, k, v, seqs.page_table, seqs.kv_lens, seqs.row_start)
    width = cache.n_kv_heads * cache.head_dim
    (kp, ks), (vp, vs) = _rows(k, width, "k"), _rows(v, width, "v")
    rows = k.shape[0]
    if rows == 0 or seqs.n_seqs == 0:
        return
    rc = call(ctx.handle, torch._C._cuda_getCurrentRawStream(index), ctypes.byref(cache.struct), ctypes.byref(seqs.struct), kp, vp,
              _dtype_code(k), rows, ks, vs)
    if rc != OK:
        raise WideError(rc, what)


@_on_device
def wide_cache_write(ctx: Context, cache: Cache, seqs: Sequences, k: torch.Tensor, v: torch.Tensor):
    """Quantise and store the new rows k, v [rows, n_kv_heads * head_dim] (bf16 or fp32)."""
    _move(ctx, "wide_cache_write", ctx.lib.wide_cache_write, cache, seqs, k, v)


@_on_device
def wide_cache_read(ctx: Context, cache: Cache, seqs: Sequences, rows: int, dtype: torch.dtype = torch.bfloat16,
                    k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None):
    """The values the cache holds for the sequences' new rows: returns (k, v) [rows, n_kv_heads * head_dim].
    Rows of no sequence are not written."""
    width = cache.n_kv_heads * cache.head_dim
    if k is None:
        k = cache.pages.new_empty((rows, width), dtype=dtype)
    if v is None:
        v = cache.pages.new_empty((rows, width), dtype=dtype)
    if k.shape[0] != rows:
        raise ValueError("k and v must have `rows` rows")
    _move(ctx, "wide_cache_read", ctx.lib.wide_cache_read, cache, seqs, k, v)
    return k, v


@_on_device
def wide_attn_cache(ctx: Context, q: torch.Tensor, cache: Cache, seqs: Sequences, n_q_heads: int, heads_per_group: int,
                    mask_bits: Optional[torch.Tensor] = None, causal: bool = True, scale: float = 0.0,
                    o: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Masked attention of the new rows q [rows, n_q_heads * head_dim] bf16 over the cache.  ``workspace``
    (uint8, attn_cache_workspace_bytes) replaces the context's own scratch, which calls on one stream share.  Rows that belong to no
    sequence, or to a row range that is none, are not written: without ``o`` they hold what the allocation held before."""
    width = n_q_heads * cache.head_dim
    qp, qs = _rows(q, width, "q")
    rows = q.shape[0]
    if o is None:
        o = q.new_empty((rows, width))
    elif o.shape != q.shape or o.dtype != q.dtype or not o.is_contiguous():
        raise ValueError("o: expected a contiguous tensor of q's shape and dtype")
    if mask_bits is not None and mask_bits.shape != (rows, (n_q_heads // max(1, heads_per_group) + 31) // 32):
        raise ValueError("mask_bits: expected [rows, ceil(n_groups / 32)]")
    if workspace is None:      # one size serves every call, so this one stays where it is (captured graphs hold its address)
        workspace = ctx._ws.get(2)
        if workspace is None:
            workspace = ctx.workspace(attn_cache_workspace_bytes(rows, n_q_heads, cache.n_kv_heads, cache.head_dim), slot=2)
    index = ctx.device.index
    _same_device(index, q, cache.pages, o, mask_bits, workspace, seqs.page_table, seqs.kv_lens, seqs.row_start)
    bits = _int32(mask_bits, "mask_bits")
    if rows == 0 or seqs.n_seqs == 0:
        return o
    rc = ctx.lib.wide_attn_cache(ctx.handle, torch._C._cuda_getCurrentRawStream(index), ctypes.byref(cache.struct),
                                 ctypes.byref(seqs.struct), qp, _dtype_code(q), rows, qs, n_q_heads, heads_per_group, bits,
                                 1 if causal else 0, float(scale), o.data_ptr(), workspace.data_ptr(), workspace.nbytes, 0)
    if rc != OK:
        raise WideError(rc, "wide_attn_cache")
    return o


def attn_cache_workspace_bytes(rows: int, n_q_heads: int, n_kv_heads: int, head_dim: int) -> int:
    return int(load_library().wide_attn_cache_workspace_bytes(rows, n_q_heads, n_kv_heads, head_dim))
