"""ctypes binding of the CAEE C ABI (include/caee.h).

Argument marshalling only: every step of the layer runs in the HIP kernels
of ``libcaee.so``.  Tensors are torch CUDA tensors (device memory); the
current torch stream of the tensors' device is passed to the library.
Importing this module fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
# CAEE_LIBRARY names another build of the library (e.g. the host-sanitized one).
LIB_PATH = os.environ.get("CAEE_LIBRARY") or os.path.join(HERE, "libcaee.so")

CAEE_OK, CAEE_ERR_INVALID_ARG, CAEE_ERR_UNSUPPORTED, CAEE_ERR_WORKSPACE, CAEE_ERR_HIP, CAEE_ERR_CAPACITY = range(6)
CAEE_F32, CAEE_BF16, CAEE_FP8_E4M3 = 0, 1, 2
KERNEL_KINDS = {"route": 0, "gate_up": 1, "down": 2, "combine": 3, "quant": 4, "plan": 5, "attention": 6, "matmul": 7}
DTYPE_CODE = {"f32": CAEE_F32, "bf16": CAEE_BF16, "fp8": CAEE_FP8_E4M3}
IMPORTANCE_CODE = {"max": 0, "sum": 1, "cir": 2}
LATENT_FORM_CODE = {"auto": 0, "absorbed": 1, "expanded": 2}
REFILL_CODE = {"score": 0, "none": 1, "random": 2, "literal": 3}


class CaeeError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"caee status {status}: {message}")
        self.status = status


class LayerDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("T", "d", "f", "E", "n_group", "topk_group", "k", "n_shared")] + [
        ("routed_scaling", ctypes.c_float), ("tau", ctypes.c_float),
        ("n_bins", ctypes.c_int32), ("importance", ctypes.c_int32),
        ("x_dtype", ctypes.c_int32), ("w_dtype", ctypes.c_int32), ("y_dtype", ctypes.c_int32),
        ("refill", ctypes.c_int32), ("seed", ctypes.c_uint32), ("keep_top1", ctypes.c_int32)]


class ExpertWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("w13", "w2", "w13_scale", "w2_scale", "sh_w13", "sh_w2", "sh_w13_scale", "sh_w2_scale")] + [
        ("layout", ctypes.c_int32)]


LAYOUT_ROWMAJOR, LAYOUT_TILED = 0, 1
STATS = 9   # entries of caee_route_out_t.stats


class OffloadDesc(ctypes.Structure):
    _fields_ = [("host_w13", ctypes.POINTER(ctypes.c_void_p)), ("host_w2", ctypes.POINTER(ctypes.c_void_p)),
                ("slot_w13", ctypes.c_void_p), ("slot_w2", ctypes.c_void_p),
                ("sh_w13", ctypes.c_void_p), ("sh_w2", ctypes.c_void_p),
                ("layout", ctypes.c_int32), ("n_cache", ctypes.c_int32), ("n_stage", ctypes.c_int32),
                ("fetch_batch", ctypes.c_int32), ("miss_cost", ctypes.c_float)]


class OffloadStats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in
                ("calls", "needed", "hits", "misses", "staged", "evictions", "bytes_h2d")] + [
        ("passes", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class RouteOut(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("topk_ids", "topk_w", "orig_ids", "masks", "stats", "bin_loads")]


class PagedPlanOut(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("cu_new", "cu_kv", "seq_len", "slots", "position", "request", "free_head", "lacking")]


class LatentDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("T", "B", "heads", "nope", "rope", "latent", "v", "block_size", "n_blocks", "max_blocks", "max_new",
                 "causal", "form", "y_dtype")] + [
        ("max_kv", ctypes.c_int64), ("q_stride", ctypes.c_int64), ("scale", ctypes.c_float)]


class LatentWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w_uk", "w_uk_t", "w_uv")]


class BlockMatmulDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("M", "N", "K", "x_dtype", "y_dtype", "layout")] + [
        ("x_stride", ctypes.c_int64), ("y_stride", ctypes.c_int64)]


def _load(path: str = LIB_PATH):
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with __graft_entry__.build() "
                          "(python -c 'import __graft_entry__ as g; g.build()')")
    # torch ships its own HIP runtime; importing it first makes the library
    # bind to that same runtime (one HIP runtime per process) instead of
    # loading a second copy that would not see the device torch opened.
    import torch  # noqa: F401
    lib = ctypes.CDLL(path)
    st = ctypes.c_int
    P = ctypes.c_void_p
    desc_p = ctypes.POINTER(LayerDesc)
    sig = {
        "caee_workspace_size": (st, [desc_p, ctypes.POINTER(ctypes.c_size_t)]),
        "caee_route_prune": (st, [desc_p, P, P, P, P, ctypes.POINTER(RouteOut), P, ctypes.c_size_t, P]),
        "caee_expert_ffn": (st, [desc_p, P, P, P, ctypes.POINTER(ExpertWeights), P, P, ctypes.c_size_t, P]),
        "caee_moe_layer": (st, [desc_p, P, P, P, P, P, ctypes.POINTER(ExpertWeights), P,
                                ctypes.POINTER(RouteOut), P, ctypes.c_size_t, P]),
        "caee_moe_layer_noalloc": (st, [desc_p, P, P, P, P, P, ctypes.POINTER(ExpertWeights), P,
                                        ctypes.POINTER(RouteOut), P]),
        "caee_pack_matrix": (st, [ctypes.c_int32, P, P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, P]),
        "caee_quantize_rows": (st, [ctypes.c_int32, P, ctypes.c_int64, ctypes.c_int64, P, P, P]),
        "caee_offload_create": (st, [desc_p, ctypes.POINTER(OffloadDesc), ctypes.POINTER(P)]),
        "caee_offload_destroy": (None, [P]),
        "caee_offload_layer": (st, [P, desc_p, P, P, P, P, ctypes.POINTER(RouteOut), P, ctypes.c_size_t, P, P]),
        "caee_offload_stats": (st, [P, ctypes.POINTER(OffloadStats)]),
        "caee_offload_residency": (st, [P, P]),
        "caee_offload_reset": (st, [P]),
        "caee_lru_step": (st, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, P, P, P, ctypes.c_int64, P, P, P, P]),
        "caee_paged_plan": (st, [ctypes.c_int32] * 4 + [P, P, P, P, ctypes.c_int32, P,
                                                        ctypes.POINTER(PagedPlanOut), P]),
        "caee_latent_store": (st, [ctypes.c_int32] * 4 + [P, ctypes.c_int64, P, ctypes.c_int64, P, P, ctypes.c_int64,
                                                          P]),
        "caee_latent_workspace_size": (st, [ctypes.POINTER(LatentDesc), ctypes.POINTER(ctypes.c_size_t)]),
        "caee_latent_attention": (st, [ctypes.POINTER(LatentDesc), P, ctypes.POINTER(LatentWeights), P, P, P, P, P, P,
                                       P, P, ctypes.c_size_t, P]),
        "caee_block_matmul_workspace_size": (st, [ctypes.POINTER(BlockMatmulDesc), ctypes.POINTER(ctypes.c_size_t)]),
        "caee_block_matmul": (st, [ctypes.POINTER(BlockMatmulDesc), P, P, P, P, P, P, ctypes.c_size_t, P]),
        "caee_status_str": (ctypes.c_char_p, [st]),
        "caee_last_error": (ctypes.c_char_p, []),
        "caee_abi_version": (ctypes.c_int, []),
        "caee_timing_enable": (st, [ctypes.c_int]),
        "caee_timing_reset": (st, []),
        "caee_timing_query": (st, [ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                   ctypes.POINTER(ctypes.c_int64)]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()


def load_library(path: str) -> None:
    """Bind this module to another build of the library (e.g. one compiled
    with different kernel tuning knobs)."""
    global lib
    lib = _load(path)


EXPORTED = ("caee_workspace_size", "caee_route_prune", "caee_expert_ffn", "caee_moe_layer", "caee_moe_layer_noalloc",
            "caee_pack_matrix", "caee_quantize_rows", "caee_offload_create", "caee_offload_destroy",
            "caee_offload_layer", "caee_offload_stats", "caee_offload_residency", "caee_offload_reset",
            "caee_lru_step", "caee_paged_plan", "caee_latent_store", "caee_latent_workspace_size",
            "caee_latent_attention", "caee_block_matmul_workspace_size", "caee_block_matmul", "caee_status_str", "caee_last_error", "caee_abi_version",
            "caee_timing_enable", "caee_timing_reset", "caee_timing_query")


def _check(status: int):
    if status != CAEE_OK:
        raise CaeeError(status, lib.caee_last_error().decode())


def abi_version() -> int:
    return lib.caee_abi_version()


@dataclass
class Layer:
    """Descriptor fields of one MoE layer call (see caee_layer_desc_t)."""

    T: int
    d: int
    f: int
    E: int
    n_group: int
    topk_group: int
    k: int
    n_shared: int
    routed_scaling: float
    tau: float = 0.0
    n_bins: int = 1
    w_dtype: str = "bf16"
    x_dtype: str = "bf16"
    y_dtype: str = "bf16"
    importance: str = "max"     # "max" | "sum" | "cir" (caee_importance_t)
    refill: str = "score"       # "score" | "none" | "random" | "literal" (caee_refill_t)
    seed: int = 0               # random refill keys
    keep_top1: bool = False     # each token's top expert mandatory in every call (not the paper's step 1)

    def desc(self) -> LayerDesc:
        return LayerDesc(self.T, self.d, self.f, self.E, self.n_group, self.topk_group, self.k,
                         self.n_shared, self.routed_scaling, self.tau, self.n_bins,
                         IMPORTANCE_CODE[self.importance],
                         DTYPE_CODE[self.x_dtype], DTYPE_CODE[self.w_dtype], DTYPE_CODE[self.y_dtype],
                         REFILL_CODE[self.refill], self.seed & 0xFFFFFFFF, 1 if self.keep_top1 else 0)

    @classmethod
    def from_shape(cls, shape, **over) -> "Layer":
        kw = dict(T=shape.T, d=shape.d, f=shape.f, E=shape.E, n_group=shape.n_group,
                  topk_group=shape.topk_group, k=shape.k, n_shared=shape.n_shared,
                  routed_scaling=shape.routed_scaling, tau=shape.tau, n_bins=shape.n_bins,
                  w_dtype=shape.w_dtype, x_dtype=shape.x_dtype, y_dtype=shape.y_dtype)
        kw.update(over)
        return cls(**kw)


def workspace_size(layer: Layer) -> int:
    n = ctypes.c_size_t(0)
    d = layer.desc()
    _check(lib.caee_workspace_size(ctypes.byref(d), ctypes.byref(n)))
    return int(n.value)


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _stream(*tensors) -> Optional[int]:
    import torch
    for t in tensors:
        if t is not None:
            if not t.is_cuda:
                raise ValueError(f"expected a tensor on a GPU, got one on {t.device}")
            # what torch.cuda.current_stream(t.device).cuda_stream returns, without the Stream object (2 us a call)
            return torch._C._cuda_getCurrentRawStream(t.get_device())
    return None


def _weights(w: dict) -> ExpertWeights:
    g = lambda n: _ptr(w.get(n))  # noqa: E731
    return ExpertWeights(g("w13"), g("w2"), g("w13_scale"), g("w2_scale"),
                         g("sh_w13"), g("sh_w2"), g("sh_w13_scale"), g("sh_w2_scale"),
                         int(w.get("layout", LAYOUT_ROWMAJOR)))


def pack_matrix(w_dtype: str, src, dst, rows: int, cols: int, count: int):
    """Repack `count` row-major [rows][cols] matrices into the tiled layout."""
    _check(lib.caee_pack_matrix(DTYPE_CODE[w_dtype], _ptr(src), _ptr(dst), rows, cols, count, _stream(src)))
    return dst


def quantize_rows(src, q, scale):
    """E4M3 codes and per-128-column fp32 scales of a bf16/fp32 [rows][cols] tensor."""
    import torch
    dt = {torch.bfloat16: CAEE_BF16, torch.float32: CAEE_F32}[src.dtype]
    _check(lib.caee_quantize_rows(dt, _ptr(src), src.shape[0], src.shape[1], _ptr(q), _ptr(scale), _stream(src)))
    return q, scale


def pack_weights(weights: dict, w_dtype: str) -> dict:
    """Tiled copy of a row-major expert weight dict (scales are shared)."""
    import torch
    out = {k: v for k, v in weights.items() if k.endswith("_scale")}
    for name in ("w13", "w2", "sh_w13", "sh_w2"):
        src = weights.get(name)
        if src is None:
            continue
        dst = torch.empty_like(src)
        if src.numel():
            pack_matrix(w_dtype, src, dst, src.shape[1], src.shape[2], src.shape[0])
        out[name] = dst
    out["layout"] = LAYOUT_TILED
    return out


def pin_host_weights(weights: dict) -> dict:
    """Page-locked host copies of the routed expert matrices (``w13``, ``w2``)
    of a device weight dict, in its layout: the host side of an offloaded
    layer.  Shared experts stay on the device."""
    import torch
    out = {"layout": int(weights.get("layout", LAYOUT_ROWMAJOR))}
    for name in ("w13", "w2"):
        src = weights[name]
        dst = torch.empty(src.shape, dtype=src.dtype, pin_memory=True)
        dst.copy_(src)
        out[name] = dst
    return out


def alloc_slots(layer: Layer, n_slots: int, device) -> tuple:
    """Device buffers for ``n_slots`` experts of ``layer`` (w13, w2)."""
    import torch
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[layer.w_dtype]
    return (torch.empty((n_slots, 2 * layer.f, layer.d), dtype=dt, device=device),
            torch.empty((n_slots, layer.d, layer.f), dtype=dt, device=device))


def _route_out(out: Optional[dict]) -> Optional[RouteOut]:
    if out is None:
        return None
    g = lambda n: _ptr(out.get(n))  # noqa: E731
    return RouteOut(g("topk_ids"), g("topk_w"), g("orig_ids"), g("masks"), g("stats"), g("bin_loads"))


def alloc_workspace(layer: Layer, device):
    import torch
    return torch.empty(max(workspace_size(layer), 256), dtype=torch.uint8, device=device)


def alloc_route_out(layer: Layer, device, full: bool = True) -> dict:
    """Device buffers for the routing results of ``layer``."""
    import torch
    T, k = layer.T, layer.k
    out = {"topk_ids": torch.empty((T, k), dtype=torch.int32, device=device),
           "topk_w": torch.empty((T, k), dtype=torch.float32, device=device)}
    if full:
        words = (layer.E + 31) // 32
        out["orig_ids"] = torch.empty((T, k), dtype=torch.int32, device=device)
        out["masks"] = torch.empty((4, words), dtype=torch.int32, device=device)
        out["stats"] = torch.empty(STATS, dtype=torch.int32, device=device)
        out["bin_loads"] = torch.empty((3, layer.n_bins), dtype=torch.float64, device=device)
    return out


def route_prune(layer: Layer, logits, bias, cost, bins, out: dict, ws) -> dict:
    d = layer.desc()
    ro = _route_out(out)
    _check(lib.caee_route_prune(ctypes.byref(d), _ptr(logits), _ptr(bias), _ptr(cost), _ptr(bins),
                                ctypes.byref(ro), _ptr(ws), ws.numel(), _stream(logits)))
    return out


def expert_ffn(layer: Layer, x, topk_ids, topk_w, weights: dict, y, ws):
    d = layer.desc()
    w = _weights(weights)
    _check(lib.caee_expert_ffn(ctypes.byref(d), _ptr(x), _ptr(topk_ids), _ptr(topk_w), ctypes.byref(w),
                               _ptr(y), _ptr(ws), ws.numel(), _stream(x)))
    return y


def moe_layer(layer: Layer, x, logits, bias, cost, bins, weights: dict, y, ws, out: Optional[dict] = None):
    d = layer.desc()
    w = _weights(weights)
    ro = _route_out(out)
    _check(lib.caee_moe_layer(ctypes.byref(d), _ptr(x), _ptr(logits), _ptr(bias), _ptr(cost), _ptr(bins),
                              ctypes.byref(w), _ptr(y), None if ro is None else ctypes.byref(ro),
                              _ptr(ws), ws.numel(), _stream(x)))
    return y


SCRATCH_BYTES = 48 << 20   # CAEE_SCRATCH_BYTES: the library's own scratch array per GPU


def moe_layer_noalloc(layer: Layer, x, logits, bias, cost, bins, weights: dict, y, out: Optional[dict] = None):
    """caee_moe_layer_noalloc: the whole layer in the library's scratch array
    (no workspace argument; allocates nothing)."""
    d = layer.desc()
    w = _weights(weights)
    ro = _route_out(out)
    _check(lib.caee_moe_layer_noalloc(ctypes.byref(d), _ptr(x), _ptr(logits), _ptr(bias), _ptr(cost), _ptr(bins),
                                      ctypes.byref(w), _ptr(y), None if ro is None else ctypes.byref(ro),
                                      _stream(x)))
    return y


# ---------------------------------------------------------------------------
# The attention block in front of the layer.

_CODES: dict = {}          # torch dtype -> caee_dtype_t, made by the first call


def _code(t) -> int:
    if not _CODES:
        import torch
        _CODES.update({torch.bfloat16: CAEE_BF16, torch.float32: CAEE_F32, torch.uint8: CAEE_FP8_E4M3,
                       torch.float8_e4m3fn: CAEE_FP8_E4M3})
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"tensor of dtype {t.dtype}: bfloat16, float32 or e4m3 codes (uint8, float8_e4m3fn) are taken")
    return code


def _need(t, name: str, dtype=None, shape=None, dense: bool = True):
    """The argument checks that only the tensors' owner can make: device, dtype, shape, layout."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if dense and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _at(t, name: str, dtype, shape) -> int:
    """Address of a dense device tensor, checked as by ``_need`` (one expression where all is well: a call of a dozen
    tensors is bound by these checks)."""
    if t.is_cuda and t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    return _need(t, name, dtype, shape).data_ptr()


def _workspace(ws) -> tuple:
    """Address and bytes of a workspace."""
    if ws is None:
        return None, 0
    _need(ws, "ws")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def alloc_paged_plan(B: int, T: int, device) -> dict:
    """Device buffers for the plan of B requests and T token entries (caee_paged_plan_out_t)."""
    import torch
    i32 = lambda n: torch.empty(n, dtype=torch.int32, device=device)  # noqa: E731
    return {"cu_new": i32(B + 1), "cu_kv": i32(B + 1), "seq_len": i32(B),
            "slots": torch.empty(T, dtype=torch.int64, device=device), "position": i32(T), "request": i32(T),
            "free_head": i32(1), "lacking": i32(1)}


def paged_plan(block_size: int, ctx_len, new_len, block_table, free_list, free_head, out: dict) -> dict:
    """Pages, slots and positions of a step's new tokens (caee_paged_plan).

    ``ctx_len``/``new_len`` [B] int32: tokens each request has in the cache and receives; ``block_table``
    [B][max_blocks] int32, updated in place; ``free_list`` int32 pages, used from ``free_head[0]`` on; ``out`` as
    made by ``alloc_paged_plan`` (its ``seq_len`` and ``free_head`` are the next call's inputs, whose ``out`` is then
    another one: no output may overlap an input)."""
    import torch
    B, T = ctx_len.shape[0], out["slots"].shape[0]
    i32, per_request, per_token, one = torch.int32, (B,), (T,), (1,)
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError(f"block_table must be [{B}][max_blocks]")
    width, n_free = block_table.shape[1], free_list.shape[0]
    position, request = out.get("position"), out.get("request")
    o = PagedPlanOut(_at(out["cu_new"], "cu_new", i32, (B + 1,)), _at(out["cu_kv"], "cu_kv", i32, (B + 1,)),
                     _at(out["seq_len"], "seq_len", i32, per_request),
                     _at(out["slots"], "slots", torch.int64, per_token),
                     None if position is None else _at(position, "position", i32, per_token),
                     None if request is None else _at(request, "request", i32, per_token),
                     _at(out["free_head"], "free_head", i32, one), _at(out["lacking"], "lacking", i32, one))
    _check(lib.caee_paged_plan(B, T, block_size, width, _at(ctx_len, "ctx_len", i32, per_request),
                               _at(new_len, "new_len", i32, per_request),
                               _at(block_table, "block_table", i32, (B, width)),
                               _at(free_list, "free_list", i32, (n_free,)), n_free,
                               _at(free_head, "free_head", i32, one), ctypes.byref(o), _stream(free_head)))
    return out


def _rows(t, name: str):
    """A 2-D tensor whose rows are dense; its row stride (of a single row, which may be any, the row's length)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (shape[1] > 1 and stride[1] != 1):
        raise ValueError(f"{name} must be 2-D with dense rows")
    return stride[0] if shape[0] > 1 else shape[1]


def latent_store(c, r, slots, cache):
    """Rows [c_t | r_t] of T tokens into ``cache`` [n_blocks][block_size][latent + rope] bf16 at ``slots`` [T] int64
    (caee_latent_store).  ``c`` [T][latent] and ``r`` [T][rope], bf16 or f32, may be slices of wider rows."""
    import torch
    cs, rs = _rows(c, "c"), _rows(r, "r")
    (T, latent), (Tr, rope), pages = c.shape, r.shape, cache.shape
    if c.dtype != r.dtype or Tr != T or len(pages) != 3 or pages[2] != latent + rope:
        raise ValueError("c, r and cache do not fit together")
    _check(lib.caee_latent_store(T, latent, rope, _code(c), c.data_ptr(), cs, r.data_ptr(), rs,
                                 _at(slots, "slots", torch.int64, (T,)), _at(cache, "cache", torch.bfloat16, pages),
                                 pages[0] * pages[1], _stream(cache)))
    return cache


@dataclass
class Latent:
    """Descriptor fields of latent attention that a layer keeps (see caee_latent_desc_t)."""

    heads: int
    nope: int
    rope: int
    latent: int
    v: int
    scale: float
    causal: bool = True
    form: str = "auto"          # "auto" | "absorbed" | "expanded" (caee_latent_form_t)

    def desc(self, T: int, B: int, max_new: int, max_kv: int, block_size: int = 1, n_blocks: int = 1,
             max_blocks: int = 1, q_stride: Optional[int] = None, y_dtype: int = CAEE_BF16) -> LatentDesc:
        qs = self.heads * (self.nope + self.rope) if q_stride is None else q_stride
        return LatentDesc(T, B, self.heads, self.nope, self.rope, self.latent, self.v, block_size, n_blocks,
                          max_blocks, max_new, 1 if self.causal else 0, LATENT_FORM_CODE[self.form], y_dtype, max_kv,
                          qs, self.scale)


def latent_workspace_size(att: Latent, T: int, B: int, max_new: int, max_kv: int) -> int:
    n = ctypes.c_size_t(0)
    d = att.desc(T, B, max_new, max_kv)
    _check(lib.caee_latent_workspace_size(ctypes.byref(d), ctypes.byref(n)))
    return int(n.value)


def alloc_latent_workspace(att: Latent, T: int, B: int, max_new: int, max_kv: int, device):
    import torch
    return torch.empty(max(latent_workspace_size(att, T, B, max_new, max_kv), 256), dtype=torch.uint8, device=device)


def pack_latent_weights(w_uk, w_uv) -> dict:
    """The weight dict of ``latent_attention`` from ``w_uk`` [heads][nope][latent] and ``w_uv`` [heads][v][latent]."""
    return {"w_uk": w_uk.contiguous(), "w_uk_t": w_uk.transpose(1, 2).contiguous(), "w_uv": w_uv.contiguous()}


def latent_attention(att: Latent, q, weights: dict, cache, block_table, plan: dict, y, ws, max_new: int, max_kv: int,
                     lse=None):
    """Latent attention of the new tokens over the paged cache (caee_latent_attention).

    ``q`` [T][heads][nope + rope] bf16 (tokens may be strided); ``weights`` as made by ``pack_latent_weights``;
    ``plan`` with ``cu_new``, ``cu_kv`` and ``seq_len`` as ``paged_plan`` writes them; ``max_new``/``max_kv``: host
    bounds of a request's new tokens and of the sum of ``seq_len``; ``y`` [T][heads][v] bf16 or f32."""
    import torch
    bf, i32, H, R = torch.bfloat16, torch.int32, att.heads, att.latent
    ws_at, ws_bytes = _workspace(ws)
    T, B = q.shape[0], block_table.shape[0]
    _need(q, "q", bf, (T, H, att.nope + att.rope), dense=False)
    if q.stride(2) != 1 or (H > 1 and q.stride(1) != att.nope + att.rope):
        raise ValueError("q must have dense heads")
    if _need(cache, "cache", bf).dim() != 3 or cache.shape[2] != R + att.rope:
        raise ValueError(f"cache must be [n_blocks][block_size][{R + att.rope}]")
    if _need(block_table, "block_table", i32).dim() != 2:
        raise ValueError("block_table must be [B][max_blocks]")
    for name, n in (("cu_new", B + 1), ("cu_kv", B + 1), ("seq_len", B)):
        _need(plan[name], name, i32, (n,))
    for name, shape in (("w_uk", (H, att.nope, R)), ("w_uk_t", (H, R, att.nope)), ("w_uv", (H, att.v, R))):
        if weights.get(name) is not None:
            _need(weights[name], name, bf, shape)
    _need(y, "y", None, (T, H, att.v))
    if lse is not None:
        _need(lse, "lse", torch.float32, (T, H))
    stride = q.stride(0) if T > 1 else H * (att.nope + att.rope)
    d = att.desc(T, B, max_new, max_kv, cache.shape[1], cache.shape[0], block_table.shape[1], stride, _code(y))
    w = LatentWeights(_ptr(weights.get("w_uk")), _ptr(weights.get("w_uk_t")), _ptr(weights.get("w_uv")))
    _check(lib.caee_latent_attention(ctypes.byref(d), _ptr(q), ctypes.byref(w), _ptr(cache), _ptr(block_table),
                                     _ptr(plan["cu_new"]), _ptr(plan["cu_kv"]), _ptr(plan["seq_len"]), _ptr(y),
                                     _ptr(lse), ws_at, ws_bytes, _stream(y)))
    return y


def _block_matmul_desc(x, N: int, y_dtype: int, layout: int, y_stride: int) -> BlockMatmulDesc:
    return BlockMatmulDesc(x.shape[0], N, x.shape[1], _code(x), y_dtype, layout, _rows(x, "x"), y_stride)


def block_matmul_workspace_size(x, N: int) -> int:
    n = ctypes.c_size_t(0)
    d = _block_matmul_desc(x, N, CAEE_F32, LAYOUT_ROWMAJOR, N)
    _check(lib.caee_block_matmul_workspace_size(ctypes.byref(d), ctypes.byref(n)))
    return int(n.value)


def alloc_block_matmul_workspace(x, N: int, device):
    import torch
    return torch.empty(max(block_matmul_workspace_size(x, N), 256), dtype=torch.uint8, device=device)


def block_matmul(x, w, w_scale, y, ws=None, x_scale=None, layout: int = LAYOUT_ROWMAJOR):
    """y = x W^T with e4m3 weights and one fp32 scale per 128x128 block (caee_block_matmul).

    ``x`` [M][K]: bf16 or f32 (quantised in the call) or e4m3 codes with ``x_scale`` [M][K/128]; rows may be strided,
    those of ``y`` [M][N] (bf16 or f32) too.  ``w`` [N][K] codes in ``layout`` order, ``w_scale``
    [ceil(N/128)][K/128].  ``ws`` as made by ``alloc_block_matmul_workspace`` (not needed for codes)."""
    import torch
    ws_at, ws_bytes = _workspace(ws)
    (M, K), N = x.shape, w.shape[0]
    if _code(_need(w, "w", None, (N, K))) != CAEE_FP8_E4M3:
        raise TypeError("w must be e4m3 codes")
    _need(w_scale, "w_scale", torch.float32, ((N + 127) // 128, K // 128))
    if x_scale is not None:
        _need(x_scale, "x_scale", torch.float32, (M, K // 128))
    ys = _rows(y, "y")
    if tuple(y.shape) != (M, N):
        raise ValueError(f"y must have shape {(M, N)}, got {tuple(y.shape)}")
    d = _block_matmul_desc(x, N, _code(y), layout, ys)
    _check(lib.caee_block_matmul(ctypes.byref(d), _ptr(x), _ptr(x_scale), _ptr(w), _ptr(w_scale), _ptr(y), ws_at,
                                 ws_bytes, _stream(y)))
    return y


def timing_enable(on: bool = True):
    _check(lib.caee_timing_enable(1 if on else 0))


def timing_reset():
    _check(lib.caee_timing_reset())


def timing_query(kind: str):
    ms = ctypes.c_double(0)
    n = ctypes.c_int64(0)
    _check(lib.caee_timing_query(KERNEL_KINDS[kind], ctypes.byref(ms), ctypes.byref(n)))
    return float(ms.value), int(n.value)


def lru_step(E: int, n_cache: int, n_stage: int, slot_of, slot_expert, slot_used, call: int, need):
    """One residency plan on host numpy arrays (caee_lru_step); the state
    arrays are updated in place.  Returns (fetch, fetch_slot, counts) with
    counts = (hits, misses, staged, evictions)."""
    import numpy as np
    for a, dt in ((slot_of, np.int32), (slot_expert, np.int32), (slot_used, np.int64)):
        if a.dtype != dt or not a.flags.c_contiguous:
            raise TypeError("state arrays must be contiguous int32/int32/int64")
    need = np.ascontiguousarray(need, dtype=np.uint8)
    fetch = np.zeros(E, np.int32)
    fetch_slot = np.zeros(E, np.int32)
    counts = np.zeros(4, np.int32)
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p)  # noqa: E731
    _check(lib.caee_lru_step(E, n_cache, n_stage, p(slot_of), p(slot_expert), p(slot_used), call, p(need),
                             p(fetch), p(fetch_slot), p(counts)))
    n = int(counts[1])
    return fetch[:n].copy(), fetch_slot[:n].copy(), tuple(int(c) for c in counts)


class Offload:
    """Offload residency handle (caee_offload_t) of one layer.

    ``host_w13``/``host_w2``: per-expert page-locked host tensors (or one
    pinned tensor [E][...] each); ``slot_w13``/``slot_w2``: device tensors
    with ``n_cache + n_stage`` expert slots; ``sh_w13``/``sh_w2``: device
    shared-expert weights (or None).  Every tensor must stay alive while the
    handle is used; the handle keeps references to them."""

    def __init__(self, layer: Layer, host_w13, host_w2, slot_w13, slot_w2, sh_w13, sh_w2, n_cache: int,
                 n_stage: int, miss_cost: float, fetch_batch: int = 4, layout: int = LAYOUT_TILED):
        E = layer.E
        h13 = list(host_w13) if isinstance(host_w13, (list, tuple)) else [host_w13[e] for e in range(E)]
        h2 = list(host_w2) if isinstance(host_w2, (list, tuple)) else [host_w2[e] for e in range(E)]
        if len(h13) != E or len(h2) != E:
            raise ValueError("one host tensor per routed expert is needed")
        self._keep = (host_w13, host_w2, h13, h2, slot_w13, slot_w2, sh_w13, sh_w2)
        self._h13 = (ctypes.c_void_p * E)(*[int(t.data_ptr()) for t in h13])
        self._h2 = (ctypes.c_void_p * E)(*[int(t.data_ptr()) for t in h2])
        self.od = OffloadDesc(ctypes.cast(self._h13, ctypes.POINTER(ctypes.c_void_p)),
                              ctypes.cast(self._h2, ctypes.POINTER(ctypes.c_void_p)),
                              _ptr(slot_w13), _ptr(slot_w2), _ptr(sh_w13), _ptr(sh_w2),
                              int(layout), int(n_cache), int(n_stage), int(fetch_batch), float(miss_cost))
        self.layer = layer
        self.E = E
        d = layer.desc()
        h = ctypes.c_void_p(None)
        _check(lib.caee_offload_create(ctypes.byref(d), ctypes.byref(self.od), ctypes.byref(h)))
        self.handle = h

    def __call__(self, layer: Layer, x, logits, bias, y, ws, out: Optional[dict] = None, copy_stream=None):
        """One layer call.  ``copy_stream``: a torch stream for the host-to-device
        copies (default: a dedicated stream of the handle)."""
        import torch
        if copy_stream is None:
            if getattr(self, "_copy_stream", None) is None:
                self._copy_stream = torch.cuda.Stream(device=x.device)
            copy_stream = self._copy_stream
        d = layer.desc()
        ro = _route_out(out)
        _check(lib.caee_offload_layer(self.handle, ctypes.byref(d), _ptr(x), _ptr(logits), _ptr(bias), _ptr(y),
                                      None if ro is None else ctypes.byref(ro), _ptr(ws), ws.numel(), _stream(x),
                                      int(copy_stream.cuda_stream)))
        return y

    def stats(self) -> dict:
        st = OffloadStats()
        _check(lib.caee_offload_stats(self.handle, ctypes.byref(st)))
        return {n: int(getattr(st, n)) for n, _ in OffloadStats._fields_ if n != "reserved"}

    def residency(self):
        import numpy as np
        a = np.zeros(self.E, np.int32)
        _check(lib.caee_offload_residency(self.handle, a.ctypes.data_as(ctypes.c_void_p)))
        return a

    def reset(self):
        _check(lib.caee_offload_reset(self.handle))

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            lib.caee_offload_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
