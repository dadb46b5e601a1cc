"""Python binding of libsnls.so (the C ABI declared in include/snls.h).

Argument marshalling only: torch supplies device memory and the current HIP
stream; every step of the computation runs in the library's HIP kernels.
There is no CPU fallback -- if libsnls.so is missing or fails to load, every
call raises.

Functions carry the C names: snls_search, snls_topk, snls_aggregate,
snls_backward, snls_aggregate_stacked, snls_chain_flows, snls_aggregate_static,
snls_gather_stacked, snls_stacked_reduce, snls_gather_reduce, snls_bias,
snls_bias_backward, snls_backward_scores, snls_cache_store, snls_cache_attend,
snls_cache_attend_points, snls_norm, snls_norm_backward, snls_dropout,
snls_rotate, snls_rotate_points, snls_project_pack, snls_project,
snls_workspace_size, snls_norm_workspace_size, snls_status_string,
snls_abi_version.
Parameters are plain dicts with keys B, T, C, H, W, HD, ws, wt, ps, stride0,
stride1, k, dist_type (see ``params_from_dict``); the position bias's with keys
radius and edges (a list), a cache's with keys B, slots, C, H, W, HD, block, the
rotary positions' with keys B, T, C, H, W, HD, pairs and theta (three numbers
each) and, where they are not 0, interleaved, row0, col0.
A cache is the tuple (k_codes, k_scales, v_codes, v_scales) that ``cache_alloc``
returns.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsnls.so")

SNLS_OK, SNLS_ERR_INVALID_ARG, SNLS_ERR_UNSUPPORTED, SNLS_ERR_HIP, SNLS_ERR_WORKSPACE, SNLS_ERR_SCRATCH = range(6)
SNLS_DIST_PROD, SNLS_DIST_L2 = 0, 1
SNLS_OP_SEARCH, SNLS_OP_AGGREGATE, SNLS_OP_BACKWARD, SNLS_OP_AGGREGATE_STACKED = 0, 1, 2, 3
SNLS_OP_GATHER_STACKED, SNLS_OP_GATHER_REDUCE = 4, 5
SNLS_OP_BIAS_BACKWARD = 6
SNLS_MAX_K = 128
SNLS_BIAS_MAX_EDGES, SNLS_BIAS_MAX_BUCKETS = 16, 4096
SNLS_STATIC_SCRATCH_BYTES = 64 << 20
SNLS_ROTATE_MAX_PAIRS, SNLS_PROJECT_MAX_CIN = 128, 1024
SYMBOLS = ("snls_search", "snls_topk", "snls_aggregate", "snls_backward", "snls_workspace_size",
           "snls_status_string", "snls_abi_version", "snls_aggregate_stacked", "snls_chain_flows",
           "snls_aggregate_static", "snls_gather_stacked", "snls_stacked_reduce", "snls_gather_reduce",
           "snls_bias", "snls_bias_backward", "snls_backward_scores", "snls_cache_store", "snls_cache_attend",
           "snls_cache_attend_points", "snls_norm", "snls_norm_backward", "snls_norm_workspace_size", "snls_dropout",
           "snls_rotate", "snls_rotate_points", "snls_project_pack", "snls_project")


class SnlsParams(ctypes.Structure):
    """Mirror of the C struct snls_params."""
    _fields_ = [("struct_size", ctypes.c_uint32)] + [
        (n, ctypes.c_int32) for n in ("B", "T", "C", "H", "W", "HD", "ws", "wt", "ps", "stride0")
    ] + [("stride1", ctypes.c_float), ("k", ctypes.c_int32), ("dist_type", ctypes.c_int32)]


class SnlsBiasParams(ctypes.Structure):
    """Mirror of the C struct snls_bias_params."""
    _fields_ = [("struct_size", ctypes.c_uint32), ("radius", ctypes.c_int32), ("n_edges", ctypes.c_int32),
                ("edges", ctypes.c_float * SNLS_BIAS_MAX_EDGES)]


class SnlsCacheParams(ctypes.Structure):
    """Mirror of the C struct snls_cache_params."""
    _fields_ = [("struct_size", ctypes.c_uint32)] + [
        (n, ctypes.c_int32) for n in ("B", "slots", "C", "H", "W", "HD", "block")]


class SnlsNormParams(ctypes.Structure):
    """Mirror of the C struct snls_norm_params."""
    _fields_ = [("struct_size", ctypes.c_uint32), ("C", ctypes.c_int32), ("frames", ctypes.c_int64),
                ("pixels", ctypes.c_int64), ("eps", ctypes.c_float), ("drop", ctypes.c_float),
                ("site", ctypes.c_uint32)]


class SnlsRotateParams(ctypes.Structure):
    """Mirror of the C struct snls_rotate_params."""
    _fields_ = [("struct_size", ctypes.c_uint32)] + [
        (n, ctypes.c_int32) for n in ("B", "T", "C", "H", "W", "HD")
    ] + [("pairs", ctypes.c_int32 * 3), ("theta", ctypes.c_float * 3)] + [
        (n, ctypes.c_int32) for n in ("interleaved", "row0", "col0")]


class SnlsProjectParams(ctypes.Structure):
    """Mirror of the C struct snls_project_params."""
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in ("cin", "cout", "parts")] + [
        ("frames", ctypes.c_int64), ("pixels", ctypes.c_int64)]


class SnlsError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__("%s failed: %s (status %d)" % (where, snls_status_string(status), status))
        self.status = status


_lib = None


def load_library():
    """Load libsnls.so once (after torch, so both share one HIP runtime)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libsnls.so is not built (%s); run python -m paper_2309_16849_amd.build" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        P, F32, I32, I64, SZ = ctypes.c_void_p, ctypes.c_float, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        PP = ctypes.POINTER(SnlsParams)
        lib.snls_search.argtypes = [P, P, P, PP, P, P, P, SZ, P]
        lib.snls_topk.argtypes = [P, P, I64, I32, I32, I32, P, P, P]
        lib.snls_aggregate.argtypes = [P, P, P, PP, F32, P, P, SZ, P]
        lib.snls_backward.argtypes = [P] * 8 + [PP, F32, P, P, P, P, P, SZ, P]
        lib.snls_aggregate_stacked.argtypes = [P, P, P, PP, F32, P, P, SZ, P]
        lib.snls_chain_flows.argtypes = [P, P, I32, I32, I32, I32, I32, P, P]
        lib.snls_aggregate_static.argtypes = [P, P, P, PP, F32, P, P]
        lib.snls_gather_stacked.argtypes = [P, P, P, PP, P, P, SZ, P]
        lib.snls_stacked_reduce.argtypes = [P, P, PP, I32, P, P]
        lib.snls_gather_reduce.argtypes = [P, P, P, P, PP, I32, P, P, SZ, P]
        PB, PC = ctypes.POINTER(SnlsBiasParams), ctypes.POINTER(SnlsCacheParams)
        lib.snls_bias.argtypes = [P, P, P, PP, PB, P, P]
        lib.snls_bias_backward.argtypes = [P, P, P, PP, PB, P, P, SZ, P]
        lib.snls_backward_scores.argtypes = [P] * 8 + [PP, F32, P, P, P, P, P, P, SZ, P]
        lib.snls_cache_store.argtypes = [P, P, P, PC, P, P, P, P, P]
        lib.snls_cache_attend.argtypes = [P] * 8 + [PC, PB, I32, F32, P, P]
        lib.snls_cache_attend_points.argtypes = [P, P, I64] + [P] * 7 + [PC, PB, I32, F32, P, P]
        PN, PR, PJ = (ctypes.POINTER(c) for c in (SnlsNormParams, SnlsRotateParams, SnlsProjectParams))
        lib.snls_norm.argtypes = [P] * 5 + [PN, P, P, P, P]
        lib.snls_norm_backward.argtypes = [P] * 6 + [PN, P, P, P, P, P, SZ, P]
        lib.snls_norm_workspace_size.argtypes = [PN]
        lib.snls_norm_workspace_size.restype = SZ
        lib.snls_dropout.argtypes = [P, P, P, I64, F32, ctypes.c_uint32, P, P]
        lib.snls_rotate.argtypes = [P, P, P, PR, I32, P, P, P]
        lib.snls_rotate_points.argtypes = [P, P, I64, P, PR, I32, P, P]
        lib.snls_project_pack.argtypes = [P, PJ, P, P, P]
        lib.snls_project.argtypes = [P, P, P, P, PJ, P, P]
        lib.snls_workspace_size.argtypes = [ctypes.c_int, PP]
        lib.snls_workspace_size.restype = SZ
        lib.snls_status_string.argtypes = [ctypes.c_int]
        lib.snls_status_string.restype = ctypes.c_char_p
        lib.snls_abi_version.argtypes = []
        for f in ("snls_search", "snls_topk", "snls_aggregate", "snls_backward", "snls_abi_version",
                  "snls_aggregate_stacked", "snls_chain_flows", "snls_aggregate_static", "snls_gather_stacked",
                  "snls_stacked_reduce", "snls_gather_reduce", "snls_bias", "snls_bias_backward",
                  "snls_backward_scores", "snls_cache_store", "snls_cache_attend", "snls_cache_attend_points",
                  "snls_norm", "snls_norm_backward", "snls_dropout", "snls_rotate", "snls_rotate_points",
                  "snls_project_pack", "snls_project"):
            getattr(lib, f).restype = ctypes.c_int
        _lib = lib
    return _lib


_PARAMS_SIZE = ctypes.sizeof(SnlsParams)


def params_from_dict(p: dict) -> SnlsParams:
    return SnlsParams(_PARAMS_SIZE, int(p["B"]), int(p["T"]), int(p["C"]), int(p["H"]), int(p["W"]), int(p["HD"]),
                      int(p["ws"]), int(p["wt"]), int(p["ps"]), int(p["stride0"]), float(p["stride1"]), int(p["k"]),
                      int(p["dist_type"]))


def grid(p: dict):
    return (p["H"] - 1) // p["stride0"] + 1, (p["W"] - 1) // p["stride0"] + 1


def n_cand(p: dict) -> int:
    return (2 * p["wt"] + 1) * p["ws"] ** 2


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _dev(t, name, shape=None):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
        raise ValueError("%s must be a contiguous float32 tensor on the GPU" % name)
    if shape is not None and t.shape != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    return t


def _room(workspace):
    """Address and bytes of a workspace, a contiguous tensor of any type on the GPU."""
    if not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous tensor on the GPU")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _new(shape, like, stream):
    """An output beside tensor like; a call on another stream than the current one keeps its memory until that is done."""
    t = torch.empty(shape, device=like.device, dtype=torch.float32)
    if stream is not None:
        t.record_stream(stream)
    return t


def _like(t, given, name, stream):
    """An output of t's shape: the given one, or a new one as by _new."""
    if given is not None:
        return _dev(given, name, t.shape)
    new = torch.empty_like(t)
    if stream is not None:
        new.record_stream(stream)
    return new


# the current stream's handle without a Stream object around it (3 us a call)
_current_raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None and _current_raw is not None:
        return _current_raw(torch.cuda.current_device())
    return (stream if stream is not None else torch.cuda.current_stream()).cuda_stream


def _check(status, where):
    if status != SNLS_OK:
        raise SnlsError(status, where)


def snls_status_string(status: int) -> str:
    return load_library().snls_status_string(int(status)).decode()


def snls_abi_version() -> int:
    return load_library().snls_abi_version()


def snls_workspace_size(op: int, p: dict) -> int:
    prm = params_from_dict(p)
    return load_library().snls_workspace_size(op, ctypes.byref(prm))


def video_shape(p: dict):
    return (p["B"], p["T"], p["C"], p["H"], p["W"])


def flow_shape(p: dict):
    return (p["B"], p["T"], 2 * p["wt"], 2, p["H"], p["W"])


def out_shape(p: dict):
    nH, nW = grid(p)
    kk = p["k"] if p["k"] > 0 else n_cand(p)
    return (p["B"], p["HD"], p["T"], nH, nW, kk)


def snls_search(q, k, flows, p: dict, dists=None, inds=None, workspace=None, stream=None):
    """Shifted non-local search; returns (dists, inds) (see include/snls.h).
    The workspace is allocated here when not given (its size may be 0)."""
    lib = load_library()
    _dev(q, "q", video_shape(p))
    _dev(k, "k", video_shape(p))
    if p["wt"] > 0 or flows is not None:
        _dev(flows, "flows", flow_shape(p))
    shp = out_shape(p)
    if dists is None:
        dists = _new(shp, q, stream)
    if inds is None:
        inds = _new(shp + (3,), q, stream)
    _dev(dists, "dists", shp)
    _dev(inds, "inds", shp + (3,))
    if workspace is None:
        workspace = workspace_for(SNLS_OP_SEARCH, p, q.device, stream)
    prm = params_from_dict(p)
    _check(lib.snls_search(_ptr(q), _ptr(k), _ptr(flows), ctypes.byref(prm), _ptr(dists), _ptr(inds),
                           *_room(workspace), _stream(stream)), "snls_search")
    return dists, inds


def snls_topk(dists_all, inds_all, k: int, dist_type: int, dists=None, inds=None, stream=None):
    """top-k of rows of candidate scores; dists_all (..., n_cand), inds_all (..., n_cand, 3)."""
    lib = load_library()
    _dev(dists_all, "dists_all")
    n_c = dists_all.shape[-1]
    lead = tuple(dists_all.shape[:-1])
    _dev(inds_all, "inds_all", lead + (n_c, 3))
    rows = dists_all.numel() // max(n_c, 1)
    if dists is None:
        dists = _new(lead + (k,), dists_all, stream)
    if inds is None:
        inds = _new(lead + (k, 3), dists_all, stream)
    _dev(dists, "dists", lead + (k,))
    _dev(inds, "inds", lead + (k, 3))
    _check(lib.snls_topk(_ptr(dists_all), _ptr(inds_all), rows, n_c, k, dist_type, _ptr(dists), _ptr(inds),
                         _stream(stream)), "snls_topk")
    return dists, inds


def workspace_for(op: int, p: dict, device, stream=None):
    """A device buffer of snls_workspace_size(op, p) bytes (torch allocations are 256-byte aligned), for calls on
    stream (default: the current one): its memory goes to other work of that stream only."""
    need = snls_workspace_size(op, p)
    if need == ctypes.c_size_t(-1).value:
        raise SnlsError(SNLS_ERR_INVALID_ARG, "snls_workspace_size")
    with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
        return torch.empty(max((need + 3) // 4, 1), device=device, dtype=torch.float32)


def snls_aggregate(v, dists, inds, p: dict, scale: float = 1.0, out=None, workspace=None, stream=None):
    """Softmax-weighted patch aggregation; returns out (B,T,C,H,W)."""
    lib = load_library()
    _dev(v, "v", video_shape(p))
    shp = out_shape(p)
    _dev(dists, "dists", shp)
    _dev(inds, "inds", shp + (3,))
    if out is None:
        out = _new(video_shape(p), v, stream)
    _dev(out, "out", video_shape(p))
    if workspace is None:
        workspace = workspace_for(SNLS_OP_AGGREGATE, p, v.device, stream)
    prm = params_from_dict(p)
    _check(lib.snls_aggregate(_ptr(v), _ptr(dists), _ptr(inds), ctypes.byref(prm), float(scale), _ptr(out),
                              *_room(workspace), _stream(stream)), "snls_aggregate")
    return out


def snls_aggregate_static(v, dists, inds, p: dict, scale: float = 1.0, out=None, stream=None):
    """snls_aggregate with the library's static scratch array as workspace
    (nothing allocated on the device beyond ``out`` when it is not given)."""
    lib = load_library()
    _dev(v, "v", video_shape(p))
    shp = out_shape(p)
    _dev(dists, "dists", shp)
    _dev(inds, "inds", shp + (3,))
    if out is None:
        out = _new(video_shape(p), v, stream)
    _dev(out, "out", video_shape(p))
    prm = params_from_dict(p)
    _check(lib.snls_aggregate_static(_ptr(v), _ptr(dists), _ptr(inds), ctypes.byref(prm), float(scale), _ptr(out),
                                     _stream(stream)), "snls_aggregate_static")
    return out


def snls_backward(q, k, v, flows, dists, inds, grad_out, p: dict, scale: float = 1.0, grad_dists=None,
                  workspace=None, stream=None):
    """Gradients (grad_q, grad_k, grad_v, grad_flows) of search + aggregation."""
    lib = load_library()
    vs, shp = video_shape(p), out_shape(p)
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (grad_out, "grad_out")):
        _dev(t, n, vs)
    _dev(dists, "dists", shp)
    _dev(inds, "inds", shp + (3,))
    if grad_dists is not None:
        _dev(grad_dists, "grad_dists", shp)
    if p["wt"] > 0 or flows is not None:
        _dev(flows, "flows", flow_shape(p))
    gq, gk, gv = (_new(vs, q, stream) for _ in range(3))
    gf = _new(flow_shape(p), q, stream)
    if workspace is None:
        workspace = workspace_for(SNLS_OP_BACKWARD, p, q.device, stream)
    prm = params_from_dict(p)
    _check(lib.snls_backward(_ptr(q), _ptr(k), _ptr(v), _ptr(flows), _ptr(dists), _ptr(inds), _ptr(grad_out),
                             _ptr(grad_dists), ctypes.byref(prm), float(scale), _ptr(gq), _ptr(gk), _ptr(gv),
                             _ptr(gf), *_room(workspace), _stream(stream)), "snls_backward")
    return gq, gk, gv, gf


def snls_aggregate_stacked(v, dists, inds, p: dict, scale: float = 1.0, stacked=None, workspace=None, stream=None):
    """Aggregation with the k neighbours kept apart; returns (B, HD, k, T, C/HD, H, W)."""
    lib = load_library()
    _dev(v, "v", video_shape(p))
    shp = out_shape(p)
    _dev(dists, "dists", shp)
    _dev(inds, "inds", shp + (3,))
    st_shape = (p["B"], p["HD"], p["k"], p["T"], p["C"] // p["HD"], p["H"], p["W"])
    if stacked is None:
        stacked = _new(st_shape, v, stream)
    _dev(stacked, "stacked", st_shape)
    if workspace is None:
        workspace = workspace_for(SNLS_OP_AGGREGATE_STACKED, p, v.device, stream)
    prm = params_from_dict(p)
    _check(lib.snls_aggregate_stacked(_ptr(v), _ptr(dists), _ptr(inds), ctypes.byref(prm), float(scale),
                                      _ptr(stacked), *_room(workspace), _stream(stream)),
           "snls_aggregate_stacked")
    return stacked


def snls_chain_flows(fflow, bflow, wt: int, flows=None, stream=None):
    """Window offsets (B, T, 2wt, 2, H, W) composed from one-step flows (B, T, 2, H, W)."""
    lib = load_library()
    _dev(fflow, "fflow")
    B, T, two, H, W = fflow.shape
    if two != 2:
        raise ValueError("fflow must be (B, T, 2, H, W)")
    _dev(bflow, "bflow", tuple(fflow.shape))
    if flows is None:
        flows = _new((B, T, 2 * wt, 2, H, W), fflow, stream)
    _dev(flows, "flows", (B, T, 2 * wt, 2, H, W))
    _check(lib.snls_chain_flows(_ptr(fflow), _ptr(bflow), B, T, H, W, int(wt), _ptr(flows), _stream(stream)),
           "snls_chain_flows")
    return flows


def stacked_shape(p: dict):
    return (p["B"], p["HD"], p["k"], p["T"], p["C"] // p["HD"], p["H"], p["W"])


def snls_gather_stacked(v, weights, inds, p: dict, stacked=None, workspace=None, stream=None):
    """The example's gather with caller weights; returns (B, HD, k, T, C/HD, H, W)."""
    lib = load_library()
    _dev(v, "v", video_shape(p))
    shp = out_shape(p)
    _dev(weights, "weights", shp)
    _dev(inds, "inds", shp + (3,))
    if stacked is None:
        stacked = _new(stacked_shape(p), v, stream)
    _dev(stacked, "stacked", stacked_shape(p))
    if workspace is None:
        workspace = workspace_for(SNLS_OP_GATHER_STACKED, p, v.device, stream)
    prm = params_from_dict(p)
    _check(lib.snls_gather_stacked(_ptr(v), _ptr(weights), _ptr(inds), ctypes.byref(prm), _ptr(stacked),
                                   *_room(workspace), _stream(stream)), "snls_gather_stacked")
    return stacked


def snls_stacked_reduce(stacked, proj, p: dict, out=None, stream=None):
    """Reduction over the k neighbours with kernel proj (Cout, C, k); returns (B, T, Cout, H, W)."""
    lib = load_library()
    _dev(stacked, "stacked", stacked_shape(p))
    _dev(proj, "proj")
    cout = proj.shape[0]
    if tuple(proj.shape) != (cout, p["C"], p["k"]):
        raise ValueError("proj must be (Cout, C, k)")
    if out is None:
        out = _new((p["B"], p["T"], cout, p["H"], p["W"]), stacked, stream)
    _dev(out, "out", (p["B"], p["T"], cout, p["H"], p["W"]))
    prm = params_from_dict(p)
    _check(lib.snls_stacked_reduce(_ptr(stacked), _ptr(proj), ctypes.byref(prm), cout, _ptr(out), _stream(stream)),
           "snls_stacked_reduce")
    return out


def snls_gather_reduce(v, weights, inds, proj, p: dict, out=None, workspace=None, stream=None):
    """Gather with caller weights and reduction over the k neighbours in one pass; returns (B, T, Cout, H, W)."""
    lib = load_library()
    _dev(v, "v", video_shape(p))
    shp = out_shape(p)
    _dev(weights, "weights", shp)
    _dev(inds, "inds", shp + (3,))
    _dev(proj, "proj")
    cout = proj.shape[0]
    if tuple(proj.shape) != (cout, p["C"], p["k"]):
        raise ValueError("proj must be (Cout, C, k)")
    if out is None:
        out = _new((p["B"], p["T"], cout, p["H"], p["W"]), v, stream)
    _dev(out, "out", (p["B"], p["T"], cout, p["H"], p["W"]))
    if workspace is None:
        workspace = workspace_for(SNLS_OP_GATHER_REDUCE, p, v.device, stream)
    prm = params_from_dict(p)
    _check(lib.snls_gather_reduce(_ptr(v), _ptr(weights), _ptr(inds), _ptr(proj), ctypes.byref(prm), cout, _ptr(out),
                                  *_room(workspace), _stream(stream)), "snls_gather_reduce")
    return out


# ------------------------------------------------------- learned position bias --

_BIAS_SIZE, _Edges = ctypes.sizeof(SnlsBiasParams), ctypes.c_float * SNLS_BIAS_MAX_EDGES


def bias_from_dict(bias: dict) -> SnlsBiasParams:
    edges = bias["edges"]  # (a list longer than the library takes is refused there)
    return SnlsBiasParams(_BIAS_SIZE, int(bias["radius"]), len(edges), _Edges(*edges[:SNLS_BIAS_MAX_EDGES]))


def bias_table_shape(bias: dict, heads: int):
    nb = 2 * len(bias["edges"]) + 1
    return (heads, 2 * bias["radius"] + 1, nb, nb)


def _here(*tensors):
    """Every given tensor is on the current device, where the call will run."""
    cur = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != cur:
            raise ValueError("tensors are on %s, the current device is cuda:%d" % (t.device, cur))


def snls_bias(dists, inds, table, p: dict, bias: dict, out=None, stream=None):
    """Scores plus the learned bias of their position; out may be dists."""
    lib = load_library()
    shp = out_shape(p)
    _dev(dists, "dists", shp)
    _dev(inds, "inds", shp + (3,))
    _dev(table, "table", bias_table_shape(bias, p["HD"]))
    if out is None:
        out = _new(shp, dists, stream)
    _dev(out, "out", shp)
    _here(dists, inds, table, out)
    prm, bprm = params_from_dict(p), bias_from_dict(bias)
    _check(lib.snls_bias(_ptr(dists), _ptr(inds), _ptr(table), ctypes.byref(prm), ctypes.byref(bprm), _ptr(out),
                         _stream(stream)), "snls_bias")
    return out


def snls_bias_backward(grad_scores, dists, inds, p: dict, bias: dict, grad_table=None, workspace=None, stream=None):
    """Gradient of the bias table from the gradient of the (biased) scores."""
    lib = load_library()
    shp = out_shape(p)
    _dev(grad_scores, "grad_scores", shp)
    _dev(dists, "dists", shp)
    _dev(inds, "inds", shp + (3,))
    if grad_table is None:
        grad_table = _new(bias_table_shape(bias, p["HD"]), dists, stream)
    _dev(grad_table, "grad_table", bias_table_shape(bias, p["HD"]))
    if workspace is None:
        workspace = workspace_for(SNLS_OP_BIAS_BACKWARD, p, dists.device, stream)
    _here(grad_scores, dists, inds, grad_table, workspace)
    prm, bprm = params_from_dict(p), bias_from_dict(bias)
    _check(lib.snls_bias_backward(_ptr(grad_scores), _ptr(dists), _ptr(inds), ctypes.byref(prm), ctypes.byref(bprm),
                                  _ptr(grad_table), *_room(workspace), _stream(stream)),
           "snls_bias_backward")
    return grad_table


def snls_backward_scores(q, k, v, flows, dists, inds, grad_out, p: dict, scale: float = 1.0, grad_dists=None,
                         workspace=None, stream=None):
    """snls_backward's gradients and that of the scores: (grad_q, grad_k, grad_v, grad_flows, grad_scores)."""
    lib = load_library()
    vs, shp = video_shape(p), out_shape(p)
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (grad_out, "grad_out")):
        _dev(t, n, vs)
    _dev(dists, "dists", shp)
    _dev(inds, "inds", shp + (3,))
    if grad_dists is not None:
        _dev(grad_dists, "grad_dists", shp)
    if p["wt"] > 0 or flows is not None:
        _dev(flows, "flows", flow_shape(p))
    gq, gk, gv = (_new(vs, q, stream) for _ in range(3))
    gf = _new(flow_shape(p), q, stream)
    gs = _new(shp, q, stream)
    if workspace is None:
        workspace = workspace_for(SNLS_OP_BACKWARD, p, q.device, stream)
    _here(q, k, v, dists, inds, grad_out, grad_dists, flows, workspace)
    prm = params_from_dict(p)
    _check(lib.snls_backward_scores(_ptr(q), _ptr(k), _ptr(v), _ptr(flows), _ptr(dists), _ptr(inds), _ptr(grad_out),
                                    _ptr(grad_dists), ctypes.byref(prm), float(scale), _ptr(gq), _ptr(gk), _ptr(gv),
                                    _ptr(gf), _ptr(gs), *_room(workspace), _stream(stream)),
           "snls_backward_scores")
    return gq, gk, gv, gf, gs


# ------------------------------------------------------- frames held in 8 bits --

_CACHE_SIZE = ctypes.sizeof(SnlsCacheParams)


def cache_from_dict(cp: dict) -> SnlsCacheParams:
    return SnlsCacheParams(_CACHE_SIZE, int(cp["B"]), int(cp["slots"]), int(cp["C"]), int(cp["H"]), int(cp["W"]),
                           int(cp["HD"]), int(cp["block"]))


def cache_shapes(cp: dict):
    """Shapes of a cache's codes and of its scales."""
    padded = (cp["C"] // cp["HD"] + 15) // 16 * 16
    lead = (cp["B"], cp["slots"], cp["HD"])
    return lead + (cp["H"], cp["W"], padded), lead + (-(-cp["H"] // cp["block"]), -(-cp["W"] // cp["block"]))


def cache_alloc(cp: dict, device):
    """The four buffers of an empty cache: (k_codes, k_scales, v_codes, v_scales)."""
    codes, scales = cache_shapes(cp)

    def one():
        return (torch.zeros(codes, device=device, dtype=torch.uint8).view(torch.float8_e4m3fn),
                torch.ones(scales, device=device, dtype=torch.float32))

    return one() + one()


def _dev_as(t, name, shape, dtypes):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.is_contiguous()):
        raise ValueError("%s must be a contiguous tensor of %s on the GPU" % (name, " or ".join(map(str, dtypes))))
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    return t


def _cache_ptrs(cache, cp):
    codes, scales = cache_shapes(cp)
    if len(cache) != 4:
        raise ValueError("a cache is (k_codes, k_scales, v_codes, v_scales)")
    for t, n in ((cache[0], "k_codes"), (cache[2], "v_codes")):
        _dev_as(t, n, codes, (torch.float8_e4m3fn, torch.uint8))
    _dev(cache[1], "k_scales", scales)
    _dev(cache[3], "v_scales", scales)
    return tuple(_ptr(t) for t in cache)


def snls_cache_store(k, v, slots, cp: dict, cache, stream=None):
    """One frame of keys and values (B, C, H, W) into the cache's slots (int32, one a video); returns the cache."""
    lib = load_library()
    shp = (cp["B"], cp["C"], cp["H"], cp["W"])
    _dev(k, "k", shp)
    _dev(v, "v", shp)
    _dev_as(slots, "slots", (cp["B"],), (torch.int32,))
    ptrs = _cache_ptrs(cache, cp)
    _here(k, v, slots, *cache)
    prm = cache_from_dict(cp)
    _check(lib.snls_cache_store(_ptr(k), _ptr(v), _ptr(slots), ctypes.byref(prm), *ptrs, _stream(stream)),
           "snls_cache_store")
    return cache


def _attend_common(cp, ages, cache, table, bias):
    _dev_as(ages, "ages", (cp["B"], cp["slots"]), (torch.int32,))
    if (table is None) != (bias is None):
        raise ValueError("table and bias go together")
    if table is not None:
        _dev(table, "table", bias_table_shape(bias, cp["HD"]))
    return _cache_ptrs(cache, cp), ctypes.byref(bias_from_dict(bias)) if bias is not None else None


def snls_cache_attend(q, flows, ages, cache, cp: dict, ws: int, scale: float = 1.0, table=None, bias=None, out=None,
                      stream=None):
    """Every pixel of a frame q (B, C, H, W) attends its shifted windows in all cached frames; returns (B, C, H, W).
    flows (B, slots, 2, H, W) or None; ages int32 (B, slots), negative for a slot that holds no frame."""
    lib = load_library()
    shp = (cp["B"], cp["C"], cp["H"], cp["W"])
    _dev(q, "q", shp)
    if flows is not None:
        _dev(flows, "flows", (cp["B"], cp["slots"], 2, cp["H"], cp["W"]))
    ptrs, bp = _attend_common(cp, ages, cache, table, bias)
    if out is None:
        out = _new(shp, q, stream)
    _dev(out, "out", shp)
    _here(q, flows, ages, table, out, *cache)
    prm = cache_from_dict(cp)
    _check(lib.snls_cache_attend(_ptr(q), _ptr(flows), _ptr(ages), *ptrs, _ptr(table), ctypes.byref(prm), bp, int(ws),
                                 float(scale), _ptr(out), _stream(stream)), "snls_cache_attend")
    return out


def snls_cache_attend_points(q, points, flows, ages, cache, cp: dict, ws: int, scale: float = 1.0, table=None,
                             bias=None, out=None, stream=None):
    """Single pixels attend the cached frames: q (n, C), points int32 (n, 3) = video, row, column, flows
    (n, slots, 2) or None; returns (n, C)."""
    lib = load_library()
    _dev(q, "q")
    n = q.shape[0]
    _dev(q, "q", (n, cp["C"]))
    _dev_as(points, "points", (n, 3), (torch.int32,))
    if flows is not None:
        _dev(flows, "flows", (n, cp["slots"], 2))
    ptrs, bp = _attend_common(cp, ages, cache, table, bias)
    if out is None:
        out = _new((n, cp["C"]), q, stream)
    _dev(out, "out", (n, cp["C"]))
    if n == 0:
        return out
    _here(q, points, flows, ages, table, out, *cache)
    prm = cache_from_dict(cp)
    _check(lib.snls_cache_attend_points(_ptr(q), _ptr(points), n, _ptr(flows), _ptr(ages), *ptrs, _ptr(table),
                                        ctypes.byref(prm), bp, int(ws), float(scale), _ptr(out), _stream(stream)),
           "snls_cache_attend_points")
    return out


# ------------------------------------------------- norm, dropout, around a layer --

_NORM_SIZE = ctypes.sizeof(SnlsNormParams)


def _features(t, name):
    """frames, C, pixels of features (..., C, H, W), or of n tokens (n, C), and the shape of a value a pixel."""
    _dev(t, name)
    s = t.shape
    if len(s) == 2:
        return s[0], s[1], 1, (s[0],)
    if len(s) < 3:
        raise ValueError("%s must be (..., C, H, W) or (n, C)" % name)
    frames = 1
    for n in s[:-3]:
        frames *= n
    return frames, s[-3], s[-2] * s[-1], tuple(s[:-3]) + tuple(s[-2:])


def dropout_site(site: int) -> int:
    """A dropout's number; a C field would take it modulo 2^32, and two sites share a mask."""
    site = int(site)
    if not 0 <= site < 1 << 32:
        raise ValueError("site must be a whole number of 32 bits, got %d" % site)
    return site


_MOST = (1 << 31) - 1  # channels beyond stay more than the library takes


def norm_params(C: int, frames: int, pixels: int, eps: float, drop: float, site: int) -> SnlsNormParams:
    return SnlsNormParams(_NORM_SIZE, min(C, _MOST), frames, pixels, float(eps), float(drop), dropout_site(site))


def _per_channel(C, **tensors):
    for n, t in tensors.items():
        if t is not None:
            _dev(t, n, (C,))


def _rng(rng, drop):
    """Address of a generator's state, a tensor of two int64: seed and step."""
    if rng is None:
        if drop > 0:
            raise ValueError("dropout needs rng, a tensor of two int64 (seed, step)")
        return None
    return _dev_as(rng, "rng", (2,), (torch.int64, torch.uint64)).data_ptr()


def snls_norm(x, gamma=None, beta=None, eps: float = 1e-5, branch=None, drop: float = 0.0, rng=None, site: int = 0,
              y=None, total=None, stats=None, stream=None):
    """Layer norm over the channels of features (..., C, H, W) or tokens (n, C), of x or of the residual sum
    x + dropout(branch); returns (y, total, stats), total being x without branch.  rng: two int64 on the GPU, seed
    and step."""
    lib = load_library()
    frames, C, pixels, px = _features(x, "x")
    _per_channel(C, gamma=gamma, beta=beta)
    if branch is not None:
        _dev(branch, "branch", x.shape)
        total = _like(x, total, "total", stream)
    elif total is not None:
        raise ValueError("total goes with branch")
    y = _like(x, y, "y", stream)
    stats = _dev(stats, "stats", (2,) + px) if stats is not None else _new((2,) + px, x, stream)
    _here(x, gamma, beta, branch, rng, y, total, stats)
    prm = norm_params(C, frames, pixels or 1, eps, drop, site)
    if pixels:
        _check(lib.snls_norm(_ptr(x), _ptr(branch), _rng(rng, drop), _ptr(gamma), _ptr(beta), ctypes.byref(prm),
                             _ptr(total), _ptr(y), _ptr(stats), _stream(stream)), "snls_norm")
    return y, x if branch is None else total, stats


def snls_norm_backward(grad_y, total, stats, gamma=None, grad_total=None, drop: float = 0.0, rng=None, site: int = 0,
                       weights: bool = True, grad_x=None, grad_branch=None, workspace=None, stream=None):
    """Gradients of snls_norm: (grad_x, grad_branch, grad_gamma, grad_beta); grad_branch is grad_x when nothing is
    dropped, the last two are None for weights=False."""
    lib = load_library()
    frames, C, pixels, px = _features(total, "total")
    _dev(grad_y, "grad_y", total.shape)
    _dev(stats, "stats", (2,) + px)
    _per_channel(C, gamma=gamma)
    if grad_total is not None:
        _dev(grad_total, "grad_total", total.shape)
    grad_x = _like(total, grad_x, "grad_x", stream)
    if grad_branch is not None or drop > 0:
        grad_branch = _like(total, grad_branch, "grad_branch", stream)
    prm = norm_params(C, frames if pixels else 0, pixels or 1, 0.0, drop, site)
    gg, gb, room = None, None, (None, 0)
    if weights:
        gg, gb = _new((C,), total, stream), _new((C,), total, stream)
        if workspace is None:
            need = lib.snls_norm_workspace_size(ctypes.byref(prm))
            if need == ctypes.c_size_t(-1).value:
                raise SnlsError(SNLS_ERR_INVALID_ARG, "snls_norm_workspace_size")
            workspace = _new(((need + 3) // 4,), total, stream)
        room = _room(workspace)
    _here(grad_y, total, stats, gamma, grad_total, rng, grad_x, grad_branch, workspace)
    _check(lib.snls_norm_backward(_ptr(grad_y), _ptr(grad_total), _ptr(total), _ptr(stats), _ptr(gamma),
                                  _rng(rng, drop), ctypes.byref(prm), _ptr(grad_x), _ptr(grad_branch), _ptr(gg),
                                  _ptr(gb), *room, _stream(stream)), "snls_norm_backward")
    return grad_x, grad_x if grad_branch is None else grad_branch, gg, gb


def snls_dropout(x, rng, drop: float, site: int = 0, residual=None, out=None, stream=None):
    """dropout(x), or residual + dropout(x); applied to a gradient it is its own backward pass.  out may be x or
    residual."""
    lib = load_library()
    _dev(x, "x")
    if residual is not None:
        _dev(residual, "residual", x.shape)
    out = _like(x, out, "out", stream)
    _here(x, residual, rng, out)
    _check(lib.snls_dropout(_ptr(x), _ptr(residual), _rng(rng, drop), x.numel(), float(drop), dropout_site(site),
                            _ptr(out), _stream(stream)), "snls_dropout")
    return out


# ------------------------------------------------------------- rotary positions --

_ROTATE_SIZE, _pack_rotate = ctypes.sizeof(SnlsRotateParams), struct.Struct("=I9i3f3i").pack  # the struct's fields


def rotate_from_dict(rp: dict) -> SnlsRotateParams:
    if len(rp["pairs"]) != 3 or len(rp["theta"]) != 3:
        raise ValueError("pairs and theta have three entries: time, row, column")
    try:  # (packing looks at the numbers' ranges, which ctypes fields do not, and takes half their time)
        return SnlsRotateParams.from_buffer_copy(_pack_rotate(
            _ROTATE_SIZE, int(rp["B"]), int(rp["T"]), int(rp["C"]), int(rp["H"]), int(rp["W"]), int(rp["HD"]),
            *rp["pairs"], *rp["theta"], int(rp.get("interleaved", 0)), int(rp.get("row0", 0)), int(rp.get("col0", 0))))
    except (struct.error, OverflowError) as e:
        raise ValueError("sizes, pairs and origins must be whole numbers of 32 bits, theta of fp32's range: %s" % e)


def snls_rotate(q, k, rp: dict, times=None, inverse: bool = False, q_out=None, k_out=None, stream=None):
    """Rotary positions of videos q and k (None for q alone); returns (q_out, k_out).  times: int64 (B, T), or None
    for 0 .. T-1.  inverse: the gradients of q and k from those of the outputs.  Outputs may be q and k."""
    lib = load_library()
    shp = video_shape(rp)
    _dev(q, "q", shp)
    q_out = _like(q, q_out, "q_out", stream)
    if k is not None:
        _dev(k, "k", shp)
        k_out = _like(k, k_out, "k_out", stream)
    elif k_out is not None:
        raise ValueError("k_out goes with k")
    if times is not None:
        _dev_as(times, "times", (rp["B"], rp["T"]), (torch.int64,))
    _here(q, k, times, q_out, k_out)
    prm = rotate_from_dict(rp)
    _check(lib.snls_rotate(_ptr(q), _ptr(k), _ptr(times), ctypes.byref(prm), int(inverse), _ptr(q_out), _ptr(k_out),
                           _stream(stream)), "snls_rotate")
    return q_out, k_out


def snls_rotate_points(q, points, rp: dict, times=None, inverse: bool = False, out=None, stream=None):
    """The same for tokens q (n, C) at points int32 (n, 3) = video, row, column; times int64 (B), or None for 0."""
    lib = load_library()
    _dev(q, "q")
    n = q.shape[0]
    _dev(q, "q", (n, rp["C"]))
    _dev_as(points, "points", (n, 3), (torch.int32,))
    if times is not None:
        _dev_as(times, "times", (rp["B"],), (torch.int64,))
    out = _like(q, out, "out", stream)
    _here(q, points, times, out)
    prm = rotate_from_dict(rp)
    _check(lib.snls_rotate_points(_ptr(q), _ptr(points), n, _ptr(times), ctypes.byref(prm), int(inverse), _ptr(out),
                                  _stream(stream)), "snls_rotate_points")
    return out


# ------------------------------------------------------------- 8-bit projections --

_PROJECT_SIZE = ctypes.sizeof(SnlsProjectParams)


def project_params(cin: int, cout: int, parts: int, frames: int, pixels: int) -> SnlsProjectParams:
    return SnlsProjectParams(_PROJECT_SIZE, min(cin, _MOST), min(cout, _MOST), parts, frames, pixels)


def snls_project_pack(w, codes=None, scales=None, stream=None):
    """Weights (cout, cin) as int8 codes and a scale per output channel: (codes, scales)."""
    lib = load_library()
    _dev(w, "w")
    if w.dim() != 2:
        raise ValueError("w must be (cout, cin)")
    cout, cin = w.shape
    if codes is None:
        codes = torch.empty(w.shape, device=w.device, dtype=torch.int8)
        if stream is not None:
            codes.record_stream(stream)
    _dev_as(codes, "codes", w.shape, (torch.int8,))
    scales = _dev(scales, "scales", (cout,)) if scales is not None else _new((cout,), w, stream)
    _here(w, codes, scales)
    prm = project_params(cin, cout, 1, 0, 1)
    _check(lib.snls_project_pack(_ptr(w), ctypes.byref(prm), _ptr(codes), _ptr(scales), _stream(stream)),
           "snls_project_pack")
    return codes, scales


def snls_project(x, codes, scales, bias=None, parts: int = 1, out=None, stream=None):
    """Product of features (..., cin, H, W) or tokens (n, cin) with 8-bit weights (cout, cin); returns
    (parts, ..., cout / parts, H, W) or (parts, n, cout / parts): parts tensors, one after the other."""
    lib = load_library()
    frames, cin, pixels, _ = _features(x, "x")
    if not isinstance(codes, torch.Tensor) or codes.dim() != 2:
        raise ValueError("codes must be (cout, cin)")
    cout, parts = codes.shape[0], int(parts)
    _dev_as(codes, "codes", (cout, cin), (torch.int8,))
    _per_channel(cout, scales=scales, bias=bias)
    if parts < 1 or cout % parts:
        raise ValueError("parts must divide cout")
    tail = (cout // parts,) + tuple(x.shape[-2:]) if x.dim() > 2 else (cout // parts,)
    shp = (parts,) + tuple(x.shape[:-3] if x.dim() > 2 else x.shape[:1]) + tail
    out = _dev(out, "out", shp) if out is not None else _new(shp, x, stream)
    _here(x, codes, scales, bias, out)
    prm = project_params(cin, cout, parts, frames, pixels or 1)
    if pixels:
        _check(lib.snls_project(_ptr(x), _ptr(codes), _ptr(scales), _ptr(bias), ctypes.byref(prm), _ptr(out),
                                _stream(stream)), "snls_project")
    return out
