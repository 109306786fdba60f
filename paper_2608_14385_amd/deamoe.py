"""Python binding of libdeamoe.so (the C ABI in include/deamoe.h).

Argument marshalling only: every step of the layer runs in the library's HIP
kernels.  PyTorch provides device memory and the current stream.  The module
raises at import of the library when libdeamoe.so is missing; there is no
fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import functools
import os
from dataclasses import dataclass

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdeamoe.so")

OK, ERR_INVALID, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = 0, -1, -2, -3, -4
F32, BF16, FP8_E4M3_B128 = 0, 1, 2
FORM_SLICE, FORM_FACTORED = 0, 1
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
SIGMA_SILU, SIGMA_NONE, SIGMA_GELU, SIGMA_RMSNORM = 0, 1, 2, 3
MAX_TOKENS = 128
SCRATCH_BYTES = 64 << 20   # library-owned workspace of deamoe_layer_forward_noalloc, per GPU

EXPORTS = ("deamoe_status_string", "deamoe_workspace_bytes", "deamoe_route",
           "deamoe_layer_forward", "deamoe_layer_forward_traced", "deamoe_baseline_forward",
           "deamoe_loaded_bytes", "deamoe_trace_points", "deamoe_layer_forward_noalloc",
           "deamoe_dispatch_workspace_bytes", "deamoe_dispatch", "deamoe_dispatch_backward",
           "deamoe_combine", "deamoe_combine_backward", "deamoe_w4_linear", "deamoe_w4_swiglu",
           "deamoe_prenorm", "deamoe_prenorm_backward", "deamoe_postnorm",
           "deamoe_postnorm_backward", "deamoe_norm_workspace_bytes")


class DeamoeError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_string(status)} ({status})")
        self.status = status


class deamoe_config(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("hidden", "n_experts", "n_depts", "top_k", "top_k_dept",
                                         "d_shared", "d_private", "d_shared_expert", "form",
                                         "score", "renorm", "sigma")] + \
               [("route_scale", C.c_float), ("w_dtype", C.c_int32), ("act_dtype", C.c_int32),
                ("max_tokens", C.c_int32), ("dept_cover", C.c_int32)]


class deamoe_weights(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("router", "dept_gate", "dept_up", "dept_down",
                                          "priv_gate", "priv_up", "priv_down", "se_gate", "se_up",
                                          "se_down")] + [("scale", C.c_void_p * 9)]


ROUTING_FIELDS = ("topk_ids", "topk_w", "tok_depts", "tok_dept_w", "tok_ndept", "dept_count",
                  "dept_offset", "dept_tokens", "exp_count", "exp_offset", "exp_tokens", "logits")


class deamoe_routing(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ROUTING_FIELDS]


class deamoe_w4_config(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("R", "K", "n", "group", "scale_dtype")]


GATE_NONE, GATE_SHARED, GATE_FULL = 0, 1, 2

_lib = None


def lib():
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing; build it with "
                              "`python -m paper_2608_14385_amd.build`")
        L = C.CDLL(LIB_PATH)
        cfgp, vp, i32 = C.POINTER(deamoe_config), C.c_void_p, C.c_int32
        L.deamoe_status_string.restype = C.c_char_p
        L.deamoe_status_string.argtypes = [C.c_int]
        L.deamoe_workspace_bytes.argtypes = [cfgp, C.POINTER(C.c_size_t)]
        L.deamoe_route.argtypes = [cfgp, i32, vp, vp, vp, vp, C.POINTER(deamoe_routing), vp,
                                   C.c_size_t, vp]
        layer_args = [cfgp, i32, vp, C.POINTER(deamoe_weights), vp, vp, C.POINTER(deamoe_routing),
                      vp, vp, C.c_size_t, vp]
        L.deamoe_layer_forward.argtypes = layer_args
        L.deamoe_baseline_forward.argtypes = layer_args
        L.deamoe_layer_forward_traced.argtypes = layer_args + [C.POINTER(C.c_void_p), i32]
        L.deamoe_layer_forward_noalloc.argtypes = [cfgp, i32, vp, C.POINTER(deamoe_weights), vp, vp,
                                                   C.POINTER(deamoe_routing), vp, vp]
        L.deamoe_trace_points.argtypes = [cfgp, i32, C.POINTER(C.c_int32)]
        L.deamoe_loaded_bytes.argtypes = [cfgp, i32, vp, vp, C.POINTER(C.c_int64),
                                          C.POINTER(C.c_int64)]
        sz, f32, szp, w4p = C.c_size_t, C.c_float, C.POINTER(C.c_size_t), C.POINTER(deamoe_w4_config)
        L.deamoe_dispatch_workspace_bytes.argtypes = [i32, i32, i32, szp]
        L.deamoe_dispatch.argtypes = [i32] * 5 + [vp] * 7 + [sz, vp]
        L.deamoe_dispatch_backward.argtypes = [i32] * 4 + [vp] * 4
        L.deamoe_combine.argtypes = [i32] * 4 + [vp] * 5
        L.deamoe_combine_backward.argtypes = [i32] * 4 + [vp] * 7
        L.deamoe_w4_linear.argtypes = [w4p, i32] + [vp] * 6
        L.deamoe_w4_swiglu.argtypes = [w4p, i32] + [vp] * 8
        L.deamoe_prenorm.argtypes = [i32] * 3 + [f32] + [vp] * 4
        L.deamoe_prenorm_backward.argtypes = [i32] * 3 + [f32] + [vp] * 7 + [sz, vp]
        L.deamoe_postnorm.argtypes = [i32] * 3 + [f32, f32, i32] + [vp] * 8
        L.deamoe_postnorm_backward.argtypes = [i32] * 3 + [f32, f32, i32] + [vp] * 13 + [sz, vp]
        L.deamoe_norm_workspace_bytes.argtypes = [i32, i32, szp]
        for f in EXPORTS:
            getattr(L, f).restype = C.c_int if f != "deamoe_status_string" else C.c_char_p
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().deamoe_status_string(status).decode()


def _check(status: int, what: str):
    if status != OK:
        raise DeamoeError(status, what)


_DT = {"f32": F32, "bf16": BF16, "fp8": FP8_E4M3_B128}


def make_config(cfg, max_tokens: int) -> deamoe_config:
    """C config from a layer description (workloads.LayerConfig or alike)."""
    return deamoe_config(hidden=cfg.hidden, n_experts=cfg.n_experts, n_depts=cfg.n_depts,
                         top_k=cfg.top_k, top_k_dept=cfg.top_k_dept, d_shared=cfg.d_shared,
                         d_private=cfg.d_private, d_shared_expert=cfg.d_shared_expert,
                         form={"slice": FORM_SLICE, "factored": FORM_FACTORED}[cfg.form],
                         score={"softmax": SCORE_SOFTMAX, "sigmoid": SCORE_SIGMOID}[cfg.score],
                         renorm=int(bool(cfg.renorm)),
                         sigma={"silu": SIGMA_SILU, "none": SIGMA_NONE, "gelu": SIGMA_GELU,
                                "rmsnorm": SIGMA_RMSNORM}[cfg.sigma],
                         route_scale=float(cfg.route_scale), w_dtype=_DT[cfg.w_dtype],
                         act_dtype=_DT[cfg.act_dtype], max_tokens=int(max_tokens),
                         dept_cover=int(getattr(cfg, "dept_cover", 0)))


_WKEYS = ("dept_gate", "dept_up", "dept_down", "priv_gate", "priv_up", "priv_down",
          "se_gate", "se_up", "se_down")


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def make_weights(w: dict) -> deamoe_weights:
    """C weight table from a dict of device tensors (keys as in workloads.weight_shapes)."""
    W = deamoe_weights()
    W.router = _ptr(w.get("router"))
    for i, k in enumerate(_WKEYS):
        setattr(W, k, _ptr(w.get(k)))
        W.scale[i] = _ptr(w.get(k + "_scale"))
    return W


def workspace_bytes(c: deamoe_config) -> int:
    n = C.c_size_t(0)
    _check(lib().deamoe_workspace_bytes(C.byref(c), C.byref(n)), "deamoe_workspace_bytes")
    return int(n.value)


def alloc_workspace(c: deamoe_config, device="cuda") -> torch.Tensor:
    return torch.empty(workspace_bytes(c), dtype=torch.uint8, device=device)


@dataclass
class Routing:
    """Device tensors receiving the routing of one step."""
    tensors: dict

    @classmethod
    def alloc(cls, cfg, T: int, device="cuda") -> "Routing":
        n, m, k = cfg.n_experts, cfg.n_depts, cfg.top_k
        i32, f32 = torch.int32, torch.float32
        shapes = {"topk_ids": ((T, k), i32), "topk_w": ((T, k), f32),
                  "tok_depts": ((T, k), i32), "tok_dept_w": ((T, k), f32),
                  "tok_ndept": ((T,), i32), "dept_count": ((m,), i32),
                  "dept_offset": ((m + 1,), i32), "dept_tokens": ((max(T * k, 1),), i32),
                  "exp_count": ((n,), i32), "exp_offset": ((n + 1,), i32),
                  "exp_tokens": ((max(T * k, 1),), i32), "logits": ((T, n), f32)}
        return cls({key: torch.full(s, -7, dtype=dt, device=device)
                    for key, (s, dt) in shapes.items()})

    def struct(self) -> deamoe_routing:
        return deamoe_routing(**{k: self.tensors[k].data_ptr() for k in ROUTING_FIELDS})

    def host(self) -> dict:
        """Host copies, with the CSR token lists cut to their used length."""
        h = {k: v.cpu().numpy() for k, v in self.tensors.items()}
        h["dept_tokens"] = h["dept_tokens"][: h["dept_offset"][-1]]
        h["exp_tokens"] = h["exp_tokens"][: h["exp_offset"][-1]]
        return h


def _stream(stream) -> int | None:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def deamoe_route(c: deamoe_config, x, router_w, routing: Routing, ws: torch.Tensor,
                 logits_in=None, router_bias=None, T: int | None = None, stream=None):
    T = int(x.shape[0]) if T is None else T
    r = routing.struct()
    _check(lib().deamoe_route(C.byref(c), T, _ptr(x), _ptr(router_w), _ptr(logits_in),
                              _ptr(router_bias), C.byref(r), _ptr(ws), ws.numel(),
                              _stream(stream)), "deamoe_route")


def _layer(fn, c, x, W, y, ws, logits_in, router_bias, routing, stream, *extra):
    r = routing.struct() if routing is not None else None
    _check(fn(C.byref(c), int(x.shape[0]), _ptr(x), C.byref(W), _ptr(logits_in),
              _ptr(router_bias), C.byref(r) if r is not None else None, _ptr(y), _ptr(ws),
              ws.numel(), _stream(stream), *extra), fn.__name__)


def deamoe_layer_forward(c: deamoe_config, x, W: deamoe_weights, y, ws, logits_in=None,
                         router_bias=None, routing: Routing | None = None, stream=None):
    _layer(lib().deamoe_layer_forward, c, x, W, y, ws, logits_in, router_bias, routing, stream)


def deamoe_layer_forward_traced(c: deamoe_config, x, W: deamoe_weights, y, ws, events: list,
                                logits_in=None, router_bias=None, routing: Routing | None = None,
                                stream=None):
    """events: raw hipEvent_t handles (ints) recorded at the stage boundaries."""
    arr = (C.c_void_p * len(events))(*events)
    _layer(lib().deamoe_layer_forward_traced, c, x, W, y, ws, logits_in, router_bias, routing,
           stream, arr, len(events))


def deamoe_layer_forward_noalloc(c: deamoe_config, x, W: deamoe_weights, y, logits_in=None,
                                 router_bias=None, routing: Routing | None = None, stream=None):
    """deamoe_layer_forward on the library's own per-GPU scratch array (no workspace)."""
    r = routing.struct() if routing is not None else None
    _check(lib().deamoe_layer_forward_noalloc(
        C.byref(c), int(x.shape[0]), _ptr(x), C.byref(W), _ptr(logits_in), _ptr(router_bias),
        C.byref(r) if r is not None else None, _ptr(y), _stream(stream)),
        "deamoe_layer_forward_noalloc")


def deamoe_baseline_forward(c: deamoe_config, x, W: deamoe_weights, y, ws, logits_in=None,
                            router_bias=None, routing: Routing | None = None, stream=None):
    _layer(lib().deamoe_baseline_forward, c, x, W, y, ws, logits_in, router_bias, routing, stream)


def deamoe_loaded_bytes(c: deamoe_config, T: int, dept_count, exp_count) -> tuple:
    import numpy as np
    dc = np.ascontiguousarray(np.asarray(dept_count, dtype=np.int32))
    ec = np.ascontiguousarray(np.asarray(exp_count, dtype=np.int32))
    wb, tb = C.c_int64(0), C.c_int64(0)
    _check(lib().deamoe_loaded_bytes(C.byref(c), T, dc.ctypes.data, ec.ctypes.data, C.byref(wb),
                                     C.byref(tb)), "deamoe_loaded_bytes")
    return int(wb.value), int(tb.value)


def deamoe_trace_points(c: deamoe_config, T: int) -> int:
    n = C.c_int32(0)
    _check(lib().deamoe_trace_points(C.byref(c), T, C.byref(n)), "deamoe_trace_points")
    return int(n.value)


class Layer:
    """Owns the config, weight table and workspace of one layer on one device."""

    def __init__(self, cfg, weights: dict, max_tokens: int, device="cuda", baseline=False):
        self.cfg = cfg
        self.c = make_config(cfg, max_tokens)
        self.weights = weights
        self.W = make_weights(weights)
        self.ws = alloc_workspace(self.c, device)
        self.baseline = baseline

    def __call__(self, x, logits_in=None, router_bias=None, routing=None, y=None, stream=None):
        if y is None:
            y = torch.empty_like(x)
        fn = deamoe_baseline_forward if self.baseline else deamoe_layer_forward
        fn(self.c, x, self.W, y, self.ws, logits_in=logits_in, router_bias=router_bias,
           routing=routing, stream=stream)
        return y


# ---------------------------------------------------------------------------
# Operators beside the layer: sorted tokens, 4-bit products, norms.  Tensors
# are contiguous and on one device, outputs are the caller's; the calls run on
# `stream` (default: the current stream of the tensors' device) and, where no
# workspace is given, take one from torch's allocator for that stream.  None of
# them, nor the classes below, is recorded by autograd: results carry no gradient
# history, also of inputs that require one; gradients are the _backward calls.


def _fits(what: str, dev: int, *tensors):
    """Every (name, tensor, dtype, shape) has that type and shape, is contiguous and on device `dev`."""
    for name, t, dtype, shape in tensors:
        if t is None:
            raise DeamoeError(ERR_INVALID, f"{what}: {name} is needed")
        if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
            raise DeamoeError(ERR_INVALID, f"{what}: {name} is {t.dtype} {tuple(t.shape)} with strides "
                              f"{t.stride()} on {t.device}; needed is {dtype} {tuple(shape)}, contiguous, "
                              f"on device {dev}")


def _act(what: str, t: torch.Tensor) -> int:
    if t.dtype is torch.bfloat16:
        return BF16
    if t.dtype is torch.float32:
        return F32
    raise DeamoeError(ERR_INVALID, f"{what}: {t.dtype} is neither bfloat16 nor float32")


def _same_device(what: str, dev: int, stream):
    if stream.device.index != dev:
        raise DeamoeError(ERR_INVALID, f"{what}: the stream is on {stream.device}, the tensors are on device {dev}")


def _on(what: str, dev: int, stream):
    """A context in which device `dev` is the current one and, where one is given, `stream` its current stream."""
    if stream is not None:
        _same_device(what, dev, stream)
        return torch.cuda.stream(stream)
    if dev >= 0 and dev != torch.cuda.current_device():
        return torch.cuda.device(dev)
    return contextlib.nullcontext()


def _call(fn, dev: int, stream, args) -> int:
    """fn(*args, stream) with device `dev` current; the stream is its current one unless given."""
    if dev < 0:
        raise DeamoeError(ERR_INVALID, f"{fn.__name__}: tensors are not on a GPU")
    if stream is not None:
        _same_device(fn.__name__, dev, stream)
    if dev != torch.cuda.current_device():
        with torch.cuda.device(dev):
            return _call(fn, dev, stream, args)
    # the raw handle: a torch.cuda.Stream made for the call costs more than the launch
    return fn(*args, torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream)


def _run(fn, dev: int, stream, *args):
    _check(_call(fn, dev, stream, args), fn.__name__)


def _run_with_workspace(fn, dev: int, stream, ws, nbytes: int, *args):
    """The same for a call whose last two arguments are its workspace: the given one, or one of torch's
    for the stream that the call runs on."""
    if ws is None and nbytes and dev >= 0:
        with contextlib.nullcontext() if stream is None else _on(fn.__name__, dev, stream):
            ws = torch.empty(nbytes, dtype=torch.uint8, device=torch.device("cuda", dev))
    elif ws is not None and (ws.get_device() != dev or not ws.is_contiguous()):
        raise DeamoeError(ERR_WORKSPACE, f"{fn.__name__}: workspace is not contiguous, or not on device {dev}")
    _run(fn, dev, stream, *args, _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size())


_INT32 = (1 << 31) - 1   # ctypes passes larger sizes on modulo 2^32


def _too_large(what: str, name: str, sizes):
    raise DeamoeError(ERR_UNSUPPORTED, f"{what}: {name} {tuple(sizes)} has sizes past 2^31 - 1")


def _bytes(fn, *args) -> int:
    if max(args) > _INT32:
        _too_large(fn.__name__, "sizes", args)
    n = C.c_size_t(0)
    _check(fn(*args, C.byref(n)), fn.__name__)
    return n.value


def _rows(what: str, t: torch.Tensor, name: str) -> tuple:
    try:
        rows, cols = t.shape
    except (AttributeError, ValueError):
        raise DeamoeError(ERR_INVALID, f"{what}: {name} is {'missing' if t is None else tuple(t.shape)}, "
                                       "needed are two dimensions") from None
    if rows > _INT32 or cols > _INT32:
        _too_large(what, name, (rows, cols))
    return rows, cols


@functools.lru_cache(maxsize=1024)   # of sizes alone; 10 pairs sorted in 8.5 us, not 8.9
def deamoe_dispatch_workspace_bytes(T: int, k: int, n: int) -> int:
    return _bytes(lib().deamoe_dispatch_workspace_bytes, T, k, n)


def deamoe_dispatch(ids, x, offset, pair, row, xs=None, ws=None, stream=None):
    """Tokens sorted by group: ids [T, k] int32 -> offset [n + 1], pair [T * k], row [T, k], and
    with xs [T * k, h] the rows of x [T, h] in that order (x may be None without xs)."""
    what, i32 = "deamoe_dispatch", torch.int32
    T, k = _rows(what, ids, "ids")
    try:
        n = offset.numel() - 1   # past 32 bits: the workspace's size refuses it
    except AttributeError:
        raise DeamoeError(ERR_INVALID, f"{what}: offset is needed") from None
    dev, h, act = ids.get_device(), 1, F32
    _fits(what, dev, ("ids", ids, i32, (T, k)), ("offset", offset, i32, (n + 1,)),
          ("pair", pair, i32, (T * k,)), ("row", row, i32, (T, k)))
    if xs is not None:
        h, act = _rows(what, x, "x")[1], _act(what, x)
        _fits(what, dev, ("x", x, x.dtype, (T, h)), ("xs", xs, x.dtype, (T * k, h)))
    _run_with_workspace(lib().deamoe_dispatch, dev, stream, ws,
                        deamoe_dispatch_workspace_bytes(T, k, n), T, k, n, h, act,
                        ids.data_ptr(), x.data_ptr() if xs is not None else None, offset.data_ptr(),
                        pair.data_ptr(), row.data_ptr(), _ptr(xs))


def deamoe_dispatch_backward(row, dxs, dx, stream=None):
    """dx [T, h]: the sum of each token's rows of dxs [T * k, h]."""
    what = "deamoe_dispatch_backward"
    (T, k), h, dev, dt = _rows(what, row, "row"), _rows(what, dx, "dx")[1], row.get_device(), dx.dtype
    act = _act(what, dx)
    _fits(what, dev, ("row", row, torch.int32, (T, k)), ("dx", dx, dt, (T, h)),
          ("dxs", dxs, dt, (T * k, h)))
    _run(lib().deamoe_dispatch_backward, dev, stream, T, k, h, act, row.data_ptr(),
         dxs.data_ptr(), dx.data_ptr())


def deamoe_combine(row, w, ys, y, stream=None):
    """y [T, h]: the sum of each token's rows of ys [T * k, h], weighted by w [T, k] (fp32)."""
    what = "deamoe_combine"
    (T, k), h, dev, dt = _rows(what, row, "row"), _rows(what, y, "y")[1], row.get_device(), y.dtype
    act = _act(what, y)
    _fits(what, dev, ("row", row, torch.int32, (T, k)), ("w", w, torch.float32, (T, k)),
          ("y", y, dt, (T, h)), ("ys", ys, dt, (T * k, h)))
    _run(lib().deamoe_combine, dev, stream, T, k, h, act, row.data_ptr(), w.data_ptr(),
         ys.data_ptr(), y.data_ptr())


def deamoe_combine_backward(row, w, ys, dy, dys=None, dw=None, stream=None):
    """dys [T * k, h] and dw [T, k] (either may be None) from dy [T, h]; w is needed for dys only,
    ys for dw only."""
    what, f32 = "deamoe_combine_backward", torch.float32
    (T, k), h, dev, dt = _rows(what, row, "row"), _rows(what, dy, "dy")[1], row.get_device(), dy.dtype
    act = _act(what, dy)
    _fits(what, dev, ("row", row, torch.int32, (T, k)), ("dy", dy, dt, (T, h)))
    if dys is not None:
        _fits(what, dev, ("dys", dys, dt, (T * k, h)), ("w", w, f32, (T, k)))
    if dw is not None:
        _fits(what, dev, ("dw", dw, f32, (T, k)), ("ys", ys, dt, (T * k, h)))
    _run(lib().deamoe_combine_backward, dev, stream, T, k, h, act, row.data_ptr(),
         w.data_ptr() if dys is not None else None, ys.data_ptr() if dw is not None else None,
         dy.data_ptr(), _ptr(dys), _ptr(dw))


def _w4(what: str, x, matrices, y, offset):
    """Checks one product's tensors: its config, rows and device."""
    codes, scale = matrices[0]
    M, K = _rows(what, x, "x")
    if codes is None or scale is None:
        raise DeamoeError(ERR_INVALID, f"{what}: codes and scale are needed")
    shape, groups = codes.shape, scale.shape[-1] if scale.dim() else 0
    if len(shape) not in (2, 3) or shape[-1] * 2 != K or scale.dim() != len(shape) or not groups or K % groups:
        raise DeamoeError(ERR_INVALID, f"{what}: codes {tuple(shape)} and scale {tuple(scale.shape)} "
                                       f"do not fit {K} columns")
    n, R, dev, sdt, bf16 = shape[0] if len(shape) == 3 else 1, shape[-2], x.get_device(), scale.dtype, torch.bfloat16
    if n > _INT32 or R > _INT32:
        _too_large(what, "codes", shape)
    if sdt is not torch.float32 and sdt is not bf16:
        raise DeamoeError(ERR_INVALID, f"{what}: scale is {sdt}")
    for c, s in matrices:
        _fits(what, dev, ("codes", c, torch.uint8, shape), ("scale", s, sdt, (*shape[:-1], groups)))
    _fits(what, dev, ("x", x, bf16, (M, K)), ("y", y, bf16, (M, R)))
    if offset is not None:
        _fits(what, dev, ("offset", offset, torch.int32, (n + 1,)))
    return deamoe_w4_config(R, K, n, K // groups, BF16 if sdt is bf16 else F32), M, dev


def deamoe_w4_linear(x, codes, scale, y, offset=None, stream=None):
    """y [M, R] = x [M, K] W^T (bf16); codes [R, K / 2] uint8 and scale [R, K / group], or stacks of
    n of both with offset [n + 1] (int32): the rows of every matrix."""
    cfg, M, dev = _w4("deamoe_w4_linear", x, ((codes, scale),), y, offset)
    _run(lib().deamoe_w4_linear, dev, stream, C.byref(cfg), M, x.data_ptr(), _ptr(offset),
         codes.data_ptr(), scale.data_ptr(), y.data_ptr())


def deamoe_w4_swiglu(x, gate_codes, gate_scale, up_codes, up_scale, y, offset=None, stream=None):
    """y = SiLU(x Wg^T) * (x Wu^T), otherwise as deamoe_w4_linear."""
    cfg, M, dev = _w4("deamoe_w4_swiglu", x, ((gate_codes, gate_scale), (up_codes, up_scale)), y,
                      offset)
    _run(lib().deamoe_w4_swiglu, dev, stream, C.byref(cfg), M, x.data_ptr(), _ptr(offset),
         gate_codes.data_ptr(), gate_scale.data_ptr(), up_codes.data_ptr(), up_scale.data_ptr(),
         y.data_ptr())


@functools.lru_cache(maxsize=1024)
def deamoe_norm_workspace_bytes(T: int, h: int) -> int:
    return _bytes(lib().deamoe_norm_workspace_bytes, T, h)


def deamoe_prenorm(x, w, u, eps: float = 1e-6, stream=None):
    """u = RMSNorm(x) * w, rows of x [T, h]; u may be x."""
    what = "deamoe_prenorm"
    (T, h), act, dev, dt = _rows(what, x, "x"), _act(what, x), x.get_device(), x.dtype
    _fits(what, dev, ("x", x, dt, (T, h)), ("w", w, dt, (h,)), ("u", u, dt, (T, h)))
    _run(lib().deamoe_prenorm, dev, stream, T, h, act, eps, x.data_ptr(), w.data_ptr(),
         u.data_ptr())


def deamoe_prenorm_backward(x, w, du, dx, dw, dres=None, eps: float = 1e-6, ws=None, stream=None):
    """dx = dres + the gradient of x from du; dw [h] fp32.  dres may be dx."""
    what = "deamoe_prenorm_backward"
    (T, h), act, dev, dt = _rows(what, x, "x"), _act(what, x), x.get_device(), x.dtype
    _fits(what, dev, ("x", x, dt, (T, h)), ("w", w, dt, (h,)), ("du", du, dt, (T, h)),
          ("dx", dx, dt, (T, h)), ("dw", dw, torch.float32, (h,)))
    if dres is not None:
        _fits(what, dev, ("dres", dres, dt, (T, h)))
    _run_with_workspace(lib().deamoe_prenorm_backward, dev, stream, ws,
                        deamoe_norm_workspace_bytes(T, h), T, h, act, eps, x.data_ptr(),
                        w.data_ptr(), du.data_ptr(), _ptr(dres), dx.data_ptr(), dw.data_ptr())


def _gate(what, gate, T, h, dt, dev) -> int:
    if gate is None:
        return GATE_NONE
    shared = gate.dim() == 1
    _fits(what, dev, ("gate", gate, dt, (h,) if shared else (T, h)))
    return GATE_SHARED if shared else GATE_FULL


def deamoe_postnorm(x, y, w, z, gate=None, res_scale: float = 1.0, w_next=None, u=None,
                    eps: float = 1e-6, stream=None):
    """z = res_scale * x + gate * RMSNorm(y) * w, rows of x and y [T, h]; gate [h], [T, h] or None (1).
    With w_next and u also u = RMSNorm(z) * w_next.  z may be x."""
    what = "deamoe_postnorm"
    (T, h), act, dev, dt = _rows(what, x, "x"), _act(what, x), x.get_device(), x.dtype
    full = (T, h)
    _fits(what, dev, ("x", x, dt, full), ("y", y, dt, full), ("w", w, dt, (h,)), ("z", z, dt, full))
    if w_next is not None:
        _fits(what, dev, ("w_next", w_next, dt, (h,)))
    if u is not None:
        _fits(what, dev, ("u", u, dt, full))
    mode = _gate(what, gate, T, h, dt, dev)
    _run(lib().deamoe_postnorm, dev, stream, T, h, act, eps, res_scale, mode, x.data_ptr(),
         y.data_ptr(), w.data_ptr(), _ptr(gate), _ptr(w_next), z.data_ptr(), _ptr(u))


def deamoe_postnorm_backward(y, w, dz, dx, dy, dw, gate=None, dgate=None, res_scale: float = 1.0,
                             z=None, w_next=None, du=None, dw_next=None, eps: float = 1e-6, ws=None,
                             stream=None):
    """Gradients of deamoe_postnorm from dz and, with a next norm (z, w_next, du, dw_next), du: dx, dy
    [T, h], dw and dw_next [h] fp32, dgate as the gate ([h]: fp32).  dx may be dz."""
    what, f32 = "deamoe_postnorm_backward", torch.float32
    (T, h), act, dev, dt = _rows(what, y, "y"), _act(what, y), y.get_device(), y.dtype
    mode, full, vec = _gate(what, gate, T, h, dt, dev), (T, h), (h,)
    _fits(what, dev, ("y", y, dt, full), ("w", w, dt, vec), ("dz", dz, dt, full), ("dx", dx, dt, full),
          ("dy", dy, dt, full), ("dw", dw, f32, vec))
    if (dgate is None) != (mode == GATE_NONE) or len({t is None for t in (z, w_next, du, dw_next)}) != 1:
        raise DeamoeError(ERR_INVALID, f"{what}: gate and dgate, and z, w_next, du and dw_next, are "
                                       "given together or not at all")
    if dgate is not None:
        _fits(what, dev, ("dgate", dgate, f32, vec) if mode == GATE_SHARED else ("dgate", dgate, dt, full))
    if du is not None:
        _fits(what, dev, ("z", z, dt, full), ("w_next", w_next, dt, vec), ("du", du, dt, full),
              ("dw_next", dw_next, f32, vec))
    _run_with_workspace(lib().deamoe_postnorm_backward, dev, stream, ws,
                        deamoe_norm_workspace_bytes(T, h), T, h, act, eps, res_scale, mode,
                        y.data_ptr(), w.data_ptr(), _ptr(gate), _ptr(z), _ptr(w_next), dz.data_ptr(),
                        _ptr(du), dx.data_ptr(), dy.data_ptr(), dw.data_ptr(), _ptr(dgate), _ptr(dw_next))


class W4Experts:
    """SwiGLU experts with 4-bit weights, for batches of any size: tokens sorted by expert, the
    experts' products over their rows, and the weighted way back.

    gate, up and down are (codes, scale) pairs: gate and up [n, d, h / 2] and [n, d, h / group], down
    [n, h, d / 2] and [n, h, d / group].

    Forward only: 4-bit products have no gradient here, and the result is detached from its inputs.
    The activations and every expert's row of the down product are rounded to bf16, the products'
    output type, before the weighted sum in fp32 (Layer keeps those rows in fp32): rows of half the
    bytes for the way back, at half a bf16 step, 2^-8, of each row's share of y."""

    def __init__(self, gate, up, down):
        self.gate, self.up, self.down = gate, up, down
        self.n, self.d, half = gate[0].shape
        self.h = 2 * half

    def __call__(self, x, topk_ids, topk_w, y=None, stream=None):
        """y [T, h] from x [T, h] (bf16), topk_ids [T, k] (int32, -1: none) and topk_w [T, k] (fp32)."""
        if stream is not None:
            with _on("W4Experts", x.get_device(), stream):
                return self(x, topk_ids, topk_w, y)
        T, k = topk_ids.shape
        new, i32 = dict(device=x.device), torch.int32
        offset, pair = torch.empty(self.n + 1, dtype=i32, **new), torch.empty(T * k, dtype=i32, **new)
        row, xs = torch.empty(T, k, dtype=i32, **new), x.new_empty(T * k, self.h)
        a, ys = x.new_empty(T * k, self.d), x.new_empty(T * k, self.h)
        y = torch.empty_like(x) if y is None else y
        deamoe_dispatch(topk_ids, x, offset, pair, row, xs)
        deamoe_w4_swiglu(xs, *self.gate, *self.up, a, offset=offset)
        deamoe_w4_linear(a, *self.down, ys, offset=offset)
        deamoe_combine(row, topk_w, ys, y)
        return y


class Block:
    """A layer between its norms: z = res_scale * x + gate * RMSNorm(layer(RMSNorm(x) * w_pre)) * w_post,
    the layer being a Layer or any callable of the normed rows.  Forward only: z is detached from x and
    the weights (deamoe_postnorm_backward and deamoe_prenorm_backward give the norms' gradients)."""

    def __init__(self, layer, w_pre, w_post, gate=None, res_scale: float = 1.0, eps: float = 1e-6,
                 w_next=None):
        self.layer, self.w_pre, self.w_post, self.gate = layer, w_pre, w_post, gate
        self.res_scale, self.eps, self.w_next = res_scale, eps, w_next

    def __call__(self, x, u=None, stream=None, **kw):
        """z, or with w_next (z, u): u is the next block's normed input, which its call takes in
        place of norming x again.  Further keyword arguments go to the layer, which runs with x's
        device and the call's stream as the current ones."""
        with _on("Block", x.get_device(), stream):
            if u is None:
                u = torch.empty_like(x)
                deamoe_prenorm(x, self.w_pre, u, eps=self.eps)
            y, z = self.layer(u, **kw), torch.empty_like(x)
            nxt = torch.empty_like(x) if self.w_next is not None else None
            deamoe_postnorm(x, y, self.w_post, z, gate=self.gate, res_scale=self.res_scale,
                            w_next=self.w_next, u=nxt, eps=self.eps)
            return z if nxt is None else (z, nxt)
