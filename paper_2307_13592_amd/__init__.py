"""Python binding of libmgn (include/mgn.h): one MeshGraphNets training step
on one MI355X mesh partition.

The functions here carry the C ABI's names and only marshal arguments
(torch device tensors -> device pointers, numpy arrays -> host pointers,
status codes -> exceptions).  Every step of the computation runs in the HIP
kernels of libmgn.so; there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import functools
import os

import numpy as np

from . import build as _build

MGN_OK, MGN_E_ARG, MGN_E_GRAPH, MGN_E_STATE, MGN_E_NOMEM, MGN_E_HIP, MGN_E_UNSUPPORTED = range(7)
MGN_FP32, MGN_BF16, MGN_E4M3 = 0, 1, 2
STATUS_NAMES = ["MGN_OK", "MGN_E_ARG", "MGN_E_GRAPH", "MGN_E_STATE", "MGN_E_NOMEM", "MGN_E_HIP", "MGN_E_UNSUPPORTED"]

# every symbol include/mgn.h declares
EXPORTS = ["mgn_create", "mgn_destroy", "mgn_last_error", "mgn_param_count", "mgn_set_params", "mgn_sgd_step",
           "mgn_get_params",
           "mgn_partition_slabs", "mgn_graph_sizes", "mgn_graph_build", "mgn_graph_validate", "mgn_set_recompute",
           "mgn_set_inference", "mgn_set_h1_stash", "mgn_rollout_update", "mgn_norm_accumulate", "mgn_norm_apply",
           "mgn_workspace_size",
           "mgn_forward", "mgn_backward", "mgn_forward_begin", "mgn_forward_block", "mgn_forward_end",
           "mgn_backward_begin", "mgn_backward_block", "mgn_backward_end", "mgn_halo_masks", "mgn_copy_latents",
           "mgn_add_latent_grads", "mgn_lockstep_forward", "mgn_lockstep_backward", "mgn_mse_grad",
           "mgn_mse_grad_global", "mgn_timing_enable", "mgn_timing_read", "mgn_forward_noalloc",
           "mgn_rows_store8", "mgn_rows_load8", "mgn_rms_norm", "mgn_rms_norm_grad", "mgn_gated_scan_work",
           "mgn_gated_scan", "mgn_gated_scan_grad", "mgn_pack_latents8", "mgn_add_latent_grads8",
           "mgn_lockstep_forward8", "mgn_lockstep_backward8",
           "mgn_layer_norm", "mgn_layer_norm_grad", "mgn_causal_conv", "mgn_causal_conv_grad",
           "mgn_selective_scan_work", "mgn_selective_scan", "mgn_selective_scan_grad_work", "mgn_selective_scan_grad",
           "mgn_grads_create", "mgn_grads_destroy", "mgn_grads_work", "mgn_grad_norm", "mgn_grad_clip"]
TIMERS = ["encode", "edge_fwd", "node_fwd", "decode", "edge_bwd", "node_bwd", "input_grad", "weight_grad",
          "other", "node_proj", "exchange"]


class MgnError(RuntimeError):
    def __init__(self, status: int, msg: str):
        self.status = status
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__(f"{name}: {msg}")


class mgn_config(C.Structure):
    _fields_ = [("latent", C.c_int32), ("n_blocks", C.c_int32), ("depth", C.c_int32), ("node_in", C.c_int32),
                ("edge_in", C.c_int32), ("node_out", C.c_int32), ("precision", C.c_int32), ("ln_eps", C.c_float)]


class mgn_halo_link(C.Structure):
    _fields_ = [("part", C.c_int32), ("owner", C.c_int32), ("recv_idx", C.c_void_p), ("send_rows", C.c_void_p),
                ("n", C.c_int64)]


class mgn_graph(C.Structure):
    _fields_ = [("n_owned", C.c_int64), ("n_halo", C.c_int64), ("n_edges", C.c_int64), ("row_ptr", C.c_void_p),
                ("send", C.c_void_p), ("trow_ptr", C.c_void_p), ("tedge", C.c_void_p)]


class mgn_ssm(C.Structure):
    _fields_ = [("steps", C.c_int64), ("rows", C.c_int64), ("cols", C.c_int32), ("n", C.c_int32), ("type", C.c_int32),
                ("softplus", C.c_int32), ("x", C.c_void_p), ("dt", C.c_void_p), ("B", C.c_void_p), ("C", C.c_void_p),
                ("z", C.c_void_p), ("A", C.c_void_p), ("D", C.c_void_p), ("dt_bias", C.c_void_p),
                ("starts", C.c_void_p)]


class mgn_ssm_grads(C.Structure):
    _fields_ = [("dx", C.c_void_p), ("ddt", C.c_void_p), ("dB", C.c_void_p), ("dC", C.c_void_p), ("dz", C.c_void_p),
                ("dA", C.c_void_p), ("dD", C.c_void_p), ("d_bias", C.c_void_p), ("accumulate", C.c_int32)]


class mgn_grad(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("type", C.c_int32)]


_byref = C.byref  # (C is also a name of the selective scan's)
_lib = None


def lib() -> C.CDLL:
    """Loads libmgn.so, building it first only if no build exists."""
    global _lib
    if _lib is None:
        if not os.path.exists(_build.LIB):
            _build.build()
        L = C.CDLL(_build.LIB)
        for name in EXPORTS:
            getattr(L, name)
        vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int32
        sig = {
            "mgn_create": (C.c_int, [vp, vp]),
            "mgn_destroy": (None, [vp]),
            "mgn_last_error": (C.c_char_p, [vp]),
            "mgn_param_count": (i64, [vp]),
            "mgn_set_params": (C.c_int, [vp, vp, C.c_int, vp]),
            "mgn_get_params": (C.c_int, [vp, vp, C.c_int, vp]),
            "mgn_sgd_step": (C.c_int, [vp, vp, C.c_float, vp]),
            "mgn_partition_slabs": (C.c_int, [vp, i64, i32, vp]),
            "mgn_graph_sizes": (C.c_int, [vp, vp, i64, vp, i64, i32, vp]),
            "mgn_graph_build": (C.c_int, [vp, vp, i64, vp, i64, i32, vp, vp, vp, vp, vp, vp]),
            "mgn_graph_validate": (C.c_int, [vp, vp, vp]),
            "mgn_set_recompute": (C.c_int, [vp, i32, i64]),
            "mgn_set_inference": (C.c_int, [vp, i32]),
            "mgn_set_h1_stash": (C.c_int, [vp, i32]),
            "mgn_rollout_update": (C.c_int, [vp, i64, i32, vp, i32, i32, vp]),
            "mgn_norm_accumulate": (C.c_int, [vp, i64, i32, vp, vp, vp]),
            "mgn_norm_apply": (C.c_int, [vp, i64, i32, vp, C.c_double, vp, vp]),
            "mgn_workspace_size": (C.c_int, [vp, vp, vp]),
            "mgn_forward": (C.c_int, [vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]),
            "mgn_backward": (C.c_int, [vp, vp, vp, C.c_int, vp, vp]),
            "mgn_forward_noalloc": (C.c_int, [vp, vp, vp, vp, vp, vp, vp]),
            "mgn_forward_begin": (C.c_int, [vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]),
            "mgn_forward_block": (C.c_int, [vp, vp]),
            "mgn_forward_end": (C.c_int, [vp, vp]),
            "mgn_backward_begin": (C.c_int, [vp, vp, vp, C.c_int, vp, vp]),
            "mgn_backward_block": (C.c_int, [vp, vp]),
            "mgn_backward_end": (C.c_int, [vp, vp]),
            "mgn_halo_masks": (C.c_int, [vp, i64, i64, vp, i64, vp, i64, i32, vp, vp, vp]),
            "mgn_copy_latents": (C.c_int, [vp, vp, vp, i64, vp, i64, vp]),
            "mgn_add_latent_grads": (C.c_int, [vp, vp, i64, vp, vp, i64, vp]),
            "mgn_lockstep_forward": (C.c_int, [i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp]),
            "mgn_lockstep_backward": (C.c_int, [i32, vp, vp, vp, C.c_int, vp, vp, i32, vp]),
            "mgn_rows_store8": (C.c_int, [vp, i32, i64, i32, vp, vp, i64, vp, vp, i64, vp]),
            "mgn_rows_load8": (C.c_int, [vp, vp, i64, i32, vp, vp, i64, vp, i32, i64, i32, vp]),
            "mgn_rms_norm": (C.c_int, [vp, vp, i32, i64, i32, vp, C.c_float, vp, vp, i32, vp, vp]),
            "mgn_rms_norm_grad": (C.c_int, [vp, i32, vp, C.c_float, vp, vp, i64, i32, vp, vp, i32, vp, vp]),
            "mgn_gated_scan_work": (C.c_int, [i64, i64, i32, vp]),
            "mgn_gated_scan": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, i64, i64, i32, vp, vp, vp, C.c_size_t, vp]),
            "mgn_gated_scan_grad": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, i64, i64, i32, vp, vp, vp, vp,
                                              C.c_size_t, vp]),
            "mgn_pack_latents8": (C.c_int, [vp, vp, i64, vp, vp, i32, vp]),
            "mgn_add_latent_grads8": (C.c_int, [vp, vp, vp, i32, vp, i64, vp]),
            "mgn_lockstep_forward8": (C.c_int, [i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, i64, i32, vp]),
            "mgn_layer_norm": (C.c_int, [vp, vp, i32, i64, i32, vp, vp, C.c_float, vp, vp, i32, vp, vp]),
            "mgn_layer_norm_grad": (C.c_int, [vp, i32, vp, C.c_float, vp, vp, i64, i32, vp, vp, vp, i32, vp, vp]),
            "mgn_causal_conv": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, i64, i64, i32, i32, vp, vp, vp]),
            "mgn_causal_conv_grad": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, vp, vp, i64, i64, i32, i32, vp, vp, vp, i32,
                                               vp, vp, vp]),
            "mgn_selective_scan_work": (C.c_int, [i64, i64, i32, i32, vp]),
            "mgn_selective_scan": (C.c_int, [vp, vp, vp, vp, vp, vp, C.c_size_t, vp]),
            "mgn_selective_scan_grad_work": (C.c_int, [i64, i64, i32, i32, vp]),
            "mgn_selective_scan_grad": (C.c_int, [vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]),
            "mgn_grads_create": (C.c_int, [vp, i64, vp]),
            "mgn_grads_destroy": (None, [vp]),
            "mgn_grads_work": (C.c_int, [vp, vp]),
            "mgn_grad_norm": (C.c_int, [vp, vp, vp, C.c_size_t, vp]),
            "mgn_grad_clip": (C.c_int, [vp, C.c_float, i32, vp, vp, C.c_size_t, vp]),
            "mgn_lockstep_backward8": (C.c_int, [i32, vp, vp, vp, C.c_int, vp, vp, i32, vp, vp, i64, i32, vp]),
            "mgn_mse_grad": (C.c_int, [vp, vp, vp, i64, i32, vp, vp, vp]),
            "mgn_mse_grad_global": (C.c_int, [vp, vp, vp, i64, i32, i64, vp, vp, vp]),
            "mgn_timing_enable": (C.c_int, [vp, C.c_int]),
            "mgn_timing_read": (C.c_int, [vp, C.c_int, vp, vp]),
        }
        for name, (res, args) in sig.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


# ------------------------------------------------------------ marshalling ---
def _dev(t):
    """Device pointer of a torch tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return C.c_void_p(t.data_ptr())


def _devt(t, dtype, name: str, shape=None, numel=None, min_numel=None):
    """_dev with the checks the C ABI cannot make (it takes no dtype, and
    no length for some buffers): torch dtype, exact shape, exact or minimum
    element count."""
    if t is None:
        raise ValueError(f"{name}: expected a device tensor, got None")
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name}: expected {numel} elements, got {t.numel()}")
    if min_numel is not None and t.numel() < min_numel:
        raise ValueError(f"{name}: expected at least {min_numel} elements, got {t.numel()}")
    return _dev(t)


def _host(a, dtype):
    if a is None:
        return None, None
    a = np.ascontiguousarray(a, dtype=dtype)
    return a, a.ctypes.data_as(C.c_void_p)


def _stream(stream):
    if stream is None:
        import torch
        return C.c_void_p(torch.cuda.current_stream().cuda_stream)
    return C.c_void_p(int(stream))


def _check(st: int, model=None):
    if st != MGN_OK:
        msg = lib().mgn_last_error(model).decode()
        raise MgnError(st, msg)


# ------------------------------------------------------------------- ABI ---
def mgn_create(latent: int, n_blocks: int, depth: int, precision: int = MGN_FP32, node_in: int = 11,
               edge_in: int = 4, node_out: int = 5, ln_eps: float = 1e-5) -> C.c_void_p:
    cfg = mgn_config(latent, n_blocks, depth, node_in, edge_in, node_out, precision, ln_eps)
    h = C.c_void_p()
    _check(lib().mgn_create(C.byref(cfg), C.byref(h)))
    return h


def mgn_destroy(model) -> None:
    lib().mgn_destroy(model)


def mgn_last_error(model=None) -> str:
    return lib().mgn_last_error(model).decode()


def mgn_param_count(model) -> int:
    return int(lib().mgn_param_count(model))


def mgn_set_params(model, params, stream=None) -> None:
    """params: float32 device tensor or host array of mgn_param_count entries."""
    if hasattr(params, "is_cuda") and params.is_cuda:
        _check(lib().mgn_set_params(model, _dev(params), 1, _stream(stream)), model)
    else:
        a, p = _host(params, np.float32)
        if a.size != mgn_param_count(model):
            raise ValueError("parameter vector has the wrong length")
        _check(lib().mgn_set_params(model, p, 0, _stream(stream)), model)


def _sgd_args(model, grad, lr: float):
    """Checked arguments of mgn_sgd_step (the C ABI takes no type and no length)."""
    import torch
    if grad.numel() != mgn_param_count(model):
        raise ValueError("gradient vector has the wrong length")
    if not np.isfinite(C.c_float(lr).value):
        raise MgnError(MGN_E_ARG, "mgn_sgd_step: learning rate is not finite")
    return _devt(grad, torch.float32, "grad"), float(lr)


def mgn_sgd_step(model, grad, lr: float, stream=None) -> None:
    """params -= lr * grad on the device (grad: float32 device tensor)."""
    _check(lib().mgn_sgd_step(model, *_sgd_args(model, grad, lr), _stream(stream)), model)


def mgn_get_params(model, stream=None) -> np.ndarray:
    out = np.empty(mgn_param_count(model), np.float32)
    _check(lib().mgn_get_params(model, out.ctypes.data_as(C.c_void_p), 0, _stream(stream)), model)
    return out


def mgn_partition_slabs(key, nparts: int) -> np.ndarray:
    k, kp = _host(key, np.int32)
    part = np.empty(k.shape[0], np.int32)
    _check(lib().mgn_partition_slabs(kp, k.shape[0], nparts, part.ctypes.data_as(C.c_void_p)))
    return part


def mgn_graph_sizes(send, recv, part, n_nodes: int, p: int):
    s, sp = _host(send, np.int32)
    r, rp = _host(recv, np.int32)
    pa, pp = _host(part, np.int32)
    sz = np.zeros(3, np.int64)
    _check(lib().mgn_graph_sizes(sp, rp, s.shape[0], pp, n_nodes, p, sz.ctypes.data_as(C.c_void_p)))
    return tuple(int(x) for x in sz)


def mgn_graph_build(send, recv, part, n_nodes: int, p: int) -> dict:
    """Host-side build of part p's local graph; returns numpy arrays."""
    no, nh, ne = mgn_graph_sizes(send, recv, part, n_nodes, p)
    s, sp = _host(send, np.int32)
    r, rp = _host(recv, np.int32)
    pa, pp = _host(part, np.int32)
    g = dict(n_owned=no, n_halo=nh, n_edges=ne, row_ptr=np.empty(no + 1, np.int32), send=np.empty(ne, np.int32),
             eperm=np.empty(ne, np.int32), trow_ptr=np.empty(no + nh + 1, np.int32), tedge=np.empty(ne, np.int32),
             l2g=np.empty(no + nh, np.int32))
    ptr = lambda k: g[k].ctypes.data_as(C.c_void_p)
    _check(lib().mgn_graph_build(sp, rp, s.shape[0], pp, n_nodes, p, ptr("row_ptr"), ptr("send"), ptr("eperm"),
                                 ptr("trow_ptr"), ptr("tedge"), ptr("l2g")))
    return g


def graph_struct(dg: dict) -> mgn_graph:
    """mgn_graph from a dict of sizes and int32 device tensors."""
    return mgn_graph(dg["n_owned"], dg["n_halo"], dg["n_edges"], _dev(dg["row_ptr"]), _dev(dg["send"]),
                     _dev(dg["trow_ptr"]), _dev(dg["tedge"]))


def mgn_graph_validate(model, graph: mgn_graph, stream=None) -> None:
    _check(lib().mgn_graph_validate(model, C.byref(graph), _stream(stream)), model)


def mgn_set_recompute(model, interval: int, chunk_edges: int = 0) -> None:
    _check(lib().mgn_set_recompute(model, int(interval), int(chunk_edges)), model)


def mgn_set_inference(model, on: bool = True) -> None:
    _check(lib().mgn_set_inference(model, int(bool(on))), model)


def mgn_set_h1_stash(model, n_blocks: int) -> None:
    _check(lib().mgn_set_h1_stash(model, int(n_blocks)), model)


MGN_NORM_MAX_COLS = 64
MGN_NORM_WORK_PER_COL = 1024


def mgn_norm_accumulate(x, stats, work, stream=None) -> None:
    """Adds the rows of x (device float32 [rows][cols]) to the running
    statistics `stats` (device float64 [1 + 2 cols]); work: device float64
    scratch of at least MGN_NORM_WORK_PER_COL * cols."""
    import torch
    if x.dim() != 2:
        raise ValueError("x: expected [rows][cols]")
    rows, cols = x.shape
    _check(lib().mgn_norm_accumulate(_devt(x, torch.float32, "x"), rows, cols,
                                     _devt(stats, torch.float64, "stats", numel=1 + 2 * cols),
                                     _devt(work, torch.float64, "work", min_numel=MGN_NORM_WORK_PER_COL * cols),
                                     _stream(stream)))


def mgn_norm_apply(x, stats, out, eps: float = 1e-8, stream=None) -> None:
    """out = (x - mean) / max(std, eps) per column (device float32; out may be x)."""
    import torch
    if x.dim() != 2:
        raise ValueError("x: expected [rows][cols]")
    rows, cols = x.shape
    _check(lib().mgn_norm_apply(_devt(x, torch.float32, "x"), rows, cols,
                                _devt(stats, torch.float64, "stats", numel=1 + 2 * cols), C.c_double(eps),
                                _devt(out, torch.float32, "out", shape=(rows, cols)), _stream(stream)))


def mgn_rollout_update(out, node_feat, col0: int = 3, stream=None) -> None:
    """node_feat[:, col0:col0 + out.shape[1]] += out (device tensors)."""
    import torch
    n, d = out.shape
    if node_feat.dim() != 2 or node_feat.shape[0] != n:
        raise ValueError("node_feat: expected [n][features] with the rows of out")
    _check(lib().mgn_rollout_update(_devt(out, torch.float32, "out"), n, d,
                                    _devt(node_feat, torch.float32, "node_feat"), int(node_feat.shape[1]), int(col0),
                                    _stream(stream)))


MGN_ROW_MAX_COLS = 8192
MGN_ROWS8_BLOCK = 128
MGN_RMS_WORK_PER_COL = 1024


def rows8_blocks(cols: int) -> int:
    """Scales of an 8-bit row of `cols` columns."""
    return -(-cols // MGN_ROWS8_BLOCK)


def _type(t, name: str, e4m3: bool = False) -> int:
    """Storage type of a row array from its torch dtype (uint8: 8-bit codes)."""
    import torch
    if t is None:
        raise ValueError(f"{name}: expected a device tensor, got None")
    if t.dtype is torch.float32:
        return MGN_FP32
    if t.dtype is torch.bfloat16:
        return MGN_BF16
    if e4m3 and t.dtype is torch.uint8:
        return MGN_E4M3
    raise ValueError(f"{name}: unsupported storage type {t.dtype}")


def _shape(t, name: str, dims: int = 2):
    if t is None or t.dim() != dims:
        raise ValueError(f"{name}: expected {'[steps]' if dims == 3 else ''}[rows][cols]")
    return t.shape


def _arr(t, name: str, dtype, shape, dev: int):
    """Device pointer of an array of this type and shape on GPU `dev` (None ->
    NULL); _run refuses a dev that is none.  One comparison per property: these
    calls are short."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    _devt(t, dtype, name, shape=shape)  # says what is wrong, but for the device
    raise ValueError(f"{name}: expected a tensor on GPU {dev}, got one on {t.device}")


def _need(p, name: str):
    if p is None:
        raise ValueError(f"{name}: expected a device tensor, got None")
    return p


def _run(fn: str, dev: int, stream, *args) -> None:
    """Calls the entry point fn(*args, stream) on GPU `dev`, its arrays';
    without a stream given, on the current one of that device."""
    import torch
    if dev < 0:
        raise ValueError(f"{fn}: expected device tensors")
    f = getattr(lib(), fn)
    if dev == torch.cuda.current_device():
        st = f(*args, torch._C._cuda_getCurrentRawStream(dev) if stream is None else int(stream))
    else:
        with torch.cuda.device(dev):
            st = f(*args, torch.cuda.current_stream().cuda_stream if stream is None else int(stream))
    if st != MGN_OK:
        _check(st)


def _on(stream, device):
    """Context in which torch allocates on `stream` (None: the current one): what
    a call on that stream writes must come from there, or the allocator could
    hand it out while work queued elsewhere still uses it."""
    import torch
    if stream is None:
        return contextlib.nullcontext()
    if int(stream) == 0:  # (torch takes no handle of 0 for a stream)
        return torch.cuda.stream(torch.cuda.default_stream(device))
    return torch.cuda.stream(torch.cuda.ExternalStream(int(stream), device=device))


def _scratch(nbytes: int, dev: int, stream):
    """Device scratch for one call on `stream`: from torch's allocator, on that
    stream, so that it is not handed out again before the call has run (and
    belongs to a HIP graph that records the call)."""
    import torch
    device = torch.device("cuda", dev) if dev >= 0 else None
    if stream is None or device is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with _on(stream, device):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _lists(a, b, rows: int, dev):
    """Pointers and length of two int32 index lists, either of them None."""
    import torch
    n = a.numel() if a is not None else b.numel() if b is not None else rows
    return _arr(a, "index list", torch.int32, (n,), dev), _arr(b, "index list", torch.int32, (n,), dev), n


def mgn_rows_store8(src, q, scale, src_rows=None, slots=None, stream=None) -> None:
    """Stores rows of src (device float32 or bfloat16 [n_src][cols]) in 8 bits:
    slot slots[i] of q (uint8 [n_slots][cols]) and scale (float32
    [n_slots][rows8_blocks(cols)]) takes row src_rows[i].  src_rows, slots:
    int32 device tensors of one length, or None for 0, 1, 2, ...; without
    either, every row of src is stored."""
    import torch
    n_src, cols = _shape(src, "src")
    n_slots, dev = _shape(q, "q")[0], src.get_device()
    rows, at, n = _lists(src_rows, slots, n_src, dev)
    _run("mgn_rows_store8", dev, stream, _need(_arr(src, "src", src.dtype, (n_src, cols), dev), "src"),
         _type(src, "src"), n_src, cols, rows, at, n, _arr(q, "q", torch.uint8, (n_slots, cols), dev),
         _need(_arr(scale, "scale", torch.float32, (n_slots, rows8_blocks(cols)), dev), "scale"), n_slots)


def mgn_rows_load8(q, scale, dst, slots=None, dst_rows=None, add: bool = False, stream=None) -> None:
    """Reads 8-bit rows back: row dst_rows[i] of dst (device float32 or
    bfloat16 [n_dst][cols]) takes the values of slot slots[i] (add: the sum of
    them and of what it holds, float32 only).  Without index tensors every
    slot is read."""
    import torch
    n_slots, cols = _shape(q, "q")
    n_dst, dev = _shape(dst, "dst")[0], q.get_device()
    rows, at, n = _lists(dst_rows, slots, n_slots, dev)
    _run("mgn_rows_load8", dev, stream, _need(_arr(q, "q", torch.uint8, (n_slots, cols), dev), "q"),
         _need(_arr(scale, "scale", torch.float32, (n_slots, rows8_blocks(cols)), dev), "scale"), n_slots, cols, at,
         rows, n, _arr(dst, "dst", dst.dtype, (n_dst, cols), dev), _type(dst, "dst"), n_dst, 1 if add else 0)


def mgn_rms_norm(x, weight, y, res=None, total=None, y_scale=None, eps: float = 1e-6, stream=None) -> None:
    """y = t / sqrt(mean(t^2) + eps) * weight for t = x + res, rows of device
    tensors.  x, res, total: float32 or bfloat16, one type; total takes t.  y:
    float32, bfloat16, or uint8 for 8-bit rows with their scales in y_scale.
    weight: float32 [cols] or None."""
    import torch
    shape = rows, cols = _shape(x, "x")
    dev, dt = x.get_device(), x.dtype
    yt = _type(y, "y", e4m3=True)
    _run("mgn_rms_norm", dev, stream, _arr(x, "x", dt, shape, dev), _arr(res, "res", dt, shape, dev), _type(x, "x"),
         rows, cols, _arr(weight, "weight", torch.float32, (cols,), dev), eps, _arr(total, "total", dt, shape, dev),
         _arr(y, "y", y.dtype, shape, dev), yt,
         None if y_scale is None else _arr(y_scale, "y_scale", torch.float32, (rows, rows8_blocks(cols)), dev))


def mgn_rms_norm_grad(total, weight, dy, dx, dweight=None, d_total=None, accumulate: bool = False, work=None,
                      eps: float = 1e-6, stream=None) -> None:
    """Backward of mgn_rms_norm: dx (the gradient of x and of res) and dweight
    (float32 [cols], overwritten or added to) from the normalised sum `total`,
    dy and the gradient d_total that reaches the sum otherwise.  work: float32
    scratch of MGN_RMS_WORK_PER_COL * cols for dweight (None: allocated)."""
    import torch
    shape = rows, cols = _shape(total, "total")
    dev, dt = total.get_device(), total.dtype
    pt = _arr(total, "total", dt, shape, dev)
    if work is not None:
        pw = _devt(work, torch.float32, "work", min_numel=MGN_RMS_WORK_PER_COL * cols)
        if work.get_device() != dev:
            raise ValueError(f"work: expected a tensor on GPU {dev}, got one on {work.device}")
    elif dweight is not None:
        work = _scratch(4 * MGN_RMS_WORK_PER_COL * cols, dev, stream)
        pw = work.data_ptr()
    else:
        pw = None
    _run("mgn_rms_norm_grad", dev, stream, pt, _type(total, "total"),
         _arr(weight, "weight", torch.float32, (cols,), dev), eps, _need(_arr(dy, "dy", dt, shape, dev), "dy"),
         _arr(d_total, "d_total", dt, shape, dev), rows, cols, _need(_arr(dx, "dx", dt, shape, dev), "dx"),
         _arr(dweight, "dweight", torch.float32, (cols,), dev), 1 if accumulate else 0, pw)


@functools.lru_cache(maxsize=256)
def mgn_gated_scan_work(steps: int, rows: int, cols: int) -> int:
    """Bytes of device scratch mgn_gated_scan and its backward need."""
    n = C.c_size_t()
    _check(lib().mgn_gated_scan_work(int(steps), int(rows), int(cols), C.byref(n)))
    return int(n.value)


def _scan_args(g, x, x_scale, starts, h0, work, stream):
    """Marshalled arguments the recurrence and its backward share."""
    import torch
    shape = T, rows, cols = _shape(g, "g", 3)
    dev = g.get_device()
    xt = _type(x, "x", e4m3=True)
    if xt != MGN_E4M3 and x.dtype is not g.dtype:
        raise ValueError(f"x: expected {g.dtype} (as g) or uint8 codes, got {x.dtype}")
    head = (_arr(g, "g", g.dtype, shape, dev), _type(g, "g"), _arr(x, "x", x.dtype, shape, dev), xt,
            None if x_scale is None else _arr(x_scale, "x_scale", torch.float32, (T, rows, rows8_blocks(cols)), dev),
            None if starts is None else _arr(starts, "starts", torch.uint8, (T,), dev),
            _arr(h0, "h0", torch.float32, (rows, cols), dev))
    if work is None:
        need = mgn_gated_scan_work(T, rows, cols)
        if need:
            work = _scratch(need, dev, stream)
        return shape, dev, head, (work.data_ptr() if need else None, need), work
    pw = _dev(work)
    if work.get_device() != dev:
        raise ValueError(f"work: expected a tensor on GPU {dev}, got one on {work.device}")
    return shape, dev, head, (pw, work.numel() * work.element_size()), work


def mgn_gated_scan(g, x, h=None, h_last=None, h0=None, starts=None, x_scale=None, work=None, stream=None) -> None:
    """h_t = sigmoid(g_t) h_{t-1} + sigmoid(-g_t) x_t along the first axis of
    device tensors [steps][rows][cols].  g, x: float32 or bfloat16, or x uint8
    codes with x_scale; h (all states) and h_last (the last; it may be h0):
    float32, either may be None; starts: uint8 [steps].  work: device scratch of
    mgn_gated_scan_work bytes (None: allocated)."""
    import torch
    shape, dev, head, tail, keep = _scan_args(g, x, x_scale, starts, h0, work, stream)
    T, rows, cols = shape
    _run("mgn_gated_scan", dev, stream, *head, T, rows, cols, _arr(h, "h", torch.float32, shape, dev),
         _arr(h_last, "h_last", torch.float32, (rows, cols), dev), *tail)


def mgn_gated_scan_grad(g, x, h, dg, dx, dh=None, dh_last=None, dh0=None, h0=None, starts=None, x_scale=None,
                        work=None, stream=None) -> None:
    """Backward of mgn_gated_scan from its arguments, its h and the float32
    gradients dh [steps][rows][cols] and dh_last [rows][cols]: dg (g's type), dx
    (x's type; g's for 8-bit x) and dh0 (float32, or None; it may be dh_last)."""
    import torch
    shape, dev, head, tail, keep = _scan_args(g, x, x_scale, starts, h0, work, stream)
    T, rows, cols = shape
    one, f32, dt = (rows, cols), torch.float32, g.dtype
    _run("mgn_gated_scan_grad", dev, stream, *head, _need(_arr(h, "h", f32, shape, dev), "h"),
         _arr(dh, "dh", f32, shape, dev), _arr(dh_last, "dh_last", f32, one, dev), T, rows, cols,
         _need(_arr(dg, "dg", dt, shape, dev), "dg"), _need(_arr(dx, "dx", dt, shape, dev), "dx"),
         _arr(dh0, "dh0", f32, one, dev), *tail)


MGN_LAYER_WORK_PER_COL = 2048
MGN_CONV_MAX_WIDTH, MGN_CONV_PARTS = 8, 1024
MGN_STATES_MAX, MGN_MARK_STEPS = 64, 8


def _given(work, name: str, nbytes: int, dev: int, stream):
    """Pointer and bytes of a call's scratch, and the tensor that holds it: the
    caller's, or one of nbytes."""
    if work is None:
        work = _scratch(nbytes, dev, stream) if nbytes else None
        return (work.data_ptr() if nbytes else None), nbytes, work
    p = _dev(work)
    if work.get_device() != dev:
        raise ValueError(f"{name}: expected a tensor on GPU {dev}, got one on {work.device}")
    return p, work.numel() * work.element_size(), work


def mgn_layer_norm(x, weight, bias, y, res=None, total=None, y_scale=None, eps: float = 1e-5, stream=None) -> None:
    """y = (t - mean(t)) / sqrt(var(t) + eps) * weight + bias for t = x + res, rows
    of device tensors.  x, res, total: float32 or bfloat16, one type; total takes t.
    y: float32, bfloat16, or uint8 for 8-bit rows with their scales in y_scale.
    weight, bias: float32 [cols] or None."""
    import torch
    shape = rows, cols = _shape(x, "x")
    dev, dt, f32 = x.get_device(), x.dtype, torch.float32
    yt = _type(y, "y", e4m3=True)
    _run("mgn_layer_norm", dev, stream, _arr(x, "x", dt, shape, dev), _arr(res, "res", dt, shape, dev), _type(x, "x"),
         rows, cols, _arr(weight, "weight", f32, (cols,), dev), _arr(bias, "bias", f32, (cols,), dev), eps,
         _arr(total, "total", dt, shape, dev), _arr(y, "y", y.dtype, shape, dev), yt,
         None if y_scale is None else _arr(y_scale, "y_scale", f32, (rows, rows8_blocks(cols)), dev))


def mgn_layer_norm_grad(total, weight, dy, dx, dweight=None, dbias=None, d_total=None, accumulate: bool = False,
                        work=None, eps: float = 1e-5, stream=None) -> None:
    """Backward of mgn_layer_norm: dx (the gradient of x and of res), dweight and
    dbias (float32 [cols], overwritten or added to) from the normalised sum `total`,
    dy and the gradient d_total that reaches the sum otherwise.  work: float32
    scratch of MGN_LAYER_WORK_PER_COL * cols for dweight and dbias (None:
    allocated)."""
    import torch
    shape = rows, cols = _shape(total, "total")
    dev, dt, f32 = total.get_device(), total.dtype, torch.float32
    pt = _arr(total, "total", dt, shape, dev)
    sums = dweight is not None or dbias is not None
    if work is not None:
        _devt(work, f32, "work", min_numel=MGN_LAYER_WORK_PER_COL * cols)
    pw, _, keep = _given(work, "work", 4 * MGN_LAYER_WORK_PER_COL * cols if sums else 0, dev, stream)
    _run("mgn_layer_norm_grad", dev, stream, pt, _type(total, "total"), _arr(weight, "weight", f32, (cols,), dev), eps,
         _need(_arr(dy, "dy", dt, shape, dev), "dy"), _arr(d_total, "d_total", dt, shape, dev), rows, cols,
         _need(_arr(dx, "dx", dt, shape, dev), "dx"), _arr(dweight, "dweight", f32, (cols,), dev),
         _arr(dbias, "dbias", f32, (cols,), dev), 1 if accumulate else 0, pw)


def _conv_args(x, weight, bias, past, starts):
    """Marshalled arguments the convolution and its backward share."""
    import torch
    shape = T, rows, cols = _shape(x, "x", 3)
    dev, f32 = x.get_device(), torch.float32
    if weight is None or weight.dim() != 2:
        raise ValueError("weight: expected [cols][width]")
    width = weight.shape[1]
    if not 1 <= width <= MGN_CONV_MAX_WIDTH:
        raise ValueError(f"weight: expected 1 .. {MGN_CONV_MAX_WIDTH} weights a column")
    before = (width - 1, rows, cols)
    return shape, dev, width, before, (
        _arr(x, "x", x.dtype, shape, dev), _type(x, "x"), _arr(weight, "weight", f32, (cols, width), dev), width,
        _arr(bias, "bias", f32, (cols,), dev), None if starts is None else _arr(starts, "starts", torch.uint8, (T,), dev),
        _arr(past, "past", x.dtype, before, dev))


def mgn_causal_conv(x, weight, y, bias=None, past=None, past_out=None, starts=None, silu: bool = False,
                    stream=None) -> None:
    """v_t = bias + sum_k weight[:, width - 1 - k] x_{t-k} along the first axis of
    device tensors [steps][rows][cols], y = v or (silu) v sigmoid(v).  x, y: float32
    or bfloat16; weight: float32 [cols][width]; bias: float32 [cols] or None; past,
    past_out [width - 1][rows][cols] of x's type: the inputs before the first step
    and those that the next window's steps see (past_out may be past), either None;
    starts: uint8 [steps]."""
    shape, dev, width, before, head = _conv_args(x, weight, bias, past, starts)
    T, rows, cols = shape
    _run("mgn_causal_conv", dev, stream, *head, T, rows, cols, 1 if silu else 0,
         _need(_arr(y, "y", x.dtype, shape, dev), "y"), _arr(past_out, "past_out", x.dtype, before, dev))


def mgn_causal_conv_grad(x, weight, dy, dx, dweight=None, dbias=None, bias=None, past=None, d_past=None,
                         d_past_out=None, starts=None, silu: bool = False, accumulate: bool = False, work=None,
                         stream=None) -> None:
    """Backward of mgn_causal_conv from its arguments, dy and d_past_out (float32
    [width - 1][rows][cols], or None): dx (x's type), dweight, dbias (float32,
    overwritten or added to) and d_past (float32), each of them or None.  work:
    float32 scratch of MGN_CONV_PARTS * cols * (width + 1) for dweight and dbias
    (None: allocated)."""
    call, keep = _causal_conv_grad(x, weight, dy, dx, dweight, dbias, bias, past, d_past, d_past_out, starts, silu,
                                   accumulate, work, stream)
    _run(*call)


def _causal_conv_grad(x, weight, dy, dx, dweight, dbias, bias, past, d_past, d_past_out, starts, silu, accumulate, work,
                      stream):
    """The checks and marshalling of mgn_causal_conv_grad: _run's arguments, and last the
    scratch that it keeps.  (Of several calls in a row none runs if one would be refused.)"""
    import torch
    shape, dev, width, before, head = _conv_args(x, weight, bias, past, starts)
    T, rows, cols = shape
    f32, floats = torch.float32, MGN_CONV_PARTS * cols * (width + 1)
    sums = dweight is not None or dbias is not None
    if work is not None:
        _devt(work, f32, "work", min_numel=floats)
    pw, _, keep = _given(work, "work", 4 * floats if sums else 0, dev, stream)
    args = (*head, _need(_arr(dy, "dy", x.dtype, shape, dev), "dy"), _arr(d_past_out, "d_past_out", f32, before, dev), T,
            rows, cols, 1 if silu else 0, _need(_arr(dx, "dx", x.dtype, shape, dev), "dx"),
            _arr(dweight, "dweight", f32, (cols, width), dev), _arr(dbias, "dbias", f32, (cols,), dev),
            1 if accumulate else 0, _arr(d_past, "d_past", f32, before, dev), pw)
    return ("mgn_causal_conv_grad", dev, stream, *args), keep


@functools.lru_cache(maxsize=256)
def mgn_selective_scan_work(steps: int, rows: int, cols: int, n: int) -> int:
    """Bytes of device scratch mgn_selective_scan needs."""
    b = C.c_size_t()
    _check(lib().mgn_selective_scan_work(int(steps), int(rows), int(cols), int(n), C.byref(b)))
    return int(b.value)


@functools.lru_cache(maxsize=256)
def mgn_selective_scan_grad_work(steps: int, rows: int, cols: int, n: int) -> int:
    """Bytes of device scratch mgn_selective_scan_grad needs."""
    b = C.c_size_t()
    _check(lib().mgn_selective_scan_grad_work(int(steps), int(rows), int(cols), int(n), C.byref(b)))
    return int(b.value)


def _ssm_args(x, dt, A, B, C_, D, dt_bias, z, starts, softplus):
    """The scan's shape, device and argument record."""
    import torch
    shape = T, rows, cols = _shape(x, "x", 3)
    dev, ty, f32 = x.get_device(), x.dtype, torch.float32
    if A is None or A.dim() != 2 or not 1 <= A.shape[1] <= MGN_STATES_MAX:
        raise ValueError(f"A: expected [cols][n], 1 <= n <= {MGN_STATES_MAX}")
    n = A.shape[1]
    return shape, dev, n, mgn_ssm(
        T, rows, cols, n, _type(x, "x"), 1 if softplus else 0, _arr(x, "x", ty, shape, dev),
        _need(_arr(dt, "dt", ty, shape, dev), "dt"), _need(_arr(B, "B", ty, (T, rows, n), dev), "B"),
        _need(_arr(C_, "C", ty, (T, rows, n), dev), "C"), _arr(z, "z", ty, shape, dev), _arr(A, "A", f32, (cols, n), dev),
        _arr(D, "D", f32, (cols,), dev), _arr(dt_bias, "dt_bias", f32, (cols,), dev),
        None if starts is None else _arr(starts, "starts", torch.uint8, (T,), dev))


def mgn_selective_marks(x, A, stream=None):
    """The array that mgn_selective_scan leaves its states in for the backward:
    float32 [ceil(steps / MGN_MARK_STEPS)][rows][cols][n]."""
    import torch
    T, rows, cols = _shape(x, "x", 3)
    with _on(stream, x.device):
        return torch.empty((-(-T // MGN_MARK_STEPS), rows, cols, A.shape[1]), dtype=torch.float32, device=x.device)


def mgn_selective_scan(x, dt, A, B, C, y, D=None, dt_bias=None, z=None, h0=None, h_last=None, marks=None, starts=None,
                       softplus: bool = False, work=None, stream=None) -> None:
    """The selective scan along the first axis of device tensors [steps][rows][cols]:
      h_t = exp(delta A) h_{t-1} + delta x B_t,  delta = dt + dt_bias (softplus: its
      softplus),  y = (sum over the states of C_t h_t + D x) z sigmoid(z).
    x, dt, z (or None), y and B, C [steps][rows][n]: float32 or bfloat16, one type; A
    float32 [cols][n]; D, dt_bias float32 [cols] or None; h0, h_last (it may be h0)
    float32 [rows][cols][n] or None; marks of mgn_selective_marks, for the backward;
    starts: uint8 [steps].  work: device scratch of mgn_selective_scan_work bytes
    (None: allocated)."""
    call, keep = _selective_scan(x, dt, A, B, C, y, D, dt_bias, z, h0, h_last, marks, starts, softplus, work, stream)
    _run(*call)


def _selective_scan(x, dt, A, B, C, y, D, dt_bias, z, h0, h_last, marks, starts, softplus, work, stream):
    """mgn_selective_scan as _causal_conv_grad."""
    import torch
    shape, dev, n, s = _ssm_args(x, dt, A, B, C, D, dt_bias, z, starts, softplus)
    T, rows, cols = shape
    f32, state = torch.float32, (rows, cols, n)
    pw, nb, keep = _given(work, "work", mgn_selective_scan_work(T, rows, cols, n) if work is None else 0, dev, stream)
    args = (_byref(s), _arr(h0, "h0", f32, state, dev), _need(_arr(y, "y", x.dtype, shape, dev), "y"),
            _arr(h_last, "h_last", f32, state, dev), _arr(marks, "marks", f32, (-(-T // MGN_MARK_STEPS),) + state, dev),
            pw, nb)
    return ("mgn_selective_scan", dev, stream, *args), keep


def mgn_selective_scan_grad(x, dt, A, B, C, marks, dy, dx, ddt, dA, dB, dC, dD=None, d_bias=None, dz=None, D=None,
                            dt_bias=None, z=None, dh_last=None, dh0=None, starts=None, softplus: bool = False,
                            accumulate: bool = False, work=None, stream=None) -> None:
    """Backward of mgn_selective_scan from its arguments, its marks, dy and dh_last
    (float32 [rows][cols][n], or None): dx, ddt, dB, dC and (with z) dz in x's type;
    dA, dD, d_bias (float32, overwritten or added to, each of them or None); dh0
    (float32, or None; it may be dh_last).  work: device scratch of
    mgn_selective_scan_grad_work bytes (None: allocated)."""
    call, keep = _selective_scan_grad(x, dt, A, B, C, marks, dy, dx, ddt, dA, dB, dC, dD, d_bias, dz, D, dt_bias, z,
                                      dh_last, dh0, starts, softplus, accumulate, work, stream)
    _run(*call)


def _selective_scan_grad(x, dt, A, B, C, marks, dy, dx, ddt, dA, dB, dC, dD, d_bias, dz, D, dt_bias, z, dh_last, dh0,
                         starts, softplus, accumulate, work, stream):
    """mgn_selective_scan_grad as _causal_conv_grad."""
    import torch
    shape, dev, n, s = _ssm_args(x, dt, A, B, C, D, dt_bias, z, starts, softplus)
    T, rows, cols = shape
    f32, ty, state, pair = torch.float32, x.dtype, (rows, cols, n), (T, rows, n)
    g = mgn_ssm_grads(_need(_arr(dx, "dx", ty, shape, dev), "dx"), _need(_arr(ddt, "ddt", ty, shape, dev), "ddt"),
                      _need(_arr(dB, "dB", ty, pair, dev), "dB"), _need(_arr(dC, "dC", ty, pair, dev), "dC"),
                      _arr(dz, "dz", ty, shape, dev), _arr(dA, "dA", f32, (cols, n), dev),
                      _arr(dD, "dD", f32, (cols,), dev), _arr(d_bias, "d_bias", f32, (cols,), dev),
                      1 if accumulate else 0)
    pw, nb, keep = _given(work, "work", mgn_selective_scan_grad_work(T, rows, cols, n) if work is None else 0, dev,
                          stream)
    args = (_byref(s), _need(_arr(marks, "marks", f32, (-(-T // MGN_MARK_STEPS),) + state, dev), "marks"),
            _need(_arr(dy, "dy", ty, shape, dev), "dy"), _arr(dh_last, "dh_last", f32, state, dev), _byref(g),
            _arr(dh0, "dh0", f32, state, dev), pw, nb)
    return ("mgn_selective_scan_grad", dev, stream, *args), keep


def _apart(fn: str, read, written) -> None:
    """Refuses two calls in a row of which the second would read, in the tensors `read`
    (None: not there), what is written by either in the tensors `written`."""
    spans = [(p, p + t.nbytes) for t in written if (p := t.data_ptr())]
    for t in read:
        if t is not None and (p := t.data_ptr()):
            q = p + t.nbytes
            for b, e in spans:
                if p < e and b < q:
                    raise MgnError(MGN_E_ARG, f"{fn}: overlapping arrays")


class mgn_grad_list:
    """Device tensors (float32 or bfloat16, contiguous, on one GPU) whose global norm
    mgn_grad_norm and mgn_grad_clip take; outs: where the clipped ones go (None: in
    place).  It is made once for a program's gradients, stands for the memory that they
    have then, and keeps that memory."""

    def __init__(self, grads, outs=None):
        grads = list(grads)
        outs = [None] * len(grads) if outs is None else list(outs)
        # (aliases: a tensor whose .data is set to another leaves its memory here)
        grads, outs = ([None if t is None else t.detach() for t in ts] for ts in (grads, outs))
        if len(outs) != len(grads):
            raise ValueError("outs: expected one for each of grads")
        if any(g is None for g in grads):
            raise ValueError("grads: expected tensors, got None")
        self._list = None
        self.tensors, self.dev = (grads, outs), grads[0].get_device() if grads else -1
        if grads and self.dev < 0:
            raise ValueError("grads[0]: expected a device tensor")
        rec = (mgn_grad * max(len(grads), 1))()
        for k, (g, o) in enumerate(zip(grads, outs)):
            ty = _type(g, f"grads[{k}]")
            rec[k] = mgn_grad(_arr(g, f"grads[{k}]", g.dtype, g.shape, self.dev),
                              _arr(o, f"outs[{k}]", g.dtype, g.shape, self.dev), g.numel(), ty)
        p = C.c_void_p()
        _check(lib().mgn_grads_create(rec, len(grads), C.byref(p)))
        self._list, self._destroy = p, lib().mgn_grads_destroy
        n = C.c_size_t()
        _check(lib().mgn_grads_work(p, C.byref(n)))
        self.work_bytes = int(n.value)

    def __del__(self):
        if getattr(self, "_list", None):
            self._destroy(self._list)
            self._list = None


def _grads(grads, norm, work, stream):
    import torch
    keep = grads = grads if isinstance(grads, mgn_grad_list) else mgn_grad_list(grads)
    dev = grads.dev if grads.dev >= 0 else norm.get_device()
    pn = _need(_arr(norm, "norm", torch.float32, (1,), dev), "norm")
    pw, nb, scratch = _given(work, "work", grads.work_bytes if work is None else 0, dev, stream)
    return dev, grads._list, pn, (pw, nb), (keep, scratch)


def mgn_grad_norm(grads, norm, work=None, stream=None) -> None:
    """norm (float32 [1], device) = sqrt of the sum of squares over all elements of
    grads, an mgn_grad_list or a sequence of tensors.  work: device scratch of the
    list's work_bytes (None: allocated)."""
    dev, p, pn, tail, keep = _grads(grads, norm, work, stream)
    _run("mgn_grad_norm", dev, stream, p, pn, *tail)


def mgn_grad_clip(grads, max_norm: float, norm, given: bool = False, work=None, stream=None) -> None:
    """Scales grads (an mgn_grad_list, into its outs; or a sequence of tensors, in
    place) by min(1, max_norm / norm); norm (float32 [1], device) takes the tensors'
    own or, given, is read.  A norm that is not finite (in float32) scales nothing."""
    dev, p, pn, tail, keep = _grads(grads, norm, work, stream)
    _run("mgn_grad_clip", dev, stream, p, float(max_norm), 1 if given else 0, pn, *tail)


def mgn_workspace_size(model, graph: mgn_graph) -> int:
    n = C.c_size_t()
    _check(lib().mgn_workspace_size(model, C.byref(graph), C.byref(n)), model)
    return int(n.value)


def mgn_forward(model, graph: mgn_graph, node_feat, edge_feat, halo, out, workspace, stream=None) -> None:
    _check(lib().mgn_forward(model, C.byref(graph), _dev(node_feat), _dev(edge_feat), _dev(halo), _dev(out),
                             _dev(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           model)


MGN_NOALLOC_WS_MAX = 128 << 20


def mgn_forward_noalloc(model, graph: mgn_graph, node_feat, edge_feat, halo, out, stream=None) -> None:
    """mgn_forward with the library's static per-GPU workspace (no caller
    workspace, no allocation)."""
    _check(lib().mgn_forward_noalloc(model, C.byref(graph), _dev(node_feat), _dev(edge_feat), _dev(halo), _dev(out),
                                     _stream(stream)), model)


def mgn_backward(model, d_out, d_params, accumulate: bool = False, d_halo=None, stream=None) -> None:
    _check(lib().mgn_backward(model, _dev(d_out), _dev(d_params), int(bool(accumulate)), _dev(d_halo),
                              _stream(stream)), model)


def mgn_forward_begin(model, graph: mgn_graph, node_feat, edge_feat, halo, out, workspace, stream=None) -> None:
    _check(lib().mgn_forward_begin(model, C.byref(graph), _dev(node_feat), _dev(edge_feat), _dev(halo), _dev(out),
                                   _dev(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           model)


def mgn_forward_block(model, stream=None) -> None:
    _check(lib().mgn_forward_block(model, _stream(stream)), model)


def mgn_forward_end(model, stream=None) -> None:
    _check(lib().mgn_forward_end(model, _stream(stream)), model)


def mgn_backward_begin(model, d_out, d_params, accumulate: bool = False, d_halo=None, stream=None) -> None:
    _check(lib().mgn_backward_begin(model, _dev(d_out), _dev(d_params), int(bool(accumulate)), _dev(d_halo),
                                    _stream(stream)), model)


def mgn_backward_block(model, stream=None) -> None:
    _check(lib().mgn_backward_block(model, _stream(stream)), model)


def mgn_backward_end(model, stream=None) -> None:
    _check(lib().mgn_backward_end(model, _stream(stream)), model)


def mgn_halo_masks(l2g_p, n_owned_p: int, part, l2g_q, n_owned_q: int, q: int):
    """Host exchange lists of part p's halo nodes owned by part q:
    (recv_idx, send_rows) int32 arrays (halo index in p, local id in q)."""
    lp, lpp = _host(l2g_p, np.int32)
    pa, pp = _host(part, np.int32)
    lq, lqp = _host(l2g_q, np.int32)
    nh = lp.shape[0] - int(n_owned_p)
    recv = np.empty(max(nh, 0), np.int32)
    send = np.empty(max(nh, 0), np.int32)
    cnt = C.c_int64()
    _check(lib().mgn_halo_masks(lpp, int(n_owned_p), nh, pp, pa.shape[0], lqp, int(n_owned_q), int(q),
                                recv.ctypes.data_as(C.c_void_p), send.ctypes.data_as(C.c_void_p), C.byref(cnt)))
    return recv[:cnt.value].copy(), send[:cnt.value].copy()


def mgn_copy_latents(owner, send_rows, recv_idx, halo_k, stream=None) -> None:
    """halo_k[recv_idx[i]] = owner's current node latents[send_rows[i]] (device tensors)."""
    _check(lib().mgn_copy_latents(owner, _dev(send_rows), _dev(recv_idx), int(send_rows.numel()), _dev(halo_k),
                                  int(halo_k.shape[0]), _stream(stream)), owner)


def mgn_add_latent_grads(owner, d_halo_k, recv_idx, send_rows, stream=None) -> None:
    """owner's dL/dv[send_rows[i]] += d_halo_k[recv_idx[i]] (device tensors)."""
    _check(lib().mgn_add_latent_grads(owner, _dev(d_halo_k), int(d_halo_k.shape[0]), _dev(recv_idx),
                                      _dev(send_rows), int(send_rows.numel()), _stream(stream)), owner)


def _slots8(q, scale):
    """8-bit slots of an exchange: (q, scale, slots, cols)."""
    import torch
    slots, cols = _shape(q, "q")
    return (_devt(q, torch.uint8, "q"), _devt(scale, torch.float32, "scale", shape=(slots, rows8_blocks(cols))), slots,
            cols)


def mgn_pack_latents8(owner, send_rows, q, scale, stream=None) -> None:
    """Slots 0 .. n-1 of q (uint8 [slots][latent]) and scale take the owner's
    current node latents[send_rows] in 8 bits (device tensors)."""
    import torch
    n = send_rows.numel()
    pq, ps, slots, cols = _slots8(q, scale)
    if slots < n:
        raise ValueError("q: expected at least as many slots as send_rows")
    _check(lib().mgn_pack_latents8(owner, _devt(send_rows, torch.int32, "send_rows"), n, pq, ps, cols,
                                   _stream(stream)), owner)


def mgn_add_latent_grads8(owner, q, scale, send_rows, stream=None) -> None:
    """owner's dL/dv[send_rows[i]] += the values of slot i (device tensors)."""
    import torch
    n = send_rows.numel()
    pq, ps, slots, cols = _slots8(q, scale)
    if slots < n:
        raise ValueError("q: expected at least as many slots as send_rows")
    _check(lib().mgn_add_latent_grads8(owner, pq, ps, cols, _devt(send_rows, torch.int32, "send_rows"), n,
                                       _stream(stream)), owner)


def _ptrs(ts):
    """C array of device pointers (NULL for None)."""
    return (C.c_void_p * len(ts))(*[None if t is None else t.data_ptr() for t in ts])


def _links(links):
    return (mgn_halo_link * max(len(links), 1))(*[mgn_halo_link(p, q, r.data_ptr(), s.data_ptr(), r.numel())
                                                  for p, q, r, s in links])


def mgn_lockstep_forward(models, graphs, node_feats, edge_feats, halos, outs, workspaces, links,
                         stream=None) -> None:
    """models, graphs (mgn_graph), device tensors per part; links: list of
    (part, owner, recv_idx, send_rows) with device int32 index tensors."""
    P = len(models)
    ms = (C.c_void_p * P)(*[m.value for m in models])
    gs = (mgn_graph * P)(*graphs)
    wb = (C.c_size_t * P)(*[w.numel() * w.element_size() for w in workspaces])
    st = lib().mgn_lockstep_forward(P, ms, gs, _ptrs(node_feats), _ptrs(edge_feats), _ptrs(halos), _ptrs(outs),
                                    _ptrs(workspaces), wb, _links(links), len(links), _stream(stream))
    _check(st)


def mgn_lockstep_forward8(models, graphs, node_feats, edge_feats, halos, outs, workspaces, links, q, scale,
                          stream=None) -> None:
    """mgn_lockstep_forward with every exchange in 8 bits; q (uint8
    [slots][latent]), scale: device scratch of as many slots as the longest link."""
    P = len(models)
    ms = (C.c_void_p * P)(*[m.value for m in models])
    gs = (mgn_graph * P)(*graphs)
    wb = (C.c_size_t * P)(*[w.numel() * w.element_size() for w in workspaces])
    st = lib().mgn_lockstep_forward8(P, ms, gs, _ptrs(node_feats), _ptrs(edge_feats), _ptrs(halos), _ptrs(outs),
                                     _ptrs(workspaces), wb, _links(links), len(links), *_slots8(q, scale),
                                     _stream(stream))
    _check(st)


def mgn_lockstep_backward(models, d_outs, d_params, d_halos, links, accumulate: bool = False, stream=None) -> None:
    P = len(models)
    ms = (C.c_void_p * P)(*[m.value for m in models])
    st = lib().mgn_lockstep_backward(P, ms, _ptrs(d_outs), _dev(d_params), int(bool(accumulate)), _ptrs(d_halos),
                                     _links(links), len(links), _stream(stream))
    _check(st)


def mgn_lockstep_backward8(models, d_outs, d_params, d_halos, links, q, scale, accumulate: bool = False,
                           stream=None) -> None:
    """mgn_lockstep_backward with the halo gradients in 8 bits (q, scale as in
    mgn_lockstep_forward8)."""
    P = len(models)
    ms = (C.c_void_p * P)(*[m.value for m in models])
    st = lib().mgn_lockstep_backward8(P, ms, _ptrs(d_outs), _dev(d_params), int(bool(accumulate)), _ptrs(d_halos),
                                      _links(links), len(links), *_slots8(q, scale), _stream(stream))
    _check(st)


def _mse_args(out, target, mask, loss, d_out):
    import torch
    if out.dim() != 2:
        raise ValueError("out: expected [n][d]")
    n, d = out.shape
    return (n, d, _devt(out, torch.float32, "out"), _devt(target, torch.float32, "target", shape=(n, d)),
            None if mask is None else _devt(mask, torch.uint8, "mask", numel=n),
            _devt(loss, torch.float32, "loss", min_numel=2), _devt(d_out, torch.float32, "d_out", shape=(n, d)))


def mgn_mse_grad(out, target, mask, loss, d_out, stream=None) -> None:
    n, d, po, pt, pm, pl, pd = _mse_args(out, target, mask, loss, d_out)
    _check(lib().mgn_mse_grad(po, pt, pm, n, d, pl, pd, _stream(stream)))


def mgn_mse_grad_global(out, target, mask, global_rows: int, loss, d_out, stream=None) -> None:
    n, d, po, pt, pm, pl, pd = _mse_args(out, target, mask, loss, d_out)
    _check(lib().mgn_mse_grad_global(po, pt, pm, n, d, int(global_rows), pl, pd, _stream(stream)))


def mgn_timing_enable(model, enable: bool = True) -> None:
    _check(lib().mgn_timing_enable(model, int(bool(enable))), model)


def mgn_timing_read(model) -> dict:
    """{timer name: (total ms, launches)} for every timer class."""
    res = {}
    for i, name in enumerate(TIMERS):
        ms, n = C.c_double(), C.c_int64()
        _check(lib().mgn_timing_read(model, i, C.byref(ms), C.byref(n)), model)
        res[name] = (ms.value, n.value)
    return res
