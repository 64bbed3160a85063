"""ctypes binding of libmoe_ffn.so (C ABI in include/moe_ffn.h).

Marshalling only: torch supplies device memory and the stream; every function
here has the name and meaning of the C entry point it calls.
"""
from __future__ import annotations

import ctypes
import dataclasses
import os
from typing import Optional

import torch

MOE_F32, MOE_BF16 = 0, 1
MODE_SERIALIZED, MODE_PERSISTENT = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None


class MoeError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {moe_status_string(status)} ({status})")
        self.status = status


class _MoeShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "H", "I", "E", "E_local", "expert_base", "k", "dtype")]


class _MoeSaved(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("topk_idx", "topk_w", "counts", "offsets", "row_of", "token_of", "slot_of", "Xp", "H1", "A", "Yp")]


EXPORTS = (
    "moe_status_string", "moe_ffn_workspace_bytes", "moe_ffn_forward", "moe_ffn_backward", "moe_ffn_backward_two_streams",
    "moe_ffn_last_status", "moe_ffn_debug_set_spin_limit", "moe_route", "moe_permute", "moe_grouped_gemm_swiglu", "moe_grouped_gemm",
    "moe_combine", "moe_microbench_workspace_bytes", "moe_microbench_swiglu_add", "moe_microbench_last_status",
    "moe_probe_mfma_bf16", "moe_probe_copy", "moe_probe_read", "moe_probe_write", "moe_microbench_swiglu_add_static_scratch",
    "moe_ffn_debug_force_device_scope", "moe_ffn_debug_layout", "moe_dispatch_to_combine",
    "moe_grouped_gemm_scatter", "moe_ffn_forward_scatter",
    "moe_layer_norm_workspace_bytes", "moe_layer_norm_forward", "moe_layer_norm_backward", "moe_dropout_add_forward",
    "moe_dropout_add_backward", "moe_dropout_add_layer_norm_forward", "moe_dropout_add_layer_norm_backward",
    "moe_balance_workspace_bytes", "moe_balance_forward", "moe_router_backward", "moe_quantize_w4", "moe_ffn_forward_w4",
)
LAYOUT_WORDS = 25   # MOE_LAYOUT_WORDS

# Argument kinds of the operators around the layer: i int, f float, p pointer, z size_t
_KINDS = {"i": ctypes.c_int32, "f": ctypes.c_float, "p": ctypes.c_void_p, "z": ctypes.c_size_t}
_BLOCK_ARGS = {
    "moe_layer_norm_workspace_bytes": "iip", "moe_layer_norm_forward": "iiipppfpppp", "moe_layer_norm_backward": "iiipppppppp" "ppzp",
    "moe_dropout_add_forward": "iiippfppp", "moe_dropout_add_backward": "iiipfppp",
    "moe_dropout_add_layer_norm_forward": "iiippfpppf" "ppppp", "moe_dropout_add_layer_norm_backward": "iiipppppp" "fpppppp" "zp",
    "moe_balance_workspace_bytes": "iip", "moe_balance_forward": "iiipppf" "ppppzp", "moe_router_backward": "iiippppp" "fpppp",
    "moe_quantize_w4": "iiiipppp", "moe_ffn_forward_w4": "ppppppppppzp",
}


def library_path() -> str:
    return os.path.join(_HERE, "libmoe_ffn.so")


def load_library() -> ctypes.CDLL:
    """Load the HIP library; raises if it has not been built (no fallback)."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise FileNotFoundError(
                f"{path} is missing: build it with `python -m paper_2605_23764_amd.build` "
                "(or __graft_entry__.build()); there is no CPU fallback")
        lib = ctypes.CDLL(path)
        lib.moe_status_string.restype = ctypes.c_char_p
        lib.moe_status_string.argtypes = [ctypes.c_int]
        for name in EXPORTS[1:]:
            getattr(lib, name).restype = ctypes.c_int
        lib.moe_microbench_workspace_bytes.restype = ctypes.c_size_t
        lib.moe_microbench_workspace_bytes.argtypes = [ctypes.c_int]
        for name, kinds in _BLOCK_ARGS.items():
            getattr(lib, name).argtypes = [_KINDS[c] for c in kinds]
        _LIB = lib
    return _LIB


def moe_status_string(status: int) -> str:
    return load_library().moe_status_string(int(status)).decode()


def make_shape(T, H, I, E, E_local, expert_base, k, dtype) -> _MoeShape:
    if isinstance(dtype, torch.dtype):
        dtype = {torch.float32: MOE_F32, torch.bfloat16: MOE_BF16}[dtype]
    return _MoeShape(T, H, I, E, E_local, expert_base, k, dtype)


def _torch_dtype(shape: _MoeShape) -> torch.dtype:
    return torch.bfloat16 if shape.dtype == MOE_BF16 else torch.float32


def moe_ffn_workspace_bytes(shape: _MoeShape):
    fwd, bwd = ctypes.c_size_t(0), ctypes.c_size_t(0)
    st = load_library().moe_ffn_workspace_bytes(ctypes.byref(shape), ctypes.byref(fwd), ctypes.byref(bwd))
    if st != 0:
        raise MoeError(st, "moe_ffn_workspace_bytes")
    return fwd.value, bwd.value


def alloc_workspace(shape: _MoeShape, device="cuda", backward: bool = False) -> torch.Tensor:
    fwd, bwd = moe_ffn_workspace_bytes(shape)
    return torch.empty(max(fwd, bwd) if backward else fwd, dtype=torch.uint8, device=device)


@dataclasses.dataclass
class Saved:
    """Device buffers of MoeSaved (torch tensors own the memory)."""
    topk_idx: torch.Tensor
    topk_w: torch.Tensor
    counts: torch.Tensor
    offsets: torch.Tensor
    row_of: torch.Tensor
    token_of: torch.Tensor
    slot_of: torch.Tensor
    Xp: Optional[torch.Tensor]
    H1: Optional[torch.Tensor]
    A: torch.Tensor
    Yp: torch.Tensor

    def c_struct(self) -> _MoeSaved:
        f = lambda t: ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)  # noqa: E731
        return _MoeSaved(*(f(getattr(self, n)) for n, _ in _MoeSaved._fields_))


def alloc_saved(shape: _MoeShape, device="cuda", store_h1: bool = False, keep_xp: bool = True) -> Saved:
    """keep_xp=False: no permuted copy of x is kept (MoeSaved.Xp = NULL); forward and backward then read x through
    the permutation."""
    T, H, I, k, El = shape.T, shape.H, shape.I, shape.k, shape.E_local
    Rm = T * min(k, El)
    dt = _torch_dtype(shape)
    i32 = dict(dtype=torch.int32, device=device)
    # +4 elements keep zero-size problems at non-null, aligned pointers
    return Saved(
        topk_idx=torch.empty(T * k + 4, **i32)[: T * k].view(T, k),
        topk_w=torch.empty(T * k + 4, dtype=torch.float32, device=device)[: T * k].view(T, k),
        counts=torch.empty(El, **i32),
        offsets=torch.empty(El + 1, **i32),
        row_of=torch.empty(T * k + 4, **i32)[: T * k].view(T, k),
        token_of=torch.empty(Rm + 4, **i32)[:Rm],
        slot_of=torch.empty(Rm + 4, **i32)[:Rm],
        Xp=torch.empty(Rm * H + 8, dtype=dt, device=device)[: Rm * H].view(Rm, H) if keep_xp else None,
        H1=torch.empty(Rm * 2 * I + 8, dtype=dt, device=device)[: Rm * 2 * I].view(Rm, 2 * I) if store_h1 else None,
        A=torch.empty(Rm * I + 8, dtype=dt, device=device)[: Rm * I].view(Rm, I),
        Yp=torch.empty(Rm * H + 8, dtype=dt, device=device)[: Rm * H].view(Rm, H),
    )


def _ptr(t: Optional[torch.Tensor]) -> ctypes.c_void_p:
    if t is None:
        return ctypes.c_void_p(0)
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _check(st: int, what: str) -> None:
    if st != 0:
        raise MoeError(st, what)


def _ws(ws: torch.Tensor):
    return _ptr(ws), ctypes.c_size_t(ws.numel() * ws.element_size())


def moe_ffn_forward(shape, x, logits, w_gate_up, w_down, out, saved: Optional[Saved], workspace,
                    mode: int = MODE_SERIALIZED, stream=None) -> None:
    sv = saved.c_struct() if saved is not None else None
    wp, wb = _ws(workspace)
    st = load_library().moe_ffn_forward(
        ctypes.byref(shape), _ptr(x), _ptr(logits), _ptr(w_gate_up), _ptr(w_down), _ptr(out),
        ctypes.byref(sv) if sv is not None else None, wp, wb, ctypes.c_int(mode), _stream(stream))
    _check(st, "moe_ffn_forward")


def moe_ffn_backward(shape, dy, x, w_gate_up, w_down, saved: Saved, dx, dw_gate_up, dw_down, dtopk_w,
                     workspace, mode: int = MODE_SERIALIZED, stream=None) -> None:
    sv = saved.c_struct()
    wp, wb = _ws(workspace)
    st = load_library().moe_ffn_backward(
        ctypes.byref(shape), _ptr(dy), _ptr(x), _ptr(w_gate_up), _ptr(w_down), ctypes.byref(sv),
        _ptr(dx), _ptr(dw_gate_up), _ptr(dw_down), _ptr(dtopk_w), wp, wb, ctypes.c_int(mode), _stream(stream))
    _check(st, "moe_ffn_backward")


def moe_ffn_backward_two_streams(shape, dy, x, w_gate_up, w_down, saved: Saved, dx, dw_gate_up, dw_down, dtopk_w,
                                 workspace, wgrad_stream, mode: int = MODE_SERIALIZED, stream=None) -> None:
    """`wgrad_stream`: a torch.cuda.Stream for the weight-gradient launches, or None (one stream)."""
    sv = saved.c_struct()
    wp, wb = _ws(workspace)
    side = ctypes.c_void_p(wgrad_stream.cuda_stream) if wgrad_stream is not None else ctypes.c_void_p(None)
    st = load_library().moe_ffn_backward_two_streams(
        ctypes.byref(shape), _ptr(dy), _ptr(x), _ptr(w_gate_up), _ptr(w_down), ctypes.byref(sv),
        _ptr(dx), _ptr(dw_gate_up), _ptr(dw_down), _ptr(dtopk_w), wp, wb, ctypes.c_int(mode), _stream(stream), side)
    _check(st, "moe_ffn_backward_two_streams")


def moe_ffn_last_status(shape, workspace) -> int:
    return load_library().moe_ffn_last_status(ctypes.byref(shape), _ptr(workspace))


def moe_ffn_debug_set_spin_limit(polls: int) -> None:
    _check(load_library().moe_ffn_debug_set_spin_limit(ctypes.c_uint32(polls)), "moe_ffn_debug_set_spin_limit")


def moe_route(shape, logits, saved: Saved, workspace, stream=None) -> None:
    sv = saved.c_struct()
    wp, wb = _ws(workspace)
    _check(load_library().moe_route(ctypes.byref(shape), _ptr(logits), ctypes.byref(sv), wp, wb, _stream(stream)),
           "moe_route")


def moe_permute(shape, x, saved: Saved, workspace, stream=None) -> None:
    sv = saved.c_struct()
    wp, wb = _ws(workspace)
    _check(load_library().moe_permute(ctypes.byref(shape), _ptr(x), ctypes.byref(sv), wp, wb, _stream(stream)),
           "moe_permute")


def moe_grouped_gemm_swiglu(shape, w_gate_up, saved: Saved, workspace, stream=None) -> None:
    sv = saved.c_struct()
    wp, wb = _ws(workspace)
    _check(load_library().moe_grouped_gemm_swiglu(ctypes.byref(shape), _ptr(w_gate_up), ctypes.byref(sv), wp, wb,
                                                  _stream(stream)), "moe_grouped_gemm_swiglu")


def moe_grouped_gemm(shape, w_down, saved: Saved, workspace, stream=None) -> None:
    sv = saved.c_struct()
    wp, wb = _ws(workspace)
    _check(load_library().moe_grouped_gemm(ctypes.byref(shape), _ptr(w_down), ctypes.byref(sv), wp, wb,
                                           _stream(stream)), "moe_grouped_gemm")


def moe_grouped_gemm_scatter(shape, w_down, saved: Saved, out, workspace, stream=None) -> None:
    sv = saved.c_struct()
    wp, wb = _ws(workspace)
    _check(load_library().moe_grouped_gemm_scatter(ctypes.byref(shape), _ptr(w_down), ctypes.byref(sv), _ptr(out), wp, wb,
                                                   _stream(stream)), "moe_grouped_gemm_scatter")


def moe_ffn_forward_scatter(shape, x, logits, w_gate_up, w_down, out, saved: Optional[Saved], workspace,
                            mode: int = MODE_SERIALIZED, stream=None) -> None:
    sv = saved.c_struct() if saved is not None else None
    wp, wb = _ws(workspace)
    st = load_library().moe_ffn_forward_scatter(
        ctypes.byref(shape), _ptr(x), _ptr(logits), _ptr(w_gate_up), _ptr(w_down), _ptr(out),
        ctypes.byref(sv) if sv is not None else None, wp, wb, ctypes.c_int(mode), _stream(stream))
    _check(st, "moe_ffn_forward_scatter")


def moe_combine(shape, saved: Saved, out, workspace, stream=None) -> None:
    sv = saved.c_struct()
    wp, wb = _ws(workspace)
    _check(load_library().moe_combine(ctypes.byref(shape), ctypes.byref(sv), _ptr(out), wp, wb, _stream(stream)),
           "moe_combine")


def moe_dispatch_to_combine(shape, x, w_gate_up, w_down, out, saved: Saved, workspace, mode: int = MODE_SERIALIZED,
                            stream=None) -> None:
    sv = saved.c_struct()
    wp, wb = _ws(workspace)
    _check(load_library().moe_dispatch_to_combine(ctypes.byref(shape), _ptr(x), _ptr(w_gate_up), _ptr(w_down), _ptr(out),
                                                  ctypes.byref(sv), wp, wb, ctypes.c_int(mode), _stream(stream)),
           "moe_dispatch_to_combine")


MB_SERIAL, MB_STATIC, MB_DYNAMIC, MB_DYNAMIC_XCD = 0, 1, 2, 3


def moe_microbench_workspace_bytes(M: int) -> int:
    return int(load_library().moe_microbench_workspace_bytes(int(M)))


def moe_microbench_swiglu_add(M, N, x, y, s, out, mode, tile_rows, workspace, stream=None) -> None:
    wp, wb = _ws(workspace)
    _check(load_library().moe_microbench_swiglu_add(ctypes.c_int(M), ctypes.c_int(N), _ptr(x), _ptr(y), _ptr(s),
                                                    _ptr(out), ctypes.c_int(mode), ctypes.c_int(tile_rows), wp, wb,
                                                    _stream(stream)),
           "moe_microbench_swiglu_add")


def moe_microbench_last_status(workspace) -> int:
    return load_library().moe_microbench_last_status(_ptr(workspace))


def moe_probe_mfma_bf16(n_workgroups, mfma_per_wave, random_operands, sink, stream=None) -> None:
    _check(load_library().moe_probe_mfma_bf16(ctypes.c_int(n_workgroups), ctypes.c_int(mfma_per_wave),
                                              ctypes.c_int(1 if random_operands else 0), _ptr(sink), _stream(stream)),
           "moe_probe_mfma_bf16")


def moe_microbench_swiglu_add_static_scratch(M, N, x, y, s, out, mode, tile_rows, status=None, stream=None) -> None:
    _check(load_library().moe_microbench_swiglu_add_static_scratch(
        ctypes.c_int(M), ctypes.c_int(N), _ptr(x), _ptr(y), _ptr(s), _ptr(out), ctypes.c_int(mode),
        ctypes.c_int(tile_rows), _ptr(status), _stream(stream)), "moe_microbench_swiglu_add_static_scratch")


def moe_ffn_debug_force_device_scope(on: bool) -> None:
    _check(load_library().moe_ffn_debug_force_device_scope(ctypes.c_int(1 if on else 0)),
           "moe_ffn_debug_force_device_scope")


def moe_ffn_debug_layout(shape, backward: bool = False):
    """The LAYOUT_WORDS integers of moe_ffn_debug_layout (offsets of the scheduler's tables in the workspace)."""
    out = (ctypes.c_int64 * LAYOUT_WORDS)()
    _check(load_library().moe_ffn_debug_layout(ctypes.byref(shape), ctypes.c_int(1 if backward else 0), out,
                                               ctypes.c_int(LAYOUT_WORDS)), "moe_ffn_debug_layout")
    return list(out)


def moe_probe_read(src, nbytes, sink, stream=None) -> None:
    _check(load_library().moe_probe_read(_ptr(src), ctypes.c_size_t(nbytes), _ptr(sink), _stream(stream)),
           "moe_probe_read")


def moe_probe_write(dst, nbytes, word=0, stream=None) -> None:
    _check(load_library().moe_probe_write(_ptr(dst), ctypes.c_size_t(nbytes), ctypes.c_uint32(word), _stream(stream)),
           "moe_probe_write")


def moe_probe_copy(src, dst, nbytes, stream=None) -> None:
    _check(load_library().moe_probe_copy(_ptr(src), _ptr(dst), ctypes.c_size_t(nbytes), _stream(stream)),
           "moe_probe_copy")


# ---- the operators around the layer: T, H and the storage type are read off the tensors, whose shapes and types are checked ----

def _args(shape, dtype, names: str, *tensors):
    """Device addresses of tensors of this shape and type; None for None.  (One call per group: a launch is 3 us of the host's time, and each
    tensor's checks a quarter of one.)"""
    out = []
    for t in tensors:
        if t is None:
            out.append(None)
        elif t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous():
            out.append(t.data_ptr())
        else:
            raise ValueError(f"{names.split()[len(out)]}: expected a contiguous device tensor of shape {tuple(shape)} and type {dtype}, got "
                             f"{tuple(t.shape)}, {t.dtype}, {t.device}")
    return out


_STORAGE = {torch.bfloat16: MOE_BF16, torch.float32: MOE_F32}


def _rows(t: torch.Tensor, name: str):
    """(shape, storage type, its MoeDtype) of a [T, H] tensor."""
    shape, dtype = t.shape, t.dtype
    if len(shape) != 2 or dtype not in _STORAGE:
        raise ValueError(f"{name}: expected a [T, H] tensor in bfloat16 or float32, got {tuple(shape)}, {dtype}")
    return shape, dtype, _STORAGE[dtype]


def _raw_stream(stream) -> int:
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _size(name: str, *args) -> int:
    n = ctypes.c_size_t(0)
    _check(getattr(load_library(), name)(*args, ctypes.addressof(n)), name)
    return n.value


def _workspace(t: Optional[torch.Tensor]):
    if t is None:
        return None, 0
    return _ptr(t).value, t.numel() * t.element_size()


def moe_layer_norm_workspace_bytes(T: int, H: int) -> int:
    return _size("moe_layer_norm_workspace_bytes", T, H)


def alloc_layer_norm_workspace(T: int, H: int, device="cuda") -> torch.Tensor:
    return torch.empty(moe_layer_norm_workspace_bytes(T, H), dtype=torch.uint8, device=device)


def moe_layer_norm_forward(x, gamma, beta, eps: float, y, mean=None, rstd=None, stream=None) -> None:
    """y = layer norm of the rows of x [T, H]; gamma, beta [H] or None; mean, rstd [T] f32 (for the backward) or None."""
    shape, dt, code = _rows(x, "x")
    T, H = shape
    x, y = _args(shape, dt, "x y", x, y)
    gamma, beta = _args((H,), dt, "gamma beta", gamma, beta)
    mean, rstd = _args((T,), torch.float32, "mean rstd", mean, rstd)
    _check(load_library().moe_layer_norm_forward(T, H, code, x, gamma, beta, eps, y, mean, rstd, _raw_stream(stream)),
           "moe_layer_norm_forward")


def moe_layer_norm_backward(dy, x, gamma, mean, rstd, dres, dx, dgamma, dbeta, workspace, stream=None) -> None:
    """dx = gradient of x, plus dres (the residual path's) if given; dgamma, dbeta [H] or None."""
    shape, dt, code = _rows(x, "x")
    T, H = shape
    dy, x, dres, dx = _args(shape, dt, "dy x dres dx", dy, x, dres, dx)
    gamma, dgamma, dbeta = _args((H,), dt, "gamma dgamma dbeta", gamma, dgamma, dbeta)
    mean, rstd = _args((T,), torch.float32, "mean rstd", mean, rstd)
    ws, wb = _workspace(workspace)
    _check(load_library().moe_layer_norm_backward(T, H, code, dy, x, gamma, mean, rstd, dres, dx, dgamma, dbeta, ws, wb,
                                                  _raw_stream(stream)), "moe_layer_norm_backward")


def moe_dropout_add_forward(v, residual, p: float, rng, out, stream=None) -> None:
    """out = residual (or 0) + dropout(v); rng: device int64 {seed, offset}, None if p == 0."""
    shape, dt, code = _rows(v, "v")
    T, H = shape
    v, residual, out = _args(shape, dt, "v residual out", v, residual, out)
    rng, = _args((2,), torch.int64, "rng", rng)
    _check(load_library().moe_dropout_add_forward(T, H, code, v, residual, p, rng, out, _raw_stream(stream)), "moe_dropout_add_forward")


def moe_dropout_add_backward(dout, p: float, rng, dv, stream=None) -> None:
    """dv = dropout's backward of dout, with the forward's p and rng contents."""
    shape, dt, code = _rows(dout, "dout")
    T, H = shape
    dout, dv = _args(shape, dt, "dout dv", dout, dv)
    rng, = _args((2,), torch.int64, "rng", rng)
    _check(load_library().moe_dropout_add_backward(T, H, code, dout, p, rng, dv, _raw_stream(stream)), "moe_dropout_add_backward")


def moe_dropout_add_layer_norm_forward(v, residual, p: float, rng, gamma, beta, eps: float, z, y, mean=None, rstd=None,
                                       stream=None) -> None:
    """z = residual (or 0) + dropout(v), y = layer norm of z."""
    shape, dt, code = _rows(v, "v")
    T, H = shape
    v, residual, z, y = _args(shape, dt, "v residual z y", v, residual, z, y)
    gamma, beta = _args((H,), dt, "gamma beta", gamma, beta)
    mean, rstd = _args((T,), torch.float32, "mean rstd", mean, rstd)
    rng, = _args((2,), torch.int64, "rng", rng)
    _check(load_library().moe_dropout_add_layer_norm_forward(T, H, code, v, residual, p, rng, gamma, beta, eps, z, y, mean, rstd,
                                                             _raw_stream(stream)), "moe_dropout_add_layer_norm_forward")


def moe_dropout_add_layer_norm_backward(dy, z, gamma, mean, rstd, dres, p: float, rng, dz, dv, dgamma, dbeta, workspace,
                                        stream=None) -> None:
    """dz = dres (or 0) + layer norm's backward at z (the residual's gradient too), dv = dropout's backward of dz."""
    shape, dt, code = _rows(z, "z")
    T, H = shape
    dy, z, dres, dz, dv = _args(shape, dt, "dy z dres dz dv", dy, z, dres, dz, dv)
    gamma, dgamma, dbeta = _args((H,), dt, "gamma dgamma dbeta", gamma, dgamma, dbeta)
    mean, rstd = _args((T,), torch.float32, "mean rstd", mean, rstd)
    rng, = _args((2,), torch.int64, "rng", rng)
    ws, wb = _workspace(workspace)
    _check(load_library().moe_dropout_add_layer_norm_backward(T, H, code, dy, z, gamma, mean, rstd, dres, p, rng, dz, dv, dgamma, dbeta,
                                                              ws, wb, _raw_stream(stream)), "moe_dropout_add_layer_norm_backward")


def moe_balance_workspace_bytes(T: int, E: int) -> int:
    return _size("moe_balance_workspace_bytes", T, E)


def alloc_balance_workspace(T: int, E: int, device="cuda") -> torch.Tensor:
    return torch.empty(moe_balance_workspace_bytes(T, E), dtype=torch.uint8, device=device)


def _router(logits, topk_idx, mask):
    """T, E, k and the mask's type (bool or uint8)."""
    if logits.dim() != 2 or topk_idx.dim() != 2:
        raise ValueError("expected logits [T, E] and topk_idx [T, k]")
    return *logits.shape, topk_idx.shape[1], torch.bool if mask is not None and mask.dtype is torch.bool else torch.uint8


def moe_balance_forward(logits, topk_idx, mask, coef: float, counts, prob_sum, loss, workspace, stream=None) -> None:
    """counts [E + 1] i32 (the last: tokens that count), prob_sum [E] f32, loss [1] f32; mask [T] bool / uint8 or None."""
    T, E, k, mask_type = _router(logits, topk_idx, mask)
    f32, i32 = torch.float32, torch.int32
    logits, = _args((T, E), f32, "logits", logits)
    topk_idx, = _args((T, k), i32, "topk_idx", topk_idx)
    mask, = _args((T,), mask_type, "mask", mask)
    counts, = _args((E + 1,), i32, "counts", counts)
    prob_sum, = _args((E,), f32, "prob_sum", prob_sum)
    loss, = _args((1,), f32, "loss", loss)
    ws, wb = _workspace(workspace)
    _check(load_library().moe_balance_forward(T, E, k, logits, topk_idx, mask, coef, counts, prob_sum, loss, ws, wb, _raw_stream(stream)),
           "moe_balance_forward")


def moe_router_backward(logits, topk_idx, topk_w, dtopk_w, mask, coef: float, counts, dloss, dlogits, stream=None) -> None:
    """dlogits [T, E] from the routing weights' gradient (topk_w, dtopk_w or both None) and the balance loss's (counts or None)."""
    T, E, k, mask_type = _router(logits, topk_idx, mask)
    f32, i32 = torch.float32, torch.int32
    logits, dlogits = _args((T, E), f32, "logits dlogits", logits, dlogits)
    topk_idx, = _args((T, k), i32, "topk_idx", topk_idx)
    topk_w, dtopk_w = _args((T, k), f32, "topk_w dtopk_w", topk_w, dtopk_w)
    mask, = _args((T,), mask_type, "mask", mask)
    counts, = _args((E + 1,), i32, "counts", counts)
    dloss, = _args((1,), f32, "dloss", dloss)
    _check(load_library().moe_router_backward(T, E, k, logits, topk_idx, topk_w, dtopk_w, mask, coef, counts, dloss, dlogits,
                                              _raw_stream(stream)), "moe_router_backward")


def alloc_w4(E_local: int, K: int, N: int, device="cuda"):
    """(q, scale) buffers of a weight tensor [E_local, K, N] in 4-bit blocks."""
    return (torch.empty(E_local, K // 32, N, 16, dtype=torch.uint8, device=device),
            torch.empty(E_local, K // 32, N, dtype=torch.uint8, device=device))


def moe_quantize_w4(w, q, scale, stream=None) -> None:
    """4-bit blocks of w [E_local, K, N] (bfloat16 or float32)."""
    if w.dim() != 3 or w.dtype not in _STORAGE:
        raise ValueError(f"w: expected an [E_local, K, N] tensor in bfloat16 or float32, got {tuple(w.shape)}, {w.dtype}")
    E, K, N = w.shape
    code = _STORAGE[w.dtype]
    w, = _args((E, K, N), w.dtype, "w", w)
    q, = _args((E, K // 32, N, 16), torch.uint8, "q", q)
    scale, = _args((E, K // 32, N), torch.uint8, "scale", scale)
    _check(load_library().moe_quantize_w4(E, K, N, code, w, q, scale, _raw_stream(stream)), "moe_quantize_w4")


def moe_ffn_forward_w4(shape, x, logits, q_gate_up, s_gate_up, q_down, s_down, out, saved: Optional[Saved], workspace,
                       stream=None) -> None:
    T, H, I, El, u8 = shape.T, shape.H, shape.I, shape.E_local, torch.uint8
    sv = saved.c_struct() if saved is not None else None
    x, out = _args((T, H), torch.bfloat16, "x out", x, out)
    logits, = _args((T, shape.E), torch.float32, "logits", logits)
    q_gate_up, = _args((El, H // 32, 2 * I, 16), u8, "q_gate_up", q_gate_up)
    s_gate_up, = _args((El, H // 32, 2 * I), u8, "s_gate_up", s_gate_up)
    q_down, = _args((El, I // 32, H, 16), u8, "q_down", q_down)
    s_down, = _args((El, I // 32, H), u8, "s_down", s_down)
    ws, wb = _workspace(workspace)
    _check(load_library().moe_ffn_forward_w4(ctypes.addressof(shape), x, logits, q_gate_up, s_gate_up, q_down, s_down, out,
                                             ctypes.addressof(sv) if sv is not None else None, ws, wb, _raw_stream(stream)),
           "moe_ffn_forward_w4")
