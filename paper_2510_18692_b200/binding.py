"""Thin ctypes binding of the C ABI in include/moga.h (argument marshalling only).

Every function takes torch CUDA tensors (used purely as device memory), passes
their pointers and the current stream to ``libmoga.so`` and raises ``MogaError``
on a non-OK status.  No arithmetic of the method happens in Python, and there is
no fallback: if the library is missing, importing this module fails.
"""
from __future__ import annotations

import ctypes
import os

import torch

from .inputs import MogaConfig

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "csrc", "libmoga.so")

EXPORTS = ("moga_workspace_bytes", "moga_scratch_bytes", "moga_status_string", "moga_route",
           "moga_permute", "moga_group_attn", "moga_unpermute", "moga_forward",
           "moga_last_device_status", "moga_sort_static", "moga_balance_stats", "moga_stga_build", "moga_gather_rows",
           "moga_static_group_attn", "moga_mean3", "moga_forward_host_bytes", "moga_forward_host",
           "moga_visual_workspace_bytes", "moga_visual_forward", "moga_selftest_wait_timeout", "moga_set_attn_kernel", "moga_forward_routed", "moga_set_fused_topk", "moga_backward",
           "moga_backward_workspace_bytes", "moga_route_backward", "moga_route_backward_workspace_bytes",
           "moga_layernorm", "moga_layernorm_backward_workspace_bytes", "moga_layernorm_backward", "moga_dropout_add",
           "moga_residual_norm", "moga_residual_norm_backward", "moga_rope_build", "moga_rope", "moga_permute_rope",
           "moga_permute_rope_backward", "moga_forward_rope", "moga_backward_rope")

MOGA_F32, MOGA_BF16 = 0, 1
MOGA_ROUTE_AUTO, MOGA_ROUTE_ALU = 0, 1
STATUS_NAMES = {0: "MOGA_OK", 1: "MOGA_ERR_INVALID_ARG", 2: "MOGA_ERR_UNSUPPORTED",
                3: "MOGA_ERR_WORKSPACE", 4: "MOGA_ERR_CUDA", 5: "MOGA_ERR_TIMEOUT",
                6: "MOGA_ERR_INTERNAL"}


class MogaShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("H", ctypes.c_int32),
                ("C", ctypes.c_int32), ("D", ctypes.c_int32), ("M", ctypes.c_int32),
                ("k", ctypes.c_int32), ("dtype", ctypes.c_int32), ("gate_mode", ctypes.c_int32),
                ("scale", ctypes.c_float), ("q_stride_b", ctypes.c_int64),
                ("q_stride_h", ctypes.c_int64), ("q_stride_n", ctypes.c_int64),
                ("route_mode", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class MogaStaticLists(ctypes.Structure):
    _fields_ = [("G", ctypes.c_int32), ("Tkv", ctypes.c_int32), ("F", ctypes.c_int32),
                ("tokens_per_frame", ctypes.c_int32), ("q_idx", ctypes.c_void_p), ("q_inv", ctypes.c_void_p),
                ("q_offsets", ctypes.c_void_p), ("kv_idx", ctypes.c_void_p), ("kv_offsets", ctypes.c_void_p)]


class MogaNorm(ctypes.Structure):
    _fields_ = [("eps", ctypes.c_float), ("per_batch", ctypes.c_int32)]


class MogaDropout(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("step", ctypes.c_void_p)]


class MogaRopeConfig(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("scaling", ctypes.c_int32), ("n_axes", ctypes.c_int32),
                ("axis_dim", ctypes.c_int32 * 3), ("grid_h", ctypes.c_int32), ("grid_w", ctypes.c_int32),
                ("start", ctypes.c_int32 * 3), ("amplitude", ctypes.c_float), ("base", ctypes.c_double),
                ("factor", ctypes.c_double * 3), ("original_length", ctypes.c_double), ("beta_slow", ctypes.c_double),
                ("beta_fast", ctypes.c_double)]


class MogaRopePlan(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("pairs", ctypes.c_int32),
                ("grid_h", ctypes.c_int32), ("grid_w", ctypes.c_int32), ("axis_pairs", ctypes.c_int32 * 3),
                ("start", ctypes.c_int32 * 3), ("amplitude", ctypes.c_float), ("turns", ctypes.c_uint64 * 64)]


class MogaError(RuntimeError):
    def __init__(self, code: int, where: str, why: str = ""):
        self.code = code
        super().__init__(f"{where}: {STATUS_NAMES.get(code, code)} ({why or status_string(code)})")


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2510_18692_b200.build` "
                      "(there is no CPU fallback)")
lib = ctypes.CDLL(LIB_PATH)
for _n in EXPORTS:
    getattr(lib, _n).restype = ctypes.c_int
for _n in ("moga_workspace_bytes", "moga_scratch_bytes", "moga_static_scratch_bytes", "moga_forward_host_bytes",
           "moga_visual_workspace_bytes", "moga_backward_workspace_bytes", "moga_route_backward", "moga_route_backward_workspace_bytes",
           "moga_layernorm_backward_workspace_bytes"):
    getattr(lib, _n).restype = ctypes.c_size_t
lib.moga_status_string.restype = ctypes.c_char_p


def status_string(code: int) -> str:
    return lib.moga_status_string(ctypes.c_int(code)).decode()


def make_shape(cfg: MogaConfig, strides=None, scale=None, route_mode=MOGA_ROUTE_AUTO) -> MogaShape:
    sb, sh, sn = strides if strides is not None else (0, 0, 0)
    return MogaShape(cfg.B, cfg.N, cfg.H, cfg.C, cfg.D, cfg.M, cfg.k,
                     MOGA_F32 if cfg.dtype == "f32" else MOGA_BF16, cfg.gate_mode,
                     cfg.scale if scale is None else scale, sb, sh, sn, route_mode, 0)


def _ptr(t):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(code: int, where: str):
    if code != 0:
        raise MogaError(code, where)


def moga_workspace_bytes(shape: MogaShape) -> int:
    return int(lib.moga_workspace_bytes(ctypes.byref(shape)))


def moga_scratch_bytes(shape: MogaShape) -> int:
    return int(lib.moga_scratch_bytes(ctypes.byref(shape)))


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """Device bytes for ``ws`` (torch's allocator returns 512-byte aligned blocks)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def moga_route(shape, X, Wr, bias, gid, gate, logits=None, ws=None):
    _check(lib.moga_route(ctypes.byref(shape), _ptr(X), _ptr(Wr), _ptr(bias), _ptr(gid), _ptr(gate),
                          _ptr(logits), _ptr(ws), ctypes.c_size_t(0 if ws is None else ws.numel()),
                          _stream()), "moga_route")


def moga_balance_stats(shape, gid, gate, alpha, F, P, loss, ws):
    _check(lib.moga_balance_stats(ctypes.byref(shape), _ptr(gid), _ptr(gate), ctypes.c_float(alpha), _ptr(F),
                                  _ptr(P), _ptr(loss), _ptr(ws), ctypes.c_size_t(ws.numel()), _stream()),
           "moga_balance_stats")


def moga_permute(shape, gid, Q, K, V, perm, inv, offsets, Qp, Kp, Vp, ws):
    _check(lib.moga_permute(ctypes.byref(shape), _ptr(gid), _ptr(Q), _ptr(K), _ptr(V), _ptr(perm),
                            _ptr(inv), _ptr(offsets), _ptr(Qp), _ptr(Kp), _ptr(Vp), _ptr(ws),
                            ctypes.c_size_t(ws.numel()), _stream()), "moga_permute")


def moga_sort_static(shape, gid, perm, inv, offsets, status_out=None):
    """Group sort with library-resident scratch: no workspace, no device allocation."""
    _check(lib.moga_sort_static(ctypes.byref(shape), _ptr(gid), _ptr(perm), _ptr(inv), _ptr(offsets),
                                _ptr(status_out), _stream()), "moga_sort_static")


def moga_group_attn(shape, Qp, Kp, Vp, offsets, Op, lse, ws):
    _check(lib.moga_group_attn(ctypes.byref(shape), _ptr(Qp), _ptr(Kp), _ptr(Vp), _ptr(offsets),
                               _ptr(Op), _ptr(lse), _ptr(ws), ctypes.c_size_t(ws.numel()),
                               _stream()), "moga_group_attn")


def moga_stga_build(F, Hh, Ww, wh, ww, shot_starts, tg, augment=True):
    """Host-side group lists of the spatial-temporal branch: dict of numpy int32 arrays
    q_idx, q_inv, q_offsets, kv_idx, kv_offsets (plus G, Tkv)."""
    import numpy as np
    shots = (ctypes.c_int32 * len(shot_starts))(*shot_starts)
    G, Tkv = ctypes.c_int32(0), ctypes.c_int32(0)
    null = ctypes.c_void_p(0)
    args = (ctypes.c_int32(F), ctypes.c_int32(Hh), ctypes.c_int32(Ww), ctypes.c_int32(wh), ctypes.c_int32(ww),
            shots, ctypes.c_int32(len(shot_starts)), ctypes.c_int32(tg), ctypes.c_int32(1 if augment else 0))
    _check(lib.moga_stga_build(*args, null, null, null, null, null, ctypes.byref(G), ctypes.byref(Tkv)),
           "moga_stga_build")
    N = F * Hh * Ww
    out = dict(q_idx=np.empty(N, np.int32), q_inv=np.empty(N, np.int32), q_offsets=np.empty(G.value + 1, np.int32),
               kv_idx=np.empty(Tkv.value, np.int32), kv_offsets=np.empty(G.value + 1, np.int32))
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    _check(lib.moga_stga_build(*args, p(out["q_idx"]), p(out["q_inv"]), p(out["q_offsets"]), p(out["kv_idx"]),
                               p(out["kv_offsets"]), ctypes.byref(G), ctypes.byref(Tkv)), "moga_stga_build")
    out.update(G=G.value, Tkv=Tkv.value)
    return out


def moga_static_scratch_bytes(shape, G) -> int:
    return int(lib.moga_static_scratch_bytes(ctypes.byref(shape), ctypes.c_int32(G)))


def moga_gather_rows(shape, idx, src, dst):
    _check(lib.moga_gather_rows(ctypes.byref(shape), _ptr(idx), ctypes.c_int32(idx.numel()), _ptr(src), _ptr(dst),
                                _stream()), "moga_gather_rows")


def moga_static_group_attn(shape, G, Tq, Tkv, Qs, Ks, Vs, q_offsets, kv_offsets, Os, lse, ws):
    _check(lib.moga_static_group_attn(ctypes.byref(shape), ctypes.c_int32(G), ctypes.c_int32(Tq), ctypes.c_int32(Tkv),
                                      _ptr(Qs), _ptr(Ks), _ptr(Vs), _ptr(q_offsets), _ptr(kv_offsets), _ptr(Os),
                                      _ptr(lse), _ptr(ws), ctypes.c_size_t(ws.numel()), _stream()),
           "moga_static_group_attn")


def moga_mean3(shape, A, Bs, inv_b, C, O):
    _check(lib.moga_mean3(ctypes.byref(shape), _ptr(A), _ptr(Bs), _ptr(inv_b), _ptr(C), _ptr(O), _stream()),
           "moga_mean3")


def moga_unpermute(shape, Op, inv, gate, O):
    _check(lib.moga_unpermute(ctypes.byref(shape), _ptr(Op), _ptr(inv), _ptr(gate), _ptr(O),
                              _stream()), "moga_unpermute")


def moga_forward(shape, X, Wr, bias, Q, K, V, O, ws, gid_out=None, gate_out=None, perm_out=None,
                 offsets_out=None):
    _check(lib.moga_forward(ctypes.byref(shape), _ptr(X), _ptr(Wr), _ptr(bias), _ptr(Q), _ptr(K),
                            _ptr(V), _ptr(O), _ptr(gid_out), _ptr(gate_out), _ptr(perm_out),
                            _ptr(offsets_out), _ptr(ws), ctypes.c_size_t(ws.numel()), _stream()),
           "moga_forward")


def moga_forward_routed(shape, gid, gate, Q, K, V, O, ws, perm_out=None, offsets_out=None):
    _check(lib.moga_forward_routed(ctypes.byref(shape), _ptr(gid), _ptr(gate), _ptr(Q), _ptr(K), _ptr(V), _ptr(O),
                                   _ptr(perm_out), _ptr(offsets_out), _ptr(ws), ctypes.c_size_t(ws.numel()),
                                   _stream()), "moga_forward_routed")


def moga_route_backward_workspace_bytes(shape) -> int:
    return int(lib.moga_route_backward_workspace_bytes(ctypes.byref(shape)))


def moga_route_backward(shape, X, Wr, logits, gid, dgate, dX, dWr, dbias, ws):
    _check(lib.moga_route_backward(ctypes.byref(shape), _ptr(X), _ptr(Wr), _ptr(logits), _ptr(gid), _ptr(dgate),
                                   _ptr(dX), _ptr(dWr), _ptr(dbias), _ptr(ws), ctypes.c_size_t(ws.numel()),
                                   _stream()), "moga_route_backward")


def moga_backward_workspace_bytes(shape) -> int:
    return int(lib.moga_backward_workspace_bytes(ctypes.byref(shape)))


def moga_backward(shape, Qp, Kp, Vp, Op, lse, gate, perm, inv, offsets, dO, dQ, dK, dV, dgate, ws):
    _check(lib.moga_backward(ctypes.byref(shape), _ptr(Qp), _ptr(Kp), _ptr(Vp), _ptr(Op), _ptr(lse), _ptr(gate),
                             _ptr(perm), _ptr(inv), _ptr(offsets), _ptr(dO), _ptr(dQ), _ptr(dK), _ptr(dV),
                             _ptr(dgate), _ptr(ws), ctypes.c_size_t(ws.numel()), _stream()), "moga_backward")


# ---- around the attention: norm, dropout, rotary positions.  These calls also check what the C side
# cannot see of a tensor: its device, type, size and contiguity.  They are called many times a layer with
# little work behind some of them, so pointers go to the C side as plain integers (argtypes below) and each
# tensor is looked at once.
_DTYPES = (torch.float32, torch.bfloat16)
_P, _I, _S = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
lib.moga_layernorm.argtypes = [_P] * 9
lib.moga_layernorm_backward.argtypes = [_P] * 11 + [_S, _P]
lib.moga_dropout_add.argtypes = [_P] * 6
lib.moga_residual_norm.argtypes = [_P] * 12
lib.moga_residual_norm_backward.argtypes = [_P] * 14 + [_S, _P]
lib.moga_rope.argtypes = [_P, _P, _P, _I, _P, _P, _P, _P, _I, _P]
lib.moga_permute_rope.argtypes = [_P, _P, _P, _I] + [_P] * 11 + [_S, _P]
lib.moga_permute_rope_backward.argtypes = [_P, _P, _P, _I] + [_P] * 8
lib.moga_forward_rope.argtypes = [_P, _P, _P, _I] + [_P] * 12 + [_S, _P]
lib.moga_backward_rope.argtypes = [_P, _P, _P, _I] + [_P] * 15 + [_S, _P]


# the current device and its current stream, without the objects that torch.cuda makes of them
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)


def _here(where, t):
    """The current device's index, which is where ``t`` has to be."""
    if not t.is_cuda or t.get_device() != _current_device():
        raise MogaError(1, where, f"a tensor on {t.device}, not on the current CUDA device")
    return t.get_device()


def _expect(where, device, dtype, numel, *tensors):
    """Addresses of contiguous tensors of ``numel`` elements on ``device`` (0 for None)."""
    out = []
    for t in tensors:
        if t is None:
            out.append(0)
        elif t.dtype is dtype and t.numel() == numel and t.is_contiguous() and t.get_device() == device:
            out.append(t.data_ptr())
        else:
            raise MogaError(1, where, f"expected {numel} contiguous elements of {dtype} on device {device}, got "
                                      f"{tuple(t.shape)} {t.dtype} on {t.device}, strides {t.stride()}")
    return out


def _expect_heads(where, device, s, *tensors):
    """Addresses of [B, H, N, D] tensors with the shape's strides, counted from a tensor's first element."""
    if not (s.q_stride_b or s.q_stride_h or s.q_stride_n) or s.N == 0:
        return _expect(where, device, _DTYPES[s.dtype], s.B * s.H * s.N * s.D, *tensors)
    need = (s.B - 1) * s.q_stride_b + (s.H - 1) * s.q_stride_h + (s.N - 1) * s.q_stride_n + s.D
    out = []
    for t in tensors:
        if t is None:
            out.append(0)
            continue
        if t.dtype is not _DTYPES[s.dtype] or t.get_device() != device:
            raise MogaError(1, where, f"expected {_DTYPES[s.dtype]} on device {device}, got {t.dtype} on {t.device}")
        if t.untyped_storage().nbytes() // t.element_size() - t.storage_offset() < need:
            raise MogaError(1, where, f"the shape's strides reach past the memory of a {tuple(t.shape)} tensor")
        out.append(t.data_ptr())
    return out


def _expect_params(where, device, s, n, *tensors):
    return _expect(where, device, torch.float32, s.C * (s.B if n.per_batch else 1), *tensors)


def _rope_args(where, device, s, plan, pos):
    """Plan, positions ([N, axes], [1, N, axes] or [B, N, axes] int32, or None) and whether they differ by batch item."""
    if pos is None:
        return ctypes.byref(plan), 0, 0
    per_batch = 1 if pos.dim() == 3 and pos.shape[0] == s.B and s.B > 1 else 0
    if tuple(pos.shape[-2:]) != (s.N, plan.n_axes):
        raise MogaError(1, where, f"pos: expected [..., {s.N}, {plan.n_axes}], got {tuple(pos.shape)}")
    return ctypes.byref(plan), _expect(where, device, torch.int32, (s.B if per_batch else 1) * s.N * plan.n_axes, pos)[0], per_batch


def _ws(where, device, ws):
    if ws.get_device() != device or not ws.is_contiguous():
        raise MogaError(1, where, f"the workspace is on {ws.device}, not on device {device}, or not contiguous")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _drop(where, device, drop):
    """The descriptor's address (None: no dropout); its step word, which the kernels read, has to be on their device."""
    step = getattr(drop, "_step", None)
    if step is not None and step.get_device() != device:
        raise MogaError(1, where, f"the dropout's step word is on {step.device}, not on device {device}")
    return None if drop is None else ctypes.byref(drop)


def make_norm(eps=1e-5, per_batch=False) -> MogaNorm:
    return MogaNorm(eps, 1 if per_batch else 0)


def make_dropout(p, seed, offset=0, step=None) -> MogaDropout:
    """``step``: None, or a CUDA int64 tensor of one element that is added to ``offset`` on the device
    (keep it alive as long as the descriptor is used)."""
    if step is not None and (not step.is_cuda or step.dtype is not torch.int64 or step.numel() != 1):
        raise MogaError(1, "make_dropout", "step: expected one int64 element on the GPU")
    d = MogaDropout(p, seed % (1 << 64), offset % (1 << 64), 0 if step is None else step.data_ptr())
    d._step = step
    return d


def moga_layernorm_backward_workspace_bytes(shape, norm) -> int:
    return int(lib.moga_layernorm_backward_workspace_bytes(ctypes.byref(shape), ctypes.byref(norm)))


def moga_layernorm(shape, norm, X, W, bias, Y, mean=None, rstd=None):
    where = "moga_layernorm"
    dev, rows = _here(where, X), shape.B * shape.N
    x, y = _expect(where, dev, _DTYPES[shape.dtype], rows * shape.C, X, Y)
    w, b = _expect_params(where, dev, shape, norm, W, bias)
    m, r = _expect(where, dev, torch.float32, rows, mean, rstd)
    _check(lib.moga_layernorm(ctypes.byref(shape), ctypes.byref(norm), x, w, b, y, m, r, _stream_of(dev)), where)


def moga_layernorm_backward(shape, norm, X, W, mean, rstd, dY, dX, dW, dbias, ws):
    where = "moga_layernorm_backward"
    dev, rows = _here(where, X), shape.B * shape.N
    x, dy, dx = _expect(where, dev, _DTYPES[shape.dtype], rows * shape.C, X, dY, dX)
    w, dw, db = _expect_params(where, dev, shape, norm, W, dW, dbias)
    m, r = _expect(where, dev, torch.float32, rows, mean, rstd)
    _check(lib.moga_layernorm_backward(ctypes.byref(shape), ctypes.byref(norm), x, w, m, r, dy, dx, dw, db,
                                       *_ws(where, dev, ws), _stream_of(dev)), where)


def moga_dropout_add(shape, drop, X, R, Y):
    """Y = R + dropout(X); R may be None."""
    where = "moga_dropout_add"
    dev = _here(where, X)
    x, r, y = _expect(where, dev, _DTYPES[shape.dtype], shape.B * shape.N * shape.C, X, R, Y)
    _check(lib.moga_dropout_add(ctypes.byref(shape), _drop(where, dev, drop), x, r, y, _stream_of(dev)), where)


def moga_residual_norm(shape, norm, drop, X, R, W, bias, Hs, Y, mean=None, rstd=None):
    """Hs = R + dropout(X) (drop may be None), Y = layer norm of the stored Hs."""
    where = "moga_residual_norm"
    dev, rows = _here(where, X), shape.B * shape.N
    x, res, h, y = _expect(where, dev, _DTYPES[shape.dtype], rows * shape.C, X, R, Hs, Y)
    w, b = _expect_params(where, dev, shape, norm, W, bias)
    m, r = _expect(where, dev, torch.float32, rows, mean, rstd)
    _check(lib.moga_residual_norm(ctypes.byref(shape), ctypes.byref(norm), _drop(where, dev, drop), x, res, w, b, h, y, m, r,
                                  _stream_of(dev)), where)


def moga_residual_norm_backward(shape, norm, drop, Hs, W, mean, rstd, dY, dH, dX, dR, dW, dbias, ws):
    where = "moga_residual_norm_backward"
    dev, rows = _here(where, Hs), shape.B * shape.N
    h, dy, dh, dx, dr = _expect(where, dev, _DTYPES[shape.dtype], rows * shape.C, Hs, dY, dH, dX, dR)
    w, dw, db = _expect_params(where, dev, shape, norm, W, dW, dbias)
    m, r = _expect(where, dev, torch.float32, rows, mean, rstd)
    _check(lib.moga_residual_norm_backward(ctypes.byref(shape), ctypes.byref(norm), _drop(where, dev, drop), h, w, m, r, dy, dh,
                                           dx, dr, dw, db, *_ws(where, dev, ws), _stream_of(dev)), where)


ROPE_LAYOUTS = {"interleaved": 0, "half": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "base": 2, "by_parts": 3}


def make_rope(axis_dims, layout="interleaved", scaling="none", base=10000.0, factor=1.0, original_length=0.0,
              beta_slow=1.0, beta_fast=32.0, amplitude=1.0, grid=(0, 0), start=(0, 0, 0)) -> MogaRopePlan:
    """The plan of rotary positions: ``axis_dims`` rotated channels of each of 1 to 3 axes, ``factor`` one
    number or one for each axis, ``grid`` (height, width) of a frame for positions taken from the token index."""
    axis_dims = [axis_dims] if isinstance(axis_dims, int) else list(axis_dims)
    n = len(axis_dims)
    if not 1 <= n <= 3:
        raise MogaError(1, "make_rope", "1 to 3 axes")
    if layout not in ROPE_LAYOUTS or scaling not in ROPE_SCALINGS:
        raise MogaError(1, "make_rope", f"layout {layout!r}, scaling {scaling!r}")
    factors = [factor] * n if isinstance(factor, (int, float)) else list(factor)
    start, grid = list(start), list(grid)
    if len(factors) != n or len(start) not in (n, 3) or len(grid) != 2:
        raise MogaError(1, "make_rope", f"factor and start: one for each of the {n} axes; grid: height and width")
    for name, values in (("axis_dims", axis_dims), ("start", start), ("grid", grid)):
        if not all(-2 ** 31 <= v < 2 ** 31 for v in values):       # the C side would take the low 32 bits
            raise MogaError(1, "make_rope", f"{name}: {values} does not fit 32 bits")
    fill = lambda v, x: v[:n] + [x] * (3 - n)
    cfg = MogaRopeConfig(ROPE_LAYOUTS[layout], ROPE_SCALINGS[scaling], n, (ctypes.c_int32 * 3)(*fill(axis_dims, 0)),
                         grid[0], grid[1], (ctypes.c_int32 * 3)(*fill(start, 0)), amplitude, base,
                         (ctypes.c_double * 3)(*fill(factors, 1.0)), original_length, beta_slow, beta_fast)
    plan = MogaRopePlan()
    _check(lib.moga_rope_build(ctypes.byref(cfg), ctypes.byref(plan)), "make_rope")
    return plan


def moga_rope(shape, plan, pos, Q, K, Qo, Ko, transpose=False):
    """K and Ko may be None; Qo may be Q, Ko may be K."""
    where = "moga_rope"
    dev = _here(where, Q)
    q, k, qo, ko = _expect_heads(where, dev, shape, Q, K, Qo, Ko)
    _check(lib.moga_rope(ctypes.byref(shape), *_rope_args(where, dev, shape, plan, pos), q, k, qo, ko,
                         1 if transpose else 0, _stream_of(dev)), where)


def moga_permute_rope(shape, plan, pos, gid, Q, K, V, perm, inv, offsets, Qp, Kp, Vp, ws):
    where = "moga_permute_rope"
    dev, T = _here(where, Q), shape.N * shape.k
    q, k, v = _expect_heads(where, dev, shape, Q, K, V)
    qp, kp, vp = _expect(where, dev, _DTYPES[shape.dtype], shape.B * shape.H * T * shape.D, Qp, Kp, Vp)
    g, p, i = _expect(where, dev, torch.int32, shape.B * T, gid, perm, inv)
    o, = _expect(where, dev, torch.int32, shape.B * (shape.M + 1), offsets)
    _check(lib.moga_permute_rope(ctypes.byref(shape), *_rope_args(where, dev, shape, plan, pos), g, q, k, v, p, i, o, qp,
                                 kp, vp, *_ws(where, dev, ws), _stream_of(dev)), where)


def moga_permute_rope_backward(shape, plan, pos, dQp, dKp, dVp, inv, dQ, dK, dV):
    where = "moga_permute_rope_backward"
    dev, T = _here(where, dQp), shape.N * shape.k
    qp, kp, vp = _expect(where, dev, _DTYPES[shape.dtype], shape.B * shape.H * T * shape.D, dQp, dKp, dVp)
    q, k, v = _expect_heads(where, dev, shape, dQ, dK, dV)
    i, = _expect(where, dev, torch.int32, shape.B * T, inv)
    _check(lib.moga_permute_rope_backward(ctypes.byref(shape), *_rope_args(where, dev, shape, plan, pos), qp, kp, vp, i, q,
                                          k, v, _stream_of(dev)), where)


def moga_forward_rope(shape, plan, pos, X, Wr, bias, Q, K, V, O, ws, gid_out=None, gate_out=None, perm_out=None,
                      offsets_out=None):
    where = "moga_forward_rope"
    dev, T = _here(where, Q), shape.B * shape.N * shape.k
    q, k, v, o = _expect_heads(where, dev, shape, Q, K, V, O)
    x, = _expect(where, dev, _DTYPES[shape.dtype], shape.B * shape.N * shape.C, X)
    w, = _expect(where, dev, torch.float32, shape.C * shape.M, Wr)
    b, = _expect(where, dev, torch.float32, shape.M, bias)
    gid, perm = _expect(where, dev, torch.int32, T, gid_out, perm_out)
    gate, = _expect(where, dev, torch.float32, T, gate_out)
    off, = _expect(where, dev, torch.int32, shape.B * (shape.M + 1), offsets_out)
    _check(lib.moga_forward_rope(ctypes.byref(shape), *_rope_args(where, dev, shape, plan, pos), x, w, b, q, k, v, o, gid,
                                 gate, perm, off, *_ws(where, dev, ws), _stream_of(dev)), where)


def moga_backward_rope(shape, plan, pos, Qp, Kp, Vp, Op, lse, gate, perm, inv, offsets, dO, dQ, dK, dV, dgate, ws):
    where = "moga_backward_rope"
    dev, T = _here(where, Qp), shape.N * shape.k
    qp, kp, vp, op = _expect(where, dev, _DTYPES[shape.dtype], shape.B * shape.H * T * shape.D, Qp, Kp, Vp, Op)
    do, dq, dk, dv = _expect_heads(where, dev, shape, dO, dQ, dK, dV)
    ls, = _expect(where, dev, torch.float32, shape.B * shape.H * T, lse)
    g, dg = _expect(where, dev, torch.float32, shape.B * T, gate, dgate)
    p, i = _expect(where, dev, torch.int32, shape.B * T, perm, inv)
    off, = _expect(where, dev, torch.int32, shape.B * (shape.M + 1), offsets)
    _check(lib.moga_backward_rope(ctypes.byref(shape), *_rope_args(where, dev, shape, plan, pos), qp, kp, vp, op, ls, g, p,
                                  i, off, do, dq, dk, dv, dg, *_ws(where, dev, ws), _stream_of(dev)), where)


def moga_forward_host_bytes(shape, heads_per_chunk) -> int:
    return int(lib.moga_forward_host_bytes(ctypes.byref(shape), ctypes.c_int32(heads_per_chunk)))


def moga_forward_host(shape, X, Wr, bias, Q, K, V, O, arena, heads_per_chunk, gid_out=None, gate_out=None):
    """Forward from host tensors (torch CPU tensors, ideally pinned); ``arena`` is a CUDA uint8 tensor."""
    _check(lib.moga_forward_host(ctypes.byref(shape), _ptr(X), _ptr(Wr), _ptr(bias), _ptr(Q), _ptr(K), _ptr(V),
                                 _ptr(O), _ptr(gid_out), _ptr(gate_out), _ptr(arena),
                                 ctypes.c_size_t(arena.numel()), ctypes.c_int32(heads_per_chunk), _stream()),
           "moga_forward_host")


def make_static_lists(lists, F, tokens_per_frame, device="cuda"):
    """Device copies of moga_stga_build's arrays wrapped for moga_visual_forward.  Returns the
    ctypes struct and the tensors that keep the device memory alive."""
    keep = {k: torch.from_numpy(lists[k]).to(device) for k in ("q_idx", "q_inv", "q_offsets", "kv_idx", "kv_offsets")}
    st = MogaStaticLists(lists["G"], lists["Tkv"], F, tokens_per_frame, *(keep[k].data_ptr() for k in
                         ("q_idx", "q_inv", "q_offsets", "kv_idx", "kv_offsets")))
    return st, keep


def moga_visual_workspace_bytes(shape, static_lists) -> int:
    return int(lib.moga_visual_workspace_bytes(ctypes.byref(shape), ctypes.byref(static_lists)))


def moga_visual_forward(shape, X, Wr, bias, Q, K, V, O, static_lists, ws):
    _check(lib.moga_visual_forward(ctypes.byref(shape), _ptr(X), _ptr(Wr), _ptr(bias), _ptr(Q), _ptr(K), _ptr(V),
                                   _ptr(O), ctypes.byref(static_lists), _ptr(ws), ctypes.c_size_t(ws.numel()),
                                   _stream()), "moga_visual_forward")


def moga_selftest_wait_timeout(ws, limit_ns):
    _check(lib.moga_selftest_wait_timeout(_ptr(ws), ctypes.c_size_t(ws.numel()), ctypes.c_uint64(limit_ns),
                                          _stream()), "moga_selftest_wait_timeout")


MOGA_ATTN_AUTO, MOGA_ATTN_SINGLE, MOGA_ATTN_PAIR = 0, 1, 2


def moga_set_fused_topk(on: bool):
    _check(lib.moga_set_fused_topk(ctypes.c_int32(1 if on else 0)), "moga_set_fused_topk")


def moga_set_attn_kernel(mode: int):
    _check(lib.moga_set_attn_kernel(ctypes.c_int32(mode)), "moga_set_attn_kernel")


def moga_last_device_status(ws):
    """(status code, detail word) of the most recent call that used ``ws``; synchronises."""
    detail = ctypes.c_uint32(0)
    code = lib.moga_last_device_status(_ptr(ws), _stream(), ctypes.byref(detail))
    return int(code), int(detail.value)
