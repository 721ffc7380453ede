"""Binding of libgcpsl.so (include/gcpsl.h), by ctypes and, for regular calls of the operators on tensors, _ops.so:
argument marshalling only.

Every computation of the hot path runs in the library's HIP kernels.  PyTorch
is used for device memory (the caller-owned buffers the C ABI works in) and
for the stream handle.  If the library has not been built, every entry point
raises; there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import NamedTuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgcpsl.so")

OK, EINVAL, ESTATE, EHIP, EUNSUPPORTED = 0, -1, -2, -3, -4
RULES = {"random": 0, "size": 1, "label_l1": 2, "label_jsd": 3}
DTYPES = {"f32": 0, "bf16": 1}
CONV3X3, MAXPOOL2, AVGPOOL, LINEAR, BATCHNORM, GROUPNORM, BLOCK = 1, 2, 3, 4, 5, 6, 7
RESIDUAL, STRIDE2 = 1, 2
SCHEDULES = {"lockstep": 0, "epoch": 1}
PAYLOAD = ("activations", "cut_grads", "client_grads", "client_model", "fusion")  # GCPSL_PAYLOAD_* order

EXPORTS = ["gcpsl_param_count", "gcpsl_state_count", "gcpsl_workspace_bytes", "gcpsl_assign", "gcpsl_create",
           "gcpsl_create_static",
           "gcpsl_sample", "gcpsl_step", "gcpsl_step_replica", "gcpsl_epoch_rounds", "gcpsl_fuse",
           "gcpsl_fuse_replicas", "gcpsl_fuse_partial", "gcpsl_fuse_finalise",
           "gcpsl_participation", "gcpsl_batch_deviation", "gcpsl_payload",
           "gcpsl_cluster_sizes", "gcpsl_tensor", "gcpsl_timing", "gcpsl_timing_read",
           "gcpsl_group_forward", "gcpsl_group_input_grad", "gcpsl_group_workspace_bytes", "gcpsl_group_weight_grad",
           "gcpsl_dropout", "gcpsl_score_workspace_bytes", "gcpsl_score", "gcpsl_score_grad",
           "gcpsl_destroy", "gcpsl_last_error"]


class GCPSLError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"gcpsl error {code}: {msg}")
        self.code = code


class Layer(C.Structure):
    _fields_ = [("kind", C.c_int32), ("cin", C.c_int32), ("cout", C.c_int32), ("flags", C.c_int32),
                ("groups", C.c_int32)]


class Desc(C.Structure):
    _fields_ = [
        ("K", C.c_int32), ("C", C.c_int32), ("B", C.c_int32), ("L", C.c_int32),
        ("H", C.c_int32), ("W", C.c_int32), ("Cin", C.c_int32), ("dtype", C.c_int32),
        ("n_examples", C.c_int64), ("n_layers", C.c_int32), ("cut", C.c_int32),
        ("layers", C.POINTER(Layer)), ("lr", C.c_float), ("momentum", C.c_float),
        ("weight_decay", C.c_float), ("nesterov", C.c_int32), ("label_smoothing", C.c_float),
        ("seed", C.c_uint64), ("max_steps", C.c_int64), ("max_window", C.c_int32),
        ("schedule", C.c_int32), ("client_of_example", C.POINTER(C.c_int32)),
        ("cluster_of_client", C.POINTER(C.c_int32)), ("images", C.c_void_p),
        ("labels", C.c_void_p), ("theta", C.c_void_p), ("momentum_buf", C.c_void_p), ("norm_state", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class KernelStat(C.Structure):
    _fields_ = [("name", C.c_char * 64), ("launches", C.c_int64), ("ms", C.c_double),
                ("flops", C.c_double), ("bytes", C.c_double)]


_lib = None


def lib():
    """Load libgcpsl.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2609_29395_amd.build`")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
    P = C.POINTER
    L.gcpsl_param_count.argtypes = [P(Desc), P(i64), P(i64)]
    L.gcpsl_state_count.argtypes = [P(Desc), P(i64)]
    L.gcpsl_workspace_bytes.argtypes = [P(Desc), P(C.c_size_t)]
    L.gcpsl_assign.argtypes = [i32, i32, i32, u64, P(i64), P(i64), i32, P(i32)]
    L.gcpsl_create.argtypes = [P(Desc), P(vp)]
    L.gcpsl_create_static.argtypes = [P(Desc), P(vp)]
    L.gcpsl_sample.argtypes = [vp, i64, i32, vp, vp]
    L.gcpsl_step.argtypes = [vp, i64, vp, vp]
    L.gcpsl_step_replica.argtypes = [vp, i64, i32, vp, vp]
    L.gcpsl_epoch_rounds.argtypes = [vp, P(i64), P(i64)]
    L.gcpsl_fuse.argtypes = [vp, vp]
    L.gcpsl_fuse_replicas.argtypes = [vp, i32, i64, P(i64), vp]
    L.gcpsl_fuse_partial.argtypes = [vp, vp, vp]
    L.gcpsl_fuse_finalise.argtypes = [vp, vp, i64, vp]
    L.gcpsl_participation.argtypes = [vp, P(i64), P(i64), P(i32)]
    L.gcpsl_batch_deviation.argtypes = [vp, P(i64), P(i64), P(i64), P(i64)]
    L.gcpsl_payload.argtypes = [vp, P(i64)]
    L.gcpsl_cluster_sizes.argtypes = [vp, P(i64)]
    L.gcpsl_tensor.argtypes = [vp, C.c_char_p, P(vp), P(i64), P(i32)]
    L.gcpsl_timing.argtypes = [vp, i32]
    L.gcpsl_timing_read.argtypes = [vp, P(KernelStat), i32, P(i32)]
    f64, size = C.c_double, C.c_size_t
    group = [i32, i32, i64, i32, i32, vp]  # dtype, G, rows, n, k, offsets
    L.gcpsl_group_forward.argtypes = group + [vp, i64, vp, i64, vp, i64, i32, f64, u64, vp, i64, vp]
    L.gcpsl_group_input_grad.argtypes = group + [vp, i64, vp, i64, vp, i64, f64, vp, i64, vp]
    L.gcpsl_group_workspace_bytes.argtypes = group[:5] + [P(size)]
    L.gcpsl_group_weight_grad.argtypes = group + [vp, i64, vp, i64, vp, i64, vp, i64, vp, size, vp]
    L.gcpsl_dropout.argtypes = [i32, i64, i64, vp, i64, f64, u64, vp, i64, vp]
    L.gcpsl_score_workspace_bytes.argtypes = [i32, i64, i32, i32, P(size)]
    L.gcpsl_score.argtypes = [i32, i64, i32, vp, i64, vp, i32, vp, vp, vp, vp, vp, vp, size, vp]
    L.gcpsl_score_grad.argtypes = [i32, i64, i32, vp, i64, vp, vp, vp, vp, vp, vp, i64, vp]
    L.gcpsl_destroy.argtypes = [vp]
    L.gcpsl_destroy.restype = None
    L.gcpsl_last_error.restype = C.c_char_p
    for name in EXPORTS:
        if name not in ("gcpsl_destroy", "gcpsl_last_error"):
            getattr(L, name).restype = C.c_int
    _lib = L
    return L


def _check(rc):
    if rc != OK:
        raise GCPSLError(rc, lib().gcpsl_last_error().decode())


def _i32p(a):
    return a.ctypes.data_as(C.POINTER(C.c_int32))


def _i64p(a):
    return a.ctypes.data_as(C.POINTER(C.c_int64))


def layers_struct(layers):
    arr = (Layer * len(layers))()
    for i, spec in enumerate(layers):
        kind = spec[0]
        if kind == "conv":
            arr[i] = Layer(CONV3X3, spec[1], spec[2], RESIDUAL if spec[3] else 0, 0)
        elif kind == "maxpool":
            arr[i] = Layer(MAXPOOL2, 0, 0, 0, 0)
        elif kind == "avgpool":
            arr[i] = Layer(AVGPOOL, 0, 0, 0, 0)
        elif kind == "linear":
            arr[i] = Layer(LINEAR, spec[1], spec[2], 0, 0)
        elif kind == "bnorm":
            arr[i] = Layer(BATCHNORM, spec[1], spec[1], 0, 0)
        elif kind == "gnorm":
            arr[i] = Layer(GROUPNORM, spec[1], spec[1], 0, spec[2])
        elif kind == "block":
            if spec[3] not in (1, 2):
                raise ValueError("block stride must be 1 or 2")
            arr[i] = Layer(BLOCK, spec[1], spec[2], STRIDE2 if spec[3] == 2 else 0, spec[4])
        else:
            raise ValueError(kind)
    return arr


def assign(rule, K, C_, seed, counts=None, hist=None):
    """gcpsl_assign: Alg. 1 cluster_of_client (host)."""
    out = np.zeros(K, dtype=np.int32)
    cnt = None if counts is None else np.ascontiguousarray(counts, dtype=np.int64)
    h = None if hist is None else np.ascontiguousarray(hist, dtype=np.int64)
    L = 0 if h is None else h.shape[1]
    _check(lib().gcpsl_assign(K, C_, RULES[rule] if isinstance(rule, str) else rule, seed,
                              None if cnt is None else _i64p(cnt), None if h is None else _i64p(h),
                              L, _i32p(out)))
    return out


def fuse_replicas(theta, weights, stream=None):
    """gcpsl_fuse_replicas: Eq. 5 in place on a [C][P] fp32 torch tensor on
    the GPU with host weights [C]."""
    if theta.dim() != 2 or theta.dtype.is_floating_point is False or theta.element_size() != 4:
        raise ValueError("theta must be a [C][P] fp32 tensor")
    if not theta.is_contiguous():
        raise ValueError("theta must be contiguous")
    w = np.ascontiguousarray(weights, dtype=np.int64)
    if w.shape != (theta.shape[0],):
        raise ValueError("weights must have one entry per replica")
    _check(lib().gcpsl_fuse_replicas(C.c_void_p(theta.data_ptr()), theta.shape[0], theta.shape[1], _i64p(w),
                                     _stream(stream)))


# ------------------------------------------ operators on tensors, without a context
#
# Tensors are on the current GPU, rows of consecutive elements (any row
# stride).  Every function returns the tensors it wrote: those given as out,
# dw, db, or new ones.  stream: a torch stream, the current one by default.
# What is newly allocated for another stream comes from that stream's memory and
# is marked as used on the current one too; as with any work of two streams, the
# caller makes `stream` wait for inputs made elsewhere, keeps them until it is
# done with them (or marks them as used there: Tensor.record_stream), and makes
# whoever reads the results wait for `stream`.
#
# Autograd does not see these calls: tensors that require a gradient are taken as
# plain ones, results never require one, and what is written (out, dw, db) does
# not count as changed.  The backward passes are the functions for them here.
#
# The smallest calls are bound by the host.  A call on the current stream that
# brings no workspace goes through csrc/bind.cpp in one native call, which
# checks, allocates and launches; what that does not take (it answers None) and
# every other call is checked here, by the same rules, with a message.

_torch = None
_types = {}
_ops = None
_ENTRIES = ["gcpsl_group_forward", "gcpsl_group_input_grad", "gcpsl_group_workspace_bytes", "gcpsl_group_weight_grad",
            "gcpsl_dropout", "gcpsl_score_workspace_bytes", "gcpsl_score", "gcpsl_score_grad"]


def _load_torch():
    global _torch
    import torch
    _types.update({torch.float32: 0, torch.bfloat16: 1})
    _torch = torch
    return torch


def _native():
    """csrc/bind.cpp's module, on the entries of the library that lib() loaded (raises if it has not been built)."""
    global _ops
    if _ops is None:
        torch = _torch or _load_torch()
        from . import _ops as module
        L = lib()
        module.init(tuple(C.cast(getattr(L, name), C.c_void_p).value for name in _ENTRIES), torch._C._cuda_getDevice,
                    torch._C._cuda_getCurrentRawStream, Scores)
        _ops = module
    return _ops


def _done(result):
    """Whether a native call made its result; raises for the library's error code."""
    if result is None:
        return False
    if result.__class__ is int:
        _check(result)
    return True


def _begin(t, stream):
    """(torch, type code, stream handle, device) of a call on t's GPU."""
    torch = _torch or _load_torch()
    code = _types.get(t.dtype)
    if code is None:
        raise ValueError(f"fp32 or bf16 tensors only, not {t.dtype}")
    device = t.get_device()
    if device < 0 or device != torch._C._cuda_getDevice():
        raise ValueError("tensors must be on the current GPU")
    handle = torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream
    return torch, code, handle, device


def _empty(like, shape, dtype, stream):
    current = None if stream is None else _torch.cuda.current_stream(like.device)
    if stream == current:
        return like.new_empty(*shape, dtype=dtype)
    # from that stream's memory: a block freed on the current stream may still be in use by work queued there
    with _torch.cuda.stream(stream):
        t = like.new_empty(*shape, dtype=dtype)
    t.record_stream(current)  # where the caller may go on with it
    return t


def _rows(t, what, dtype, device, rows=None, cols=None):
    """(address, row stride) of a [rows][cols] tensor."""
    shape = t.shape
    if len(shape) != 2 or t.dtype != dtype or t.get_device() != device:
        raise ValueError(f"{what} must be a [rows][cols] {dtype} tensor on the same GPU")
    r, c = shape
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        raise ValueError(f"{what} must be ({rows}, {cols}), is {tuple(shape)}")
    ld, step = t.stride()
    if step != 1 and c > 1:
        raise ValueError(f"{what}: a row's elements must be consecutive")
    return t.data_ptr(), (ld if r > 1 else c)


def _out(like, out, rows, cols, dtype, device, stream):
    """(tensor, address, row stride) of a [rows][cols] result: out, or a new one."""
    if out is None:
        out = _empty(like, (rows, cols), dtype, stream)
        return out, out.data_ptr(), cols
    return out, *_rows(out, "out", dtype, device, rows, cols)


def _vector(t, what, dtype, n, device):
    """Address of a vector of n elements, None for None."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != (n,) or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} vector of {n} on the same GPU")
    return t.data_ptr()


def _offsets(t, torch, device):
    if t.dim() != 1 or t.shape[0] < 2:
        raise ValueError("offsets must be a vector of G + 1 entries")
    G = t.shape[0] - 1
    return _vector(t, "offsets", torch.int32, G + 1, device), G


def _weights(t, what, dtype, device, shape):
    """(address, stride from group to group) of [G][n][k] weights or [G][n]
    biases, each group's consecutive."""
    if t.shape != shape or t.dtype != dtype or t.get_device() != device:
        raise ValueError(f"{what} must be {dtype} {shape} on the same GPU, is {t.dtype} {tuple(t.shape)}")
    st = t.stride()
    if (st[-1] != 1 and shape[-1] > 1) or (len(shape) == 3 and shape[1] > 1 and st[1] != shape[2]):
        raise ValueError(f"{what}: a group's entries must be consecutive")
    return t.data_ptr(), (st[0] if shape[0] > 1 else shape[1] * (shape[2] if len(shape) == 3 else 1))


def _workspace(like, workspace, nbytes, device, stream):
    """(address, bytes, tensor to keep) of a call's workspace."""
    if workspace is None:
        if nbytes == 0:
            return None, 0, None
        workspace = _empty(like, (nbytes,), _torch.uint8, stream)
    elif workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous on the same GPU")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def group_forward(x, offsets, w, bias=None, relu=False, p=0.0, seed=0, out=None, stream=None):
    """gcpsl_group_forward: [rows][n] = dropout(relu(W_g x_r + b_g)) of x
    [rows][k], rows offsets[g] to offsets[g + 1] through w[g] of [G][n][k]
    and bias[g] of [G][n] (fp32)."""
    if stream is None:
        r = (_ops or _native()).group_forward(x, offsets, w, bias, relu, p, seed, out)
        if _done(r):
            return r
    torch, code, handle, device = _begin(x, stream)
    dtype = x.dtype
    xp, ldx = _rows(x, "x", dtype, device)
    off, G = _offsets(offsets, torch, device)
    rows, k = x.shape
    n = w.shape[1] if w.dim() == 3 else -1
    wp, w_gs = _weights(w, "w", dtype, device, (G, n, k))
    bp, b_gs = (None, 0) if bias is None else _weights(bias, "bias", torch.float32, device, (G, n))
    y, yp, ldy = _out(x, out, rows, n, dtype, device, stream)
    _check(lib().gcpsl_group_forward(code, G, rows, n, k, off, xp, ldx, wp, w_gs, bp, b_gs, 1 if relu else 0, p, seed,
                                     yp, ldy, handle))
    return y


def group_input_grad(dy, offsets, w, gate=None, p=0.0, out=None, stream=None):
    """gcpsl_group_input_grad: [rows][k] = W_g^T dy_r of dy [rows][n]; with
    the layer's input as gate, which a ReLU and a dropout of probability p
    made, the gradient through those."""
    if stream is None:
        r = (_ops or _native()).group_input_grad(dy, offsets, w, gate, p, out)
        if _done(r):
            return r
    torch, code, handle, device = _begin(dy, stream)
    dtype = dy.dtype
    dp, lddy = _rows(dy, "dy", dtype, device)
    off, G = _offsets(offsets, torch, device)
    rows, n = dy.shape
    k = w.shape[2] if w.dim() == 3 else -1
    wp, w_gs = _weights(w, "w", dtype, device, (G, n, k))
    gp, ldg = (None, 0) if gate is None else _rows(gate, "gate", dtype, device, rows, k)
    dx, xp, lddx = _out(dy, out, rows, k, dtype, device, stream)
    _check(lib().gcpsl_group_input_grad(code, G, rows, n, k, off, dp, lddy, wp, w_gs, gp, ldg, p, xp, lddx, handle))
    return dx


@functools.lru_cache(maxsize=1024)
def _group_workspace_bytes(code, G, rows, n, k):
    b = C.c_size_t()
    _check(lib().gcpsl_group_workspace_bytes(code, G, rows, n, k, C.byref(b)))
    return b.value


def group_workspace_bytes(dtype, G, rows, n, k):
    """gcpsl_group_workspace_bytes for "f32" or "bf16" tensors."""
    return _group_workspace_bytes(DTYPES[dtype], G, rows, n, k)


def group_weight_grad(dy, x, offsets, dw=None, db=None, bias=True, workspace=None, stream=None):
    """gcpsl_group_weight_grad: (dw [G][n][k], db [G][n]) in fp32 from dy
    [rows][n] and x [rows][k]; db is None with bias=False."""
    if stream is None and workspace is None:
        r = (_ops or _native()).group_weight_grad(dy, x, offsets, dw, db, bias)
        if _done(r):
            return r
    torch, code, handle, device = _begin(dy, stream)
    dp, lddy = _rows(dy, "dy", dy.dtype, device)
    off, G = _offsets(offsets, torch, device)
    rows, n = dy.shape
    xp, ldx = _rows(x, "x", dy.dtype, device, rows)
    k = x.shape[1]
    if dw is None:
        dw = _empty(dy, (G, n, k), torch.float32, stream)
        wp, w_gs = dw.data_ptr(), n * k
    else:
        wp, w_gs = _weights(dw, "dw", torch.float32, device, (G, n, k))
    if db is not None:
        bp, b_gs = _weights(db, "db", torch.float32, device, (G, n))
    elif bias:
        db = _empty(dy, (G, n), torch.float32, stream)
        bp, b_gs = db.data_ptr(), n
    else:
        bp, b_gs = None, 0
    ptr, size, keep = _workspace(dy, workspace, _group_workspace_bytes(code, G, rows, n, k), device, stream)
    _check(lib().gcpsl_group_weight_grad(code, G, rows, n, k, off, dp, lddy, xp, ldx, wp, w_gs, bp, b_gs, ptr, size,
                                         handle))
    return dw, db


def dropout(x, p, seed, out=None, stream=None):
    """gcpsl_dropout of x [rows][cols]; out may be x.  The same call on the
    output's gradient is the backward pass."""
    if stream is None:
        r = (_ops or _native()).dropout(x, p, seed, out)
        if _done(r):
            return r
    torch, code, handle, device = _begin(x, stream)
    xp, ldx = _rows(x, "x", x.dtype, device)
    rows, cols = x.shape
    y, yp, ldy = _out(x, out, rows, cols, x.dtype, device, stream)
    _check(lib().gcpsl_dropout(code, rows, cols, xp, ldx, p, seed, yp, ldy, handle))
    return y


class Scores(NamedTuple):
    logp: object       # [rows] log probability of each row's label (None without labels)
    entropy: object    # [rows]
    lse: object        # [rows] log sum of exponentials
    top_logp: object   # [rows][top], in decreasing order
    top_class: object  # [rows][top] int32


@functools.lru_cache(maxsize=1024)
def _score_workspace_bytes(code, rows, L, top):
    b = C.c_size_t()
    _check(lib().gcpsl_score_workspace_bytes(code, rows, L, top, C.byref(b)))
    return b.value


def score_workspace_bytes(dtype, rows, L, top=0):
    """gcpsl_score_workspace_bytes for "f32" or "bf16" logits."""
    return _score_workspace_bytes(DTYPES[dtype], rows, L, top)


def score(logits, labels=None, top=0, workspace=None, stream=None):
    """gcpsl_score of logits [rows][L] and int32 labels [rows]."""
    if stream is None and workspace is None:
        r = (_ops or _native()).score(logits, labels, top)
        if _done(r):
            return r
    torch, code, handle, device = _begin(logits, stream)
    zp, ldz = _rows(logits, "logits", logits.dtype, device)
    rows, L = logits.shape
    yp = _vector(labels, "labels", torch.int32, rows, device)
    ptr, size, keep = _workspace(logits, workspace, _score_workspace_bytes(code, rows, L, top), device, stream)
    # one allocation for all results: an allocation and a view cost the host about a microsecond each
    held = _empty(logits, (rows * (3 + 2 * top),), torch.float32, stream)
    logp, entropy, lse, top_logp, top_class = held.split_with_sizes((rows, rows, rows, rows * top, rows * top))
    hp = held.data_ptr()
    _check(lib().gcpsl_score(code, rows, L, zp, ldz, yp, top, None if labels is None else hp, hp + 4 * rows,
                             hp + 8 * rows, hp + 12 * rows, hp + (12 + 4 * top) * rows, ptr, size, handle))
    return Scores(None if labels is None else logp, entropy, lse, top_logp.view(rows, top),
                  top_class.view(torch.int32).view(rows, top))


def score_grad(logits, labels, lse, entropy=None, g_logp=None, g_entropy=None, out=None, stream=None):
    """gcpsl_score_grad: the loss's gradient by the logits [rows][L], given
    those by logp (g_logp [rows]) and by entropy (g_entropy [rows]), of which
    one may be None; out may be the logits."""
    if stream is None:
        r = (_ops or _native()).score_grad(logits, labels, lse, entropy, g_logp, g_entropy, out)
        if _done(r):
            return r
    torch, code, handle, device = _begin(logits, stream)
    zp, ldz = _rows(logits, "logits", logits.dtype, device)
    rows, L = logits.shape
    yp = _vector(labels, "labels", torch.int32, rows, device)
    f32 = torch.float32
    dz, dp, lddz = _out(logits, out, rows, L, logits.dtype, device, stream)
    _check(lib().gcpsl_score_grad(code, rows, L, zp, ldz, yp, _vector(lse, "lse", f32, rows, device),
                                  _vector(entropy, "entropy", f32, rows, device),
                                  _vector(g_logp, "g_logp", f32, rows, device),
                                  _vector(g_entropy, "g_entropy", f32, rows, device), dp, lddz, handle))
    return dz


def make_desc(cfg, client_of_example, cluster_of_client, max_steps=None, max_window=1, schedule="lockstep"):
    """Host part of gcpsl_desc for a workload (device pointers filled by Context)."""
    d = Desc()
    d.K, d.C, d.B, d.L = cfg["K"], cfg["C"], cfg["B"], cfg["L"]
    d.H, d.W, d.Cin = cfg["H"], cfg["W"], cfg["Cin"]
    d.dtype = DTYPES[cfg["dtype"]]
    d.n_examples = cfg["N_ex"]
    keep = {"layers": layers_struct(cfg["layers"]),
            "coe": np.ascontiguousarray(client_of_example, dtype=np.int32),
            "coc": np.ascontiguousarray(cluster_of_client, dtype=np.int32)}
    d.n_layers = len(cfg["layers"])
    d.cut = cfg["cut"]
    d.layers = C.cast(keep["layers"], C.POINTER(Layer))
    d.lr, d.momentum = cfg["lr"], cfg["momentum"]
    d.weight_decay = cfg.get("weight_decay", 0.0)
    d.nesterov = 1 if cfg.get("nesterov", False) else 0
    d.label_smoothing = cfg.get("label_smoothing", 0.0)
    d.seed = cfg["seed"]
    d.max_steps = max_steps if max_steps is not None else cfg["T"]
    d.max_window = max_window
    d.schedule = SCHEDULES[schedule]
    d.client_of_example = _i32p(keep["coe"])
    d.cluster_of_client = _i32p(keep["coc"])
    return d, keep


def param_count(desc):
    P, Pc = C.c_int64(), C.c_int64()
    _check(lib().gcpsl_param_count(C.byref(desc), C.byref(P), C.byref(Pc)))
    return P.value, Pc.value


def state_count(desc):
    S = C.c_int64()
    _check(lib().gcpsl_state_count(C.byref(desc), C.byref(S)))
    return S.value


def workspace_bytes(desc):
    n = C.c_size_t()
    _check(lib().gcpsl_workspace_bytes(C.byref(desc), C.byref(n)))
    return n.value


def _stream(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


class Context:
    """One gcpsl_ctx with the caller-owned device buffers it works in."""

    def __init__(self, cfg, images, labels, client_of_example, cluster_of_client, theta0,
                 max_steps=None, max_window=1, device="cuda", schedule="lockstep", norm_state0=None,
                 static=False):
        """static: gcpsl_create_static (the library's own workspace, no
        workspace tensor here; `tensor` is then unavailable)."""
        import torch
        self.cfg = cfg
        self.schedule = schedule
        desc, self._keep = make_desc(cfg, client_of_example, cluster_of_client, max_steps, max_window, schedule)
        self.P, self.P_client = param_count(desc)
        t0 = torch.as_tensor(np.asarray(theta0, dtype=np.float32))
        if t0.numel() != self.P:
            raise ValueError(f"theta0 has {t0.numel()} entries, the model has {self.P}")
        self.images = torch.from_numpy(np.array(images, dtype=np.float32)).to(device)
        self.labels = torch.from_numpy(np.array(labels, dtype=np.int32)).to(device)
        self.theta = t0.to(device).reshape(1, -1).repeat(cfg["C"], 1).contiguous()
        self.mom = torch.zeros_like(self.theta)
        self.S = state_count(desc)
        ns0 = np.zeros(self.S, dtype=np.float32) if norm_state0 is None else np.asarray(norm_state0, np.float32)
        if ns0.size != self.S:
            raise ValueError(f"norm_state0 has {ns0.size} entries, the model has {self.S}")
        self.norm_state = (torch.as_tensor(ns0).to(device).reshape(1, -1).repeat(cfg["C"], 1).contiguous()
                           if self.S else None)
        desc.images = self.images.data_ptr()
        desc.labels = self.labels.data_ptr()
        desc.theta = self.theta.data_ptr()
        desc.momentum_buf = self.mom.data_ptr()
        desc.norm_state = self.norm_state.data_ptr() if self.S else None
        self.static = static
        if static:
            self.workspace = None
            desc.workspace, desc.workspace_bytes = None, 0
        else:
            nbytes = workspace_bytes(desc)
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
            base = self.workspace.data_ptr()
            desc.workspace = base + (-base) % 256
            desc.workspace_bytes = nbytes
        self.desc = desc
        h = C.c_void_p()
        create = lib().gcpsl_create_static if static else lib().gcpsl_create
        _check(create(C.byref(desc), C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            lib().gcpsl_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def sample(self, step, nsteps=1, idx_out=None, stream=None):
        ptr = None if idx_out is None else C.c_void_p(idx_out.data_ptr())
        _check(lib().gcpsl_sample(self._h, step, nsteps, ptr, _stream(stream)))

    def step(self, step, loss_out=None, stream=None):
        ptr = None if loss_out is None else C.c_void_p(loss_out.data_ptr())
        _check(lib().gcpsl_step(self._h, step, ptr, _stream(stream)))

    def step_replica(self, step, replica, loss_out=None, stream=None):
        ptr = None if loss_out is None else C.c_void_p(loss_out.data_ptr())
        _check(lib().gcpsl_step_replica(self._h, step, replica, ptr, _stream(stream)))

    def epoch_rounds(self):
        """(r_n per cluster, R = slots of a system epoch) of the epoch schedule."""
        out = np.zeros(self.cfg["C"], dtype=np.int64)
        R = C.c_int64()
        _check(lib().gcpsl_epoch_rounds(self._h, _i64p(out), C.byref(R)))
        return out, R.value

    def fuse(self, stream=None):
        _check(lib().gcpsl_fuse(self._h, _stream(stream)))

    def fuse_partial(self, partial, stream=None):
        """gcpsl_fuse_partial into a device fp64 tensor of P + S entries."""
        if partial.numel() != self.P + self.S or partial.element_size() != 8 or not partial.is_contiguous():
            raise ValueError("partial must be a contiguous fp64 tensor of P + S entries")
        _check(lib().gcpsl_fuse_partial(self._h, C.c_void_p(partial.data_ptr()), _stream(stream)))

    def fuse_finalise(self, partial, W, stream=None):
        """gcpsl_fuse_finalise from a device fp64 tensor of P + S entries."""
        if partial.numel() != self.P + self.S or partial.element_size() != 8 or not partial.is_contiguous():
            raise ValueError("partial must be a contiguous fp64 tensor of P + S entries")
        _check(lib().gcpsl_fuse_finalise(self._h, C.c_void_p(partial.data_ptr()), int(W), _stream(stream)))

    def batch_deviation(self):
        """(sum of numerators, batches, denominator B |D|, per-step numerators
        [T_h][C] with -1 where no batch was drawn) of Sec. V-E's batch
        deviation (synchronises)."""
        sn, nb, den = C.c_int64(), C.c_int64(), C.c_int64()
        per = np.zeros((self.desc.max_steps, self.cfg["C"]), dtype=np.int64)
        _check(lib().gcpsl_batch_deviation(self._h, C.byref(sn), C.byref(nb), C.byref(den), _i64p(per)))
        T = self.participation()[1] // self.cfg["K"]
        return sn.value, nb.value, den.value, per[:T]

    def payload(self):
        """{category: bytes} of Sec. V-E's logical payload (synchronises)."""
        out = np.zeros(len(PAYLOAD), dtype=np.int64)
        _check(lib().gcpsl_payload(self._h, _i64p(out)))
        return {k: int(v) for k, v in zip(PAYLOAD, out)}

    def participation(self):
        a, t = C.c_int64(), C.c_int64()
        T = self.desc.max_steps
        per = np.zeros((T, self.cfg["C"]), dtype=np.int32)
        _check(lib().gcpsl_participation(self._h, C.byref(a), C.byref(t), _i32p(per)))
        steps = t.value // self.cfg["K"] if self.cfg["K"] else 0
        return a.value, t.value, per[:steps]

    def cluster_sizes(self):
        out = np.zeros(self.cfg["C"], dtype=np.int64)
        _check(lib().gcpsl_cluster_sizes(self._h, _i64p(out)))
        return out

    def timing(self, on):
        _check(lib().gcpsl_timing(self._h, 1 if on else 0))

    def timing_read(self, cap=64):
        """{kernel: dict(launches, ms, flops, bytes)} of the launches recorded
        since the last read (synchronises)."""
        arr = (KernelStat * cap)()
        n = C.c_int32()
        _check(lib().gcpsl_timing_read(self._h, arr, cap, C.byref(n)))
        return {arr[i].name.decode(): dict(launches=arr[i].launches, ms=arr[i].ms, flops=arr[i].flops,
                                           bytes=arr[i].bytes) for i in range(min(n.value, cap))}

    def tensor(self, name):
        """torch view of a named workspace tensor (gcpsl_tensor)."""
        import torch
        if self.workspace is None:
            raise ValueError("a static context's workspace is the library's own; it has no tensor view")
        ptr, n, dt = C.c_void_p(), C.c_int64(), C.c_int32()
        _check(lib().gcpsl_tensor(self._h, name.encode(), C.byref(ptr), C.byref(n), C.byref(dt)))
        tdt = {0: torch.float32, 1: torch.bfloat16, -1: torch.int32, -2: torch.uint8}[dt.value]
        esz = torch.tensor([], dtype=tdt).element_size()
        off = ptr.value - self.workspace.data_ptr()
        return self.workspace[off:off + n.value * esz].view(tdt)
