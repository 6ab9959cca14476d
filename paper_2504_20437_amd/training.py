"""Training operators of ``libgalore.so``: 8-bit activation checkpoints and the
weight gradient from them, microscaled 4-bit products, and the norms of a block.

Argument marshalling only, as in the rest of the binding: every tensor's device,
dtype, shape and strides are checked before any device access, work is enqueued on
the current stream or the one given, outputs and workspaces not given are
allocated there.

Codes come as a pair of tensors. For a matrix of ``cols`` columns, in blocks of 32
(``nb = ceil(cols / 32)``): 8-bit checkpoints hold int8 codes (..., rows, 32 nb),
4-bit matrices uint8 codes (..., rows, 16 nb), two to a byte; either has uint8
scales (..., rows, nb rounded up to a multiple of 4).

Autograd does not see these calls: what they return has no graph, also where an
input requires gradients, so that a loss formed from it leaves those inputs without
a gradient. The backward pass is the caller's: each forward call has its gradient
here (galore_norm_block_backward, galore_checkpoint_weight_grad, galore_mx4_matmul on
the operand by columns), to be called by hand or from the backward of a
torch.autograd.Function.
"""
from __future__ import annotations

import ctypes
import functools
import inspect

import torch

from . import _check, _torch_stream, lib

_Tensor = torch.Tensor
GATE_NONE, GATE_VECTOR, GATE_TOKENS = 0, 1, 2
_CODE = {torch.float32: 0, torch.bfloat16: 1}


class MxMatrix(ctypes.Structure):
    """galore_mx_t"""
    _fields_ = [("codes", ctypes.c_void_p), ("ldq", ctypes.c_int64), ("stride_q", ctypes.c_int64),
                ("scales", ctypes.c_void_p), ("lds", ctypes.c_int64), ("stride_s", ctypes.c_int64)]


def declare(lib):
    vp, sz, i32, i64, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    mx = ctypes.POINTER(MxMatrix)
    for name, args, res in (
        ("galore_mx_scale_bytes", [i64], i64),
        ("galore_checkpoint_pack", [vp, i32, i64, i64, i64, i64, mx, i32, vp], i32),
        ("galore_checkpoint_unpack", [mx, i64, i64, vp, i32, i64, i64, i32, vp], i32),
        ("galore_checkpoint_weight_grad_workspace_size", [i64, i64, i64, i32], sz),
        ("galore_checkpoint_weight_grad", [vp, i32, i64, i64, mx, i64, i64, i64, vp, i32, i64, i64, i32, i32, vp, sz, vp],
         i32),
        ("galore_mx4_quantize", [vp, i32, i64, i64, i64, i64, mx, mx, i32, vp], i32),
        ("galore_mx4_dequantize", [mx, i64, i64, vp, i32, i64, i64, i32, vp], i32),
        ("galore_mx4_matmul", [mx, mx, i64, i64, i64, vp, i32, i64, i64, i32, vp], i32),
        ("galore_norm_block", [vp, i64, vp, i64, i32, vp, vp, vp, i64, i32, f32, f32, i64, i64, vp, i64, vp, i64, vp, mx,
                               mx, mx, vp], i32),
        ("galore_norm_block_backward_workspace_size", [i64, i64], sz),
        ("galore_norm_block_backward", [vp, i64, vp, i64, i32, vp, i64, vp, i64, mx, mx, vp, vp, vp, vp, i64, i32, f32,
                                        i64, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, sz, vp], i32),
    ):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, res


# ---- argument checks ------------------------------------------------------------------
#
# A call on few tokens takes less time on the GPU than its marshalling takes here, so
# each check is made once, on the plain attributes of a tensor.


def _fail(name, want, t):
    got = "%s %s %s on %s" % (t.dtype, tuple(t.shape), t.stride(), t.device) if isinstance(t, _Tensor) else type(t).__name__
    raise ValueError("%s must be %s, got %s" % (name, want, got))


def _code(dtype):
    code = _CODE.get(dtype)
    if code is None:
        raise ValueError("dtype must be float32 or bfloat16")
    return code


def _float(t, name, dims=(2, 3)):
    """the dtype code of a row-major float32 or bfloat16 device tensor"""
    code = _CODE.get(t.dtype) if isinstance(t, _Tensor) else None
    if code is None or t.dim() not in dims or not t.is_cuda or (t.stride(-1) != 1 and t.shape[-1] > 1):
        _fail(name, "a row-major float32 or bfloat16 tensor of %s dimensions on a GPU" % " or ".join(map(str, dims)), t)
    return code


def _pitch(t):
    """row pitch and matrix stride of a row-major tensor (a size of one leaves its stride free: the packed one then)"""
    shape = t.shape
    rows = shape[-2]
    if t.is_contiguous():
        return shape[-1], rows * shape[-1]
    s = t.stride()
    ld = s[-2] if rows > 1 else shape[-1]
    return ld, s[0] if len(s) == 3 and shape[0] > 1 else rows * ld


def _given(t, name, shape, dtype, device):
    """(pointer, row pitch, matrix stride) of a row-major tensor of this shape"""
    if not isinstance(t, _Tensor) or t.dtype != dtype or t.shape != shape or t.device != device:
        _fail(name, "%s %s on %s" % (dtype, tuple(shape), device), t)
    cols, rows = shape[-1], shape[-2]
    if t.is_contiguous():
        return t.data_ptr(), cols, rows * cols
    s = t.stride()
    if s[-1] != 1 and cols > 1:
        _fail(name, "row-major", t)
    ld = s[-2] if rows > 1 else cols
    return t.data_ptr(), ld, s[0] if len(s) == 3 and shape[0] > 1 else rows * ld


def _vector(t, name, length, device):
    """pointer of a float32 vector"""
    if (not isinstance(t, _Tensor) or t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != length or
            t.device != device or (t.stride(0) != 1 and length > 1)):
        _fail(name, "a float32 vector of %d on %s" % (length, device), t)
    return t.data_ptr()


def _stats(t, tokens, device):
    """pointer of the (tokens, 2) statistics"""
    p, ld, _ = _given(t, "rstd", (tokens, 2), torch.float32, device)
    if ld != 2:
        _fail("rstd", "contiguous", t)
    return p


def _mx(codes, scales, rows, cols, bits, lead, device, name):
    """the struct of a pair of codes and scales, checked"""
    nb = (cols + 31) // 32
    qp, ldq, sq = _given(codes, name + " codes", lead + (rows, nb * 4 * bits), torch.int8 if bits == 8 else torch.uint8, device)
    sp, lds, ss = _given(scales, name + " scales", lead + (rows, (nb + 3) // 4 * 4), torch.uint8, device)
    if (qp | ldq | sq) % 16:
        raise ValueError("%s codes must start on 16 bytes, every row of them" % name)
    if (sp | lds | ss) % 4:
        raise ValueError("%s scales must start on 4 bytes, every row of them" % name)
    return MxMatrix(qp, ldq, sq, sp, lds, ss)


def _pair(given, rows, cols, bits, lead, device, name):
    """((codes, scales), struct) of the given pair, or of a new one"""
    if given is not None:
        codes, scales = given
        return (codes, scales), _mx(codes, scales, rows, cols, bits, lead, device, name)
    nb = (cols + 31) // 32
    width, ns = nb * 4 * bits, (nb + 3) // 4 * 4
    codes = torch.empty(lead + (rows, width), dtype=torch.int8 if bits == 8 else torch.uint8, device=device)
    scales = torch.empty(lead + (rows, ns), dtype=torch.uint8, device=device)
    return (codes, scales), MxMatrix(codes.data_ptr(), width, rows * width, scales.data_ptr(), ns, rows * ns)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _on_stream(call):
    """Runs call(stream handle, *args, **kw) with the given stream (the keyword ``stream``; the current one by default)
    and the device of the call's first tensor as the current ones, so that outputs are allocated there too."""
    signature = inspect.signature(call)
    own = list(signature.parameters.values())[1:]
    name = own[0].name

    @functools.wraps(call)
    def run(*args, stream=None, **kw):
        first = args[0] if args else kw.get(name)
        if not isinstance(first, _Tensor) or not first.is_cuda:
            _fail(name, "a tensor on a GPU", first)
        index = first.device.index
        if stream is None and index == torch.cuda.current_device():
            if _raw_stream is not None:
                return call(_raw_stream(index), *args, **kw)
            return call(torch.cuda.current_stream().cuda_stream, *args, **kw)
        ts = _torch_stream(stream, first.device)
        with torch.cuda.device(index), torch.cuda.stream(ts):
            return call(ts.cuda_stream, *args, **kw)
    run.__signature__ = signature.replace(
        parameters=own + [inspect.Parameter("stream", inspect.Parameter.KEYWORD_ONLY, default=None)])
    return run


def _workspace(workspace, need, device):
    """(tensor kept alive, pointer, bytes)"""
    if workspace is None:
        if not need:
            return None, None, 0
        workspace = torch.empty((need,), dtype=torch.uint8, device=device)
    elif (not isinstance(workspace, _Tensor) or workspace.dim() != 1 or not workspace.is_contiguous() or
          workspace.device != device):
        _fail("workspace", "a contiguous 1-D tensor on %s" % device, workspace)
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _batch(lead):
    return lead[0] if lead else 1


# ---- 8-bit checkpoints ----------------------------------------------------------------


def galore_checkpoint_empty(tokens: int, cols: int, batch=None, device="cuda"):
    """(codes, scales) for a checkpoint of tokens x cols values (``batch`` of them if given)."""
    return _pair(None, tokens, cols, 8, () if batch is None else (batch,), torch.device(device), "")[0]


@_on_stream
def galore_checkpoint_pack(_h, X: torch.Tensor, out=None):
    """8-bit checkpoint (codes, scales) of X ((tokens, cols) or (batch, tokens, cols))."""
    dt = _float(X, "X")
    shape = X.shape
    lead, tokens, cols = tuple(shape[:-2]), shape[-2], shape[-1]
    pair, q = _pair(out, tokens, cols, 8, lead, X.device, "out")
    ld, st = _pitch(X)
    _check(lib.galore_checkpoint_pack(X.data_ptr(), dt, tokens, cols, ld, st, q, _batch(lead), _h),
           "galore_checkpoint_pack")
    return pair


def _decode(fn, name, bits, h, codes, scales, cols, dtype, out):
    if codes.dim() not in (2, 3):
        _fail("codes", "a 2-D or 3-D tensor", codes)
    shape, dev = codes.shape, codes.device
    lead, rows = tuple(shape[:-2]), shape[-2]
    q = _mx(codes, scales, rows, cols, bits, lead, dev, "given")
    if out is None:
        code = _code(dtype)
        out = torch.empty(lead + (rows, cols), dtype=dtype, device=dev)
        p, ld, st = out.data_ptr(), cols, rows * cols
    else:
        code = _float(out, "out")
        p, ld, st = _given(out, "out", lead + (rows, cols), out.dtype, dev)
    _check(fn(q, rows, cols, p, code, ld, st, _batch(lead), h), name)
    return out


@_on_stream
def galore_checkpoint_unpack(_h, codes: torch.Tensor, scales: torch.Tensor, cols: int, dtype=torch.bfloat16, out=None):
    """The values of a checkpoint, exact in either dtype."""
    return _decode(lib.galore_checkpoint_unpack, "galore_checkpoint_unpack", 8, _h, codes, scales, cols, dtype, out)


def galore_checkpoint_weight_grad_workspace_size(tokens: int, m: int, n: int, batch: int = 1) -> int:
    return int(lib.galore_checkpoint_weight_grad_workspace_size(tokens, m, n, batch))


@_on_stream
def galore_checkpoint_weight_grad(_h, dY: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, n: int, G=None,
                                  accumulate: bool = False, dtype=None, workspace=None):
    """Weight gradient G (m x n) = dY^T X of a linear layer Y = X W^T, from the incoming gradient dY ((tokens, m) or
    (batch, tokens, m)) and the 8-bit checkpoint of its input X (tokens x n); added to G with ``accumulate``. G is
    allocated in ``dtype`` (dY's by default) where it is not given."""
    dt = _float(dY, "dY")
    shape, dev = dY.shape, dY.device
    lead, tokens, m = tuple(shape[:-2]), shape[-2], shape[-1]
    batch = _batch(lead)
    q = _mx(codes, scales, tokens, n, 8, lead, dev, "checkpoint")
    if G is None:
        if accumulate:
            raise ValueError("accumulate needs G")
        dtype = dtype or dY.dtype
        gt = _code(dtype)
        G = torch.empty(lead + (m, n), dtype=dtype, device=dev)
        gp, ldg, sg = G.data_ptr(), n, m * n
    else:
        gt = _float(G, "G")
        gp, ldg, sg = _given(G, "G", lead + (m, n), G.dtype, dev)
    need = lib.galore_checkpoint_weight_grad_workspace_size(tokens, m, n, batch)
    workspace, wp, wb = _workspace(workspace, need, dev)
    ld, st = _pitch(dY)
    _check(lib.galore_checkpoint_weight_grad(dY.data_ptr(), dt, ld, st, q, tokens, m, n, gp, gt, ldg, sg,
                                             1 if accumulate else 0, batch, wp, wb, _h),
           "galore_checkpoint_weight_grad")
    return G


# ---- microscaled 4-bit floating point ---------------------------------------------------


@_on_stream
def galore_mx4_quantize(_h, X: torch.Tensor, rows: bool = True, columns: bool = False, out=None, out_columns=None):
    """X ((m, n) or (batch, m, n)) in 4-bit codes: with ``rows`` (codes, scales) in blocks along its rows, with
    ``columns`` those of its transpose, in blocks along its columns; both, in this order, from one read of X."""
    dt = _float(X, "X")
    if not rows and not columns:
        raise ValueError("rows, columns or both")
    shape, dev = X.shape, X.device
    lead, m, n = tuple(shape[:-2]), shape[-2], shape[-1]
    a = b = ()
    q = qt = None
    if rows:
        a, q = _pair(out, m, n, 4, lead, dev, "out")
    if columns:
        b, qt = _pair(out_columns, n, m, 4, lead, dev, "out_columns")
    ld, st = _pitch(X)
    _check(lib.galore_mx4_quantize(X.data_ptr(), dt, m, n, ld, st, q, qt, _batch(lead), _h), "galore_mx4_quantize")
    return a + b


@_on_stream
def galore_mx4_dequantize(_h, codes: torch.Tensor, scales: torch.Tensor, cols: int, dtype=torch.bfloat16, out=None):
    """The values of a 4-bit matrix, exact in either dtype."""
    return _decode(lib.galore_mx4_dequantize, "galore_mx4_dequantize", 4, _h, codes, scales, cols, dtype, out)


@_on_stream
def galore_mx4_matmul(_h, A: torch.Tensor, A_scales: torch.Tensor, B: torch.Tensor, B_scales: torch.Tensor, k: int, C=None,
                      dtype=torch.bfloat16):
    """C (m x n) = A B^T of 4-bit matrices A (m x k) and B (n x k), blocks along k. C carries no autograd graph."""
    if A.dim() not in (2, 3):
        _fail("A", "a 2-D or 3-D tensor", A)
    if not isinstance(B, _Tensor) or B.dim() != A.dim():
        _fail("B", "a tensor of as many dimensions as A", B)
    shape, dev = A.shape, A.device
    lead, m, n = tuple(shape[:-2]), shape[-2], B.shape[-2]
    qa = _mx(A, A_scales, m, k, 4, lead, dev, "A")
    qb = _mx(B, B_scales, n, k, 4, lead, dev, "B")
    if C is None:
        ct = _code(dtype)
        C = torch.empty(lead + (m, n), dtype=dtype, device=dev)
        cp, ld, st = C.data_ptr(), n, m * n
    else:
        ct = _float(C, "C")
        cp, ld, st = _given(C, "C", lead + (m, n), C.dtype, dev)
    _check(lib.galore_mx4_matmul(qa, qb, m, n, k, cp, ct, ld, st, _batch(lead), _h), "galore_mx4_matmul")
    return C


# ---- the norms of a block ---------------------------------------------------------------


def _gate(gate, name, shape, dtype, device):
    """(pointer, pitch, mode)"""
    if gate is None:
        return None, 0, GATE_NONE
    if isinstance(gate, _Tensor) and gate.dim() == 1:
        return _vector(gate, name, shape[1], device), 0, GATE_VECTOR
    p, ld, _ = _given(gate, name, shape, dtype, device)
    return p, ld, GATE_TOKENS


def _out(t, name, like):
    """(tensor, pointer, pitch) of the given tensor, or of a new one of the same shape as `like`"""
    shape = like.shape
    if t is None:
        t = torch.empty_like(like) if like.is_contiguous() else torch.empty(shape, dtype=like.dtype, device=like.device)
        return t, t.data_ptr(), shape[1]
    p, ld, _ = _given(t, name, shape, like.dtype, like.device)
    return t, p, ld


def _out_vector(t, name, like, length, device):
    """(tensor, pointer) of the given float32 vector, or of a new one like the checked `like`"""
    if t is None:
        t = torch.empty_like(like)
        return t, t.data_ptr()
    return t, _vector(t, name, length, device)


@_on_stream
def galore_norm_block(_h, X: torch.Tensor, Y: torch.Tensor, w_post: torch.Tensor, w_pre: torch.Tensor, gate=None,
                      alpha: float = 1.0, eps: float = 1e-5, H=None, Z=None, rstd=None, checkpoints=False):
    """The norms after and before a block with its gate and residual scale:

        H = X + alpha gate norm(Y) w_post,   Z = norm(H) w_pre

    X, Y: (tokens, d), the residual stream and the block's output; gate: None, a float32 vector of d, or a tensor like
    X; H may be X. Returns (H, Z, rstd, y8, h8, z8): rstd (tokens, 2) and the 8-bit checkpoints of Y, H and Z for the
    backward pass, None where not asked for. ``checkpoints``: True for all three, or a triple of (codes, scales), True
    or None. The results carry no autograd graph: their gradients are galore_norm_block_backward's."""
    dt = _float(X, "X", (2,))
    shape, dtype, dev = X.shape, X.dtype, X.device
    tokens, d = shape
    yp, ldy, _ = _given(Y, "Y", shape, dtype, dev)
    wo, wp = _vector(w_post, "w_post", d, dev), _vector(w_pre, "w_pre", d, dev)
    gp, ldgate, mode = _gate(gate, "gate", shape, dtype, dev)
    H, hp, ldh = _out(H, "H", X)
    Z, zp, ldz = _out(Z, "Z", X)
    if rstd is None:
        rstd = torch.empty((tokens, 2), dtype=torch.float32, device=dev)
        rp = rstd.data_ptr()
    else:
        rp = _stats(rstd, tokens, dev)
    y8 = h8 = z8 = qy = qh = qz = None
    if checkpoints:
        want = (True, True, True) if checkpoints is True else checkpoints
        (y8, qy), (h8, qh), (z8, qz) = [
            (None, None) if c is None else _pair(None if c is True else c, tokens, d, 8, (), dev, "checkpoint") for c in want]
    _check(lib.galore_norm_block(X.data_ptr(), _pitch(X)[0], yp, ldy, dt, wo, wp, gp, ldgate, mode, alpha, eps, tokens, d,
                                 hp, ldh, zp, ldz, rp, qy, qh, qz, _h), "galore_norm_block")
    return H, Z, rstd, y8, h8, z8


def galore_norm_block_backward_workspace_size(tokens: int, d: int) -> int:
    return int(lib.galore_norm_block_backward_workspace_size(tokens, d))


@_on_stream
def galore_norm_block_backward(_h, dZ: torch.Tensor, dH, H, Y, rstd: torch.Tensor, w_post: torch.Tensor,
                               w_pre: torch.Tensor, gate=None, alpha: float = 1.0, dX=None, dY=None, dgate=None,
                               dw_post=None, dw_pre=None, workspace=None):
    """Gradients of galore_norm_block: (dX, dY, dgate, dw_post, dw_pre) from dZ and dH (None for zero). H and Y: both
    the tensors of the forward pass or both their 8-bit checkpoints (codes, scales). dX may be dH; dgate is None
    without a gate, else like the gate."""
    dt = _float(dZ, "dZ", (2,))
    shape, dtype, dev = dZ.shape, dZ.dtype, dZ.device
    tokens, d = shape
    dhp, lddh = None, 0
    if dH is not None:
        dhp, lddh, _ = _given(dH, "dH", shape, dtype, dev)
    h8 = y8 = hp = yp = None
    ldh = ldy = 0
    if isinstance(H, _Tensor) and isinstance(Y, _Tensor):
        hp, ldh, _ = _given(H, "H", shape, dtype, dev)
        yp, ldy, _ = _given(Y, "Y", shape, dtype, dev)
    elif isinstance(H, (tuple, list)) and isinstance(Y, (tuple, list)):
        h8 = _mx(*H, tokens, d, 8, (), dev, "H")
        y8 = _mx(*Y, tokens, d, 8, (), dev, "Y")
    else:
        raise ValueError("H and Y must both be tensors or both be checkpoints")
    rp = _stats(rstd, tokens, dev)
    wo, wp = _vector(w_post, "w_post", d, dev), _vector(w_pre, "w_pre", d, dev)
    gp, ldgate, mode = _gate(gate, "gate", shape, dtype, dev)
    dX, dxp, lddx = _out(dX, "dX", dZ)
    dY, dyp, lddy = _out(dY, "dY", dZ)
    dgp, lddg = None, 0
    if gate is not None:
        if dgate is None and mode == GATE_VECTOR:
            dgate, dgp = _out_vector(None, "dgate", gate, d, dev)
        elif dgate is None:
            dgate, dgp, lddg = _out(None, "dgate", gate)
        else:
            dgp, lddg, dmode = _gate(dgate, "dgate", shape, dtype, dev)
            if dmode != mode:
                _fail("dgate", "like the gate", dgate)
    elif dgate is not None:
        raise ValueError("dgate without a gate")
    dw_post, dwop = _out_vector(dw_post, "dw_post", w_post, d, dev)
    dw_pre, dwpp = _out_vector(dw_pre, "dw_pre", w_pre, d, dev)
    workspace, wsp, wsb = _workspace(workspace, lib.galore_norm_block_backward_workspace_size(tokens, d), dev)
    _check(lib.galore_norm_block_backward(
        dZ.data_ptr(), _pitch(dZ)[0], dhp, lddh, dt, hp, ldh, yp, ldy, h8, y8, rp, wo, wp, gp, ldgate, mode, alpha, tokens,
        d, dxp, lddx, dyp, lddy, dgp, lddg, dwop, dwpp, wsp, wsb, _h), "galore_norm_block_backward")
    return dX, dY, dgate, dw_post, dw_pre
