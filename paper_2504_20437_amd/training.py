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
"""
from __future__ import annotations

import ctypes

import torch

from . import _check, _handle, _torch_stream, lib

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


def _fail(name, want, t):
    got = "%s %s on %s" % (t.dtype, tuple(t.shape), t.device) if isinstance(t, torch.Tensor) else type(t).__name__
    raise ValueError("%s must be %s, got %s" % (name, want, got))


def _float(t, name, device=None):
    """the dtype code of a float32 or bfloat16 device tensor, 2-D or 3-D, row-major"""
    if not isinstance(t, torch.Tensor) or t.dtype not in _CODE or t.dim() not in (2, 3):
        _fail(name, "a 2-D or 3-D float32 or bfloat16 tensor", t)
    if not t.is_cuda or (device is not None and t.device != device):
        _fail(name, "on %s" % (device if device is not None else "a GPU"), t)
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError("%s must be row-major" % name)
    return _CODE[t.dtype]


def _expect(t, name, shape, dtype, device):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or tuple(t.shape) != tuple(shape) or t.device != device:
        _fail(name, "%s %s on %s" % (dtype, tuple(shape), device), t)
    if t.dim() and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError("%s must be row-major" % name)


def _pitch(t):
    """row pitch and matrix stride of a row-major tensor (a size of one leaves its stride free: the packed one then)"""
    rows, cols = t.shape[-2], t.shape[-1]
    ld = t.stride(-2) if rows > 1 else cols
    return ld, t.stride(0) if t.dim() == 3 and t.shape[0] > 1 else rows * ld


def _batch(t):
    return t.shape[0] if t.dim() == 3 else 1


def _blocks(cols):
    nb = (cols + 31) // 32
    return nb, (nb + 3) // 4 * 4


def _mx(codes, scales, rows, cols, bits, lead, device, name):
    """the struct of a pair of codes and scales, checked"""
    nb, ns = _blocks(cols)
    _expect(codes, name + " codes", lead + (rows, nb * 4 * bits), torch.int8 if bits == 8 else torch.uint8, device)
    _expect(scales, name + " scales", lead + (rows, ns), torch.uint8, device)
    ldq, sq = _pitch(codes)
    lds, ss = _pitch(scales)
    if codes.data_ptr() % 16 or ldq % 16 or sq % 16:
        raise ValueError("%s codes must start on 16 bytes, every row of them" % name)
    if scales.data_ptr() % 4 or lds % 4 or ss % 4:
        raise ValueError("%s scales must start on 4 bytes, every row of them" % name)
    return MxMatrix(codes.data_ptr(), ldq, sq, scales.data_ptr(), lds, ss)


def _empty_mx(rows, cols, bits, lead, device):
    nb, ns = _blocks(cols)
    return (torch.empty(lead + (rows, nb * 4 * bits), dtype=torch.int8 if bits == 8 else torch.uint8, device=device),
            torch.empty(lead + (rows, ns), dtype=torch.uint8, device=device))


def _pair(given, rows, cols, bits, lead, device):
    if given is None:
        return _empty_mx(rows, cols, bits, lead, device)
    codes, scales = given
    return codes, scales


class _On:
    """the given stream as the current one, where it is not that already"""

    def __init__(self, stream, device):
        self.stream = _torch_stream(stream, device)
        self.switch = torch.cuda.stream(self.stream) if stream is not None else None
        # a call on another device than the current one launches there
        self.device = torch.cuda.device(device) if device.index != torch.cuda.current_device() else None

    def __enter__(self):
        if self.device is not None:
            self.device.__enter__()
        if self.switch is not None:
            self.switch.__enter__()
        return _handle(self.stream)

    def __exit__(self, *exc):
        if self.switch is not None:
            self.switch.__exit__(*exc)
        if self.device is not None:
            self.device.__exit__(*exc)


def _workspace(workspace, need, device):
    """(tensor kept alive, pointer, bytes)"""
    if workspace is None:
        if not need:
            return None, None, 0
        workspace = torch.empty((need,), dtype=torch.uint8, device=device)
    if workspace.dim() != 1 or not workspace.is_contiguous() or workspace.device != device:
        _fail("workspace", "a contiguous 1-D tensor on %s" % device, workspace)
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


# ---- 8-bit checkpoints ----------------------------------------------------------------


def galore_checkpoint_empty(tokens: int, cols: int, batch=None, device="cuda"):
    """(codes, scales) for a checkpoint of tokens x cols values (``batch`` of them if given)."""
    return _empty_mx(tokens, cols, 8, () if batch is None else (batch,), torch.device(device))


def galore_checkpoint_pack(X: torch.Tensor, out=None, stream=None):
    """8-bit checkpoint (codes, scales) of X ((tokens, cols) or (batch, tokens, cols))."""
    dt = _float(X, "X")
    tokens, cols = X.shape[-2:]
    lead, dev = tuple(X.shape[:-2]), X.device
    with _On(stream, dev) as h:
        codes, scales = _pair(out, tokens, cols, 8, lead, dev)
        q = _mx(codes, scales, tokens, cols, 8, lead, dev, "out")
        ld, st = _pitch(X)
        _check(lib.galore_checkpoint_pack(X.data_ptr(), dt, tokens, cols, ld, st, q, _batch(X), h),
               "galore_checkpoint_pack")
    return codes, scales


def galore_checkpoint_unpack(codes: torch.Tensor, scales: torch.Tensor, cols: int, dtype=torch.bfloat16, out=None,
                             stream=None):
    """The values of a checkpoint, exact in either dtype."""
    return _decode(lib.galore_checkpoint_unpack, "galore_checkpoint_unpack", 8, codes, scales, cols, dtype, out, stream)


def _decode(fn, name, bits, codes, scales, cols, dtype, out, stream):
    if not isinstance(codes, torch.Tensor) or codes.dim() not in (2, 3) or not codes.is_cuda:
        _fail("codes", "a 2-D or 3-D tensor on a GPU", codes)
    lead, rows, dev = tuple(codes.shape[:-2]), codes.shape[-2], codes.device
    if out is not None:
        dtype = out.dtype
    if dtype not in _CODE:
        raise ValueError("dtype must be float32 or bfloat16")
    with _On(stream, dev) as h:
        q = _mx(codes, scales, rows, cols, bits, lead, dev, "given")
        if out is None:
            out = torch.empty(lead + (rows, cols), dtype=dtype, device=dev)
        else:
            _expect(out, "out", lead + (rows, cols), dtype, dev)
        ld, st = _pitch(out)
        _check(fn(q, rows, cols, out.data_ptr(), _CODE[dtype], ld, st, _batch(codes), h), name)
    return out


def galore_checkpoint_weight_grad_workspace_size(tokens: int, m: int, n: int, batch: int = 1) -> int:
    return int(lib.galore_checkpoint_weight_grad_workspace_size(tokens, m, n, batch))


def galore_checkpoint_weight_grad(dY: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, n: int, G=None,
                                  accumulate: bool = False, dtype=None, workspace=None, stream=None):
    """Weight gradient G (m x n) = dY^T X of a linear layer Y = X W^T, from the incoming gradient dY ((tokens, m) or
    (batch, tokens, m)) and the 8-bit checkpoint of its input X (tokens x n); added to G with ``accumulate``. G is
    allocated in ``dtype`` (dY's by default) where it is not given."""
    dt = _float(dY, "dY")
    tokens, m = dY.shape[-2:]
    lead, dev, batch = tuple(dY.shape[:-2]), dY.device, _batch(dY)
    if accumulate and G is None:
        raise ValueError("accumulate needs G")
    with _On(stream, dev) as h:
        q = _mx(codes, scales, tokens, n, 8, lead, dev, "checkpoint")
        if G is None:
            G = torch.empty(lead + (m, n), dtype=dtype or dY.dtype, device=dev)
        elif tuple(G.shape) != lead + (m, n):
            _fail("G", "of shape %s" % (lead + (m, n),), G)
        gt = _float(G, "G", dev)
        need = lib.galore_checkpoint_weight_grad_workspace_size(tokens, m, n, batch)
        workspace, wp, wb = _workspace(workspace, need, dev)
        ld, st = _pitch(dY)
        ldg, sg = _pitch(G)
        _check(lib.galore_checkpoint_weight_grad(dY.data_ptr(), dt, ld, st, q, tokens, m, n, G.data_ptr(), gt, ldg, sg,
                                                 1 if accumulate else 0, batch, wp, wb, h),
               "galore_checkpoint_weight_grad")
    return G


# ---- microscaled 4-bit floating point ---------------------------------------------------


def galore_mx4_quantize(X: torch.Tensor, rows: bool = True, columns: bool = False, out=None, out_columns=None, stream=None):
    """X ((m, n) or (batch, m, n)) in 4-bit codes: with ``rows`` (codes, scales) in blocks along its rows, with
    ``columns`` those of its transpose, in blocks along its columns; both, in this order, from one read of X."""
    dt = _float(X, "X")
    m, n = X.shape[-2:]
    lead, dev = tuple(X.shape[:-2]), X.device
    if not rows and not columns:
        raise ValueError("rows, columns or both")
    with _On(stream, dev) as h:
        q = qt = None
        got = ()
        if rows:
            got = _pair(out, m, n, 4, lead, dev)
            q = _mx(*got, m, n, 4, lead, dev, "out")
        if columns:
            t = _pair(out_columns, n, m, 4, lead, dev)
            qt = _mx(*t, n, m, 4, lead, dev, "out_columns")
            got = got + t
        ld, st = _pitch(X)
        _check(lib.galore_mx4_quantize(X.data_ptr(), dt, m, n, ld, st, q, qt, _batch(X), h), "galore_mx4_quantize")
    return got


def galore_mx4_dequantize(codes: torch.Tensor, scales: torch.Tensor, cols: int, dtype=torch.bfloat16, out=None,
                          stream=None):
    """The values of a 4-bit matrix, exact in either dtype."""
    return _decode(lib.galore_mx4_dequantize, "galore_mx4_dequantize", 4, codes, scales, cols, dtype, out, stream)


def galore_mx4_matmul(A: torch.Tensor, A_scales: torch.Tensor, B: torch.Tensor, B_scales: torch.Tensor, k: int, C=None,
                      dtype=torch.bfloat16, stream=None):
    """C (m x n) = A B^T of 4-bit matrices A (m x k) and B (n x k), blocks along k."""
    if not isinstance(A, torch.Tensor) or A.dim() not in (2, 3) or not A.is_cuda:
        _fail("A", "a 2-D or 3-D tensor on a GPU", A)
    if not isinstance(B, torch.Tensor) or B.dim() != A.dim():
        _fail("B", "of as many dimensions as A", B)
    lead, m, n, dev = tuple(A.shape[:-2]), A.shape[-2], B.shape[-2], A.device
    with _On(stream, dev) as h:
        qa = _mx(A, A_scales, m, k, 4, lead, dev, "A")
        qb = _mx(B, B_scales, n, k, 4, lead, dev, "B")
        if C is None:
            C = torch.empty(lead + (m, n), dtype=dtype, device=dev)
        elif tuple(C.shape) != lead + (m, n):
            _fail("C", "of shape %s" % (lead + (m, n),), C)
        ct = _float(C, "C", dev)
        ld, st = _pitch(C)
        _check(lib.galore_mx4_matmul(qa, qb, m, n, k, C.data_ptr(), ct, ld, st, _batch(A), h), "galore_mx4_matmul")
    return C


# ---- the norms of a block ---------------------------------------------------------------


def _gate(gate, X, name="gate"):
    """(pointer, pitch, mode)"""
    if gate is None:
        return None, 0, GATE_NONE
    if isinstance(gate, torch.Tensor) and gate.dim() == 1:
        _vector(gate, name, X)
        return gate.data_ptr(), 0, GATE_VECTOR
    _expect(gate, name, X.shape, X.dtype, X.device)
    return gate.data_ptr(), _pitch(gate)[0], GATE_TOKENS


def _vector(t, name, X):
    _expect(t, name, (X.shape[1],), torch.float32, X.device)
    return t.data_ptr()


def _rows(t, name, X):
    """(pointer, pitch) of a tensor like X, allocated if None"""
    if t is None:
        t = torch.empty(X.shape, dtype=X.dtype, device=X.device)
    else:
        _expect(t, name, X.shape, X.dtype, X.device)
    return t, t.data_ptr(), _pitch(t)[0]


def galore_norm_block(X: torch.Tensor, Y: torch.Tensor, w_post: torch.Tensor, w_pre: torch.Tensor, gate=None,
                      alpha: float = 1.0, eps: float = 1e-5, H=None, Z=None, rstd=None, checkpoints=False, stream=None):
    """The norms after and before a block with its gate and residual scale:

        H = X + alpha gate norm(Y) w_post,   Z = norm(H) w_pre

    X, Y: (tokens, d), the residual stream and the block's output; gate: None, a float32 vector of d, or a tensor like
    X; H may be X. Returns (H, Z, rstd, y8, h8, z8): rstd (tokens, 2) and the 8-bit checkpoints of Y, H and Z for the
    backward pass, None where not asked for. ``checkpoints``: True for all three, or a triple of (codes, scales), True
    or None."""
    dt = _float(X, "X")
    if X.dim() != 2:
        _fail("X", "2-D", X)
    _expect(Y, "Y", X.shape, X.dtype, X.device)
    tokens, d = X.shape
    dev = X.device
    wo, wp = _vector(w_post, "w_post", X), _vector(w_pre, "w_pre", X)
    gp, ldgate, mode = _gate(gate, X)
    if checkpoints is True or checkpoints is False or checkpoints is None:
        checkpoints = (checkpoints or None,) * 3
    with _On(stream, dev) as h:
        H, hp, ldh = _rows(H, "H", X)
        Z, zp, ldz = _rows(Z, "Z", X)
        if rstd is None:
            rstd = torch.empty((tokens, 2), dtype=torch.float32, device=dev)
        else:
            _expect(rstd, "rstd", (tokens, 2), torch.float32, dev)
            if not rstd.is_contiguous():
                raise ValueError("rstd must be contiguous")
        pairs = [None if c is None else _pair(None if c is True else c, tokens, d, 8, (), dev) for c in checkpoints]
        mx = [None if c is None else _mx(*c, tokens, d, 8, (), dev, "checkpoint") for c in pairs]
        _check(lib.galore_norm_block(X.data_ptr(), _pitch(X)[0], Y.data_ptr(), _pitch(Y)[0], dt, wo, wp, gp, ldgate, mode,
                                     alpha, eps, tokens, d, hp, ldh, zp, ldz, rstd.data_ptr(), mx[0], mx[1], mx[2], h),
               "galore_norm_block")
    return (H, Z, rstd, *pairs)


def galore_norm_block_backward_workspace_size(tokens: int, d: int) -> int:
    return int(lib.galore_norm_block_backward_workspace_size(tokens, d))


def galore_norm_block_backward(dZ: torch.Tensor, dH, H, Y, rstd: torch.Tensor, w_post: torch.Tensor, w_pre: torch.Tensor,
                               gate=None, alpha: float = 1.0, dX=None, dY=None, dgate=None, dw_post=None, dw_pre=None,
                               workspace=None, stream=None):
    """Gradients of galore_norm_block: (dX, dY, dgate, dw_post, dw_pre) from dZ and dH (None for zero). H and Y: both
    the tensors of the forward pass or both their 8-bit checkpoints (codes, scales). dX may be dH; dgate is None
    without a gate, else like the gate."""
    dt = _float(dZ, "dZ")
    if dZ.dim() != 2:
        _fail("dZ", "2-D", dZ)
    tokens, d = dZ.shape
    dev = dZ.device
    if dH is not None:
        _expect(dH, "dH", dZ.shape, dZ.dtype, dev)
    packed = not isinstance(H, torch.Tensor)
    if packed == isinstance(Y, torch.Tensor):
        raise ValueError("H and Y must both be tensors or both be checkpoints")
    _expect(rstd, "rstd", (tokens, 2), torch.float32, dev)
    if not rstd.is_contiguous():
        raise ValueError("rstd must be contiguous")
    wo, wp = _vector(w_post, "w_post", dZ), _vector(w_pre, "w_pre", dZ)
    gp, ldgate, mode = _gate(gate, dZ)
    with _On(stream, dev) as h:
        if packed:
            (hc, hs), (yc, ys) = H, Y
            h8 = _mx(hc, hs, tokens, d, 8, (), dev, "H")
            y8 = _mx(yc, ys, tokens, d, 8, (), dev, "Y")
            hp = yp = None
            ldh = ldy = 0
        else:
            _expect(H, "H", dZ.shape, dZ.dtype, dev)
            _expect(Y, "Y", dZ.shape, dZ.dtype, dev)
            h8 = y8 = None
            hp, ldh, yp, ldy = H.data_ptr(), _pitch(H)[0], Y.data_ptr(), _pitch(Y)[0]
        dX, dxp, lddx = _rows(dX, "dX", dZ)
        dY, dyp, lddy = _rows(dY, "dY", dZ)
        if gate is None:
            if dgate is not None:
                raise ValueError("dgate without a gate")
            dgp, lddg = None, 0
        else:
            if dgate is None:
                dgate = torch.empty(gate.shape, dtype=gate.dtype, device=dev)
            dgp, lddg, _ = _gate(dgate, dZ, "dgate")
            if dgate.dim() != gate.dim():
                _fail("dgate", "like the gate", dgate)
        if dw_post is None:
            dw_post = torch.empty((d,), dtype=torch.float32, device=dev)
        if dw_pre is None:
            dw_pre = torch.empty((d,), dtype=torch.float32, device=dev)
        need = lib.galore_norm_block_backward_workspace_size(tokens, d)
        workspace, wsp, wsb = _workspace(workspace, need, dev)
        _check(lib.galore_norm_block_backward(
            dZ.data_ptr(), _pitch(dZ)[0], None if dH is None else dH.data_ptr(), 0 if dH is None else _pitch(dH)[0], dt, hp,
            ldh, yp, ldy, h8, y8, rstd.data_ptr(), wo, wp, gp, ldgate, mode, alpha, tokens, d, dxp, lddx, dyp, lddy, dgp,
            lddg, _vector(dw_post, "dw_post", dZ), _vector(dw_pre, "dw_pre", dZ), wsp, wsb, h),
            "galore_norm_block_backward")
    return dX, dY, dgate, dw_post, dw_pre
