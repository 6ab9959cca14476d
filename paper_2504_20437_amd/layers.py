"""Operators between linear layers: the embedding and its gradient, dropout, the norms
of heads with their rotation, and a gated linear recurrence.

Argument marshalling only, as in ``training.py``: every tensor's device, dtype, shape
and strides are checked before any device access, work is enqueued on the current
stream or the one given, outputs and workspaces not given are allocated there.
Autograd does not see these calls. What each keeps for its backward pass: nothing
(embedding, dropout), its inputs (head norms; or their 8-bit checkpoints), its inputs
and one state every 64 tokens (recurrence).
"""
from __future__ import annotations

import ctypes

import torch

from . import _check, lib
from .training import (MxMatrix, _batch, _code, _fail, _float, _given, _mx, _on_stream, _out_vector, _pair, _pitch, _Tensor,
                       _vector, _workspace)

_STEP = 64   # tokens from one kept state of the recurrence to the next


class HeadsMatrix(ctypes.Structure):
    """galore_heads_t"""
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


def declare(lib):
    vp, sz, i32, i64, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    u64, u32 = ctypes.c_uint64, ctypes.c_uint32
    mx, heads = ctypes.POINTER(MxMatrix), ctypes.POINTER(HeadsMatrix)
    for name, args, res in (
        ("galore_embedding", [vp, i32, i64, vp, i32, i64, i64, i64, f32, vp, i32, i64, vp], i32),
        ("galore_embedding_grad_workspace_size", [i64, i64, i64], sz),
        ("galore_embedding_grad", [vp, i32, i64, vp, i32, i64, i64, i64, f32, vp, i32, i64, i32, vp, sz, vp], i32),
        ("galore_dropout", [vp, i64, i64, i32, vp, i64, i64, i64, i64, f32, u64, u32, vp, i64, i64, mx, i32, vp], i32),
        ("galore_head_norm", [heads, i32, heads, i32, i32, i64, i64, vp, vp, vp, i64, i64, i64, vp, i32, i32, f32, heads,
                              heads, vp], i32),
        ("galore_head_norm_backward_workspace_size", [i64, i32, i32, i64], sz),
        ("galore_head_norm_backward", [heads, i32, heads, i32, i32, i64, i64, heads, heads, mx, mx, vp, vp, vp, i64, i64,
                                       i64, vp, i32, i32, f32, heads, heads, vp, vp, vp, sz, vp], i32),
        ("galore_recurrence_states", [i64], i64),
        ("galore_recurrence_workspace_size", [i64, i64, i32], sz),
        ("galore_recurrence", [vp, i64, i64, vp, i64, i64, i32, i64, i64, vp, vp, i32, i64, vp, i64, i64, vp, vp, i32, vp,
                               sz, vp], i32),
        ("galore_recurrence_backward", [vp, i64, i64, vp, i64, i64, vp, i64, i64, i32, i64, i64, vp, vp, vp, vp, i32, i64,
                                        vp, i64, i64, vp, i64, i64, vp, i32, vp, sz, vp], i32),
    ):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, res


def _indices(t, name, device, length=None):
    """(pointer, bytes) of a vector of int32 or int64"""
    if (not isinstance(t, _Tensor) or t.dtype not in (torch.int32, torch.int64) or t.dim() != 1 or t.device != device or
            not t.is_contiguous() or (length is not None and t.shape[0] != length)):
        _fail(name, "a contiguous vector of %sint32 or int64 on %s" % ("" if length is None else "%d " % length, device), t)
    return t.data_ptr(), 4 if t.dtype == torch.int32 else 8


def _packed(t, name, shape, device):
    """pointer of a contiguous float32 tensor"""
    if not isinstance(t, _Tensor) or t.dtype != torch.float32 or t.shape != shape or t.device != device or \
            not t.is_contiguous():
        _fail(name, "a contiguous float32 tensor %s on %s" % (tuple(shape), device), t)
    return t.data_ptr()


def _empty(like):
    """a contiguous tensor of the same shape and type (empty_like is the cheapest call that makes one)"""
    t = torch.empty_like(like)
    return t if t.is_contiguous() else torch.empty(like.shape, dtype=like.dtype, device=like.device)


def _matrix(t, name, like):
    """(tensor, pointer, row pitch, matrix stride) of the given tensor, or of a new one of `like`'s shape and type"""
    if t is None:
        t = _empty(like)
        shape = like.shape
        return t, t.data_ptr(), shape[-1], shape[-2] * shape[-1]
    return (t,) + _given(t, name, like.shape, like.dtype, like.device)


# ---- embedding ------------------------------------------------------------------------


@_on_stream
def galore_embedding(_h, ids: torch.Tensor, W: torch.Tensor, scale: float = 1.0, out=None, dtype=None):
    """Rows scale W[ids] (tokens, d) of the embedding W (vocab, d), in ``dtype`` (W's by default). A negative id is padding
    and gives a row of zeros, one past the vocabulary a row of NaN."""
    dev = ids.device
    ip, ib = _indices(ids, "ids", dev)
    tokens = ids.shape[0]
    wt = _float(W, "W", (2,))
    if W.device != dev:
        _fail("W", "on %s" % dev, W)
    vocab, d = W.shape
    if out is None:
        dtype = dtype or W.dtype
        ot = _code(dtype)
        out = torch.empty((tokens, d), dtype=dtype, device=dev)
        op, ldo = out.data_ptr(), d
    else:
        ot = _float(out, "out", (2,))
        op, ldo, _ = _given(out, "out", (tokens, d), out.dtype, dev)
    _check(lib.galore_embedding(ip, ib, tokens, W.data_ptr(), wt, vocab, d, _pitch(W)[0], scale, op, ot, ldo, _h),
           "galore_embedding")
    return out


def galore_embedding_grad_workspace_size(tokens: int, vocab: int, d: int) -> int:
    return int(lib.galore_embedding_grad_workspace_size(tokens, vocab, d))


@_on_stream
def galore_embedding_grad(_h, ids: torch.Tensor, dY: torch.Tensor, vocab: int, scale: float = 1.0, G=None,
                          accumulate: bool = False, dtype=None, workspace=None):
    """Gradient G (vocab, d) of the embedding's matrix, as galore_step takes it: row v is scale times the sum of the rows of
    dY (tokens, d) whose id is v; added to G with ``accumulate``, else zero where no token has the id. G is allocated in
    ``dtype`` (dY's by default) where it is not given. Padding (ids under zero) has no gradient."""
    dev = ids.device
    ip, ib = _indices(ids, "ids", dev)
    tokens = ids.shape[0]
    yt = _float(dY, "dY", (2,))
    if dY.shape[0] != tokens or dY.device != dev:
        _fail("dY", "a row for each of %d ids on %s" % (tokens, dev), dY)
    d = dY.shape[1]
    if G is None:
        if accumulate:
            raise ValueError("accumulate needs G")
        dtype = dtype or dY.dtype
        gt = _code(dtype)
        G = torch.empty((vocab, d), dtype=dtype, device=dev)
        gp, ldg = G.data_ptr(), d
    else:
        gt = _float(G, "G", (2,))
        gp, ldg, _ = _given(G, "G", (vocab, d), G.dtype, dev)
    workspace, wp, wb = _workspace(workspace, lib.galore_embedding_grad_workspace_size(tokens, vocab, d), dev)
    _check(lib.galore_embedding_grad(ip, ib, tokens, dY.data_ptr(), yt, _pitch(dY)[0], vocab, d, scale, gp, gt, ldg,
                                     1 if accumulate else 0, wp, wb, _h), "galore_embedding_grad")
    return G


# ---- dropout ----------------------------------------------------------------------------


@_on_stream
def galore_dropout(_h, X: torch.Tensor, p: float, seed: int, index: int = 0, residual=None, out=None, checkpoint=None):
    """Dropout of X ((tokens, cols) or (batch, tokens, cols)) with chance p, added to ``residual`` if it is given. Returns
    (Y, y8): y8 is Y's 8-bit checkpoint with ``checkpoint`` (True or a pair of codes and scales), else None. The mask is
    made from (seed, index, place) and not stored: the gradient of X is the same call on Y's gradient, without residual.
    Take another seed or index (below 2^32) for each layer and step. out may be X or the residual."""
    dt = _float(X, "X")
    shape, dev = X.shape, X.device
    lead, tokens, cols = tuple(shape[:-2]), shape[-2], shape[-1]
    if not 0 <= seed < 2 ** 64 or not 0 <= index < 2 ** 32:
        raise ValueError("seed must be in [0, 2^64) and index in [0, 2^32)")
    rp, ldr, sr = None, 0, 0
    if residual is not None:
        rp, ldr, sr = _given(residual, "residual", shape, X.dtype, dev)
    out, yp, ldy, sy = _matrix(out, "out", X)
    y8 = q = None
    if checkpoint is not None and checkpoint is not False:
        y8, q = _pair(None if checkpoint is True else checkpoint, tokens, cols, 8, lead, dev, "checkpoint")
    ld, st = _pitch(X)
    _check(lib.galore_dropout(X.data_ptr(), ld, st, dt, rp, ldr, sr, tokens, cols, p, seed, index, yp, ldy, sy, q,
                              _batch(lead), _h), "galore_dropout")
    return out, y8


# ---- norms of heads with their rotation ---------------------------------------------------


def _heads(t, name, shape, dtype, device):
    """the struct of a (tokens, heads, d) tensor"""
    if not isinstance(t, _Tensor) or t.dtype != dtype or t.shape != shape or t.device != device:
        _fail(name, "%s %s on %s" % (dtype, tuple(shape), device), t)
    s = t.stride()
    if s[2] != 1 and shape[2] > 1:
        _fail(name, "a tensor with packed heads", t)
    return HeadsMatrix(t.data_ptr(), s[0], s[1])


def _heads_out(t, name, like, shape):
    if t is None:
        t = _empty(like)
        return t, HeadsMatrix(t.data_ptr(), shape[1] * shape[2], shape[2])
    return t, _heads(t, name, shape, like.dtype, like.device)


def _rotation(table, positions, tokens, device):
    """(table pointer, rows, pitch, rot, positions pointer, bytes)"""
    if not isinstance(table, _Tensor) or table.dim() != 2:
        _fail("table", "a float32 (positions, rot) tensor on %s" % device, table)
    shape = table.shape
    tp, ldt, _ = _given(table, "table", shape, torch.float32, device)
    pp, pb = (None, 4) if positions is None else _indices(positions, "positions", device, tokens)
    return tp, shape[0], ldt, shape[1], pp, pb


def _head_shapes(Q, K, q_name, k_name):
    dt = _float(Q, q_name, (3,))
    q, k = Q.shape, K.shape if isinstance(K, _Tensor) else ()
    if len(k) != 3 or k[0] != q[0] or k[2] != q[2]:
        _fail(k_name, "of as many tokens and values to a head as %s" % q_name, K)
    return dt, q, k, Q.device


@_on_stream
def galore_head_norm(_h, Q: torch.Tensor, K: torch.Tensor, w_q: torch.Tensor, w_k: torch.Tensor, table: torch.Tensor,
                     positions=None, interleaved: bool = False, eps: float = 1e-5, Q_out=None, K_out=None):
    """Norms of queries Q (tokens, heads, d) and keys K (tokens, key heads, d) for each head, times w_q and w_k (float32, d),
    and their rotation by position: (Q_out, K_out), which may be Q and K. Q and K may be views of one product's output, or
    of (heads, tokens, d) tensors. table: float32 (positions, rot), rot / 2 cosines and rot / 2 sines a row, for pairs
    (k, k + rot / 2) of a head's values, or (2 k, 2 k + 1) with ``interleaved``. positions: int32 or int64, a token's own
    number if None; a negative one is padding and gives zeros, one past the table NaN."""
    dt, qs, ks, dev = _head_shapes(Q, K, "Q", "K")
    (tokens, hq, d), hk, dtype = qs, ks[1], Q.dtype
    q, k = _heads(Q, "Q", qs, dtype, dev), _heads(K, "K", ks, dtype, dev)
    wq, wk = _vector(w_q, "w_q", d, dev), _vector(w_k, "w_k", d, dev)
    tp, rows, ldt, rot, pp, pb = _rotation(table, positions, tokens, dev)
    Q_out, qo = _heads_out(Q_out, "Q_out", Q, qs)
    K_out, ko = _heads_out(K_out, "K_out", K, ks)
    _check(lib.galore_head_norm(q, hq, k, hk, dt, tokens, d, wq, wk, tp, rows, ldt, rot, pp, pb, 1 if interleaved else 0,
                                eps, qo, ko, _h), "galore_head_norm")
    return Q_out, K_out


def galore_head_norm_backward_workspace_size(tokens: int, q_heads: int, k_heads: int, d: int) -> int:
    return int(lib.galore_head_norm_backward_workspace_size(tokens, q_heads, k_heads, d))


@_on_stream
def galore_head_norm_backward(_h, dQ: torch.Tensor, dK: torch.Tensor, Q, K, w_q: torch.Tensor, w_k: torch.Tensor,
                              table: torch.Tensor, positions=None, interleaved: bool = False, eps: float = 1e-5, dQ_in=None,
                              dK_in=None, dw_q=None, dw_k=None, workspace=None):
    """Gradients of galore_head_norm from those of its outputs: (dQ_in, dK_in, dw_q, dw_k); dQ_in and dK_in may be dQ and
    dK. Q and K: both as they went into the forward pass, or both 8-bit checkpoints (codes, scales) of (tokens, heads d)."""
    dt, qs, ks, dev = _head_shapes(dQ, dK, "dQ", "dK")
    (tokens, hq, d), hk, dtype = qs, ks[1], dQ.dtype
    gq, gk = _heads(dQ, "dQ", qs, dtype, dev), _heads(dK, "dK", ks, dtype, dev)
    q = k = q8 = k8 = None
    if isinstance(Q, _Tensor) and isinstance(K, _Tensor):
        q, k = _heads(Q, "Q", qs, dtype, dev), _heads(K, "K", ks, dtype, dev)
    elif isinstance(Q, (tuple, list)) and isinstance(K, (tuple, list)):
        q8, k8 = _mx(*Q, tokens, hq * d, 8, (), dev, "Q"), _mx(*K, tokens, hk * d, 8, (), dev, "K")
    else:
        raise ValueError("Q and K must both be tensors or both be checkpoints")
    wq, wk = _vector(w_q, "w_q", d, dev), _vector(w_k, "w_k", d, dev)
    tp, rows, ldt, rot, pp, pb = _rotation(table, positions, tokens, dev)
    dQ_in, qo = _heads_out(dQ_in, "dQ_in", dQ, qs)
    dK_in, ko = _heads_out(dK_in, "dK_in", dK, ks)
    dw_q, dwq = _out_vector(dw_q, "dw_q", w_q, d, dev)
    dw_k, dwk = _out_vector(dw_k, "dw_k", w_k, d, dev)
    workspace, wp, wb = _workspace(workspace, lib.galore_head_norm_backward_workspace_size(tokens, hq, hk, d), dev)
    _check(lib.galore_head_norm_backward(gq, hq, gk, hk, dt, tokens, d, q, k, q8, k8, wq, wk, tp, rows, ldt, rot, pp, pb,
                                         1 if interleaved else 0, eps, qo, ko, dwq, dwk, wp, wb, _h),
           "galore_head_norm_backward")
    return dQ_in, dK_in, dw_q, dw_k


# ---- gated linear recurrence ---------------------------------------------------------------


def galore_recurrence_workspace_size(tokens: int, d: int, batch: int = 1) -> int:
    return int(lib.galore_recurrence_workspace_size(tokens, d, batch))


def _sequences(offsets, lead, batch, device):
    """(pointer, bytes, sequences)"""
    if offsets is None:
        return None, 4, batch
    if lead:
        raise ValueError("offsets belong to packed sequences of shape (tokens, d)")
    p, nbytes = _indices(offsets, "offsets", device)
    if offsets.shape[0] < 2:
        _fail("offsets", "the bounds of one sequence or more", offsets)
    return p, nbytes, offsets.shape[0] - 1


@_on_stream
def galore_recurrence(_h, X: torch.Tensor, F: torch.Tensor, h0=None, offsets=None, H=None, last=None, states=False,
                      workspace=None):
    """Gated linear recurrence H_t = a H_{t-1} + (1 - a) X_t, a = sigmoid(F_t), in each channel of X and F ((tokens, d) or
    (batch, tokens, d)). Each matrix is a sequence, or, with ``offsets`` (int32 or int64, ascending), the tokens from
    offsets[s] to offsets[s + 1] of X (tokens, d) are; tokens of no sequence are left as they are in H. h0: float32
    (sequences, d), zeros if None. Returns (H, last, states): last, float32 (sequences, d), holds the states after the last
    tokens; ``states`` (True, or a float32 tensor (..., ceil(tokens / 64), d)) those that galore_recurrence_backward needs,
    else None. H may be X or F; last may be h0 without offsets, so that single tokens step their states in place."""
    dt = _float(X, "X")
    shape, dev = X.shape, X.device
    lead, tokens, d = tuple(shape[:-2]), shape[-2], shape[-1]
    batch = _batch(lead)
    fp, ldf, sf = _given(F, "F", shape, X.dtype, dev)
    op, ob, n = _sequences(offsets, lead, batch, dev)
    h0p = None if h0 is None else _packed(h0, "h0", (n, d), dev)
    H, hp, ldh, sh = _matrix(H, "H", X)
    if last is None:
        last = torch.empty((n, d), dtype=torch.float32, device=dev) if h0 is None else torch.empty_like(h0)
        lp = last.data_ptr()
    else:
        lp = _packed(last, "last", (n, d), dev)
    if states is True:
        states = torch.empty(lead + (-(-tokens // _STEP), d), dtype=torch.float32, device=dev)
    elif states is False:
        states = None
    sp = None if states is None else _packed(states, "states", lead + (-(-tokens // _STEP), d), dev)
    workspace, wp, wb = _workspace(workspace, lib.galore_recurrence_workspace_size(tokens, d, batch), dev)
    ld, st = _pitch(X)
    _check(lib.galore_recurrence(X.data_ptr(), ld, st, fp, ldf, sf, dt, tokens, d, h0p, op, ob, n, hp, ldh, sh, lp, sp, batch,
                                 wp, wb, _h), "galore_recurrence")
    return H, last, states


@_on_stream
def galore_recurrence_backward(_h, dH: torch.Tensor, X: torch.Tensor, F: torch.Tensor, states: torch.Tensor, h0=None,
                               dlast=None, offsets=None, dX=None, dF=None, dh0=None, workspace=None):
    """Gradients of galore_recurrence, (dX, dF, dh0), from dH and dlast (that of ``last``, zeros if None). X, F, h0 and
    offsets as in the forward pass, states as it returned them. dX and dF may be dH, X or F."""
    dt = _float(dH, "dH")
    shape, dev = dH.shape, dH.device
    lead, tokens, d = tuple(shape[:-2]), shape[-2], shape[-1]
    batch = _batch(lead)
    xp, ldx, sx = _given(X, "X", shape, dH.dtype, dev)
    fp, ldf, sf = _given(F, "F", shape, dH.dtype, dev)
    op, ob, n = _sequences(offsets, lead, batch, dev)
    sp = _packed(states, "states", lead + (-(-tokens // _STEP), d), dev)
    h0p = None if h0 is None else _packed(h0, "h0", (n, d), dev)
    dlp = None if dlast is None else _packed(dlast, "dlast", (n, d), dev)
    dX, dxp, lddx, sdx = _matrix(dX, "dX", dH)
    dF, dfp, lddf, sdf = _matrix(dF, "dF", dH)
    if dh0 is None:
        dh0 = torch.empty((n, d), dtype=torch.float32, device=dev)
        dhp = dh0.data_ptr()
    else:
        dhp = _packed(dh0, "dh0", (n, d), dev)
    workspace, wp, wb = _workspace(workspace, lib.galore_recurrence_workspace_size(tokens, d, batch), dev)
    ld, st = _pitch(dH)
    _check(lib.galore_recurrence_backward(dH.data_ptr(), ld, st, xp, ldx, sx, fp, ldf, sf, dt, tokens, d, sp, h0p, dlp, op,
                                          ob, n, dxp, lddx, sdx, dfp, lddf, sdf, dhp, batch, wp, wb, _h),
           "galore_recurrence_backward")
    return dX, dF, dh0
