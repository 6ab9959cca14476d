"""Plain 64-bit forms of the training operators, on the CPU with numpy: block
codes, the products over them, the norms of a block and their gradients."""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def _nearest_even(u, values):
    """index of the value nearest to each u >= 0 (u at most the largest), ties to the even index"""
    hi = np.minimum(np.searchsorted(values, u, side="left"), len(values) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = values[hi] - u, u - values[lo]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def _scale_exponents(x, largest, floor, top):
    """x (rows, cols) in blocks: values (rows, nb, 32), exponents, which blocks hold a NaN or Inf"""
    rows, cols = x.shape
    nb = -(-cols // 32)
    v = np.zeros((rows, nb * 32))
    v[:, :cols] = x
    v = v.reshape(rows, nb, 32)
    bad = ~np.isfinite(v).all(axis=2)
    v = np.where(bad[:, :, None], 0.0, v)
    m, e = np.frexp(np.abs(v).max(axis=2) / largest)    # m in [.5, 1): the smallest power of two not below
    e = np.where(m > 0.5, e, e - 1)
    e = np.where(m > 0, np.clip(e, floor, top), floor)
    return v, e, bad


def _pad4(scales):
    return np.pad(scales, ((0, 0), (0, -scales.shape[1] % 4))).astype(np.uint8)


def mx8_encode(x):
    """(codes int8 (rows, 32 nb), scales uint8 (rows, nb padded to 4))"""
    v, e, bad = _scale_exponents(np.asarray(x, np.float64), 127, -125, 121)
    u = np.minimum(np.abs(v) * np.exp2(-e.astype(np.float64))[:, :, None], 127)
    c = np.sign(v) * _nearest_even(u, np.arange(128.0))
    scales = np.where(bad, 255, e + 133)
    return c.reshape(x.shape[0], -1).astype(np.int8), _pad4(scales)


def _units(scales, cols, shift):
    s = scales.astype(np.int64)[:, np.arange(cols) // 32]
    return np.where(s == 255, np.nan, np.exp2((s - shift).astype(np.float64)))


def mx8_decode(codes, scales, cols):
    return codes[:, :cols].astype(np.float64) * _units(scales, cols, 133)


def mx4_encode(x):
    v, e, bad = _scale_exponents(np.asarray(x, np.float64), 6, -124, 125)
    u = np.minimum(np.abs(v) * np.exp2(-e.astype(np.float64))[:, :, None], 6)
    q = _nearest_even(u, E2M1) | (np.signbit(v).astype(np.int64) << 3)
    q = np.where(bad[:, :, None], 0, q).reshape(x.shape[0], -1)
    return (q[:, 0::2] | (q[:, 1::2] << 4)).astype(np.uint8), _pad4(np.where(bad, 255, e + 127))


def mx4_decode(codes, scales, cols):
    q = np.stack((codes & 15, codes >> 4), axis=2).reshape(codes.shape[0], -1)[:, :cols]
    v = np.where(q & 8, -E2M1[q & 7], E2M1[q & 7])
    return v * _units(scales, cols, 127)


def norms(x, y, w_post, w_pre, gate, alpha, eps):
    ry = 1 / np.sqrt((y * y).mean(1, keepdims=True) + eps)
    h = x + alpha * gate * (y * ry) * w_post
    rh = 1 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return h, h * rh * w_pre, np.concatenate((ry, rh), axis=1)


def norms_backward(dz, dh, h, y, rstd, w_post, w_pre, gate, alpha):
    """dx, dy, the gate's gradient for each token, dw_post, dw_pre"""
    ry, rh = rstd[:, :1], rstd[:, 1:]
    n, u = h * rh, y * ry
    a = dz * w_pre
    dx = dh + rh * (a - n * (a * n).mean(1, keepdims=True))
    g = alpha * dx * gate * w_post
    dy = ry * (g - u * (g * u).mean(1, keepdims=True))
    return dx, dy, alpha * dx * u * w_post, (alpha * dx * gate * u).sum(0), (dz * n).sum(0)
