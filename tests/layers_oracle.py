"""Plain 64-bit forms of the operators between linear layers, on the CPU with numpy:
embedding, dropout, head norms with rotation, gated recurrence, and their gradients."""
import numpy as np


def lookup(ids, w, scale):
    y = np.zeros((len(ids), w.shape[1]))
    for t, i in enumerate(ids):
        y[t] = 0.0 if i < 0 else np.nan if i >= len(w) else w[i].astype(np.float64) * scale
    return y


def embedding_grad(ids, dy, vocab, scale):
    """(G, the sums of magnitudes, the counts)"""
    g, mag, n = np.zeros((vocab, dy.shape[1])), np.zeros((vocab, dy.shape[1])), np.zeros(vocab, np.int64)
    for t, i in enumerate(ids):
        if 0 <= i < vocab:
            g[i] += dy[t]
            mag[i] += np.abs(dy[t])
            n[i] += 1
    return g * scale, mag * abs(scale), n


def philox4x32(counter, key):
    """ten rounds on Python integers"""
    c, k = list(counter), list(key)
    for _ in range(10):
        p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xffffffff, (p >> 32) ^ c[3] ^ k[1], p & 0xffffffff]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return c


def dropout_bits(seed, index, batch, tokens, cols):
    """the 16 random bits of every value"""
    u = np.zeros((batch, tokens, -(-cols // 8) * 8), np.int64)
    for b in range(batch):
        for t in range(tokens):
            for j in range(-(-cols // 8)):
                w = philox4x32((j, t, b, index), (seed & 0xffffffff, seed >> 32))
                u[b, t, 8 * j:8 * j + 8] = [h for x in w for h in (x & 0xffff, x >> 16)]
    return u[:, :, :cols]


def pairs(d, rot, interleaved):
    """the places of the rotated pairs"""
    k = np.arange(rot // 2)
    return (2 * k, 2 * k + 1) if interleaved else (k, k + rot // 2)


def head_norm(x, w, cos, sin, interleaved, eps):
    """x (tokens, heads, d); cos, sin (tokens, rot / 2). (y, n)"""
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r * w
    y = n.copy()
    i, j = pairs(x.shape[-1], 2 * cos.shape[1], interleaved)
    c, s = cos[:, None, :], sin[:, None, :]
    y[..., i] = n[..., i] * c - n[..., j] * s
    y[..., j] = n[..., i] * s + n[..., j] * c
    return y, n


def head_norm_backward(dy, x, w, cos, sin, interleaved, eps):
    """dx, dw, and bounds of what was summed for them: magnitudes for dx and for dw"""
    d = x.shape[-1]
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    i, j = pairs(d, 2 * cos.shape[1], interleaved)
    c, s = cos[:, None, :], sin[:, None, :]
    m, mag = dy.copy(), np.abs(dy)
    m[..., i] = dy[..., i] * c + dy[..., j] * s
    m[..., j] = dy[..., j] * c - dy[..., i] * s
    mag[..., i] = np.abs(dy[..., i] * c) + np.abs(dy[..., j] * s)
    mag[..., j] = np.abs(dy[..., j] * c) + np.abs(dy[..., i] * s)
    p = m * w
    dx = r * (p - x * r * r * (p * x).mean(-1, keepdims=True))
    bound = r * (mag * np.abs(w) + np.abs(x) * r * r * (mag * np.abs(w * x)).mean(-1, keepdims=True))
    return dx, (m * x * r).sum((0, 1)), bound, (mag * np.abs(x) * r).sum((0, 1))


def sigmoid(f):
    """(sigmoid(f), sigmoid(-f))"""
    e = np.exp(-np.abs(f))
    big, small = 1 / (1 + e), e / (1 + e)
    return np.where(f >= 0, big, small), np.where(f >= 0, small, big)


def recurrence(x, f, h0, bounds):
    """x, f (tokens, d), h0 (sequences, d), bounds: sequences + 1. h (0 outside the sequences), the state before each
    token, the last states, and for h a bound of its terms times their ages"""
    a, z = sigmoid(f)
    h, before, age = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)
    last = h0.copy()
    for s in range(len(bounds) - 1):
        state, mag, k = h0[s].copy(), np.abs(h0[s]), np.abs(h0[s])
        for t in range(bounds[s], bounds[s + 1]):
            before[t] = state
            state = a[t] * state + z[t] * x[t]
            k = a[t] * (k + mag) + z[t] * np.abs(x[t])
            mag = a[t] * mag + z[t] * np.abs(x[t])
            h[t], age[t] = state, k
        last[s] = state
    return h, before, last, age


def recurrence_backward(dh, x, f, h0, dlast, bounds):
    """dx, df, dh0 and bounds of their terms times their ages"""
    a, z = sigmoid(f)
    _, before, _, age = recurrence(x, f, h0, bounds)
    aged = np.zeros_like(x)
    dx, df, dx_k, df_k = (np.zeros_like(x) for _ in range(4))
    dh0, dh0_k = dlast.copy(), np.abs(dlast)
    for s in range(len(bounds) - 1):
        aged[bounds[s]:bounds[s + 1]] = np.concatenate((np.abs(h0[s:s + 1]), age[bounds[s]:bounds[s + 1] - 1]))[
            :bounds[s + 1] - bounds[s]]
        c, mag, k = dlast[s].copy(), np.abs(dlast[s]), np.abs(dlast[s])
        for t in range(bounds[s + 1] - 1, bounds[s] - 1, -1):
            g, gm, gk = dh[t] + c, np.abs(dh[t]) + mag, np.abs(dh[t]) + k
            dx[t], dx_k[t] = z[t] * g, z[t] * (gk + gm)
            df[t] = g * (before[t] - x[t]) * a[t] * z[t]
            df_k[t] = a[t] * z[t] * ((gk + gm) * (np.abs(before[t]) + np.abs(x[t])) + gm * aged[t])
            c, mag, k = a[t] * g, a[t] * gm, a[t] * (gk + gm)
        dh0[s], dh0_k[s] = c, k + mag
    return dx, df, dh0, dx_k, df_k, dh0_k
