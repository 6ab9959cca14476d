"""The operators between linear layers at the ends of what they take: gates past the range of exp, against the 64-bit
forms.

Tolerances as in test_layers_ops.py: E = 2^-24 is half a step of fp32; a term of a recurrence that has gone through k
steps is within 10 k E, and the oracle sums the terms times k. A gate (or one less it) under G = 2^-125 may count as zero:
that moves what it weighs by G times its magnitude, in every step."""
import numpy as np
import pytest
import torch

import layers_oracle as lo
from test_layers_ops import DTYPES, E, close, n64, randn

G = 2.0 ** -125
INF, NAN = float("inf"), float("nan")
LOGITS = [-INF, -1e30, -1000.0, -104.0, -100.0, -90.0, -89.0, -88.0, -87.5, -87.0, -86.5, -85.0, -81.0, -80.0, -79.5, -60.0,
          60.0, 79.5, 80.0, 81.0, 85.0, 86.5, 87.0, 87.5, 88.0, 89.0, 100.0, 104.0, 1000.0, 1e30, INF]


@pytest.fixture(scope="module")
def gl():
    import paper_2504_20437_amd
    return paper_2504_20437_amd


def test_oracle_gates():
    """the oracle's gates at the ends, against their definition"""
    a, z = lo.sigmoid(np.array([-INF, -100.0, -85.0, 0.0, 85.0, 100.0, INF]))
    want = [0.0, 1 / (1 + np.exp(100.0)), 1 / (1 + np.exp(85.0)), 0.5]
    assert np.allclose(a[:4], want, rtol=1e-15, atol=0) and np.allclose(z[3:], want[::-1], rtol=1e-15, atol=0)
    assert a[-1] == z[0] == 1.0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens", [1, 3, 8, 9, 150])
@pytest.mark.parametrize("packed", [False, True])
def test_gates_past_the_range_of_exp(gl, dtype, tokens, packed):
    """every logit in a channel of its own, on every third token (the others forget little); states and inputs large
    enough to show what a gate that should be gone leaves of them"""
    d = len(LOGITS)
    f = torch.full((tokens, d), 3.0)
    f[::3] = torch.tensor(LOGITS)
    f = f.to(dtype).cuda()
    x, dh = randn((tokens, d), 1, dtype), randn((tokens, d), 2, dtype)
    h0, dlast = 1e30 * randn((1, d), 3), randn((1, d), 4)
    offsets = torch.tensor([0, tokens], device="cuda") if packed else None
    H, last, states = gl.galore_recurrence(x, f, h0=h0, offsets=offsets, states=True)
    x64, f64, z0, zl = n64(x), n64(f), n64(h0), n64(dlast)
    h, before, end, age = lo.recurrence(x64, f64, z0, [0, tokens])
    peak = np.maximum(np.abs(z0[0]), np.abs(x64).max(0))             # of any state, in each channel
    close(H, h, 10 * E * age + G * tokens * peak, dtype)
    close(last, end, 10 * E * age[-1] + G * tokens * peak, torch.float32)
    got = gl.galore_recurrence_backward(dh, x, f, states, h0=h0, dlast=dlast, offsets=offsets)
    dx, df, dh0, dx_k, df_k, dh0_k = lo.recurrence_backward(n64(dh), x64, f64, z0, zl, [0, tokens])
    carry = np.abs(n64(dh)).sum(0) + np.abs(zl[0])                   # of any carry
    close(got[0], dx, 10 * E * dx_k + G * tokens * carry, dtype)
    # df is a product of a carry, two gates and (state before - x): each may move by its own G
    close(got[1], df, 10 * E * df_k + 4 * G * tokens * carry * peak, dtype)
    close(got[2], dh0, 10 * E * dh0_k + G * tokens * carry, torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens", [1, 20, 300])
def test_a_gate_of_minus_infinity_forgets(gl, dtype, tokens):
    """nothing of the state before is left, whatever its size: the state is x"""
    x, f = randn((tokens, 9), 1, dtype), torch.full((tokens, 9), -INF, dtype=dtype, device="cuda")
    h0 = torch.full((1, 9), 3e38, device="cuda")
    H, last, states = gl.galore_recurrence(x, f, h0=h0, states=True)
    close(H, n64(x), 8 * E * np.abs(n64(x)), dtype)
    close(last, n64(x[-1:]), 8 * E * np.abs(n64(x[-1:])), torch.float32)
    dx, df, dh0 = gl.galore_recurrence_backward(x, x, f, states, h0=h0)
    close(dx, n64(x), 8 * E * np.abs(n64(x)), dtype)
    assert (df == 0).all() and (dh0 == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens", [5, 200])
def test_gates_that_are_no_numbers(gl, dtype, tokens):
    """NaN from the token on in its channel, and nowhere else; backward up to it"""
    x, f, dh = randn((tokens, 7), 1, dtype), randn((tokens, 7), 2, dtype), randn((tokens, 7), 3, dtype)
    at = tokens // 2
    f[at, 4] = NAN
    H, last, states = gl.galore_recurrence(x, f, states=True)
    zero = np.zeros((1, 7))
    h, _, end, age = lo.recurrence(n64(x), n64(f), zero, [0, tokens])
    assert np.isnan(h[at:, 4]).all() and not np.isnan(np.delete(h, 4, 1)).any()
    close(H, h, 10 * E * np.nan_to_num(age), dtype)
    close(last, end, 10 * E * np.nan_to_num(age[-1]), torch.float32)
    got = gl.galore_recurrence_backward(dh, x, f, states)
    want = lo.recurrence_backward(n64(dh), n64(x), n64(f), zero, zero, [0, tokens])
    for g, w, k, t in ((got[0], want[0], want[3], dtype), (got[1], want[1], want[4], dtype), (got[2], want[2], want[5], torch.float32)):
        close(g, w, 10 * E * np.nan_to_num(k), t)
