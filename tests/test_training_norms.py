"""The norms' gradients against autograd, and the calls that write over an input at widths of several waves."""
import pytest
import torch

import test_training_ops as ops
import training_oracle as ora
from test_training_ops import ALPHA, DTYPES, EPS, checkpoint, close, host, norm_inputs, on, values


@pytest.fixture(scope="module")
def gl():
    import paper_2504_20437_amd
    return paper_2504_20437_amd


def rms(v):
    return (v * v).mean(1, keepdim=True).add(EPS).rsqrt()


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("gate", ["none", "vector", "tokens"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,d", [(7, 96), (40, 1025), (5, 4097), (3, 8200)])
def test_gradients_against_autograd(gl, t, d, dtype, gate, packed):
    """torch differentiates the forward formulas in 64 bits, statistics and all, at the H and Y that the kernel reads.

    The kernel takes the statistics rounded to fp32: at most six of them stand in a term, 8 U more than the bounds of
    the comparison with the formulas."""
    x, y, wo, wp, gt = norm_inputs(t, d, dtype, gate, t + d)
    dz, dh = values(t, d, dtype, 5, "gradients"), values(t, d, dtype, 6, "gradients")
    h = torch.from_numpy(ora.norms(host(x), host(y), host(wo), host(wp), 1.0 if gt is None else host(gt), ALPHA, EPS)[0])
    h = h.to(DTYPES[dtype])
    if packed:
        h_in, y_in = checkpoint(h), checkpoint(y)
        h64, y64 = (torch.from_numpy(ora.mx8_decode(host(c), host(s), d)) for c, s in (h_in, y_in))
    else:
        h_in, y_in, h64, y64 = on(h), on(y), h.double(), y.double()
    leaves = [v.double().clone().requires_grad_() for v in (h64, y64, wo, wp)]
    hv, yv, wov, wpv = leaves
    gv = torch.ones(1, dtype=torch.float64) if gt is None else gt.double().clone().requires_grad_()
    rstd = torch.cat((rms(y64), rms(h64)), dim=1)
    got = gl.galore_norm_block_backward(on(dz), on(dh), h_in, y_in, on(rstd.float()), on(wo), on(wp), on(gt), alpha=ALPHA)

    # Z and the stream, as functions of H; then the block's part of H, as one of Y and the weights
    ((hv * rms(hv) * wpv) * dz.double()).sum().add((hv * dh.double()).sum()).backward()
    dx = hv.grad
    (ALPHA * gv * (yv * rms(yv)) * wov * dx).sum().backward()

    a = torch.abs
    ry, rh = rstd[:, :1], rstd[:, 1:]
    n, u, p = a(h64 * rh), a(y64 * ry), a(dz.double() * wp.double())
    sx = a(dh.double()) + rh * (p + n * (p * n).mean(1, keepdim=True))
    ga = a(gv.detach())
    g = ALPHA * sx * ga * a(wo.double())
    bounds = [(got[0], dx, sx, d), (got[1], yv.grad, ry * (g + u * (g * u).mean(1, keepdim=True)), 2 * d + 16),
              (got[3], wov.grad, (ALPHA * sx * ga * u).sum(0), d + t + 16),
              (got[4], wpv.grad, (a(dz.double()) * n).sum(0), d + t)]
    if gt is not None:
        each = ALPHA * sx * u * a(wo.double())
        bounds.append((got[2], gv.grad, each if gate == "tokens" else each.sum(0), d + 16 + (t if gate == "vector" else 0)))
    for value, want, size, count in bounds:
        close(value, want.numpy(), size.numpy(), count + 8)


@pytest.mark.gpu
@pytest.mark.parametrize("gate", ["none", "vector", "tokens"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [513, 1025, 2049, 4097, 8193])
def test_in_place_at_wide_rows(gl, d, dtype, gate):
    """the group across a row's end is read with the group before it, which another wave writes"""
    t = 300
    x, y, wo, wp, gt = norm_inputs(t, d, dtype, gate, d)
    y, wo, wp, gt = on(y), on(wo), on(wp), on(gt)
    H, Z, R, *_ = gl.galore_norm_block(on(x), y, wo, wp, gt, alpha=ALPHA)
    dz, dh = on(values(t, d, dtype, 5, "gradients")), values(t, d, dtype, 6, "gradients")
    want = gl.galore_norm_block_backward(dz, on(dh), H, y, R, wo, wp, gt, alpha=ALPHA)
    for pad, offset in ((0, 0), (7, 0), (3, 1)):
        xd = on(x, pad, offset)
        out = gl.galore_norm_block(xd, y, wo, wp, gt, alpha=ALPHA, H=xd)
        assert out[0] is xd and torch.equal(xd, H) and torch.equal(out[1], Z) and torch.equal(out[2], R)
        dx = on(dh, pad, offset)
        got = gl.galore_norm_block_backward(dz, dx, H, y, R, wo, wp, gt, alpha=ALPHA, dX=dx)
        assert got[0] is dx and all(p is q is None or torch.equal(p, q) for p, q in zip(got, want))
