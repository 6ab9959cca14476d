"""One backward pass of the example against the definition, on the operands that it used."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U, B = 2.0 ** -24, 2.0 ** -8       # largest relative rounding errors of fp32 and bfloat16


@pytest.fixture
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import lean_training
    finally:
        sys.path.pop(0)
    return lean_training


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,d,hidden", [(256, 256, 688), (100, 96, 203)])
def test_gradients_of_one_step(example, monkeypatch, tokens, d, hidden):
    gl = example.gl
    acts, grads, steps = [], [], []
    pack, step = gl.galore_checkpoint_pack, example.Weight.step

    def keep_activation(a, *args, **kw):
        acts.append(a.clone())
        return pack(a, *args, **kw)

    def keep_step(self, dy, x8, tau, lr):
        steps.append((self, dy.clone(), x8))
        return step(self, dy, x8, tau, lr)

    # the weights stay as they are: every product of the pass is of the same operands
    monkeypatch.setattr(gl, "galore_checkpoint_pack", keep_activation)
    monkeypatch.setattr(gl, "galore_step", lambda G, *args, **kw: grads.append(G.clone()))
    monkeypatch.setattr(example.Weight, "step", keep_step)
    model = example.Model(d, hidden, 2, 16)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    out, saved = model.forward(torch.randn((tokens, d), generator=g, device="cuda").bfloat16())
    model.backward((1e-3 * torch.randn((tokens, d), generator=g, device="cuda")).bfloat16(), saved, 0, 0.0)
    assert len(acts) == 2 and len(steps) == 4 and len(grads) == 4
    for i, a in enumerate(reversed(acts)):
        (w2, dy, a8), (w1, da, z8) = steps[2 * i], steps[2 * i + 1]
        on = a > 0
        # units that are on, though their checkpoint holds zero for them, are in the test
        assert (on & (gl.galore_checkpoint_unpack(*a8, hidden) == 0)).any()
        # through the product and the ReLU, with the derivative of the activation that was
        dq = gl.galore_mx4_dequantize(*gl.galore_mx4_quantize(dy), d, dtype=torch.float32).double()
        wc = gl.galore_mx4_dequantize(*w2.columns, d, dtype=torch.float32).double()      # W2^T
        want, size = dq @ wc.t() * on, dq.abs() @ wc.abs().t()
        assert ((da.double() - want).abs() <= B * want.abs() + 2 * (d + 4) * U * size).all()
        assert (da[~on] == 0).all()
        # and the weight gradients of both layers
        for G, grad, x8, n in ((grads[2 * i], dy, a8, hidden), (grads[2 * i + 1], da, z8, d)):
            x = gl.galore_checkpoint_unpack(*x8, n, dtype=torch.float32).double()
            want, size = grad.double().t() @ x, grad.double().abs().t() @ x.abs()
            assert ((G.double() - want).abs() <= B * want.abs() + 2 * (tokens + 4) * U * size).all()
