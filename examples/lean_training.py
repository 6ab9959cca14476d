"""A training step that holds little: residual MLP blocks whose activations live in
8 bits between the passes, whose products run in 4 bits, and whose weights are
stepped by GaLore.

    h, z = norm_block(x, y)            norm after the block before, gate, residual, next norm
    a = relu(z W1^T), y = a W2^T       4-bit products, z and a kept as 8-bit checkpoints,
                                       and one bit a value for where a > 0

backward: data gradients in 4 bits (weights in blocks along their columns), weight
gradients from the checkpoints, the norms' gradients from the checkpoints of y and
h, one galore_step for each weight. Synthetic data: the targets are a random
network's answers.

    python examples/lean_training.py --steps 60
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2504_20437_amd as gl  # noqa: E402


def pack_positive(a):
    """Which values of a are positive, one bit each. The ReLU's derivative is taken from these, not from the checkpoint
    of a: a small positive value, under half a step of its block's codes, is a zero there."""
    bits = torch.nn.functional.pad(a > 0, (0, -a.shape[1] % 8)).view(a.shape[0], -1, 8)
    return (bits << torch.arange(8, dtype=torch.uint8, device=a.device)).sum(-1, dtype=torch.uint8)


def unpack_positive(bits, cols):
    """True where pack_positive saw a positive value"""
    m = bits.unsqueeze(-1) >> torch.arange(8, dtype=torch.uint8, device=bits.device) & 1
    return m.view(bits.shape[0], -1)[:, :cols] != 0


class Weight:
    """A matrix under GaLore: fp32 weight and moments, its projector, its 4-bit forms for the products."""

    def __init__(self, out_features, in_features, rank, generator):
        self.w = torch.randn((out_features, in_features), generator=generator, device="cuda") / in_features ** 0.5
        self.rank = rank
        s, l = sorted((out_features, in_features))
        self.p = torch.empty((s, rank), device="cuda")
        self.m = torch.zeros((rank, l), device="cuda")
        self.v = torch.zeros((rank, l), device="cuda")

    def quantize(self):
        """4-bit codes along the rows, for the forward product, and along the columns, for the backward one"""
        q = gl.galore_mx4_quantize(self.w, rows=True, columns=True)
        self.rows, self.columns = q[:2], q[2:]

    def forward(self, x):
        """x W^T of bf16 activations"""
        return gl.galore_mx4_matmul(*gl.galore_mx4_quantize(x), *self.rows, self.w.shape[1])

    def data_gradient(self, dy):
        return gl.galore_mx4_matmul(*gl.galore_mx4_quantize(dy), *self.columns, self.w.shape[0])

    def step(self, dy, x8, tau, lr):
        """weight gradient from the checkpoint of the input, then one GaLore step"""
        g = gl.galore_checkpoint_weight_grad(dy, *x8, self.w.shape[1])
        gl.galore_step(g, self.w, self.p, self.m, self.v, self.rank, p=8, q=1, seed=7, tau=tau, T=20, lr=lr, alpha=1.0,
                       flags=gl.GALORE_STEP_ALIGN)


class Block:
    def __init__(self, d, hidden, rank, generator):
        self.w1, self.w2 = Weight(hidden, d, rank, generator), Weight(d, hidden, rank, generator)
        # the norm before this block, and the norm after it with its gate
        self.pre = torch.ones(d, device="cuda")
        self.post = torch.ones(d, device="cuda")
        self.gate = torch.full((d,), 0.5, device="cuda")


class Model:
    """blocks over a residual stream; stream i + 1 = stream i + alpha gate norm(block i)"""

    def __init__(self, d, hidden, blocks, rank, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.blocks = [Block(d, hidden, rank, g) for _ in range(blocks)]
        self.last = torch.ones(d, device="cuda")     # the norm before the output
        self.none = torch.zeros(d, device="cuda")    # nothing comes before the first block
        self.ones = torch.ones(d, device="cuda")
        self.alpha = blocks ** -0.5

    def _norm(self, i, x, y, saved):
        """the norms between block i - 1 and block i (or the output)"""
        before = self.blocks[i - 1] if i else None
        w_pre = self.blocks[i].pre if i < len(self.blocks) else self.last
        post, gate = (before.post, before.gate) if before else (self.ones, self.none)
        h, z, rstd, y8, h8, z8 = gl.galore_norm_block(x, y, post, w_pre, gate, alpha=self.alpha, checkpoints=saved)
        return h, z, (post, w_pre, gate, rstd, y8, h8), z8

    def forward(self, x, saved=True):
        """(output, what the backward pass needs)"""
        kept, y = [], x
        for i, b in enumerate(self.blocks):
            b.w1.quantize()
            b.w2.quantize()
            x, z, norm, z8 = self._norm(i, x, y, saved)
            a = torch.relu(b.w1.forward(z))
            a8, on = (gl.galore_checkpoint_pack(a), pack_positive(a)) if saved else (None, None)
            y = b.w2.forward(a)
            kept.append((norm, z8, a8, on))
        _, z, norm, _ = self._norm(len(self.blocks), x, y, saved)
        return z, (kept, norm)

    def backward(self, dz, saved, tau, lr):
        """steps every weight; the gradient of the input is not asked for"""
        kept, norm = saved
        dh = None
        for i in range(len(self.blocks), 0, -1):
            b = self.blocks[i - 1]
            dh, dy = self._norm_step(dz, dh, norm, lr)
            norm, z8, a8, on = kept[i - 1]
            da = b.w2.data_gradient(dy).masked_fill_(~unpack_positive(on, b.w2.w.shape[1]), 0)
            dz = b.w1.data_gradient(da)
            b.w2.step(dy, a8, tau, lr)
            b.w1.step(da, z8, tau, lr)
        self._norm_step(dz, dh, norm, lr)

    def _norm_step(self, dz, dh, norm, lr):
        post, w_pre, gate, rstd, y8, h8 = norm
        dx, dy, dgate, dpost, dpre = gl.galore_norm_block_backward(dz, dh, h8, y8, rstd, post, w_pre, gate, alpha=self.alpha)
        w_pre -= lr * dpre / (dpre.norm() + 1e-12)
        if gate is not self.none:                    # vectors: normalised gradient steps
            post -= lr * dpost / (dpost.norm() + 1e-12)
            gate -= lr * dgate / (dgate.norm() + 1e-12)
        return dx, dy


def train(steps, tokens=1024, d=512, hidden=1376, blocks=4, rank=64, lr=0.01, seed=0):
    """losses of `steps` steps, each on new tokens"""
    model, teacher = Model(d, hidden, blocks, rank, seed), Model(d, hidden, blocks, rank, seed + 1)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 2)
    losses = []
    for tau in range(steps):
        x = torch.randn((tokens, d), generator=g, device="cuda").bfloat16()
        target = teacher.forward(x, saved=False)[0].float()
        out, saved = model.forward(x)
        diff = out.float() - target
        losses.append((diff ** 2).mean())
        model.backward((2.0 / diff.numel() * diff).bfloat16(), saved, tau, lr)
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=1024)
    a = ap.parse_args()
    for step, loss in enumerate(train(a.steps, a.tokens)):
        if step % 10 == 0 or step == a.steps - 1:
            print("step %d loss %.5f" % (step, loss), flush=True)
