"""Which form of a training operator's kernel a call takes, each form against the
others, offsets past 32 bits, and the operators together in a training step."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import test_training_ops as ops
import training_oracle as ora
from test_training_ops import check_grad, check_product, checkpoint, codes4, host, values

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_20437_amd", "csrc")

SHIM = """
#include "dispatch.hpp"
using namespace galore;
extern "C" {
int few_rows_(long M, long N, long K) { return mx4_few_rows(M, N, K); }
int tile_(long M, long N, long b) { return mx4_tile(M, N, b); }
int wide_(long T, long m, long n, long b, long ok, long fp32) { return weight_grad_plan(T, m, n, b, ok, fp32).wide; }
int splits_(long T, long m, long n, long b, long ok, long fp32) { return weight_grad_plan(T, m, n, b, ok, fp32).splits; }
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    src, out = str(d / "shim.cpp"), str(d / "librules.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
    lib = ctypes.CDLL(out)
    return lambda name, *a: getattr(lib, name + "_")(*[ctypes.c_long(v) for v in a])


@pytest.fixture(scope="module")
def gl():
    import paper_2504_20437_amd
    return paper_2504_20437_amd


# ---- rules (CPU) ------------------------------------------------------------------------


@pytest.mark.parametrize("m,n,k,few", [(1, 11008, 4096, 1), (8, 11008, 4096, 1), (16, 11008, 4096, 0), (32, 4096, 4096, 1),
                                       (33, 64, 64, 0), (32, 64, 64, 1)])
def test_few_rows(rule, m, n, k, few):
    assert rule("few_rows", m, n, k) == few


@pytest.mark.parametrize("m,n,batch,tile", [(8192, 11008, 1, 0), (4096, 4096, 1, 0), (4096, 4096 - 256, 1, 1), (2048, 2048, 1, 1),
                                            (512, 4096, 1, 2), (64, 64, 1, 2), (256, 256, 256, 0)])
def test_product_tiles(rule, m, n, batch, tile):
    assert rule("tile", m, n, batch) == tile


@pytest.mark.parametrize("t,m,n,ok,fp32,wide,splits", [
    (8192, 11008, 4096, 1, 0, 1, 1), (4096, 2048, 5461, 1, 0, 1, 1), (8192, 1024, 2736, 1, 0, 1, 5),
    (8192, 512, 1376, 1, 0, 1, 10), (256, 512, 1376, 1, 0, 0, 1), (1, 512, 1376, 1, 0, 0, 1), (509, 2048, 5461, 1, 1, 0, 1),
    (1024, 4096, 4096, 1, 1, 1, 1), (8192, 1024, 2736, 1, 1, 1, 2), (8192, 512, 1376, 1, 1, 1, 10),
    (1000, 1024, 1024, 1, 1, 0, 4), (0, 64, 64, 0, 0, 0, 1)])
def test_weight_grad_plan(rule, t, m, n, ok, fp32, wide, splits):
    assert rule("wide", t, m, n, 1, ok, fp32) == wide
    assert rule("splits", t, m, n, 1, ok, fp32) == splits


def test_weight_grad_workspace_holds_every_plan(rule, gl):
    for t in (1, 33, 300, 2000, 9000):
        for m, n in ((64, 64), (136, 100), (512, 1376), (2048, 2048)):
            need = gl.galore_checkpoint_weight_grad_workspace_size(t, m, n)
            for ok, fp32 in ((1, 0), (0, 0), (1, 1), (0, 1)):
                s = rule("splits", t, m, n, 1, ok and t >= 32, fp32)
                assert s == 1 or need >= 4 * s * m * n


# ---- forms against the definition ----------------------------------------------------------


@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,m,n,dy,split", [(4000, 1032, 1290, "bf16", 1), (4001, 1030, 1300, "bf16", 1),
                                            (4090, 1290, 1032, "bf16", 1), (3000, 1021, 2700, "f32", 1),
                                            (1025, 4090, 2040, "f32", 0), (1030, 4091, 2030, "f32", 0)])
def test_wide_weight_grad(rule, gl, t, m, n, dy, split, out):
    """wide tiles, with the tokens split and not, the last stage, the last split and the last columns ragged"""
    fp32 = dy == "f32"
    assert rule("wide", t, m, n, 1, 1, fp32) and (rule("splits", t, m, n, 1, 1, fp32) > 1) == split
    g, x = values(t, m, dy, 1, "gradients"), values(t, n, "f32", 2)
    q = checkpoint(x)
    start = torch.randn((m, n), generator=torch.Generator().manual_seed(3)).to(out)
    G = start.cuda()
    gl.galore_checkpoint_weight_grad(g.cuda(), *q, n, G=G, accumulate=True)
    check_grad(G, host(g), ora.mx8_decode(host(q[0]), host(q[1]), n), host(start))


@pytest.mark.gpu
@pytest.mark.parametrize("t", [4000, 4001])
def test_wide_weight_grad_last_word(rule, gl, t):
    """an odd number of gradients in rows on 4 bytes: the last word of the last token holds one of them"""
    m, n = 1031, 1300
    assert rule("wide", t, m, n, 1, 1, 0)
    g, x = values(t, m, "bf16", 1, "gradients"), values(t, n, "f32", 2)
    g[-1] = 3.0                                                     # the last token counts
    dy = torch.full((t, m + 1), float("nan"), dtype=torch.bfloat16, device="cuda")[:, :m]
    dy.copy_(g)
    q = checkpoint(x)
    G = gl.galore_checkpoint_weight_grad(dy, *q, n, dtype=torch.float32)
    check_grad(G, host(g), ora.mx8_decode(host(q[0]), host(q[1]), n), np.zeros((m, n)))


@pytest.mark.gpu
@pytest.mark.parametrize("t,m,n", [(64, 4088, 4000), (65, 4086, 4000), (95, 4088, 4000), (97, 4090, 3990)])
def test_wide_weight_grad_few_tokens(rule, gl, t, m, n):
    assert rule("wide", t, m, n, 1, 1, 0)
    g, x = values(t, m, "bf16", t, "gradients"), values(t, n, "f32", 2)
    x[t - 1, 40] = float("nan")                       # in the last token: one block of columns
    q = checkpoint(x)
    G = host(gl.galore_checkpoint_weight_grad(g.cuda(), *q, n, dtype=torch.float32))
    xh = ora.mx8_decode(host(q[0]), host(q[1]), n)
    assert np.isnan(G[:, 32:64]).all()
    keep = np.r_[0:32, 64:n]
    check_grad(torch.from_numpy(G[:, keep]), host(g), xh[:, keep])


@pytest.mark.gpu
def test_wide_weight_grad_batched(rule, gl):
    t, m, n, b = 70, 2048, 1100, 6
    assert rule("wide", t, m, n, b, 1, 0)
    g = torch.stack([values(t, m, "bf16", i, "gradients") for i in range(b)])
    pairs = [checkpoint(values(t, n, "f32", 20 + i)) for i in range(b)]
    G = gl.galore_checkpoint_weight_grad(g.cuda(), torch.stack([p[0] for p in pairs]), torch.stack([p[1] for p in pairs]), n)
    for i in (0, 3, b - 1):
        check_grad(G[i], host(g[i]), ora.mx8_decode(*map(host, pairs[i]), n))


@pytest.mark.gpu
@pytest.mark.parametrize("k", [32, 64, 224, 256, 257, 512, 513, 768, 1000])
def test_wide_product_depths(gl, k):
    """one stage, two, three and ragged ones, with what lies behind a row's end the NaN byte"""
    m, n = 4096, 4104
    a, b = codes4(values(m, k, "f32", 1)), codes4(values(n, k, "f32", 2))
    nb = (k + 31) // 32
    a[1][:, nb:] = 255
    b[1][:, nb:] = 255
    C = gl.galore_mx4_matmul(*a, *b, k, dtype=torch.float32)
    ah, bh = ora.mx4_decode(host(a[0]), host(a[1]), k), ora.mx4_decode(host(b[0]), host(b[1]), k)
    rows, cols = np.r_[0:40, 2000:2040, m - 40:m], np.r_[0:40, 3000:3040, n - 40:n]
    check_product(C[torch.from_numpy(rows).cuda()][:, torch.from_numpy(cols).cuda()], ah[rows], bh[cols])


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(1200, 700), (4096, 4096)])
def test_product_forms_agree_on_integers(gl, m, n):
    """small integers are exact in every form: the tiles, the rows of B in registers, and fp32 sums in any order"""
    k = 640
    g = torch.Generator().manual_seed(5)
    x, y = (torch.tensor([0., 1, -1, 2, -2, 3, 4, 6])[torch.randint(0, 8, (r, k), generator=g)] for r in (m, n))
    a, b = codes4(x), codes4(y)
    want = x.cuda() @ y.t().cuda()
    assert torch.equal(gl.galore_mx4_matmul(*a, *b, k, dtype=torch.float32), want)
    for rows in (1, 16, 17, 32, 33, 64, 65, 300):
        assert torch.equal(gl.galore_mx4_matmul(a[0][:rows], a[1][:rows], *b, k, dtype=torch.float32), want[:rows])


# ---- offsets past 32 bits -----------------------------------------------------------------


def stretched(t, pitch):
    """the same rows at a long pitch (bytes past 4 GiB from the first to the last)"""
    big = torch.empty((t.shape[0], pitch), dtype=t.dtype, device="cuda")
    big[:, :t.shape[1]] = t
    return big[:, :t.shape[1]]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_codes_past_32_bits(gl, dtype):
    rows, cols = 300, 200
    x = values(rows, cols, dtype, 1).cuda()
    far = stretched(x, 1 << 23)                       # 300 x 2^23 elements
    q, want = gl.galore_checkpoint_pack(far), gl.galore_checkpoint_pack(x)
    assert all(torch.equal(a, b) for a, b in zip(q, want))
    for a, b in zip(gl.galore_mx4_quantize(far, columns=True), gl.galore_mx4_quantize(x, columns=True)):
        assert torch.equal(a, b)
    del far
    fq = (stretched(q[0], 1 << 24), stretched(q[1], 1 << 22))
    assert torch.equal(gl.galore_checkpoint_unpack(*fq, cols, dtype=torch.float32),
                       gl.galore_checkpoint_unpack(*q, cols, dtype=torch.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(72, 200), (4096, 4096)])
def test_weight_grad_past_32_bits(gl, dtype, m, n):
    t = 520
    g, x = values(t, m, dtype, 1, "gradients").cuda(), values(t, n, "f32", 2)
    q = checkpoint(x)
    want = gl.galore_checkpoint_weight_grad(g, *q, n, dtype=torch.float32)
    far = stretched(g, 1 << 22)
    fq = (stretched(q[0], 1 << 23), stretched(q[1], 1 << 23))
    assert torch.equal(gl.galore_checkpoint_weight_grad(far, *fq, n, dtype=torch.float32), want)
    G = stretched(torch.zeros_like(want), 1 << 21)
    gl.galore_checkpoint_weight_grad(g, *q, n, G=G)
    assert torch.equal(G, want)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(20, 1100), (300, 1100), (4096, 4096)])
def test_product_past_32_bits(gl, m, n):
    k = 300
    a, b = codes4(values(m, k, "f32", 1)), codes4(values(n, k, "f32", 2))
    want = gl.galore_mx4_matmul(*a, *b, k, dtype=torch.float32)
    pitch = 1 << 22 if n == 1100 else 1 << 21         # past and below the wide kernel's limit of pitches
    fb = (stretched(b[0], pitch), stretched(b[1], pitch))
    assert torch.equal(gl.galore_mx4_matmul(*a, *fb, k, dtype=torch.float32), want)
    fa = [stretched(v, pitch) for v in a]
    assert torch.equal(gl.galore_mx4_matmul(*fa, *b, k, dtype=torch.float32), want)


@pytest.mark.gpu
def test_norms_past_32_bits(gl):
    t, d = 600, 300
    x, y = values(t, d, "bf16", 1).cuda(), values(t, d, "bf16", 2).cuda()
    w = torch.ones(d, device="cuda")
    H, Z, R, y8, h8, _ = gl.galore_norm_block(x, y, w, w, checkpoints=True)
    fx = stretched(x, 1 << 22)
    out = stretched(torch.zeros_like(x), 1 << 22)
    FH, FZ, FR, *_ = gl.galore_norm_block(fx, y, w, w, H=fx, Z=out)
    assert torch.equal(FH, H) and torch.equal(FZ, Z) and torch.equal(FR, R)
    dz = values(t, d, "bf16", 3).cuda()
    want = gl.galore_norm_block_backward(dz, x, H, y, R, w, w)
    got = gl.galore_norm_block_backward(stretched(dz, 1 << 22), x, FH, y, R, w, w, dX=out)
    assert all(torch.equal(a, b) for a, b in zip((got[0], got[1], got[3], got[4]), (want[0], want[1], want[3], want[4])))


# ---- together ------------------------------------------------------------------------------


@pytest.mark.gpu
def test_training_step_learns():
    """the example's loss: each step's tokens are new, so that it falls only if the gradients are right"""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import lean_training
    losses = lean_training.train(40, tokens=512, d=256, hidden=688, blocks=2, rank=32)
    assert all(np.isfinite(losses))
    assert np.mean(losses[-5:]) < 0.6 * losses[0]


@pytest.mark.gpu
def test_training_gradients_against_autograd(gl):
    """one linear layer between two norms, from the 4-bit operands and 8-bit checkpoints that the operators used:
    autograd in 64 bits on the same values gives the same gradients"""
    t, d = 96, 160
    g = torch.Generator().manual_seed(0)
    x, y0 = (torch.randn((t, d), generator=g).bfloat16().cuda() for _ in range(2))
    w = (torch.randn((d, d), generator=g) / d ** 0.5).cuda()
    ones = torch.ones(d, device="cuda")
    h, z, r1, y8, h8, z8 = gl.galore_norm_block(x, y0, ones, ones, checkpoints=True)
    wq = gl.galore_mx4_quantize(w, columns=True)
    zq = gl.galore_mx4_quantize(z)
    y = gl.galore_mx4_matmul(*zq, *wq[:2], d)
    dy = (1e-2 * torch.randn((t, d), generator=g)).bfloat16().cuda()
    G = gl.galore_checkpoint_weight_grad(dy, *z8, d, dtype=torch.float32)
    dz = gl.galore_mx4_matmul(*gl.galore_mx4_quantize(dy), *wq[2:], d)
    # the forward value, and the gradients, of the decoded operands
    zd = gl.galore_mx4_dequantize(*zq, d, dtype=torch.float32).double()
    wr = gl.galore_mx4_dequantize(*wq[:2], d, dtype=torch.float32).double()
    wc = gl.galore_mx4_dequantize(*wq[2:], d, dtype=torch.float32).double().t()
    z8d = gl.galore_checkpoint_unpack(*z8, d, dtype=torch.float32).double().requires_grad_()
    wv = wr.clone().requires_grad_()
    (z8d @ wv.t() * dy.double()).sum().backward()
    size = dy.double().abs().t() @ z8d.detach().abs()
    assert ((G.double() - wv.grad).abs() <= (t + 4) * 2.0 ** -24 * size).all()
    assert ((y.double() - zd @ wr.t()).abs() <= 2.0 ** -8 * (zd.abs() @ wr.abs().t())).all()
    dq = gl.galore_mx4_dequantize(*gl.galore_mx4_quantize(dy), d, dtype=torch.float32).double()
    assert ((dz.double() - dq @ wc).abs() <= 2.0 ** -8 * (dq.abs() @ wc.abs())).all()


@pytest.mark.gpu
@pytest.mark.parametrize("gate", ["none", "vector", "tokens"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,d", [(530, 2731), (520, 6000), (513, 8200)])
def test_norm_backward_walks_over_wide_rows(gl, t, d, dtype, gate):
    """several rows to a workgroup in the forms of wide rows: the next row held, read when it is due, vectors read again"""
    ops.test_norm_block_backward(gl, t, d, dtype, gate)


@pytest.mark.gpu
@pytest.mark.parametrize("t", [1, 1500])
def test_graph_replays(gl, t):
    """the operators in a graph: every replay, with eager work between, equals the calls themselves on its inputs"""
    m, n = 256, 288
    gen = torch.Generator(device="cuda").manual_seed(t)

    def new(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)

    x, y, dz, dy = new(t, n), new(t, n), new(t, n), new(t, m)
    wo, wp, gate, weight = new(n, dtype=torch.float32), new(n, dtype=torch.float32), new(n, dtype=torch.float32), new(m, n)

    def step():
        h, z, rstd, y8, h8, z8 = gl.galore_norm_block(x, y, wo, wp, gate, checkpoints=True)
        w, ws, wt, wts = gl.galore_mx4_quantize(weight, columns=True)
        out = gl.galore_mx4_matmul(*gl.galore_mx4_quantize(z), w, ws, n)
        dx = gl.galore_mx4_matmul(*gl.galore_mx4_quantize(dy), wt, wts, m)
        g = gl.galore_checkpoint_weight_grad(dy, *z8, n, dtype=torch.float32)
        return [h, z, out, dx, g, gl.galore_checkpoint_unpack(*z8, n),
                *gl.galore_norm_block_backward(dz, dx, h8, y8, rstd, wo, wp, gate)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(4):
        for v in (x, y, dz, dy):
            v.copy_(new(*v.shape))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in held]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
