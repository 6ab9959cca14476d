"""8-bit checkpoints, the weight gradient from them, 4-bit products and the norms
of a block, against the plain 64-bit forms of training_oracle.

Tolerances. U = 2^-24 is the largest relative rounding error of fp32, B = 2^-8 of bfloat16. Codes, scales
and decoded values are exact. A sum of K products in fp32, in any order, is off by
at most about K U of the sum of their magnitudes; a result rounded to bfloat16 by B
of itself more."""
import numpy as np
import pytest
import torch

import training_oracle as ora

U, B = 2.0 ** -24, 2.0 ** -8
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def gl():
    import paper_2504_20437_amd
    return paper_2504_20437_amd


def host(t):
    return t.detach().cpu().double().numpy() if t.dtype.is_floating_point else t.detach().cpu().numpy()


def values(rows, cols, dtype, seed, kind="activations"):
    """a CPU tensor of `dtype`; tokens of unequal size, some of them zero"""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g) * torch.exp(2 * torch.randn((rows, 1), generator=g))
    if rows > 3:
        x[rows // 2] = 0
        x[1, : cols // 2] = 0
    if kind == "gradients":
        x *= 1e-4
    return x.to(DTYPES[dtype])


def place(x, pad=0, offset=0):
    """x on the GPU in rows of a longer pitch that start `offset` elements in, the rest NaN"""
    if not pad and not offset:
        return x.cuda()
    big = torch.full((x.shape[0], x.shape[1] + pad + offset), float("nan"), dtype=x.dtype, device="cuda")
    big[:, offset:offset + x.shape[1]] = x.cuda()
    return big[:, offset:offset + x.shape[1]]


def checkpoint(x):
    """codes and scales of a CPU tensor, on the GPU, by the oracle"""
    c, s = ora.mx8_encode(host(x))
    return torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()


# ---- the oracle itself (CPU) ----------------------------------------------------------


def test_oracle_codes_by_hand():
    x = np.zeros((1, 33))
    x[0, :4] = [127.0, -126.5, 0.5, 1.5]          # unit 1: ties to even
    x[0, 32] = 128.0                              # unit 2
    c, s = ora.mx8_encode(x)
    assert c[0, :4].tolist() == [127, -126, 0, 2] and c[0, 32] == 64
    assert s.tolist() == [[133, 134, 0, 0]]
    x = np.zeros((1, 40))
    x[0, :8] = [6, -5, 3.5, 2.5, 0.25, 0.75, -0.2, 1.25]
    x[0, 32] = 6.1
    c, s = ora.mx4_encode(x)
    assert s.tolist() == [[127, 128, 0, 0]]
    assert ora.mx4_decode(c, s, 40)[0, :8].tolist() == [6, -4, 4, 2, 0, 1, 0, 1]
    assert ora.mx4_decode(c, s, 40)[0, 32] == 6


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(0)
    t, d, alpha, eps = 5, 7, 0.7, 1e-3
    x, y, a, b = (rng.standard_normal((t, d)) for _ in range(4))
    w_post, w_pre, gate = (rng.standard_normal(d) + 1.5 for _ in range(3))
    p = [x, y, gate, w_post, w_pre]

    def loss():
        h, z, _ = ora.norms(x, y, w_post, w_pre, gate, alpha, eps)
        return (h * a).sum() + (z * b).sum()
    h, _, rstd = ora.norms(x, y, w_post, w_pre, gate, alpha, eps)
    dx, dy, dg, dwo, dwp = ora.norms_backward(b, a, h, y, rstd, w_post, w_pre, gate, alpha)
    for v, grad in zip(p, (dx, dy, dg.sum(0), dwo, dwp)):
        for i in np.ndindex(v.shape):
            keep, step = v[i], 1e-5
            v[i] = keep + step
            up = loss()
            v[i] = keep - step
            down = loss()
            v[i] = keep
            # central differences: truncation of order step^2, rounding of 1e-16 / step
            assert abs((up - down) / (2 * step) - grad[i]) < 1e-7 * (1 + abs(grad[i]))


# ---- refusals (CPU: nothing is enqueued) ----------------------------------------------


FAKE = 0x10000


def struct(gl, **kw):
    from paper_2504_20437_amd.training import MxMatrix
    a = dict(codes=FAKE, ldq=1024, stride_q=1 << 20, scales=FAKE, lds=64, stride_s=1 << 16)
    a.update(kw)
    return MxMatrix(a["codes"], a["ldq"], a["stride_q"], a["scales"], a["lds"], a["stride_s"])


BAD_STRUCTS = [(dict(codes=None), -1), (dict(scales=None), -1), (dict(codes=FAKE + 8), -1), (dict(scales=FAKE + 2), -1),
               (dict(ldq=1000), -2), (dict(ldq=16), -2), (dict(lds=62), -2), (dict(lds=0), -2),
               (dict(stride_q=16), -2), (dict(stride_s=4), -2), (dict(stride_q=(1 << 20) + 8), -2),
               (dict(stride_s=(1 << 16) + 2), -2)]


@pytest.mark.parametrize("kw,code", BAD_STRUCTS)
def test_struct_rejects(gl, kw, code):
    bad, ok = struct(gl, **kw), struct(gl)
    lib = gl.lib
    assert lib.galore_checkpoint_pack(FAKE, 0, 64, 200, 200, 64 * 200, bad, 2, None) == code
    assert lib.galore_checkpoint_unpack(bad, 64, 200, FAKE, 0, 200, 64 * 200, 2, None) == code
    assert lib.galore_checkpoint_weight_grad(FAKE, 0, 96, 64 * 96, bad, 64, 96, 200, FAKE, 0, 200, 96 * 200, 0, 2, None,
                                             0, None) == code
    assert lib.galore_mx4_quantize(FAKE, 0, 64, 200, 200, 64 * 200, bad, None, 2, None) == code
    assert lib.galore_mx4_quantize(FAKE, 0, 200, 64, 64, 64 * 200, None, struct(gl, **dict(kw)), 2, None) == code
    assert lib.galore_mx4_dequantize(bad, 64, 200, FAKE, 0, 200, 64 * 200, 2, None) == code
    assert lib.galore_mx4_matmul(bad, ok, 64, 96, 200, FAKE, 0, 96, 64 * 96, 2, None) == code
    assert lib.galore_mx4_matmul(ok, bad, 64, 96, 200, FAKE, 0, 96, 64 * 96, 2, None) == code


def test_checkpoint_rejects(gl):
    lib, ok = gl.lib, struct(gl)
    assert lib.galore_checkpoint_pack(None, 0, 64, 200, 200, 0, ok, 1, None) == -1
    assert lib.galore_checkpoint_pack(FAKE, 2, 64, 200, 200, 0, ok, 1, None) == -1
    assert lib.galore_checkpoint_pack(FAKE, 0, 64, 200, 200, 0, None, 1, None) == -1
    for rows, cols, ld, st, batch in ((-1, 200, 200, 0, 1), (64, 0, 200, 0, 1), (64, 200, 199, 0, 1), (64, 200, 200, 0, 0),
                                      (64, 200, 200, 64 * 200 - 1, 2), (64, 200, 200, 1 << 30, 65536),
                                      ((1 << 28) + 1, 200, 200, 0, 1), (64, (1 << 28) + 1, 1 << 29, 0, 1)):
        assert lib.galore_checkpoint_pack(FAKE, 0, rows, cols, ld, st, ok, batch, None) == -2
        assert lib.galore_checkpoint_unpack(ok, rows, cols, FAKE, 0, ld, st, batch, None) == -2
        assert lib.galore_mx4_quantize(FAKE, 0, rows, cols, ld, st, ok, None, batch, None) == -2
        assert lib.galore_mx4_dequantize(ok, rows, cols, FAKE, 0, ld, st, batch, None) == -2
    assert lib.galore_mx4_quantize(FAKE, 0, 64, 200, 200, 0, None, None, 1, None) == -1
    # no tokens: nothing to do, no pointers needed
    assert lib.galore_checkpoint_pack(None, 0, 0, 200, 200, 0, struct(gl, codes=None, scales=None), 1, None) == 0
    assert lib.galore_mx4_matmul(struct(gl, codes=None, scales=None), ok, 0, 96, 200, None, 0, 96, 0, 1, None) == 0


def test_weight_grad_rejects(gl):
    def call(dy=FAKE, dt=0, ldy=96, t=64, m=96, n=200, g=FAKE, gt=0, ldg=200, batch=1, ws=None, wb=0):
        return gl.lib.galore_checkpoint_weight_grad(dy, dt, ldy, 0, struct(gl), t, m, n, g, gt, ldg, 0, 0, batch, ws, wb, None)
    assert call(dy=None) == -1 and call(g=None) == -1 and call(dt=5) == -1 and call(gt=-1) == -1
    assert call(ldy=95) == -2 and call(ldg=199) == -2 and call(m=0) == -2 and call(n=0) == -2 and call(t=-1) == -2
    assert call(ws=FAKE + 1, wb=1 << 30) == -3
    need = gl.galore_checkpoint_weight_grad_workspace_size(8192, 96, 200)
    assert need > 0 and call(t=8192, ws=FAKE, wb=need - 1) == -3
    assert gl.galore_checkpoint_weight_grad_workspace_size(8192, 11008, 4096) == 0
    assert gl.galore_checkpoint_weight_grad_workspace_size(0, 96, 200) == 0


def test_matmul_rejects(gl):
    def call(m=64, n=96, k=200, c=FAKE, ct=0, ldc=96, batch=1):
        return gl.lib.galore_mx4_matmul(struct(gl), struct(gl), m, n, k, c, ct, ldc, 0, batch, None)
    assert call(c=None) == -1 and call(ct=3) == -1
    assert call(m=-1) == -2 and call(n=0) == -2 and call(k=0) == -2 and call(ldc=95) == -2 and call(batch=0) == -2


def test_norm_rejects(gl):
    def fwd(x=FAKE, ldx=64, y=FAKE, dt=0, wo=FAKE, wp=FAKE, gate=FAKE, ldg=64, mode=1, alpha=1.0, eps=1e-5, t=8, d=64,
            h=FAKE, z=FAKE, ldz=64, r=FAKE, y8=None):
        return gl.lib.galore_norm_block(x, ldx, y, 64, dt, wo, wp, gate, ldg, mode, alpha, eps, t, d, h, 64, z, ldz, r, y8,
                                        None, None, None)
    for kw in (dict(x=None), dict(y=None), dict(dt=2), dict(wo=None), dict(wp=None), dict(gate=None), dict(mode=3),
               dict(mode=-1), dict(alpha=float("nan")), dict(eps=0.0), dict(eps=float("inf")), dict(h=None), dict(z=None),
               dict(r=None), dict(y8=struct(gl, codes=None)), dict(mode=2, gate=None)):
        assert fwd(**kw) == -1, kw
    for kw in (dict(ldx=63), dict(ldz=63), dict(t=-1), dict(d=0), dict(d=16385, ldx=1 << 15, ldz=1 << 15),
               dict(mode=2, ldg=63), dict(y8=struct(gl, ldq=32))):
        assert fwd(**kw) == -2, kw
    need = gl.galore_norm_block_backward_workspace_size(8, 64)

    def bwd(dz=FAKE, h=FAKE, y=FAKE, h8=None, y8=None, r=FAKE, gate=FAKE, dgate=FAKE, mode=1, dx=FAKE, dwo=FAKE, ws=FAKE,
            wb=need, lddx=64, alpha=1.0):
        return gl.lib.galore_norm_block_backward(dz, 64, None, 0, 0, h, 64, y, 64, h8, y8, r, FAKE, FAKE, gate, 64, mode,
                                                 alpha, 8, 64, dx, lddx, FAKE, 64, dgate, 64, dwo, FAKE, ws, wb, None)
    for kw in (dict(dz=None), dict(h=None), dict(y=None), dict(h8=struct(gl)), dict(h8=struct(gl), y8=struct(gl)),
               dict(r=None), dict(gate=None), dict(dgate=None), dict(mode=7), dict(dx=None), dict(dwo=None),
               dict(alpha=float("inf"))):
        assert bwd(**kw) == -1, kw
    assert bwd(lddx=63) == -2
    for kw in (dict(ws=None), dict(ws=FAKE + 8), dict(wb=need - 1)):
        assert bwd(**kw) == -3, kw
    assert gl.galore_norm_block_backward_workspace_size(0, 64) == 0
    assert gl.galore_norm_block_backward_workspace_size(8, 16385) == 0


def test_binding_rejects(gl):
    """before any device access"""
    x = torch.zeros((4, 64))
    for call in (lambda: gl.galore_checkpoint_pack(x), lambda: gl.galore_mx4_quantize(x),
                 lambda: gl.galore_checkpoint_pack(x.double()), lambda: gl.galore_checkpoint_pack(x[0]),
                 lambda: gl.galore_checkpoint_unpack(x.to(torch.int8), x, 64),
                 lambda: gl.galore_mx4_matmul(x, x, x, x, 64),
                 lambda: gl.galore_checkpoint_weight_grad(x, x, x, 64),
                 lambda: gl.galore_norm_block(x, x, x[0], x[0]),
                 lambda: gl.galore_norm_block_backward(x, None, x, x, x, x[0], x[0])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_binding_rejects_mismatched_tensors(gl):
    x = torch.zeros((6, 70), device="cuda")
    codes, scales = gl.galore_checkpoint_pack(x)
    w = torch.ones(70, device="cuda")
    r = torch.ones((6, 2), device="cuda")
    for call in (lambda: gl.galore_checkpoint_unpack(codes, scales, 97),
                 lambda: gl.galore_checkpoint_unpack(codes.cpu(), scales, 70),
                 lambda: gl.galore_checkpoint_unpack(codes, scales[:, :2], 70),
                 lambda: gl.galore_checkpoint_unpack(codes, scales, 70, dtype=torch.float16),
                 lambda: gl.galore_checkpoint_pack(x.t()),
                 lambda: gl.galore_checkpoint_pack(x, out=(codes.to(torch.uint8), scales)),
                 lambda: gl.galore_checkpoint_weight_grad(x[:5], codes, scales, 70),
                 lambda: gl.galore_checkpoint_weight_grad(x, codes, scales, 70, accumulate=True),
                 lambda: gl.galore_checkpoint_weight_grad(x, codes, scales, 70, G=torch.zeros((70, 71), device="cuda")),
                 lambda: gl.galore_checkpoint_weight_grad(x, codes, scales, 70, workspace=torch.zeros(8)),
                 lambda: gl.galore_mx4_quantize(x, rows=False, columns=False),
                 lambda: gl.galore_norm_block(x, x, w[:-1], w),
                 lambda: gl.galore_norm_block(x, x.bfloat16(), w, w),
                 lambda: gl.galore_norm_block(x, x, w, w, gate=w.bfloat16()),
                 lambda: gl.galore_norm_block_backward(x, None, x, (codes, scales), r, w, w),
                 lambda: gl.galore_norm_block_backward(x, None, x, x, r[:, :1], w, w),
                 lambda: gl.galore_norm_block_backward(x, None, x, x, r, w, w, dgate=w)):
        with pytest.raises(ValueError):
            call()


# ---- codes ------------------------------------------------------------------------------


SHAPES = [(1, 1), (1, 31), (3, 32), (2, 33), (5, 128), (130, 100), (64, 257), (7, 4096), (200, 513), (33, 5461)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_checkpoint_codes(gl, rows, cols, dtype):
    x = values(rows, cols, dtype, rows + cols)
    for pad, offset in ((0, 0), (5, 1)):
        codes, scales = gl.galore_checkpoint_pack(place(x, pad, offset))
        c, s = ora.mx8_encode(host(x))
        assert np.array_equal(host(scales), s)
        assert np.array_equal(host(codes), c)
        for out in ("f32", "bf16"):
            assert np.array_equal(host(gl.galore_checkpoint_unpack(codes, scales, cols, dtype=DTYPES[out])),
                                  ora.mx8_decode(c, s, cols))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES + [(128, 128), (129, 127), (4096, 7)])
def test_mx4_codes(gl, rows, cols, dtype):
    x = values(rows, cols, dtype, rows * cols)
    row = [torch.from_numpy(v) for v in ora.mx4_encode(host(x))]
    col = [torch.from_numpy(v) for v in ora.mx4_encode(host(x).T)]
    for pad, offset in ((0, 0), (3, 1)):
        xd = place(x, pad, offset)
        got = [t.cpu() for t in gl.galore_mx4_quantize(xd)]
        both = [t.cpu() for t in gl.galore_mx4_quantize(xd, columns=True)]
        only = [t.cpu() for t in gl.galore_mx4_quantize(xd, rows=False, columns=True)]
        for a, b in zip(got + both + only, row + row + col + col):
            assert torch.equal(a, b)
    for out in ("f32", "bf16"):
        back = gl.galore_mx4_dequantize(both[0].cuda(), both[1].cuda(), cols, dtype=DTYPES[out])
        assert np.array_equal(host(back), ora.mx4_decode(*[t.numpy() for t in row], cols))


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_code_edges(gl, bits, dtype):
    """ties, signed zeros, blocks on both sides of a power of two, the type's ends, subnormals, NaN and Inf"""
    big = torch.finfo(DTYPES[dtype]).max
    rows = [[0.0, -0.0], [1.0], [127.0, 126.5, 0.5, 1.5, -2.5], [127.5, 1], [6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25],
            [6.0625, 1], [big, -big], [big / 2, 1.0], [2.0 ** -120, 2.0 ** -126], [2.0 ** -126], [1e-40, -1e-44], [1e-30, 1e30],
            [float("nan"), 1.0], [float("inf"), 2.0], [-float("inf")], [3.0 * 2.0 ** -124, 2.0 ** -124]]
    x = torch.zeros((len(rows), 70))
    for i, r in enumerate(rows):
        x[i, 32:32 + len(r)] = torch.tensor(r)
        x[i, 69] = 1.0
    x = x.to(DTYPES[dtype])
    xh = host(x)
    if bits == 8:
        c, s = ora.mx8_encode(xh)
        codes, scales = gl.galore_checkpoint_pack(x.cuda())
        back, want = gl.galore_checkpoint_unpack(codes, scales, 70, dtype=torch.float32), ora.mx8_decode(c, s, 70)
    else:
        c, s = ora.mx4_encode(xh)
        codes, scales = gl.galore_mx4_quantize(x.cuda())
        back, want = gl.galore_mx4_dequantize(codes, scales, 70, dtype=torch.float32), ora.mx4_decode(c, s, 70)
        ct, st = ora.mx4_encode(xh.T)
        tc, ts = gl.galore_mx4_quantize(x.cuda(), rows=False, columns=True)
        assert np.array_equal(host(tc), ct) and np.array_equal(host(ts), st)
    assert np.array_equal(host(scales), s) and np.array_equal(host(codes), c)
    assert np.array_equal(host(back), want, equal_nan=True)
    assert np.isnan(host(back)[12, 32:64]).all() and np.isfinite(host(back)[12, :32]).all()


@pytest.mark.gpu
def test_decode_any_scale(gl):
    """scale bytes that the encoder does not write are read as what they stand for"""
    scales = torch.arange(256, dtype=torch.uint8).reshape(64, 4)
    c8 = torch.full((64, 128), 3, dtype=torch.int8)
    c4 = torch.full((64, 64), 0x2b, dtype=torch.uint8)      # -1.5, 1
    with np.errstate(over="ignore"):
        want8 = ora.mx8_decode(c8.numpy(), scales.numpy(), 128).astype(np.float32)
        want4 = ora.mx4_decode(c4.numpy(), scales.numpy(), 128).astype(np.float32)
    for dt in (torch.float32, torch.bfloat16):
        got8 = gl.galore_checkpoint_unpack(c8.cuda(), scales.cuda(), 128, dtype=dt).float().cpu().numpy()
        got4 = gl.galore_mx4_dequantize(c4.cuda(), scales.cuda(), 128, dtype=dt).float().cpu().numpy()
        assert np.array_equal(got8, want8, equal_nan=True) and np.array_equal(got4, want4, equal_nan=True)


@pytest.mark.gpu
def test_codes_batched_strided(gl):
    x = torch.stack([values(37, 75, "bf16", i) for i in range(3)])
    room = torch.zeros((3, 40, 128), dtype=torch.int8, device="cuda")
    sroom = torch.full((3, 40, 12), 9, dtype=torch.uint8, device="cuda")
    out = (room[:, :37, :96], sroom[:, :37, :4])
    xd = torch.full((3, 41, 90), float("nan"), dtype=torch.bfloat16, device="cuda")[:, :37, 3:78]
    xd.copy_(x.cuda())
    codes, scales = gl.galore_checkpoint_pack(xd, out=out)
    back = torch.full((3, 38, 77), 7.0, device="cuda")
    gl.galore_checkpoint_unpack(codes, scales, 75, out=back[:, :37, 1:76])
    rows = gl.galore_mx4_quantize(xd, columns=True)
    for b in range(3):
        c, s = ora.mx8_encode(host(x[b]))
        assert np.array_equal(host(codes[b]), c) and np.array_equal(host(scales[b]), s)
        assert np.array_equal(host(back[b, :37, 1:76]), ora.mx8_decode(c, s, 75))
        for got, want in zip(rows, ora.mx4_encode(host(x[b])) + ora.mx4_encode(host(x[b]).T)):
            assert np.array_equal(host(got[b]), want)
    assert (room[:, 37:] == 0).all() and (room[:, :, 96:] == 0).all() and (sroom[:, :, 4:] == 9).all()
    assert (back[:, 37] == 7).all() and (back[:, :, 0] == 7).all() and (back[:, :, 76] == 7).all()


# ---- weight gradient ----------------------------------------------------------------------


GRADS = [(1, 1, 1), (1, 130, 40), (5, 33, 257), (31, 64, 96), (64, 128, 128), (100, 129, 127), (513, 96, 200),
         (2049, 200, 72), (333, 300, 700)]


def check_grad(G, dy, x, start=None):
    """G against dy^T x (+ start) in 64 bits"""
    want = dy.T @ x + (0 if start is None else start)
    tol = (dy.shape[0] + 4) * U * (np.abs(dy).T @ np.abs(x) + (0 if start is None else np.abs(start)))
    if G.dtype == torch.bfloat16:
        tol = tol + B * (np.abs(want) + tol)
    err = np.abs(host(G) - want)
    assert (err <= tol).all(), (err - tol).max()


@pytest.mark.gpu
@pytest.mark.parametrize("dy,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("t,m,n", GRADS)
def test_weight_grad(gl, t, m, n, dy, out):
    g = values(t, m, dy, t + m, "gradients")
    x = values(t, n, "f32", t + n)
    q = checkpoint(x)
    xh = ora.mx8_decode(host(q[0]), host(q[1]), n)
    for pad, offset in ((0, 0), (3, 1)):
        G = gl.galore_checkpoint_weight_grad(place(g, pad, offset), *q, n, dtype=DTYPES[out])
        check_grad(G, host(g), xh)
    # added to what is there, into rows of a longer pitch, and without the workspace
    start = torch.randn((m, n + 3), generator=torch.Generator().manual_seed(1)).to(DTYPES[out])
    room = start.cuda()
    gl.galore_checkpoint_weight_grad(g.cuda(), *q, n, G=room[:, 1:n + 1], accumulate=True)
    check_grad(room[:, 1:n + 1], host(g), xh, host(start[:, 1:n + 1]))
    assert torch.equal(room[:, n + 1:].cpu(), start[:, n + 1:]) and torch.equal(room[:, 0].cpu(), start[:, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("dy", ["bf16", "f32"])
def test_weight_grad_split_agrees(gl, dy):
    """with the tokens split over workgroups and without"""
    t, m, n = 1500, 130, 100
    g, q = values(t, m, dy, 2, "gradients"), checkpoint(values(t, n, "f32", 3))
    assert gl.galore_checkpoint_weight_grad_workspace_size(t, m, n) > 0
    xh = ora.mx8_decode(host(q[0]), host(q[1]), n)
    G = torch.empty((m, n), device="cuda")
    gd = g.cuda()
    check_grad(gl.galore_checkpoint_weight_grad(gd, *q, n, dtype=torch.float32), host(g), xh)
    from paper_2504_20437_amd.training import MxMatrix
    s = MxMatrix(q[0].data_ptr(), q[0].stride(0), 0, q[1].data_ptr(), q[1].stride(0), 0)
    torch.cuda.synchronize()
    assert gl.lib.galore_checkpoint_weight_grad(gd.data_ptr(), 1 if dy == "bf16" else 0, m, 0, s, t, m, n, G.data_ptr(), 0,
                                                n, 0, 0, 1, None, 0, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    check_grad(G, host(g), xh)


@pytest.mark.gpu
def test_weight_grad_large_tiles(gl):
    """the widest tiles of the launch rules, with ragged edges"""
    t, m, n = 70, 3600, 4000
    g, x = values(t, m, "bf16", 4, "gradients"), values(t, n, "f32", 5)
    q = checkpoint(x)
    G = gl.galore_checkpoint_weight_grad(g.cuda(), *q, n, dtype=torch.float32)
    check_grad(G, host(g), ora.mx8_decode(host(q[0]), host(q[1]), n))


@pytest.mark.gpu
def test_weight_grad_batched(gl):
    t, m, n, b = 65, 70, 40, 3
    g = torch.stack([values(t, m, "bf16", i, "gradients") for i in range(b)])
    pairs = [checkpoint(values(t, n, "f32", 10 + i)) for i in range(b)]
    codes, scales = torch.stack([p[0] for p in pairs]), torch.stack([p[1] for p in pairs])
    G = gl.galore_checkpoint_weight_grad(g.cuda(), codes, scales, n)
    for i in range(b):
        check_grad(G[i], host(g[i]), ora.mx8_decode(host(codes[i]), host(scales[i]), n))


@pytest.mark.gpu
def test_weight_grad_no_tokens_and_nonfinite(gl):
    q = gl.galore_checkpoint_empty(0, 40)
    G = gl.galore_checkpoint_weight_grad(torch.zeros((0, 70), device="cuda"), *q, 40)
    assert (G == 0).all()
    start = torch.ones((70, 40), device="cuda")
    assert (gl.galore_checkpoint_weight_grad(torch.zeros((0, 70), device="cuda"), *q, 40, G=start, accumulate=True) == 1).all()
    x = values(40, 70, "f32", 1)
    x[3, 5] = float("nan")
    q = gl.galore_checkpoint_pack(x.cuda())
    dy = values(40, 50, "bf16", 2)
    dy[7, 9] = float("inf")
    dy[8] = 0
    G = host(gl.galore_checkpoint_weight_grad(dy.cuda(), *q, 70, dtype=torch.float32))
    bad = ~np.isfinite(G)
    assert bad[:, :32].all() and bad[9].all()                       # the NaN's block of columns, the Inf's row
    assert not np.delete(bad[:, 32:], 9, axis=0).any()


# ---- 4-bit product ---------------------------------------------------------------------------


PRODUCTS = [(1, 1, 1), (1, 40, 33), (1, 1000, 520), (3, 17, 4096), (16, 100, 129), (17, 64, 256), (33, 130, 300),
            (64, 96, 1000), (65, 64, 32), (100, 130, 257), (130, 257, 700), (300, 200, 64), (257, 1000, 96)]


def check_product(C, a, b):
    want = a @ b.T
    tol = (a.shape[1] + 4) * U * (np.abs(a) @ np.abs(b).T)
    if C.dtype == torch.bfloat16:
        tol = tol + B * (np.abs(want) + tol)
    err = np.abs(host(C) - want)
    assert (err <= tol).all(), (err - tol).max()


def codes4(x):
    return [torch.from_numpy(v).cuda() for v in ora.mx4_encode(host(x))]


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_mx4_matmul(gl, m, n, k, out):
    a, b = codes4(values(m, k, "f32", m + k)), codes4(values(n, k, "f32", n + k + 1))
    C = gl.galore_mx4_matmul(*a, *b, k, dtype=DTYPES[out])
    ah, bh = (ora.mx4_decode(host(q[0]), host(q[1]), k) for q in (a, b))
    check_product(C, ah, bh)
    # bytes past the last block hold anything: rows of a longer pitch, NaN scales in the padding
    wide = [torch.full((q.shape[0], q.shape[1] + 32), 255, dtype=torch.uint8, device="cuda") for q in a]
    for w, q in zip(wide, a):
        w[:, :q.shape[1]] = q
    nb = (k + 31) // 32
    wide[1][:, nb:] = 255
    b[1][:, nb:] = 255
    room = torch.full((m, n + 2), 5.0, dtype=DTYPES[out], device="cuda")
    gl.galore_mx4_matmul(wide[0][:, :a[0].shape[1]], wide[1][:, :a[1].shape[1]], *b, k, C=room[:, 1:n + 1])
    assert torch.equal(room[:, 1:n + 1], C)
    assert (room[:, 0] == 5).all() and (room[:, n + 1] == 5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(4097, 4000, 300), (2100, 1930, 520)])
def test_mx4_matmul_large_tiles(gl, m, n, k):
    a, b = codes4(values(m, k, "f32", 1)), codes4(values(n, k, "f32", 2))
    C = gl.galore_mx4_matmul(*a, *b, k, dtype=torch.float32)
    check_product(C, *(ora.mx4_decode(host(q[0]), host(q[1]), k) for q in (a, b)))


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 20, 70, 200])
def test_mx4_matmul_batched_and_nan(gl, m):
    n, k, nb = 50, 200, 3
    a = [codes4(values(m, k, "f32", i)) for i in range(nb)]
    b = [codes4(values(n, k, "f32", 9 + i)) for i in range(nb)]
    b[1][1][7, 2] = 255                              # one block of one weight row is NaN
    C = gl.galore_mx4_matmul(*[torch.stack(v) for v in zip(*a)], *[torch.stack(v) for v in zip(*b)], k, dtype=torch.float32)
    for i in range(nb):
        ah, bh = (ora.mx4_decode(host(q[0]), host(q[1]), k) for q in (a[i], b[i]))
        if i == 1:
            assert np.isnan(host(C[i])[:, 7]).all()
            keep = np.arange(n) != 7
            check_product(C[i][:, torch.from_numpy(keep).cuda()], ah, bh[keep])
        else:
            check_product(C[i], ah, bh)


@pytest.mark.gpu
def test_mx4_matmul_scale_ends(gl):
    """products of the largest and smallest scales: zero or Inf where fp32 says so, exact between"""
    a = codes4(torch.full((70, 64), 2.0 ** 100))
    for f in (2.0 ** -100, 2.0 ** -90, 2.0 ** 20):
        b = codes4(torch.full((40, 64), f))
        assert (gl.galore_mx4_matmul(*a, *b, 64, dtype=torch.float32) == 64 * 2.0 ** 100 * f).all()
    assert gl.galore_mx4_matmul(*a, *a, 64, dtype=torch.float32).isinf().all()
    zero = gl.galore_mx4_matmul(*codes4(torch.zeros((70, 64))), *a, 64)
    assert (zero == 0).all()


# ---- norms -----------------------------------------------------------------------------------


NORMS = [(1, 1), (3, 7), (5, 64), (2, 511), (9, 512), (3, 513), (6, 1024), (2, 1025), (3, 2047), (2, 4096), (3, 5461),
         (2, 8192), (2, 8193), (1, 16384)]
ALPHA, EPS = 0.7, 1e-5


def norm_inputs(t, d, dtype, gate, seed):
    x, y = values(t, d, dtype, seed), values(t, d, dtype, seed + 1)
    g = torch.Generator().manual_seed(seed)
    w_post, w_pre = 1 + 0.3 * torch.randn(d, generator=g), 1 + 0.3 * torch.randn(d, generator=g)
    gt = None
    if gate == "vector":
        gt = torch.randn(d, generator=g)
    elif gate == "tokens":
        gt = torch.randn((t, d), generator=g).to(DTYPES[dtype])
    return x, y, w_post, w_pre, gt


def on(t, pad=0, offset=0):
    return None if t is None else t.cuda() if t.dim() == 1 else place(t, pad, offset)


def close(got, want, size, count):
    """within (count + 16) U of the sum of magnitudes `size`, and the rounding to bf16"""
    tol = (count + 16) * U * size
    if got.dtype == torch.bfloat16:
        tol = tol + B * (np.abs(want) + tol)
    err = np.abs(host(got) - want)
    assert (err <= tol + 1e-37).all(), (err / (tol + 1e-37)).max()


@pytest.mark.gpu
@pytest.mark.parametrize("gate", ["none", "vector", "tokens"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,d", NORMS)
def test_norm_block(gl, t, d, dtype, gate):
    x, y, wo, wp, gt = norm_inputs(t, d, dtype, gate, t + d)
    xh, yh, gh = host(x), host(y), 1.0 if gt is None else host(gt)
    h, z, rstd = ora.norms(xh, yh, host(wo), host(wp), gh, ALPHA, EPS)
    size = np.abs(xh) + np.abs(h - xh)
    for pad, offset in ((0, 0), (3, 1)):
        H, Z, R, y8, h8, z8 = gl.galore_norm_block(on(x, pad, offset), on(y, pad, offset), on(wo), on(wp),
                                                   on(gt, pad, offset), alpha=ALPHA, eps=EPS, checkpoints=True)
        close(H, h, size, d)
        # a relative error of rstd(h): that of the sum, and the error of h in it
        spread = 1 + np.sqrt((size ** 2).mean(1, keepdims=True)) * rstd[:, 1:]
        close(R[:, :1], rstd[:, :1], np.abs(rstd[:, :1]), d)
        close(R[:, 1:], rstd[:, 1:], np.abs(rstd[:, 1:]) * spread, d)
        # z: the error of h, and that of rstd(h), at most as large as h's
        zsize = np.abs(host(wp)) * rstd[:, 1:] * (size + np.abs(h) * spread)
        close(Z, z, zsize, 2 * d)
        c, s = ora.mx8_encode(yh)
        assert np.array_equal(host(y8[0]), c) and np.array_equal(host(y8[1]), s)
        # checkpoints of h and z: a step of the code, twice where the last bit moved the scale
        for q, want in ((h8, h), (z8, z)):
            nb = (d + 31) // 32
            amax = np.zeros((t, nb * 32))
            amax[:, :d] = np.abs(want)
            amax = np.repeat(amax.reshape(t, nb, 32).max(2), 32, axis=1)[:, :d]
            assert (np.abs(host(gl.galore_checkpoint_unpack(*q, d, dtype=torch.float32)) - want) <= 1.01 * amax / 127 + 2.0 ** -120).all()
            assert (host(q[1])[:, nb:] == 0).all() and (host(q[0])[:, d:] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_block_in_place_and_parts(gl, dtype):
    x, y, wo, wp, gt = norm_inputs(37, 200, dtype, "vector", 3)
    args = (on(y), on(wo), on(wp), on(gt))
    H, Z, R, *none = gl.galore_norm_block(on(x), *args, alpha=ALPHA)
    assert none == [None, None, None]
    xd = on(x)
    out = gl.galore_norm_block(xd, *args, alpha=ALPHA, H=xd, checkpoints=(None, True, None))
    assert out[0] is xd and torch.equal(xd, H) and torch.equal(out[1], Z) and out[3] is None and out[5] is None
    none = gl.galore_norm_block(on(x)[:0], *[a if a.dim() == 1 else a[:0] for a in args], checkpoints=True)
    assert none[0].shape == (0, 200) and none[3][0].shape == (0, 224)


def check_backward(got, dz, dh, hh, yh, rstd, wo, wp, gt, t, d):
    dx, dy, dgate, dwo, dwp = got
    gh = 1.0 if gt is None else host(gt)
    want = ora.norms_backward(dz, dh, hh, yh, rstd, wo, wp, gh, ALPHA)
    a = np.abs
    ry, rh = rstd[:, :1], rstd[:, 1:]
    n, u, p = a(hh * rh), a(yh * ry), a(dz * wp)
    sx = a(dh) + rh * (p + n * (p * n).mean(1, keepdims=True))      # magnitudes that dx is the sum of
    g = ALPHA * sx * a(gh) * a(wo)
    close(dx, want[0], sx, d)
    close(dy, want[1], ry * (g + u * (g * u).mean(1, keepdims=True)), 2 * d + 16)
    per_token = ALPHA * sx * u * a(wo)
    close(dwo, want[3], (ALPHA * sx * a(gh) * u).sum(0), d + t + 16)
    close(dwp, want[4], (a(dz) * n).sum(0), d + t)
    if gt is None:
        assert dgate is None
    elif gt.dim() == 1:
        close(dgate, want[2].sum(0), per_token.sum(0), d + t + 16)
    else:
        close(dgate, want[2], per_token, d + 16)


@pytest.mark.gpu
@pytest.mark.parametrize("gate", ["none", "vector", "tokens"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,d", NORMS + [(1500, 40), (700, 1100)])
def test_norm_block_backward(gl, t, d, dtype, gate):
    x, y, wo, wp, gt = norm_inputs(t, d, dtype, gate, t + d)
    dz, dh = values(t, d, dtype, 5, "gradients"), values(t, d, dtype, 6, "gradients")
    h, _, rstd = ora.norms(host(x), host(y), host(wo), host(wp), 1.0 if gt is None else host(gt), ALPHA, EPS)
    h = torch.from_numpy(h).to(DTYPES[dtype])
    R = torch.from_numpy(rstd).float()
    common = (host(R), host(wo), host(wp), gt, t, d)
    for pad, offset in ((0, 0), (3, 1)):
        got = gl.galore_norm_block_backward(*(on(v, pad, offset) for v in (dz, dh, h, y)), on(R), on(wo), on(wp),
                                            on(gt, pad, offset), alpha=ALPHA)
        check_backward(got, host(dz), host(dh), host(h), host(y), *common)
    # from checkpoints, without a gradient along the stream
    h8, y8 = checkpoint(h), checkpoint(y)
    got = gl.galore_norm_block_backward(on(dz), None, h8, y8, on(R), on(wo), on(wp), on(gt), alpha=ALPHA)
    check_backward(got, host(dz), np.zeros((t, d)), *(ora.mx8_decode(host(c), host(s), d) for c, s in (h8, y8)), *common)


@pytest.mark.gpu
def test_norm_block_backward_in_place_and_empty(gl):
    t, d = 19, 300
    x, y, wo, wp, gt = norm_inputs(t, d, "f32", "tokens", 4)
    H, Z, R, *_ = gl.galore_norm_block(on(x), on(y), on(wo), on(wp), on(gt))
    dz, dh = values(t, d, "f32", 5).cuda(), values(t, d, "f32", 6).cuda()
    a = gl.galore_norm_block_backward(dz, dh, H, on(y), R, on(wo), on(wp), on(gt))
    b = gl.galore_norm_block_backward(dz, dh, H, on(y), R, on(wo), on(wp), on(gt), dX=dh)
    assert b[0] is dh and all(torch.equal(p, q) for p, q in zip(a, b))
    e = torch.zeros((0, d), device="cuda")
    dx, dy, dg, dwo, dwp = gl.galore_norm_block_backward(e, None, e, e, R[:0], on(wo), on(wp), torch.ones(d, device="cuda"))
    assert dx.shape == (0, d) and (dg == 0).all() and (dwo == 0).all() and (dwp == 0).all()


@pytest.mark.gpu
def test_norm_gradients_against_differences(gl):
    """the kernels' gradients along a direction against central differences of the 64-bit forward pass"""
    t, d = 6, 96
    x, y, wo, wp, gt = norm_inputs(t, d, "f32", "vector", 8)
    x, y = x / x.abs().max(), y / y.abs().max()
    dz, dh = (torch.randn((t, d), generator=torch.Generator().manual_seed(i)) for i in (1, 2))
    H, Z, R, *_ = gl.galore_norm_block(on(x), on(y), on(wo), on(wp), on(gt), alpha=ALPHA, eps=1e-2)
    grads = gl.galore_norm_block_backward(on(dz), on(dh), H, on(y), R, on(wo), on(wp), on(gt), alpha=ALPHA)
    at = [host(v) for v in (x, y, gt, wo, wp)]
    rng = np.random.default_rng(0)

    def loss(p):
        h, z, _ = ora.norms(p[0], p[1], p[3], p[4], p[2], ALPHA, 1e-2)
        return (h * host(dh)).sum() + (z * host(dz)).sum()
    for i, g in enumerate(grads):
        v = rng.standard_normal(at[i].shape)
        step = 1e-5
        diff = (loss([p + step * v * (j == i) for j, p in enumerate(at)]) -
                loss([p - step * v * (j == i) for j, p in enumerate(at)])) / (2 * step)
        got = host(g)
        # 2 (d + t) fp32 roundings of terms whose sizes add up to at most about ten times |g| |v|
        assert abs((got * v).sum() - diff) <= 20 * (d + t) * U * np.abs(got * v).sum() + 1e-7


@pytest.mark.gpu
def test_results_do_not_vary_and_streams(gl):
    """the same bits twice, and on another stream than the current one, filled there"""
    t, m, n = 2100, 140, 200
    g, x = values(t, m, "bf16", 1, "gradients").cuda(), values(t, n, "bf16", 2).cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = []
    for stream in (None, None, side):
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            q = gl.galore_checkpoint_pack(x * 1.0, stream=stream)
        G = gl.galore_checkpoint_weight_grad(g, *q, n, dtype=torch.float32, stream=stream)
        a = gl.galore_mx4_quantize(x, stream=stream)
        C = gl.galore_mx4_matmul(*a, a[0][:50].contiguous() if stream is None else a[0][:50], a[1][:50], n, stream=stream)
        w = torch.ones(n, device="cuda")
        torch.cuda.synchronize()
        f = gl.galore_norm_block(x, x, w, w, stream=stream)
        bw = gl.galore_norm_block_backward(x, x, f[0], x, f[2], w, w, stream=stream)
        torch.cuda.synchronize()
        out.append([*q, G, *a, C, *f[:3], bw[0], bw[1], bw[3], bw[4]])
    for other in out[1:]:
        assert all(torch.equal(p, q) for p, q in zip(out[0], other))
