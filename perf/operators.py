"""Performance cases of the training operators around the GaLore path.

GaLore keeps the optimizer's state small, so what a training program still holds
are the activations of the forward pass, and what it still computes are the
products and norms of its blocks. The cases stand for

* ``pack``      an activation written as an 8-bit checkpoint and read back;
* ``grad``      a linear layer's weight gradient from its incoming gradient and
                the 8-bit checkpoint of its input (the gradient that the GaLore
                step then projects);
* ``quant``     a matrix as microscaled 4-bit floating point, in blocks along
                its rows (for the forward product) and along its columns (for
                the backward one), and both read back;
* ``product``   the product of two such operands;
* ``forward``   the norms after and before a block with the block's gate and
                residual scale, with or without the 8-bit checkpoints that the
                backward pass wants;
* ``backward``  their gradients, from plain activations or from checkpoints.

Hidden and intermediate sizes are those of the Llama-shaped workloads of 60M to
7B parameters; token counts run from one to a long batch.

Formats. A row of `cols` values is nb = ceil(cols / 32) blocks of 32. A block has
one scale byte E for 2^(E - 127), NaN where E = 255; a row of scales is padded to
a multiple of four bytes.
8-bit checkpoint: int8 codes c of c 2^(E - 133), 32 nb bytes a row; the smallest E
with the block's largest magnitude at most 127 2^(E - 133), 8 <= E <= 254.
4-bit: E2M1 codes (sign, then 0, .5, 1, 1.5, 2, 3, 4, 6), element 2i in the low
nibble of byte i, 16 nb bytes a row; the smallest E with the block's largest
magnitude at most 6 2^(E - 127), 3 <= E <= 252. Both round half to even, to the
largest code at most; codes past the row's end are zero.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-5
ALPHA = 0.5


def listed():
    return [
        # one 1B-shaped MLP activation: rows of 5461 bf16 values start on no 16-byte boundary
        {"name": "pack-2048x5461-bf16", "kind": "pack", "t": 2048, "n": 5461, "dtype": "bf16"},
        # a long batch of 7B-shaped block inputs
        {"name": "pack-16384x4096-bf16", "kind": "pack", "t": 16384, "n": 4096, "dtype": "bf16"},
        # 1B-shaped gate/up weight, a short micro-batch, gradients kept in fp32, ragged in every size
        {"name": "grad-509t-2048x5461-f32", "kind": "grad", "t": 509, "m": 2048, "n": 5461, "dtype": "f32",
         "out": "f32"},
        # 7B-shaped gate/up weight, a long batch, gradient in the type that the subspace update reads
        {"name": "grad-8192t-11008x4096-bf16", "kind": "grad", "t": 8192, "m": 11008, "n": 4096, "dtype": "bf16",
         "out": "bf16"},
        # 1B-shaped weight in fp32, both orientations
        {"name": "quant-2048x5461-f32", "kind": "quant", "m": 2048, "n": 5461, "dtype": "f32"},
        # 7B-shaped activations or incoming gradients of a long batch, both orientations
        {"name": "quant-8192x4096-bf16", "kind": "quant", "m": 8192, "n": 4096, "dtype": "bf16"},
        # one token through a 7B-shaped gate/up weight: the weight's bytes bound it
        {"name": "product-1x11008x4096-bf16", "kind": "product", "m": 1, "n": 11008, "k": 4096, "out": "bf16"},
        # a long batch through the same weight
        {"name": "product-8192x11008x4096-bf16", "kind": "product", "m": 8192, "n": 11008, "k": 4096, "out": "bf16"},
        # one token of a 7B-shaped model: latency
        {"name": "forward-1x4096-bf16", "kind": "forward", "t": 1, "d": 4096, "dtype": "bf16", "gate": "vector",
         "saved": "none"},
        # a 1B-shaped training batch that writes its checkpoints
        {"name": "forward-4096x2048-bf16-saved", "kind": "forward", "t": 4096, "d": 2048, "dtype": "bf16",
         "gate": "vector", "saved": "packed"},
        # a 350M-shaped model in fp32 with a gate of its own for each token, an odd number of tokens
        {"name": "backward-1003x1024-f32", "kind": "backward", "t": 1003, "d": 1024, "dtype": "f32",
         "gate": "tokens", "saved": "plain"},
        # a long 7B-shaped batch, the activations held in 8 bits
        {"name": "backward-8192x4096-bf16-saved", "kind": "backward", "t": 8192, "d": 4096, "dtype": "bf16",
         "gate": "vector", "saved": "packed"},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def _hidden(rng, lo, hi):
    """mostly round sizes, odd ones among them"""
    d = _log(rng, lo, hi)
    return max(lo, d // 64 * 64) if rng.random() < 0.6 else d


def draw(rng):
    kind = rng.choice(["pack", "grad", "grad", "quant", "product", "product", "forward", "backward"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "pack":
        return {"kind": kind, "t": _log(rng, 1, 16384), "n": _hidden(rng, 64, 4096), "dtype": dtype}
    if kind == "grad":
        return {"kind": kind, "t": _log(rng, 1, 8192), "m": _hidden(rng, 256, 4096), "n": _hidden(rng, 256, 8192),
                "dtype": dtype, "out": "f32" if dtype == "f32" else rng.choice(["bf16", "f32"])}
    if kind == "quant":
        return {"kind": kind, "m": _log(rng, 1, 8192), "n": _hidden(rng, 64, 4096), "dtype": dtype}
    if kind == "product":
        return {"kind": kind, "m": _log(rng, 1, 8192), "n": _hidden(rng, 256, 8192), "k": _hidden(rng, 256, 4096),
                "out": rng.choice(["bf16", "bf16", "f32"])}
    gate = rng.choice(["none", "vector", "tokens"])
    c = {"kind": kind, "t": _log(rng, 1, 8192), "d": _hidden(rng, 64, 4096), "dtype": dtype, "gate": gate}
    c["saved"] = rng.choice(["none" if kind == "forward" else "plain", "packed"])
    return c


def work(c):
    kind = c["kind"]
    b8, b4 = 1 + 1 / 32, 0.5 + 1 / 32          # bytes of an 8-bit and of a 4-bit value with its share of a scale
    if kind == "pack":
        e, s = c["t"] * c["n"], SIZE[c["dtype"]]
        return {"bytes": e * (2 * s + 2 * b8), "flops": 4.0 * e}
    if kind == "grad":
        t, m, n = c["t"], c["m"], c["n"]
        return {"bytes": t * m * SIZE[c["dtype"]] + t * n * b8 + m * n * SIZE[c["out"]], "flops": 2.0 * t * m * n}
    if kind == "quant":
        e, s = c["m"] * c["n"], SIZE[c["dtype"]]
        return {"bytes": e * (s + 4 * b4 + 2 * 2), "flops": 8.0 * e}
    if kind == "product":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": (m + n) * k * b4 + m * n * SIZE[c["out"]], "flops": 2.0 * m * n * k}
    e, s = c["t"] * c["d"], SIZE[c["dtype"]]
    packed = c["saved"] == "packed"
    rows = s if c["gate"] == "tokens" else 0
    if kind == "forward":
        return {"bytes": e * (4 * s + rows + (3 * (2 * b8 + 2) if packed else 0)) + 16.0 * c["d"], "flops": 12.0 * e}
    return {"bytes": e * (4 * s + 2 * rows + 2 * (b8 if packed else s)) + 24.0 * c["d"], "flops": 30.0 * e}


# ---- inputs ---------------------------------------------------------------------------


def _activation(g, t, n, dtype):
    """tokens of unequal size, a few channels much larger than the others, some tokens of padding"""
    x = torch.randn((t, n), generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn((t, 1), generator=g, device="cuda"))
    x *= 1.0 + 19.0 * (torch.rand((1, n), generator=g, device="cuda") < 0.01)
    if t > 8:
        x *= torch.rand((t, 1), generator=g, device="cuda") >= 0.02
    return x.to(dtype)


def _gradient(g, t, n, dtype):
    """small, of unequal size from token to token, zero where the loss is masked"""
    x = 1e-3 * torch.randn((t, n), generator=g, device="cuda")
    x *= torch.exp(torch.randn((t, 1), generator=g, device="cuda"))
    if t > 8:
        x *= torch.rand((t, 1), generator=g, device="cuda") >= 0.05
    return x.to(dtype)


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(c)
    kind = c["kind"]
    dtype = DTYPES.get(c.get("dtype"))
    if kind == "pack":
        s["x"] = _activation(g, c["t"], c["n"], dtype)
    elif kind == "grad":
        s["dy"] = _gradient(g, c["t"], c["m"], dtype)
        s["codes"], s["scales"] = _pack(_activation(g, c["t"], c["n"], torch.float32))
    elif kind == "quant":
        s["x"] = _activation(g, c["m"], c["n"], dtype)
    elif kind == "product":
        s["a"], s["a_scales"] = _quantize(_activation(g, c["m"], c["k"], torch.float32))
        s["b"], s["b_scales"] = _quantize(0.02 * torch.randn((c["n"], c["k"]), generator=g, device="cuda"))
    else:
        t, d = c["t"], c["d"]
        s["w_post"] = 1.0 + 0.1 * torch.randn(d, generator=g, device="cuda")
        s["w_pre"] = 1.0 + 0.1 * torch.randn(d, generator=g, device="cuda")
        s["gate"] = None
        if c["gate"] == "vector":
            s["gate"] = torch.rand(d, generator=g, device="cuda")
        elif c["gate"] == "tokens":
            s["gate"] = torch.sigmoid(torch.randn((t, d), generator=g, device="cuda")).to(dtype)
        x, y = _activation(g, t, d, dtype), _activation(g, t, d, dtype)
        if kind == "forward":
            s["x"], s["y"] = x, y
        else:
            s["dz"], s["dh"] = _gradient(g, t, d, dtype), _gradient(g, t, d, dtype)
            h, _, s["rstd"] = _norms(x.float(), y.float(), s["w_post"], s["w_pre"], s["gate"])
            if c["saved"] == "packed":
                s["h"], s["y"] = _pack(h), _pack(y.float())
            else:
                s["h"], s["y"] = h.to(dtype), y
    return s


# ---- the plain forms ------------------------------------------------------------------


def _blocks(x, top, less, least, most, step):
    """x (rows, cols) in blocks of 32 over its blocks' units 2^(E - 127 - step), and the scale bytes: E is the exponent
    field of the largest magnitude, less `less`, and one more where its fraction is over `top`"""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    v = torch.zeros((rows, 32 * nb), dtype=torch.float32, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, nb, 32)
    bits = v.abs().amax(2).view(torch.int32)
    e = ((bits >> 23) - less + ((bits & 0x7fffff) > top)).clamp(least, most)
    scales = torch.zeros((rows, (nb + 3) // 4 * 4), dtype=torch.uint8, device=x.device)
    bad = bits >= 0x7f800000
    inverse = ((254 + step - e) << 23).view(torch.float32)  # 2^-(E - 127 - step)
    scales[:, :nb] = torch.where(bad, torch.full_like(e, 255), e).to(torch.uint8)
    u = v * inverse.unsqueeze(2)
    return torch.where(bad.unsqueeze(2), torch.zeros_like(u), u).reshape(rows, 32 * nb), scales


def _pack(x):
    u, scales = _blocks(x, 0x7e0000, 0, 8, 254, 6)
    return torch.round(u).clamp(-127, 127).to(torch.int8), scales


def _factors(scales, nb, step):
    """2^(E - 127 - step) for every value of a row of nb blocks"""
    e = scales[:, :nb].to(torch.int32)
    f = torch.ldexp(torch.ones((), device=scales.device), e - 127 - step)
    return torch.where(e == 255, torch.full_like(f, math.nan), f).repeat_interleave(32, dim=1)


def _unpack(codes, scales, cols):
    return (codes.float() * _factors(scales, codes.shape[1] // 32, 6))[:, :cols]


def _quantize(x):
    u, scales = _blocks(x, 0x400000, 2, 3, 252, 0)
    a = u.abs().clamp(max=6)
    # the steps are .5 up to 2, 1 up to 4 and 2 up to 6
    q = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, torch.round(a) + 2, torch.round(0.5 * a) + 4))
    q = q.to(torch.uint8) | (torch.signbit(u).to(torch.uint8) << 3)
    return q[:, 0::2] | (q[:, 1::2] << 4), scales


def _dequantize(codes, scales, cols):
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    v = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), dim=2).reshape(codes.shape[0], -1)
    return (v * _factors(scales, codes.shape[1] // 16, 0))[:, :cols]


def _rstd(x):
    return torch.rsqrt((x * x).mean(1) + EPS)


def _norms(x, y, w_post, w_pre, gate):
    ry = _rstd(y)
    u = y * ry[:, None] * w_post
    if gate is not None:
        u = u * gate.float()
    h = x + ALPHA * u
    rh = _rstd(h)
    return h, h * rh[:, None] * w_pre, torch.stack((ry, rh), 1)


def _norms_backward(dz, dh, h, y, rstd, w_post, w_pre, gate):
    ry, rh = rstd[:, :1], rstd[:, 1:]
    nh, ny = h * rh, y * ry
    a = dz * w_pre
    dx = dh + rh * (a - nh * (a * nh).mean(1, keepdim=True))
    b = ALPHA * dx
    s = b * ny                                   # the gradient of gate * w_post
    if gate is None:
        dgate, gated, dw_post = None, b * w_post, s.sum(0)
    else:
        gate = gate.float()
        gated = b * gate * w_post
        dw_post = (s * gate).sum(0)
        dgate = s * w_post
        if gate.dim() == 1:
            dgate = dgate.sum(0)
    dy = ry * (gated - ny * (gated * ny).mean(1, keepdim=True))
    return dx, dy, dgate, dw_post, (dz * nh).sum(0)


def _plain(s):
    kind = s["kind"]
    if kind == "pack":
        codes, scales = _pack(s["x"].float())
        return {"x": _unpack(codes, scales, s["n"]).to(s["x"].dtype), "scales": scales}
    if kind == "grad":
        x = _unpack(s["codes"], s["scales"], s["n"])
        return torch.matmul(s["dy"].float().t(), x).to(DTYPES[s["out"]])
    if kind == "quant":
        x = s["x"].float()
        rows, row_scales = _quantize(x)
        cols, col_scales = _quantize(x.t())
        return {"rows": _dequantize(rows, row_scales, s["n"]).to(torch.bfloat16), "row_scales": row_scales,
                "columns": _dequantize(cols, col_scales, s["m"]).to(torch.bfloat16), "column_scales": col_scales}
    if kind == "product":
        a = _dequantize(s["a"], s["a_scales"], s["k"])
        return torch.matmul(a, _dequantize(s["b"], s["b_scales"], s["k"]).t()).to(DTYPES[s["out"]])
    dtype = DTYPES[s["dtype"]]
    if kind == "forward":
        h, z, rstd = _norms(s["x"].float(), s["y"].float(), s["w_post"], s["w_pre"], s["gate"])
        r = {"h": h.to(dtype), "z": z.to(dtype), "rstd": rstd}
        if s["saved"] == "packed":
            r["y8"] = _unpack(*_pack(s["y"].float()), s["d"]).to(torch.bfloat16)
            r["h8"] = _unpack(*_pack(h), s["d"]).to(torch.bfloat16)
            r["z8"] = _unpack(*_pack(z), s["d"]).to(torch.bfloat16)
        return r
    if s["saved"] == "packed":
        h, y = _unpack(*s["h"], s["d"]), _unpack(*s["y"], s["d"])
    else:
        h, y = s["h"].float(), s["y"].float()
    dx, dy, dgate, dw_post, dw_pre = _norms_backward(s["dz"].float(), s["dh"].float(), h, y, s["rstd"], s["w_post"],
                                                     s["w_pre"], s["gate"])
    r = {"dx": dx.to(dtype), "dy": dy.to(dtype), "dw_post": dw_post, "dw_pre": dw_pre}
    if dgate is not None:
        r["dgate"] = dgate.to(s["gate"].dtype)
    return r


# ---- the framework's calls --------------------------------------------------------------


def _own(s):
    import paper_2504_20437_amd as gl
    kind = s["kind"]
    if kind == "pack":
        codes, scales = gl.galore_checkpoint_pack(s["x"])
        return {"x": gl.galore_checkpoint_unpack(codes, scales, s["n"], dtype=s["x"].dtype), "scales": scales}
    if kind == "grad":
        return gl.galore_checkpoint_weight_grad(s["dy"], s["codes"], s["scales"], s["n"], dtype=DTYPES[s["out"]])
    if kind == "quant":
        rows, row_scales, cols, col_scales = gl.galore_mx4_quantize(s["x"], rows=True, columns=True)
        return {"rows": gl.galore_mx4_dequantize(rows, row_scales, s["n"]), "row_scales": row_scales,
                "columns": gl.galore_mx4_dequantize(cols, col_scales, s["m"]), "column_scales": col_scales}
    if kind == "product":
        return gl.galore_mx4_matmul(s["a"], s["a_scales"], s["b"], s["b_scales"], s["k"], dtype=DTYPES[s["out"]])
    if kind == "forward":
        saved = s["saved"] == "packed"
        h, z, rstd, y8, h8, z8 = gl.galore_norm_block(s["x"], s["y"], s["w_post"], s["w_pre"], s["gate"], alpha=ALPHA,
                                                      eps=EPS, checkpoints=saved)
        r = {"h": h, "z": z, "rstd": rstd}
        if saved:
            r["y8"] = gl.galore_checkpoint_unpack(*y8, s["d"])
            r["h8"] = gl.galore_checkpoint_unpack(*h8, s["d"])
            r["z8"] = gl.galore_checkpoint_unpack(*z8, s["d"])
        return r
    dx, dy, dgate, dw_post, dw_pre = gl.galore_norm_block_backward(s["dz"], s["dh"], s["h"], s["y"], s["rstd"],
                                                                   s["w_post"], s["w_pre"], s["gate"], alpha=ALPHA)
    r = {"dx": dx, "dy": dy, "dw_post": dw_post, "dw_pre": dw_pre}
    if dgate is not None:
        r["dgate"] = dgate
    return r


def run(state):
    return _own(state) if own else _plain(state)


# ---- the same from the definitions, in 64 bits ------------------------------------------


def _round64(x, largest, floor, values, bias):
    """x, in blocks of 32 along its rows, rounded to `values` (the non-negative ones, ascending) times each block's
    scale: the smallest power of two, 2^floor or more, that brings the block's magnitudes to `largest` or under. And
    the exponents plus `bias`."""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    v = torch.nn.functional.pad(x.double(), (0, 32 * nb - cols)).view(rows, nb, 32)
    mantissa, exponent = torch.frexp(v.abs().amax(2) / largest)
    exponent = torch.where(mantissa > 0.5, exponent, exponent - 1)
    exponent = torch.where(mantissa > 0, exponent, torch.full_like(exponent, floor)).clamp(min=floor)
    unit = torch.pow(torch.full((), 2.0, dtype=torch.float64, device=x.device), exponent.double()).unsqueeze(2)
    u = (v / unit).abs()
    above = torch.bucketize(u, values).clamp(max=len(values) - 1)    # the first value that is not below u
    below = (above - 1).clamp(min=0)
    up, down = values[above] - u, u - values[below]
    even = (above % 2 == 0)
    pick = torch.where((up < down) | ((up == down) & even), values[above], values[below])
    got = (torch.sign(v) * pick * unit).view(rows, 32 * nb)[:, :cols]
    scales = torch.zeros((rows, (nb + 3) // 4 * 4), dtype=torch.uint8, device=x.device)
    scales[:, :nb] = (exponent + bias).to(torch.uint8)
    return got, scales


def _pack64(x):
    return _round64(x, 127, -125, torch.arange(128, dtype=torch.float64, device=x.device), 133)


def _quantize64(x):
    values = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    return _round64(x, 6, -124, values, 127)


def _values64(codes, scales, cols, bits):
    """what codes and scales stand for, from the bits"""
    if bits == 8:
        v, shift = codes.double(), 133
    else:
        n = torch.stack((codes & 15, codes >> 4), dim=2).reshape(codes.shape[0], -1).long()
        sign, e, f = n >> 3, (n >> 1) & 3, (n & 1).double()
        v = torch.where(e == 0, 0.5 * f, (1 + 0.5 * f) * torch.pow(2.0, (e - 1).double()))
        v, shift = torch.where(sign == 1, -v, v), 127
    block = torch.arange(cols, device=codes.device) // 32
    return v[:, :cols] * torch.pow(2.0, scales.double() - shift)[:, block]


def exact(c, seed):
    s = prepare(c, seed)
    kind = c["kind"]
    if kind == "pack":
        x, scales = _pack64(s["x"])
        return {"x": x, "scales": scales}
    if kind == "grad":
        return torch.matmul(s["dy"].double().t().contiguous(), _values64(s["codes"], s["scales"], c["n"], 8))
    if kind == "quant":
        rows, row_scales = _quantize64(s["x"])
        cols, col_scales = _quantize64(s["x"].t())
        return {"rows": rows, "row_scales": row_scales, "columns": cols, "column_scales": col_scales}
    if kind == "product":
        a, b = _values64(s["a"], s["a_scales"], c["k"], 4), _values64(s["b"], s["b_scales"], c["k"], 4)
        return torch.matmul(a, b.t().contiguous())
    d = c["d"]
    gate = torch.ones((), dtype=torch.float64, device="cuda") if s["gate"] is None else s["gate"].double()
    w_post, w_pre = s["w_post"].double(), s["w_pre"].double()
    if kind == "forward":
        x, y = s["x"].double(), s["y"].double()
        sy = torch.sqrt((y ** 2).sum(1, keepdim=True) / d + EPS)
        h = x + gate * (ALPHA * w_post) * (y / sy)
        sh = torch.sqrt((h ** 2).sum(1, keepdim=True) / d + EPS)
        z = w_pre * (h / sh)
        r = {"h": h, "z": z, "rstd": torch.cat((1 / sy, 1 / sh), 1)}
        if c["saved"] == "packed":
            # a last bit of h or z decides between two codes, so only y's are fixed
            r["y8"], r["h8"], r["z8"] = _pack64(y)[0], None, None
        return r
    if c["saved"] == "packed":
        h, y = _values64(*s["h"], d, 8), _values64(*s["y"], d, 8)
    else:
        h, y = s["h"].double(), s["y"].double()
    dz, dh, r = s["dz"].double(), s["dh"].double(), s["rstd"].double()
    ry, rh = r[:, 0:1], r[:, 1:2]
    p = dz * w_pre * rh
    dx = dh + p - h * rh ** 2 * ((p * h).sum(1, keepdim=True) / d)
    q = ALPHA * dx * gate * w_post * ry
    dy = q - y * ry ** 2 * ((q * y).sum(1, keepdim=True) / d)
    out = {"dx": dx, "dy": dy, "dw_post": (ALPHA * dx * gate * y * ry).sum(0), "dw_pre": (dz * h * rh).sum(0)}
    if s["gate"] is not None:
        per_token = ALPHA * dx * w_post * y * ry
        out["dgate"] = per_token.sum(0) if s["gate"].dim() == 1 else per_token
    return out
