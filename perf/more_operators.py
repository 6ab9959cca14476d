"""Performance cases of the operators that stand between a model's linear layers.

A training step in little memory has, beside its products, its norms and its
optimizer, an embedding, dropout, the rotation of queries and keys, and a mixing of
tokens. None of these keeps anything for its backward pass that can be made again.
The cases stand for

* ``lookup``      rows of the embedding matrix for token ids, scaled;
* ``embgrad``     the embedding matrix's gradient, in the form that a subspace
                  update reads: rows of the incoming gradient summed by token id;
* ``dropout``     dropout of a block's output, added to the residual stream or kept
                  as an 8-bit checkpoint too (the backward pass is the same call on
                  the incoming gradient);
* ``rotate``      the norms of queries and keys for each head and the rotation by
                  position;
* ``rotateback``  their gradients, from plain queries and keys or 8-bit checkpoints;
* ``scan``        a gated linear recurrence over tokens;
* ``scanback``    its gradients.

Hidden sizes and heads are those of the Llama-shaped workloads of 60M to 7B
parameters, token counts run from one to a long batch.

Definitions.
Lookup: out[t] = scale W[id]; a negative id is padding, whose row is zero and which
has no gradient. Gradient: G[v] = scale times the sum of the rows t with id v.
Dropout: element c of row t of matrix b has 16 random bits, from Philox4x32-10 with the
key (seed's low word, high word) and the counter (c // 8, t, b, index): word
(c % 8) // 2, its low half where c is even. It is kept where they are T = round(65536 p)
or more, and multiplied by 65536 / (65536 - T).
Rotation: n = x (mean x^2 + eps)^(-1/2) w over a head, then for the first `rot` values
(y_i, y_j) = (n_i cos - n_j sin, n_i sin + n_j cos), j = i + rot / 2, or (2 i, 2 i + 1)
interleaved; a row of the table holds the cosines, then the sines.
Recurrence: a = sigmoid(f), h_t = a_t h_{t-1} + (1 - a_t) x_t in each channel, from h0;
packed sequences lie one after the other, their bounds in `offsets`.
8-bit checkpoint: blocks of 32 along a row, a scale byte E each, codes c of value
c 2^(E - 133), |c| <= 127, the smallest E >= 8 that clips none; half to even.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-5
BASE = 10000.0
STEP = 64            # tokens from one kept state of the recurrence to the next


def listed():
    return [
        # one token of a 7B-shaped model that answers: latency
        {"name": "lookup-1-32000x4096-bf16", "kind": "lookup", "t": 1, "v": 32000, "d": 4096, "dtype": "bf16",
         "out": "bf16"},
        # a short micro-batch of a 350M-shaped model trained in fp32: most of G is rows that no token has
        {"name": "embgrad-1003-32000x1024-f32", "kind": "embgrad", "t": 1003, "v": 32000, "d": 1024, "dtype": "f32",
         "out": "f32"},
        # a long batch of a 7B-shaped model, gradient in the type that the subspace update reads
        {"name": "embgrad-16384-32000x4096-bf16", "kind": "embgrad", "t": 16384, "v": 32000, "d": 4096,
         "dtype": "bf16", "out": "bf16"},
        # 1B-shaped MLP activations in fp32 added to a stream, ragged in both sizes
        {"name": "dropout-509x5461-f32-residual", "kind": "dropout", "b": 1, "t": 509, "d": 5461, "dtype": "f32",
         "p": 0.1, "residual": True, "saved": False},
        # a long 7B-shaped batch before a linear layer, kept in 8 bits for its weight gradient
        {"name": "dropout-16384x4096-bf16-saved", "kind": "dropout", "b": 1, "t": 16384, "d": 4096, "dtype": "bf16",
         "p": 0.1, "residual": False, "saved": True},
        # one token of a 7B-shaped model, 32 heads of 128: latency
        {"name": "rotate-1-32+32x128-bf16", "kind": "rotate", "t": 1, "hq": 32, "hk": 32, "d": 128, "rot": 128,
         "inter": False, "dtype": "bf16"},
        # a long batch, eight query heads to a key head
        {"name": "rotate-8192-32+4x128-bf16", "kind": "rotate", "t": 8192, "hq": 32, "hk": 4, "d": 128, "rot": 128,
         "inter": False, "dtype": "bf16"},
        # heads of 80 in fp32, a part of them rotated in neighbouring pairs, an odd number of tokens
        {"name": "rotateback-1003-16+2x80-f32", "kind": "rotateback", "t": 1003, "hq": 16, "hk": 2, "d": 80, "rot": 32,
         "inter": True, "dtype": "f32", "saved": "plain"},
        # a long 7B-shaped batch whose queries and keys are held in 8 bits
        {"name": "rotateback-8192-32+32x128-bf16-saved", "kind": "rotateback", "t": 8192, "hq": 32, "hk": 32, "d": 128,
         "rot": 128, "inter": False, "dtype": "bf16", "saved": "packed"},
        # one token of each of 16 sequences, states in and out
        {"name": "scan-16x1x2048-bf16", "kind": "scan", "b": 16, "t": 1, "d": 2048, "dtype": "bf16", "packed": 0,
         "h0": True, "saved": False},
        # a long 1B-shaped batch, states kept for the backward pass
        {"name": "scan-4x8192x2048-bf16-saved", "kind": "scan", "b": 4, "t": 8192, "d": 2048, "dtype": "bf16",
         "packed": 0, "h0": False, "saved": True},
        # 7B-shaped documents packed into one long row
        {"name": "scanback-8192x4096-bf16-packed", "kind": "scanback", "b": 1, "t": 8192, "d": 4096, "dtype": "bf16",
         "packed": 11, "h0": False},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def _hidden(rng, lo, hi):
    """mostly round sizes, odd ones among them"""
    d = _log(rng, lo, hi)
    return max(lo, d // 64 * 64) if rng.random() < 0.6 else d


def draw(rng):
    kind = rng.choice(["lookup", "embgrad", "embgrad", "dropout", "dropout", "rotate", "rotateback", "scan", "scan",
                       "scanback", "scanback"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("lookup", "embgrad"):
        return {"kind": kind, "t": _log(rng, 1, 8192), "v": _log(rng, 100, 32000), "d": _hidden(rng, 64, 4096),
                "dtype": dtype, "out": rng.choice([dtype, "f32"])}
    if kind == "dropout":
        return {"kind": kind, "b": rng.choice([1, 1, 2, 3]), "t": _log(rng, 1, 2700), "d": _hidden(rng, 64, 4096),
                "dtype": dtype, "p": rng.choice([0.05, 0.1, 0.25, 0.5]), "residual": rng.random() < 0.5,
                "saved": rng.random() < 0.5}
    if kind in ("rotate", "rotateback"):
        hk = rng.choice([1, 2, 4, 8])
        d = rng.choice([64, 64, 128, 128, 80, 96, 40, 256, 75])
        c = {"kind": kind, "t": _log(rng, 1, 4096), "hq": hk * rng.choice([1, 2, 4]), "hk": hk, "d": d,
             "rot": rng.choice([d // 2 * 2, d // 2 * 2, d // 4 * 2, d // 16 * 4]), "inter": rng.random() < 0.3,
             "dtype": dtype}
        if kind == "rotateback":
            c["saved"] = rng.choice(["plain", "packed"])
        return c
    b = rng.choice([1, 1, 2, 8])
    c = {"kind": kind, "b": b, "t": max(1, _log(rng, 1, 8192) // b), "d": _hidden(rng, 64, 2048), "dtype": dtype,
         "packed": rng.choice([0, 1, 5, 40]) if b == 1 else 0, "h0": rng.random() < 0.5}
    if kind == "scan":
        c["saved"] = rng.random() < 0.5
    return c


def _frequencies(v):
    """how often a token id comes up, by rank: falling as one over the rank"""
    r = np.arange(1, v + 1, dtype=np.float64)
    return np.log1p(1 / r) / math.log(v + 1)


def work(c):
    kind, s = c["kind"], SIZE[c["dtype"]]
    b8 = 1 + 1 / 32                           # bytes of an 8-bit value with its share of a scale
    if kind in ("lookup", "embgrad"):
        t, v, d, o = c["t"], c["v"], c["d"], SIZE[c["out"]]
        if kind == "embgrad":
            return {"bytes": 8.0 * t + t * d * s + v * d * o, "flops": 1.0 * t * d}
        rows = float((1 - (1 - _frequencies(v)) ** t).sum())     # that come up at all
        return {"bytes": 8.0 * t + rows * d * s + t * d * o, "flops": 1.0 * t * d}
    if kind == "dropout":
        e = c["b"] * c["t"] * c["d"]
        # ten rounds of two products and four exclusive ors for eight values
        return {"bytes": e * (2 * s + (s if c["residual"] else 0) + (b8 + 2 if c["saved"] else 0)),
                "flops": e * (60 / 8 + 3)}
    if kind in ("rotate", "rotateback"):
        e = c["t"] * (c["hq"] + c["hk"]) * c["d"]
        other = 4.0 * c["t"] * (1 + c["rot"]) + 8.0 * c["d"]
        if kind == "rotate":
            return {"bytes": 2 * e * s + other, "flops": 8.0 * e}
        return {"bytes": e * (2 * s + (b8 if c["saved"] == "packed" else s)) + other + 8.0 * c["d"], "flops": 18.0 * e}
    e = c["b"] * c["t"] * c["d"]
    states = 4.0 * c["b"] * -(-c["t"] // STEP) * c["d"]
    row = 4.0 * max(c["b"], c["packed"]) * c["d"]     # a state of every sequence
    if kind == "scan":
        return {"bytes": 3 * e * s + (states if c["saved"] else 0) + row * (2 if c["h0"] else 1), "flops": 10.0 * e}
    return {"bytes": 5 * e * s + states + row * (3 if c["h0"] else 2), "flops": 24.0 * e}


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


def _token_ids(g, t, v):
    """ids as text has them, a few of them padding"""
    rank = torch.exp(torch.rand(t, generator=g, device="cuda", dtype=torch.float64) * math.log(v + 1)).long() - 1
    ids = torch.randperm(v, generator=g, device="cuda")[rank.clamp(0, v - 1)]
    if t > 8:
        ids = torch.where(torch.rand(t, generator=g, device="cuda") < 0.02, torch.full_like(ids, -1), ids)
    return ids


def _bounds(g, t, n):
    """bounds of n sequences over t tokens, some of them short"""
    cut = (t * torch.rand(n - 1, generator=g, device="cuda") ** 1.5).int().clamp(0, t).sort().values
    ends = torch.tensor([0, t], dtype=torch.int32, device="cuda")
    return torch.cat((ends[:1], cut.int(), ends[1:]))


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(c)
    kind, dtype, t, d = c["kind"], DTYPES[c["dtype"]], c["t"], c["d"]
    if kind in ("lookup", "embgrad"):
        s["ids"] = _token_ids(g, t, c["v"])
        s["scale"] = float(np.float32(d ** 0.5))
        if kind == "lookup":
            s["w"] = (0.02 * torch.randn((c["v"], d), generator=g, device="cuda")).to(dtype)
        else:
            s["dy"] = _gradient(g, t, d, dtype)
    elif kind == "dropout":
        s["seed"] = int(torch.randint(0, 2 ** 62, (1,), generator=torch.Generator().manual_seed(seed)))
        s["index"] = seed % 1000
        s["x"] = _activation(g, c["b"] * t, d, dtype).view(c["b"], t, d)
        s["r"] = _activation(g, c["b"] * t, d, dtype).view(c["b"], t, d) if c["residual"] else None
    elif kind in ("rotate", "rotateback"):
        hq, hk, rot = c["hq"], c["hk"], c["rot"]
        s["w_q"] = 1.0 + 0.1 * torch.randn(d, generator=g, device="cuda")
        s["w_k"] = 1.0 + 0.1 * torch.randn(d, generator=g, device="cuda")
        # a batch of documents, each counted from its own start
        start = int(torch.randint(0, 4096, (1,), generator=torch.Generator().manual_seed(seed)))
        s["positions"] = ((torch.arange(t, device="cuda") + start) % 4096).int()
        angle = torch.arange(4096, device="cuda", dtype=torch.float64)[:, None] * \
            BASE ** (-2 * torch.arange(rot // 2, device="cuda", dtype=torch.float64) / max(rot, 1))
        s["table"] = torch.cat((angle.cos(), angle.sin()), 1).float()
        # queries, keys and values as one product leaves them
        qkv = _activation(g, t, (hq + 2 * hk) * d, dtype)
        q, k = qkv[:, :hq * d], qkv[:, hq * d:(hq + hk) * d]
        if kind == "rotate":
            s["q"], s["k"] = q.unflatten(1, (hq, d)), k.unflatten(1, (hk, d))
        else:
            s["dq"] = _gradient(g, t, hq * d, dtype).view(t, hq, d)
            s["dk"] = _gradient(g, t, hk * d, dtype).view(t, hk, d)
            if c["saved"] == "packed":
                s["q"], s["k"] = _pack(q.float()), _pack(k.float())
            else:
                s["q"], s["k"] = q.unflatten(1, (hq, d)), k.unflatten(1, (hk, d))
    else:
        b, n = c["b"], c["packed"]
        lead = (b, t, d) if not n else (t, d)
        s["x"] = _activation(g, b * t, d, dtype).view(lead)
        # most gates forget slowly
        s["f"] = (2.0 + 1.5 * torch.randn((b * t, d), generator=g, device="cuda")).to(dtype).view(lead)
        s["offsets"] = _bounds(g, t, n) if n else None
        s["h0"] = torch.randn((n or b, d), generator=g, device="cuda") if c["h0"] else None
        if kind == "scanback":
            s["dh"] = _gradient(g, b * t, d, dtype).view(lead)
            s["dlast"] = 1e-3 * torch.randn((n or b, d), generator=g, device="cuda")
            h, _, entering = _scan(s)
            del h
            s["states"] = entering
    return s


# ---- the plain forms ------------------------------------------------------------------


def _pack(x):
    """8-bit checkpoint of x (rows, cols): codes and scales"""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    v = torch.zeros((rows, 32 * nb), dtype=torch.float32, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, nb, 32)
    bits = v.abs().amax(2).view(torch.int32)
    e = ((bits >> 23) + ((bits & 0x7fffff) > 0x7e0000)).clamp(8, 254)
    scales = torch.zeros((rows, (nb + 3) // 4 * 4), dtype=torch.uint8, device=x.device)
    scales[:, :nb] = e.to(torch.uint8)
    u = v * ((260 - e) << 23).view(torch.float32).unsqueeze(2)      # 2^(133 - E)
    return torch.round(u).clamp(-127, 127).to(torch.int8).view(rows, 32 * nb), scales


def _unpack(codes, scales, cols):
    e = scales[:, :codes.shape[1] // 32].to(torch.int32)
    unit = torch.ldexp(torch.ones((), device=scales.device), e - 133)
    return (codes.float() * unit.repeat_interleave(32, dim=1))[:, :cols]


def _random16(seed, index, b, t, groups):
    """(b, t, 8 groups) random 16-bit numbers"""
    def grid(n, dim):
        shape = [1, 1, 1]
        shape[dim] = n
        return torch.arange(n, device="cuda").view(shape).expand(b, t, groups)
    low = 0xffffffff
    x = [grid(groups, 2), grid(t, 1), grid(b, 0), torch.full((b, t, groups), index, dtype=torch.int64, device="cuda")]
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p0, p1 = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [(p1 >> 32 & low) ^ x[1] ^ k0, p1 & low, (p0 >> 32 & low) ^ x[3] ^ k1, p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([h for w in x for h in (w & 0xffff, w >> 16)], dim=3).view(b, t, 8 * groups)


def _dropout(s):
    b, t, d = s["x"].shape
    cut = int(round(65536 * s["p"]))
    kept = _random16(s["seed"], s["index"], b, t, (d + 7) // 8)[:, :, :d] >= cut
    y = torch.where(kept, s["x"].float() * float(np.float32(65536 / (65536 - cut))), torch.zeros((), device="cuda"))
    return y + s["r"].float() if s["residual"] else y


def _rotate(n, table, positions, inter, back):
    """the rotation of n (tokens, heads, d) by its table's rows, or its transpose"""
    half = table.shape[1] // 2
    cos, sin = table[positions.long()][:, None, :half], table[positions.long()][:, None, half:]
    if back:
        sin = -sin
    out = n.clone()
    first = slice(0, 2 * half, 2) if inter else slice(0, half)
    second = slice(1, 2 * half, 2) if inter else slice(half, 2 * half)
    out[..., first] = n[..., first] * cos - n[..., second] * sin
    out[..., second] = n[..., first] * sin + n[..., second] * cos
    return out


def _heads(x, w, s):
    n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    return _rotate(n, s["table"], s["positions"], s["inter"], False)


def _heads_backward(dy, x, w, s):
    dn = _rotate(dy, s["table"], s["positions"], s["inter"], True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    u, p = x * r, dn * w
    return r * (p - u * (p * u).mean(-1, keepdim=True)), (dn * u).sum((0, 1))


def _prefix(a, b):
    """b_t := b_t + a_t b_{t-1} in turn along the second axis, by doubling"""
    k = 1
    while k < a.shape[1]:
        b = torch.cat((b[:, :k], b[:, k:] + a[:, k:] * b[:, :-k]), 1)
        a = torch.cat((a[:, :k], a[:, k:] * a[:, :-k]), 1)
        k *= 2
    return b


def _sequences(s):
    """first and last tokens of the sequences that have any (as a mask over (batch, tokens)), and for each such token its
    sequence, in the order of a boolean index; the sequences without tokens"""
    b, t = (1, s["t"]) if s["offsets"] is not None else (s["b"], s["t"])
    first = torch.zeros((b, t), dtype=torch.bool, device="cuda")
    last = torch.zeros((b, t), dtype=torch.bool, device="cuda")
    if s["offsets"] is None:
        first[:, 0] = True
        last[:, -1] = True
        owner = torch.arange(b, device="cuda")
        return first, last, owner, owner[:0]
    o = s["offsets"].long()
    length = o[1:] - o[:-1]
    some = torch.nonzero(length > 0).view(-1)
    first[0, o[:-1][some]] = True
    last[0, o[1:][some] - 1] = True
    return first, last, some, torch.nonzero(length == 0).view(-1)


def _gates(s):
    shape = (1,) + tuple(s["x"].shape) if s["x"].dim() == 2 else tuple(s["x"].shape)
    f = s["f"].float().view(shape)
    return s["x"].float().view(shape), torch.sigmoid(f), torch.sigmoid(-f)


def _scan(s):
    """h, the last states, and the states that enter every STEP tokens"""
    x, a, z = _gates(s)
    first, last, some, none = _sequences(s)
    h0 = s["h0"] if s["h0"] is not None else torch.zeros((s["packed"] or s["b"], s["d"]), device="cuda")
    u = z * x
    u[first] += a[first] * h0[some]
    h = _prefix(torch.where(first[..., None], torch.zeros((), device="cuda"), a), u)
    end = torch.empty_like(h0)
    end[some] = h[last]
    end[none] = h0[none]
    entering = torch.zeros((x.shape[0], -(-x.shape[1] // STEP), x.shape[2]), device="cuda")
    if s["offsets"] is None:
        entering[:, 0] = h0
    entering[:, 1:] = h[:, STEP - 1:-1:STEP]
    return h.view(s["x"].shape), end, entering if s["x"].dim() == 3 else entering[0]


def _scan_backward(s):
    x, a, z = _gates(s)
    first, last, some, none = _sequences(s)
    h0 = s["h0"] if s["h0"] is not None else torch.zeros_like(s["dlast"])
    # states before each token: from those kept, over at most STEP tokens
    b, t, d = x.shape
    n = s["states"].shape[-2]
    pad = torch.nn.functional.pad
    shape = (b * n, STEP, d)
    u = z * x
    u[first] += a[first] * h0[some]
    start = torch.where(first[..., None], torch.zeros((), device="cuda"), a)
    u = pad(u, (0, 0, 0, n * STEP - t)).view(shape)
    start = pad(start, (0, 0, 0, n * STEP - t)).view(shape)
    entering = s["states"].reshape(b * n, 1, d)
    u[:, :1] += start[:, :1] * entering
    h = _prefix(start, u)
    before = torch.cat((entering, h[:, :-1]), 1).view(b, n * STEP, d)[:, :t].clone()
    before[first] = h0[some]
    g = s["dh"].float().view(x.shape).clone()
    g[last] += s["dlast"][some]
    after = torch.zeros_like(a)
    after[:, :-1] = a[:, 1:]
    after[last] = 0
    g = _prefix(after.flip(1), g.flip(1)).flip(1)
    dh0 = torch.empty_like(h0)
    dh0[some] = (a * g)[first]
    dh0[none] = s["dlast"][none]
    return (z * g).view(s["x"].shape), (g * (before - x) * a * z).view(s["x"].shape), dh0


def _plain(s):
    kind, dtype = s["kind"], DTYPES[s["dtype"]]
    if kind == "lookup":
        y = s["w"][s["ids"].clamp(min=0)].float() * s["scale"]
        return torch.where((s["ids"] < 0)[:, None], torch.zeros_like(y), y).to(DTYPES[s["out"]])
    if kind == "embgrad":
        kept = s["ids"] >= 0
        g = torch.zeros((s["v"], s["d"]), device="cuda")
        g.index_add_(0, s["ids"][kept], s["dy"][kept].float())
        return (g * s["scale"]).to(DTYPES[s["out"]])
    if kind == "dropout":
        y = _dropout(s)
        r = {"y": y.to(dtype)}
        if s["saved"]:
            r["y8"] = _unpack(*_pack(y.view(-1, s["d"])), s["d"]).to(torch.bfloat16).view(y.shape)
        return r
    if kind == "rotate":
        return {"q": _heads(s["q"].float(), s["w_q"], s).to(dtype), "k": _heads(s["k"].float(), s["w_k"], s).to(dtype)}
    if kind == "rotateback":
        q, k = s["q"], s["k"]
        if s["saved"] == "packed":
            q = _unpack(*q, s["hq"] * s["d"]).view(s["t"], s["hq"], s["d"])
            k = _unpack(*k, s["hk"] * s["d"]).view(s["t"], s["hk"], s["d"])
        dq, dw_q = _heads_backward(s["dq"].float(), q.float(), s["w_q"], s)
        dk, dw_k = _heads_backward(s["dk"].float(), k.float(), s["w_k"], s)
        return {"dq": dq.to(dtype), "dk": dk.to(dtype), "dw_q": dw_q, "dw_k": dw_k}
    if kind == "scan":
        h, last, entering = _scan(s)
        r = {"h": h.to(dtype), "last": last}
        if s["saved"]:
            r["states"] = entering
        return r
    dx, df, dh0 = _scan_backward(s)
    return {"dx": dx.to(dtype), "df": df.to(dtype), "dh0": dh0}


# ---- the framework's calls --------------------------------------------------------------


def _own(s):
    import paper_2504_20437_amd as gl
    kind = s["kind"]
    if kind == "lookup":
        return gl.galore_embedding(s["ids"], s["w"], scale=s["scale"], dtype=DTYPES[s["out"]])
    if kind == "embgrad":
        return gl.galore_embedding_grad(s["ids"], s["dy"], s["v"], scale=s["scale"], dtype=DTYPES[s["out"]])
    if kind == "dropout":
        y, y8 = gl.galore_dropout(s["x"], s["p"], s["seed"], s["index"], residual=s["r"],
                                  checkpoint=True if s["saved"] else None)
        r = {"y": y}
        if s["saved"]:
            r["y8"] = gl.galore_checkpoint_unpack(*y8, s["d"])
        return r
    if kind == "rotate":
        q, k = gl.galore_head_norm(s["q"], s["k"], s["w_q"], s["w_k"], s["table"], s["positions"],
                                   interleaved=s["inter"], eps=EPS)
        return {"q": q, "k": k}
    if kind == "rotateback":
        dq, dk, dw_q, dw_k = gl.galore_head_norm_backward(s["dq"], s["dk"], s["q"], s["k"], s["w_q"], s["w_k"],
                                                          s["table"], s["positions"], interleaved=s["inter"], eps=EPS)
        return {"dq": dq, "dk": dk, "dw_q": dw_q, "dw_k": dw_k}
    if kind == "scan":
        h, last, states = gl.galore_recurrence(s["x"], s["f"], h0=s["h0"], offsets=s["offsets"], states=s["saved"])
        r = {"h": h, "last": last}
        if s["saved"]:
            r["states"] = states
        return r
    dx, df, dh0 = gl.galore_recurrence_backward(s["dh"], s["x"], s["f"], s["states"], h0=s["h0"], dlast=s["dlast"],
                                                offsets=s["offsets"])
    return {"dx": dx, "df": df, "dh0": dh0}


def run(state):
    return _own(state) if own else _plain(state)


# ---- the same from the definitions, in 64 bits ------------------------------------------


def _values64(codes, scales, cols):
    block = torch.arange(cols, device=codes.device) // 32
    return codes.double()[:, :cols] * torch.pow(2.0, scales.double() - 133)[:, block]


def _kept64(c, s):
    """which elements dropout keeps, on the host in unsigned words"""
    b, t, d = s["x"].shape
    word, wide = np.uint64(0xffffffff), np.uint64(32)
    j, i, m = np.meshgrid(np.arange((d + 7) // 8, dtype=np.uint64), np.arange(t, dtype=np.uint64),
                          np.arange(b, dtype=np.uint64), indexing="ij")
    r = [j, i, m, np.full_like(j, s["index"])]
    key = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32]
    for n in range(10):
        left, right = np.uint64(3528531795) * r[0], np.uint64(3449720151) * r[2]
        k = [np.uint64((key[0] + n * 2654435769) % 2 ** 32), np.uint64((key[1] + n * 3144134277) % 2 ** 32)]
        r = [(right >> wide) ^ r[1] ^ k[0], right & word, (left >> wide) ^ r[3] ^ k[1], left & word]
    half = [np.uint64(0), np.uint64(16)]
    u = np.stack([r[e // 2] >> half[e % 2] & np.uint64(0xffff) for e in range(8)], axis=1)   # (groups, 8, t, b)
    u = u.reshape(-1, t, b).transpose(2, 1, 0)[:, :, :d]
    return torch.from_numpy(np.ascontiguousarray(u >= np.uint64(round(65536 * c["p"])))).cuda()


def _angles64(s):
    """cos + i sin of every rotated pair of every token"""
    row = s["table"][s["positions"].long()].double()
    half = row.shape[1] // 2
    return torch.complex(row[:, :half], row[:, half:])[:, None, :]


def _turn64(n, s, turn):
    rot = s["table"].shape[1]
    head, rest = n[..., :rot], n[..., rot:]
    pairs = head.unflatten(-1, (rot // 2, 2)) if s["inter"] else head.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    z = torch.complex(pairs[..., 0].contiguous(), pairs[..., 1].contiguous()) * turn
    pairs = torch.stack((z.real, z.imag), -1)
    head = pairs.flatten(-2) if s["inter"] else pairs.transpose(-1, -2).flatten(-2)
    return torch.cat((head, rest), -1)


def _documents(c, s):
    """(batch row, first token, end) of every sequence"""
    if s["offsets"] is None:
        return [(i, 0, c["t"]) for i in range(c["b"])]
    o = s["offsets"].tolist()
    return [(0, o[i], o[i + 1]) for i in range(len(o) - 1)]


def _scan64(c, s):
    """h of every token, the state before it, and the last states; token by token, all sequences in step"""
    docs = _documents(c, s)
    x = s["x"].double().view(c["b"], c["t"], c["d"])
    f = s["f"].double().view(c["b"], c["t"], c["d"])
    h, before = torch.empty_like(x), torch.empty_like(x)
    state = s["h0"].double().clone() if s["h0"] is not None else x.new_zeros((len(docs), c["d"]))
    rows = torch.tensor([r for r, _, _ in docs], device="cuda")
    starts = torch.tensor([a for _, a, _ in docs], device="cuda")
    order = sorted(range(len(docs)), key=lambda i: docs[i][2] - docs[i][1], reverse=True)
    length = [docs[i][2] - docs[i][1] for i in order]
    order_t = torch.tensor(order, device="cuda")
    n = len(docs)
    for k in range(length[0] if length else 0):
        while length[n - 1] <= k:
            n -= 1
        who = order_t[:n]
        r, at = rows[who], starts[who] + k
        before[r, at] = state[who]
        gate = 1 / (1 + torch.exp(-f[r, at]))
        state[who] = gate * state[who] + (1 - gate) * x[r, at]
        h[r, at] = state[who]
    return h, before, state


def exact(c, seed):
    s = prepare(c, seed)
    kind = c["kind"]
    if kind == "lookup":
        y = s["w"].double()[s["ids"]] * s["scale"]
        y[s["ids"] < 0] = 0
        return y
    if kind == "embgrad":
        order = s["ids"].argsort(stable=True)
        order = order[s["ids"][order] >= 0]
        g = torch.zeros((c["v"], c["d"]), dtype=torch.float64, device="cuda")
        ids, counts = s["ids"][order].unique_consecutive(return_counts=True)
        for part, n, i in zip(order.split(counts.tolist()), counts.tolist(), ids.tolist()):
            g[i] = s["dy"][part].double().sum(0) * s["scale"]
        return g
    if kind == "dropout":
        cut = round(65536 * c["p"])
        y = torch.where(_kept64(c, s), s["x"].double() / (1 - cut / 65536), torch.zeros((), device="cuda", dtype=torch.float64))
        r = {"y": y if s["r"] is None else y + s["r"].double()}
        if c["saved"]:
            r["y8"] = None        # a last bit of y decides between two codes
        return r
    if kind in ("rotate", "rotateback"):
        turn = _angles64(s)
        out = {}
        for name, heads in (("q", c["hq"]), ("k", c["hk"])):
            w = s["w_" + name].double()
            x = s[name]
            x = _values64(*x, heads * c["d"]).view(c["t"], heads, c["d"]) if c.get("saved") == "packed" else x.double()
            norm = torch.sqrt((x ** 2).sum(-1, keepdim=True) / c["d"] + EPS)
            if kind == "rotate":
                out[name] = _turn64(w * (x / norm), s, turn)
                continue
            dn = _turn64(s["d" + name].double(), s, turn.conj())
            out["dw_" + name] = (dn * (x / norm)).flatten(0, 1).sum(0)
            out["d" + name] = dn * w / norm - x * ((dn * w * x).sum(-1, keepdim=True) / (c["d"] * norm ** 3))
        return out
    h, before, last = _scan64(c, s)
    shape = s["x"].shape
    if kind == "scan":
        r = {"h": h.view(shape), "last": last}
        if c["saved"]:
            # what enters a run of STEP tokens: the state after the token before it
            n = -(-c["t"] // STEP)
            states = h.new_zeros((c["b"], n, c["d"]))
            if s["offsets"] is None and s["h0"] is not None:
                states[:, 0] = s["h0"].double()
            for i in range(1, n):
                states[:, i] = h[:, STEP * i - 1]
            r["states"] = states if s["x"].dim() == 3 else states[0]
        return r
    x, f = s["x"].double().view(h.shape), s["f"].double().view(h.shape)
    gate = 1 / (1 + torch.exp(-f))
    dx, df = torch.empty_like(x), torch.empty_like(x)
    dh = s["dh"].double().view(h.shape)
    carry = s["dlast"].double().clone()
    docs = _documents(c, s)
    rows = torch.tensor([r for r, _, _ in docs], device="cuda")
    ends = torch.tensor([e for _, _, e in docs], device="cuda")
    order = sorted(range(len(docs)), key=lambda i: docs[i][2] - docs[i][1], reverse=True)
    length = [docs[i][2] - docs[i][1] for i in order]
    order_t = torch.tensor(order, device="cuda")
    n = len(docs)
    for k in range(length[0] if length else 0):
        while length[n - 1] <= k:
            n -= 1
        who = order_t[:n]
        r, at = rows[who], ends[who] - 1 - k
        g = dh[r, at] + carry[who]
        a = gate[r, at]
        dx[r, at] = (1 - a) * g
        df[r, at] = g * (before[r, at] - x[r, at]) * a * (1 - a)
        carry[who] = a * g
    return {"dx": dx.view(shape), "df": df.view(shape), "dh0": carry}
