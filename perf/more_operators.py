"""What the operators for a residual block of a caller's own cost, and what they compute in plain torch.

  norm        h = x + scale act(gate) N(y), z = N(h): the norms after and before a block fused with its gate and residual scale
  norm_grad   the gradients of all of these from dz and dh
  linear8     y = x W^T in 8-bit integers: x quantised row by row (alone, or as the norm before the projection leaves it), scales per row and channel
  product8    the product alone, of operands that are quantised already
  adamw       one AdamW step over many tensors, states in 32 or in 8 bits

With own = False, run() uses elementary torch operations in 32 bits; with own = True, the library's entry points.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}
_EPS = 1e-6
_B1, _B2, _ADAM_EPS, _LR = 0.9, 0.999, 1e-8, 1e-3


def listed():
    return [
        # one query's row, normalised before its projection
        dict(name="norm_single", kind="norm", n=1, d=256, x="bf16", b="bf16", norm="rms", form="pre", post=False, gate="none", scale=False, bias=False, train=False),
        # the 2 B + N slots of the large-graph batch (B = N = 8,192): a block's output joins the fp32 rows, the next block's input leaves
        dict(name="norm_batch", kind="norm", n=24_576, d=200, x="f32", b="bf16", norm="layer", form="both", post=False, gate="none", scale=True, bias=True, train=True),
        # a text encoder's residual stream, gated, norms on both sides of the block
        dict(name="norm_large", kind="norm", n=32_768, d=4096, x="bf16", b="bf16", norm="rms", form="both", post=True, gate="sigmoid", scale=True, bias=False, train=True),
        # the gradients over the batch's slots
        dict(name="norm_grad_batch", kind="norm_grad", n=24_576, d=256, x="f32", b="bf16", norm="layer", form="both", post=True, gate="silu", scale=True, bias=True),
        # the gradients of the text encoder's residual stream
        dict(name="norm_grad_large", kind="norm_grad", n=16_384, d=4096, x="bf16", b="bf16", norm="rms", form="both", post=True, gate="sigmoid", scale=True, bias=False),
        # one entity's text features projected
        dict(name="linear8_single", kind="linear8", M=1, N=256, K=768, x="bf16", o="bf16", first="quantize", add=False),
        # the projection of a batch's slots, normalised before it, added to their shallow rows
        dict(name="linear8_batch", kind="linear8", M=24_576, N=256, K=768, x="bf16", o="bf16", first="norm", add=True),
        # a large product
        dict(name="product8_large", kind="product8", M=8192, N=4096, K=8192, o="bf16", add=False),
        # the encoder's two matrices and its vectors
        dict(name="adamw_small", kind="adamw", count=8, n=2 * 256 * 768, p="f32", g="f32", bits=32, copy="none"),
        # a hundred tensors of a text encoder with bf16 gradients and a bf16 copy of the weights, states in 8 bits
        dict(name="adamw_many_8bit", kind="adamw", count=100, n=20_000_000, p="f32", g="bf16", bits=8, copy="bf16"),
        # a dense table of 400,000 rows of 256
        dict(name="adamw_large", kind="adamw", count=1, n=400_000 * 256, p="f32", g="f32", bits=32, copy="none"),
        # the same kind of table with states in 8 bits
        dict(name="adamw_large_8bit", kind="adamw", count=1, n=250_000 * 256, p="f32", g="f32", bits=8, copy="none"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["norm", "norm_grad", "linear8", "product8", "adamw"], [24, 22, 22, 12, 20])[0]
    t = lambda: rng.choice(["f32", "bf16", "f16"])
    if kind in ("norm", "norm_grad"):
        d = rng.choice([8 * _log_int(rng, 1, 1024), 8 * _log_int(rng, 1, 1024), _log_int(rng, 3, 8192)])
        n = _log_int(rng, 1, 65_536)
        while n * d > 60_000_000:
            n = max(1, n // 2)
        form = rng.choice(["pre", "post", "both", "both"])
        c = dict(kind=kind, n=n, d=d, x=t(), b=t(), norm=rng.choice(["rms", "layer"]), form=form, post=form != "pre" and rng.random() < 0.6,
                 gate=rng.choice(["none", "sigmoid", "silu", "plain"]) if form != "pre" else "none", scale=form != "pre" and rng.random() < 0.6)
        c["bias"] = c["norm"] == "layer" and rng.random() < 0.7 and (form != "post" or c["post"])
        return dict(c, train=rng.random() < 0.5) if kind == "norm" else c
    if kind in ("linear8", "product8"):
        M, N, K = _log_int(rng, 1, 32_768), _log_int(rng, 16, 8192), _log_int(rng, 32, 16_384)
        while M * N * K > 8192 * 4096 * 8192 // 2 or M * N > 60_000_000 or M * K > 100_000_000:
            M, N, K = max(1, M * 2 // 3), max(16, N * 3 // 4), max(32, K * 3 // 4)
        c = dict(kind=kind, M=M, N=N, K=K, o=t(), add=rng.random() < 0.4)
        if kind == "product8":
            return c
        c["first"] = rng.choice(["quantize", "quantize", "norm"]) if K <= 8192 else "quantize"
        if c["first"] == "norm":
            # (the norm's own last bit decides a value beside the middle of two integers: outputs of 16 bits do not see that)
            c["o"] = rng.choice(["bf16", "f16"])
        return dict(c, x=t())
    return dict(kind=kind, count=_log_int(rng, 1, 120), n=_log_int(rng, 1000, 40_000_000), p=rng.choice(["f32", "f32", "bf16", "f16"]), g=t(), bits=rng.choice([32, 8]),
                copy=rng.choice(["none", "bf16", "f16"]))


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _cdiv(a, b):
    return -(-a // b)


def _rows(gen, rows, cols, dev):
    """Rows of different sizes and columns of different ranges, as activations have."""
    x = torch.randn((rows, cols), generator=gen, device=dev)
    return x.mul_(torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device=dev))).mul_(0.5 + torch.rand((1, cols), generator=gen, device=dev))


def _sizes(c):
    """Matrices and vectors in turn; lengths of every remainder."""
    big = _cdiv(c["count"], 2)
    return [max(1, c["n"] // big + 5 * (i % 7) - 3 * i % 11) if i % 2 == 0 else 1 + (977 * i) % 4096 for i in range(c["count"])] if c["count"] > 1 else [c["n"]]


def _inputs(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    c, s = case, {"case": case, "dev": dev}
    vector = lambda d, mid, spread: torch.randn(d, generator=gen, device=dev).mul_(spread).add_(mid)
    if c["kind"] in ("norm", "norm_grad"):
        n, d, TX, TB = c["n"], c["d"], _TYPES[c["x"]], _TYPES[c["b"]]
        s["x"] = _rows(gen, n, d, dev).add_(0.3).to(TX)
        has_y = c["form"] != "pre"
        s["y"] = _rows(gen, n, d, dev).mul_(0.5).to(TB) if has_y else None
        s["gate"] = torch.randn((n, d), generator=gen, device=dev).mul_(1.5).to(TB) if c["gate"] != "none" else None
        s["w1"] = vector(d, 1.0, 0.2) if c["post"] else None
        s["b1"] = vector(d, 0.0, 0.1) if c["post"] and c["bias"] else None
        s["scale"] = vector(d, 0.1, 0.05) if c["scale"] else None
        s["w2"] = vector(d, 1.0, 0.2) if c["form"] != "post" else None
        s["b2"] = vector(d, 0.0, 0.1) if c["form"] != "post" and c["bias"] else None
        if c["kind"] == "norm_grad":
            s["dz"] = _rows(gen, n, d, dev).mul_(0.01).to(TB) if c["form"] != "post" else None
            s["dh"] = _rows(gen, n, d, dev).mul_(0.01).to(TX)
    elif c["kind"] in ("linear8", "product8"):
        M, N, K = c["M"], c["N"], c["K"]
        s["x"] = _rows(gen, M, K, dev)
        w = torch.randn((N, K), generator=gen, device=dev).mul_(torch.exp(0.3 * torch.randn((N, 1), generator=gen, device=dev)) * K ** -0.5)
        s["w"], s["w_scales"] = _quantize(w)
        s["w"] = _padded(s["w"])
        if c["kind"] == "product8":
            s["a"], s["a_scales"] = _quantize(s.pop("x"))
            s["a"] = _padded(s["a"])
        else:
            s["x"] = s["x"].to(_TYPES[c["x"]])
            s["norm_w"] = vector(K, 1.0, 0.2) if c["first"] == "norm" else None
        s["addend"] = torch.randn((M, N), generator=gen, device=dev).to(_TYPES[c["o"]]) if c["add"] else None
    else:
        # tensors one after the other in flat buffers, each at a multiple of 128 elements; what lies between them is zero and stays so
        sizes = _sizes(c)
        blocks = [_cdiv(k, 128) for k in sizes]
        first = [sum(blocks[:i]) for i in range(len(blocks))]
        nb = sum(blocks)
        s["spans"] = [(128 * f, 128 * f + k) for f, k in zip(first, sizes)]
        ids = torch.repeat_interleave(torch.arange(len(sizes), device=dev), torch.tensor(blocks, device=dev))
        s["tensor_of_block"] = ids
        s["block_in_tensor"] = torch.arange(nb, device=dev) - torch.tensor(first, device=dev)[ids]
        s["decay"] = [0.1 if i % 2 == 0 else 0.0 for i in range(len(sizes))]
        real = (s["block_in_tensor"][:, None] * 128 + torch.arange(128, device=dev)) < torch.tensor(sizes, device=dev)[ids][:, None]
        s["p"] = (torch.randn((nb, 128), generator=gen, device=dev).mul_(0.05) * real).to(_TYPES[c["p"]]).view(-1)
        size = torch.exp(1.0 * torch.randn((nb, 1), generator=gen, device=dev)) * 1e-3          # rows' gradients differ in size
        g = torch.randn((nb, 128), generator=gen, device=dev).mul_(size) * real
        m, v = g * 0.3, (g.abs() * 0.5 + 0.5 * size * real).square_()
        g.add_(torch.randn((nb, 128), generator=gen, device=dev).mul_(0.5 * size) * real)
        s["g"] = g.to(_TYPES[c["g"]]).view(-1)
        if c["bits"] == 32:
            s["m"], s["v"], s["ms"], s["vs"] = m.view(-1), v.view(-1), None, None
        else:
            for name, a, bias, t in (("m", m, 7, torch.float8_e4m3fn), ("v", v, 14, torch.float8_e5m2)):
                top = a.abs().amax(1, keepdim=True)
                scale = torch.where(top > 0, torch.ldexp(torch.ones_like(top), torch.frexp(top)[1] - 1 - bias), torch.ones_like(top))
                s[name], s[name + "s"] = (a / scale).to(t).view(-1), scale.view(-1).contiguous()
        s["copy"] = torch.zeros(nb * 128, dtype=_TYPES[c["copy"]], device=dev) if c["copy"] != "none" else None
        s["step"], s["seed"] = 1000 + seed % 977, (seed * 0x9E3779B97F4A7C15 + 11) % (1 << 63)
    return s


def _padded(q):
    """The same matrix with rows a multiple of 16 bytes apart."""
    rows, cols = q.shape
    wide = torch.zeros((rows, _cdiv(cols, 16) * 16), dtype=q.dtype, device=q.device)
    wide[:, :cols] = q
    return wide[:, :cols]


def prepare(case, seed):
    s, c = _inputs(case, seed), case
    dev = s["dev"]
    if c["kind"] in ("norm", "norm_grad"):
        n, d = c["n"], c["d"]
        has_y, has_z = c["form"] != "pre", c["form"] != "post"
        if c["kind"] == "norm":
            s["h"] = torch.empty((n, d), dtype=_TYPES[c["x"]], device=dev) if has_y else None
            s["z"] = torch.empty((n, d), dtype=_TYPES[c["b"]], device=dev) if has_z else None
            s["stats"] = torch.empty((n, 4), device=dev) if c["train"] else None
        else:
            # what the forward pass left behind: mean and reciprocal deviation of both norms' rows
            s["stats"] = _forward(s, c)[2]
            for name, of in (("dx", "x"), ("dy", "y"), ("dgate", "gate"), ("dw1", "w1"), ("db1", "b1"), ("dscale", "scale"), ("dw2", "w2"), ("db2", "b2")):
                s[name] = torch.empty_like(s[of]) if s[of] is not None else None
    elif c["kind"] in ("linear8", "product8"):
        s["out"] = torch.empty((c["M"], c["N"]), dtype=_TYPES[c["o"]], device=dev)
        if c["kind"] == "linear8":
            s["a"] = torch.empty((c["M"], _cdiv(c["K"], 16) * 16), dtype=torch.int8, device=dev)[:, :c["K"]]
            s["a_scales"] = torch.empty(c["M"], device=dev)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _norm(u, kind):
    """(normalised rows, mean, reciprocal deviation)."""
    mu = u.mean(1, keepdim=True) if kind == "layer" else torch.zeros((u.shape[0], 1), device=u.device, dtype=u.dtype)
    u = u - mu
    r = torch.rsqrt((u * u).mean(1, keepdim=True) + _EPS)
    return u * r, mu, r


def _act(gate, kind):
    """act(g) and its derivative."""
    g = gate.float()
    if kind == "plain":
        return g, torch.ones_like(g)
    sig = torch.sigmoid(g)
    return (sig, sig * (1 - sig)) if kind == "sigmoid" else (g * sig, sig * (1 + g * (1 - sig)))


def _forward(s, c):
    """h, z (in 32 bits) and the statistics [n, 4]: mean and reciprocal deviation of y's rows, then of h's (0 where a norm is not taken)."""
    h, zero = s["x"].float(), torch.zeros((c["n"], 1), device=s["dev"])
    stats = [zero, zero, zero, zero]
    if s["y"] is not None:
        a = s["y"].float()
        if s["w1"] is not None:
            a, stats[0], stats[1] = _norm(a, c["norm"])
            a = a * s["w1"]
            a = a + s["b1"] if s["b1"] is not None else a
        a = a * _act(s["gate"], c["gate"])[0] if s["gate"] is not None else a
        h = h + (a * s["scale"] if s["scale"] is not None else a)
    z = None
    if s["w2"] is not None:
        z, stats[2], stats[3] = _norm(h, c["norm"])
        z = z * s["w2"]
        z = z + s["b2"] if s["b2"] is not None else z
    return h, z, torch.cat(stats, 1)


def _through_norm(c, normed, r, kind):
    """The gradient of a norm's input from c = weight times the gradient of its output."""
    c_mean = c.mean(1, keepdim=True) if kind == "layer" else 0.0
    return r * (c - c_mean - normed * (c * normed).mean(1, keepdim=True))


def _backward(s, c):
    h = _forward(s, c)[0]
    mu1, r1, mu2, r2 = s["stats"].split(1, 1)
    got = dict.fromkeys(("dx", "dy", "dgate", "dw1", "db1", "dscale", "dw2", "db2"))
    dh = s["dh"].float()
    if s["w2"] is not None:
        normed, dz = (h - mu2) * r2, s["dz"].float()
        got["dw2"] = (dz * normed).sum(0)
        got["db2"] = dz.sum(0) if s["b2"] is not None else None
        dh = dh + _through_norm(dz * s["w2"], normed, r2, c["norm"])
    got["dx"] = dh.to(s["x"].dtype)
    if s["y"] is not None:
        normed = (s["y"].float() - mu1) * r1 if s["w1"] is not None else s["y"].float()
        a = normed * s["w1"] if s["w1"] is not None else normed
        a = a + s["b1"] if s["b1"] is not None else a
        e = dh * s["scale"] if s["scale"] is not None else dh
        act = None
        if s["gate"] is not None:
            act, slope = _act(s["gate"], c["gate"])
            got["dgate"] = (e * a * slope).to(s["gate"].dtype)
            e = e * act
        if s["scale"] is not None:
            got["dscale"] = (dh * (a * act if act is not None else a)).sum(0)
        if s["w1"] is not None:
            got["dw1"] = (e * normed).sum(0)
            got["db1"] = e.sum(0) if s["b1"] is not None else None
            e = _through_norm(e * s["w1"], normed, r1, c["norm"])
        got["dy"] = e.to(s["y"].dtype)
    return got


def _quantize(x):
    """8-bit integers and a scale for each row."""
    most = x.abs().amax(1, keepdim=True).float()
    scale = torch.where(most > 0, (most / torch.full_like(most, 127.0)).clamp_(min=2.0 ** -126), torch.ones_like(most))
    # (64 bits: a quotient rounded to 32 falls on the middle of two integers where the true one does not)
    return (x.double() / scale.double()).round_().to(torch.int8), scale[:, 0].contiguous()


def _product(a, sa, b, sb, addend, out_type):
    c = torch.matmul(a.float(), b.float().t()) * sa[:, None] * sb
    return (c if addend is None else c + addend.float()).to(out_type)


def _mul32(a, b):
    """High and low words of the product of a word tensor and a word constant, in int64."""
    low = a * (b & 0xFFFF)
    t = a * (b >> 16) + (low >> 16)
    return t >> 16, ((t & 0xFFFF) << 16) | (low & 0xFFFF)


def _noise(s):
    """The two 16-bit numbers of every element: Philox4x32 with ten rounds, four elements to a counter."""
    at = (s["block_in_tensor"][:, None] * 32 + torch.arange(32, device=s["dev"])).view(-1)
    c0, c1 = at & 0xFFFFFFFF, (s["tensor_of_block"] * 64).repeat_interleave(32) + (at >> 32)
    c2, c3 = torch.full_like(c0, s["step"] & 0xFFFFFFFF), torch.full_like(c0, (1 << 30) + (s["step"] >> 32))
    k0, k1 = s["seed"] & 0xFFFFFFFF, s["seed"] >> 32
    for _ in range(10):
        h0, l0 = _mul32(c0, 0xD2511F53)
        h1, l1 = _mul32(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], 1).view(-1, 128)
    return (words & 0xFFFF).to(torch.int32), (words >> 16).to(torch.int32)


def _rounded(a, half, bits, bias, top):
    """(8-bit values, scales) of rows of 128: powers of two as scales, rounded up where the 16-bit number is at least what is missing."""
    most = a.abs().amax(1, keepdim=True)
    scale = torch.ldexp(torch.ones_like(most), (torch.frexp(most)[1] - 1 - top).clamp_(min=-126))
    scale = torch.where(most > 0, scale, torch.ones_like(scale))
    # as 32-bit patterns whose exponents are the 8-bit type's, the type's subnormal values among their own
    shift = 23 - bits
    code = ((a.abs() / scale) * 2.0 ** (bias - 127)).view(torch.int32)
    code = (code + (half << (shift - 16)) + (1 << (shift - 17))) >> shift
    return code, scale


def _adamw(s, c):
    p, g = s["p"].view(-1, 128).float(), s["g"].view(-1, 128).float()
    m, v = s["m"].view(-1, 128).float(), s["v"].view(-1, 128).float()
    if c["bits"] == 8:
        m, v = m * s["ms"][:, None], v * s["vs"][:, None]
    m = m * _B1 + g * (1 - _B1)
    v = v * _B2 + (g * g) * (1 - _B2)
    t = s["step"] + 1
    keep = torch.tensor([1 - _LR * w for w in s["decay"]], device=s["dev"])[s["tensor_of_block"]][:, None]
    p = p * keep - (_LR / (1 - _B1 ** t)) * m / (torch.sqrt(v) / math.sqrt(1 - _B2 ** t) + _ADAM_EPS)
    s["p"].view(-1, 128).copy_(p)
    if s["copy"] is not None:
        s["copy"].view(-1, 128).copy_(p)
    if c["bits"] == 32:
        s["m"].view(-1, 128).copy_(m)
        s["v"].view(-1, 128).copy_(v)
    else:
        low, high = _noise(s)
        code, scale = _rounded(m, low, 3, 7, 7)
        s["m"].view(torch.uint8).view(-1, 128).copy_(code | (torch.signbit(m).to(torch.int32) << 7))
        s["ms"].copy_(scale[:, 0])
        code, scale = _rounded(v, high, 2, 15, 14)
        s["v"].view(torch.uint8).view(-1, 128).copy_(torch.where(v > 0, code.clamp(min=1), code))       # (a positive one stays positive)
        s["vs"].copy_(scale[:, 0])
    return [s[k] for k in ("p", "m", "v", "ms", "vs", "copy")]


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    if c["kind"] == "norm":
        h, z, stats = _forward(s, c)
        return [h.to(s["x"].dtype) if s["y"] is not None else None, z.to(_TYPES[c["b"]]) if z is not None else None, stats if c["train"] else None]
    if c["kind"] == "norm_grad":
        return _backward(s, c)
    if c["kind"] == "adamw":
        return _adamw(s, c)
    if c["kind"] == "product8":
        return _product(s["a"], s["a_scales"], s["w"], s["w_scales"], s["addend"], _TYPES[c["o"]])
    x = s["x"]
    if c["first"] == "norm":
        x = _norm(x.float(), "rms")[0] * s["norm_w"]
    return _product(*_quantize(x), s["w"], s["w_scales"], s["addend"], _TYPES[c["o"]])


def _run_own(s, c):
    import paper_2211_12281_b200 as K
    act = "plain" if c.get("gate", "none") == "none" else c["gate"]
    if c["kind"] == "norm":
        K.block_norm(s["x"], z=s["z"], pre_weight=s["w2"], pre_bias=s["b2"], y=s["y"], h=s["h"], gate=s["gate"], gate_act=act, post_weight=s["w1"],
                     post_bias=s["b1"], scale=s["scale"], kind=c["norm"], eps=_EPS, stats=s["stats"])
        return [s["h"], s["z"], s["stats"]]
    if c["kind"] == "norm_grad":
        K.block_norm_grad(s["x"], s["stats"], s["dx"], dz=s["dz"], dh=s["dh"], pre_weight=s["w2"], dpre_weight=s["dw2"], dpre_bias=s["db2"], y=s["y"], dy=s["dy"],
                          gate=s["gate"], dgate=s["dgate"], gate_act=act, post_weight=s["w1"], post_bias=s["b1"], dpost_weight=s["dw1"], dpost_bias=s["db1"],
                          scale=s["scale"], dscale=s["dscale"], kind=c["norm"])
        return {k: s[k] for k in ("dx", "dy", "dgate", "dw1", "db1", "dscale", "dw2", "db2")}
    if c["kind"] == "adamw":
        if "optimizer" not in s:       # the object that a training program makes once for its parameters
            cut = lambda a: [None if a is None else a[i:j] for i, j in s["spans"]]
            blocks = lambda a: None if a is None else [a[i // 128:_cdiv(j, 128)] for i, j in s["spans"]]
            s["optimizer"] = K.AdamW(cut(s["p"]), cut(s["g"]), cut(s["m"]), cut(s["v"]), blocks(s["ms"]), blocks(s["vs"]),
                                     copies=None if s["copy"] is None else cut(s["copy"]), weight_decay=s["decay"])
        s["optimizer"].step(s["step"], _LR, beta1=_B1, beta2=_B2, eps=_ADAM_EPS, seed=s["seed"])
        return [s[k] for k in ("p", "m", "v", "ms", "vs", "copy")]
    if c["kind"] == "linear8":
        if c["first"] == "norm":
            K.block_norm(s["x"], z=s["a"], z_scales=s["a_scales"], pre_weight=s["norm_w"], kind="rms", eps=_EPS)
        else:
            K.int8_quantize(s["x"], s["a"], s["a_scales"])
    K.int8_matmul(s["a"], s["a_scales"], s["w"], s["w_scales"], s["out"], addend=s["addend"])
    return s["out"]


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] in ("norm", "norm_grad"):
        n, d, X, B = c["n"], c["d"], _SIZE[c["x"]], _SIZE[c["b"]]
        y, g, z = c["form"] != "pre", c["gate"] != "none", c["form"] != "post"
        vectors = 4 * d * (c["post"] + c["scale"] + z + c["bias"] * (c["post"] + z))
        if c["kind"] == "norm":
            return dict(bytes=n * d * (X * (1 + y) + B * (y + g + z)) + vectors + 16 * n * c["train"], flops=n * d * (4 * z + 4 * c["post"] + 2 * y + 4 * g))
        return dict(bytes=n * d * (X * 3 + B * (2 * y + 2 * g + z)) + 2 * vectors + 16 * n, flops=n * d * (12 * z + 12 * c["post"] + 4 * y + 8 * g))
    if c["kind"] in ("linear8", "product8"):
        M, N, K, O = c["M"], c["N"], c["K"], _SIZE[c["o"]]
        a = M * K * _SIZE[c["x"]] + (4 * K if c["first"] == "norm" else 0) if c["kind"] == "linear8" else M * (K + 4)
        return dict(bytes=a + N * (K + 4) + M * N * O * (2 if c["add"] else 1), flops=2 * M * N * K)
    n, blocks = sum(_sizes(c)), sum(_cdiv(k, 128) for k in _sizes(c))
    states = 16 * n if c["bits"] == 32 else 4 * n + 16 * blocks
    return dict(bytes=n * (2 * _SIZE[c["p"]] + _SIZE[c["g"]] + _SIZE.get(c["copy"], 0)) + states, flops=14 * n)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _norm64(u, layer):
    mu = u.sum(1, keepdim=True) / u.shape[1] * layer
    var = ((u - mu) ** 2).sum(1, keepdim=True) / u.shape[1]
    return mu, 1 / torch.sqrt(var + _EPS)


def _exact_norm(c, s):
    """Forward in 64 bits; the gradients by differentiating it."""
    f = {k: s[k].double() for k in ("x", "y", "gate", "w1", "b1", "scale", "w2", "b2") if s.get(k) is not None}
    grad = c["kind"] == "norm_grad"
    if grad:
        f = {k: v.requires_grad_() for k, v in f.items()}
    layer = 1.0 if c["norm"] == "layer" else 0.0
    with torch.set_grad_enabled(grad):
        h, none = f["x"], torch.zeros((c["n"], 1), dtype=torch.float64, device=s["dev"])
        stats = [none] * 4
        if "y" in f:
            a = f["y"]
            if "w1" in f:
                mu, r = _norm64(a, layer)
                stats[:2] = mu, r
                a = (a - mu) * r * f["w1"] + f.get("b1", 0.0)
            if "gate" in f:
                sig = 1 / (1 + torch.exp(-f["gate"]))
                a = a * {"plain": lambda: f["gate"], "sigmoid": lambda: sig, "silu": lambda: f["gate"] * sig}[c["gate"]]()
            h = h + f.get("scale", 1.0) * a
        z = None
        if "w2" in f:
            mu, r = _norm64(h, layer)
            stats[2:] = mu, r
            z = (h - mu) * r * f["w2"] + f.get("b2", 0.0)
        if not grad:
            return [h if "y" in f else None, z, torch.cat(stats, 1) if c["train"] else None]
        total = (h * s["dh"].double()).sum()
        if z is not None:
            total = total + (z * s["dz"].double()).sum()
        got = dict(zip(f, torch.autograd.grad(total, list(f.values()))))
    return {"d" + k: got.get(k) for k in ("x", "y", "gate", "w1", "b1", "scale", "w2", "b2")}


def _philox_np(index, high, step, seed):
    m, low = np.uint64(32), np.uint64(0xFFFFFFFF)
    x = [index & low, high.astype(np.uint64) + (index >> m), np.full_like(index, step % 2 ** 32), np.full_like(index, 2 ** 30 + step // 2 ** 32)]
    for r in range(10):
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(q >> m) ^ x[1] ^ np.uint64((seed + r * 0x9E3779B9) % 2 ** 32), q & low, (p >> m) ^ x[3] ^ np.uint64((seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32), p & low]
    return np.stack(x, 1).reshape(-1, 128)


def _state64(a, half, mantissa, smallest, top):
    """8-bit values and scales of rows of 128 doubles, rounded up with the probability that the 16-bit number stands for."""
    most = a.abs().amax(1, keepdim=True)
    scale = torch.exp2((torch.floor(torch.log2(most)) - top).clamp(min=-126))
    scale = torch.where(most > 0, scale, torch.ones_like(scale))
    y = a.abs() / scale
    step = torch.exp2(torch.floor(torch.log2(y)).clamp(min=smallest) - mantissa)
    return torch.floor(y / step + (half + 0.5) / 65536) * step * torch.sign(a), scale[:, 0], step


def _exact_adamw(c, s):
    if c["bits"] == 8 and s["p"].numel() > 80_000_000:
        return None
    f32 = lambda x: x.float().double()
    b1, b2 = (float(np.float32(b)) for b in (_B1, _B2))
    o1, o2 = (float(np.float32(1 - b)) for b in (_B1, _B2))
    p, g, m, v = (s[k].view(-1, 128).double() for k in "pgmv")
    if c["bits"] == 8:
        m, v = m * s["ms"].double()[:, None], v * s["vs"].double()[:, None]
    # the moments are numbers of 32 bits: each product and sum is rounded to them, before a state of 8 bits is made of them
    m, v = f32(f32(m * b1) + f32(g * o1)), f32(f32(v * b2) + f32(f32(g * g) * o2))
    t = s["step"] + 1
    keep = torch.tensor([1 - _LR * w for w in s["decay"]], dtype=torch.float64, device=s["dev"])[s["tensor_of_block"]][:, None]
    p = p * keep - _LR / (1 - _B1 ** t) * m / (torch.sqrt(v / (1 - _B2 ** t)) + _ADAM_EPS)
    copy = p.view(-1) if s["copy"] is not None else None
    if c["bits"] == 32:
        return [p.view(-1), m.view(-1), v.view(-1), None, None, copy]
    index = (s["block_in_tensor"].cpu().numpy().astype(np.uint64)[:, None] * np.uint64(32) + np.arange(32, dtype=np.uint64)).reshape(-1)
    high = np.repeat(s["tensor_of_block"].cpu().numpy() * 64, 32)
    words = torch.from_numpy(_philox_np(index, high, s["step"], s["seed"]).astype(np.int64)).to(s["dev"])
    qm, ms, _ = _state64(m, words % 65536, 3, -6, 7)
    qv, vs, least = _state64(v, words // 65536, 2, -14, 14)
    qv = torch.where((v > 0) & (qv == 0), least, qv)
    return [p.view(-1), qm.view(-1), qv.view(-1), ms, vs, copy]


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] in ("norm", "norm_grad"):
        return _exact_norm(c, s)
    if c["kind"] == "adamw":
        return _exact_adamw(c, s)
    if c["kind"] == "product8":
        r = s["a"].double() @ s["w"].double().t() * s["a_scales"].double()[:, None] * s["w_scales"].double()
    else:
        x = s["x"].double()
        if c["first"] == "norm":
            x = x / torch.sqrt((x ** 2).sum(1, keepdim=True) / c["K"] + _EPS) * s["norm_w"].double()
        most = x.abs().amax(1)
        scale = (most / 127).float().double()
        scale = torch.where(most > 0, scale, torch.ones_like(scale))
        r = torch.round(x / scale[:, None]) @ s["w"].double().t() * scale[:, None] * s["w_scales"].double()
    return r + s["addend"].double() if c["add"] else r
