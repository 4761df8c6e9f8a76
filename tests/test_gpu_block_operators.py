"""The operators for a residual block against plain forms in 64 bits: norms around a gated block and their gradients, products in 8-bit
integers, AdamW over many tensors, and a block trained and served with them.  Tolerances count roundings: half a step of the
output's type (eps / 2) for the last one, U = 2^-24 for each fp32 operation before it, carried through the formulas to first order
(and 5 % more, for what is of second order)."""
import math

import numpy as np
import pytest

from test_gpu_row_operators import K, T, U, _check, _gen, _strided, _type  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- norms -----------------------------------------------------------------------------------------------------------

def _depth(d):
    """Additions that one term of a row's sum goes through at most: 8 or 32 in a thread (more where a row is gone over in steps of 1,024), then
    five exchanges, a sum over warps in five, and the products with 1 / d and eps."""
    return 32 + -(-d // 1024) + 12


class Value:
    """Numbers in 64 bits and how far their fp32 form may be off."""

    def __init__(self, v, tol):
        self.v, self.tol = v, tol


def _norm64(T, u, eps, layer, d):
    """(centred, r, relative tolerance of r, mean) of rows of a Value; `centred` is a Value."""
    D = _depth(d) * U
    mu = u.v.mean(1, keepdim=True) * layer
    dmu = (u.tol.mean(1, keepdim=True) + D * u.v.abs().mean(1, keepdim=True)) * layer
    c = Value(u.v - mu, u.tol + dmu + U * (u.v - mu).abs())
    var = (c.v ** 2).mean(1, keepdim=True)
    r = 1 / T.sqrt(var + eps)
    # a sum of squares, each off by 2 |c| tol; rsqrtf is within two units, 4 U; 1/2 of the argument's relative error
    rho = ((c.v.abs() * c.tol).mean(1, keepdim=True) + D * var) * r * r + 6 * U
    return c, r, rho, mu


def _normed(c, r, rho):
    n = c.v * r
    return Value(n, r * c.tol + n.abs() * (rho + U))


def _act64(T, g, kind):
    """act(g) and its derivative, as Values.  The exponent g log2 e of e = 2^(-g log2 e) is off by half a step of itself and the constant's half step: e by
    2 U |g| ln 2 log2 e < 2 U |g| at most, the instruction adds 2^-22.5 < 3 U, the sum U, the reciprocal's unit 2 U; s = 1 / (1 + e) has the share e / (1 + e) < 1
    of what e is off.  The derivative s (1 - s) is off by s's error twice and three roundings, (1 - s) of at most 1."""
    if kind == "plain":
        return Value(g, T.zeros_like(g)), Value(T.ones_like(g), T.zeros_like(g))
    s = 1 / (1 + T.exp(-g))
    off = (6 + 2 * g.abs()) * U
    if kind == "sigmoid":
        return Value(s, off * s), Value(s * (1 - s), (2 * off + 3 * U) * s)
    return Value(g * s, (off + U) * (g * s).abs()), Value(s * (1 + g * (1 - s)), (2 * off + 5 * U) * (1 + g.abs()) * s)


def _block64(T, f, act, eps, layer, d):
    """Forward in 64 bits with tolerances: a dict of Values."""
    zero = T.zeros_like(f["x"])
    o = {"h": Value(f["x"], zero)}
    if f.get("y") is not None:
        yn = Value(f["y"], zero)
        if f.get("w1") is not None:
            c, o["r1"], o["rho1"], o["mu1"] = _norm64(T, yn, eps, layer, d)
            yn = _normed(c, o["r1"], o["rho1"])
            a = Value(yn.v * f["w1"], yn.tol * f["w1"].abs())
            if f.get("b1") is not None:
                a = Value(a.v + f["b1"], a.tol)
            a.tol = a.tol + U * a.v.abs()
        else:
            a = yn
        o["yn"], o["a"] = yn, a
        if f.get("gate") is not None:
            o["act"], o["slope"] = _act64(T, f["gate"], act)
            a = Value(a.v * o["act"].v, a.tol * o["act"].v.abs() + a.v.abs() * o["act"].tol + U * (a.v * o["act"].v).abs())
        o["u"] = a
        s = f["scale"] if f.get("scale") is not None else T.ones((), dtype=T.float64, device="cuda")
        h = f["x"] + s * a.v
        o["h"] = Value(h, (s * a.tol).abs() + U * h.abs())
    if f.get("w2") is not None:
        c, o["r2"], o["rho2"], o["mu2"] = _norm64(T, o["h"], eps, layer, d)
        hn = _normed(c, o["r2"], o["rho2"])
        z = hn.v * f["w2"] + (f["b2"] if f.get("b2") is not None else 0)
        o["hn"], o["z"] = hn, Value(z, hn.tol * f["w2"].abs() + U * z.abs())
    return o


def _through(T, c, n, r, rho, layer, D):
    """r (c - mean(c) - n mean(c n)) of Values c, n."""
    A = Value(c.v.mean(1, keepdim=True) * layer, (c.tol.mean(1, keepdim=True) + D * c.v.abs().mean(1, keepdim=True)) * layer)
    cn = c.v * n.v
    B = Value(cn.mean(1, keepdim=True), (c.tol * n.v.abs() + c.v.abs() * n.tol).mean(1, keepdim=True) + (D + U) * cn.abs().mean(1, keepdim=True))
    v = r * (c.v - A.v - n.v * B.v)
    parts = c.v.abs() + A.v.abs() + (n.v * B.v).abs()
    return Value(v, r * (c.tol + A.tol + n.v.abs() * B.tol + B.v.abs() * n.tol + 4 * U * parts) + v.abs() * (rho + U))


def _block_grad64(T, f, o, act, layer, d, dz, dh):
    D, one = _depth(d) * U, T.ones((), dtype=T.float64, device="cuda")
    n = f["x"].shape[0]
    rows = (n // 592 + 120) * U                   # a row's term: its turn in the CTA, up to 32 teams, the CTAs' sums by eights and the eight
    column = lambda t: Value(t.v.sum(0), t.tol.sum(0) + rows * t.v.abs().sum(0))
    times = lambda a, b, k=1: Value(a.v * b.v, a.tol * b.v.abs() + a.v.abs() * b.tol + k * U * (a.v * b.v).abs())
    exact = lambda v: Value(v, T.zeros_like(v))
    g = {}
    top = exact(dh if dh is not None else T.zeros_like(f["x"]))
    if dz is not None:
        c = times(exact(dz), exact(f["w2"]))
        back = _through(T, c, o["hn"], o["r2"], o["rho2"], layer, D)
        top = Value(top.v + back.v, back.tol + U * (top.v + back.v).abs())
        g["dw2"], g["db2"] = column(times(exact(dz), o["hn"], 0)), column(exact(dz))
    g["dx"] = top
    if f.get("y") is not None:
        s = exact(f["scale"]) if f.get("scale") is not None else exact(one)
        w1 = exact(f["w1"]) if f.get("w1") is not None else exact(one)
        ac, slope = (o["act"], o["slope"]) if "act" in o else (exact(one), exact(one))
        u, e = times(ac, top), times(s, top)
        if "act" in o:
            g["dgate"] = times(times(slope, o["a"]), e)
        S1, S0 = column(times(u, o["yn"], 0)), column(u)
        q = times(times(u, s), w1)
        if f.get("w1") is not None:
            g["dw1"], g["db1"] = times(s, S1), times(s, S0)
            g["dy"] = _through(T, q, o["yn"], o["r1"], o["rho1"], layer, D)
        else:
            g["dy"] = q
        if f.get("scale") is not None:
            ds = times(w1, S1)
            if f.get("b1") is not None:
                b = times(exact(f["b1"]), S0)
                ds = Value(ds.v + b.v, ds.tol + b.tol + U * (ds.v + b.v).abs())
            g["dscale"] = ds
    return g


def _inputs(T, g, n, d, tx, tb, form, post, gate, scale, bias, extra=0, shift=0):
    """Tensors of a block, rows `extra` elements apart."""
    def rows(t, mul=1.0, add=0.0):
        m = _strided(T, n, d, _type(T, t), extra, shift)
        m.copy_(T.randn((n, d), generator=g, device="cuda") * T.exp(0.5 * T.randn((n, 1), generator=g, device="cuda")) * mul + add)
        return m
    vector = lambda mid, spread: T.randn(d, generator=g, device="cuda") * spread + mid
    f = dict(x=rows(tx, 1.0, 0.3), y=None, gate=None, w1=None, b1=None, scale=None, w2=None, b2=None)
    if form != "pre":
        f["y"] = rows(tb, 0.5, -0.1)
        f["gate"] = rows(tb, 1.5) if gate != "none" else None
        f["w1"], f["scale"] = vector(1.0, 0.2) if post else None, vector(0.1, 0.5) if scale else None
        f["b1"] = vector(0.0, 0.2) if post and bias else None
    if form != "post":
        f["w2"], f["b2"] = vector(1.0, 0.2), vector(0.0, 0.2) if bias else None
    return f


def _double(f):
    return {k: v.double() for k, v in f.items() if v is not None}


NORM_CASES = [
    # n, d, x type, block type, form, post, gate, scale, bias, kind
    (1, 1, "f32", "f32", "pre", False, "none", False, True, "rms"), (1, 256, "bf16", "bf16", "pre", False, "none", False, False, "rms"),
    (3, 1, "bf16", "f32", "both", True, "sigmoid", True, True, "layer"), (7, 5, "f32", "f16", "both", True, "silu", True, True, "layer"),
    (33, 8, "f32", "f32", "both", False, "plain", True, False, "rms"), (65, 63, "f16", "f16", "both", True, "sigmoid", False, True, "rms"),
    (100, 64, "f32", "bf16", "post", True, "none", True, False, "layer"), (257, 65, "bf16", "f16", "both", True, "plain", True, True, "layer"),
    (40, 128, "f16", "f32", "post", False, "silu", False, False, "rms"), (19, 129, "f32", "f32", "both", False, "none", False, True, "layer"),
    (1000, 200, "f32", "bf16", "both", False, "none", True, True, "layer"), (31, 256, "bf16", "bf16", "both", True, "silu", True, False, "rms"),
    (9, 257, "f16", "bf16", "pre", False, "none", False, True, "layer"), (50, 512, "f32", "f32", "both", True, "sigmoid", True, True, "layer"),
    (12, 513, "bf16", "bf16", "both", True, "sigmoid", True, True, "rms"), (30, 1000, "f32", "f16", "both", True, "plain", True, False, "layer"),
    (5, 1024, "f32", "f32", "pre", False, "none", False, False, "rms"), (17, 1025, "bf16", "f32", "both", True, "silu", True, True, "layer"),
    (700, 2048, "bf16", "bf16", "both", True, "sigmoid", True, False, "rms"), (6, 4095, "f16", "f16", "both", True, "sigmoid", True, True, "layer"),
    (5, 4096, "f32", "f32", "both", True, "silu", True, True, "layer"), (4, 4104, "f32", "bf16", "both", True, "silu", True, True, "layer"),
    (3, 8192, "bf16", "bf16", "both", True, "plain", True, False, "rms"), (2, 8193, "f32", "f16", "both", True, "sigmoid", True, True, "layer"),
    (70, 96, "bf16", "bf16", "both", True, "silu", True, False, "rms"), (11, 768, "bf16", "f16", "both", True, "sigmoid", True, True, "layer"), (40, 704, "f32", "f32", "both", True, "silu", True, False, "rms"),
    (9, 1200, "f32", "bf16", "both", False, "plain", True, True, "layer"), (160, 1600, "bf16", "bf16", "both", True, "none", False, False, "rms"), (5, 5001, "bf16", "f32", "both", True, "silu", True, True, "layer"),
    (300, 5000, "bf16", "bf16", "both", True, "sigmoid", True, False, "rms"), (2, 6144, "f32", "f32", "post", True, "plain", True, False, "layer"),
    (3, 20_000, "bf16", "f32", "both", True, "silu", True, True, "rms"), (2, 9000, "f16", "f16", "pre", False, "none", False, True, "layer"),
    (70, 50, "f32", "bf16", "both", True, "sigmoid", True, True, "layer"), (9, 100, "bf16", "bf16", "both", True, "silu", True, False, "rms"), (33, 250, "f16", "f32", "pre", False, "none", False, True, "layer"),
    (200, 1002, "bf16", "bf16", "both", True, "sigmoid", True, True, "layer"), (6, 2050, "f32", "f32", "both", True, "plain", True, False, "rms"), (5, 4098, "bf16", "f16", "both", True, "silu", True, True, "layer"),
    (3, 8190, "f32", "bf16", "post", True, "sigmoid", True, True, "layer")]
LAYOUTS = [(0, 0), (8, 8), (3, 1)]


@pytest.mark.parametrize("n,d,tx,tb,form,post,gate,scale,bias,kind", NORM_CASES)
def test_block_norm(T, K, n, d, tx, tb, form, post, gate, scale, bias, kind):
    for extra, shift in LAYOUTS:
        f = _inputs(T, _gen(T, n + d), n, d, tx, tb, form, post, gate, scale, bias, extra, shift)
        o = _block64(T, _double(f), gate, float(np.float32(1e-5)), float(kind == "layer"), d)
        h = _strided(T, n, d, _type(T, tx), extra, shift) if form != "pre" else None
        z = _strided(T, n, d, _type(T, tb), extra, shift) if form != "post" else None
        guards = []
        for out in (h, z):
            if out is not None and extra and n > 1:
                guards.append(out.as_strided((n - 1, extra), (d + extra, 1), out.storage_offset() + d))
                guards[-1].fill_(7.0)
        stats = T.full((n, 4), float("nan"), device="cuda")
        args = dict(pre_weight=f["w2"], pre_bias=f["b2"], y=f["y"], gate=f["gate"], gate_act="plain" if gate == "none" else gate, post_weight=f["w1"],
                    post_bias=f["b1"], scale=f["scale"], kind=kind, eps=1e-5)
        K.block_norm(f["x"], z=z, h=h, stats=stats, **args)
        if h is not None:
            _check(T, h, o["h"].v, 1.05 * o["h"].tol, "h")
        if z is not None:
            _check(T, z, o["z"].v, 1.05 * o["z"].tol, "z")
        assert all((x == 7.0).all() for x in guards)
        for i, name in ((0, "1"), (2, "2")):
            if "r" + name in o:
                r = o["r" + name][:, 0]
                assert ((stats[:, i + 1].double() - r).abs() <= 1.05 * (o["rho" + name][:, 0] + U) * r).all()
                assert kind == "layer" or (stats[:, i] == 0).all()
            else:
                assert (stats[:, i:i + 2] == 0).all()
        # without statistics, with one result alone, and in place: the same bits
        if form == "both":
            h2, z2 = T.empty((n, d), dtype=h.dtype, device="cuda"), T.empty((n, d), dtype=z.dtype, device="cuda")
            for out in (dict(z=z2), dict(h=h2)):
                if extra == 0 and shift == 0:
                    K.block_norm(f["x"], **dict(args, **out))
                    assert T.equal(*((z2, z) if "z" in out else (h2, h)))
            K.block_norm(f["x"], z=f["y"], h=f["x"], **args)
            assert T.equal(f["x"], h) and T.equal(f["y"], z)


@pytest.mark.parametrize("n,d,tx,tb,form,post,gate,scale,bias,kind", NORM_CASES)
def test_block_norm_grad(T, K, n, d, tx, tb, form, post, gate, scale, bias, kind):
    for extra, shift in LAYOUTS:
        g = _gen(T, 3 * n + d)
        f = _inputs(T, g, n, d, tx, tb, form, post, gate, scale, bias, extra, shift)
        more = _inputs(T, g, n, d, tx, tb, "both", False, "none", False, False, extra, shift)
        dz, dh = more["y"] if form != "post" else None, more["x"] if n % 2 == 1 or form == "post" else None
        layer, act = float(kind == "layer"), "plain" if gate == "none" else gate
        f64 = _double(f)
        o = _block64(T, f64, gate, float(np.float32(1e-5)), layer, d)
        want = _block_grad64(T, f64, o, gate, layer, d, dz.double() if dz is not None else None, dh.double() if dh is not None else None)
        stats = T.empty((n, 4), device="cuda")
        outs = dict(z=T.empty((n, d), dtype=_type(T, tb), device="cuda")) if form != "post" else dict(h=T.empty((n, d), dtype=_type(T, tx), device="cuda"))
        args = dict(pre_weight=f["w2"], y=f["y"], gate=f["gate"], gate_act=act, post_weight=f["w1"], post_bias=f["b1"], scale=f["scale"], kind=kind)
        K.block_norm(f["x"], stats=stats, pre_bias=f["b2"], eps=1e-5, **outs, **args)
        of = dict(dx="x", dy="y", dgate="gate", dw1="w1", db1="b1", dscale="scale", dw2="w2", db2="b2")
        name = dict(dw1="dpost_weight", db1="dpost_bias", dw2="dpre_weight", db2="dpre_bias")
        got = {}
        for k, v in of.items():
            if f[v] is not None:
                got[k] = _strided(T, n, d, f[v].dtype, extra, shift) if f[v].dim() == 2 else T.full((d,), float("nan"), device="cuda")
        call = lambda outs, **kw: K.block_norm_grad(f["x"], stats, dz=dz, dh=dh, **{name.get(k, k): v for k, v in outs.items()}, **dict(args, **kw))
        call(got)
        for k, v in got.items():
            _check(T, v, want[k].v, 1.05 * want[k].tol, k)
        vectors = [k for k in got if got[k].dim() == 1]
        # the same bits again; added to what is there; alone
        again = {k: T.full_like(v, float("nan")) for k, v in got.items() if v.dim() == 1 or extra == 0 and shift == 0}
        call(again)
        assert all(T.equal(again[k], got[k]) for k in again)
        if vectors:
            old = {k: T.randn(d, generator=g, device="cuda") for k in vectors}
            sums = {k: v.clone() for k, v in old.items()}
            call(sums, accumulate=True)
            assert all(T.equal(sums[k], old[k] + got[k]) for k in vectors)
        # in place of the operands
        call({k: f[of[k]] for k in got if k in ("dx", "dy", "dgate")})
        assert all(T.equal(f[of[k]], got[k]) for k in got if k in ("dx", "dy", "dgate"))


@pytest.mark.parametrize("d", [64, 256, 1024, 4096])
def test_block_norm_takes_vectors_that_start_anywhere(T, K, d):
    """Vectors between multiples of 16 bytes, beside rows that are not: within the roundings of the aligned ones."""
    n, g = 33, _gen(T, d)
    f = _inputs(T, g, n, d, "bf16", "bf16", "both", True, "silu", True, True)
    dz = T.randn((n, d), generator=g, device="cuda").to(T.bfloat16)
    for k in ("w1", "b1", "scale", "w2", "b2"):
        f[k] = T.cat([f[k][:1], f[k]])[1:]
        assert f[k].data_ptr() % 16 == 4
    o = _block64(T, _double(f), "silu", float(np.float32(1e-6)), 1.0, d)
    z, h, stats = T.empty_like(f["y"]), T.empty_like(f["x"]), T.empty((n, 4), device="cuda")
    args = dict(pre_weight=f["w2"], y=f["y"], gate=f["gate"], gate_act="silu", post_weight=f["w1"], post_bias=f["b1"], scale=f["scale"], kind="layer")
    K.block_norm(f["x"], z=z, h=h, pre_bias=f["b2"], stats=stats, **args)
    _check(T, z, o["z"].v, 1.05 * o["z"].tol, "z")
    _check(T, h, o["h"].v, 1.05 * o["h"].tol, "h")
    want = _block_grad64(T, _double(f), o, "silu", 1.0, d, dz.double(), None)
    out = T.zeros(5 * d + 1, device="cuda")[1:].view(5, d)
    dy = T.empty_like(f["y"])
    K.block_norm_grad(f["x"], stats, dz=dz, dy=dy, dpost_weight=out[0], dpost_bias=out[1], dscale=out[2], dpre_weight=out[3], dpre_bias=out[4], **args)
    for got, k in ((dy, "dy"), (out[0], "dw1"), (out[1], "db1"), (out[2], "dscale"), (out[3], "dw2"), (out[4], "db2")):
        _check(T, got, want[k].v, 1.05 * want[k].tol, k)


@pytest.mark.parametrize("kind,act", [("rms", "plain"), ("layer", "sigmoid"), ("layer", "silu")])
def test_block_norm_grad_against_differences(T, K, kind, act):
    """Central differences of the formula in 64 bits: with steps of 1e-4 they are within 1e-8 times a third derivative (below 100 here) of the slope;
    the kernel's gradients are within 1e-5 of their size (some 100 roundings)."""
    n, d, eps = 3, 6, float(np.float32(1e-5))
    g = _gen(T, 5)
    f = _inputs(T, g, n, d, "f32", "f32", "both", True, act, True, True)
    dz, dh = T.randn((n, d), generator=g, device="cuda"), T.randn((n, d), generator=g, device="cuda")
    f64 = _double(f)

    def loss(f):
        o = _block64(T, f, act, eps, float(kind == "layer"), d)
        return float((o["z"].v * dz.double()).sum() + (o["h"].v * dh.double()).sum())

    stats, z = T.empty((n, 4), device="cuda"), T.empty((n, d), device="cuda")
    args = dict(pre_weight=f["w2"], y=f["y"], gate=f["gate"], gate_act=act, post_weight=f["w1"], post_bias=f["b1"], scale=f["scale"], kind=kind)
    K.block_norm(f["x"], z=z, stats=stats, pre_bias=f["b2"], eps=1e-5, **args)
    got = {k: T.empty_like(f[k]) for k in f}
    K.block_norm_grad(f["x"], stats, got["x"], dz=dz, dh=dh, dy=got["y"], dgate=got["gate"], dpost_weight=got["w1"], dpost_bias=got["b1"], dscale=got["scale"],
                      dpre_weight=got["w2"], dpre_bias=got["b2"], **args)
    for k, v in f64.items():
        flat = v.view(-1)
        for i in range(flat.numel()):
            at = float(flat[i])
            flat[i] = at + 1e-4
            up = loss(f64)
            flat[i] = at - 1e-4
            slope = (up - loss(f64)) / 2e-4
            flat[i] = at
            assert abs(float(got[k].view(-1)[i]) - slope) <= 2e-6 + 1e-5 * max(1.0, float(got[k].abs().max())), (k, i)


@pytest.mark.parametrize("d", [24, 100, 256, 700, 2000, 9000])
def test_block_norm_in_8_bits(T, K, d):
    """z as int8 is what int8_quantize makes of the fp32 z, but for the last bits of that z: scales within them, integers within one where those decide."""
    n = 37
    g = _gen(T, d)
    f = _inputs(T, g, n, d, "bf16", "bf16", "both", True, "sigmoid", True, False)
    args = dict(pre_weight=f["w2"], y=f["y"], gate=f["gate"], gate_act="sigmoid", post_weight=f["w1"], scale=f["scale"], kind="rms", eps=1e-5)
    z8, s8 = T.empty((n, (d + 15) // 16 * 16), dtype=T.int8, device="cuda")[:, :d], T.empty(n, device="cuda")
    h = T.empty((n, d), dtype=T.bfloat16, device="cuda")
    K.block_norm(f["x"], z=z8, z_scales=s8, h=h, **args)
    o = _block64(T, _double(f), "sigmoid", float(np.float32(1e-5)), 0.0, d)
    most, tol = o["z"].v.abs().amax(1), 1.05 * o["z"].tol.amax(1)
    assert ((s8.double() - most / 127).abs() <= (tol + most * U) / 127 * 1.01).all()
    off = (z8.double() - o["z"].v / s8.double()[:, None]).abs()
    assert (off <= 0.5 + 1.05 * o["z"].tol / s8.double()[:, None]).all()
    _check(T, h, o["h"].v, 1.05 * o["h"].tol, "h")
    # a row with a NaN or an infinity stands for NaN, one of zeros for zeros
    x = T.randn((4, d), generator=g, device="cuda")
    x[1], x[2, d // 2], x[3, d - 1] = 0.0, float("nan"), float("inf")
    z8, s8 = z8[:4], s8[:4]
    K.block_norm(x, z=z8, z_scales=s8, pre_weight=T.ones(d, device="cuda"))
    v = z8.float() * s8[:, None]
    assert T.isfinite(v[0]).all() and (v[1] == 0).all() and T.isnan(v[2:]).all()


def test_block_norm_of_hard_rows(T, K):
    """A mean far from zero, rows of zeros, infinities and NaNs that stay in their rows, values at the ends of the range."""
    for d in (40, 250, 600, 3000, 10_000):
        w = T.ones(d, device="cuda")
        x = T.randn((6, d), device="cuda", generator=_gen(T, d))
        x[1] = x[1] * 0.01 + 1000.0
        x[2] = 0.0
        x[3, 1], x[4, d - 1] = float("inf"), float("nan")
        x[5] *= 1e-30
        z = T.empty_like(x)
        K.block_norm(x, z=z, pre_weight=w, kind="layer", eps=1e-5)
        good = T.tensor([0, 1, 2, 5], device="cuda")
        o = _block64(T, dict(x=x[good].double(), w2=w.double()), "none", float(np.float32(1e-5)), 1.0, d)
        _check(T, z[good], o["z"].v, 1.05 * o["z"].tol, d)
        assert (z[2] == 0).all() and T.isnan(z[3:5]).all()


@pytest.mark.parametrize("d", [200, 600, 5000])
def test_block_norm_of_no_rows(T, K, d):
    x, w = T.empty((0, d), device="cuda"), T.ones(d, device="cuda")
    K.block_norm(x, z=T.empty_like(x), pre_weight=w)
    dw = T.full((d,), 3.0, device="cuda")
    K.block_norm_grad(x, T.empty((0, 4), device="cuda"), T.empty_like(x), dz=x, pre_weight=w, dpre_weight=dw, accumulate=True)
    assert (dw == 3).all()
    K.block_norm_grad(x, T.empty((0, 4), device="cuda"), T.empty_like(x), dz=x, pre_weight=w, dpre_weight=dw)
    assert (dw == 0).all()


def test_block_norm_beyond_two_to_the_31_elements(T, K):
    n, d = 8_400_000, 256
    x = T.empty((n, d), dtype=T.bfloat16, device="cuda")
    x.view(-1)[:1 << 20].normal_()
    rows = T.arange(0, n, 4096, device="cuda")
    x.fill_(1.0)
    x[-5:] = T.arange(d, device="cuda") / 16.0
    x[8_388_607:8_388_609] = 3.0 - T.arange(d, device="cuda") / 8.0
    w = T.linspace(0.5, 1.5, d, device="cuda")
    stats = T.empty((n, 4), device="cuda")
    z = T.empty_like(x)
    K.block_norm(x, z=z, pre_weight=w, kind="rms", eps=1e-5, stats=stats)
    at = T.cat([rows, T.tensor([8_388_606, 8_388_607, 8_388_608, n - 6, n - 5, n - 1], device="cuda")])
    o = _block64(T, dict(x=x[at].double(), w2=w.double()), "none", float(np.float32(1e-5)), 0.0, d)
    _check(T, z[at], o["z"].v, 1.05 * o["z"].tol)
    dw = T.empty(d, device="cuda")
    K.block_norm_grad(x, stats, x, dz=z, pre_weight=w, dpre_weight=dw)
    hn = T.ones(d, dtype=T.float64, device="cuda") / math.sqrt(1 + float(np.float32(1e-5)))
    want = (n - 7) * hn * z[0].double()               # all but seven rows are the same
    for i in (8_388_607, 8_388_608, *range(n - 5, n)):
        row = (x[0].double() * 0 + (T.arange(d, device="cuda").double() / 16 if i >= n - 5 else 3 - T.arange(d, device="cuda").double() / 8))
        row = row.to(T.bfloat16).double()
        want = want + z[i].double() * row / T.sqrt((row ** 2).mean() + float(np.float32(1e-5)))
    # rows are added 1,774 to a team, eight teams, 592 CTAs by eights
    assert ((dw.double() - want).abs() <= (1774 + 8 + 74 + 8 + 60) * U * n * z[0].double().abs().clamp(min=1)).all()


# ---- 8-bit integers --------------------------------------------------------------------------------------------------

def _int8(T, rows, cols, extra=0):
    return T.zeros((rows, (cols + 15) // 16 * 16 + extra), dtype=T.int8, device="cuda")[:, :cols]


def _quantized64(T, x):
    most = x.double().abs().amax(1)
    s = T.where(most > 0, (most / 127).float().clamp(min=2.0 ** -126), T.ones((), device="cuda"))
    return T.round(x.double() / s.double()[:, None]).to(T.int8), s


@pytest.mark.parametrize("tx", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,extra,shift", [(1, 1, 0, 0), (1, 768, 0, 0), (5, 7, 0, 0), (33, 8, 8, 0), (100, 100, 3, 1), (64, 1023, 0, 0), (9, 1024, 0, 0), (17, 1025, 0, 1),
                                                   (7, 4096, 0, 0), (3, 8192, 8, 8), (5, 8193, 0, 0), (2, 30_001, 1, 0), (3000, 256, 0, 0)])
def test_int8_quantize(T, K, tx, rows, cols, extra, shift):
    g = _gen(T, rows + cols)
    x = _strided(T, rows, cols, _type(T, tx), extra, shift)
    x.copy_(T.randn((rows, cols), generator=g, device="cuda") * T.exp(2 * T.randn((rows, 1), generator=g, device="cuda")))
    # every other row full of middles: the largest value is 127 times a power of two, the others (k + 1/2) times that
    halves = (T.randint(-127, 127, (rows, cols), generator=g, device="cuda") + 0.5) * 0.25
    x[::2] = halves[::2].to(x.dtype)
    x[::2, cols // 2] = 127 * 0.25
    if rows > 4:
        x[3] = 0.0
    q, s = _int8(T, rows, cols, 16), T.full((rows,), float("nan"), device="cuda")
    wide = q.as_strided((rows, q.stride(0)), (q.stride(0), 1))
    wide[:, cols:] = 77
    K.int8_quantize(x, q, s)
    wq, ws = _quantized64(T, x)
    assert T.equal(q, wq) and T.equal(s, ws) and (wide[:, cols:] == 77).all()


def test_int8_quantize_at_the_ends_of_the_range(T, K):
    for t in (T.float32, T.bfloat16):
        x = T.zeros((6, 40), device="cuda", dtype=t)
        x[0, 3], x[1, 39], x[2, 0] = float("inf"), float("nan"), -float("inf")
        x[0, 4] = float("nan")
        x[3] = T.linspace(-1, 1, 40, device="cuda") * 1e-40                    # below the normal numbers
        x[4] = T.linspace(-1, 1, 40, device="cuda") * 3e38
        x[5] = T.linspace(-1, 1, 40, device="cuda") * 2.0 ** -125
        q, s = _int8(T, 6, 40), T.empty(6, device="cuda")
        K.int8_quantize(x, q, s)
        assert T.isnan(q[:3].float() * s[:3, None]).all()
        wq, ws = _quantized64(T, x[3:])
        assert T.equal(q[3:], wq) and T.equal(s[3:], ws)


PRODUCTS = [
    # M, N, K, out, addend, extra columns of out, shift
    (1, 1, 1, "f32", False, 0, 0), (1, 256, 768, "bf16", False, 0, 0), (1, 4096, 4096, "f32", True, 0, 0), (3, 17, 33, "f16", True, 1, 1), (16, 1000, 2048, "bf16", True, 0, 0),
    (128, 128, 128, "f32", True, 0, 0), (129, 127, 130, "f32", True, 3, 0), (200, 64, 16_000, "bf16", False, 0, 0), (1000, 1001, 100, "bf16", True, 0, 0),
    (1000, 1002, 100, "f16", True, 0, 0), (4096, 256, 768, "f32", True, 0, 0), (5000, 777, 512, "bf16", True, 1, 1), (24_576, 256, 768, "bf16", True, 0, 0),
    (2500, 4096, 2048, "f32", False, 0, 0), (4096, 4095, 4096, "bf16", True, 0, 0), (4100, 4096, 2050, "bf16", False, 8, 8), (65, 8192, 8000, "f16", False, 0, 0),
    (20_000, 70, 300, "f32", False, 2, 0), (40_000, 512, 64, "bf16", False, 0, 0), (8192, 2048, 3000, "f32", True, 4, 4),
    (200, 8000, 1500, "f16", True, 1, 0), (16_384, 512, 512, "bf16", True, 0, 0), (9800, 222, 2500, "bf16", True, 0, 0), (250, 9999, 9000, "f32", True, 1, 1), (3001, 300, 3000, "bf16", True, 1, 1)]


@pytest.mark.parametrize("M,N,Kd,to,add,extra,shift", PRODUCTS)
def test_int8_matmul(T, K, M, N, Kd, to, add, extra, shift):
    g = _gen(T, M + N + Kd)
    a, b = _int8(T, M, Kd), _int8(T, N, Kd, 32)
    a.copy_(T.randint(-128, 128, (M, Kd), generator=g, device="cuda", dtype=T.int8))
    b.copy_(T.randint(-128, 128, (N, Kd), generator=g, device="cuda", dtype=T.int8))
    b.as_strided((N, b.stride(0) - Kd), (b.stride(0), 1), Kd).fill_(99)                 # what lies between the rows is not read
    sa, sb = (T.rand(k, generator=g, device="cuda") * 0.01 + 1e-4 for k in (M, N))
    out = _strided(T, M, N, _type(T, to), extra, shift)
    addend = _strided(T, M, N, _type(T, to), extra, shift)
    addend.copy_(T.randn((M, N), generator=g, device="cuda") * 10)
    if extra and M > 1:
        guard = out.as_strided((M - 1, extra), (N + extra, 1), out.storage_offset() + N)
        guard.fill_(7.0)
    status = T.zeros(1, dtype=T.int32, device="cuda")
    K.int8_matmul(a, sa, b, sb, out, addend=addend if add else None, status=status)
    total = a.double() @ b.double().t()                 # exact: below 2^53
    want = total * sa.double()[:, None] * sb.double()
    tol = want.abs() * 3 * U                            # to fp32, two products
    if add:
        want = want + addend.double()
        tol = tol + want.abs() * U
    _check(T, out, want, 1.01 * tol)
    assert status.item() == 0
    if extra and M > 1:
        assert (guard == 7.0).all()
    if add:                                             # in place of the addend: the same bits
        K.int8_matmul(a, sa, b, sb, addend, addend=addend)
        assert T.equal(addend, out)
    else:
        again = T.empty((M, N), dtype=out.dtype, device="cuda")
        K.int8_matmul(a, sa, b, sb, again)
        assert T.equal(again, out)


def test_int8_matmul_sums_up_to_the_last_bit(T, K):
    """131,071 products of the largest magnitude fill 32 bits, and sums of any order and any share of K are the same."""
    Kd = 131_071
    for M, N in ((1, 8), (130, 200), (300, 40)):
        a, b = _int8(T, M, Kd), _int8(T, N, Kd)
        a.fill_(-128)
        b.fill_(-128)
        b[1] = 127
        out = T.empty((M, N), device="cuda")
        K.int8_matmul(a, T.ones(M, device="cuda"), b, T.ones(N, device="cuda"), out)
        want = T.full((M, N), 128.0 * 128 * Kd, dtype=T.float64, device="cuda")
        want[:, 1] = -128.0 * 127 * Kd
        assert T.equal(out, want.float())
        with pytest.raises(K.KgeError) as e:
            K.int8_matmul(_int8(T, M, Kd + 1), T.ones(M, device="cuda"), _int8(T, N, Kd + 1), T.ones(N, device="cuda"), out)
        assert e.value.code == -5


@pytest.mark.parametrize("M,N,Kd", [(5, 40, 64), (4, 300, 4096), (700, 600, 256), (4500, 4200, 2048)])
def test_int8_matmul_of_scales_far_from_one(T, K, M, N, Kd):
    g = _gen(T, M)
    a, b = _int8(T, M, Kd), _int8(T, N, Kd)
    a.copy_(T.randint(-127, 128, (M, Kd), generator=g, device="cuda", dtype=T.int8))
    b.copy_(T.randint(-127, 128, (N, Kd), generator=g, device="cuda", dtype=T.int8))
    for one, other in ((1e-30, 1e30), (1e36, 1e-36), (2.0 ** -126, 2.0 ** 100), (1e-25, 1e-25), (1e25, 1e20)):
        sa, sb = T.full((M,), one, device="cuda"), T.full((N,), other, device="cuda")
        out = T.empty((M, N), device="cuda")
        K.int8_matmul(a, sa, b, sb, out)
        want = (a.double() @ b.double().t()) * sa.double()[0] * sb.double()[0]
        if one * other > 1e38:
            assert T.equal(out, T.where(want == 0, want, want.sign() * float("inf")).float())
        else:
            _check(T, out, want, want.abs() * 3.03 * U)
    sa, sb = T.ones(M, device="cuda"), T.ones(N, device="cuda")
    sa[M // 2], sb[N - 1] = float("inf"), float("nan")
    a[M // 2] = 0
    b[N - 1] = 0
    K.int8_matmul(a, sa, b, sb, out)
    nan = T.isnan(out)
    assert nan[M // 2].all() and nan[:, N - 1].all() and int(nan.sum()) == M + N - 1


def test_int8_waits_that_run_out_are_reported(T, K):
    ran_out = False
    for M, N, Kd in ((1, 4096, 4096), (24_576, 256, 768), (4096, 4096, 4096), (20_000, 64, 300), (16_384, 512, 512)):
        g = _gen(T, M)
        a, b = _int8(T, M, Kd), _int8(T, N, Kd)
        a.copy_(T.randint(-127, 128, (M, Kd), generator=g, device="cuda", dtype=T.int8))
        b.copy_(T.randint(-127, 128, (N, Kd), generator=g, device="cuda", dtype=T.int8))
        sa, sb = T.ones(M, device="cuda"), T.ones(N, device="cuda")
        out, status = T.empty((M, N), device="cuda"), T.zeros(1, dtype=T.int32, device="cuda")
        K.int8_matmul(a, sa, b, sb, out, status=status)
        want = out.clone()
        assert status.item() == 0
        try:
            for tries in (1, 1, 1, 2, 4, 16, 64):
                assert K.lib().kge_debug_set_product_wait_limit(tries) == 0
                K.int8_matmul(a, sa, b, sb, out, status=status)
                assert status.item() in (0, -11)
                ran_out |= status.item() != 0
                if status.item() == 0:
                    assert T.equal(out, want)
                status.zero_()
        finally:
            K.lib().kge_debug_set_product_wait_limit(0)
        out.fill_(float("nan"))
        K.int8_matmul(a, sa, b, sb, out, status=status)
        assert status.item() == 0 and T.equal(out, want)
    assert ran_out


# ---- AdamW -----------------------------------------------------------------------------------------------------------

def _words(n, index, step, seed):
    """The 32-bit words of elements 0 .. n - 1 of the index-th tensor: Philox4x32-10, four elements to a counter."""
    m, low = np.uint64(32), np.uint64(0xFFFFFFFF)
    at = np.arange((n + 3) // 4, dtype=np.uint64)
    x = [at & low, np.uint64(64 * index) + (at >> m), np.full_like(at, step % 2 ** 32), np.full_like(at, 2 ** 30 + step // 2 ** 32)]
    for r in range(10):
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(q >> m) ^ x[1] ^ np.uint64((seed + r * 0x9E3779B9) % 2 ** 32), q & low, (p >> m) ^ x[3] ^ np.uint64((seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32), p & low]
    return np.stack(x, 1).reshape(-1)[:n]


def _blocks(T, a):
    """[blocks of 128, 128], zeros behind the end."""
    return T.nn.functional.pad(a.reshape(-1), (0, -a.numel() % 128)).view(-1, 128)


def _round8(T, a, half, mantissa, smallest, top):
    """Values (in 64 bits) and scales [blocks] of a state in 8 bits."""
    n = a.numel()
    w = _blocks(T, a)
    half = _blocks(T, T.from_numpy(half.astype(np.float64)).to(a.device))
    most = w.abs().amax(1, keepdim=True)
    scale = T.where(most > 0, T.exp2((T.floor(T.log2(most)) - top).clamp(min=-126)), T.ones_like(most))
    y = w.abs() / scale
    step = T.exp2(T.floor(T.log2(y)).clamp(min=smallest) - mantissa)
    return (T.floor(y / step + (half + 0.5) / 65536) * step * T.sign(w)).view(-1)[:n], scale[:, 0], step.view(-1)[:n]


def _values(T, q, scales):
    n = q.numel()
    return q.float().view(-1) * scales.repeat_interleave(128)[:n]


def _adamw64(T, p, g, m, v, i, lr, b1, b2, eps, wd, step, seed, bits, gs=1.0):
    """(p, its tolerance, m, v, m as stored with scales, v as stored with scales)."""
    f = lambda x: x.float().double()
    f1, o1, f2, o2 = (float(np.float32(x)) for x in (b1, 1 - b1, b2, 1 - b2))
    g = f(g.double() * float(np.float32(gs)))
    m = f(f(m.double() * f1) + f(g * o1))
    v = f(f(v.double() * f2) + f(f(g * g) * o2))
    t = step + 1
    change = lr / (1 - b1 ** t) * m / (T.sqrt(v / (1 - b2 ** t)) + float(np.float32(eps)))
    new = p.double() * (1 - lr * wd) - change
    # 1 - lr wd, its product, the final sum; of the change: the square root's instruction (2^-23, two units), the constant it is multiplied by and their sum
    # with eps (one each), the reciprocal's instruction (two), the product with m, lr / (1 - b1^t) (one each)
    tol = U * (2 * p.double().abs() + 8 * change.abs() + new.abs())
    if bits == 32:
        return new, tol, m, v, None, None
    w = _words(p.numel(), i, step, seed)
    qm = _round8(T, m, w & 0xFFFF, 3, -6, 7)
    qv = _round8(T, v, w >> 16, 2, -14, 14)
    qv = (T.where((v > 0) & (qv[0] == 0), qv[2], qv[0]), qv[1])
    return new, tol, m, v, qm[:2], qv


def _states(T, g, sizes, bits, shift=0):
    m, v, ms, vs = [], [], [], []
    for n in sizes:
        a = T.randn(n, generator=g, device="cuda") * 1e-3
        b = (T.randn(n, generator=g, device="cuda") * 1e-3).square_() + 1e-12
        if bits == 32:
            m.append(T.zeros(n + shift, device="cuda")[shift:].copy_(a))
            v.append(T.zeros(n + shift, device="cuda")[shift:].copy_(b))
        else:
            for x, to, scales, t, top in ((a, m, ms, T.float8_e4m3fn, 7), (b, v, vs, T.float8_e5m2, 14)):
                most = _blocks(T, x).abs().amax(1) if n else T.zeros(0, device="cuda")
                s = T.exp2(T.floor(T.log2(most.clamp(min=1e-30))) - top)
                q = T.zeros(n + shift, device="cuda", dtype=T.uint8)[shift:]
                q.copy_((_blocks(T, x) / s[:, None]).view(-1)[:n].to(t).view(T.uint8))
                to.append(q.view(t))
                scales.append(s.contiguous())
    return m, v, (ms if bits == 8 else None), (vs if bits == 8 else None)


SIZES = [1, 127, 0, 128, 129, 4095, 4096, 4097, 2048, 100_003]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("tp,tg,copy,shift,sizes,step,gs", [
    ("f32", "f32", None, 0, SIZES, 0, 1.0), ("f32", "bf16", "bf16", 0, SIZES, 7, 0.5), ("bf16", "bf16", None, 0, SIZES, 999, 1.0), ("f16", "f32", "bf16", 0, [5000], 3, 0.1),
    ("f32", "f16", "f16", 1, SIZES, 12_345_678_901, 1.0), ("bf16", "f32", "f16", 3, SIZES, 1, 1.0), ("f32", "f32", None, 0, [300 + 7 * i for i in range(41)], 50, 1.0),
    ("f32", "f32", "bf16", 0, [1 + i % 400 for i in range(1000)], 2, 2.0), ("f32", "bf16", None, 0, [200 + 9 * i for i in range(30)], 4, 1.0)])
def test_adamw(T, K, bits, tp, tg, copy, shift, sizes, step, gs):
    g = _gen(T, len(sizes) + step % 1000)
    at = lambda n, t: T.zeros(n + shift, dtype=_type(T, t), device="cuda")[shift:]
    params = [at(n, tp).copy_(T.randn(n, generator=g, device="cuda") * 0.05) for n in sizes]
    grads = [at(n, tg).copy_(T.randn(n, generator=g, device="cuda") * 1e-3) for n in sizes]
    if len(sizes) > 5:
        grads[4] = None
    m, v, ms, vs = _states(T, g, sizes, bits, shift)
    copies = [at(n, copy) for n in sizes] if copy else None
    decay = [0.1 if i % 3 else 0.0 for i in range(len(sizes))]
    lr, b1, b2, eps, seed = 1e-3, 0.9, 0.95, 1e-6, 0x123456789ABCDEF5
    old = [x.clone() for x in params]
    state = lambda i: (m[i], v[i]) if bits == 32 else (_values(T, m[i], ms[i]), _values(T, v[i], vs[i]))
    want = [None if grads[i] is None else _adamw64(T, params[i], grads[i], *state(i), i, lr, b1, b2, eps, decay[i], step, seed, bits, gs) for i in range(len(sizes))]
    before = [x.clone() for x in m]
    K.AdamW(params, grads, m, v, ms, vs, copies=copies, weight_decay=decay).step(step, lr, beta1=b1, beta2=b2, eps=eps, seed=seed, grad_scale=gs)
    for i, x in enumerate(want):
        if x is None:
            assert T.equal(params[i], old[i]) and T.equal(m[i].view(T.uint8), before[i].view(T.uint8))
            continue
        if sizes[i] == 0:
            continue
        _check(T, params[i], x[0], x[1], f"p{i}")
        if copies:
            _check(T, copies[i], x[0], x[1], f"copy{i}")
        if bits == 32:
            assert T.equal(m[i].double(), x[2]) and T.equal(v[i].double(), x[3])
        else:
            for q, s, (wq, ws) in ((m[i], ms[i], x[4]), (v[i], vs[i], x[5])):
                assert T.equal(s.double(), ws)
                differ = q.double() != wq
                # a value that is subnormal in 8 bits is one in the kernel's fp32 pattern too, rounded there at 2^-20 (m; v: 2^-21) of the type's last unit: a decision nearer than half
                # of that to its border may fall the other way, with a probability of 2^-20 an element (ten times that many are let pass, and two)
                assert int(differ.sum()) <= 2 + sizes[i] // 100_000


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_from_nothing_and_on_device_numbers(T, K, bits):
    """The first steps from zero states; captured with the step, the rate and the gradients' factor on the device, replays are the eager calls."""
    sizes = [1000, 37, 4500]
    g = _gen(T, 9)
    start = [T.randn(n, generator=g, device="cuda") for n in sizes]
    grads = [T.randn(n, generator=g, device="cuda") for n in sizes]

    def fresh():
        z = (lambda n, t: T.zeros(n, dtype=t, device="cuda"))
        m = [z(n, T.float32 if bits == 32 else T.float8_e4m3fn) for n in sizes]
        v = [z(n, T.float32 if bits == 32 else T.float8_e5m2) for n in sizes]
        s = [None if bits == 32 else [z((n + 127) // 128, T.float32) for n in sizes] for _ in range(2)]
        p = [x.clone() for x in start]
        return p, m, v, s, K.AdamW(p, grads, m, v, s[0], s[1], weight_decay=0.1)

    p, m, v, s, opt = fresh()
    for k in range(4):
        opt.step(10 + k, 1e-2 * 0.5 ** k, seed=3, grad_scale=0.25)
    p2, m2, v2, s2, opt2 = fresh()
    step, lr, gs = T.zeros(1, dtype=T.int64, device="cuda"), T.ones(1, device="cuda"), T.full((1,), 0.25, device="cuda")
    graph = T.cuda.CUDAGraph()
    with T.cuda.graph(graph):
        opt2.step(10, 1e-2, seed=3, step_dev=step, lr_dev=lr, grad_scale_dev=gs)
        step.add_(1)
        lr.mul_(0.5)
    for _ in range(4):
        graph.replay()
    for i in range(len(sizes)):
        # the same doubles on both sides, expm1 within a unit of theirs: one rounding to fp32 apart at most, in each of four steps
        assert ((p2[i] - p[i]).abs() <= 4 * 4 * U * (start[i].abs() + 0.1)).all()
        assert T.equal(m2[i].view(T.uint8), m[i].view(T.uint8)) and T.equal(v2[i].view(T.uint8), v[i].view(T.uint8))
    one = fresh()
    one[4].step(0, 0.01, eps=1e-8, seed=1)
    for i in range(len(sizes)):        # m / (1 - b1) is the gradient itself, so the first step moves each element by lr, but for the decay
        assert ((one[0][i] - start[i] * (1 - 0.01 * 0.1) + 0.01 * grads[i].sign()).abs() <= 1e-6 + 0.01 * 1e-8 / grads[i].abs()).all()


def test_adamw_refuses_tensors_that_overlap(T, K):
    flat, g = T.zeros(4096, device="cuda"), T.zeros(1000, device="cuda")
    p, m, v = flat[:1000], flat[1000:2000], flat[2000:3000]
    K.AdamW([p], [g], [m], [v]).step(0, 0.1)
    K.AdamW([p], [flat[3000:4000]], [m], [v]).step(0, 0.1)
    for bad in (lambda: K.AdamW([p], [g], [flat[999:1999]], [v]), lambda: K.AdamW([p, p], [g, g], [m, flat[3000:4000]], [v, T.zeros(1000, device="cuda")]),
                lambda: K.AdamW([p], [p], [m], [v]), lambda: K.AdamW([p], [flat[2999:3999]], [m], [v]), lambda: K.AdamW([p], [g], [m], [v]).set_grads([m]),
                lambda: K.AdamW([p], [g], [m], [v]).set_grads([g, g]), lambda: K.AdamW([], [g], [], []), lambda: K.AdamW([p], [g.double()], [m], [v]),
                lambda: K.AdamW([p], [g.cpu()], [m], [v])):
        with pytest.raises(K.KgeError) as e:
            bad()
        assert e.value.code == -1
    K.AdamW([], [], [], []).step(0, 0.1)


def test_adamw_rounds_right_on_average(T, K):
    """What a state in 8 bits is on average over elements (and so over steps) is what it would be in 32: within five standard deviations."""
    n = 1 << 20
    p, grad = T.zeros(n, device="cuda"), T.full((n,), 1.1e-3, device="cuda")
    m, v = T.zeros(n, dtype=T.float8_e4m3fn, device="cuda"), T.zeros(n, dtype=T.float8_e5m2, device="cuda")
    ms, vs = T.zeros(n // 128, device="cuda"), T.zeros(n // 128, device="cuda")
    opt = K.AdamW([p], [grad], [m], [v], [ms], [vs])
    wm, wv, var_m, var_v = 0.0, 0.0, 0.0, 0.0
    for k in range(60):
        opt.step(k, 0.0, seed=77)
        wm, wv = 0.9 * wm + 0.1 * 1.1e-3, 0.999 * wv + 0.001 * 1.1e-3 ** 2
        # a rounding moves a value by less than a step (an eighth, a quarter of it), and what moved it fades
        var_m, var_v = 0.81 * var_m + (1.3 * wm / 8) ** 2 / 4, 0.998 * var_v + (1.5 * wv / 4) ** 2 / 4
    am, av = float(_values(T, m, ms).double().mean()), float(_values(T, v, vs).double().mean())
    assert abs(am - wm) <= 5 * math.sqrt(var_m / n) + 2.0 ** -16 * wm * 10
    assert abs(av - wv) <= 5 * math.sqrt(var_v / n) + 2.0 ** -16 * wv * 60


def test_adamw_keeps_trouble_in_its_block(T, K):
    n = 1000
    g = _gen(T, 3)
    p, grad = T.randn(n, generator=g, device="cuda"), T.randn(n, generator=g, device="cuda")
    grad[200], grad[700] = float("nan"), float("inf")
    grad[300] = 0.0
    m, v = T.zeros(n, dtype=T.float8_e4m3fn, device="cuda"), T.zeros(n, dtype=T.float8_e5m2, device="cuda")
    ms, vs = T.zeros(8, device="cuda"), T.zeros(8, device="cuda")
    old = p.clone()
    K.AdamW([p], [grad], [m], [v], [ms], [vs]).step(0, 0.1, seed=1)
    bad = T.zeros(n, dtype=T.bool, device="cuda")
    bad[[200, 700]] = True
    assert T.isnan(p[bad]).all() and T.isfinite(p[~bad]).all() and p[300] == old[300]
    block = T.arange(n, device="cuda") // 128
    for x in (_values(T, m, ms), _values(T, v, vs)):
        assert T.equal(T.isnan(x), (block == 1) | (block == 5))
    # elements far below their block's largest keep a positive v, and the next step stays within a few lr
    grad = T.full((256,), 1e-12, device="cuda")
    grad[::128] = 1e4
    p, m, v = T.zeros(256, device="cuda"), T.zeros(256, dtype=T.float8_e4m3fn, device="cuda"), T.zeros(256, dtype=T.float8_e5m2, device="cuda")
    opt = K.AdamW([p], [grad], [m], [v], [T.zeros(2, device="cuda")], [T.zeros(2, device="cuda")])
    for k in range(50):
        was = p.clone()
        opt.step(k, 1e-3, seed=5)
        assert (v.float() > 0).all() and ((p - was).abs() <= 2e-2).all()


def test_adamw_beyond_two_to_the_31_elements(T, K):
    n = (1 << 31) + 1000
    p, g = T.zeros(n, dtype=T.bfloat16, device="cuda"), T.zeros(n, dtype=T.bfloat16, device="cuda")
    m, v = T.zeros(n, dtype=T.float8_e4m3fn, device="cuda"), T.zeros(n, dtype=T.float8_e5m2, device="cuda")
    ms, vs = T.zeros((n + 127) // 128, device="cuda"), T.zeros((n + 127) // 128, device="cuda")
    spots = [0, 5, (1 << 31) - 1, 1 << 31, n - 1]
    for i, k in enumerate(spots):
        g[k] = float(i + 1)
    K.AdamW([p], [g], [m], [v], [ms], [vs]).step(0, 0.5, seed=9)
    assert int((p != 0).sum()) == len(spots) and all(float(p[k]) == -0.5 for k in spots)
    assert int((ms != 1).sum()) == 4 and int((m.view(T.uint8) != 0).sum(dtype=T.int64)) == len(spots)


# ---- together --------------------------------------------------------------------------------------------------------

def test_block_trained_and_served(T, K):
    """z = N(x), y = z W^T, h = x + s sigmoid(g) N(y), loss = h . c: three steps of training against the same in 64 bits, then served in 8-bit integers."""
    n, d, lr = 300, 256, 1e-2
    g = _gen(T, 1)
    x, gate, c = (T.randn((n, d), generator=g, device="cuda") for _ in range(3))
    names = ("W", "w_pre", "w_post", "scale")
    par = dict(W=T.randn((d, d), generator=g, device="cuda") * d ** -0.5, w_pre=T.ones(d, device="cuda"), w_post=T.ones(d, device="cuda"), scale=T.full((d,), 0.5, device="cuda"))
    ref = {k: v.double().requires_grad_() for k, v in par.items()}
    rm, rv = ({k: T.zeros_like(v) for k, v in ref.items()} for _ in range(2))
    grads = {k: T.empty_like(v) for k, v in par.items()}
    state = lambda: [T.zeros(v.numel(), device="cuda") for v in par.values()]
    opt = K.AdamW([par[k] for k in names], [grads[k] for k in names], state(), state(), weight_decay=[0.1, 0.0, 0.0, 0.0])
    z, h, dy, dz = (T.empty((n, d), device="cuda") for _ in range(4))
    s1, s2, dh = T.empty((n, 4), device="cuda"), T.empty((n, 4), device="cuda"), T.empty((n, d), device="cuda")
    rms = lambda u, w: u * T.rsqrt((u * u).mean(1, keepdim=True) + 1e-6) * w
    for step in range(3):
        K.block_norm(x, z=z, pre_weight=par["w_pre"], stats=s1)
        y = z @ par["W"].t()
        K.block_norm(x, y=y, h=h, gate=gate, gate_act="sigmoid", post_weight=par["w_post"], scale=par["scale"], stats=s2)
        K.block_norm_grad(x, s2, dx=dh, dh=c, y=y, dy=dy, gate=gate, gate_act="sigmoid", post_weight=par["w_post"], dpost_weight=grads["w_post"], scale=par["scale"],
                          dscale=grads["scale"])
        T.matmul(dy.t(), z, out=grads["W"])
        T.matmul(dy, par["W"], out=dz)
        K.block_norm_grad(x, s1, dx=dh, dh=dh, dz=dz, pre_weight=par["w_pre"], dpre_weight=grads["w_pre"])
        opt.step(step, lr)
        leaf = x.double().requires_grad_()
        out = leaf + ref["scale"] * T.sigmoid(gate.double()) * rms(rms(leaf, ref["w_pre"]) @ ref["W"].t(), ref["w_post"])
        (out * c.double()).sum().backward()
        # (fp32 products of 256 terms between: some 1e-6 of a gradient's largest)
        assert ((h - out.detach()).abs() <= 2e-5 * out.detach().abs().max()).all() and ((dh - leaf.grad).abs() <= 2e-5 * leaf.grad.abs().max()).all()
        with T.no_grad():
            for k, v in ref.items():
                assert ((grads[k] - v.grad).abs() <= 2e-5 * v.grad.abs().max()).all(), k
                rm[k], rv[k] = 0.9 * rm[k] + 0.1 * v.grad, 0.999 * rv[k] + 0.001 * v.grad ** 2
                t = step + 1
                v.mul_(1 - lr * (0.1 if k == "W" else 0.0)).sub_(lr * (rm[k] / (1 - 0.9 ** t)) / ((rv[k] / (1 - 0.999 ** t)).sqrt() + 1e-8))
                v.grad = None
                # a step moves an element by lr; gradients near zero may turn it, others follow them
                assert float(((par[k] - v).abs() > 1e-3 * lr).double().mean()) <= 0.01, k
    wq, ws = _int8(T, d, d), T.empty(d, device="cuda")
    K.int8_quantize(par["W"], wq, ws)
    q, s = _int8(T, n, d), T.empty(n, device="cuda")
    y8, h8 = T.empty((n, d), device="cuda"), T.empty((n, d), device="cuda")

    def serve():
        K.block_norm(x, z=q, z_scales=s, pre_weight=par["w_pre"])
        K.int8_matmul(q, s, wq, ws, y8)
        K.block_norm(x, y=y8, h=h8, gate=gate, gate_act="sigmoid", post_weight=par["w_post"], scale=par["scale"])

    serve()
    # (the integers are summed first: of products with the scales, 62 bits long, a sum that is zero would not be zero in 64 bits)
    plain = (q.double() @ wq.double().t()) * s.double()[:, None] * ws.double()
    _check(T, y8, plain, plain.abs() * 3.03 * U)
    o = _block64(T, dict(x=x.double(), y=y8.double(), gate=gate.double(), w1=par["w_post"].double(), scale=par["scale"].double()), "sigmoid", float(np.float32(1e-6)), 0.0, d)
    _check(T, h8, o["h"].v, 1.05 * o["h"].tol)
    # integers of 7 bits and a sign: each operand within half of a 127th of its row's largest value
    z64 = rms(x.double(), par["w_pre"].double())
    w64 = par["W"].double()
    bound = (s.double()[:, None] / 2 * 1.001) @ w64.abs().sum(1)[None, :] + z64.abs().sum(1)[:, None] * (ws.double() / 2)[None, :] + d * s.double()[:, None] * ws.double() / 4
    assert ((y8.double() - z64 @ w64.t()).abs() <= bound * 1.01).all()
    # captured and replayed on another stream, beside another graph of the same calls
    want = h8.clone()
    stream, graphs = T.cuda.Stream(), []
    for _ in range(2):
        graphs.append(T.cuda.CUDAGraph())
        with T.cuda.graph(graphs[-1], stream=stream):
            serve()
    h8.zero_()
    with T.cuda.stream(stream):
        graphs[0].replay()
        graphs[1].replay()
    T.cuda.synchronize()
    assert T.equal(h8, want)


def test_calls_on_two_streams_do_not_share_anything(T, K):
    """Gradients of vectors (which need scratch) and products on two streams at once are what they are alone."""
    streams = [T.cuda.Stream(), T.cuda.Stream()]
    jobs = []
    for i in range(2):
        g = _gen(T, 40 + i)
        n, d = 3000 + i, 400
        f = _inputs(T, g, n, d, "f32", "bf16", "both", True, "silu", True, True)
        dz, stats, z = T.randn((n, d), generator=g, device="cuda").to(T.bfloat16), T.empty((n, 4), device="cuda"), T.empty((n, d), dtype=T.bfloat16, device="cuda")
        args = dict(pre_weight=f["w2"], y=f["y"], gate=f["gate"], gate_act="silu", post_weight=f["w1"], post_bias=f["b1"], scale=f["scale"], kind="layer")
        K.block_norm(f["x"], z=z, stats=stats, pre_bias=f["b2"], **args)
        dw = [T.empty(d, device="cuda") for _ in range(5)]

        def call(f=f, stats=stats, dz=dz, args=args, dw=dw):
            K.block_norm_grad(f["x"], stats, dz=dz, dpre_weight=dw[0], dpre_bias=dw[1], dpost_weight=dw[2], dpost_bias=dw[3], dscale=dw[4], **args)
        call()
        jobs.append((call, dw, [x.clone() for x in dw]))
    T.cuda.synchronize()
    for _ in range(20):
        for s, (call, dw, _) in zip(streams, jobs):
            with T.cuda.stream(s):
                for x in dw:
                    x.fill_(float("nan"))
                call()
    T.cuda.synchronize()
    for _, dw, want in jobs:
        assert all(T.equal(a, b) for a, b in zip(dw, want))
