"""What the rows-features-dropout operators of the library cost, and what they compute in plain torch.

  lookup      rows of a table times a scale, for a list of ids                          (the batch's slots, a prompt's tokens)
  grad        its gradient: the rows' gradients summed by id into a dense table gradient
  dropout     kept where a counter-based 16-bit number reaches the threshold; backward = the same call on the gradient
  quantize    8-bit floating point with a scale for each block of 128, one or both orientations
  product     C = A B^T (+ C0) of two such operands
  linear      one training pass of a projection: y = x W^T, dx = dy W, dW = dy^T x, all operands quantised in the pass

With own = False, run() uses elementary torch operations in 32 bits; with own = True, the library's entry points.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_FP8 = {"e4m3": (torch.float8_e4m3fn, 448.0), "e5m2": (torch.float8_e5m2, 57344.0)}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one entity's row, as a service that answers one query at a time reads it
        dict(name="lookup_single", kind="lookup", n=1, E=100_000, d=256, t="bf16", o="bf16", scale=16.0, pad=0.0),
        # the 2 B + N slots of the large-graph batch (B = N = 8,192) at the ragged row width
        dict(name="lookup_batch", kind="lookup", n=24_576, E=2_000_000, d=200, t="f32", o="f32", scale=1.0, pad=0.0),
        # gradient of the smallest training configuration's slots (B = 64, N = 128, d = 32, 1,000 entities)
        dict(name="grad_small", kind="grad", n=256, E=1000, d=32, g="f32", o="f32", scale=1.0, pad=0.0, acc=False),
        # the large-graph batch into a table of 100,000 rows
        dict(name="grad_batch", kind="grad", n=24_576, E=100_000, d=128, g="f32", o="f32", scale=1.0, pad=0.0, acc=False),
        # half a million text tokens with a few very frequent ids, bf16 gradients into an fp32 table gradient
        dict(name="grad_long", kind="grad", n=500_000, E=120_001, d=256, g="bf16", o="f32", scale=16.0, pad=0.05, acc=False),
        # the smallest configuration's rows
        dict(name="dropout_small", kind="dropout", n=256 * 32, x="f32", o="f32", p=0.1, res=False),
        # 100,000 rows of 768 projected features in bf16, added to what they are a residual of
        dict(name="dropout_large", kind="dropout", n=100_000 * 768, x="bf16", o="bf16", p=0.1, res=True),
        # the text features of 100,000 entities made ready for 8-bit products
        dict(name="quantize_features", kind="quantize", rows=100_000, cols=768, x="bf16", f="e4m3", block=1, forms="row", pow2=False),
        # one entity's features projected
        dict(name="product_single", kind="product", M=1, N=256, K=768, fa="e4m3", fb="e4m3", ba=1, bb=128, o="bf16", add=False),
        # the projection of a batch's slots, added to their shallow rows
        dict(name="product_batch", kind="product", M=24_576, N=256, K=768, fa="e4m3", fb="e4m3", ba=1, bb=128, o="f32", add=True),
        # a large square-ish product
        dict(name="product_large", kind="product", M=8192, N=4096, K=8192, fa="e4m3", fb="e4m3", ba=1, bb=128, o="bf16", add=False),
        # one training pass of the projection over a batch's slots
        dict(name="linear_train", kind="linear", T=24_576, I=768, O=256, x="bf16", g="bf16", o="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["lookup", "grad", "dropout", "quantize", "product", "linear"], [20, 25, 15, 10, 22, 8])[0]
    t = lambda: rng.choice(["f32", "bf16", "f16"])
    if kind in ("lookup", "grad"):
        d = rng.choice([8 * rng.randint(2, 64), 8 * rng.randint(2, 64), rng.randint(5, 300)])
        n, E = _log_int(rng, 1, 500_000), _log_int(rng, 100, 500_000)
        while E * d > 40_000_000:
            E //= 2
        while n * d > 128_000_000:
            n //= 2
        c = dict(kind=kind, n=max(1, n), E=E, d=d, o=t(), scale=rng.choice([1.0, 0.5, round(math.sqrt(d), 3)]), pad=rng.choice([0.0, 0.1]))
        return dict(c, t=t()) if kind == "lookup" else dict(c, g=t(), acc=rng.random() < 0.3)
    if kind == "dropout":
        return dict(kind=kind, n=_log_int(rng, 1, 70_000_000), x=t(), o=t(), p=rng.choice([0.05, 0.1, 0.25, 0.5]), res=rng.random() < 0.5)
    if kind == "quantize":
        rows, cols = _log_int(rng, 1, 60_000), _log_int(rng, 16, 4096)
        while rows * cols > 75_000_000:
            rows //= 2
        return dict(kind=kind, rows=rows, cols=cols, x=t(), f=rng.choice(["e4m3", "e4m3", "e5m2"]), block=rng.choice([1, 1, 128]),
                    forms=rng.choice(["row", "column", "both"]), pow2=rng.random() < 0.3)
    if kind == "product":
        M, N, K = _log_int(rng, 1, 32_768), _log_int(rng, 16, 8192), _log_int(rng, 32, 16_384)
        while M * N * K > 8192 * 4096 * 8192 // 2 or M * N > 60_000_000 or M * K > 100_000_000:
            M, N, K = max(1, M * 2 // 3), max(16, N * 3 // 4), max(32, K * 3 // 4)
        return dict(kind=kind, M=M, N=N, K=K, fa=rng.choice(["e4m3", "e4m3", "e5m2"]), fb=rng.choice(["e4m3", "e4m3", "e5m2"]),
                    ba=rng.choice([1, 1, 128]), bb=rng.choice([1, 128]), o=t(), add=rng.random() < 0.4)
    return dict(kind=kind, T=_log_int(rng, 64, 32_768), I=16 * rng.randint(4, 64), O=16 * rng.randint(4, 40), x=t(), g=t(), o=rng.choice(["f32", "bf16"]))


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _ids(gen, n, E, pad, dev):
    """Ids whose frequency falls like 1 / rank, in an order of their own; `pad` of them are padding (-1)."""
    u = torch.rand(n, generator=gen, device=dev, dtype=torch.float64)
    rank = (torch.exp(u * math.log(E + 1.0)).long() - 1).clamp_(0, E - 1)
    ids = torch.randperm(E, generator=gen, device=dev)[rank]
    if pad:
        ids = torch.where(torch.rand(n, generator=gen, device=dev) < pad, torch.full_like(ids, -1), ids)
    return ids.to(torch.int32)


def _rows(gen, rows, cols, dev, spread=True):
    """Rows of different sizes with heavier tails than a normal's, as features and their gradients have."""
    x = torch.randn((rows, cols), generator=gen, device=dev)
    if spread:
        x = x * torch.exp(0.7 * torch.randn((rows, 1), generator=gen, device=dev)) * (0.5 + torch.rand((1, cols), generator=gen, device=dev))
    return x


def _inputs(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    c, s = case, {"case": case, "dev": dev}
    if c["kind"] == "lookup":
        s["table"] = _rows(gen, c["E"], c["d"], dev, False).mul_(0.1).to(_TYPES[c["t"]])
        s["ids"] = _ids(gen, c["n"], c["E"], c["pad"], dev)
    elif c["kind"] == "grad":
        s["ids"] = _ids(gen, c["n"], c["E"], c["pad"], dev)
        s["grads"] = _rows(gen, c["n"], c["d"], dev).mul_(0.01).to(_TYPES[c["g"]])
        s["old"] = _rows(gen, c["E"], c["d"], dev, False).mul_(0.1).to(_TYPES[c["o"]]) if c["acc"] else None
    elif c["kind"] == "dropout":
        s["x"] = torch.randn(c["n"], generator=gen, device=dev).to(_TYPES[c["x"]])
        s["residual"] = torch.randn(c["n"], generator=gen, device=dev).to(_TYPES[c["o"]]) if c["res"] else None
        s["seed"], s["step"], s["site"] = (seed * 0x9E3779B97F4A7C15 + 7) % (1 << 63), 1000 + seed % 977, 3
    elif c["kind"] == "quantize":
        s["x"] = _rows(gen, c["rows"], c["cols"], dev).to(_TYPES[c["x"]])
    elif c["kind"] == "product":
        for name, rows in (("a", c["M"]), ("b", c["N"])):
            x = _rows(gen, rows, c["K"], dev)
            if name == "b":
                x.mul_(c["K"] ** -0.5)
            q, sc = _quantize(x, c["f" + name], c["b" + name], False)
            s[name], s[name + "_scales"] = _padded(q), sc
        s["addend"] = torch.randn((c["M"], c["N"]), generator=gen, device=dev).to(_TYPES[c["o"]]) if c["add"] else None
    else:
        s["x"] = _rows(gen, c["T"], c["I"], dev).to(_TYPES[c["x"]])
        s["w"] = torch.randn((c["O"], c["I"]), generator=gen, device=dev).mul_(1.0 / math.sqrt(c["I"]))
        s["dy"] = _rows(gen, c["T"], c["O"], dev).mul_(0.01).to(_TYPES[c["g"]])
    return s


def _padded(q):
    """The same matrix with rows a multiple of 16 bytes apart."""
    rows, cols = q.shape
    wide = torch.zeros((rows, (cols + 15) // 16 * 16), dtype=torch.uint8, device=q.device)
    wide[:, :cols] = q.view(torch.uint8)
    return wide.view(q.dtype)[:, :cols]


def _empty8(rows, cols, dtype, dev):
    return torch.empty((rows, (cols + 15) // 16 * 16), dtype=dtype, device=dev)[:, :cols]


def _cdiv(a, b):
    return -(-a // b)


def prepare(case, seed):
    s, c = _inputs(case, seed), case
    dev = s["dev"]
    if c["kind"] == "lookup":
        s["out"] = torch.empty((c["n"], c["d"]), dtype=_TYPES[c["o"]], device=dev)
    elif c["kind"] == "grad":
        s["out"] = s["old"] if c["acc"] else torch.empty((c["E"], c["d"]), dtype=_TYPES[c["o"]], device=dev)
    elif c["kind"] == "dropout":
        s["out"] = torch.empty(c["n"], dtype=_TYPES[c["o"]], device=dev)
    elif c["kind"] == "quantize":
        s["q"] = _operand(c["rows"], c["cols"], c["f"], c["block"], dev) if c["forms"] != "column" else (None, None)
        s["qt"] = _operand(c["cols"], c["rows"], c["f"], c["block"], dev) if c["forms"] != "row" else (None, None)
    elif c["kind"] == "product":
        s["out"] = torch.empty((c["M"], c["N"]), dtype=_TYPES[c["o"]], device=dev)
    else:
        T, I, O = c["T"], c["I"], c["O"]
        s["xq"], s["xt"] = _operand(T, I, "e4m3", 1, dev), _operand(I, T, "e4m3", 1, dev)
        s["wq"], s["wt"] = _operand(O, I, "e4m3", 128, dev), _operand(I, O, "e4m3", 128, dev)
        s["gq"], s["gt"] = _operand(T, O, "e4m3", 1, dev), _operand(O, T, "e4m3", 1, dev)
        s["y"], s["dx"] = (torch.empty((T, w), dtype=_TYPES[c["o"]], device=dev) for w in (O, I))
        s["dw"] = torch.empty((O, I), device=dev)
    return s


def _operand(rows, cols, fmt, block, dev):
    """An empty 8-bit operand [rows, cols] and its scales [blocks of cols, rows (or blocks of rows)]."""
    return (_empty8(rows, cols, _FP8[fmt][0], dev),
            torch.empty((_cdiv(cols, 128), rows if block == 1 else _cdiv(rows, 128)), device=dev))


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _lookup(table, ids, scale, out_type):
    ok = (ids >= 0) & (ids < table.shape[0])
    rows = table[torch.where(ok, ids, torch.zeros_like(ids))].float() * scale
    return torch.where(ok[:, None], rows, torch.zeros_like(rows)).to(out_type)


def _grad(ids, grads, rows, scale, old, out_type):
    ok = (ids >= 0) & (ids < rows)
    g = grads.float()
    g = torch.where(ok[:, None], g, torch.zeros_like(g))
    total = torch.zeros((rows, g.shape[1]), device=g.device).index_add_(0, torch.where(ok, ids, torch.zeros_like(ids)), g) * scale
    return (total if old is None else old.float() + total).to(out_type)


def _mul32(a, b):
    """High and low words of the product of a word tensor and a word constant, in int64."""
    low = a * (b & 0xFFFF)
    t = a * (b >> 16) + (low >> 16)
    return t >> 16, ((t & 0xFFFF) << 16) | (low & 0xFFFF)


def _halves(n, seed, step, site, dev):
    """The 16-bit numbers of elements 0 .. n - 1: Philox4x32 with ten rounds, eight elements to a counter."""
    c0 = torch.arange((n + 7) // 8, device=dev, dtype=torch.int64)
    c1, c2, c3 = (torch.full_like(c0, v) for v in (step & 0xFFFFFFFF, step >> 32, 0x80000000 | site))
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        h0, l0 = _mul32(c0, 0xD2511F53)
        h1, l1 = _mul32(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:n]


def _dropout(x, p, seed, step, site, residual, out_type):
    cut = round(p * 65536)
    y = torch.where(_halves(x.numel(), seed, step, site, x.device) >= cut, x.float() * (65536.0 / (65536 - cut)), torch.zeros((), device=x.device))
    return (y if residual is None else residual.float() + y).to(out_type)


def _quantize(x, fmt, block, pow2):
    """8-bit values and scales [blocks of columns, rows or blocks of rows] of x, in blocks of 128 columns (and `block` rows)."""
    dtype, top = _FP8[fmt]
    rows, cols = x.shape
    kb, rb = _cdiv(cols, 128), _cdiv(rows, block)
    x = x.float()
    wide = torch.zeros((rb * block, kb * 128), device=x.device)
    wide[:rows, :cols] = x
    most = wide.abs().view(rb, block, kb, 128).amax((1, 3))
    scale = (most / torch.full_like(most, top)).clamp_(min=2.0 ** -126)
    if pow2:
        mant, e = torch.frexp(scale)
        scale = torch.ldexp(torch.ones_like(scale), e - (mant == 0.5).to(e.dtype))
    scale = torch.where(most > 0, scale, torch.ones_like(scale))
    # (64 bits: a quotient rounded to 32 falls on the middle of two 8-bit values where the true one does not)
    y = wide.view(rb, block, kb, 128).double() / scale.double()[:, None, :, None]
    bits, least = (3, -6) if fmt == "e4m3" else (2, -14)
    last = torch.ldexp(torch.ones_like(y), (torch.frexp(y)[1] - 1).clamp_(min=least) - bits)
    q = ((y / last).round_() * last).view(rb * block, kb * 128)[:rows, :cols].to(dtype)
    return q, scale.t().contiguous()


def _values(q, scales):
    """The values that an operand stands for, in 32 bits."""
    rows, cols = q.shape
    s = scales if scales.shape[1] == rows else scales.repeat_interleave(128, 1)[:, :rows]
    return q.float() * s.repeat_interleave(128, 0)[:cols].t()


def _product(a, sa, b, sb, addend, out_type):
    c = torch.matmul(_values(a, sa), _values(b, sb).t())
    return (c if addend is None else c + addend.float()).to(out_type)


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    if c["kind"] == "lookup":
        return _lookup(s["table"], s["ids"], c["scale"], _TYPES[c["o"]])
    if c["kind"] == "grad":
        g = _grad(s["ids"], s["grads"], c["E"], c["scale"], s["out"] if c["acc"] else None, _TYPES[c["o"]])
        return s["out"].copy_(g) if c["acc"] else g
    if c["kind"] == "dropout":
        return _dropout(s["x"], c["p"], s["seed"], s["step"], s["site"], s["residual"], _TYPES[c["o"]])
    if c["kind"] == "quantize":
        return [None if s[name][0] is None else _quantize(x, c["f"], c["block"], c["pow2"])
                for name, x in (("q", s["x"]), ("qt", s["x"].t()))]
    if c["kind"] == "product":
        return _product(s["a"], s["a_scales"], s["b"], s["b_scales"], s["addend"], _TYPES[c["o"]])
    o = _TYPES[c["o"]]
    y = _product(*_quantize(s["x"], "e4m3", 1, False), *_quantize(s["w"], "e4m3", 128, False), None, o)
    dx = _product(*_quantize(s["dy"], "e4m3", 1, False), *_quantize(s["w"].t(), "e4m3", 128, False), None, o)
    dw = _product(*_quantize(s["dy"].t(), "e4m3", 1, False), *_quantize(s["x"].t(), "e4m3", 1, False), None, torch.float32)
    return dict(y=y, dx=dx, dw=dw)


def _run_own(s, c):
    import paper_2211_12281_b200 as K
    if c["kind"] == "lookup":
        K.embedding_lookup(s["table"], s["ids"], s["out"], scale=c["scale"])
        return s["out"]
    if c["kind"] == "grad":
        K.embedding_grad(s["ids"], s["grads"], s["out"], scale=c["scale"], accumulate=c["acc"])
        return s["out"]
    if c["kind"] == "dropout":
        K.dropout(s["x"], s["out"], c["p"], s["seed"], s["step"], site=s["site"], residual=s["residual"])
        return s["out"]
    if c["kind"] == "quantize":
        K.fp8_quantize(s["x"], *s["q"], *s["qt"], block_rows=c["block"], pow2=c["pow2"])
        return [None if s[name][0] is None else s[name] for name in ("q", "qt")]
    if c["kind"] == "product":
        K.fp8_matmul(s["a"], s["a_scales"], s["b"], s["b_scales"], s["out"], addend=s["addend"])
        return s["out"]
    K.fp8_quantize(s["x"], *s["xq"], *s["xt"])
    K.fp8_quantize(s["w"], *s["wq"], *s["wt"], block_rows=128)
    K.fp8_matmul(*s["xq"], *s["wq"], s["y"])
    K.fp8_quantize(s["dy"], *s["gq"], *s["gt"])
    K.fp8_matmul(*s["gq"], *s["wt"], s["dx"])
    K.fp8_matmul(*s["gt"], *s["xt"], s["dw"])
    return dict(y=s["y"], dx=s["dx"], dw=s["dw"])


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def _operand_bytes(rows, cols, block):
    return rows * cols + 4 * _cdiv(cols, 128) * (rows if block == 1 else _cdiv(rows, 128))


def work(case):
    c = case
    if c["kind"] == "lookup":
        rows = min(c["n"], c["E"])          # a row that several ids name is read once
        return dict(bytes=4 * c["n"] + c["d"] * (rows * _SIZE[c["t"]] + c["n"] * _SIZE[c["o"]]), flops=c["n"] * c["d"])
    if c["kind"] == "grad":
        table = 2 * min(c["n"], c["E"]) if c["acc"] else c["E"]
        return dict(bytes=4 * c["n"] + c["d"] * (c["n"] * _SIZE[c["g"]] + table * _SIZE[c["o"]]), flops=c["n"] * c["d"])
    if c["kind"] == "dropout":
        return dict(bytes=c["n"] * (_SIZE[c["x"]] + _SIZE[c["o"]] * (2 if c["res"] else 1)), flops=2 * c["n"])
    if c["kind"] == "quantize":
        forms = [(c["rows"], c["cols"])] * (c["forms"] != "column") + [(c["cols"], c["rows"])] * (c["forms"] != "row")
        return dict(bytes=c["rows"] * c["cols"] * _SIZE[c["x"]] + sum(_operand_bytes(r, k, c["block"]) for r, k in forms), flops=2 * c["rows"] * c["cols"])
    if c["kind"] == "product":
        return dict(bytes=_operand_bytes(c["M"], c["K"], c["ba"]) + _operand_bytes(c["N"], c["K"], c["bb"]) +
                    c["M"] * c["N"] * _SIZE[c["o"]] * (2 if c["add"] else 1), flops=2 * c["M"] * c["N"] * c["K"])
    T, I, O = c["T"], c["I"], c["O"]
    return dict(bytes=T * I * _SIZE[c["x"]] + 4 * O * I + T * O * _SIZE[c["g"]] + T * (I + O) * _SIZE[c["o"]] + 4 * O * I, flops=6 * T * I * O)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _philox_np(n, seed, step, site):
    m, low = np.uint64(32), np.uint64(0xFFFFFFFF)
    x = np.zeros((4, (n + 7) // 8), dtype=np.uint64)
    x[0] = np.arange(x.shape[1], dtype=np.uint64)
    x[1], x[2], x[3] = step & 0xFFFFFFFF, step >> 32, 0x80000000 + site
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for r in range(10):
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = np.stack([(q >> m) ^ x[1] ^ np.uint64((key[0] + r * 0x9E3779B9) % 2 ** 32), q & low,
                      (p >> m) ^ x[3] ^ np.uint64((key[1] + r * 0xBB67AE85) % 2 ** 32), p & low])
    return np.ascontiguousarray(x.T.astype("<u4")).view("<u2").reshape(-1)[:n]


def _fp8_round64(y, fmt):
    """The nearest 8-bit value (ties to the even one) of doubles within the type's range."""
    bits, least = (3, -6) if fmt == "e4m3" else (2, -14)
    e = torch.frexp(y)[1].to(torch.float64) - 1
    step = torch.exp2(torch.clamp(e, min=least) - bits)
    return torch.round(y / step) * step


def _operand64(x, fmt, block, pow2=False):
    """(8-bit values, scales spread over the elements, scales) in 64 bits."""
    x = x.double()
    rows, cols = x.shape
    top = _FP8[fmt][1]
    pad = torch.nn.functional.pad(x.abs(), (0, -cols % 128, 0, -rows % block))
    most = pad.reshape(pad.shape[0] // block, block, -1, 128).amax(3).amax(1)
    # the scale is what is stored, in 32 bits; the values are rounded by it
    sc = torch.exp2(torch.ceil(torch.log2(most / top))) if pow2 else (most / top).float().double()
    sc = torch.where(most > 0, sc, torch.ones_like(sc))
    spread = sc.repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    return _fp8_round64(x / spread, fmt), spread, sc.t().contiguous()


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "lookup":
        ids = s["ids"].long()
        rows = s["table"].double()[ids.clamp(min=0)] * c["scale"]
        rows[ids < 0] = 0
        return rows
    if c["kind"] == "grad":
        ids = s["ids"].long()
        total = torch.zeros((c["E"], c["d"]), dtype=torch.float64, device=s["dev"])
        total.index_add_(0, ids[ids >= 0], s["grads"][ids >= 0].double())
        total *= c["scale"]
        return total + s["old"].double() if c["acc"] else total
    if c["kind"] == "dropout":
        if c["n"] > 80_000_000:
            return None
        keep = torch.from_numpy(_philox_np(c["n"], s["seed"], s["step"], s["site"]).astype(np.int32)).to(s["dev"]) >= round(c["p"] * 65536)
        y = s["x"].double() / (1.0 - round(c["p"] * 65536) / 65536)
        y[~keep] = 0
        return y + s["residual"].double() if c["res"] else y
    if c["kind"] == "quantize":
        got = []
        for form, x in (("row", s["x"]), ("column", s["x"].t())):
            if c["forms"] in (form, "both"):
                q, _, sc = _operand64(x, c["f"], c["block"], c["pow2"])
                got.append([q, sc])
            else:
                got.append(None)
        return got
    if c["kind"] == "product":
        def values(q, sc):
            rows, cols = q.shape
            at = torch.arange(rows, device=q.device) // (1 if sc.shape[1] == rows else 128)
            return q.to(torch.float32).double() * sc.double()[torch.arange(cols, device=q.device)[None, :] // 128, at[:, None]]
        r = values(s["a"], s["a_scales"]) @ values(s["b"], s["b_scales"]).t()
        return r + s["addend"].double() if c["add"] else r

    def prod(a, fa, b, fb):
        (qa, ua, _), (qb, ub, _) = _operand64(a, "e4m3", fa), _operand64(b, "e4m3", fb)
        return (qa * ua) @ (qb * ub).t()
    x, w, dy = s["x"], s["w"], s["dy"]
    return dict(y=prod(x, 1, w, 128), dx=prod(dy, 1, w.t(), 128), dw=prod(dy.t(), 1, x.t(), 1))
