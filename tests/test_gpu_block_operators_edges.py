"""The operators for a residual block at the ends of what they take: the smallest scales, gates far from zero, rows without columns.  Tolerances count roundings of
U = 2^-24."""
import pytest

from test_gpu_block_operators import _int8, _quantized64
from test_gpu_row_operators import K, T, U, _gen  # noqa: F401

pytestmark = pytest.mark.gpu


def test_int8_quantize_of_middles_at_the_smallest_scales(T, K):
    """fp32 rows whose scale is a small odd number of units of 2^-149, full of the two values next to each middle: half a unit decides."""
    rows, least = 500, 2.0 ** -149
    g = _gen(T, 1)
    s = (2 ** 23 + 1 + 2 * T.randint(0, 2 ** 22, (rows, 1), generator=g, device="cuda")).double()                  # units; 2^-126 to 2^-125
    middle = (T.arange(127, device="cuda").double() + 0.5) * s
    x = T.cat([T.floor(middle), T.ceil(middle), 127 * s], 1) * least
    x = T.where(T.rand(x.shape, generator=g, device="cuda") < 0.5, -x, x).float()
    q, scales = _int8(T, rows, x.shape[1]), T.empty(rows, device="cuda")
    K.int8_quantize(x, q, scales)
    wq, ws = _quantized64(T, x)          # (quotients of integers below 2^31: in 64 bits right, or a middle exactly)
    assert T.equal(scales, ws) and T.equal(scales.double() / least, s[:, 0])
    assert T.equal(q, wq)


@pytest.mark.parametrize("tx", ["float32", "bfloat16"])
def test_int8_quantize_of_rows_without_columns(T, K, tx):
    """They hold no value but zero: scale 1."""
    for rows in (1, 9, 3000):
        scales = T.full((rows + 1,), float("nan"), device="cuda")
        K.int8_quantize(T.empty((rows, 0), dtype=getattr(T, tx), device="cuda"), _int8(T, rows, 16)[:, :0], scales[:rows])
        assert (scales[:rows] == 1).all() and T.isnan(scales[rows])


@pytest.mark.parametrize("gate,tx,tb", [("sigmoid", "float32", "float32"), ("silu", "float32", "float32"), ("sigmoid", "float32", "bfloat16"), ("silu", "float32", "float16")])
@pytest.mark.parametrize("d", [64, 250, 257, 600, 998, 4096, 5000, 9000])
def test_gates_far_from_zero(T, K, d, gate, tx, tb):
    """h = 0 + act(g) 1, dgate = act'(g), dy = act(g) for gates up to 120 from zero.  The power's instruction is within 2^-22 (4 U; CUDA's own function two units, the
    same), what its argument's rounding left out is made up for to one rounding (U), the sum with one U, the reciprocal's instruction 2 U: 8 U, of which a sigmoid far
    below zero takes all.  Below the normal numbers: two units of 2^-149 of the power, one rounding."""
    n, tx, tb = 40, getattr(T, tx), getattr(T, tb)
    g = T.linspace(-120, 120, n * d, dtype=T.float64, device="cuda").flip(0).view(d, n).t().to(tb).contiguous()
    g[3, d // 2], g[7, 0] = -1e4, 1e4
    one, x, stats = T.ones((n, d), dtype=tb, device="cuda"), T.zeros((n, d), dtype=tx, device="cuda"), T.empty((n, 4), device="cuda")
    h, dy, dg = T.empty_like(x), T.empty_like(one), T.empty_like(one)
    K.block_norm(x, y=one, h=h, gate=g, gate_act=gate, stats=stats)
    K.block_norm_grad(x, stats, dh=T.ones_like(x), y=one, dy=dy, gate=g, dgate=dg, gate_act=gate)
    v = g.double()
    s = T.where(v < 0, T.exp(v) / (1 + T.exp(v)), 1 / (1 + T.exp(-v)))
    off, least = 8 * U, 3 * 2.0 ** -149
    want, tol = (s, off * s + least) if gate == "sigmoid" else (v * s, v.abs() * ((off + U) * s + least) + least)
    half = lambda t: T.finfo(t).eps / 2 if t is not T.float32 else 0.0           # (the product with one and the sum with zero are exact)
    small = lambda t: T.finfo(t).smallest_normal * T.finfo(t).eps / 2
    assert ((h.double() - want).abs() <= 1.01 * tol).all()
    assert ((dy.double() - want).abs() <= 1.01 * tol + half(tb) * want.abs() + small(tb)).all()
    # s (1 - s): twice what s is off, three roundings of s at most; s (1 + g (1 - s)): five, of (1 + |g|) s at most
    slope = s * (1 - s) if gate == "sigmoid" else s * (1 + v * (1 - s))
    tol = ((2 * off + 3 * U) * s if gate == "sigmoid" else (2 * off + 5 * U) * (1 + v.abs()) * s) + 2 * least * (1 + v.abs())
    assert ((dg.double() - slope).abs() <= 1.01 * tol + half(tb) * slope.abs() + small(tb)).all()


@pytest.mark.parametrize("d", [64, 600, 4096, 9000])
def test_infinite_gates(T, K, d):
    """An infinite gate's sigmoid is 0 or 1, a NaN's NaN, and neighbours are what they are alone."""
    g = T.zeros((3, d), device="cuda")
    g[0, 0], g[0, d - 1], g[1, 5], g[2, 7] = float("inf"), -float("inf"), float("nan"), -90.0
    h = T.empty_like(g)
    K.block_norm(T.zeros_like(g), y=T.ones_like(g), h=h, gate=g, gate_act="sigmoid")
    want = T.full_like(g, 0.5)
    want[0, 0], want[0, d - 1], want[2, 7] = 1.0, 0.0, 8.194012623990515e-40
    good = ~T.isnan(g)
    assert T.isnan(h[1, 5]) and ((h - want).abs() <= 9 * U * want + 3 * 2.0 ** -149)[good].all()


@pytest.mark.parametrize("gate,tx,tb", [("sigmoid", "bfloat16", "bfloat16"), ("silu", "bfloat16", "float16"), ("silu", "float16", "float16")])
@pytest.mark.parametrize("d", [64, 250, 257, 998, 4096])
def test_gates_far_from_zero_among_16_bits(T, K, d, gate, tx, tb):
    """h, all of which is rounded to 16 bits: act(g) within 2^-16 of itself before that, a sigmoid below 2^-126 may be 0."""
    n, tx, tb = 40, getattr(T, tx), getattr(T, tb)
    g = T.linspace(-120, 120, n * d, dtype=T.float64, device="cuda").flip(0).view(d, n).t().to(tb).contiguous()
    if gate == "sigmoid":
        g[3, d // 2], g[7, 0] = -float("inf"), float("inf")
    h = T.empty((n, d), dtype=tx, device="cuda")
    K.block_norm(T.zeros_like(h), y=T.ones_like(g), h=h, gate=g, gate_act=gate)
    v = g.double()
    s = T.where(v < 0, T.exp(v) / (1 + T.exp(v)), 1 / (1 + T.exp(-v)))
    want, least = (s, 2.0 ** -126) if gate == "sigmoid" else (v * s, v.abs() * 2.0 ** -126)
    step = T.finfo(tx)
    assert ((h.double() - want).abs() <= (2.0 ** -16 + step.eps / 2) * 1.01 * want.abs() + least + step.smallest_normal * step.eps / 2).all()
