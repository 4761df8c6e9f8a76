"""Results of the operators for a residual block that must not depend on how a call is cut up: products in 8-bit integers row by row, and rows, columns and tensors
that a kernel comes to in its second and third turn."""
import numpy as np
import pytest

import test_gpu_block_operators as block
from test_gpu_block_operators import _int8
from test_gpu_row_operators import K, T, _check, _gen  # noqa: F401

pytestmark = pytest.mark.gpu


def _fma(T, x, y, z):
    """x y + z of fp32 numbers, rounded once: in 64 bits the product is exact, and a sum that is not is made odd, so that it is no middle of two fp32 numbers."""
    p, z = x.double() * y.double(), z.double()
    s = p + z
    back = s - p
    off = (p - (s - back)) + (z - back)
    even = (s.view(T.int64) & 1) == 0
    return T.where((off != 0) & even, T.nextafter(s, T.where(off > 0, float("inf"), -float("inf")).double()), s).float()


# (large enough, in turn, for tiles of 128 x 128 on two CTAs an SM, of 256 x 256, of 128 x 128 on one, of 128 x 64; few of their rows alone share K in a cluster)
@pytest.mark.parametrize("M,N,Kd", [(20_000, 300, 1536), (20_000, 300, 7680), (700, 3000, 5000), (30_000, 40, 1600), (300, 500, 2000)])
def test_int8_matmul_of_a_row_does_not_depend_on_the_others(T, K, M, N, Kd):
    g = _gen(T, M + N)
    a, b = _int8(T, M, Kd), _int8(T, N, Kd)
    a.copy_(T.randint(-127, 128, (M, Kd), generator=g, device="cuda", dtype=T.int8))
    b.copy_(T.randint(-127, 128, (N, Kd), generator=g, device="cuda", dtype=T.int8))
    sa, sb = (T.exp(2 * T.randn(k, generator=g, device="cuda")) for k in (M, N))
    total = (a.double() @ b.double().t()).float()                # exact before it is rounded
    addend = T.randn((M, N), generator=g, device="cuda") * 1e3
    for far in (False, True):
        if far:                                                  # scales far from one change nothing in other rows and columns
            sa[2], sa[M - 40], sb[N // 2], sb[7] = 2.0 ** -80 / 3, 3 * 2.0 ** 70, 2.0 ** 65 / 3, -5 * 2.0 ** -90
        swap = ((sa.abs() < 2.0 ** -63) | (sa.abs() > 2.0 ** 63))[:, None] | (sb.abs() < 2.0 ** -63) | (sb.abs() > 2.0 ** 63)
        swap &= sb.abs() < sa.abs()[:, None]
        first, last = T.where(swap, sb, sa[:, None]), T.where(swap, sa[:, None], sb)
        for plus in (None, addend):
            want = total * first * last if plus is None else _fma(T, total * first, last, plus)
            out = T.empty((M, N), device="cuda")
            K.int8_matmul(a, sa, b, sb, out, addend=plus)
            assert T.equal(out, want)
            for rows in (slice(0, 1), slice(0, 5), slice(100, 229), slice(M - 50, M)):
                some = T.empty((rows.stop - rows.start, N), device="cuda")
                K.int8_matmul(a[rows], sa[rows], b, sb, some, addend=None if plus is None else plus[rows])
                assert T.equal(some, out[rows])


# Rows enough for every team of every kernel to come to its second and third (with the next row's loads under way, where the kernel has them), and a rest: one team for
# each width that has its own, rows that move eight elements at a time, two, or one.
TURNS = [
    # n, d, x type, block type, form, post, gate, scale, bias, kind
    (40_001, 8, "f32", "bf16", "both", True, "silu", True, True, "layer"), (40_001, 50, "bf16", "bf16", "both", True, "sigmoid", True, False, "rms"),
    (40_001, 64, "bf16", "f16", "both", True, "plain", True, True, "layer"), (40_001, 64, "f32", "f32", "pre", False, "none", False, False, "rms"),
    (20_003, 128, "f32", "f32", "both", True, "sigmoid", True, True, "layer"), (30_011, 104, "bf16", "bf16", "pre", False, "none", False, True, "layer"),
    (10_007, 200, "f32", "bf16", "both", False, "none", True, True, "layer"), (10_007, 250, "f16", "f16", "both", True, "silu", True, False, "rms"),
    (10_007, 256, "bf16", "bf16", "both", True, "silu", True, True, "layer"), (8003, 400, "f32", "bf16", "both", True, "silu", True, True, "layer"),
    (8003, 512, "bf16", "bf16", "both", True, "sigmoid", False, False, "rms"), (6003, 768, "f16", "bf16", "both", True, "plain", True, False, "rms"),
    (3001, 998, "bf16", "bf16", "both", True, "sigmoid", True, True, "layer"), (6003, 1000, "bf16", "f32", "both", True, "silu", True, False, "rms"),
    (6003, 1024, "f32", "f32", "post", True, "sigmoid", True, True, "layer"), (2501, 1600, "bf16", "bf16", "both", True, "sigmoid", True, True, "layer"),
    (3001, 1400, "f32", "bf16", "pre", False, "none", False, True, "rms"), (2501, 2050, "bf16", "bf16", "both", True, "none", True, False, "rms"),
    (2501, 4096, "bf16", "bf16", "both", True, "sigmoid", True, False, "rms"), (2501, 4096, "f32", "bf16", "both", True, "silu", True, True, "layer"),
    (701, 5000, "f32", "f16", "both", True, "sigmoid", True, True, "layer"), (1203, 8192, "bf16", "bf16", "both", True, "silu", True, False, "rms"), (400, 9002, "bf16", "bf16", "both", True, "silu", True, True, "layer")]


@pytest.mark.parametrize("n,d,tx,tb,form,post,gate,scale,bias,kind", TURNS)
def test_block_norm_over_several_turns(T, K, n, d, tx, tb, form, post, gate, scale, bias, kind):
    block.test_block_norm(T, K, n, d, tx, tb, form, post, gate, scale, bias, kind)


@pytest.mark.parametrize("n,d,tx,tb,form,post,gate,scale,bias,kind", TURNS)
def test_block_norm_grad_over_several_turns(T, K, n, d, tx, tb, form, post, gate, scale, bias, kind):
    block.test_block_norm_grad(T, K, n, d, tx, tb, form, post, gate, scale, bias, kind)


# (more than 740 CTAs' elements: each takes two turns; with room for 12, 40 and 340 tensors in a launch)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("tp,tg,copy,shift,sizes,step,gs", [
    ("f32", "f32", "bf16", 0, [1_000_003, 700_001, 2049, 300_007, 129], 3, 1.0), ("bf16", "bf16", None, 1, [2_000_001, 4097, 5, 4095], 8, 0.5),
    ("f32", "bf16", None, 0, [70_001 + 511 * i for i in range(30)], 5, 1.0), ("f16", "f16", "bf16", 0, [50_001 + 97 * i for i in range(60)], 1, 1.0)])
def test_adamw_of_two_turns(T, K, bits, tp, tg, copy, shift, sizes, step, gs):
    block.test_adamw(T, K, bits, tp, tg, copy, shift, sizes, step, gs)


@pytest.mark.parametrize("n,d", [(40_001, 48), (20_003, 120), (10_007, 256), (10_007, 250), (8003, 512), (6003, 768), (6003, 1000), (3001, 1001), (2501, 4096), (300, 9000)])
def test_norms_of_a_row_do_not_depend_on_the_others(T, K, n, d):
    """h, z, statistics, integers and their scales of rows among many are what they are alone."""
    g = _gen(T, n)
    f = block._inputs(T, g, n, d, "f32", "bf16", "both", True, "silu", True, True)
    args = dict(pre_weight=f["w2"], pre_bias=f["b2"], gate_act="silu", post_weight=f["w1"], post_bias=f["b1"], scale=f["scale"], kind="layer")

    def call(rows, in8):
        x, y, gate = (f[k][rows] for k in ("x", "y", "gate"))
        m = x.shape[0]
        z = _int8(T, m, d) if in8 else T.empty((m, d), dtype=T.bfloat16, device="cuda")
        h, stats, scales = T.empty((m, d), device="cuda"), T.empty((m, 4), device="cuda"), T.empty(m, device="cuda") if in8 else None
        K.block_norm(x, z=z, y=y, h=h, gate=gate, stats=stats, z_scales=scales, **args)
        return [h, z, stats] + ([scales] if in8 else [])
    for in8 in (False, True):
        whole = call(slice(0, n), in8)
        for rows in (slice(0, 2), slice(n // 2, n // 2 + 33), slice(n - 7, n)):
            assert all(T.equal(a[rows], b) for a, b in zip(whole, call(rows, in8)))


@pytest.mark.parametrize("n,d", [(8_400_000, 256), (8_360_000, 257)])
def test_block_norm_grad_of_few_rows_beyond_two_to_the_31_elements(T, K, n, d):
    """dz is zero but in nine rows, on both sides of element 2^31 and at the ends: the vectors' gradients are those rows' alone, and all other rows' are zero."""
    at = (1 << 31) // d
    at = T.tensor([0, 4999, at - 2, at - 1, at, at + 1, n - 600, n - 2, n - 1], device="cuda")
    g = _gen(T, d)
    few = block._inputs(T, g, 9, d, "bf16", "bf16", "both", True, "silu", True, True)
    dz = T.randn((9, d), generator=g, device="cuda").to(T.bfloat16)
    f = dict(few)
    for k in ("x", "y", "gate"):
        f[k] = T.full((n, d), 1.0, dtype=T.bfloat16, device="cuda")
        f[k][at] = few[k]
    f64 = block._double(few)
    o = block._block64(T, f64, "silu", float(np.float32(1e-5)), 1.0, d)
    args = dict(pre_weight=f["w2"], y=f["y"], gate=f["gate"], gate_act="silu", post_weight=f["w1"], post_bias=f["b1"], scale=f["scale"], kind="layer")
    z, stats = T.empty((n, d), dtype=T.bfloat16, device="cuda"), T.empty((n, 4), device="cuda")
    K.block_norm(f["x"], z=z, pre_bias=f["b2"], stats=stats, eps=1e-5, **args)
    _check(T, z[at], o["z"].v, 1.05 * o["z"].tol, "z")
    z.zero_()
    z[at] = dz
    want = block._block_grad64(T, f64, o, "silu", 1.0, d, dz.double(), None)
    names = dict(dw1="dpost_weight", db1="dpost_bias", dscale="dscale", dw2="dpre_weight", db2="dpre_bias")
    got = {k: T.empty(d, device="cuda") for k in names}
    K.block_norm_grad(f["x"], stats, dx=z, dz=z, dy=f["y"], dgate=f["gate"], **{names[k]: v for k, v in got.items()}, **args)
    got.update(dx=z[at], dy=f["y"][at], dgate=f["gate"][at])
    for k, v in got.items():
        _check(T, v, want[k].v, 1.05 * want[k].tol, k)
    for rows in (z, f["y"], f["gate"]):
        rows[at] = 0
        assert not rows.any()
