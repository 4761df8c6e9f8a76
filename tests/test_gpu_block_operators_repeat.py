"""Results of the operators for a residual block that must not depend on how a call is cut up: products in 8-bit integers row by row, and rows, columns and tensors
that a kernel comes to in its second and third turn."""
import pytest

from test_gpu_block_operators import _int8
from test_gpu_row_operators import K, T, _gen  # noqa: F401

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
