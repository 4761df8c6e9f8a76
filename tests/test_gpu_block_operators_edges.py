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
