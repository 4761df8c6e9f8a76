"""Refusals and sizes of the operators on rows at the ends of their ranges, without a GPU (the pointers are never followed)."""
import pytest

from test_row_operators_cpu import GRAD, K, _call  # noqa: F401

INT32_MAX = (1 << 31) - 1


@pytest.mark.parametrize("n", [4, 4000])
@pytest.mark.parametrize("dim", [INT32_MAX, INT32_MAX - 200, INT32_MAX - 1023])
def test_grad_refuses_widths_that_its_counters_do_not_hold(K, n, dim):
    """Columns are counted in 32 bits, in steps of up to 256 beyond the last one; widths that this would carry past 2^31 are turned down."""
    assert _call(K, "kge_embedding_grad", GRAD, GRAD, n=n, dim=dim, ld_grads=dim, ld_table=dim, scratch_bytes=1 << 62) == -5
    assert K.embedding_grad_scratch_bytes(10, dim, n) == 0


def test_wait_limit_of_the_product_is_checked(K):
    fn = K.lib().kge_debug_set_product_wait_limit
    assert fn(-1) == -1 and fn(5) == 0 and fn(0) == 0


@pytest.mark.parametrize("block_rows", [0, -1, 64, 256])
def test_binding_refuses_blocks_of_other_heights(K, block_rows):
    import torch
    with pytest.raises(K.KgeError) as e:
        K.fp8_quantize(torch.zeros((4, 64)), torch.zeros((4, 64), dtype=torch.float8_e4m3fn), torch.zeros((1, 4)), block_rows=block_rows)
    assert e.value.code == -1 and "block_rows" in str(e.value)


@pytest.mark.parametrize("rows,dim,n", [(10, 8, (1 << 32) + 5), (10, (1 << 32) + 8, 5000), (1 << 70, 8, 5000), (10, 8, -(1 << 40))])
def test_scratch_sizes_of_numbers_that_are_cut_off_are_refused(K, rows, dim, n):
    """Not the size for what is left of the number in 32 (or 64) bits."""
    with pytest.raises(K.KgeError) as e:
        K.embedding_grad_scratch_bytes(rows, dim, n)
    assert e.value.code == -1
