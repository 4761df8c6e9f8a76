"""Numbers that the operators for a residual block take, without a GPU."""
import fractions

import numpy as np
import pytest


@pytest.mark.parametrize("decay", [0, 0.1, np.float32(0.1), np.float64(0.1), np.int32(1), fractions.Fraction(1, 10)])
def test_adamw_takes_any_number_as_weight_decay(decay):
    import paper_2211_12281_b200 as K
    K.AdamW([], [], [], [], weight_decay=decay).step(0, 0.1)
