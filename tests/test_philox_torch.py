import numpy as np
import pytest

from oracle import operators_oracle as orc
from tests.philox_torch import dropout_factors


@pytest.mark.parametrize("n,h,p,seed,offset", [(5, 37, 0.3, 0x9ABCDEF012345678, (7 << 32) + 11), (3, 8, 0.0, 1, 2),
                                               (2, 16, 1.0, -5, -1), (4, 20, 2.0 ** -17 * 1.5, 3, (1 << 63) + 9)])
def test_matrix_form_is_the_scalar_oracle(n, h, p, seed, offset):
    want = orc.dropout_factors(n, h, p, seed, offset)
    assert np.array_equal(dropout_factors(n, h, p, seed, offset).numpy(), want)
    assert np.array_equal(dropout_factors(1, h, p, seed, offset, first_row=n - 1).numpy(), want[n - 1:])
