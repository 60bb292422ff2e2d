"""The weight gradient of fp32 dY down to the smallest values: three bf16 terms hold what of a value lies at 2^-133 and above, so values of 2^-110
and more exactly, and smaller ones to an absolute 2^-133."""
import numpy as np
import pytest

import act_reference as ref
from test_act_wgrad import inputs, wgrad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d_out,d_in", [(1, 40, 70), (64, 130, 96), (1000, 40, 70)])
@pytest.mark.parametrize("power", [-104, -112, -118, -123, -130, -145])
def test_down_to_the_smallest_values(rows, d_out, d_in, power):
    """As in test_act_wgrad, each sum of n terms within (n + 8) 2^-24 sum |terms|; beside it what the terms leave out, below 2^-133 a value of
    dY, and a subnormal result's own last bit at each of at most 3 n sums."""
    dy, codes, byte = inputs(rows, d_out, d_in, "f32")
    dy = dy * 50 * 2.0 ** power                            # values around 2^power, in fp32
    a, b = dy.double().numpy(), ref.decode(codes, byte, d_in)
    out = wgrad(dy, codes, byte, d_in)
    left_out = np.where(np.abs(a) < 2.0 ** -110, 2.0 ** -133, 0.0)
    size = np.abs(a).T @ np.abs(b)
    assert (np.abs(out - a.T @ b) <= (rows + 8) * 2.0 ** -24 * size + left_out.T @ np.abs(b) + 3 * rows * 2.0 ** -149).all()
