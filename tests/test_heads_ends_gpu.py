"""Norm and rotation of query and key heads at the ends of what a call may ask for."""
import pytest
import torch

from paper_2511_11248_b200 import binding as B

pytestmark = pytest.mark.gpu


def test_as_many_tokens_as_their_number_can_say():
    """2^31 - 1 heads of eight values, in place: 32 GB.  Equal values have themselves as the root of their mean square."""
    T = 2 ** 31 - 1
    x = torch.full((T * 8,), 3.0, dtype=torch.float16, device="cuda")
    x[-8:] = -1.0
    w = torch.full((8,), 0.5, dtype=torch.float16, device="cuda")
    B.tman_norm_rotate(x, 8, x, 8, B.DTYPE_F16, T, 1, 0, 8, 0, 0, w, None, 0.0, None, None)
    assert bool((x[-8:] == -0.5).all())
    assert all(bool((part == 0.5).all()) for part in x[:-8].split(1 << 31))
