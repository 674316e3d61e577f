"""Norm and rotation of query and key heads at the ends of what a call may ask for."""
import numpy as np
import pytest
import torch

from i8_common import f64, rows_on_device, up, within
from oracle import i8_oracle as io
from paper_2511_11248_b200 import binding as B, helpers as H

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


@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("T,width,rot", [(1, 128, 128), (9, 64, 32), (700, 256, 256), (3, 40, 16)])
def test_heads_of_any_size_of_bf16(T, width, rot, eps):
    """Squares of bf16 numbers beyond 2^64, or their sums, are beyond 32 bits, and those of numbers below 2^-74 are nothing there: the norm is right all the same."""
    rng = np.random.default_rng(T + width)
    exponents = np.array([-130, -110, -80, -70, -66, -60, -30, 0, 30, 57, 60, 64, 80, 100, 125])
    heads = len(exponents)
    x = rng.standard_normal((T, heads, width)).clip(-3.5, 3.5) * 2.0 ** exponents[:, None]
    x[:, :, 1::7] *= 2.0 ** -5
    xd, xv = rows_on_device(x.reshape(T, -1), heads * width, torch.bfloat16)
    w = up(rng.uniform(0.5, 1.5, width)).bfloat16()
    pos, freq = np.arange(T, dtype=np.int32), (10000.0 ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)
    y = H.alloc_matrix(T, heads * width, torch.bfloat16)
    B.tman_norm_rotate(xd, heads * width, y, heads * width, B.DTYPE_BF16, T, heads, 0, width, rot, 0, w, None, eps, up(pos), up(freq))
    ref, size = io.norm_rotate(xv.reshape(T, heads, width), f64(w), float(np.float32(eps)), pos, freq, rot, 0)
    # as for other sizes (2^-16 of the magnitudes that a value is made of), bf16's least number in place of fp16's
    within(f64(y), ref.reshape(T, -1), (2.0 ** -8 * np.abs(ref) + 2.0 ** -16 * size + 2.0 ** -134).reshape(T, -1))
