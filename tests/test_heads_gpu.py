"""Norm and rotation of query and key heads on the GPU, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from i8_common import TYPES, f64, rows_on_device, up, within
from oracle import i8_oracle as io
from paper_2511_11248_b200 import binding as B, helpers as H

pytestmark = pytest.mark.gpu

# In 32 bits: the mean of squares (width additions, 2^-24 each, halved by the root), root, products: below 2^-17 of a value of 256 (2^-18 of 128); sine and
# cosine of an angle reduced to 32 bits: 2^-21; so each value is off by 2^-16 of the magnitudes it is made of, besides the output's rounding
# (fp16 below 2^-14: half of its step, 2^-25).
SLACK = 2.0 ** -16


def check(y, x, qw, kw, qh, kh, width, eps, pos, freq, rot, adjacent, ty):
    T = len(x)
    x = x.reshape(T, -1, width)
    parts = [io.norm_rotate(p, w, eps, pos, freq, rot, adjacent) for p, w in ((x[:, :qh], qw), (x[:, qh:qh + kh], kw))]
    ref, size = (np.concatenate([p[i] for p in parts], 1).reshape(T, -1) for i in (0, 1))
    within(y, ref, io.HALF_STEP[ty] * np.abs(ref) + SLACK * size + 2.0 ** -25)


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("T,qh,kh,width,rot,adjacent,norm", [
    (1, 32, 8, 128, 128, 0, True), (1, 1, 0, 64, 64, 0, True), (3, 28, 4, 128, 64, 0, True), (2, 0, 3, 256, 256, 1, True), (5, 7, 1, 96, 96, 0, True),
    (4, 3, 2, 96, 32, 1, False), (9, 2, 2, 8, 0, 0, True), (2, 5, 5, 24, 16, 0, True), (700, 3, 1, 128, 128, 0, True), (601, 16, 2, 64, 32, 1, True),
    (33, 4, 4, 256, 128, 0, False), (3, 40, 40, 248, 240, 0, True)])
def test_norm_and_rotation(T, qh, kh, width, rot, adjacent, norm, ty):
    rng = np.random.default_rng(T + qh + width + rot)
    tt, code = TYPES[ty]
    row = (qh + kh) * width
    xd, xv = rows_on_device(rng.standard_normal((T, row)) * np.exp(rng.standard_normal((T, 1))), row + 40, tt)
    qw, kw = ((up(rng.uniform(0.2, 2.0, width)).to(tt) if norm else None) for _ in range(2))
    pos = rng.integers(0, 200000, T).astype(np.int32)
    freq = (10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)
    y = H.alloc_matrix(T, row + 8, tt)
    B.tman_norm_rotate(xd, row + 40, y, row + 8, code, T, qh, kh, width, rot, adjacent, qw, kw, 1e-6, up(pos), up(freq))
    check(f64(y[:, :row]), xv, None if qw is None else f64(qw), None if kw is None else f64(kw), qh, kh, width, 1e-6, pos, freq, rot, adjacent, ty)
    assert bool(torch.isnan(y[:, row:]).all())
    # in place, the rest of the rows as it was
    before = xd.clone()
    B.tman_norm_rotate(xd, row + 40, xd, row + 40, code, T, qh, kh, width, rot, adjacent, qw, kw, 1e-6, up(pos), up(freq))
    assert torch.equal(xd[:, :row].contiguous().view(torch.int16), y[:, :row].contiguous().view(torch.int16))
    assert torch.equal(xd[:, row:].contiguous().view(torch.int16), before[:, row:].contiguous().view(torch.int16))


@pytest.mark.parametrize("pos", [0, 1, -5, 1 << 20, 2 ** 31 - 1, -2 ** 31])
def test_far_positions(pos):
    rng = np.random.default_rng(1)
    xd, xv = rows_on_device(rng.standard_normal((1, 128)), 128, torch.float16)
    freq = (10000.0 ** (-np.arange(0, 128, 2) / 128)).astype(np.float32)
    y = H.alloc_matrix(1, 128, torch.float16)
    p = np.array([pos], dtype=np.int32)
    B.tman_norm_rotate(xd, 128, y, 128, B.DTYPE_F16, 1, 1, 0, 128, 128, 0, None, None, 0.0, up(p), up(freq))
    check(f64(y), xv, None, None, 1, 0, 128, 0.0, p, freq, 128, 0, "f16")


def test_heads_of_zeros_of_numbers_at_the_ends_and_of_none():
    x = np.zeros((4, 128))
    x[1] = 60000.0
    x[2] = 2.0 ** -24
    x[3, 7] = np.nan
    xd, xv = rows_on_device(x, 128, torch.float16)
    w = torch.ones(128, dtype=torch.float16, device="cuda")
    y = H.alloc_matrix(4, 128, torch.float16)
    freq, pos = np.ones(64, dtype=np.float32), np.arange(4, dtype=np.int32)
    B.tman_norm_rotate(xd, 128, y, 128, B.DTYPE_F16, 4, 1, 0, 128, 128, 0, w, None, 1e-20, up(pos), up(freq))
    got = f64(y)
    assert np.isnan(got[3]).all()
    check(got[:3], xv[:3], np.ones(128), None, 1, 0, 128, 1e-20, pos[:3], freq, 128, 0, "f16")
