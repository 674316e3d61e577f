"""Decode with microscaled 4-bit floating point at the ends of the range of 32 bits: what fits the output is right, whatever intermediate sums would be."""
import numpy as np
import pytest
import torch

from oracle import f4_oracle as fo
from paper_2511_11248_b200 import binding as B, helpers as H
from test_f4_gpu import f64, pack_on_device, to_device

pytestmark = pytest.mark.gpu


def check(x, codes, scales, rs, block, ty, floor=0.0):
    """Half a step of the type, 2^-23 of S = sum |x w| for every addition in 32 bits, the header's 2^-20 of the block's largest value times the weights'
    magnitudes (of 2^-17 of the row's where that is more; `floor`: of the smallest magnitudes), and half the type's smallest value."""
    dtype, code = (torch.float16, B.DTYPE_F16) if ty == "f16" else (torch.bfloat16, B.DTYPE_BF16)
    (M, K), N = x.shape, codes.shape[0]
    packed = pack_on_device(codes, scales, rs, block)
    dev, held = to_device(x, K, dtype)
    ws, y = H.alloc_workspace_f4(B.OP_GEMV, M, K, N, block), H.alloc_matrix(M, N, dtype)
    B.tman_mpgemv_f4(packed, dev, K, y, N, code, M, K, N, block, ws)
    assert B.tman_read_status(ws) == 0
    w = fo.values(codes, scales, rs, block)
    ref, S = held @ w.T, np.abs(held) @ np.abs(w).T
    assert np.abs(ref).max() < float(torch.finfo(dtype).max)
    top = np.abs(held).reshape(M, -1, block).max(-1)
    if block == 16:
        top = np.maximum(top, 2.0 ** -17 * top.max(1, keepdims=True))
    unit = np.maximum(2.0 ** -20 * top, floor)
    tol = (2.0 ** -8 if ty == "bf16" else 2.0 ** -11) * np.abs(ref) + (K / 64 + 32) * 2.0 ** -23 * S + unit @ np.abs(w).reshape(N, -1, block).sum(-1).T
    tol += 2.0 ** -134 if ty == "bf16" else 2.0 ** -25
    got = f64(y)
    bad = int((~(np.abs(got - ref) <= tol)).sum())
    assert bad == 0, f"{bad} of {got.size}"


SIZES = [(1, 512, 130), (3, 4096, 200), (8, 4096, 72), (2, 1040, 19001)]      # (several shares of k, the last: one)


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("rows,weights_row", [(1e33, 1e-6), (1e35, 1e-30), (1e-33, 1e20), (1e-30, 2.0 ** 90), (1.0, 2.0 ** -120), (1e30, -1e-10)])
def test_row_scales_of_weights_bring_the_sums_into_range(M, K, N, rows, weights_row):
    """The sums of activations times block scales leave 32 bits, or their precision, upwards or downwards; times the weights' row scale they are ordinary."""
    rng = np.random.default_rng(K + N)
    small = rows < 1
    codes = rng.integers(0, 16, (N, K)).astype(np.uint8)
    scales = rng.integers(1, 9, (N, K // 16)).astype(np.uint8) if small else rng.integers(0x70, 0x7F, (N, K // 16)).astype(np.uint8)
    check(rng.standard_normal((M, K)) * rows, codes, scales, np.full(N, weights_row, np.float32), 16, "bf16")


def test_row_scales_that_are_no_ordinary_numbers():
    """Zero and subnormal row scales of weights, and the largest."""
    rng = np.random.default_rng(1)
    M, K, N = 2, 2048, 150
    codes, scales = rng.integers(0, 16, (N, K)).astype(np.uint8), rng.integers(0x10, 0x20, (N, K // 16)).astype(np.uint8)
    rs = np.zeros(N, np.float32)
    rs[1::3], rs[2::3] = 2.0 ** -140, 3e38
    x = rng.standard_normal((M, K))
    x[0] *= 1e-4
    check(x * 1e-4, codes, scales, rs, 16, "bf16")


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_the_largest_rows_times_weights_of_one(M, K, N, block):
    """Outputs next to the largest number of bf16, each of one activation: a digit's column counts up to twice what the digits together do."""
    rng = np.random.default_rng(N)
    K += -K % block
    x = rng.uniform(1.0, 1.98, (M, K)) * 2.0 ** 127 * rng.choice([-1.0, 1.0], (M, K))
    x[:, 1::2] = rng.standard_normal((M, K // 2))
    x[0, ::3] = 2.0 ** 127
    codes = np.zeros((N, K), np.uint8)
    codes[np.arange(N), rng.integers(0, K, N)] = rng.choice([2, 10, 1], N)      # 1, -1, 0.5
    scales = np.full((N, K // block), 127 if block == 32 else 0x38, np.uint8)
    check(x, codes, scales, np.ones(N, np.float32), block, "bf16")


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("top", [2.0 ** -100, 2.0 ** -115, 2.0 ** -124, 2.0 ** -128, 2.0 ** -133])
def test_the_smallest_rows(M, K, N, block, top):
    """Down to the type's smallest value a block's numbers are as exact as the header says: off by 2^-141 at most where 2^-21 of the
    block's largest is less."""
    rng = np.random.default_rng(N + 1)
    K += -K % block
    x = rng.uniform(-1.0, 1.0, (M, K)) * top
    codes = rng.integers(0, 16, (N, K)).astype(np.uint8)
    scales = rng.integers(150, 156, (N, K // 32)).astype(np.uint8) if block == 32 else rng.integers(0x30, 0x50, (N, K // 16)).astype(np.uint8)
    check(x, codes, scales, np.full(N, 2.0 ** 25, np.float32), block, "bf16", floor=2.0 ** -141)


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("low", [True, False])
def test_the_smallest_and_largest_block_scales(M, K, N, low):
    """Weights under the scales 2^-127 to 2^-125, or 2^125 to 2^127, and activations that bring the outputs to ordinary sizes: by the decode product, and
    with both operands in 4 bits (quantized activations are exact operands, so that only sums and the type's half step remain)."""
    rng = np.random.default_rng(N + low)
    K += -K % 32
    codes = rng.integers(0, 16, (N, K)).astype(np.uint8)
    scales = rng.integers(0, 3, (N, K // 32)).astype(np.uint8) if low else rng.integers(252, 255, (N, K // 32)).astype(np.uint8)
    x = rng.standard_normal((M, K)) * (2.0 ** 110 if low else 2.0 ** -120)
    check(x, codes, scales, np.ones(N, np.float32), 32, "bf16", floor=2.0 ** -141)
    packed = pack_on_device(codes, scales, np.ones(N, np.float32), 32)
    for rows in (M, 70):
        many = np.tile(x, (-(-rows // M), 1))[:rows]
        dev, held = to_device(many, K, torch.bfloat16)
        a, ws, y = H.alloc_f4(rows, K, 32), H.alloc_workspace_f4(B.OP_GEMM, rows, K, N, 32), H.alloc_matrix(rows, N, torch.bfloat16)
        B.tman_quantize_rows_f4(dev, K, B.DTYPE_BF16, rows, K, 32, a)
        B.tman_mpgemm_f4(packed, a, y, N, B.DTYPE_BF16, rows, K, N, 32, ws)
        assert B.tman_read_status(ws) == 0
        v, w = fo.values(*fo.quantize(held, 32), 32), fo.values(codes, scales, np.ones(N), 32)
        ref, S = v @ w.T, np.abs(v) @ np.abs(w).T
        bad = int((~(np.abs(f64(y) - ref) <= 2.0 ** -8 * np.abs(ref) + (K / 64 + 32) * 2.0 ** -23 * S)).sum())
        assert bad == 0, f"{bad} of {ref.size}"
