"""Microscaled 4-bit floating point on the GPU against the oracle in 64 bits: packing, quantization and dequantization bit for bit, the products
to the roundings that they make."""
import numpy as np
import pytest
import torch

from oracle import f4_oracle as fo
from paper_2511_11248_b200 import binding as B, helpers as H

pytestmark = pytest.mark.gpu

TYPES = {"f16": (torch.float16, B.DTYPE_F16), "bf16": (torch.bfloat16, B.DTYPE_BF16)}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def up(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def activations(M, K, rng, spread=1.0):
    x = rng.standard_normal((M, K)) * np.exp(spread * rng.standard_normal((M, 1)))
    x[:, rng.choice(K, max(1, K // 100), replace=False)] *= 20.0
    return x


def to_device(x, ld, dtype):
    """x [M][K] as the first columns of rows of ld values; the columns behind are NaN.  Returns the device view and the values it holds."""
    wide = torch.full((x.shape[0], ld), float("nan"), dtype=dtype, device="cuda")
    wide[:, :x.shape[1]] = up(x).to(dtype)
    return wide, f64(wide[:, :x.shape[1]])


def weights(N, K, block, rng):
    codes = rng.integers(0, 16, (N, K)).astype(np.uint8)
    if block == 32:
        return codes, rng.integers(112, 122, (N, K // 32)).astype(np.uint8), np.ones(N, dtype=np.float32)
    return codes, rng.integers(0x08, 0x7F, (N, K // 16)).astype(np.uint8), rng.uniform(1e-4, 1e-3, N).astype(np.float32)


def pack_on_device(codes, scales, rs, block):
    N, K = codes.shape
    packed = H.alloc_f4(N, K, block)
    B.tman_pack_f4(up(codes[:, 0::2] | (codes[:, 1::2] << 4)), up(scales), up(rs), N, K, block, packed)
    return packed


def check_product(y, x, w, block, ty, exact_operands):
    """|y - x w^T| <= half a step of y's type + what the sums in 32 bits may lose: every addition 2^-23 of the partial sums, which are at most
    S = sum |x w|, in K / 64 + 32 additions (an instruction's products count as one); 16-bit activations as fixed-point numbers of
    their block: 2^-20 of its largest value in each."""
    ref = x @ w.T
    S = np.abs(x) @ np.abs(w).T
    K = x.shape[1]
    tol = HALF_STEP[ty] * np.abs(ref) + (K / 64 + 32) * 2.0 ** -23 * S + 2.0 ** -24
    if not exact_operands:
        top = np.abs(x).reshape(x.shape[0], -1, block).max(-1)
        tol += 2.0 ** -20 * (top @ np.abs(w).reshape(w.shape[0], -1, block).sum(-1).T)
    got = f64(y)
    assert np.isfinite(got).all()
    worst = np.max(np.abs(got - ref) / tol)
    assert worst <= 1.0, worst


SHAPES = [(1, 32), (3, 96), (8, 128), (9, 160), (40, 1056), (128, 256), (129, 288), (257, 640), (1001, 1184)]


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("rows,K", SHAPES + [(2, 16), (130, 1040)])
def test_pack_writes_the_layout_and_unpack_reads_it(rows, K, block):
    if K % block:
        K += block - K % block
    rng = np.random.default_rng(rows * 1000 + K + block)
    codes, scales, rs = weights(rows, K, block, rng)
    packed = pack_on_device(codes, scales, rs, block)
    assert np.array_equal(packed.cpu().numpy(), fo.pack(codes, scales, rs, block))
    ws = H.alloc_workspace_f4(B.OP_AUX, 1, K, rows, block)
    c = H.guarded_bytes(rows * K // 2, "codes")
    s = H.guarded_bytes(rows * (K // block), "scales")
    r = H.guarded_bytes(rows * 4, "row scales").view(torch.float32)
    B.tman_unpack_f4(packed, rows, K, block, c, s, r, ws)
    assert B.tman_read_status(ws) == 0
    c = c.cpu().numpy().reshape(rows, K // 2)
    assert np.array_equal(c & 15, codes[:, 0::2]) and np.array_equal(c >> 4, codes[:, 1::2])
    assert np.array_equal(s.cpu().numpy().reshape(rows, -1), scales)
    assert np.array_equal(r.cpu().numpy(), rs)


def unpacked(packed, rows, K, block):
    ws = H.alloc_workspace_f4(B.OP_AUX, 1, K, rows, block)
    c = torch.empty((rows, K // 2), dtype=torch.uint8, device="cuda")
    s = torch.empty((rows, K // block), dtype=torch.uint8, device="cuda")
    r = torch.empty(rows, dtype=torch.float32, device="cuda")
    B.tman_unpack_f4(packed, rows, K, block, c, s, r, ws)
    assert B.tman_read_status(ws) == 0
    c = c.cpu().numpy()
    return np.stack((c & 15, c >> 4), -1).reshape(rows, K), s.cpu().numpy(), r.cpu().numpy()


def quantize_and_compare(x, ld, block, ty):
    dtype, code = TYPES[ty]
    rows, K = x.shape
    dev, held = to_device(x, ld, dtype)
    packed = H.alloc_f4(rows, K, block)
    packed.fill_(0xA5)
    B.tman_quantize_rows_f4(dev, ld, code, rows, K, block, packed)
    c, s, r = unpacked(packed, rows, K, block)
    want_c, want_s, want_r = fo.quantize(held, block)
    assert np.array_equal(r, want_r.astype(np.float32))
    assert np.array_equal(s, want_s)
    fine = np.repeat(np.isfinite(held).reshape(rows, -1, block).all(-1), block, axis=1)
    assert np.array_equal(c[fine], want_c[fine])
    ws = H.alloc_workspace_f4(B.OP_AUX, 1, K, rows, block)
    out = H.alloc_matrix(rows, ld, dtype, fill=7.0)
    B.tman_dequant_rows_f4(packed, rows, K, block, out, ld, code, ws)
    assert B.tman_read_status(ws) == 0
    want = torch.from_numpy(fo.values(want_c, want_s, want_r, block)).to(dtype)
    want[~torch.from_numpy(fine)] = float("nan")
    got = out.cpu()
    assert bool((got[:, K:] == 7.0).all())
    assert torch.equal(torch.nan_to_num(got[:, :K], nan=12345.0), torch.nan_to_num(want, nan=12345.0))
    return held, want_s


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("rows,K,pad", [(1, 32, 0), (1, 4096, 0), (3, 96, 8), (8, 1120, 0), (37, 2080, 24), (300, 640, 0), (7, 18944, 0), (2, 65568, 0)])
def test_quantize_and_dequantize(rows, K, pad, block, ty):
    rng = np.random.default_rng(rows + K + block)
    quantize_and_compare(activations(rows, K, rng, spread=2.0), K + pad, block, ty)


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("block", [32, 16])
def test_quantize_every_finite_value_of_the_type(block, ty):
    """All 2^16 bit patterns, shuffled; those that are not finite make their block NaN."""
    rng = np.random.default_rng(5)
    bits = rng.permutation(65536).astype(np.uint16).reshape(64, 1024)
    dtype, code = TYPES[ty]
    dev = torch.from_numpy(bits.view(np.int16)).cuda().view(dtype)
    for fill in (False, True):
        x = dev.clone()
        if fill:                                      # without the values that are not finite, and with rows of one magnitude
            x = torch.nan_to_num(x, nan=0.0, posinf=1.0, neginf=-1.0)
            x = x.flatten()[x.flatten().abs().float().argsort()].view(64, 1024)
        quantize_and_compare(f64(x), 1024, block, ty)


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("block", [32, 16])
def test_quantize_ties(block, ty):
    """x = (half way between two codes) x (every scale a block can have): exact ties go to the even code."""
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    x = np.zeros((16, 64))
    for i in range(16):
        for b in range(64 // block):
            s = (8 + i % 8) / 8.0 * 2.0 ** (b - 2 + i // 8) if block == 16 else 2.0 ** (i + b - 8)
            x[i, b * block:b * block + 7] = ties * s
            x[i, b * block + 7] = 6 * s
            x[i, b * block + 8:b * block + 15] = -ties * s
    quantize_and_compare(x, 64, block, ty)


@pytest.mark.parametrize("block", [32, 16])
def test_quantize_rows_of_zeros_infinities_and_the_smallest_values(block):
    for ty in ("f16", "bf16"):
        tiny = 2.0 ** -24 if ty == "f16" else 2.0 ** -133
        x = np.zeros((6, 128))
        x[1, 5] = np.inf
        x[1, 100] = 3.0
        x[2, 70] = np.nan
        x[2, 3] = -2.0
        x[3, :] = tiny
        x[4, ::3] = -tiny
        x[5, :] = 65504.0 if ty == "f16" else 3.0e38
        quantize_and_compare(x, 128, block, ty)


GEMV = [(1, 32, 1), (1, 4096, 1024), (2, 160, 200), (3, 1056, 1001), (4, 512, 128), (5, 2080, 257), (7, 96, 130), (8, 1024, 264), (8, 14336, 520), (1, 18944, 72),
        (6, 128, 4100)]


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("M,K,N", GEMV)
def test_gemv(M, K, N, block, ty):
    rng = np.random.default_rng(M * 7 + K + N + block)
    dtype, code = TYPES[ty]
    codes, scales, rs = weights(N, K, block, rng)
    packed = pack_on_device(codes, scales, rs, block)
    dev, held = to_device(activations(M, K, rng), K + 8, dtype)
    ws = H.alloc_workspace_f4(B.OP_GEMV, M, K, N, block)
    y = H.alloc_matrix(M, N + 3, dtype)
    for _ in range(2):                                # the second call finds the first one's workspace
        y.fill_(float("nan"))
        B.tman_mpgemv_f4(packed, dev, K + 8, y, N + 3, code, M, K, N, block, ws)
        assert B.tman_read_status(ws) == 0
        assert bool(torch.isnan(y[:, N:]).all())
        check_product(y[:, :N], held, fo.values(codes, scales, rs, block), block, ty, exact_operands=False)


# As many tiles as there are SMs or more, so that one CTA has all of k, and rings that are full (K of 16 units and more): of an odd M the products'
# last columns reach behind the digits of the last stage.
@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("M,K,N", [(1, 4096, 14336), (3, 4096, 18944), (5, 4096, 18944), (7, 4352, 18945), (8, 1376, 18944), (1, 5152, 19001)])
def test_gemv_with_a_full_ring_and_whole_rows_of_k(M, K, N, block, ty):
    test_gemv(M, K, N, block, ty)


GEMM = [(1, 32, 1), (1, 4096, 1024), (2, 288, 130), (9, 160, 200), (16, 1056, 1001), (33, 640, 257), (100, 512, 384), (128, 1024, 264), (129, 2080, 136), (200, 4096, 96),
        (257, 96, 513), (300, 1184, 1000), (520, 256, 72), (1030, 768, 520), (17, 18944, 200)]


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("M,K,N", GEMM)
def test_gemm(M, K, N, block, ty):
    rng = np.random.default_rng(M * 7 + K + N + block)
    dtype, code = TYPES[ty]
    codes, scales, rs = weights(N, K, block, rng)
    packed = pack_on_device(codes, scales, rs, block)
    dev, held = to_device(activations(M, K, rng), K, dtype)
    a = H.alloc_f4(M, K, block)
    a.fill_(0xFF)                                     # bytes that belong to no row are anything, scales that are NaN among them
    B.tman_quantize_rows_f4(dev, K, code, M, K, block, a)
    ws = H.alloc_workspace_f4(B.OP_GEMM, M, K, N, block)
    y = H.alloc_matrix(M, N + 3, dtype)
    for _ in range(2):
        y.fill_(float("nan"))
        B.tman_mpgemm_f4(packed, a, y, N + 3, code, M, K, N, block, ws)
        assert B.tman_read_status(ws) == 0
        assert bool(torch.isnan(y[:, N:]).all())
        check_product(y[:, :N], fo.values(*fo.quantize(held, block), block), fo.values(codes, scales, rs, block), block, ty, exact_operands=True)


@pytest.mark.parametrize("block", [32, 16])
def test_a_block_that_is_not_finite_makes_its_row_nan_and_no_other(block):
    rng = np.random.default_rng(3)
    M, K, N = 5, 512, 300
    codes, scales, rs = weights(N, K, block, rng)
    packed = pack_on_device(codes, scales, rs, block)
    x = activations(M, K, rng)
    x[1, 200] = np.nan
    x[3, 17] = np.inf
    dev, _ = to_device(x, K, torch.float16)
    a = H.alloc_f4(M, K, block)
    B.tman_quantize_rows_f4(dev, K, 0, M, K, block, a)
    ws = H.alloc_workspace_f4(B.OP_GEMM, M, K, N, block)
    y = H.alloc_matrix(M, N, torch.float16, fill=0.0)
    B.tman_mpgemm_f4(packed, a, y, N, 0, M, K, N, block, ws)
    assert B.tman_read_status(ws) == 0
    assert torch.isnan(y).cpu().all(1).tolist() == [False, True, False, True, False]
    assert torch.isnan(y).cpu().any(1).tolist() == [False, True, False, True, False]


def test_headers_that_do_not_match_leave_the_output():
    rng = np.random.default_rng(4)
    M, K, N, block = 3, 256, 40, 32
    codes, scales, rs = weights(N, K, block, rng)
    packed = pack_on_device(codes, scales, rs, block)
    other = pack_on_device(*weights(N, K, 16, rng), 16)          # a buffer of the other block, large enough
    dev, _ = to_device(activations(M, K, rng), K, torch.float16)
    a = H.alloc_f4(M, K, block)
    B.tman_quantize_rows_f4(dev, K, 0, M, K, block, a)
    y = H.alloc_matrix(M, N, torch.float16, fill=3.0)
    out = H.alloc_matrix(N, K, torch.float16, fill=3.0)
    bad_a = torch.zeros_like(a)
    ws = H.alloc_workspace_f4(B.OP_GEMV, M, K, N, block)
    B.tman_mpgemv_f4(other, dev, K, y, N, 0, M, K, N, block, ws)
    assert B.tman_read_status(ws) == 5
    for w_buf, a_buf in ((other, a), (packed, bad_a)):
        ws = H.alloc_workspace_f4(B.OP_GEMM, M, K, N, block)
        B.tman_mpgemm_f4(w_buf, a_buf, y, N, 0, M, K, N, block, ws)
        assert B.tman_read_status(ws) == 5
    ws = H.alloc_workspace_f4(B.OP_AUX, M, K, N, block)
    B.tman_dequant_rows_f4(other, N, K, block, out, K, 0, ws)
    assert B.tman_read_status(ws) == 5
    c, s = H.guarded_bytes(N * K // 2, "codes"), H.guarded_bytes(N * K // 32, "scales")
    c.fill_(9), s.fill_(9)
    ws = H.alloc_workspace_f4(B.OP_AUX, M, K, N, block)
    B.tman_unpack_f4(other, N, K, block, c, s, None, ws)
    assert B.tman_read_status(ws) == 5
    assert bool((y == 3.0).all()) and bool((out == 3.0).all()) and bool((c == 9).all()) and bool((s == 9).all())


# few tiles and a long reduction: shares of k of a tile on a cluster of pairs of CTAs
@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("M,K,N", [(65, 4096, 256), (100, 2048, 1000), (129, 8256, 300), (250, 14336, 513), (600, 5152, 96), (1030, 2080, 250)])
def test_gemm_of_few_tiles(M, K, N, block):
    test_gemm(M, K, N, block, "bf16")


@pytest.mark.parametrize("M,K,N", [(20, 512, 264), (300, 512, 520), (300, 4096, 264), (201, 4096, 131)])
def test_row_scales_whose_product_leaves_the_range(M, K, N):
    """Row scales of 2^36 and about 2^93: their product is no fp32 number, the sums times both are.  Odd channels have one weight, 2^-10 x 2^36, even
    ones none: exact products, so that only the type's half step is left, and zeros stay zeros."""
    rng = np.random.default_rng(M + N)
    codes = np.zeros((N, K), np.uint8)
    codes[1::2, 0] = 1                                # 0.5
    scales = np.ones((N, K // 16), np.uint8)          # e4m3 2^-9
    packed = pack_on_device(codes, scales, np.full(N, 2.0 ** 36, np.float32), 16)
    x = rng.uniform(0.5, 1.0, (M, K)) * 2.0 ** 104
    x[:, :16] *= 2.0 ** -8
    dev, held = to_device(x, K, torch.bfloat16)
    a = H.alloc_f4(M, K, 16)
    B.tman_quantize_rows_f4(dev, K, B.DTYPE_BF16, M, K, 16, a)
    ws, y = H.alloc_workspace_f4(B.OP_GEMM, M, K, N, 16), H.alloc_matrix(M, N, torch.bfloat16)
    B.tman_mpgemm_f4(packed, a, y, N, B.DTYPE_BF16, M, K, N, 16, ws)
    assert B.tman_read_status(ws) == 0
    ref = np.zeros((M, N))
    ref[:, 1::2] = fo.values(*fo.quantize(held, 16), 16)[:, :1] * 2.0 ** 26
    got = f64(y)
    assert np.all(got[:, ::2] == 0)
    assert np.all(np.abs(got - ref) <= HALF_STEP["bf16"] * np.abs(ref))
