"""Products with both operands in 4-bit floating point as prompts run them: every height of a tile, pairs of CTAs that go round several tiles, shares of k, outputs
that leave L2; and the quantization of long rows in front of them."""
import numpy as np
import pytest
import torch

from oracle import f4_oracle as fo
from paper_2511_11248_b200 import binding as B, helpers as H
from test_f4_gpu import TYPES, activations, check_product, pack_on_device, quantize_and_compare, to_device, weights
from test_f4_plan import PROMPTS, SHARES, rounds

pytestmark = pytest.mark.gpu


def product(M, K, N, block, ty, pad):
    """The product twice, bit for bit the same, everything else untouched; channels at the tiles' borders and some between against the oracle."""
    rng = np.random.default_rng(M * 7 + K + N + block)
    dtype, code = TYPES[ty]
    codes, scales, rs = weights(N, K, block, rng)
    packed = pack_on_device(codes, scales, rs, block)
    dev, held = to_device(activations(M, K, rng), K, dtype)
    a = H.alloc_f4(M, K, block)
    a.fill_(0xFF)
    B.tman_quantize_rows_f4(dev, K, code, M, K, block, a)
    ws = H.alloc_workspace_f4(B.OP_GEMM, M, K, N, block)
    y = H.alloc_matrix(M, N + pad, dtype)
    B.tman_mpgemm_f4(packed, a, y, N + pad, code, M, K, N, block, ws)
    first = y.clone()
    for _ in range(2):
        y.fill_(float("nan"))
        B.tman_mpgemm_f4(packed, a, y, N + pad, code, M, K, N, block, ws)
        assert torch.equal(y[:, :N], first[:, :N])
    assert B.tman_read_status(ws) == 0
    assert bool(torch.isnan(y[:, N:]).all()) and bool(torch.isfinite(y[:, :N]).all())
    at = np.unique(np.concatenate([[c for t in range(0, N, 128) for c in (t, t + 1, t + 127) if c < N], [N - 1, max(N - 2, 0)], rng.integers(0, N, 100)]))
    x = fo.values(*fo.quantize(held, block), block)
    check_product(y[:, torch.from_numpy(at).cuda()], x, fo.values(codes[at], scales[at], rs[at], block), block, ty, exact_operands=True)


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("case", PROMPTS, ids=lambda c: "-".join(map(str, c[:4])))
def test_products_of_many_tiles(case, block):
    M, K, N, rows, shares, n, first, past = case
    p = B.tman_debug_f4_plan(1, M, K, N, block)
    assert (p["pair"], p["rows"], p["shares"], rounds(p), p["flags"]) == (1, rows, shares, n, first | past << 1)
    product(M, K, N, block, "bf16" if M % 4 else "f16", 2 * (N % 3) if N % 2 == 0 else N % 4)


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("case", SHARES, ids=lambda c: "-".join(map(str, c)))
def test_products_in_shares_of_k(case, block):
    M, K, N, rows, shares = case
    p = B.tman_debug_f4_plan(1, M, K, N, block)
    assert (p["pair"], p["rows"], p["shares"]) == (1, rows, shares)
    product(M, K, N, block, "f16" if N % 2 else "bf16", 0)


# where streams of weights and pairs of CTAs meet, short and long rings, one share of k and several
@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("K,N", [(288, 200), (14336, 264), (4096, 1001), (2080, 9472), (1056, 9601), (4096, 14336)])
@pytest.mark.parametrize("M", [41, 48, 49, 63, 64, 65])
def test_products_of_few_rows(M, K, N, block):
    product(M, K, N, block, "f16" if M % 2 else "bf16", 0)


# block 16: each number of values that a thread of the quantization holds
@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("rows,K,pad", [(300, 2048, 0), (297, 4112, 8), (300, 8208, 0), (299, 14336, 0), (296, 14352, 8), (300, 18944, 0), (301, 20480, 8), (298, 20496, 0),
                                        (296, 32768, 0), (296, 32784, 0), (295, 24576, 0), (295, 24592, 0)])
def test_quantize_long_rows(rows, K, pad, block):
    if K % block:
        K, pad = K + 16, 0
    rng = np.random.default_rng(rows + K + block)
    quantize_and_compare(activations(rows, K, rng, spread=2.0), K + pad, block, "bf16" if rows % 2 else "f16")
