"""Products of 8-bit integers with scales per token and channel on the GPU, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from i8_common import TYPES, f64, rows_on_device, up, within, workspace
from oracle import i8_oracle as io
from paper_2511_11248_b200 import binding as B, helpers as H

pytestmark = pytest.mark.gpu

# A product is an exact integer, rounded to 24 bits, times two scales: three roundings of 2^-24 in front of the output's own; fp16 outputs below
# 2^-14 are off by half of their step, 2^-25 (bf16: 2^-134)
LEAST = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def tolerance(ref, ty):
    return (io.HALF_STEP[ty] + 2.0 ** -22) * np.abs(ref) + LEAST[ty]


def activations(M, K, rng):
    x = rng.standard_normal((M, K)) * np.exp(rng.standard_normal((M, 1)))
    x[:, rng.choice(K, max(1, K // 100), replace=False)] *= 20.0
    return x


def weights(N, K, rng):
    return rng.integers(-127, 128, (N, K)).astype(np.int8), (rng.uniform(0.5, 1.5, N) * 2e-4).astype(np.float32)


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("M,K,pad", [(1, 16, 0), (3, 48, 8), (5, 4096, 0), (129, 1040, 264), (2, 18944, 0), (1, 131056, 8), (1000, 3584, 0)])
def test_token_quantization_is_the_oracles_bit_for_bit(M, K, pad, ty):
    rng = np.random.default_rng(M * 7 + K)
    tt, code = TYPES[ty]
    x = activations(M, K, rng)
    if M > 2:
        x[0] = 0
        x[1] *= 1e-7 if ty == "f16" else 1e-38        # subnormal numbers of the type
        x[2] = np.rint(x[2] * 10) * 0.5                # quotients on and next to halves
        x[2, 0] = 63.5
        x[2] = x[2].clip(-63.5, 63.5)
    xd, xv = rows_on_device(x, K + pad, tt)
    a = H.guarded_bytes(M * K, "codes").view(torch.int8).view(M, K)
    s = H.guarded_bytes(M * 4, "scales").view(torch.float32)
    B.tman_quantize_tokens_i8(xd, K + pad, code, M, K, a, s)
    want, scale = io.quantize_tokens(xv)
    assert np.array_equal(s.cpu().numpy(), scale)
    assert np.array_equal(a.cpu().numpy(), want)
    if ty == "f16" and pad == 0:                       # the call for contiguous fp16 rows
        a2, s2 = torch.empty_like(a), torch.empty_like(s)
        B.tman_quantize_rows_i8(xd, M, K, a2, s2)
        assert torch.equal(a, a2) and torch.equal(s, s2)


SHAPES = [(1, 16, 1), (1, 64, 148), (2, 80, 7), (3, 1040, 1001), (4, 4096, 64), (5, 528, 4737), (8, 2048, 2056), (7, 3584, 300), (1, 14336, 33), (8, 18944, 50)]


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("M,K,N", SHAPES + [(3, 65552, 40), (8, 131056, 9)])
def test_decode(M, K, N, ty):
    rng = np.random.default_rng(M + K + N)
    tt, code = TYPES[ty]
    xd, xv = rows_on_device(activations(M, K, rng), K + 8, tt)
    w, ws_ = weights(N, K, rng)
    y = H.alloc_matrix(M, N + 3, tt)
    ws = workspace(B.tman_workspace_bytes_i8(B.OP_GEMV, M, K, N))
    B.tman_mpgemv_i8(up(w), K, up(ws_), xd, K + 8, y, N + 3, code, M, K, N, ws)
    assert B.tman_read_status(ws) == 0
    a, s = io.quantize_tokens(xv)
    ref = io.product(a, s, w, ws_)
    within(f64(y[:, :N]), ref, tolerance(ref, ty))
    assert bool(torch.isnan(y[:, N:]).all())
    # the two calls it stands for give the same bits
    ad, sd, y2 = torch.empty(M, K, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda"), torch.empty(M, N, dtype=tt, device="cuda")
    B.tman_quantize_tokens_i8(xd, K + 8, code, M, K, ad, sd)
    ws2 = workspace(B.tman_workspace_bytes_i8(B.OP_GEMM, M, K, N))
    B.tman_mpgemm_i8(up(w), K, up(ws_), ad, sd, y2, N, code, M, K, N, ws2)
    assert torch.equal(y[:, :N].contiguous().view(torch.int16), y2.view(torch.int16))


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("M,K,N", [(9, 16, 1), (16, 128, 128), (17, 1040, 1001), (40, 4096, 1000), (64, 144, 257), (65, 256, 4096), (128, 3584, 512), (200, 272, 300),
                                   (257, 1024, 520), (777, 640, 1111), (1030, 512, 2048), (2049, 208, 700)])
def test_prefill(M, K, N, ty):
    rng = np.random.default_rng(M + K + N)
    tt, code = TYPES[ty]
    a = rng.integers(-127, 128, (M, K)).astype(np.int8)
    s = rng.uniform(0.01, 0.1, M).astype(np.float32)
    w, ws_ = weights(N, K, rng)
    wide = np.full((N, K + 32), 77, dtype=np.int8)
    wide[:, :K] = w
    y = H.alloc_matrix(M, N + 5, tt)
    ws = workspace(B.tman_workspace_bytes_i8(B.OP_GEMM, M, K, N))
    B.tman_mpgemm_i8(up(wide), K + 32, up(ws_), up(a), up(s), y, N + 5, code, M, K, N, ws)
    assert B.tman_read_status(ws) == 0
    ref = (a.astype(np.float64) @ w.astype(np.float64).T) * s.astype(np.float64)[:, None] * ws_.astype(np.float64)
    within(f64(y[:, :N]), ref, tolerance(ref, ty))
    assert bool(torch.isnan(y[:, N:]).all())


@pytest.mark.parametrize("M", [1, 8, 40, 300])
def test_sums_at_the_ends_of_32_bits_and_scales_at_the_ends_of_theirs(M):
    K, N = 131056, 24
    a = np.full((M, K), -128, dtype=np.int8)
    w = np.full((N, K), -128, dtype=np.int8)
    w[1::3] = 127
    w[2::3, ::2] = 127
    s = np.full(M, 1e-3, dtype=np.float32)
    ws_ = np.full(N, 1e-6, dtype=np.float32)
    for i, (one, two) in enumerate([(1e30, 1e-34), (1e-30, 1e26), (3e38, 1e-38), (1e-38, 1e30), (1e-44, 1e38), (0.0, 1.0)]):
        if i < M:
            s[i] = one
        ws_[i * 3 % N] = two
    y = H.alloc_matrix(M, N, torch.bfloat16)
    ws = workspace(B.tman_workspace_bytes_i8(B.OP_GEMM, M, K, N))
    B.tman_mpgemm_i8(up(w), K, up(ws_), up(a), up(s), y, N, B.DTYPE_BF16, M, K, N, ws)
    assert B.tman_read_status(ws) == 0
    ref = io.product(a, s, w, ws_)
    big = np.abs(ref) >= 3.3961775e38                    # rounds to an infinity of bf16
    ref[big] = np.sign(ref[big]) * np.inf
    within(f64(y), ref, tolerance(np.where(np.isinf(ref), 0, ref), "bf16"))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("ty", ["f16", "bf16"])
def test_a_row_that_is_no_number_is_nan_and_the_others_are_right(bad, ty):
    rng = np.random.default_rng(5)
    M, K, N = 6, 1040, 65
    tt, code = TYPES[ty]
    x = activations(M, K, rng)
    x[2, 700] = bad
    x[4, 0] = bad
    xd, xv = rows_on_device(x, K, tt)
    w, ws_ = weights(N, K, rng)
    ref = io.product(*io.quantize_tokens(xv), w, ws_)
    y = H.alloc_matrix(M, N, tt, fill=0.0)
    ws = workspace(B.tman_workspace_bytes_i8(B.OP_GEMV, M, K, N))
    B.tman_mpgemv_i8(up(w), K, up(ws_), xd, K, y, N, code, M, K, N, ws)
    within(f64(y), ref, tolerance(np.nan_to_num(ref), ty))
    for rows in (M, 60):
        a, s = torch.empty(rows, K, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
        y2 = H.alloc_matrix(rows, N, tt, fill=0.0)
        B.tman_quantize_tokens_i8(xd.repeat(rows // M, 1), K, code, rows, K, a, s)
        ws2 = workspace(B.tman_workspace_bytes_i8(B.OP_GEMM, rows, K, N))
        B.tman_mpgemm_i8(up(w), K, up(ws_), a, s, y2, N, code, rows, K, N, ws2)
        assert torch.equal(y2.view(torch.int16), y.repeat(rows // M, 1).view(torch.int16)) or rows != M
        within(f64(y2), np.tile(ref, (rows // M, 1)), tolerance(np.nan_to_num(np.tile(ref, (rows // M, 1))), ty))


def test_quantized_weights_are_used_by_the_call_behind_them_and_replays_see_new_ones():
    """A weight matrix quantized on the device directly in front of the products that read it, on a stream of its own, captured and replayed with other
    contents."""
    rng = np.random.default_rng(9)
    K, N, M = 1024, 777, 33
    st = torch.cuda.Stream()
    x16 = torch.empty(N, K, dtype=torch.float16, device="cuda")
    t16 = torch.empty(M, K, dtype=torch.float16, device="cuda")
    w, s = torch.empty(N, K, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    a, sa = torch.empty(M, K, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    y1, yg = H.alloc_matrix(8, N, torch.float16), H.alloc_matrix(M, N, torch.float16)
    ws1, wsg = workspace(B.tman_workspace_bytes_i8(B.OP_GEMV, 8, K, N)), workspace(B.tman_workspace_bytes_i8(B.OP_GEMM, M, K, N))
    st.wait_stream(torch.cuda.current_stream())

    def calls():
        B.tman_quantize_tokens_i8(x16, K, B.DTYPE_F16, N, K, w, s, stream=st)
        B.tman_mpgemv_i8(w, K, s, t16, K, y1, N, B.DTYPE_F16, 8, K, N, ws1, stream=st)
        B.tman_quantize_tokens_i8(t16, K, B.DTYPE_F16, M, K, a, sa, stream=st)
        B.tman_mpgemm_i8(w, K, s, a, sa, yg, N, B.DTYPE_F16, M, K, N, wsg, stream=st)

    with torch.cuda.stream(st):
        calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        calls()
    for _ in range(4):
        xw, xt = rng.standard_normal((N, K)) * 0.02, rng.standard_normal((M, K))
        with torch.cuda.stream(st):
            x16.copy_(up(xw).half())
            t16.copy_(up(xt).half())
            graph.replay()
        st.synchronize()
        wq, wsc = io.quantize_tokens(f64(x16))
        aq, asc = io.quantize_tokens(f64(t16))
        ref = io.product(aq, asc, wq, wsc)
        within(f64(yg), ref, tolerance(ref, "f16"))
        within(f64(y1), ref[:8], tolerance(ref[:8], "f16"))


def test_offsets_beyond_32_bits():
    """Weights of 2^32 bytes and more: rows far apart, the last of them the only ones that are looked at."""
    K, N = 131056, 33000
    w = torch.zeros(N, K, dtype=torch.int8, device="cuda")
    rng = np.random.default_rng(3)
    tail = rng.integers(-127, 128, (40, K)).astype(np.int8)
    w[-40:] = up(tail)
    s = torch.full((N,), 1e-3, device="cuda")
    for M in (2, 70):
        a = rng.integers(-127, 128, (M, K)).astype(np.int8)
        sa = np.full(M, 1e-4, dtype=np.float32)
        y = H.alloc_matrix(M, N, torch.bfloat16)
        ws = workspace(B.tman_workspace_bytes_i8(B.OP_GEMM, M, K, N))
        B.tman_mpgemm_i8(w, K, s, up(a), up(sa), y, N, B.DTYPE_BF16, M, K, N, ws)
        assert B.tman_read_status(ws) == 0
        ref = io.product(a, sa, tail, np.full(40, 1e-3, dtype=np.float32))
        within(f64(y[:, -40:]), ref, tolerance(ref, "bf16"))
        assert bool((y[:, :-40] == 0).all())
