"""Microscaled 4-bit floating point in use: runs of calls over shared buffers, streams, graphs, weights quantized on the device, large offsets."""
import numpy as np
import pytest
import torch

from oracle import f4_oracle as fo
from paper_2511_11248_b200 import binding as B, helpers as H
from test_f4_gpu import activations, check_product, f64, pack_on_device, to_device, weights

pytestmark = pytest.mark.gpu


def layer(M, K, N, block, seed):
    """A linear layer's buffers, and what a call of it gives alone."""
    rng = np.random.default_rng(seed)
    packed = pack_on_device(*weights(N, K, block, rng), block)
    dev, held = to_device(activations(M, K, rng), K, torch.float16)
    return packed, dev, H.alloc_f4(M, K, block), H.alloc_workspace_f4(B.OP_GEMM, M, K, N, block), H.alloc_matrix(M, N, torch.float16)


def linear(packed, x, a, ws, y, M, K, N, block, stream=None):
    B.tman_quantize_rows_f4(x, K, 0, M, K, block, a, stream=stream)
    B.tman_mpgemm_f4(packed, a, y, N, 0, M, K, N, block, ws, stream=stream)


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("M,K", [(1, 1024), (5, 4096), (40, 2048), (100, 1024), (300, 512)])
def test_a_run_of_layers_passes_its_buffers_on(M, K, block):
    """Every layer reads what the one before wrote, into the same two matrices and one packed buffer, without a wait between the calls: the same
    bits as with a wait after each."""
    rng = np.random.default_rng(M + K)
    depth = 12
    ws = H.alloc_workspace_f4(B.OP_GEMM, M, K, K, block)
    packs = []
    for _ in range(depth):
        codes, scales, rs = weights(K, K, block, rng)
        if block == 32:
            scales = rng.integers(118, 121, scales.shape).astype(np.uint8)      # outputs of about the inputs' size
        else:
            scales = rng.integers(0x30, 0x38, scales.shape).astype(np.uint8)
            rs[:] = 0.4 / np.sqrt(K)
        packs.append(pack_on_device(codes, scales, rs, block))
    a = H.alloc_f4(M, K, block)
    x0 = to_device(rng.standard_normal((M, K)), K, torch.float16)[0]
    wait = [False]

    def step(i, src, dst):
        if M <= 8 and i % 2:
            B.tman_mpgemv_f4(packs[i], src, K, dst, K, 0, M, K, K, block, ws)
        else:
            B.tman_quantize_rows_f4(src, K, 0, M, K, block, a)
            if wait[0]:
                torch.cuda.synchronize()
            B.tman_mpgemm_f4(packs[i], a, dst, K, 0, M, K, K, block, ws)
        if wait[0]:
            torch.cuda.synchronize()

    def run(bufs):
        bufs[0].copy_(x0)
        for i in range(depth):
            step(i, bufs[i % 2], bufs[(i + 1) % 2])
        torch.cuda.synchronize()
        return bufs[depth % 2].clone()

    bufs = [H.alloc_matrix(M, K, torch.float16), H.alloc_matrix(M, K, torch.float16)]
    wait[0] = True
    want = run(bufs)
    assert bool(torch.isfinite(want).all())
    wait[0] = False
    for _ in range(10):
        assert torch.equal(run(bufs), want)
    # the same run captured in a graph and replayed
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        for i in range(depth):
            step(i, bufs[i % 2], bufs[(i + 1) % 2])
    for _ in range(5):
        bufs[0].copy_(x0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(bufs[depth % 2], want)
    assert B.tman_read_status(ws) == 0


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("M", [3, 200])
def test_weights_quantized_just_before_their_product(M, block):
    """A weight matrix that a quantization wrote on the same stream, used at once, again and again with other contents; calls that let their
    successors start early lie between."""
    rng = np.random.default_rng(M)
    K, N = 1024, 512
    w = [to_device(rng.standard_normal((N, K)) * 0.02, K, torch.float16) for _ in range(4)]
    dev, held = to_device(activations(M, K, rng), K, torch.float16)
    packed, a = H.alloc_f4(N, K, block), H.alloc_f4(M, K, block)
    ws, ws_v = H.alloc_workspace_f4(B.OP_GEMM, M, K, N, block), H.alloc_workspace_f4(B.OP_GEMV, min(M, 8), K, N, block)
    small = layer(2, 512, 256, block, 9)
    outs = [H.alloc_matrix(M, N, torch.float16) for _ in range(8)]
    B.tman_quantize_rows_f4(dev, K, 0, M, K, block, a)
    for rep in range(8):
        B.tman_quantize_rows_f4(w[rep % 4][0], K, 0, N, K, block, packed)
        if rep >= 4:                                  # a kernel that starts early between the quantization and its product
            B.tman_mpgemv_f4(small[0], small[1], 512, small[4], 256, 0, 2, 512, 256, block, small[3])
        if M <= 8:
            B.tman_mpgemv_f4(packed, dev, K, outs[rep], N, 0, M, K, N, block, ws_v)
        else:
            B.tman_mpgemm_f4(packed, a, outs[rep], N, 0, M, K, N, block, ws)
    torch.cuda.synchronize()
    x = held if M <= 8 else fo.values(*fo.quantize(held, block), block)
    for rep in range(8):
        check_product(outs[rep], x, fo.values(*fo.quantize(w[rep % 4][1], block), block), block, "f16", exact_operands=M > 8)


@pytest.mark.parametrize("block", [32, 16])
def test_calls_on_several_streams_at_once(block):
    """Different layers on four streams, each with its own buffers, all of them at once and again: the bits that each gives alone."""
    shapes = [(1, 2048, 1024), (20, 1024, 2048), (150, 1024, 1024), (400, 512, 512)]
    layers = [(layer(M, K, N, block, 50 + M), (M, K, N)) for M, K, N in shapes]
    wants = []
    for (packed, x, a, ws, y), (M, K, N) in layers:
        linear(packed, x, a, ws, y, M, K, N, block)
        torch.cuda.synchronize()
        wants.append(y.clone())
    streams = [torch.cuda.Stream() for _ in shapes]
    for _ in range(20):
        for ((packed, x, a, ws, y), (M, K, N)), s in zip(layers, streams):
            y.fill_(float("nan"))
            s.wait_stream(torch.cuda.current_stream())
            for _ in range(3):
                linear(packed, x, a, ws, y, M, K, N, block, stream=s)
        torch.cuda.synchronize()
        for ((_, _, _, ws, y), _), want in zip(layers, wants):
            assert torch.equal(y, want)
            assert B.tman_read_status(ws) == 0


def test_beside_the_other_decode_calls():
    """Table-lookup decode, 4-bit decode, prefill and 4-bit products in turn on one stream, each reading what the one before wrote."""
    from paper_2511_11248_b200 import synth
    K = 1024
    c = synth.make_case("mix", 2, K, K, 4, 64, 77, 0.002, 0.004)
    devc = H.device_case(c)
    packed_int = H.pack_case(c, devc)
    ws_v, ws_m = H.alloc_workspace(B.OP_GEMV, 2, K, K, 4, 64), H.alloc_workspace(B.OP_GEMM, 2, K, K, 4, 64)
    rng = np.random.default_rng(8)
    codes, scales, rs = weights(K, K, 32, rng)
    packed = pack_on_device(codes, rng.integers(118, 121, scales.shape).astype(np.uint8), rs, 32)
    ws, a = H.alloc_workspace_f4(B.OP_GEMM, 2, K, K, 32), H.alloc_f4(2, K, 32)
    bufs = [H.alloc_matrix(2, K, torch.float16) for _ in range(2)]
    calls = [lambda s, d: B.tman_mpgemv(packed_int, s, d, 2, K, K, 4, 64, ws_v),
             lambda s, d: B.tman_mpgemv_f4(packed, s, K, d, K, 0, 2, K, K, 32, ws),
             lambda s, d: B.tman_mpgemm(packed_int, s, d, 2, K, K, 4, 64, ws_m),
             lambda s, d: (B.tman_quantize_rows_f4(s, K, 0, 2, K, 32, a), B.tman_mpgemm_f4(packed, a, d, K, 0, 2, K, K, 32, ws))]

    def run(wait):
        bufs[0].copy_(devc["x"])
        for i in range(16):
            calls[i % 4](bufs[i % 2], bufs[(i + 1) % 2])
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return bufs[0].clone()

    want = run(True)
    assert bool(torch.isfinite(want).all())
    for _ in range(20):
        assert torch.equal(run(False), want)


@pytest.mark.parametrize("block", [32, 16])
def test_not_finite_activations_make_their_row_nan(block):
    rng = np.random.default_rng(6)
    M, K, N = 6, 4096, 300
    packed = pack_on_device(*weights(N, K, block, rng), block)
    x = activations(M, K, rng)
    x[1, 4000], x[4, 3] = np.nan, -np.inf
    for ty, code in ((torch.float16, 0), (torch.bfloat16, 1)):
        dev, _ = to_device(x, K, ty)
        ws = H.alloc_workspace_f4(B.OP_GEMV, M, K, N, block)
        y = H.alloc_matrix(M, N, ty, fill=0.0)
        B.tman_mpgemv_f4(packed, dev, K, y, N, code, M, K, N, block, ws)
        assert B.tman_read_status(ws) == 0
        assert torch.isnan(y).cpu().all(1).tolist() == [False, True, False, False, True, False]
        assert torch.isnan(y).cpu().any(1).tolist() == [False, True, False, False, True, False]


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("scale", [1e-30, 2.0 ** -126, 1e30])
def test_gemv_of_the_smallest_and_largest_bf16_rows(scale, block):
    """Rows of any magnitude beside ordinary ones: relative to the row, the same tolerance."""
    rng = np.random.default_rng(7)
    M, K, N = 4, 512, 96
    codes, scales, rs = weights(N, K, block, rng)
    packed = pack_on_device(codes, scales, rs, block)
    x = rng.standard_normal((M, K))
    x[1:3] *= scale
    x[3, ::7] = 0.0
    dev, held = to_device(x, K, torch.bfloat16)
    ws = H.alloc_workspace_f4(B.OP_GEMV, M, K, N, block)
    y = H.alloc_matrix(M, N, torch.bfloat16)
    B.tman_mpgemv_f4(packed, dev, K, y, N, 1, M, K, N, block, ws)
    assert B.tman_read_status(ws) == 0
    w = fo.values(codes, scales, rs, block)
    ref, got = held @ w.T, f64(y)
    S = np.abs(held) @ np.abs(w).T
    # half a step of bf16, 2^-16 of the terms' magnitudes for the sums and the fixed-point numbers, and the smallest magnitudes of fp32 and bf16
    assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -16 * S + 2.0 ** -133)


@pytest.mark.parametrize("block", [32, 16])
def test_offsets_beyond_32_bits(block):
    """A weight matrix whose codes alone take 2.3 GB: single channels of the product, and rows of the dequantization, at both ends."""
    N, K = 70001, 65536
    g = torch.Generator(device="cuda").manual_seed(block)
    codes = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda", generator=g)
    scales = torch.randint(112, 120, (N, K // 32), dtype=torch.uint8, device="cuda", generator=g) if block == 32 else \
        torch.randint(8, 100, (N, K // 16), dtype=torch.uint8, device="cuda", generator=g)
    rs = torch.full((N,), 2.0 ** -8, device="cuda")
    packed = torch.empty(B.tman_packed_bytes_f4(N, K, block), dtype=torch.uint8, device="cuda")
    B.tman_pack_f4(codes, scales, rs, N, K, block, packed)
    rng = np.random.default_rng(1)
    dev, held = to_device(rng.standard_normal((2, K)), K, torch.float16)
    ws = H.alloc_workspace_f4(B.OP_GEMM, 2, K, N, block)
    y, y4 = H.alloc_matrix(2, N, torch.float16), H.alloc_matrix(2, N, torch.float16)
    a = H.alloc_f4(2, K, block)
    B.tman_mpgemv_f4(packed, dev, K, y, N, 0, 2, K, N, block, ws)
    B.tman_quantize_rows_f4(dev, K, 0, 2, K, block, a)
    B.tman_mpgemm_f4(packed, a, y4, N, 0, 2, K, N, block, ws)
    assert B.tman_read_status(ws) == 0
    rows = np.unique(np.concatenate([[0, 1, N - 1, N - 2], rng.integers(0, N, 40)]))
    at = torch.from_numpy(rows).cuda()
    c = codes[at].cpu().numpy()
    w = fo.values(np.stack((c & 15, c >> 4), -1).reshape(len(rows), K), scales[at].cpu().numpy(), np.full(len(rows), 2.0 ** -8), block)
    check_product(y[:, at], held, w, block, "f16", exact_operands=False)
    check_product(y4[:, at], fo.values(*fo.quantize(held, block), block), w, block, "f16", exact_operands=True)
    del codes, scales
    out = torch.empty((N, K), dtype=torch.float16, device="cuda")
    B.tman_dequant_rows_f4(packed, N, K, block, out, K, 0, ws)
    assert B.tman_read_status(ws) == 0
    assert torch.equal(out[at].cpu(), torch.from_numpy(w).to(torch.float16))
    again = torch.zeros_like(packed)
    B.tman_quantize_rows_f4(out, K, 0, N, K, block, again)      # what a quantization of the values gives: the same values
    B.tman_dequant_rows_f4(again, N, K, block, out, K, 0, ws)
    want = fo.values(*fo.quantize(torch.from_numpy(w).to(torch.float16).double().numpy(), block), block)
    assert torch.equal(out[at].cpu(), torch.from_numpy(want).to(torch.float16))


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("M", [2, 40, 300])
def test_weights_rewritten_between_calls(M, block):
    """One weight buffer written anew before every product, by a quantization, a packing or a copy, with another quantization in between, so that
    the product may start early: every product is of what was written last."""
    rng = np.random.default_rng(10 + M)
    K, N = 512, 2600
    w = [to_device(rng.standard_normal((N, K)) * 10.0 ** (i - 2), K, torch.float16) for i in range(3)]
    dev, held = to_device(activations(M, K, rng), K, torch.float16)
    packed, a = H.alloc_f4(N, K, block), H.alloc_f4(M, K, block)
    images, plain = [], []
    for x, h in w:
        B.tman_quantize_rows_f4(x, K, 0, N, K, block, packed)
        images.append(packed.clone())
        c, s, r = fo.quantize(h, block)
        plain.append((torch.from_numpy(c[:, 0::2] | (c[:, 1::2] << 4)).cuda(), torch.from_numpy(s).cuda(), torch.from_numpy(r).float().cuda()))
    ws = H.alloc_workspace_f4(B.OP_GEMM, M, K, N, block)
    outs = [H.alloc_matrix(M, N, torch.float16) for _ in range(9)]
    for i, y in enumerate(outs):
        if i % 2 == 0:
            B.tman_quantize_rows_f4(w[i % 3][0], K, 0, N, K, block, packed)
        elif i % 4 == 1:
            B.tman_pack_f4(*plain[i % 3], N, K, block, packed)
        else:
            packed.copy_(images[i % 3])
        B.tman_quantize_rows_f4(dev, K, 0, M, K, block, a)
        if M <= 8:
            B.tman_mpgemv_f4(packed, dev, K, y, N, 0, M, K, N, block, ws)
        else:
            B.tman_mpgemm_f4(packed, a, y, N, 0, M, K, N, block, ws)
    torch.cuda.synchronize()
    x = held if M <= 8 else fo.values(*fo.quantize(held, block), block)
    for i, y in enumerate(outs):
        check_product(y, x, fo.values(*fo.quantize(w[i % 3][1], block), block), block, "f16", exact_operands=M > 8)


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("M", [2, 300])
def test_a_captured_product_of_weights_quantized_on_another_stream(M, block):
    """One graph, two streams joined by events: every replay's product is of the weights that this replay quantized."""
    rng = np.random.default_rng(20 + M)
    K, N = 1024, 2600
    dev, held = to_device(activations(M, K, rng), K, torch.float16)
    src = torch.zeros((N, K), dtype=torch.float16, device="cuda")
    packed, a = H.alloc_f4(N, K, block), H.alloc_f4(M, K, block)
    ws, y = H.alloc_workspace_f4(B.OP_GEMM, M, K, N, block), H.alloc_matrix(M, N, torch.float16)
    B.tman_quantize_rows_f4(dev, K, 0, M, K, block, a)
    B.tman_quantize_rows_f4(src, K, 0, N, K, block, packed)
    B.tman_mpgemm_f4(packed, a, y, N, 0, M, K, N, block, ws)
    torch.cuda.synchronize()
    main, side, g = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=main):
        side.wait_stream(main)
        with torch.cuda.stream(side):
            B.tman_quantize_rows_f4(src, K, 0, N, K, block, packed, stream=side)
        main.wait_stream(side)
        B.tman_mpgemm_f4(packed, a, y, N, 0, M, K, N, block, ws, stream=main)
    x = fo.values(*fo.quantize(held, block), block)
    for i in range(3):
        w, h = to_device(rng.standard_normal((N, K)) * 4.0 ** -i, K, torch.float16)
        src.copy_(w)
        g.replay()
        torch.cuda.synchronize()
        assert B.tman_read_status(ws) == 0
        check_product(y, x, fo.values(*fo.quantize(h, block), block), block, "f16", exact_operands=True)
