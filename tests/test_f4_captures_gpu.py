"""Eager and captured calls of microscaled 4-bit floating point on the same stream and the same weights."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2511_11248_b200 import binding as B, helpers as H
from test_f4_gpu import activations, pack_on_device, to_device, weights

pytestmark = pytest.mark.gpu
PROGRAMMATIC = 1                                      # cudaGraphDependencyType


def capture(stream, body):
    g = torch.cuda.CUDAGraph(keep_graph=True)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=stream):
        body()
    return g


def edge_types(g):
    """Of the edges of a graph that is a chain, from its first node to its last."""
    driver, graph, n = C.CDLL("libcuda.so.1"), C.c_void_p(g.raw_cuda_graph()), C.c_size_t(0)
    assert driver.cuGraphGetEdges_v2(graph, None, None, None, C.byref(n)) == 0
    ends, begins, data = (C.c_void_p * n.value)(), (C.c_void_p * n.value)(), (C.c_uint8 * (8 * n.value))()      # (edge data: from port, to port, type, 5 reserved)
    assert driver.cuGraphGetEdges_v2(graph, ends, begins, data, C.byref(n)) == 0
    follow = {ends[i]: (begins[i], data[8 * i + 2]) for i in range(n.value)}
    assert len(follow) == n.value
    at, = set(follow) - {b for b, _ in follow.values()}
    types = []
    while at in follow:
        at, t = follow[at]
        types.append(t)
    return types


# every kernel that quantizes
@pytest.mark.parametrize("ty", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("block,rows,K", [(32, 40, 512), (32, 2400, 512), (16, 40, 512), (16, 40, 8448), (16, 40, 32896), (16, 300, 512), (16, 300, 4096), (16, 300, 8192),
                                          (16, 300, 8448), (16, 300, 16384), (16, 300, 20736), (16, 300, 32896)])
def test_edges_of_a_captured_product(block, rows, K, ty):
    """Behind the quantization of its weights a product waits for all of it, behind another quantization it may start early."""
    code = B.DTYPE_F16 if ty == torch.float16 else B.DTYPE_BF16
    w, x = torch.zeros((rows, K), dtype=ty, device="cuda"), torch.zeros((2, K), dtype=ty, device="cuda")
    packed, a, y = H.alloc_f4(rows, K, block), H.alloc_f4(2, K, block), H.alloc_matrix(2, rows, ty)
    ws = H.alloc_workspace_f4(B.OP_GEMM, 2, K, rows, block)
    s = torch.cuda.Stream()

    def of_w():
        B.tman_quantize_rows_f4(w, K, code, rows, K, block, packed)

    def of_a():
        B.tman_quantize_rows_f4(x, K, code, 2, K, block, a)

    for first, second, last in ((of_w, of_a, PROGRAMMATIC), (of_a, of_w, 0)):
        g = capture(s, lambda: (first(), second(), B.tman_mpgemm_f4(packed, a, y, rows, code, 2, K, rows, block, ws)))
        types = edge_types(g)
        assert types[-1] == last and all(t == PROGRAMMATIC for t in types[:-1]), types
        g = capture(s, lambda: (first(), second(), B.tman_mpgemv_f4(packed, x, K, y, rows, code, 2, K, rows, block, ws)))
        assert edge_types(g)[-1] == last


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("M", [2, 40, 300])
def test_captures_between_a_quantization_and_its_product(M, block):
    """Weights quantized eagerly; while that runs, a product of them and another quantization are captured on the same stream; then the eager
    product: of the weights that were written last, like the replay."""
    rng = np.random.default_rng(M + block)
    K, N = 2048, 8192
    x, _ = to_device(activations(M, K, rng), K, torch.float16)
    w = [to_device(rng.standard_normal((N, K)) * 4.0 ** -i, K, torch.float16)[0] for i in range(3)]
    packed, a, other = H.alloc_f4(N, K, block), H.alloc_f4(M, K, block), H.alloc_f4(M, K, block)
    ws, y, y_graph = H.alloc_workspace_f4(B.OP_GEMM, M, K, N, block), H.alloc_matrix(M, N, torch.float16), H.alloc_matrix(M, N, torch.float16)
    s = torch.cuda.Stream()

    def product(out):
        if M <= 8:
            B.tman_mpgemv_f4(packed, x, K, out, N, 0, M, K, N, block, ws)
        else:
            B.tman_mpgemm_f4(packed, a, out, N, 0, M, K, N, block, ws)

    wants = []
    B.tman_quantize_rows_f4(x, K, 0, M, K, block, a)
    for v in w:
        B.tman_quantize_rows_f4(v, K, 0, N, K, block, packed)
        torch.cuda.synchronize()
        product(y)
        wants.append(y.clone())
    torch.cuda.synchronize()
    for rep in range(6):
        with torch.cuda.stream(s):
            B.tman_quantize_rows_f4(w[rep % 3], K, 0, N, K, block, packed)
            g = torch.cuda.CUDAGraph()
            g.capture_begin()
            product(y_graph)
            B.tman_quantize_rows_f4(x, K, 0, M, K, block, other)
            g.capture_end()
            product(y)
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, wants[rep % 3]) and torch.equal(y_graph, wants[rep % 3])
    assert B.tman_read_status(ws) == 0


@pytest.mark.parametrize("block", [32, 16])
def test_a_product_behind_the_replay_of_its_weights_quantization(block):
    rng = np.random.default_rng(block)
    M, K, N = 3, 2048, 8192
    x, _ = to_device(activations(M, K, rng), K, torch.float16)
    w = [to_device(rng.standard_normal((N, K)) * 4.0 ** -i, K, torch.float16)[0] for i in range(3)]
    src, packed = torch.empty_like(w[0]), H.alloc_f4(N, K, block)
    ws, y = H.alloc_workspace_f4(B.OP_GEMV, M, K, N, block), H.alloc_matrix(M, N, torch.float16)
    s = torch.cuda.Stream()
    g = capture(s, lambda: B.tman_quantize_rows_f4(src, K, 0, N, K, block, packed))
    want = []
    for v in w:
        B.tman_quantize_rows_f4(v, K, 0, N, K, block, packed)
        torch.cuda.synchronize()
        B.tman_mpgemv_f4(packed, x, K, y, N, 0, M, K, N, block, ws)
        want.append(y.clone())
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for rep in range(12):
            src.copy_(w[rep % 3])
            g.replay()
            B.tman_mpgemv_f4(packed, x, K, y, N, 0, M, K, N, block, ws)
            s.synchronize()
            assert torch.equal(y, want[rep % 3])
    assert B.tman_read_status(ws) == 0
