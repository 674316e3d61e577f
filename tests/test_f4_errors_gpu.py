"""A call of microscaled 4-bit floating point whose launch fails says so, and the calls behind it do not."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2511_11248_b200 import binding as B, helpers as H
from test_f4_gpu import pack_on_device, up, weights

pytestmark = pytest.mark.gpu


class Legacy:
    cuda_stream = 1


def test_a_failed_launch_is_not_reported_by_the_next_call():
    """While a blocking stream is captured, a launch on the legacy default stream fails (and ends the capture); nothing reaches the GPU."""
    rng = np.random.default_rng(0)
    N, K = 64, 256
    codes, scales, rs = weights(N, K, 32, rng)
    packed = pack_on_device(codes, scales, rs, 32)
    args = up(codes[:, 0::2] | (codes[:, 1::2] << 4)), up(scales), up(rs)
    out, x = H.alloc_matrix(N, K, torch.float16), torch.zeros((2, K), dtype=torch.float16, device="cuda")
    y, a = H.alloc_matrix(2, N, torch.float16), H.alloc_f4(2, K, 32)
    ws = H.alloc_workspace_f4(B.OP_GEMM, 2, K, N, 32)
    B.tman_quantize_rows_f4(x, K, 0, 2, K, 32, a)
    torch.cuda.synchronize()
    driver, s, g = C.CDLL("libcuda.so.1"), C.c_void_p(), C.c_void_p()
    assert driver.cuStreamCreate(C.byref(s), 0) == 0
    calls = (lambda t: B.tman_dequant_rows_f4(packed, N, K, 32, out, K, 0, ws, stream=t), lambda t: B.tman_quantize_rows_f4(x, K, 0, 2, K, 32, a, stream=t),
             lambda t: B.tman_mpgemv_f4(packed, x, K, y, N, 0, 2, K, N, 32, ws, stream=t), lambda t: B.tman_mpgemm_f4(packed, a, y, N, 0, 2, K, N, 32, ws, stream=t))
    for call in calls:
        assert driver.cuStreamBeginCapture_v2(s, 0) == 0
        with pytest.raises(B.TmanError) as e:
            call(Legacy)
        assert e.value.status == 6
        driver.cuStreamEndCapture(s, C.byref(g))
        B.tman_pack_f4(*args, N, K, 32, packed)             # asks the runtime for the last error
        call(None)
    torch.cuda.synchronize()
    assert B.tman_read_status(ws) == 0
    assert driver.cuStreamDestroy_v2(s) == 0
