"""Microscaled 4-bit floating point without a GPU: buffer sizes, refusals before any launch, and pins of the oracle's format."""
import ctypes as C

import numpy as np
import pytest

from oracle import f4_oracle as fo


@pytest.fixture(scope="module")
def lib():
    from paper_2511_11248_b200 import build, binding
    build.build()
    return binding.lib()


class Fake:
    """Stands for a device tensor: an address and a size, never read."""

    def __init__(self, address, nbytes):
        self.address, self.nbytes = address, nbytes

    def data_ptr(self):
        return self.address

    def numel(self):
        return self.nbytes

    def element_size(self):
        return 1


def test_packed_bytes_follow_the_layout(lib):
    from paper_2511_11248_b200 import binding as B
    for rows, K, block in [(1, 32, 32), (1, 16, 16), (8, 128, 32), (129, 160, 32), (1001, 1040, 16), (4096, 14336, 32), (18944, 3584, 16)]:
        assert B.tman_packed_bytes_f4(rows, K, block) == fo.sections(rows, K, block)[3]


@pytest.mark.parametrize("rows,K,block", [(0, 32, 32), (1, 0, 32), (1, 48, 32), (1, 24, 16), (1, 64, 64), (-3, 32, 32), (1, 32, 0)])
def test_bad_shapes_are_refused(lib, rows, K, block):
    from paper_2511_11248_b200 import binding as B
    for call in (lambda: B.tman_packed_bytes_f4(rows, K, block), lambda: B.tman_workspace_bytes_f4(1, 4, K, rows, block)):
        with pytest.raises(B.TmanError) as e:
            call()
        assert e.value.status == 2


def _calls(B, **over):
    """Every call with arguments that are right except for `over`; nothing is launched as long as one is wrong."""
    a = dict(K=256, N=40, M=4, block=32, dtype=0, ldx=256, ldy=40, x=Fake(1 << 20, 4096), y=Fake(1 << 21, 4096), ws=Fake(1 << 22, 1 << 24),
             w=Fake(1 << 23, 1 << 20), a=Fake(1 << 24, 1 << 20), stream=Stream())
    a.update(over)
    g = type("A", (), a)
    return {
        "quantize": lambda: B.tman_quantize_rows_f4(g.x, g.ldx, g.dtype, g.M, g.K, g.block, g.a, stream=g.stream),
        "dequant": lambda: B.tman_dequant_rows_f4(g.a, g.M, g.K, g.block, g.x, g.ldx, g.dtype, g.ws, stream=g.stream),
        "gemv": lambda: B.tman_mpgemv_f4(g.w, g.x, g.ldx, g.y, g.ldy, g.dtype, g.M, g.K, g.N, g.block, g.ws, stream=g.stream),
        "gemm": lambda: B.tman_mpgemm_f4(g.w, g.a, g.y, g.ldy, g.dtype, g.M, g.K, g.N, g.block, g.ws, stream=g.stream),
    }


class Stream:
    cuda_stream = 0


ALL = ("quantize", "dequant", "gemv", "gemm")


@pytest.mark.parametrize("over,status,calls", [
    (dict(K=0), 2, ALL), (dict(K=80), 2, ALL), (dict(block=64), 2, ALL), (dict(M=0), 2, ALL), (dict(M=9), 2, ("gemv",)), (dict(N=0), 2, ("gemv", "gemm")),
    (dict(dtype=2), 3, ALL), (dict(ldx=248), 2, ("quantize", "dequant", "gemv")), (dict(ldx=260), 2, ("quantize", "dequant", "gemv")),
    (dict(ldy=39), 2, ("gemv", "gemm")), (dict(x=Fake((1 << 20) + 8, 4096)), 2, ("quantize", "dequant", "gemv")),
    (dict(y=Fake((1 << 21) + 1, 4096)), 2, ("gemv", "gemm")), (dict(ws=Fake((1 << 22) + 16, 1 << 24)), 2, ("dequant", "gemv", "gemm")),
    (dict(ws=Fake(1 << 22, 128)), 4, ("dequant", "gemv", "gemm")), (dict(w=Fake(1 << 23, 1000)), 4, ("gemv", "gemm")),
    (dict(w=Fake((1 << 23) + 128, 1 << 20)), 2, ("gemv", "gemm")), (dict(a=Fake(1 << 24, 1000)), 4, ("quantize", "dequant", "gemm")),
    (dict(a=Fake((1 << 24) + 64, 1 << 20)), 2, ("quantize", "dequant", "gemm")),
    (dict(x=Fake(0, 4096)), 1, ("quantize", "dequant", "gemv")), (dict(y=Fake(0, 4096)), 1, ("gemv", "gemm")), (dict(w=Fake(0, 1 << 20)), 1, ("gemv", "gemm")),
    (dict(a=Fake(0, 1 << 20)), 1, ("quantize", "dequant", "gemm")), (dict(ws=Fake(0, 1 << 24)), 1, ("dequant", "gemv", "gemm"))])
def test_wrong_arguments_are_refused_before_any_launch(lib, over, status, calls):
    from paper_2511_11248_b200 import binding as B
    table = _calls(B, **over)
    for name in calls:
        with pytest.raises(B.TmanError) as e:
            table[name]()
        assert e.value.status == status, name


def test_pack_refusals(lib):
    out = C.c_size_t(0)
    assert lib.tman_packed_bytes_f4(8, 64, 32, None) == 1
    assert lib.tman_workspace_bytes_f4(3, 1, 64, 8, 32, C.byref(out)) == 3
    assert lib.tman_workspace_bytes_f4(0, 9, 64, 8, 32, C.byref(out)) == 2
    big, ws = 1 << 20, 1 << 24
    assert lib.tman_pack_f4(None, 4096, None, 8, 64, 32, ws, big, None) == 1
    assert lib.tman_pack_f4(4096, None, None, 8, 64, 32, ws, big, None) == 1
    assert lib.tman_pack_f4(4096, 4096, None, 8, 64, 32, None, big, None) == 1
    assert lib.tman_pack_f4(4096, 4096, None, 8, 64, 32, ws, 100, None) == 4
    assert lib.tman_pack_f4(4096, 4096, None, 8, 64, 32, ws + 16, big, None) == 2
    assert lib.tman_pack_f4(4096, 4096, 4098, 8, 64, 16, ws, big, None) == 2
    assert lib.tman_unpack_f4(ws, 100, 8, 64, 32, 4096, 4096, None, ws, 256, None) == 4
    assert lib.tman_unpack_f4(ws, big, 8, 64, 32, 4096, 4096, None, ws, 64, None) == 4
    assert lib.tman_unpack_f4(ws, big, 8, 64, 32, 4096, 4096, None, None, 256, None) == 1
    assert lib.tman_unpack_f4(ws, big, 8, 65, 32, 4096, 4096, None, ws, 256, None) == 2


def test_oracle_rounds_to_nearest_even_and_saturates():
    v = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.2500001, 4.999999, 7.0])
    assert list(fo.E2M1[fo.nearest(v, fo.E2M1[:8])]) == [0, 1, 1, 2, 2, 4, 4, 0.5, 4, 6]
    g = fo.e4m3_values()
    assert g[0x7E] == 448 and np.isnan(g[0x7F]) and g[1] == 2.0 ** -9 and g[8] == 2.0 ** -6 and g[0x38] == 1.0


def test_oracle_quantization_of_known_blocks():
    x = np.zeros((1, 32))
    x[0, :4] = [12.0, -3.0, 1.0, 0.25]            # top 12 = 1.5 x 2^3: scale 2
    c, s, _ = fo.quantize(x, 32)
    assert s[0, 0] == 128 and list(fo.E2M1[c[0, :4]]) == [6, -1.5, 0.5, 0]
    c, s, r = fo.quantize(x, 16)                   # row scale: 12 <= 2688 r -> 2^-7; block scale 12 / 6 x 128 = 256
    assert r[0] == 2.0 ** -7 and fo.e4m3_values()[s[0, 0]] == 256 and s[0, 1] == 0 and list(fo.E2M1[c[0, :4]]) == [6, -1.5, 0.5, 0]


# ---- what no run shows -------------------------------------------------------------------------------------------------------------------


def _digit_ring(M, stages, units, rng, warps=16):
    """The decode kernel's ring: digit warps (row m, every `teams`-th unit), the loading warp and the multiplying one take turns in any order that
    their waits allow.  A wait for a free slot sees parity alone.  Returns what went wrong."""
    teams = min(warps // M, stages)
    actors = [(t, m) for t in range(teams) for m in range(M)]
    at = {w: w[0] for w in actors}
    freed, arrived, loaded, consumed = [0] * stages, [0] * units, 0, 0
    free = lambda i: i < stages or (freed[i % stages] & 1) != ((i // stages - 1) & 1)
    while consumed < units:
        moves = [w for w in actors if at[w] < units and free(at[w])]
        if loaded < units and free(loaded):
            moves.append("load")
        if loaded > consumed and arrived[consumed] == M:
            moves.append("multiply")
        if not moves:
            return "stuck"
        move = moves[rng.integers(len(moves))]
        i = loaded if move == "load" else at.get(move, 0)
        if move != "multiply" and i - stages >= consumed:
            return "slot overwritten"
        if move == "load":
            loaded += 1
        elif move == "multiply":
            freed[consumed % stages] += 1
            consumed += 1
        else:
            arrived[i] += 1
            at[move] += teams
    return "done"


@pytest.mark.parametrize("M", range(1, 9))
def test_ring_of_the_decode_kernel(M):
    rng = np.random.default_rng(M)
    for stages in range(1, 8):
        for units in (1, 2, 5, 9, 16, 33):
            assert _digit_ring(M, stages, units, rng) == "done"


def test_what_a_predecessor_wrote_is_read_behind_the_wait_by_ordinary_loads():
    import os
    import re
    from paper_2511_11248_b200 import build
    kernels = {}
    for name in ("f4_rows.cu", "f4_stream.cuh", "f4_pair.cuh"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, name)).read())
        assert not re.search(r"__ldg\(|ld\.global\.nc|__ldlu\(|const [^,()]*__restrict__", text), name
        for m in re.finditer(r"__global__ void[^;{]*?(\w+_kernel)\s*\([^)]*\)\s*\{(?P<body>.*?)\n\}", text, re.S):
            kernels[m[1]] = m["body"]
    early = {k for k, body in kernels.items() if "grid_wait();" in body}
    assert early == {"f4_quantize_kernel", "f4_quantize16_kernel", "f4_row_scales_kernel", "f4_dequant_kernel", "f4_stream_kernel", "f4_pair_kernel"}
    for k in early:
        body = kernels[k]
        before = body[:body.index("grid_wait();")]
        assert "grid_launch_next" not in before, k
        # in front of the wait only weights are loaded and only shared memory written
        assert not re.search(r"load_a\(|p\.x\b|ld_dependent|atomicCAS\(p\.status", before), k


def test_marks_of_quantized_buffers_tell_streams_devices_and_threads_apart(tmp_path):
    import subprocess
    from paper_2511_11248_b200 import build
    (tmp_path / "m.cpp").write_text("""
#include "f4_marks.h"
#include <thread>
using M = tman::F4Marks;
int main()
{
    M m;
    int a = 0, b = 0;
    m.note(0, 0, &a); m.note(1, 0, &b);                       // the default stream of two devices
    if (m.take(0, 0, &a) != M::kHere || m.take(0, 0, &a) != M::kNone) return 1;
    if (m.take(0, 0, &b) != M::kNone || m.take(1, 0, &b) != M::kHere) return 2;
    m.note(0, 1, &a);                                          // the default stream by its other name
    if (m.take(0, 0, &a) != M::kHere) return 3;
    m.note(0, 2, &a);                                          // the per-thread stream of two threads
    std::thread([&] { m.note(0, 2, &b); }).join();
    if (m.take(0, 2, &a) != M::kHere || m.take(0, 2, &b) != M::kElsewhere) return 4;
    m.note(0, 64, &a); m.note(0, 64, &b);                      // the last one of a stream
    if (m.take(0, 64, &a) != M::kNone || m.take(0, 128, &b) != M::kElsewhere || m.take(0, 64, &b) != M::kHere) return 5;
    return 0;
}
""")
    exe = tmp_path / "m"
    subprocess.run(["g++", "-std=c++17", "-pthread", "-I", build.CSRC, str(tmp_path / "m.cpp"), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0
