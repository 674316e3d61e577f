"""Order of kernels on a stream, checked on the sources, since no run shows a kernel that happened to start late enough.  A kernel that is launched with
programmatic stream serialization may start while the one ahead of it runs: it has to wait before it touches what that one reads or writes, and it may
let its own successor start only behind that wait, because the successor's wait covers the kernel directly ahead and no other."""
import os
import re

import pytest

from paper_2511_11248_b200 import build

ATTRIBUTE = "cudaLaunchAttributeProgrammaticStreamSerialization"
WAIT = re.compile(r'\bgrid_wait\(\)|griddepcontrol\.wait;')
SIGNAL = re.compile(r'\bgrid_launch_next\(\)|griddepcontrol\.launch_dependents;')
# kernels that are launched in plain stream order only
PLAIN = {"f4_relayout_kernel", "ws_fill_kernel", "wait_timeout_kernel", "quantize_rows_kernel", "pack_kernel", "unpack_kernel", "debug_indices_kernel",
         "dequant_ternary_int8_kernel", "debug_luts_kernel"}
# these let the next kernel start at once (include/tman.h, stream order of the packed buffer)
SIGNAL_FIRST = {"mpgemv_kernel", "decode_digits_kernel", "decode_mma_kernel"}


def sources():
    for name in sorted(os.listdir(build.CSRC)):
        if name.endswith((".cu", ".cuh")) and name != "microbench.cu":
            with open(os.path.join(build.CSRC, name)) as f:
                yield name, re.sub(r"//[^\n]*", "", f.read())


def kernels():
    """(file, kernel, body) of every kernel."""
    found = []
    for name, text in sources():
        for m in re.finditer(r"__global__ void\s+(?:__launch_bounds__\((?:[^()]|\([^()]*\))*\)\s*)?(\w+)\s*\([^{;]*?\)\s*\{(.*?)\n\}", text, re.S):
            found.append((name, m[1], m[2]))
    return found


EARLY = [k for k in kernels() if k[1] not in PLAIN]
ids = lambda v: v if isinstance(v, str) and v.endswith("_kernel") else ""


def test_every_kernel_is_found_and_plain_launches_are_plain():
    assert len(kernels()) == sum(len(re.findall(r"__global__ void", text)) for _, text in sources())
    assert PLAIN <= {k[1] for k in kernels()} and SIGNAL_FIRST <= {k[1] for k in kernels()}
    for name, text in sources():
        if ATTRIBUTE not in text:
            assert not [k for k in kernels() if k[0] == name and k[1] not in PLAIN] or name.endswith(".cuh"), name


@pytest.mark.parametrize("name,kernel,body", EARLY, ids=ids)
def test_a_kernel_that_may_start_early_waits_and_lets_the_next_one_start_behind_that(name, kernel, body):
    waits, signals = [m.start() for m in WAIT.finditer(body)], [m.start() for m in SIGNAL.finditer(body)]
    assert waits, f"{kernel} ({name}) is launched with {ATTRIBUTE} and never waits"
    assert not signals or min(waits) < min(signals) or kernel in SIGNAL_FIRST, kernel


@pytest.mark.parametrize("name,kernel,body", [k for k in EARLY if re.match(r"(i8_|norm_|append_|read_cache_|attend_)", k[1])], ids=ids)
def test_activations_are_read_behind_the_wait(name, kernel, body):
    """Of the 8-bit operators, which have no rule about what the kernels ahead write: nothing is loaded ahead of the wait (prefetches into L2 apart)."""
    assert not re.search(r"ld\.global|ld_dependent\(|load_runs\(|__ldg\(|atomic", body[:WAIT.search(body).start()]), kernel


def test_scales_that_a_warp_passes_on_through_shared_memory_are_behind_a_barrier():
    """i8_pair_kernel: a lane writes tokens' scales that the others of its warp read; a vote orders no memory."""
    body = next(k[2] for k in kernels() if k[1] == "i8_pair_kernel")
    writes = [m.start() for m in re.finditer(r"token_scale\[warp - 2\]\[i\] = ", body)]
    assert len(writes) == 2
    for at in writes:
        after = body[at:]
        barrier = re.search(r"__syncwarp\(\);|__syncthreads\(\);", after)
        wait = after.index("mbar_wait(")                   # what stands between a write and the reads of the same tile
        assert barrier and (barrier.start() < wait or not re.search(r"store16\(|token_scale", after[wait:barrier.start()])), after[:200]
