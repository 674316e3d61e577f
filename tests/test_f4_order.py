"""When a product of 4-bit floating-point weights may fetch them early: the host's bookkeeping (csrc/f4_order.h, csrc/f4_marks.h) against a stand-in
for the CUDA runtime.  What it has to prevent, a product that reads half-written weights, is not run anywhere."""
import subprocess

import pytest

RUNTIME = """
#pragma once
#include <cstddef>
typedef struct Stream *cudaStream_t; typedef struct Node *cudaGraphNode_t; typedef struct Graph *cudaGraph_t;
typedef enum { cudaSuccess = 0, cudaErrorInvalidDeviceFunction = 98, cudaErrorOther = 999 } cudaError_t;
typedef enum { cudaStreamCaptureStatusNone = 0, cudaStreamCaptureStatusActive = 1 } cudaStreamCaptureStatus;
typedef enum { cudaGraphNodeTypeKernel = 0, cudaGraphNodeTypeMemset = 2, cudaGraphNodeTypeEmpty = 5 } cudaGraphNodeType;
struct cudaGraphEdgeData { unsigned char from_port, to_port, type; };
struct cudaKernelNodeParams { void *func; void **kernelParams; };
struct Node { cudaGraphNodeType type; cudaError_t error; const void *func; void *params[5]; };
extern int g_device; extern bool g_capturing; extern cudaError_t g_error; extern cudaGraphNode_t g_ahead[4]; extern size_t g_n;
inline cudaError_t cudaGetLastError() { return cudaSuccess; }
inline cudaError_t cudaGetDevice(int *d) { *d = g_device; return g_error; }
inline cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus *s) { *s = g_capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone; return g_error; }
inline cudaError_t cudaStreamGetCaptureInfo_v3(cudaStream_t, cudaStreamCaptureStatus *s, unsigned long long *, cudaGraph_t *, const cudaGraphNode_t **n,
                                               const cudaGraphEdgeData **, size_t *count)
{ *s = cudaStreamCaptureStatusActive; *n = g_ahead; *count = g_n; return cudaSuccess; }
inline cudaError_t cudaGraphNodeGetType(cudaGraphNode_t n, cudaGraphNodeType *t) { *t = n->type; return cudaSuccess; }
inline cudaError_t cudaGraphKernelNodeGetParams(cudaGraphNode_t n, cudaKernelNodeParams *p) { p->func = (void *)n->func; p->kernelParams = n->params; return n->error; }
"""

PRELUDE = """
#include "f4_order.h"
#include <initializer_list>
#include <thread>
#include <type_traits>
#define REQUIRE(c) do { if (!(c)) return __LINE__; } while (0)
int g_device = 0; bool g_capturing = false; cudaError_t g_error = cudaSuccess; cudaGraphNode_t g_ahead[4]; size_t g_n = 0;
using namespace tman;
static int quantizer, w, a, v;
static bool writes(const cudaKernelNodeParams &n, const void *packed) { return n.func == &quantizer && *(void **)n.kernelParams[4] == packed; }
static cudaStream_t stream(size_t h) { return (cudaStream_t)h; }
struct Order : F4Order {                                     // calls whose launches succeed, by one thread
    bool note(cudaStream_t s, const void *packed) { Call c; if (!begin(s, packed, c)) return false; end(c, true); return true; }
    bool pending(cudaStream_t s, const void *packed, Writes writes) { const Call c = ahead(s, packed, writes); behind(c, true); return c.pending; }
};
"""


@pytest.fixture
def run(tmp_path):
    from paper_2511_11248_b200 import build

    def go(body):
        (tmp_path / "cuda_runtime.h").write_text(RUNTIME)
        (tmp_path / "t.cpp").write_text(PRELUDE + "int main()\n{\n" + body + "\nreturn 0;\n}\n")
        exe = tmp_path / "t"
        subprocess.run(["g++", "-std=c++17", "-pthread", "-I", str(tmp_path), "-I", build.CSRC, str(tmp_path / "t.cpp"), "-o", str(exe)], check=True)
        line = subprocess.run([str(exe)], timeout=60).returncode
        assert line == 0, (PRELUDE + "int main()\n{\n" + body).splitlines()[line - 1]
    return go


def test_a_captured_product_leaves_the_mark_of_an_eager_quantization(run):
    run("""
Order o;
REQUIRE(!o.pending(stream(64), &w, writes));
REQUIRE(o.note(stream(64), &w));                         // eager quantization of w
g_capturing = true;
REQUIRE(!o.pending(stream(64), &w, writes));             // captured: nothing ahead of it in its graph
g_capturing = false;
REQUIRE(o.pending(stream(64), &w, writes));              // eager, behind the quantization still
REQUIRE(!o.pending(stream(64), &w, writes));""")


def test_a_captured_quantization_does_not_replace_the_mark_of_an_eager_one(run):
    run("""
Order o;
REQUIRE(o.note(stream(64), &w));
g_capturing = true;
REQUIRE(o.note(stream(64), &a));
g_capturing = false;
REQUIRE(!o.pending(stream(64), &a, writes) && o.pending(stream(64), &w, writes));""")


def test_a_captured_product_asks_the_nodes_ahead_of_it(run):
    run("""
Order o;
void *pw = &w, *pa = &a;
Node qw = {cudaGraphNodeTypeKernel, cudaSuccess, &quantizer, {0, 0, 0, 0, &pw}}, qa = {cudaGraphNodeTypeKernel, cudaSuccess, &quantizer, {0, 0, 0, 0, &pa}},
     other = {cudaGraphNodeTypeKernel, cudaSuccess, &v, {0, 0, 0, 0, &pw}}, foreign = {cudaGraphNodeTypeKernel, cudaErrorInvalidDeviceFunction, nullptr, {}},
     fill = {cudaGraphNodeTypeMemset, cudaErrorOther, nullptr, {}}, odd = {cudaGraphNodeTypeKernel, cudaErrorOther, nullptr, {}};
g_capturing = true;
REQUIRE(o.note(stream(64), &w));
auto ahead = [&](std::initializer_list<Node *> n) { g_n = 0; for (Node *p : n) g_ahead[g_n++] = p; return o.pending(stream(64), &w, writes); };
REQUIRE(ahead({&qw}) && ahead({&qw}));                   // asked of the graph, not remembered
REQUIRE(!ahead({&qa}) && !ahead({&other}) && !ahead({&foreign}) && !ahead({&fill}) && !ahead({}));
REQUIRE(ahead({&qa, &fill, &qw}));                       // of several streams joined by events
REQUIRE(ahead({&odd}));                                  // not known: plain order""")


def test_a_runtime_that_fails_means_plain_order(run):
    run("""
Order o;
REQUIRE(o.note(stream(64), &a));
g_error = cudaErrorOther;
REQUIRE(!o.note(stream(64), &w) && o.pending(stream(64), &v, writes));""")


def test_quantizations_of_two_threads_on_one_stream(run):
    """Begun in one order and launched in the other: the product of either waits, until a quantization has gone through alone."""
    run("""
Order o;
F4Order::Call cw, ca;
REQUIRE(o.begin(stream(64), &w, cw) && o.begin(stream(64), &a, ca));
REQUIRE(o.pending(stream(64), &w, writes));               // under way
o.end(cw, true); o.end(ca, true);                         // (launched the other way around)
REQUIRE(o.pending(stream(64), &w, writes) && o.pending(stream(64), &a, writes) && o.pending(stream(64), &w, writes));
REQUIRE(!o.pending(stream(128), &w, writes));
REQUIRE(o.note(stream(64), &a));
REQUIRE(!o.pending(stream(64), &w, writes) && o.pending(stream(64), &a, writes) && !o.pending(stream(64), &a, writes));""")


def test_a_mark_is_taken_when_its_product_has_been_launched(run):
    """Two threads' products of the same weights behind one quantization: whichever is launched first waits for it."""
    run("""
Order o;
REQUIRE(o.note(stream(64), &w));
const F4Order::Call one = o.ahead(stream(64), &w, writes), two = o.ahead(stream(64), &w, writes);
REQUIRE(one.pending && two.pending);
o.behind(two, false);                                     // its launch failed
REQUIRE(o.ahead(stream(64), &w, writes).pending);
o.behind(one, true);
REQUIRE(!o.ahead(stream(64), &w, writes).pending);""")


def test_a_quantization_whose_launch_failed_hides_no_other(run):
    run("""
Order o;
F4Order::Call c;
REQUIRE(o.note(stream(64), &w));
REQUIRE(o.begin(stream(64), &a, c));
o.end(c, false);
REQUIRE(o.pending(stream(64), &w, writes));""")


def test_more_streams_than_the_table_holds(run):
    """Nothing is allocated, and a stream that had to make room is one whose products wait: once, then they know that nothing is under way."""
    run("""
static_assert(std::is_trivially_destructible<F4Marks>::value, "no memory of its own");
Order o;
for (size_t s = 1; s <= 64; ++s) REQUIRE(o.note(stream(64 * s), &w));
REQUIRE(!o.pending(stream(64 * 100), &a, writes));        // a stream without quantizations
REQUIRE(o.note(stream(64 * 65), &w));                     // the first one made room
REQUIRE(o.ahead(stream(64), &w, writes).pending && o.pending(stream(64), &a, writes));
REQUIRE(!o.pending(stream(64), &a, writes) && !o.pending(stream(64), &w, writes));
for (size_t s = 66; s <= 400; ++s) REQUIRE(o.note(stream(64 * s), &w) && o.ahead(stream(64 * s), &w, writes).pending);
for (size_t s = 1; s <= 400; ++s) REQUIRE(o.pending(stream(64 * s), &w, writes) && !o.pending(stream(64 * s), &w, writes));""")


def test_more_threads_in_a_quantization_than_the_table_holds(run):
    run("""
Order o;
F4Order::Call c[80];
for (size_t s = 0; s < 80; ++s) REQUIRE(o.begin(stream(64 * (s + 1)), &w, c[s]));
for (size_t s = 0; s < 80; ++s) REQUIRE(o.ahead(stream(64 * (s + 1)), &w, writes).pending);
for (size_t s = 0; s < 80; ++s) { o.end(c[s], true); REQUIRE(o.ahead(stream(64 * (s + 1)), &w, writes).pending); }
for (size_t s = 0; s < 80; ++s) REQUIRE(o.ahead(stream(64 * (s + 1)), &w, writes).pending);
for (size_t s = 0; s < 80; ++s) REQUIRE(o.note(stream(64 * (s + 1)), &a) && !o.ahead(stream(64 * (s + 1)), &w, writes).pending);""")


@pytest.mark.parametrize("name,alloc", [("f4_stream.cuh", "tcgen05_alloc("), ("f4_pair.cuh", "tcgen05_alloc2(")])
def test_tensor_memory_is_taken_behind_the_wait_and_ahead_of_the_signal(name, alloc):
    """A kernel ahead may signal before it takes its own tensor memory: with this kernel's taken ahead of the wait, each would wait for the other.
    Read from the source, since a run that shows it would hang."""
    import os
    import re
    from paper_2511_11248_b200 import build
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, name)).read())
    body = re.search(r"__global__ void[^;{]*?_kernel\s*\([^)]*\)\s*\{(.*?)\n\}", text, re.S)[1]
    assert body.count(alloc) == 1 and body.count("grid_launch_next();") == 1
    at = body.index(alloc)
    # the last thing that this warp does before it is the wait: in its own branch, or in front of all branches
    before = body[:at]
    wait, branch = before.rindex("grid_wait();"), max(before.rfind("} else if (warp == 1) {"), before.rfind("    if (warp == 1) {"))
    assert wait > branch or "if (" not in before[wait:branch].replace("if (warp == 1) {", "")
    assert at < body.index("grid_launch_next();")
