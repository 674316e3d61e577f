// Whether a product may fetch its weights before the kernel ahead of it has ended, host side.
//
// A quantization lets its successor start when it has itself begun.  A product behind it that reads what it writes as weights is launched in plain
// stream order.  What lies ahead of a product is, of an eager call, what its stream ran last (marks); of a captured call, the nodes that the
// captured launch will depend on, which the graph says by itself.  A capture runs nothing: captured calls neither leave nor take marks.
#pragma once

#include "f4_marks.h"

#include <atomic>

#include <cuda_runtime.h>

namespace tman {

class F4Order {
public:
    // Whether the kernel of a graph node is a quantization that writes `packed`.
    using Writes = bool (*)(const cudaKernelNodeParams &node, const void *packed);

    struct Call {
        const void *packed;
        int device;
        uintptr_t handle;
        bool captured, pending;                  // pending (of a product): it has to wait for all of what is ahead
    };

    // A quantization of `packed` on s: begin, the launch, end.  False: a CUDA call failed, nothing to launch or to end.
    bool begin(cudaStream_t s, const void *packed, Call &c)
    {
        noted_.store(true, std::memory_order_release);
        if (!place(s, packed, c) || !state(s, c)) return false;
        if (c.captured) captured_.store(true, std::memory_order_release);
        else marks_.begin(c.device, c.handle);
        return true;
    }
    void end(const Call &c, bool launched)
    {
        if (c.captured) return;
        if (launched) marks_.note(c.device, c.handle, c.packed);
        else marks_.drop(c.device, c.handle);
    }
    // A product of `packed` on s: ahead, the launch, behind.
    Call ahead(cudaStream_t s, const void *packed, Writes writes)
    {
        Call c = {};
        if (!noted_.load(std::memory_order_acquire)) return c;      // nothing quantized in this process: no lock
        if (!place(s, packed, c)) return unknown(c);
        // (Another stream's quantization is ordered before the product by an event, a replayed one by the end of its graph: full dependencies.)
        c.pending = marks_.find(c.device, c.handle, packed) == F4Marks::kHere;
        if (!c.pending && !captured_.load(std::memory_order_acquire)) return c;      // whether it is captured makes no difference
        if (!state(s, c)) return unknown(c);
        if (c.captured) c.pending = captured_behind(s, packed, writes);
        return c;
    }
    void behind(const Call &c, bool launched)
    {
        if (launched && c.pending && !c.captured) (void)marks_.take(c.device, c.handle, c.packed);
    }

private:
    static bool ok(cudaError_t e)
    {
        if (e != cudaSuccess) (void)cudaGetLastError();
        return e == cudaSuccess;
    }
    static bool place(cudaStream_t s, const void *packed, Call &c)
    {
        c = {packed, 0, reinterpret_cast<uintptr_t>(s), false, false};
        return ok(cudaGetDevice(&c.device));
    }
    static bool state(cudaStream_t s, Call &c)
    {
        cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
        if (!ok(cudaStreamIsCapturing(s, &st))) return false;
        c.captured = st != cudaStreamCaptureStatusNone;
        return true;
    }
    static Call unknown(Call c)                  // plain order, and no mark is taken
    {
        c.captured = c.pending = true;
        return c;
    }
    // Only a kernel can let its successor start early; one that this library does not know by its function is no quantization.
    static bool captured_behind(cudaStream_t s, const void *packed, Writes writes)
    {
        cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
        const cudaGraphNode_t *nodes = nullptr;
        const cudaGraphEdgeData *edges = nullptr;
        size_t n = 0;
        if (!ok(cudaStreamGetCaptureInfo_v3(s, &st, nullptr, nullptr, &nodes, &edges, &n))) return true;
        for (size_t i = 0; i < n; ++i) {
            cudaGraphNodeType type = cudaGraphNodeTypeEmpty;
            if (!ok(cudaGraphNodeGetType(nodes[i], &type))) return true;
            if (type != cudaGraphNodeTypeKernel) continue;
            cudaKernelNodeParams node = {};
            const cudaError_t e = cudaGraphKernelNodeGetParams(nodes[i], &node);
            if (e != cudaSuccess) (void)cudaGetLastError();
            if (e == cudaErrorInvalidDeviceFunction) continue;
            if (e != cudaSuccess || writes(node, packed)) return true;
        }
        return false;
    }

    F4Marks marks_;
    std::atomic<bool> noted_{false}, captured_{false};      // quantizations there were, captured ones
};

}  // namespace tman
