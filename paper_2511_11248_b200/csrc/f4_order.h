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

    // A quantization of `packed` is about to be launched on s.  False: a CUDA call failed.
    bool note(cudaStream_t s, const void *packed)
    {
        noted_.store(true, std::memory_order_release);
        int dev = 0;
        bool capturing = false;
        if (!state(s, dev, capturing)) return false;
        if (!capturing) marks_.note(dev, reinterpret_cast<uintptr_t>(s), packed);
        return true;
    }
    // Whether a product of `packed` on s has to wait for all of what is ahead; asked once a launch.
    bool pending(cudaStream_t s, const void *packed, Writes writes)
    {
        if (!noted_.load(std::memory_order_acquire)) return false;      // nothing quantized in this process: no lock
        int dev = 0;
        bool capturing = false;
        if (!state(s, dev, capturing)) return true;
        if (capturing) return captured_behind(s, packed, writes);
        // (Another stream's quantization is ordered before the product by an event, a replayed one by the end of its graph: full dependencies.)
        return marks_.take(dev, reinterpret_cast<uintptr_t>(s), packed) == F4Marks::kHere;
    }

private:
    static bool ok(cudaError_t e)
    {
        if (e != cudaSuccess) (void)cudaGetLastError();
        return e == cudaSuccess;
    }
    static bool state(cudaStream_t s, int &dev, bool &capturing)
    {
        cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
        if (!ok(cudaGetDevice(&dev)) || !ok(cudaStreamIsCapturing(s, &st))) return false;
        capturing = st != cudaStreamCaptureStatusNone;
        return true;
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
    std::atomic<bool> noted_{false};
};

}  // namespace tman
