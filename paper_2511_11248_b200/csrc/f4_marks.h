// Which packed buffer the last eager quantization of each stream wrote.  A stream is a handle on a device: the default stream's handle is the same on every
// device, and the per-thread one's in every thread.
#pragma once

#include <cstdint>
#include <mutex>
#include <thread>
#include <vector>

namespace tman {

class F4Marks {
public:
    // handle: the cudaStream_t's bits; 1 is the legacy default stream by name, 2 the calling thread's
    void note(int device, uintptr_t handle, const void *packed)
    {
        const Key k = key(device, handle);
        std::lock_guard<std::mutex> lock(mutex_);
        for (Mark &m : marks_)
            if (m.key == k) { m.packed = packed; return; }
        marks_.push_back({k, packed});
    }
    enum Found { kNone, kElsewhere, kHere };      // kHere: on this stream, and forgotten now
    Found take(int device, uintptr_t handle, const void *packed)
    {
        const Key k = key(device, handle);
        Found found = kNone;
        std::lock_guard<std::mutex> lock(mutex_);
        for (Mark &m : marks_) {
            if (m.packed != packed) continue;
            if (m.key == k) { m.packed = nullptr; return kHere; }
            if (m.key.device == device) found = kElsewhere;
        }
        return found;
    }

private:
    struct Key {
        int device;
        uintptr_t handle;
        std::thread::id thread;                   // of the per-thread stream only
        bool operator==(const Key &o) const { return device == o.device && handle == o.handle && thread == o.thread; }
    };
    static Key key(int device, uintptr_t handle)
    {
        if (handle == 1) handle = 0;
        return {device, handle, handle == 2 ? std::this_thread::get_id() : std::thread::id()};
    }
    struct Mark { Key key; const void *packed; };
    std::mutex mutex_;
    std::vector<Mark> marks_;
};

}  // namespace tman
