// Which packed buffer the last eager quantization of each stream wrote.  A stream is a handle on a device: the default stream's handle is the same on every
// device, and the per-thread one's in every thread.  The table has a fixed size and allocates nothing: the stream that was not used for longest makes
// room for a new one, and from then on a stream that is not there counts as one whose last quantization is not known.
#pragma once

#include <cstdint>
#include <mutex>
#include <thread>

namespace tman {

class F4Marks {
public:
    // A quantization: begin, its launch, then note, or drop if the launch failed.  Threads that share a stream may have several of them between
    // begin and note, and the order of their launches is not that of these calls: then whichever is asked for may be the last one, until one
    // alone has gone through.
    // handle: the cudaStream_t's bits; 1 is the legacy default stream by name, 2 the calling thread's
    void begin(int device, uintptr_t handle)
    {
        std::lock_guard<std::mutex> lock(mutex_);
        Mark &m = at(key(device, handle));
        m.mixed = m.writing++ > 0;
    }
    void note(int device, uintptr_t handle, const void *packed)
    {
        std::lock_guard<std::mutex> lock(mutex_);
        Mark &m = at(key(device, handle));
        if (m.writing > 0) --m.writing;
        m.packed = packed;
    }
    void drop(int device, uintptr_t handle)
    {
        std::lock_guard<std::mutex> lock(mutex_);
        Mark &m = at(key(device, handle));
        if (m.writing > 0) --m.writing;
        m.mixed = true;                           // (what was launched before may be the last one still)
    }
    // A product: find, its launch, then take.  (A mark taken ahead of the launch would let another thread's product of the same weights go first,
    // early.)
    enum Found { kNone, kElsewhere, kHere };      // kHere: on this stream
    Found find(int device, uintptr_t handle, const void *packed)
    {
        std::lock_guard<std::mutex> lock(mutex_);
        return look(key(device, handle), packed, false);
    }
    Found take(int device, uintptr_t handle, const void *packed)      // and forgotten
    {
        std::lock_guard<std::mutex> lock(mutex_);
        const Key k = key(device, handle);
        const Found found = look(k, packed, true);
        if (lost_ && !slot(k)) at(k).mixed = false;      // (behind a product in plain order nothing is under way)
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
    struct Mark {
        Key key;
        const void *packed;
        int writing;                              // quantizations between begin and note
        bool mixed;                               // some of them were there together, or what was there is not known
        uint64_t used;                            // 0: free
    };
    Mark *slot(const Key &k)
    {
        for (Mark &m : marks_)
            if (m.used && m.key == k) {
                m.used = ++clock_;
                return &m;
            }
        return nullptr;
    }
    Mark &at(const Key &k)
    {
        if (Mark *m = slot(k)) return *m;
        Mark *to = nullptr;
        for (Mark &m : marks_)
            if (m.writing == 0 && (!to || m.used < to->used)) to = &m;
        const bool unknown = lost_;
        if (!to) to = &spare_;                    // (every stream of the table is between begin and note: this one is not kept)
        if (to == &spare_ || to->packed || to->mixed) lost_ = true;
        *to = {k, nullptr, 0, unknown, ++clock_};
        return *to;
    }
    Found look(const Key &k, const void *packed, bool forget)
    {
        if (Mark *m = slot(k)) {
            const bool here = m->packed == packed;
            if (here && forget) m->packed = nullptr;
            if (here || m->writing > 0 || m->mixed) return kHere;
        } else if (lost_)
            return kHere;
        for (const Mark &m : marks_)
            if (m.used && m.packed == packed && m.key.device == k.device) return kElsewhere;
        return kNone;
    }
    static constexpr int kStreams = 64;
    std::mutex mutex_;
    Mark marks_[kStreams] = {}, spare_ = {};
    uint64_t clock_ = 0;
    bool lost_ = false;                           // a stream with a mark has made room
};

}  // namespace tman
