// Host memory that a blocking call reads back into (host code; the allocator is a parameter, so that a test can refuse).
#pragma once
#include <atomic>
#include <mutex>
#include <new>

namespace sals {

// A block of BYTES, for one call at a time.  Pinned, as a wait for the device and 8 KB from it take 11 us, into other memory 22; making
// and freeing it takes 25 us and waits for every stream of the process, so up to KEEP blocks, all alike, are kept from call to call.  Where pinned
// memory is refused it is ordinary memory, freed behind the call; p is null if there is neither.  Nothing is thrown.
template <typename ALLOC, size_t BYTES, int KEEP> struct HostBlock {
    void* p = nullptr;
    bool idle = false;   // set behind the last wait: no copy into the block is under way
    // running: the runtime is known to be at work (it is behind the first pinned block, too)
    explicit HostBlock(bool running = false)
    {
        {
            const std::lock_guard<std::mutex> hold(lock());
            for (void*& k : kept())
                if (k) { p = k; k = nullptr; pinned = true; return; }
        }
        // Ordinary memory first: where there is none, a runtime whose first use this may be is not asked, as it throws then or ends the process.
        void* const spare = ::operator new(BYTES, std::nothrow);
        if (!spare && !running && !ran().load()) return;
        try {
            p = ALLOC::pin(BYTES);
        } catch (...) {
            p = nullptr;
        }
        pinned = p != nullptr;
        if (pinned) { ran().store(true); ::operator delete(spare); }
        else p = spare;
    }
    ~HostBlock()
    {
        if (!pinned) { ::operator delete(p); return; }
        if (idle) {
            const std::lock_guard<std::mutex> hold(lock());
            for (void*& k : kept())
                if (!k) { k = p; return; }
        }
        ALLOC::unpin(p);
    }
    HostBlock(const HostBlock&) = delete;
    HostBlock& operator=(const HostBlock&) = delete;

private:
    typedef void* Blocks[KEEP];
    static std::mutex& lock() { static std::mutex m; return m; }
    static Blocks& kept() { static Blocks b = {}; return b; }
    static std::atomic<bool>& ran() { static std::atomic<bool> r{false}; return r; }
    bool pinned = false;
};

}  // namespace sals
