// What has to be told to the runtime once for each device, not once for a process.
#pragma once

#include <atomic>
#include <stdint.h>

namespace ar {

// set() is called for a device until it has succeeded there once; a failure is
// reported and tried again by the next call.  Several threads may call it for one
// device at the same time, so set() has to bear being repeated.
class OncePerDevice {
    std::atomic<uint64_t> done_{0};  // a bit for each of the first 64 devices; others are set every time

public:
    template <typename F> bool operator()(int device, F set)
    {
        const uint64_t bit = device >= 0 && device < 64 ? 1ull << device : 0;
        if (done_.load(std::memory_order_relaxed) & bit) return true;
        if (!set()) return false;
        done_.fetch_or(bit, std::memory_order_relaxed);
        return true;
    }
};

}  // namespace ar
