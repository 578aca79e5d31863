// What has to be done once per device of a process (host code).
#pragma once
#include <atomic>
#include <stdint.h>

namespace tsm {

// Runs f() (true: it worked) unless it has worked for this device before.  Host threads may come together: f() may then run in each of
// them, and none goes on before it has worked.  Devices from 64 on are done every time.
class OncePerDevice {
    std::atomic<uint64_t> done_{0};

public:
    template <typename F> bool operator()(int device, F f) {
        const uint64_t bit = device >= 0 && device < 64 ? (uint64_t)1 << device : 0;
        if (done_.load(std::memory_order_acquire) & bit) return true;
        if (!f()) return false;
        done_.fetch_or(bit, std::memory_order_release);
        return true;
    }
};

}  // namespace tsm
