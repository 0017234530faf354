// What has to be done once on each device of a process, as letting a kernel have large LDS there.
#pragma once

#include <atomic>
#include <cstdint>

namespace alt {

class OncePerDevice {
    std::atomic<uint64_t> done_{0};        // a bit for each of the first 64 devices; on others it is done every time

public:
    // f() and what it returned, 0 for success, where no call for this device has succeeded yet; 0 where one has.  (Threads that come at once all call it.)
    template <typename F>
    auto operator()(int device, F f) -> decltype(f())
    {
        const uint64_t bit = device >= 0 && device < 64 ? (uint64_t)1 << device : 0;
        if (done_.load(std::memory_order_acquire) & bit) return (decltype(f()))0;
        const auto e = f();
        if (e == (decltype(f()))0) done_.fetch_or(bit, std::memory_order_release);
        return e;
    }
};

}  // namespace alt
