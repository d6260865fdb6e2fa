// What launches ask a device only once: kernel attributes, how many clusters are resident.  An answer belongs to a device and a
// question; contexts on several threads may ask at the same time (they get the same answer).  A question that failed is asked
// again the next time, and leaves no error behind for a later check of the launch.
#pragma once
#include <cuda_runtime.h>

#include <atomic>

namespace glance {

constexpr int kMaxDevices = 64;

inline int current_device() {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return -1;
    }
    return dev;
}

// (objects of static storage: all zeros, nothing asked yet)
template <int QUESTIONS>
struct Answers {
    std::atomic<int> known[kMaxDevices][QUESTIONS];

    // ask(): the answer, above 0, or 0 if the question failed; then `otherwise` is what the caller goes by
    template <class Ask>
    int get(int dev, int question, int otherwise, Ask ask) {
        const bool kept = dev >= 0 && dev < kMaxDevices;
        int n = kept ? known[dev][question].load(std::memory_order_relaxed) : 0;
        if (n > 0) return n;
        n = ask();
        if (n < 1) {
            (void)cudaGetLastError();
            return otherwise;
        }
        if (kept) known[dev][question].store(n, std::memory_order_relaxed);
        return n;
    }
};

}  // namespace glance
