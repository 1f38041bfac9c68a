// What the host keeps of a kernel between launches, per device.  Plain C++: any number of threads may launch at once.
#pragma once
#include <atomic>
#include <cstdint>
#include <mutex>

namespace dct {

constexpr int kMaxDevices = 64;

// The most dynamic shared memory a kernel has been allowed on each device.  It only grows: a thread that asks for less while another
// asks for more must not have the last word.
class SharedLimit {
public:
    // set(bytes) allows that much and returns 0, or an error, which is passed on
    template <typename Set> int raise(int dev, uint32_t bytes, Set&& set) {
        if (allowed_[dev].load(std::memory_order_acquire) >= bytes) return 0;
        std::lock_guard<std::mutex> lock(mu_);
        if (allowed_[dev].load(std::memory_order_relaxed) >= bytes) return 0;
        const int error = set(bytes);
        if (error == 0) allowed_[dev].store(bytes, std::memory_order_release);
        return error;
    }

private:
    std::mutex mu_;
    std::atomic<uint32_t> allowed_[kMaxDevices] = {};
};

// How many clusters of 2, 4 or 8 CTAs each device holds at a time, for launches of one kernel that differ in nothing else that
// matters to it.
class ClusterCounts {
public:
    // count(): as many as the device says, at least 1; asked for once per device and size (by several threads perhaps, with one answer)
    template <typename Count> uint32_t get(int dev, uint32_t cluster, Count&& count) {
        std::atomic<uint32_t>& word = words_[dev][cluster == 2 ? 0 : cluster == 4 ? 1 : 2];
        uint32_t n = word.load(std::memory_order_relaxed);
        if (n == 0) {
            n = count();
            word.store(n, std::memory_order_relaxed);
        }
        return n;
    }

private:
    std::atomic<uint32_t> words_[kMaxDevices][3] = {};
};

}  // namespace dct
