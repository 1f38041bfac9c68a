// What the host keeps of a kernel between launches, per device.  Plain C++.
#pragma once
#include <atomic>
#include <cstdint>

namespace dct {

constexpr int kMaxDevices = 64;

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
