"""What the host keeps of a kernel between launches (csrc/launch_words.h), compiled for the CPU with stand-ins for the calls
that ask the device."""
import subprocess

from paper_2010_08899_b200.build import CSRC

PROGRAM = r"""
#include <chrono>
#include <cstdio>
#include <thread>
#include "launch_words.h"
using namespace dct;
using namespace std::chrono;

// a limit that two threads raise, the smaller one in the middle of its call when the larger one comes
static int racing_limit() {
    static SharedLimit limit;
    std::atomic<int> attribute{0}, smaller_is_in{0}, larger_is_set{0};
    std::thread smaller([&] {
        limit.raise(0, 100, [&](uint32_t bytes) {
            smaller_is_in = 1;
            const auto until = steady_clock::now() + milliseconds(300);
            while (!larger_is_set && steady_clock::now() < until) std::this_thread::yield();
            attribute = static_cast<int>(bytes);
            return 0;
        });
    });
    std::thread larger([&] {
        while (!smaller_is_in) std::this_thread::yield();
        limit.raise(0, 200, [&](uint32_t bytes) {
            attribute = static_cast<int>(bytes);
            larger_is_set = 1;
            return 0;
        });
    });
    smaller.join();
    larger.join();
    return attribute;
}

int main() {
    std::printf("%d\n", racing_limit());
    static SharedLimit limit;
    int calls = 0;
    auto set = [&](uint32_t) { ++calls; return 0; };
    auto refuse = [&](uint32_t) { ++calls; return 1; };
    limit.raise(3, 50, set);
    limit.raise(3, 40, set);                   // allowed already
    limit.raise(4, 40, set);                   // another device
    const int twice = calls, refused = limit.raise(3, 60, refuse);
    limit.raise(3, 60, set);                   // a refusal is not kept
    std::printf("%d %d %d\n", twice, refused, calls);
    static ClusterCounts counts;
    int asked = 0;
    auto say = [&](uint32_t n) { return [&asked, n] { ++asked; return n; }; };
    for (uint32_t turn = 0; turn < 2; ++turn)
        for (int dev = 0; dev < 2; ++dev)
            for (uint32_t cluster = 2; cluster <= 8; cluster *= 2) std::printf("%u ", counts.get(dev, cluster, say(100 * dev + cluster)));
    std::printf("%d\n", asked);
}
"""


def test_limits_only_grow_and_counts_are_kept_per_device_and_size(tmp_path):
    src, exe = tmp_path / "words.cpp", tmp_path / "words"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-pthread", "-I", CSRC, str(src), "-o", str(exe)])
    race, limits, counts = subprocess.run([str(exe)], capture_output=True, text=True, check=True, timeout=60).stdout.splitlines()
    assert race == "200"
    assert limits == "2 1 4"
    assert counts.split() == ["2", "4", "8", "102", "104", "108"] * 2 + ["6"]
