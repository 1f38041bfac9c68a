"""What the host keeps of a kernel between launches (csrc/launch_words.h), compiled for the CPU with stand-ins for the calls
that ask the device."""
import subprocess

from paper_2010_08899_b200.build import CSRC

PROGRAM = r"""
#include <cstdio>
#include "launch_words.h"
using namespace dct;

int main() {
    static ClusterCounts counts;
    int asked = 0;
    auto say = [&](uint32_t n) { return [&asked, n] { ++asked; return n; }; };
    for (uint32_t turn = 0; turn < 2; ++turn)
        for (int dev = 0; dev < 2; ++dev)
            for (uint32_t cluster = 2; cluster <= 8; cluster *= 2) std::printf("%u ", counts.get(dev, cluster, say(100 * dev + cluster)));
    std::printf("%d\n", asked);
}
"""


def test_counts_are_kept_per_device_and_size(tmp_path):
    src, exe = tmp_path / "words.cpp", tmp_path / "words"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-pthread", "-I", CSRC, str(src), "-o", str(exe)])
    counts = subprocess.run([str(exe)], capture_output=True, text=True, check=True, timeout=60).stdout
    assert counts.split() == ["2", "4", "8", "102", "104", "108"] * 2 + ["6"]
