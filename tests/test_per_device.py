"""csrc/per_device.h on the host: every device's value is made once, its own, whatever the number of threads."""
import os
import subprocess

from paper_2608_26140_b200 import build as abuild

PROGRAM = r"""
#include <atomic>
#include <cstdio>
#include <thread>
#include <vector>
#include "per_device.h"

int main() {
    static acache::PerDevice<std::array<int, 2>, 4> table;
    std::atomic<int> made[6] = {};
    std::atomic<int> wrong{0};
    std::vector<std::thread> threads;
    for (int t = 0; t < 16; ++t)
        threads.emplace_back([&, t] {
            for (int i = 0; i < 1000; ++i) {
                const int device = (t + i) % 4;
                const auto v = table.of(device, [&](std::array<int, 2>& x) {
                    ++made[device];
                    x[0] = 10 * device;
                    std::this_thread::yield();
                    x[1] = x[0] + 1;
                });
                if (v[0] != 10 * device || v[1] != 10 * device + 1) ++wrong;
            }
        });
    for (auto& t : threads) t.join();
    for (int i = 0; i < 2; ++i) table.of(5, [&](std::array<int, 2>&) { ++made[5]; });
    std::printf("%d %d %d %d %d %d\n", wrong.load(), made[0].load(), made[1].load(), made[2].load(), made[3].load(), made[5].load());
}
"""


def test_one_value_for_each_device(tmp_path):
    src, exe = tmp_path / "p.cpp", tmp_path / "p"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-pthread", "-I", abuild.CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    assert out == ["0", "1", "1", "1", "1", "2"]


def test_the_8_bit_attention_keeps_no_table_for_the_whole_process():
    """Its kernels' attributes and cluster counts are the current device's."""
    for name in ("kv8_attn.cu", "kv8_attn_tc.cu"):
        with open(os.path.join(abuild.CSRC, name)) as f:
            text = f.read()
        assert "static int" not in text and "static bool" not in text, name
        assert text.count("cudaFuncSetAttribute") == 1 and text.index("PerDevice<") < text.index("cudaFuncSetAttribute"), name
