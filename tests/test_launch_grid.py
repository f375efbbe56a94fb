"""Launch sizes (host code alone, compiled by g++): no launch of 2^32 threads or more, whatever the number of jobs."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_13716_amd", "csrc")

PROGRAM = r"""
#include "grid.h"
#include <cstdio>
#include <initializer_list>
int main() {
    const long long jobs[] = {1, 2, 255, 4194303, 4194304, 4194305, 16777216, 16777217, 1LL << 32, 1LL << 40};
    for (int threads : {64, 128, 256, 512, 1024})
        for (long long j : jobs) {
            const unsigned long long g = capgnn::stride_grid(j, threads);
            const bool whole = (unsigned long long)j * threads <= 1ull << 30;
            if (g < 1 || g > (unsigned long long)j || g * threads >= 1ull << 32 || (whole && g != (unsigned long long)j)) {
                std::printf("%lld jobs, %d threads: %llu workgroups\n", j, threads, g);
                return 1;
            }
        }
    return 0;
}
"""


def test_no_launch_passes_32_bits_of_threads(tmp_path):
    src, exe = tmp_path / "grid.cpp", tmp_path / "grid"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    done = subprocess.run([str(exe)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout


def test_workgroups_that_stride_take_their_number_from_there():
    """launches over rows times chunks: the only limit in the sources is the one tested above"""
    text = open(os.path.join(CSRC, "answers.hip")).read()
    assert "1 << 24" not in text and text.count("stride_grid(") == 2
