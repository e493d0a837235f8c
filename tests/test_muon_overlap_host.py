"""Which matrices of a call the orthogonalisation takes for overlapping: the
host's check against all bytes of small spans (CPU only)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MAIN = r"""
#include "ckpt_muon.cpp"
#include <cstdio>
#include <random>
int main()
{
    std::mt19937 rng(1);
    const auto below = [&](uint32_t n) { return (uint32_t)(rng() % n); };
    int refused = 0, wrong = 0;
    for (int round = 0; round < 400000; ++round) {
        const uint32_t n = 2 + below(3), e = below(2) ? 2 : 4, ld = 1 + below(9); // most matrices share a pitch, as slices do
        std::vector<Span> spans;
        std::vector<int> use(400, 0); // 1: read, 2: written
        bool meets = false;
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t rows = 1 + below(6), l = below(4) ? ld : 1 + below(9), cols = 1 + below(l), at = below(40) * e;
            const bool written = below(2);
            spans.emplace_back((const void*)(uintptr_t)at, rows, cols, l, e, written);
            for (uint32_t r = 0; r < rows; ++r)
                for (uint32_t b = 0; b < cols * e; ++b) {
                    int& u = use[at + r * l * e + b];
                    meets |= u == 2 || (u == 1 && written);
                    u = std::max(u, written ? 2 : 1);
                }
        }
        refused += meets;
        wrong += overlap(spans) != meets;
    }
    std::printf("%d %d\n", refused, wrong);
}
"""


def test_overlaps_are_those_of_the_matrices_own_bytes(tmp_path):
    src, exe = tmp_path / "m.cpp", tmp_path / "m"
    src.write_text(MAIN)
    csrc = os.path.join(ROOT, "paper_2607_01646_amd", "csrc")
    # (the operators' other functions are not called)
    subprocess.run(["g++", "-O2", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", csrc, str(src), "-o",
                    str(exe), "-Wl,--unresolved-symbols=ignore-all"], check=True)
    refused, wrong = map(int, subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split())
    assert 100000 < refused < 350000 and wrong == 0
