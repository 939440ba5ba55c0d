"""The window that the planners hand to the kernels: the arithmetic of its masks, with
the largest windows and sinks, stays within 32 bits."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# a key tile's distances as the kernels form them: rows and keys of a tile of 128, from 127 below the tile on
CODE = r"""
#include <cstdio>
#include "fnpu_internal.h"
int main() {
    const int32_t sizes[] = {1, 2, 127, 4096, INT32_MAX - 1024, INT32_MAX - 1023, INT32_MAX};
    for (int32_t size : sizes) {
        const fnpu::Window w = fnpu::make_window(size, size);
        bool fits = true;
        for (int64_t hi = -128; hi < 256; ++hi)
            for (int64_t q = 0; q < 128; q += 32) {
                const int64_t lo = hi - w.size - q;
                fits = fits && lo >= INT32_MIN && w.size + int64_t{128} <= INT32_MAX;
            }
        for (int64_t tile : {16, 64, 128}) fits = fits && w.sinks + tile - 1 <= INT32_MAX;
        std::printf("%d %d %d\n", w.size, w.sinks, fits ? 1 : 0);
    }
}
"""


def test_the_largest_windows_leave_room_for_a_tile(tmp_path):
    src, exe = tmp_path / "w.cpp", tmp_path / "w"
    src.write_text(CODE)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2606_04415_gb300", "csrc"), "-I", os.path.join(cuda, "include"),
                    str(src), "-o", str(exe)], check=True)
    rows = [tuple(map(int, line.split())) for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()]
    most = 2 ** 31 - 1 - 1024
    assert rows == [(n, n, 1) for n in (1, 2, 127, 4096, most)] + [(most, most, 1)] * 2
