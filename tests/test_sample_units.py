"""The 32-bit counters of sampling's histograms of weights (no GPU): no sum that they can have to hold leaves them."""
import subprocess

from paper_2603_17942_b200 import build as esp_build

PROGRAM = r"""
#include <stdio.h>
#include "esp_paged.h"
int main() {
    using namespace esp;
    for (int slices = 1; slices <= SAMPLE_MAX_SLICES; ++slices)
        for (int blocks = 1; blocks <= 8; blocks *= 2) {
            const unsigned elements = (unsigned)((slices + 2 * blocks - 1) / (2 * blocks) * 2 * SAMPLE_SLICE), unit = sample_unit(elements);     // of a block of a cluster
            const unsigned long long most = (unsigned long long)elements * unit;
            if (unit < 1 || unit > SAMPLE_UNIT || most > 0xffffffffull || (unit < SAMPLE_UNIT && most + elements <= 0xffffffffull)) {
                printf("%d slices, %d blocks: unit %u\n", slices, blocks, unit);
                return 1;
            }
        }
    return 0;
}
"""


def test_no_bin_overflows(tmp_path):
    src, exe = str(tmp_path / "units.cu"), str(tmp_path / "units")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([esp_build.NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", esp_build.CSRC, "-o", exe, src], check=True, capture_output=True, text=True)
    done = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert done.returncode == 0, done.stdout
