"""Eviction as far as it goes without a GPU: how many blocks a list has."""
import subprocess

from paper_2603_17942_b200 import build as esp_build

PROGRAM = r"""
#include <stdio.h>
#include "esp_paged.h"
int main() {
    using namespace esp;
    for (int kv_cap : {1, 16, 2049, 5001, 8192, 8193, 16384, 32768, 65536, 131072, 1 << 30})
        for (int max_kv : {1, 16, 2049, 5000, 8192, 8193, 32768, 32769, 65536, 1 << 30})
            for (int lists : {1, 26, 37, 38, 74, 75, 148, 149, 256, 1000, 1 << 27}) {
                int32_t as_needed = -1;
                const int n = evict_blocks(kv_cap, (max_kv + 1) / 2, lists, 148, &as_needed);
                const auto holds = [](long long keys) { return keys <= 8192 ? 1 : (keys <= 16384 ? 2 : (keys <= 32768 ? 4 : 8)); };
                const int most = holds(kv_cap);
                const bool full = (long long)lists * most > 296;
                const long long even = (max_kv + 1) / 2 * 2ll;
                if (as_needed != full || n != (full ? holds(even < kv_cap ? even : kv_cap) : most)) {
                    printf("table for %d, scratch for %d, %d lists: %d blocks, as needed %d\n", kv_cap, max_kv, lists, n, as_needed);
                    return 1;
                }
            }
    // a step at its budget: 256 lists of 2049 keys in tables for 64k positions
    int32_t as_needed = 0;
    return evict_blocks(65536, 1025, 256, 148, &as_needed) != 1 || !as_needed;
}
"""


def test_blocks_of_a_list(tmp_path):
    """Where the GPU is full, by the longest list that the scratch is made for, not by how many positions a row of the table has room for."""
    src, exe = str(tmp_path / "blocks.cu"), str(tmp_path / "blocks")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([esp_build.NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", esp_build.CSRC, "-o", exe, src], check=True, capture_output=True, text=True)
    done = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert done.returncode == 0, done.stdout
