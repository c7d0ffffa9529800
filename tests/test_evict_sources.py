"""Eviction's second kernel looks up no place that the sequence does not have, whatever it finds in `kept`.  The rule is the kernel's own, compiled for
the host; no GPU is needed."""
import os
import subprocess

from paper_2407_13885_b200 import build

PROGRAM = r"""
#include "cache_evict.cuh"
#include <climits>
#include <cstdio>

int main() {
    const int kept[] = {INT_MIN, -1, 0, 1, 5, 6, 7, 99, 100, 101, 1 << 28, INT_MAX}, lengths[] = {0, 1, 6, 100, 1 << 28};
    for (int k : kept)
        for (int n : lengths)
            for (int t : {0, 1, 5, 99}) {
                const int s = attnw::evict::source_of(k, t, n);
                if (s != -1 && (s < t || s >= n)) return std::printf("kept %d, key %d of %d: %d\n", k, t, n, s), 1;
                if (k >= t && k < n && s != k) return std::printf("kept %d, key %d of %d is left out\n", k, t, n), 1;
            }
}
"""


def test_places_outside_the_sequence_are_not_looked_up(tmp_path):
    source, program = tmp_path / "sources.cu", tmp_path / "sources"
    source.write_text(PROGRAM)
    csrc = os.path.dirname(build.SOURCES[0])
    subprocess.run([build.nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I" + csrc, "-o", str(program), str(source)], check=True)
    done = subprocess.run([str(program)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
