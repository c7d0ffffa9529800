"""The one-pass attention kernel's end after a wait that gave up: of each stage it waits for the last copy, and for no other, whose parity would
be that of a copy that is never asked for.  The rule is the kernel's own, compiled for the host; no GPU is needed."""
import os
import subprocess

from paper_2407_13885_b200 import build

PROGRAM = r"""
#include "attn_onepass.cuh"
#include <cstdio>

using namespace attnw::av1;

template <int STAGES, bool TWO_ISSUERS>
int check(const char* what) {
    for (int kind = 0; kind < (TWO_ISSUERS ? 2 : 1); ++kind)
        for (int loads = 0; loads < 40; ++loads) {
            int last[STAGES], asked[STAGES] = {};
            for (int& l : last) l = -1;
            Tiles<STAGES, TWO_ISSUERS> tile(kind);
            for (int it = 0; it < loads; ++it, tile.next()) last[tile.stage] = it;
            Tiles<STAGES, TWO_ISSUERS> again(kind);
            for (int it = 0; it < loads; ++it, again.next())
                if (again.last_of_stage(it, loads)) {
                    ++asked[again.stage];
                    if (last[again.stage] != it) return std::printf("%s: copy %d of %d is not the last of stage %d\n", what, it, loads, again.stage), 1;
                }
            for (int s = 0; s < STAGES; ++s)
                if (asked[s] != (last[s] >= 0)) return std::printf("%s: stage %d is asked %d times after %d copies\n", what, s, asked[s], loads), 1;
        }
    return 0;
}

template <int D>
int check_all() {
    return check<Smem<D>::kStages, Smem<D>::two_issuers(kWhole)>("two query tiles") || check<Smem<D>::kStages + 1, Smem<D>::two_issuers(kSplit)>("split") ||
           check<Smem<D>::kStages + 1, Smem<D>::two_issuers(kCluster)>("cluster");
}

int main() { return check_all<64>() || check_all<128>(); }
"""


def test_the_last_copy_of_each_stage_is_waited_for(tmp_path):
    source, program = tmp_path / "unwinding.cu", tmp_path / "unwinding"
    source.write_text(PROGRAM)
    csrc = os.path.dirname(build.SOURCES[0])
    subprocess.run([build.nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I" + csrc, "-o", str(program), str(source)], check=True)
    done = subprocess.run([str(program)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
