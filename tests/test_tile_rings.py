"""The one-pass attention kernel's ring of key and value tiles: no stage serves both issuing warps, each of which follows its own kind of tile by the
parity of a stage's uses.  The rule is the kernel's own, compiled for the host; no GPU is needed."""
import os
import subprocess

from paper_2407_13885_b200 import build

PROGRAM = r"""
#include "attn_onepass.cuh"
#include <cstdio>

using namespace attnw::av1;

template <int STAGES, bool TWO_ISSUERS>
int check(const char* what) {
    int user[STAGES], uses[STAGES] = {};
    for (int& u : user) u = -1;
    Tiles<STAGES, TWO_ISSUERS> of_kind[2] = {Tiles<STAGES, TWO_ISSUERS>(0), Tiles<STAGES, TWO_ISSUERS>(1)};
    for (int n = 0; n < 200; ++n)
        for (int kind = 0; kind < 2; ++kind) {
            Tiles<STAGES, TWO_ISSUERS>& p = of_kind[TWO_ISSUERS ? kind : 0];
            const int issuer = TWO_ISSUERS ? kind : 0;
            if (p.stage < 0 || p.stage >= STAGES) return std::printf("%s: stage %d\n", what, p.stage), 1;
            if (user[p.stage] >= 0 && user[p.stage] != issuer) return std::printf("%s: stage %d has two issuers\n", what, p.stage), 1;
            user[p.stage] = issuer;
            if (p.parity != (uses[p.stage]++ & 1u)) return std::printf("%s: use %d of stage %d has the wrong parity\n", what, uses[p.stage] - 1, p.stage), 1;
            p.next();
        }
    for (int s = 0; s < STAGES; ++s)
        if (uses[s] == 0) return std::printf("%s: stage %d is never used\n", what, s), 1;
    return 0;
}

template <int D>
int check_all() {
    return check<Smem<D>::kStages, Smem<D>::two_issuers(kWhole)>("two query tiles") || check<Smem<D>::kStages + 1, Smem<D>::two_issuers(kSplit)>("split") ||
           check<Smem<D>::kStages + 1, Smem<D>::two_issuers(kCluster)>("cluster");
}

int main() { return check_all<64>() || check_all<128>(); }
"""


def test_no_stage_serves_two_issuers(tmp_path):
    source, program = tmp_path / "rings.cu", tmp_path / "rings"
    source.write_text(PROGRAM)
    csrc = os.path.dirname(build.SOURCES[0])
    subprocess.run([build.nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I" + csrc, "-o", str(program), str(source)], check=True)
    done = subprocess.run([str(program)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
