"""What k_fp4_few does about its copies when a wait ran out, against a model of its
stages' barriers: every combination of how far the producer and the quantising warps had
come leaves each phase that copies land in complete, and no arrival in another one."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SRC = r"""
#include <algorithm>
#include <cstdio>
#include <vector>
#include "fp4_settle.h"

struct Barrier {
    int need, have = 0, done = 0;
    void arrive() {
        if (++have == need) { have = 0; ++done; }
    }
};

// Steps of a stage ring: agent 0 is the producer.  False for a state that cannot be: step k
// is taken only when all have taken step k - stages.
template <int WARPS> bool reachable(const int* came, int stages) {
    for (int a = 0; a <= WARPS; ++a)
        for (int b = 0; b <= WARPS; ++b)
            if (came[a] > came[b] + stages) return false;
    return true;
}

template <int WARPS> int check(const int* came, int stages) {
    std::vector<Barrier> bar(stages, Barrier{WARPS + 1});
    const int most = *std::max_element(came, came + WARPS + 1);
    for (int k = 0; k < most; ++k)
        for (int a = 0; a <= WARPS; ++a)
            if (k < came[a]) bar[k % stages].arrive();
    std::vector<int> waited(stages, 0);
    moara::settle_few<WARPS>(
        came[0], came + 1, stages, [&](int s) { bar[s].arrive(); },
        [&](int s, uint32_t parity) { waited[s] = bar[s].done > 0 && ((bar[s].done - 1) & 1) == static_cast<int>(parity) ? 1 : -1; });
    for (int s = 0; s < stages; ++s) {
        const int phases = came[0] > s ? (came[0] - 1 - s) / stages + 1 : 0;       // that copies landed in
        if (waited[s] != (phases > 0 ? 1 : 0) || bar[s].done != phases) return 1;
    }
    return 0;
}

int main() {
    int tried = 0;
    for (int stages = 1; stages <= 4; ++stages) {
        const int top = 2 * stages + 2;
        int c[5];
        for (c[0] = 0; c[0] <= top; ++c[0]) {
            if (check<0>(c, stages)) return 1;
            for (c[1] = 0; c[1] <= top; ++c[1])
                for (c[2] = 0; c[2] <= top; ++c[2])
                    for (c[3] = 0; c[3] <= top; ++c[3])
                        for (c[4] = 0; c[4] <= top; ++c[4]) {
                            if (!reachable<4>(c, stages)) continue;
                            ++tried;
                            if (check<4>(c, stages)) {
                                std::printf("stages %d: %d %d %d %d %d\n", stages, c[0], c[1], c[2], c[3], c[4]);
                                return 2;
                            }
                        }
        }
    }
    return tried > 1000 ? 0 : 3;
}
"""


def test_every_way_to_give_up(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    if shutil.which("g++") is None or not os.path.exists(os.path.join(inc, "cuda_runtime.h")):
        pytest.skip("no host compiler or CUDA headers")
    (tmp_path / "t.cpp").write_text(SRC)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", inc, "-I", os.path.join(ROOT, "paper_2609_15037_gb300", "csrc"),
                    str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    p = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout
