"""Host check of how a list of places is divided among runs: compiles the library's argument header with g++, so
that what is undefined ends the program."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2307_04339_amd", "csrc")

SRC = r"""
#include <cstdio>
#include "seq_args.h"
using namespace miriam;
int main() {
    long bad = 0;
    const Runs none = runs_of(0, 0);           // a batch without new tokens
    if (none.runs != 0 || none.run != 0 || none.more != 0) ++bad;
    const int places[] = {0, 1, 2, 3, 511, 512, 513, 4000, 99991, (1 << 30) + 7, 0x7fffffff};
    for (int n : places)
        for (int runs = 1; runs <= 1024; ++runs) {
            const Runs r = runs_of(n, runs);
            if (r.start(0) != 0 || r.start(runs) != n) ++bad;
            for (int k = 0; k < runs; ++k) {
                const int len = r.start(k + 1) - r.start(k);
                if (r.start(k) != (int)((long long)k * n / runs) || (len != n / runs && len != n / runs + 1)) ++bad;
            }
        }
    std::printf("bad %ld\n", bad);
    return bad != 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_runs_cover_their_places(tmp_path):
    src, exe = tmp_path / "runs.cpp", tmp_path / "runs"
    src.write_text(SRC)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
