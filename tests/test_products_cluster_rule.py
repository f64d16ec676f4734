"""The rule by which a mixture-of-experts layer runs in one cluster or on every SM
(rr_internal.h), compiled and asked on the host."""
import os
import subprocess

import pytest

from paper_2512_22492_gb300 import build as B

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "rr_internal.h"
int main(int argc, char** argv) {
    for (int i = 1; i + 1 < argc; i += 2) std::printf("%d\n", rr_moe_cluster(std::atoll(argv[i]), std::atoi(argv[i + 1])));
    return 0;
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    at = tmp_path_factory.mktemp("rule")
    (at / "rule.cpp").write_text(PROGRAM)
    exe = str(at / "rule")
    subprocess.check_call(["g++", "-std=c++17", "-I", B.INCLUDE, "-I", B.CSRC, "-I",
                           os.path.join(B._cuda_home(), "include"), str(at / "rule.cpp"), "-o", exe, "-ldl"])

    def ask(*pairs):
        out = subprocess.check_output([exe] + [str(v) for p in pairs for v in p], text=True, timeout=60)
        return [int(v) for v in out.split()]
    return ask


def test_a_whole_gpu(rule):
    assert rule((1, 16), (150_000, 16), (1 << 18, 16), ((1 << 18) + 1, 16), (2_400_000, 16), (2_500_000, 16),
                (1 << 40, 16)) == [8, 8, 8, 16, 16, 0, 0]


def test_no_room_for_the_cluster(rule):
    """Never a cluster that the device cannot place: the grid takes the layer."""
    assert rule((150_000, 8), (1_000_000, 8), (2_500_000, 8)) == [8, 0, 0]
    assert rule((150_000, 0), (1_000_000, 0), (2_500_000, 0)) == [0, 0, 0]
