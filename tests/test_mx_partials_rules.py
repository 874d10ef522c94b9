"""The partial sums' GPU tests reach every tile shape that can leave them (csrc/mx_rules.h, compiled with the host compiler)."""
import ctypes
import os
import subprocess

import pytest

from test_gpu_mx_partials import ONE_SLICE_FROM, SIZES, slice_length

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_04147_amd", "csrc")
PROGRAM = """
#include "mx_rules.h"
extern "C" {
int slices(int N, int K) { return mx_slices(K, mx_split(N, K, false)); }
int slice(int K) { return mx_slice(K, 4); }
int choose(int M, int N, int K) { return mx_choose(M, N, K, slices(N, K), false); }
int choose_all(int M, int N, int K) { return mx_choose_all(M, N, K, slices(N, K)); }
int kinds() { return MX_N_KINDS; }
int results(int k) { return mx_kind(k).results; }
int halves(int k) { return mx_kind(k).halves; }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(d / "rules.cpp"), "-o", str(d / "rules.so")], check=True)
    return ctypes.CDLL(str(d / "rules.so"))


def test_every_listed_size_leaves_the_partial_sums_of_its_shape(rules):
    for kind, slices, M, N, K in SIZES:
        assert (rules.choose(M, N, K), rules.slices(N, K)) == (kind, slices) and rules.choose_all(M, N, K) < 0, (kind, M, N, K)
        assert rules.slice(K) == slice_length(K) and N <= ONE_SLICE_FROM
    assert rules.slices(ONE_SLICE_FROM, 1 << 20) == 1


def test_every_shape_of_sums_is_listed_with_several_slices(rules):
    sums = [k for k in range(rules.kinds()) if rules.results(k) & 1]
    assert {(k, 4) for k in sums} <= {s[:2] for s in SIZES}
    # three slices, an odd number of partial sums: every shape that walks two of them (and more)
    assert {(k, 3) for k in sums if rules.halves(k)} <= {s[:2] for s in SIZES}


def test_a_context_takes_them_too(rules):
    """Down projection of the forwards under test, three slices at the rows of one to five blocks: shapes of few rows."""
    shapes = {rules.choose(M, 2048, 2304) for M in (24, 32, 64, 90, 192, 320)}
    assert rules.slices(2048, 2304) == 3 and {0, 1, 2, 3} <= shapes
