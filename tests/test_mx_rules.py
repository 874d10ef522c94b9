"""The rules that cut a microscaled product (csrc/mx_rules.h), compiled with the host compiler, and that the GPU tests reach every shape."""
import ctypes
import os
import subprocess

import pytest

from test_gpu_mx_shapes import ALL, SIZES

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_04147_amd", "csrc")
PROGRAM = """
#include "mx_rules.h"
extern "C" {
int split(int N, int K, int swiglu) { return mx_split(N, K, swiglu); }
int slice(int K, int s) { return mx_slice(K, s); }
int slices(int K, int s) { return mx_slices(K, s); }
int choose(int M, int N, int K, int swiglu) { return mx_choose(M, N, K, mx_slices(K, mx_split(N, K, swiglu)), swiglu); }
int choose_all(int M, int N, int K, int swiglu) { return mx_choose_all(M, N, K, mx_slices(K, mx_split(N, K, swiglu))); }
int all_kinds() { return MX_N_ALL_KINDS; }
int kinds() { return MX_N_KINDS; }
int results(int k) { return mx_kind(k).results; }
int halves(int k) { return mx_kind(k).halves; }
int lds(int k) {
    const MxKind& x = mx_kind(k);
    const int waves = x.wn * x.wm, bn = x.wn * x.tn * 32, bm = x.wm * x.tm * 32, g = x.kc / 128;
    const int w = bn * x.kc / 2 / 1024, r = bm * x.kc / 1024, s = (bn / 32 * g + 7) / 8 + (bm / 32 * g + 7) / 8;
    return w % waves || r % waves ? -1 : x.nst * (w + r + (s + waves - 1) / waves * waves) * 1024;
}
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(d / "rules.cpp"), "-o", str(d / "rules.so")], check=True)
    return ctypes.CDLL(str(d / "rules.so"))


def test_slices_cover_the_columns(rules):
    for N in (1, 512, 4096, 8192, 8193, 37888):
        for swiglu in (0, 1):
            for K in list(range(32, 6000, 32)) + [12288, 18944, 1 << 20]:
                s = rules.split(N, K, swiglu)
                n, length = rules.slices(K, s), rules.slice(K, s)
                assert 1 <= n <= s <= 4 and length % 256 == 0
                assert (n - 1) * length < K <= n * length
                # never two: a shape that walks them both would leave one sum where the others leave two, which a consumer adds to
                # its residual one after the other
                assert n != 2
                # the count of slices alone gives the same cut: kernels are told nothing else
                assert rules.slice(K, n) == length and rules.slices(K, n) == n


def test_every_shape_is_one_that_a_call_can_take(rules):
    for k in range(rules.kinds()):
        assert 0 < rules.lds(k) <= 160 * 1024
        assert rules.results(k) in (1, 2, 3) and not (rules.halves(k) and rules.results(k) != 1)
    for M in (1, 7, 32, 33, 64, 100, 160, 500, 2304, 1 << 20):
        for N in (1, 64, 4096, 12288, 1 << 20):
            for K in (32, 1024, 4096, 18944, 1 << 20):
                if M * N <= 1 << 33:
                    k = rules.choose(M, N, K, 0)
                    assert rules.results(k) & 1 and (not rules.halves(k) or rules.slices(K, rules.split(N, K, 0)) > 1)
                    if N % 64 == 0:
                        assert rules.results(rules.choose(M, N, K, 1)) & 2


def test_the_gpu_tests_reach_every_shape(rules):
    reached = set()
    for kind, M, N, K, result in SIZES:
        assert rules.choose(M, N, K, int(result == "swiglu")) == kind, (kind, M, N, K, result)
        if rules.choose_all(M, N, K, int(result == "swiglu")) < 0:
            reached.add((kind, result))
    for k in range(rules.kinds()):
        wanted = {"swiglu"} if rules.results(k) == 2 else {"fp32"} if rules.halves(k) else {"fp32", "bf16"}
        if rules.results(k) == 3:
            wanted.add("swiglu")
        assert wanted <= {r for kk, r in reached if kk == k}, k
    reached = {(rules.choose_all(M, N, K, 0), result) for _, M, N, K, result in ALL}
    assert all(rules.choose_all(M, N, K, 0) == kind for kind, M, N, K, _ in ALL)
    assert reached == {(k, r) for k in range(rules.all_kinds()) for r in ("fp32", "bf16")}
    assert all(rules.choose_all(M, N, K, int(N > 8192)) < 0 for M in (1, 64, 2304) for N in (64, 8192, 8256) for K in (32, 2016)) and rules.choose_all(8, 4096, 4096, 1) < 0
    assert all(rules.choose_all(9000, N, K, 0) < 0 <= rules.choose_all(M, N, K, 0) for M in (1, 50, 300, 1000, 2304) for N, K in ((2047, 2080), (4097, 2336), (8191, 2048), (4096, 4096)))
