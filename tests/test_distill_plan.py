"""How mpt_distill_topk chooses the clusters that share a long row, with the device's answers faked: no GPU."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1710_03740_b200", "csrc")
SOURCE = """
#include "distill_plan.h"
extern "C" int choose(int *known, int B, int C, const int *answers, int *asked)
{
    int (&k)[mpt::kDistillClusters] = *(int (*)[mpt::kDistillClusters])known;
    return mpt::distill_cluster_log2(k, B, C, [&](int ctas) {
        int i = 0;
        while ((1 << i) < ctas) i++;
        asked[i]++;
        return answers[i];
    });
}
"""
FULL = [148, 74, 35, 16]


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    lib = C.CDLL(str(d / "plan.so"))

    def call(B, classes, answers, known=None):
        known = known if known is not None else (C.c_int * 4)()
        asked = (C.c_int * 4)()
        got = lib.choose(known, B, classes, (C.c_int * 4)(*answers), asked)
        return got, list(known), list(asked)
    return call


@pytest.mark.parametrize("B,classes,size", [(512, 793471, 1), (700, 131072, 0), (10, 250000, 3), (1, 40000, 2), (148, 40000, 0), (100000, 60000, 0)])
def test_choices(choose, B, classes, size):
    """The measured ones, and 1 x 40000, where 4 and 8 CTAs cost the same 23000 classes: the fewer."""
    assert choose(B, classes, FULL)[0] == size


@pytest.mark.parametrize("none", [0, -1])
def test_sizes_that_do_not_fit_are_left_out(choose, none):
    """0: no such cluster is resident; -1: the question itself failed.  Every other size still serves the call."""
    for gone in range(4):
        answers = [none if i == gone else FULL[i] for i in range(4)]
        for B, classes in ((512, 793471), (700, 131072), (10, 250000), (148, 40000)):
            got = choose(B, classes, answers)[0]
            assert got >= 0 and got != gone
    assert choose(10, 250000, [148, none, none, none])[0] == 0
    assert choose(10, 250000, [none] * 4)[0] == -1


def test_answers_are_kept_and_errors_asked_again(choose):
    known = (C.c_int * 4)()
    assert choose(10, 250000, [148, 74, 0, -1], known) == (1, [148, 74, -1, 0], [1, 1, 1, 1])
    assert choose(10, 250000, FULL, known) == (3, [148, 74, -1, 16], [0, 0, 0, 1])

