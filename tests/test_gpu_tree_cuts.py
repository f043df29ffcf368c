"""GPU tests of tree attention in the cuts that test_gpu_tree.LONG leaves out: with it, every form of workgroup is taken with a pair's entries
whole, in runs and in runs dealt out by the lengths (test_host_tree_rules.py holds the two lists to that).  The tests are those of LONG."""
import pytest

import paper_2509_00419_amd as lv
import test_gpu_tree as tests
from test_gpu_tree import BF, FP

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return lv.Context(0)


# The rows of a form's workgroups ("few": fp32 on the vector ALUs), and how the entries are cut.
CUTS = [
    # dtype, B, T, Hq, Hkv, d, slots, page, rows, entries
    (BF, 3, 9, 6, 2, 64, 300, 0, "32", "whole"), (BF, 2, 1, 28, 4, 64, 1024, 64, "32", "whole"),
    (BF, 1, 5, 8, 2, 64, 2000, 0, "32", "runs"), (BF, 1, 2, 14, 2, 64, 4096, 16, "32", "runs"),
    (BF, 9, 1, 4, 4, 64, 14300, 0, "32", "dealt"), (BF, 9, 4, 28, 4, 64, 14336, 256, "32", "dealt"),
    (BF, 49, 34, 3, 3, 64, 2960, 0, "64", "dealt"), (BF, 11, 107, 2, 2, 64, 5813, 0, "128", "runs"),
    (BF, 43, 167, 13, 13, 64, 5334, 0, "256", "runs"),
    (BF, 16, 1, 28, 4, 128, 1100, 0, "32", "whole"), (BF, 8, 4, 40, 8, 128, 512, 32, "32", "whole"),
    (BF, 1, 3, 8, 2, 128, 2000, 0, "32", "runs"), (BF, 1, 4, 28, 4, 128, 4096, 128, "32", "runs"),
    (BF, 15, 2, 4, 1, 128, 16500, 0, "32", "dealt"), (BF, 4, 4, 16, 4, 128, 16384, 64, "32", "dealt"),
    (BF, 41, 34, 1, 1, 128, 5019, 0, "64", "dealt"), (BF, 31, 66, 17, 17, 128, 4105, 0, "128", "runs"),
    (BF, 103, 149, 6, 6, 128, 5109, 0, "256", "runs"),
    (FP, 7, 1, 2, 2, 64, 17700, 0, "few", "dealt"), (FP, 1, 5, 1, 1, 64, 65, 0, "32", "whole"), (FP, 4, 8, 4, 4, 64, 128, 16, "32", "whole"),
    (FP, 11, 5, 4, 4, 64, 2674, 0, "32", "dealt"), (FP, 6, 33, 1, 1, 64, 11024, 0, "64", "dealt"), (FP, 2, 66, 4, 4, 64, 5239, 0, "128", "dealt"),
    (FP, 7, 1, 1, 1, 128, 17600, 0, "few", "dealt"), (FP, 7, 2, 2, 2, 128, 16384, 64, "few", "dealt"), (FP, 1, 5, 1, 1, 128, 8215, 0, "64", "dealt"),
    (FP, 11, 65, 4, 4, 128, 266, 0, "128", "runs"),
]


def shape(case):
    return "-".join(map(str, case[1:]))


@pytest.mark.parametrize("kind", ["chain", "tree"])
@pytest.mark.parametrize("case", CUTS, ids=shape)
def test_every_cut_matches_the_formula(ctx, case, kind):
    tests.test_every_cut_matches_the_formula(ctx, *case[:8], kind)


@pytest.mark.parametrize("case", CUTS, ids=shape)
def test_every_cut_survives_logits_that_grow_and_values_that_are_large(ctx, case):
    tests.test_every_cut_survives_logits_that_grow_and_values_that_are_large(ctx, *case[:8])


# Nine sequences of one KV head, as that test has them.
UNSEEN = [
    # dtype, T, Hq, d, slots, rows, entries
    (BF, 3, 7, 64, 200, "32", "whole"), (BF, 3, 7, 64, 4200, "32", "runs"), (BF, 27, 1, 128, 200, "32", "whole"), (BF, 4, 6, 128, 4200, "32", "runs"),
    (BF, 2, 4, 128, 20000, "32", "runs"), (FP, 9, 1, 64, 120, "32", "whole"), (FP, 9, 1, 128, 300, "64", "runs"),
]


@pytest.mark.parametrize("case", UNSEEN, ids=shape)
def test_no_cut_lets_in_what_a_row_does_not_see(ctx, case):
    tests.test_no_cut_lets_in_what_a_row_does_not_see(ctx, *case[:5])
