"""GPU tests: the calls of test_gpu_tree.py that are compared with the oracle by check_attn, with no NaN let through.  Its largest error skips
rows that are not in use, whose reference is NaN, and so any NaN that a call wrote; in these calls no row in use sees one."""
import pytest
import torch

import paper_2509_00419_amd as lv
import test_gpu_tree as tests
from test_gpu_tree import ATTN, BF, FP

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return lv.Context(0)


@pytest.fixture(autouse=True)
def no_nan(monkeypatch):
    plain = tests.check_attn

    def check(*args, **kw):
        out, lse = plain(*args, **kw)
        assert not bool(torch.isnan(out).any()) and not bool(torch.isnan(lse).any())
        return out, lse
    monkeypatch.setattr(tests, "check_attn", check)


@pytest.mark.parametrize("case", ATTN, ids=lambda c: "-".join(map(str, c)))
def test_every_shape(ctx, case):
    tests.test_tree_attention_matches_the_oracle(ctx, *case)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_rows_without_entries(ctx, dtype):
    tests.test_rows_without_entries_short_heads_and_long_bounds(ctx, dtype)


@pytest.mark.parametrize("dtype,T,G", [(BF, 5, 2), (BF, 64, 3), (FP, 5, 2), (FP, 1, 3), (BF, 1, 3)])
def test_pages_outside_the_pool(ctx, dtype, T, G):
    if T > 1:
        tests.test_what_a_row_does_not_see_adds_nothing(ctx, dtype, T, G)
    c = tests.Caches(dtype, [[60 + T]], 128, 128, 16, 13)
    c.pages[0, 0, 1], c.pages[0, 0, 2] = -1, 10 ** 6                        # entries 16 .. 47 are nowhere
    q = torch.randn(1, T, G, 128, generator=torch.Generator().manual_seed(12)).to(dtype)
    tests.check_attn(ctx, c, q, dtype)
    c.pages[0, 0] = -5                                                      # all of them
    tests.check_attn(ctx, c, q, dtype)


@pytest.mark.parametrize("dtype,gain", [(BF, 40.0), (FP, 40.0), (BF, 0.0), (FP, 400.0)])
def test_far_and_equal_logits(ctx, dtype, gain):
    tests.test_far_and_equal_logits(ctx, dtype, gain)


def test_strided_queries_and_outputs(ctx):
    tests.test_strided_queries_and_outputs(ctx)
