"""GPU tests of the drafted-token calls at the edges of what they take."""
import pytest
import torch

import paper_2509_00419_amd as lv
from test_gpu_tree import BF, DEV, Caches

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return lv.Context(0)


def test_append_of_no_rows_with_positions_and_queries(ctx):
    c = Caches(BF, [[3, 5], [0, 16]], 16, 64).dev()
    keep = c.k.clone()
    k, q = torch.empty(2, 0, 2, 64, dtype=BF, device=DEV), torch.empty(2, 0, 8, 64, dtype=BF, device=DEV)
    freq = torch.ones(32, device=DEV)
    out, turned = ctx.kv_append(k, k, c.k, c.v, c.len, pos=torch.empty(2, 0, dtype=torch.int32, device=DEV), inv_freq=freq, q=q)
    assert torch.equal(out, c.len) and turned.shape == q.shape and torch.equal(c.k, keep)
    out, turned = ctx.kv_append(k, k, c.k, c.v, c.len, pos=torch.empty(3, 2, 0, dtype=torch.int32, device=DEV), inv_freq=freq,
                                sections=(8, 12, 12), q=q, q_out=q, length_out=c.len)
    assert out is c.len and turned is q and c.len.tolist() == [[3, 5], [0, 16]]
