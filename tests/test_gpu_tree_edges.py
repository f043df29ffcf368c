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


def test_a_refused_device_is_not_reported_by_the_next_call(ctx):
    """The C API on a device that does not exist (nothing is launched), then a call that is all right."""
    import ctypes as C

    from paper_2509_00419_amd import binding as bd
    c = Caches(BF, [[3, 5]], 16, 64).dev()
    cache = bd.Cache(c.k.data_ptr(), c.v.data_ptr(), None, None, None, None, 16, 0, 0, 0)
    d = bd.AppendDesc(bd.BF16, 1, 0, 0, 2, 64, 0, 0, 1, (C.c_int32 * 3)(), 2, 0)
    out = torch.zeros_like(c.len)
    for context, status in ((lv.Context(99), 4), (ctx, 0)):
        s = torch.cuda.current_stream().cuda_stream
        assert bd.lib.lvlm_kv_append(context._h, s, C.byref(d), C.byref(bd.AppendSrc()), C.byref(cache), c.len.data_ptr(), out.data_ptr()) == status
    assert torch.equal(out, c.len)
