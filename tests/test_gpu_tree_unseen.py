"""GPU tests of what a drafted row sees and does not see where values are no numbers: tree_attn against the formula in 64 bits, every
live element compared (a NaN fails), and to the bit against the same call over caches that hold numbers there.

Tolerances as in test_gpu_tree.py."""
import pytest
import torch

import paper_2509_00419_amd as lv
from test_gpu_tree import BF, DEV, FP, U, Caches, dense

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return lv.Context(0)


# One row in use that does not see itself.  Rows to a KV head and slots that take workgroups of 32, 64, 128 and 256 rows, and of up to
# four in fp32, with the entries whole and in runs; the drafted row is the last of a whole tile of 32, or not.
ALONE = [
    # dtype, B, T, Hq, Hkv, d, length
    (BF, 1, 1, 4, 4, 128, 32), (BF, 1, 1, 7, 1, 64, 256), (BF, 2, 1, 28, 4, 128, 1024), (BF, 2, 5, 16, 4, 128, 97), (BF, 1, 1, 8, 1, 128, 4096),
    (BF, 9, 1, 70, 1, 64, 4096), (BF, 33, 1, 80, 2, 128, 256), (BF, 9, 1, 150, 1, 128, 2048), (BF, 33, 1, 500, 4, 64, 1024),
    (BF, 9, 2, 1000, 2, 128, 640), (BF, 33, 1, 600, 2, 64, 1024),
    (FP, 1, 1, 8, 1, 64, 64), (FP, 1, 1, 8, 1, 128, 4096), (FP, 3, 6, 8, 2, 64, 640), (FP, 33, 1, 80, 2, 64, 256), (FP, 33, 1, 300, 2, 128, 608),
    (FP, 1, 1, 4, 4, 64, 32), (FP, 2, 2, 2, 1, 128, 4096),
]


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,d,length", ALONE)
def test_a_row_that_does_not_see_itself_stays_clear_of_its_own_value(ctx, dtype, B, T, Hq, Hkv, d, length):
    c = Caches(dtype, [[length] * Hkv] * B, length, d, 0, length).dev()
    q = torch.randn(B, T, Hq, d, generator=torch.Generator().manual_seed(T)).to(dtype).to(DEV)
    n_rows = [1] * B
    rows = torch.tensor(n_rows, dtype=torch.int32, device=DEV)
    words = torch.zeros(B, T, (T + 31) // 32, dtype=torch.int32, device=DEV)
    ref, ref_lse, weight = dense(c, q, n_rows, torch.zeros(B, T, T, dtype=torch.bool, device=DEV))
    e = (d + 4) * U * float(q.abs().double().sum(-1).max() * c.k.abs().max().double()) * d ** -0.5
    tol = weight * (2 * e + (length + 8) * U) + 1e-30
    if dtype == BF:
        tol = tol + 2.0 ** -8 * (weight + ref.abs())
    clean = None
    for bad_k, bad_v in ((0.0, 1.0), (float("nan"), float("nan")), (float("inf"), float("-inf")), (1.0, float("inf"))):
        c.k[:, :, length - 1], c.v[:, :, length - 1] = bad_k, bad_v
        out = torch.full((B, T, Hq, d), 7.0, dtype=dtype, device=DEV)
        lse = torch.full((B, Hq, T), 7.0, device=DEV)
        ctx.tree_attn(q, c.k, c.v, c.len, mask=words, n_rows=rows, out=out, row_lse=lse)
        assert bool((out[:, 1:] == 7.0).all()) and bool((lse[:, :, 1:] == 7.0).all())
        assert bool(((out[:, :1].double() - ref[:, :1]).abs() <= tol[:, :1]).all()), (bad_k, bad_v)
        assert bool(((lse[:, :, 0].double() - ref_lse[:, :, 0]).abs() <= e + (length + 4) * U + 4 * U * ref_lse[:, :, 0].abs()).all())
        clean = out if clean is None else clean
        assert torch.equal(out, clean), (bad_k, bad_v)


@pytest.mark.parametrize("L,at", [(40, 35), (40, 3), (300, 290), (64, 60)])
@pytest.mark.parametrize("dtype,T,G", [(BF, 1, 8), (BF, 5, 2), (BF, 1, 300), (FP, 1, 8), (FP, 5, 4), (FP, 1, 2)])
def test_what_a_row_sees_is_not_hidden_by_a_weight_of_zero(ctx, dtype, T, G, L, at):
    """An entry whose weight is below what fp32 holds: times an infinity that is no finite number, in any tile."""
    d = 64
    c = Caches(dtype, [[L + T]], 320, d, 0, L).dev()
    c.k[0, 0, at] = -8.0
    q = torch.full((1, T, G, d), 4.0, device=DEV).to(dtype)                  # (logit -256; the others' are a hundredth of that)
    c.k[0, 0, :at].mul_(0.01)
    c.k[0, 0, at + 1:].mul_(0.01)
    clean, clean_lse = ctx.tree_attn(q, c.k, c.v, c.len, want_lse=True)
    c.v[0, 0, at, 3], c.v[0, 0, at, 40] = float("inf"), float("nan")
    out, lse = ctx.tree_attn(q, c.k, c.v, c.len, want_lse=True)
    odd = torch.tensor([3, 40], device=DEV)
    assert not bool(torch.isfinite(out[..., odd].float()).any())
    keep = torch.ones(d, dtype=torch.bool, device=DEV)
    keep[odd] = False
    assert torch.equal(out[..., keep], clean[..., keep]) and torch.equal(lse, clean_lse)
