"""GPU tests of the drafted-token calls at the edges of what they take."""
import math

import pytest
import torch

import paper_2509_00419_amd as lv
import test_gpu_tree as tests
from test_gpu_parity import _guarded
from test_gpu_tree import BF, DEV, LONG, Caches
from test_gpu_tree_cuts import CUTS

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


@pytest.mark.parametrize("adjacent", [False, True])
def test_far_positions_turn_as_exactly_as_near_ones(ctx, adjacent):
    """Unit keys and queries become the cosine and sine of their angles: 2^-25 of a turn off at most (2 pi 2^-25), by which either changes as
    much at most, and 4 ulp of a number up to 1 (2^-22) for the function itself; the products are with 1 and 0.  Frequencies of hundreds,
    positions near the last there are: 2^38 turns, of which one 64-bit word keeps 2^-15."""
    from fractions import Fraction
    two_pi = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798214808651")
    T, d = 37, 64
    g = torch.Generator().manual_seed(5)
    freq = torch.cat([torch.rand(28, generator=g) * 500 + 500, torch.tensor([1.0, 0.5, 1e-6, 0.0])])
    pos = torch.randint(2 ** 30, 2 ** 31 - 1, (1, T), generator=g, dtype=torch.int64)
    pos[0, ::3] *= -1
    pos[0, :2] = torch.tensor([2 ** 31 - 1, -2 ** 31])
    want = torch.empty(T, 32, 2, dtype=torch.float64)
    for t in range(T):
        for c in range(32):
            turns = int(pos[0, t]) * Fraction(float(freq[c])) / two_pi
            part = 2 * math.pi * float(turns - round(turns))
            want[t, c, 0], want[t, c, 1] = math.cos(part), math.sin(part)
    one = torch.zeros(1, T, 1, d)
    one[..., 0::2] = 1.0
    if not adjacent:
        one = torch.cat([torch.ones(1, T, 1, 32), torch.zeros(1, T, 1, 32)], dim=-1)
    one = one.to(DEV)
    c = Caches(torch.float32, [[0]], 48, d).dev()
    _, q = ctx.kv_append(one, one, c.k, c.v, c.len, pos=pos.to(torch.int32).to(DEV), inv_freq=freq.to(DEV), adjacent=adjacent, q=one)
    for x in (c.k[0, 0, :T], q[0, :, 0]):
        x = x.double().cpu()
        x = x.view(T, 32, 2) if adjacent else x.view(T, 2, 32).transpose(1, 2)
        assert float((x - want).abs().max()) <= 2 * math.pi * 2.0 ** -25 + 2.0 ** -22


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_as_many_lists_as_a_call_may_have(ctx, dtype):
    """2^23 - 2 lists of one entry: a row's result is its value.  fp32: the probability is not 1 where the scaled logit was rounded, and is divided by
    itself: three roundings, and that of the product, of 2^-24 each."""
    B, H, d = 12282, 683, 64
    g = torch.Generator(device=DEV).manual_seed(3)
    k, v, q = (torch.randn(B, H, 1, d, generator=g, device=DEV).to(dtype) for _ in range(3))
    length = torch.ones(B, H, dtype=torch.int32, device=DEV)
    out, lse = ctx.tree_attn(q.view(B, 1, H, d), k, v, length, want_lse=True)
    v = v.view(B, 1, H, d)
    if dtype == BF:
        assert torch.equal(out, v)
    else:
        assert bool(((out - v).abs() <= 4 * 2.0 ** -24 * v.abs()).all())
    for b, h in ((0, 0), (B // 2, 5), (B - 1, H - 1)):
        x = q[b, h, 0].double() * k[b, h, 0].double() * d ** -0.5
        off = abs(float(lse[b, h, 0]) - float(x.sum()))
        assert off <= 2.0 ** -24 * ((d + 4) * float(x.abs().sum()) + 5 + 4 * abs(float(x.sum())))       # (as in test_gpu_tree.py)


@pytest.mark.parametrize("case", [c for c in LONG[:16] + CUTS if c[7] == 0 and c[1] * c[4] <= 100], ids=lambda c: "-".join(map(str, c[1:7])))
def test_tree_attention_stays_within_the_workspace_it_asked_for(case):
    """A guard band behind exactly that many bytes; heads longer than the bound, empty, and in between."""
    dtype, B, T, Hq, Hkv, d, slots = case[:7]
    lens = torch.randint(0, 2 * slots, (B, Hkv), generator=torch.Generator().manual_seed(slots))
    lens[0, 0], lens[-1, -1] = slots + 9, 0
    c = Caches(dtype, lens.tolist(), slots + 9, d, 0, slots).dev()
    q = torch.randn(B, T, Hq, d, generator=torch.Generator().manual_seed(T)).to(dtype).to(DEV)
    _guarded(lambda context, reserve: context.tree_attn(q, c.k, c.v, c.len, len_bound=slots, reserve=reserve))


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_append_and_commit_of_as_many_sequences_as_a_call_may_have(ctx, dtype):
    """65535 sequences, counts that have to be clamped: entries where they belong, lengths, and what stays as it was."""
    B, H, d, room, T = 65535, 2, 64, 4, 3
    g = torch.Generator(device=DEV).manual_seed(9)
    k, v = (torch.randn(B, T, H, d, generator=g, device=DEV).to(dtype) for _ in range(2))
    kc, vc = (torch.zeros(B, H, room, d, dtype=dtype, device=DEV) for _ in range(2))
    length = (torch.arange(B * H, device=DEV, dtype=torch.int32) % 2).view(B, H)
    n = torch.randint(-2, T + 4, (B,), generator=g, device=DEV, dtype=torch.int32)
    out, _ = ctx.kv_append(k, v, kc, vc, length, n_new=n)
    took = n.clamp(0, T)
    assert torch.equal(out, length + took[:, None])
    slot = torch.arange(room, device=DEV).view(1, 1, room) - length.unsqueeze(-1)           # new row of each slot
    held = (slot >= 0) & (slot < took.view(B, 1, 1))
    for new, cache in ((k, kc), (v, vc)):
        want = torch.gather(new.transpose(1, 2), 2, slot.clamp(0, T - 1).unsqueeze(-1).expand(-1, -1, -1, d).long())
        assert torch.equal(cache, torch.where(held.unsqueeze(-1), want, torch.zeros_like(want)))
    keep = kc.clone()
    path = torch.tensor([[1, 2, 7]], dtype=torch.int32, device=DEV).expand(B, 3).contiguous()
    done = ctx.tree_commit(kc, vc, length, path, took)
    # rows 1 and 2 move to places 0 and 1 where they lie in the slots; row 7 never does
    moved = torch.minimum(took, torch.full_like(took, 2)).view(B, 1)
    assert torch.equal(done, length + moved)
    for i in range(2):
        here = moved > i
        to, come = (length + i).long().clamp(max=room - 1), (length + i + 1).long().clamp(max=room - 1)
        row = torch.gather(keep, 2, torch.where(here, come, to).view(B, H, 1, 1).expand(B, H, 1, d))
        assert torch.equal(torch.gather(kc, 2, to.view(B, H, 1, 1).expand(B, H, 1, d)), row)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (torch.float32, 64)])
def test_as_many_rows_as_a_list_may_have(ctx, dtype, d):
    tests.test_every_cut_matches_the_formula(ctx, dtype, 1, 1024, 63, 1, d, 1100, 0, "tree")


@pytest.mark.parametrize("dtype,T", [(BF, 1), (BF, 70), (torch.float32, 1), (torch.float32, 5)])
def test_the_longest_list_there_can_be(ctx, dtype, T):
    """2^24 slots of one head.  Queries of zero weigh all entries alike, so every sum is one of whole numbers below 2^25, and a row is the
    mean of what it sees: as far as fp32 holds a quotient, and the fold's sums, 64 roundings of 2^-24."""
    L, d = 1 << 24, 64
    k, v = (torch.zeros(1, 1, L, d, dtype=dtype, device=DEV) for _ in range(2))
    k.normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    v[0, 0, : L // 2] = 1.0
    v[0, 0, L - T:] = 64.0
    length = torch.tensor([[L]], dtype=torch.int32, device=DEV)
    q = torch.zeros(1, T, 1, d, dtype=dtype, device=DEV)
    out, lse = ctx.tree_attn(q, k, v, length, want_lse=True)
    for t in range(T):
        seen = L - T + t + 1
        mean = (L // 2 + 64.0 * (t + 1)) / seen
        step = 2.0 ** -8 if dtype == BF else 0.0
        assert float((out[0, t, 0].double() - mean).abs().max()) <= mean * (72 * 2.0 ** -24 + step), t
        assert abs(float(lse[0, 0, t]) - math.log(seen)) <= 72 * 2.0 ** -24 + 4 * 2.0 ** -24 * math.log(seen)
