"""GPU parity of the drafted-token calls against the oracle (float64), through the torch binding.

Tolerances count roundings, elementwise.  u = 2^-24 (half a step of fp32).
  turned rows   angle off by 2 pi (2^-26 turns of fp32 + what 64 bits lose, |pos| 2^-50), sine and cosine by 4 ulp, a product and a
                sum: (|x_i| + |x_j|) (2^-21 + |pos| 2^-50); bf16 half a step of the result more (2^-8).
  logits        a dot product of d terms in fp32, the scale and the change to base 2: (d + 4) u sum |q| |k| scale =: e
  lse           e + (entries + 4) u + 4 u |lse|
  rows          weights off by 2 e + (entries + 8) u relatively, of sum p |v|; bf16: each probability and the result half a step more.
"""
import numpy as np
import pytest
import torch

import paper_2509_00419_amd as lv
from oracle import lvlm_oracle as O

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
BF, FP = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    return lv.Context(0)


def f64(t):
    return t.detach().cpu().double().numpy()


def host(t):
    return None if t is None else t.detach().cpu().numpy() if t.dtype not in (BF, FP) else f64(t)


class Caches:
    """Caches of given lengths: head-major with `spare` slots behind, or in shuffled pages of a pool with `extra` unused ones."""

    def __init__(self, dtype, lens, room, d, page=0, seed=0, extra=3):
        g = torch.Generator().manual_seed(seed)
        self.len = torch.tensor(lens, dtype=torch.int32)
        B, H = self.len.shape
        if page:
            wide = -(-room // page)
            n_pages = B * H * wide + extra
            self.pages = torch.randperm(n_pages, generator=g)[:B * H * wide].to(torch.int32).view(B, H, wide)
            shape = (n_pages, page)
        else:
            self.pages, shape = None, (B, H, room)
        self.k = torch.randn(*shape, d, generator=g).to(dtype)
        self.v = torch.randn(*shape, d, generator=g).to(dtype)
        self.score = torch.rand(*shape, generator=g)
        self.kind = torch.randint(0, 3, shape, generator=g).to(torch.uint8)
        self.pos = torch.randint(0, 9999, shape, generator=g).to(torch.int32)

    def dev(self):
        c = Caches.__new__(Caches)
        c.__dict__.update({k: None if x is None else x.to(DEV) for k, x in self.__dict__.items()})
        return c


def lens_of(B, H, most, ragged, seed):
    r = np.random.default_rng(seed)
    return (r.integers(0, most + 1, (B, H)) if ragged else np.full((B, H), most)).tolist()


def tree_of(T, seed):
    r = np.random.default_rng(seed)
    return np.array([-1 if t == 0 or r.random() < 0.1 else r.integers(max(0, t - 5), t) for t in range(T)], dtype=np.int32)


def check_attn(ctx, c, q, dtype, *, parents=None, mask=None, n_rows=None, len_bound=0, scale=None, out=None):
    """One call against the oracle; mask: bool [B, T, T].  Returns what the call wrote."""
    B, T, Hq, d = q.shape
    dv = c.dev()
    words = None
    if parents is not None:
        words = lv.tree_mask(torch.from_numpy(np.stack(parents))).to(DEV)
        mask = np.stack([O.tree_mask(p) for p in parents])
    elif mask is not None:
        bits = np.zeros((B, T, -(-T // 32) * 32), dtype=np.uint64)
        bits[..., :T] = mask
        w = (bits.reshape(B, T, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)
        words = torch.from_numpy(w).to(DEV)
    rows = None if n_rows is None else torch.tensor(n_rows, dtype=torch.int32, device=DEV)
    qd = q.to(DEV)
    out = torch.full((B, T, Hq, d), 7.0, dtype=dtype, device=DEV) if out is None else out
    lse = torch.full((B, Hq, T), 7.0, device=DEV)
    ctx.tree_attn(qd, dv.k, dv.v, dv.len, mask=words, n_rows=rows, pages=dv.pages, len_bound=len_bound, scale=scale, out=out, row_lse=lse)
    torch.cuda.synchronize()
    ref, ref_lse, weight = O.tree_attn(f64(q), f64(c.k), f64(c.v), host(c.len), mask=mask, n_rows=n_rows, pages=host(c.pages), scale=scale,
                                       len_bound=len_bound)
    got, got_lse = f64(out), f64(lse)
    left = np.isnan(weight)                                             # rows past n_rows
    assert np.array_equal(got[left], np.full(int(left.sum()), 7.0))
    assert np.array_equal(got_lse[np.isnan(ref_lse)], np.full(int(np.isnan(ref_lse).sum()), 7.0))
    kmax = np.abs(f64(c.k)[np.isfinite(f64(c.k))]).max()
    n = int(c.len.max().clamp(min=0)) + 1
    e = (d + 4) * U * np.abs(f64(q)).sum(-1).max() * kmax * (d ** -0.5 if scale is None else scale)
    with np.errstate(invalid="ignore"):
        tol = weight * (2 * e + (n + 8) * U) + 1e-30
        if dtype == BF:
            tol = tol + 2.0 ** -8 * (weight + np.abs(ref))
        worst = np.nanmax(np.abs(got - ref) / tol)
    assert worst <= 1.0, worst
    live = ~np.isnan(ref_lse)
    fin = live & np.isfinite(ref_lse)
    assert np.array_equal(got_lse[live & ~fin], ref_lse[live & ~fin])
    assert np.all(np.abs(got_lse[fin] - ref_lse[fin]) <= e + (n + 4) * U + 4 * U * np.abs(ref_lse[fin]))
    return out, lse


ATTN = [
    # dtype, B, T, Hq, Hkv, d, entries before the drafts, ragged, page, kind of mask
    (BF, 1, 1, 4, 1, 128, 0, False, 0, "chain"),              # a row that sees itself alone
    (BF, 2, 1, 28, 4, 128, 300, True, 0, "chain"),            # plain decoding, group of seven
    (BF, 3, 1, 8, 8, 64, 33, True, 16, "tree"),               # one head to a group, pages of half a tile
    (BF, 1, 2, 16, 1, 128, 31, False, 32, "tree"),            # one KV head, a group of sixteen
    (BF, 2, 7, 12, 4, 64, 129, True, 64, "tree"),
    (BF, 1, 32, 8, 8, 128, 64, False, 0, "tree"),
    (BF, 2, 33, 6, 2, 128, 95, True, 16, "tree"),             # the drafts reach over tiles and pages
    (BF, 1, 64, 48, 8, 128, 700, False, 128, "tree"),         # 384 rows to a KV head
    (BF, 1, 65, 4, 2, 64, 500, True, 256, "tree"),            # three words of a mask
    (BF, 1, 100, 10, 2, 128, 1, False, 0, "chain"),           # 500 rows, hardly anything before them
    (BF, 2, 130, 2, 2, 64, 40, True, 32, "chain"),
    (BF, 1, 257, 3, 1, 128, 17, False, 0, "chain"),
    (BF, 4, 5, 40, 8, 128, 1000, True, 0, "tree"),            # group of five
    (BF, 1, 3, 8, 2, 128, 5000, False, 64, "tree"),           # few rows, many entries: cut into runs
    (FP, 1, 1, 4, 4, 64, 256, False, 0, "chain"),
    (FP, 2, 9, 4, 2, 128, 75, True, 16, "tree"),
    (FP, 1, 27, 4, 4, 64, 320, True, 32, "tree"),
    (FP, 1, 70, 7, 1, 64, 50, False, 0, "chain"),
    (FP, 3, 40, 8, 2, 128, 0, False, 128, "tree"),            # nothing but the drafts
    (FP, 1, 2, 6, 2, 64, 3000, False, 0, "tree"),
]


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,d,before,ragged,page,kind", ATTN)
def test_tree_attention_matches_the_oracle(ctx, dtype, B, T, Hq, Hkv, d, before, ragged, page, kind):
    seed = T * 1000 + before
    n_rows = np.random.default_rng(seed).integers(1, T + 1, B).tolist() if ragged else None
    lens = np.array(lens_of(B, Hkv, before, ragged, seed)) + (np.array(n_rows)[:, None] if ragged else T)
    c = Caches(dtype, lens.tolist(), before + T + 5, d, page, seed)
    q = torch.randn(B, T, Hq, d, generator=torch.Generator().manual_seed(seed + 1)).to(dtype)
    parents = [tree_of(T, seed + b) for b in range(B)] if kind == "tree" else None
    check_attn(ctx, c, q, dtype, parents=parents, n_rows=n_rows)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_rows_without_entries_short_heads_and_long_bounds(ctx, dtype):
    """Masks that leave rows empty, no row in use, heads shorter than the drafts, lengths of zero and below, bounds that cut."""
    B, T, Hq, Hkv, d = 5, 6, 4, 2, 64
    c = Caches(dtype, [[6, 40], [0, 3], [-5, 6], [77, 60], [9, 9]], 77, d, 0, 5)
    q = torch.randn(B, T, Hq, d, generator=torch.Generator().manual_seed(6)).to(dtype)
    mask = np.random.default_rng(7).random((B, T, T)) < 0.4
    mask[0, 2] = mask[1, 0] = mask[2, 5] = False
    check_attn(ctx, c, q, dtype, mask=mask, n_rows=[6, 2, 6, 6, 0])
    check_attn(ctx, c, q, dtype, mask=mask, n_rows=[-3, 9, 1, 5, 6])        # counts are clamped
    check_attn(ctx, c, q, dtype, n_rows=[6, 2, 6, 6, 0], len_bound=50)      # entries at or beyond the bound are not read
    check_attn(ctx, c, q, dtype, mask=np.zeros((B, T, T), bool))


@pytest.mark.parametrize("dtype,T,G", [(BF, 5, 2), (BF, 64, 3), (FP, 5, 2)])
def test_what_a_row_does_not_see_adds_nothing(ctx, dtype, T, G):
    """NaN and infinities in stale slots, in other branches' keys and values, and in pages outside the pool."""
    d, before = 128, 40
    c = Caches(dtype, [[before + T]], 128, d, 16, 11)
    flat = c.pages[0, 0].long()

    def at(slot):
        return int(flat[slot // 16]), slot % 16
    for s in range(before + T, 128):                                        # behind the last entry
        c.k[at(s)] = float("nan")
        c.v[at(s)] = float("inf")
    q = torch.randn(1, T, G, d, generator=torch.Generator().manual_seed(12)).to(dtype)
    parents = [np.array([-1] + [0] * (T - 1), dtype=np.int32)]              # siblings: each sees row 0 and itself
    clean, clean_lse = check_attn(ctx, c, q, dtype, parents=parents)
    clean, clean_lse = clean.clone(), clean_lse.clone()
    for bad_k, bad_v in ((float("nan"), float("nan")), (float("inf"), -float("inf")), (1.0, float("inf"))):
        c.k[at(before + 3)] = bad_k
        c.v[at(before + 3)] = bad_v
        dv = c.dev()
        lse = torch.empty(1, G, T, device=DEV)
        out, _ = ctx.tree_attn(q.to(DEV), dv.k, dv.v, dv.len, mask=lv.tree_mask(torch.from_numpy(parents[0]))[None].to(DEV), pages=dv.pages,
                               row_lse=lse)
        torch.cuda.synchronize()
        others = [t for t in range(T) if t != 3]
        assert torch.equal(out[:, others], clean[:, others]) and torch.equal(lse[:, :, others], clean_lse[:, :, others])
        assert not bool(torch.isfinite(out[:, 3].float()).all())            # the row itself sees it
    c = Caches(dtype, [[60 + T]], 128, d, 16, 13)
    c.pages[0, 0, 1], c.pages[0, 0, 2] = -1, 10 ** 6                        # entries 16 .. 47 are nowhere
    check_attn(ctx, c, q, dtype, parents=parents)


@pytest.mark.parametrize("dtype,gain", [(BF, 40.0), (FP, 40.0), (BF, 0.0), (FP, 400.0)])
def test_far_and_equal_logits(ctx, dtype, gain):
    """Logits hundreds apart that grow along the entries (the running maximum moves), and all alike."""
    d, L, T = 64, 600, 3
    c = Caches(dtype, [[L]], L, d, 0, 17)
    c.k[0, 0] = (c.k[0, 0].float() * 0.01 + torch.linspace(0, 1, L)[:, None]).to(dtype)
    q = torch.full((1, T, 2, d), gain / d ** 0.5).to(dtype)
    check_attn(ctx, c, q, dtype)


def test_strided_queries_and_outputs(ctx):
    """q as a slice of a fused projection, out with another order of axes."""
    B, T, Hq, Hkv, d = 2, 6, 8, 2, 128
    c = Caches(BF, [[50, 20], [33, 6]], 64, d, 0, 19)
    fused = torch.randn(B, T, Hq + 4, d, generator=torch.Generator().manual_seed(20)).to(BF).to(DEV)
    store = torch.full((B, Hq, T, d), 7.0, dtype=BF, device=DEV)
    dv = c.dev()
    got, _ = ctx.tree_attn(fused[:, :, 2:2 + Hq], dv.k, dv.v, dv.len, out=store.transpose(1, 2))
    ref, _ = ctx.tree_attn(fused[:, :, 2:2 + Hq].contiguous(), dv.k, dv.v, dv.len)
    check_attn(ctx, c, fused[:, :, 2:2 + Hq].contiguous().cpu(), BF)
    torch.cuda.synchronize()
    assert torch.equal(store.transpose(1, 2), ref) and got.data_ptr() == store.data_ptr()


def test_one_row_is_decode_attention(ctx):
    """T = 1 over a head-major cache is lvlm_decode_attn without an append: fp32 to the roundings of both."""
    c = Caches(FP, [[700, 5], [64, 129]], 704, 64, 0, 23)
    q = torch.randn(2, 1, 8, 64, generator=torch.Generator().manual_seed(24)).to(DEV)
    dv = c.dev()
    out, _ = ctx.tree_attn(q, dv.k, dv.v, dv.len)
    ref = ctx.decode_attn(q[:, 0].contiguous(), None, None, dv.k, dv.v, None, None, None, dv.len)
    torch.cuda.synchronize()
    assert (out[:, 0] - ref).abs().max() <= 1e-5


# Shapes that take every way a call is cut: up to 4 (fp32), 32, 64, 128 and 256 rows to a workgroup, with the entries whole and in runs, over more
# steps than travel at a time.
LONG = [
    # dtype, B, T, Hq, Hkv, d, slots, page
    (BF, 33, 70, 8, 8, 64, 200, 0), (BF, 9, 130, 8, 1, 64, 4200, 0), (BF, 33, 40, 8, 8, 64, 200, 0), (BF, 5, 40, 14, 1, 64, 4200, 0),
    (BF, 33, 70, 14, 2, 64, 1100, 0), (BF, 33, 70, 14, 2, 64, 1024, 64), (BF, 9, 70, 14, 1, 64, 4200, 0), (BF, 9, 70, 14, 1, 64, 4096, 256),
    (BF, 33, 40, 8, 4, 128, 200, 0), (BF, 9, 130, 14, 1, 128, 2100, 0), (BF, 33, 11, 16, 4, 128, 1100, 0), (BF, 5, 40, 8, 8, 128, 4096, 16),
    (BF, 9, 500, 14, 1, 128, 600, 0), (BF, 9, 500, 14, 1, 128, 768, 32), (BF, 5, 1000, 2, 1, 128, 4200, 0), (BF, 9, 333, 16, 8, 128, 1100, 0),
    (FP, 9, 130, 14, 1, 64, 200, 0), (FP, 1, 1, 2, 1, 64, 1100, 0), (FP, 33, 11, 16, 4, 64, 200, 0), (FP, 1, 1, 2, 1, 64, 4200, 0),
    (FP, 33, 1, 8, 4, 64, 1024, 32), (FP, 33, 40, 8, 4, 128, 200, 0), (FP, 33, 40, 2, 1, 128, 608, 32), (FP, 33, 130, 2, 2, 128, 1100, 0),
    (FP, 1, 1, 8, 1, 64, 600, 0), (FP, 1, 1, 8, 1, 64, 4200, 0), (FP, 16, 1, 14, 2, 64, 1100, 0), (FP, 33, 1, 32, 4, 128, 200, 0),
    (FP, 1, 1, 8, 1, 128, 200, 0), (FP, 2, 4, 2, 2, 64, 200, 0), (FP, 3, 3, 4, 4, 64, 4096, 16), (FP, 2, 4, 3, 3, 128, 2048, 64),
    (FP, 5, 1, 4, 4, 128, 96, 0), (FP, 33, 2, 8, 8, 128, 1100, 0), (FP, 2, 1, 4, 4, 64, 37, 0),
]


def dense(c, q, n_rows, mask):
    """The formula in 64 bits with whole matrices, a head at a time on the GPU: out, lse, sum of p |v|; rows not in use are NaN."""
    B, T, Hq, d = q.shape
    H = c.len.shape[1]
    G = Hq // H
    out, weight = (torch.full((B, T, Hq, d), float("nan"), dtype=torch.float64, device=DEV) for _ in range(2))
    lse = torch.full((B, Hq, T), float("nan"), dtype=torch.float64, device=DEV)
    kf, vf = c.k.flatten(0, -2), c.v.flatten(0, -2)
    room = c.k.shape[2] if c.pages is None else c.pages.shape[2] * c.k.shape[1]
    for b in range(B):
        n = T if n_rows is None else n_rows[b]
        for g in range(H):
            L = int(c.len[b, g])
            s = torch.arange(L, device=DEV)
            rows = s + (b * H + g) * room if c.pages is None else c.pages[b, g, s // c.k.shape[1]].long() * c.k.shape[1] + s % c.k.shape[1]
            k, v = kf[rows].double(), vf[rows].double()
            sees = torch.ones(n, L, dtype=torch.bool, device=DEV)
            sees[:, L - n:] = torch.ones(n, n, device=DEV).tril().bool() if mask is None else mask[b, :n, :n]
            for h in range(g * G, g * G + G):
                z = (q[b, :n, h].double() @ k.t().contiguous() * d ** -0.5).masked_fill(~sees, float("-inf"))
                lse[b, h, :n] = torch.logsumexp(z, -1)
                p = torch.softmax(z, -1)
                out[b, :n, h], weight[b, :n, h] = p @ v, p @ v.abs()
    return out, lse, weight


def against_dense(ctx, c, q, dtype, n_rows, parents, clean=None, but=None):
    """One call against the formula (of the caches `clean`, without drafted row `but`, if given)."""
    B, T, Hq, d = q.shape
    words = mask = None
    if parents is not None:
        words = lv.tree_mask(torch.from_numpy(np.stack(parents))).to(DEV)
        mask = torch.from_numpy(np.stack([O.tree_mask(p) for p in parents])).to(DEV)
    rows = None if n_rows is None else torch.tensor(n_rows, dtype=torch.int32, device=DEV)
    out = torch.full((B, T, Hq, d), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((B, Hq, T), 7.0, device=DEV)
    ctx.tree_attn(q, c.k, c.v, c.len, mask=words, n_rows=rows, pages=c.pages, out=out, row_lse=lse)
    clean = clean or c
    ref, ref_lse, weight = dense(clean, q, n_rows, mask)
    if but is not None:
        assert not bool(torch.isfinite(out[:, but].float()).all())
        ref[:, but], ref_lse[:, :, but], out[:, but], lse[:, :, but] = float("nan"), float("nan"), 7.0, 7.0
    e = (d + 4) * U * float(q.abs().double().sum(-1).max() * clean.k.abs().max().double()) * d ** -0.5
    n = int(c.len.max())
    tol = weight * (2 * e + (n + 8) * U) + 1e-30
    if dtype == BF:
        tol = tol + 2.0 ** -8 * (weight + ref.abs())
    unused = torch.isnan(ref)
    assert bool((out[unused] == 7.0).all()) and bool((lse[torch.isnan(ref_lse)] == 7.0).all())
    off = ((out.double() - ref).abs() / tol)[~unused]
    assert bool((off <= 1.0).all()), float(off.max())
    off = ((lse.double() - ref_lse).abs() - (e + (n + 4) * U + 4 * U * ref_lse.abs()))[~torch.isnan(ref_lse)]
    assert bool((off <= 0.0).all()), float(off.max())
    return out, lse


@pytest.mark.parametrize("kind", ["chain", "tree"])
@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,d,slots,page", LONG)
def test_every_cut_matches_the_formula(ctx, dtype, B, T, Hq, Hkv, d, slots, page, kind):
    seed = B * T + slots
    r = np.random.default_rng(seed)
    n_rows = [T] + r.integers(1, T + 1, B - 1).tolist()
    most = slots - T
    lens = np.array(n_rows)[:, None] + np.where(r.random((B, Hkv)) < 0.5, most, r.integers(0, most + 1, (B, Hkv)))
    c = Caches(dtype, lens.tolist(), slots, d, page, seed).dev()
    q = torch.randn(B, T, Hq, d, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)
    parents = [tree_of(T, seed + b) for b in range(B)] if kind == "tree" else None
    against_dense(ctx, c, q, dtype, n_rows, parents)


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,d,slots,page", LONG)
def test_every_cut_survives_logits_that_grow_and_values_that_are_large(ctx, dtype, B, T, Hq, Hkv, d, slots, page):
    """Along the entries the logits rise by 300 (beyond any fixed reference), then by 40 with values near the end of the type, where
    sums relative to the first entries would overflow."""
    g = torch.Generator().manual_seed(slots)
    c = Caches(dtype, [[slots] * Hkv] * B, slots, d, page, slots).dev()
    rise = (torch.randn(slots, d, generator=g) * 0.01 + torch.linspace(0, 1, slots)[:, None]).to(dtype).to(DEV)
    s = torch.arange(slots, device=DEV)
    for b in range(B):
        for h in range(Hkv):
            if page:
                c.k[c.pages[b, h, s // page].long(), s % page] = rise
            else:
                c.k[b, h] = rise
    for gain, large in ((300.0, 1.0), (40.0, 1e30)):
        c.v.mul_(large)
        against_dense(ctx, c, torch.full((B, T, Hq, d), gain / d ** 0.5, device=DEV).to(dtype), dtype, None, None)


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,d,slots", [(BF, 16, 32, 32, 8, 128, 4096), (BF, 33, 4, 16, 8, 128, 8192), (FP, 9, 2, 8, 8, 64, 8192),
                                                       (BF, 3, 200, 8, 2, 128, 8192), (FP, 20, 9, 4, 4, 64, 2048)])
def test_runs_dealt_out_by_the_lengths(ctx, dtype, B, T, Hq, Hkv, d, slots):
    """Long calls share out what the heads hold: all of it, nothing, one long list among empty ones, anything between."""
    r = np.random.default_rng(B)
    q = torch.randn(B, T, Hq, d, generator=torch.Generator().manual_seed(T)).to(dtype).to(DEV)
    c = Caches(dtype, [[slots] * Hkv] * B, slots, d, 0, B).dev()
    for lens in (np.full((B, Hkv), slots), np.full((B, Hkv), T), np.where(np.arange(B * Hkv).reshape(B, Hkv) == B * Hkv // 2, slots, T),
                 np.where(r.random((B, Hkv)) < 0.1, slots - 7, T + 1), T + (r.random((B, Hkv)) ** 3 * (slots - T)).astype(int)):
        c.len = torch.from_numpy(lens.astype(np.int32)).to(DEV)
        against_dense(ctx, c, q, dtype, None, None)
    c.len = torch.zeros(B, Hkv, dtype=torch.int32, device=DEV)              # and nothing at all, but for one row in one head
    c.len[B // 2, Hkv // 2] = 1
    out, lse = ctx.tree_attn(q, c.k, c.v, c.len, want_lse=True)
    G, h = Hq // Hkv, Hkv // 2
    heads = slice(h * G, h * G + G)
    assert torch.equal(out[B // 2, T - 1, heads], c.v[B // 2, h, :1].expand(G, d))
    out[B // 2, T - 1, heads] = 0
    assert not bool(out.any()) and int(torch.isfinite(lse).sum()) == G


@pytest.mark.parametrize("dtype,T,Hq,d,slots", [(BF, 1000, 2, 128, 4200), (BF, 70, 14, 64, 4200), (FP, 40, 2, 128, 608), (BF, 130, 8, 64, 4200),
                                             (FP, 2, 2, 64, 4200), (FP, 4, 1, 128, 608), (FP, 3, 1, 64, 200)])
def test_no_cut_lets_in_what_a_row_does_not_see(ctx, dtype, T, Hq, d, slots):
    """NaN and infinities in the keys and values of one drafted row, and behind the last entry."""
    B = 9
    c = Caches(dtype, [[slots - 37]] * B, slots, d, 0, slots).dev()
    q = torch.randn(B, T, Hq, d, generator=torch.Generator().manual_seed(T)).to(dtype).to(DEV)
    parents = [np.array([-1] + [0] * (T - 1), dtype=np.int32)] * B           # siblings: each sees row 0 and itself
    clean = c.dev()
    clean.k, clean.v = c.k.clone(), c.v.clone()
    c.k[:, :, slots - 37:], c.v[:, :, slots - 37:] = float("nan"), float("inf")
    against_dense(ctx, c, q, dtype, None, parents, clean)
    at = slots - 37 - T + T // 2
    for bad_k, bad_v in ((float("nan"), float("nan")), (0.0, float("inf"))):
        c.k[:, :, at], c.v[:, :, at] = bad_k, bad_v
        against_dense(ctx, c, q, dtype, None, parents, clean, T // 2)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("L", [1, 40, 97, 256])
def test_an_infinite_value_gives_an_infinity_and_no_nan(ctx, dtype, L):
    """The last entry, seen by the one row and repeated in the rest of its tile."""
    c = Caches(dtype, [[L]], 256, 64, 0, L).dev()
    c.v[0, 0, L - 1, ::2] = float("inf")
    c.v[0, 0, L - 1, 1::4] = float("-inf")
    q = torch.randn(1, 1, 2, 64, generator=torch.Generator().manual_seed(L)).to(dtype).to(DEV)
    out, _ = ctx.tree_attn(q, c.k, c.v, c.len)
    assert bool((out[..., ::2] == float("inf")).all()) and bool((out[..., 1::4] == float("-inf")).all())
    assert bool(torch.isfinite(out[..., 3::4].float()).all())


# ---- append ---------------------------------------------------------------------------------------------------------


APPEND = [
    # dtype, B, T, Hq, Hkv, d, before, ragged, page, rot_dim, adjacent, sections, first position
    (FP, 1, 1, 4, 4, 64, 0, False, 0, 64, False, None, 0),
    (BF, 2, 1, 28, 4, 128, 300, True, 64, 128, False, (16, 24, 24), 2113),
    (BF, 3, 5, 8, 2, 128, 30, True, 16, 128, True, None, 40000),
    (FP, 2, 9, 6, 3, 128, 77, True, 32, 64, False, None, 1 << 24),          # half of the channels turn; far positions
    (BF, 1, 33, 4, 1, 64, 15, False, 16, 32, True, (4, 12), 7),
    (FP, 1, 40, 2, 2, 64, 3, True, 0, 16, False, None, (1 << 31) - 50),     # the last positions there are
    (BF, 2, 70, 0, 3, 128, 11, True, 128, 128, False, None, -35),           # no queries; positions below zero
    (BF, 1, 300, 5, 5, 64, 100, False, 256, 64, False, (0, 32, 0), 900000),
    (FP, 5, 17, 0, 2, 128, 8, True, 16, 0, False, None, 0),                 # nothing turns
]


def check_append(c, before, new, opts, got, dtype):
    """got: device caches after the call and (length_out, q_out), against the oracle."""
    ref = O.kv_append(f64(new[0]), f64(new[1]), f64(c.k), f64(c.v), before, pages=host(c.pages), score=host(c.score), kind=host(c.kind),
                      orig_pos=host(c.pos), **opts)
    dv, len_out, q_out = got
    assert np.array_equal(host(len_out), ref[5])
    assert np.array_equal(host(dv.kind), ref[3]) and np.array_equal(host(dv.pos), ref[4]) and np.array_equal(host(dv.score), ref[2])
    assert np.array_equal(f64(dv.v), ref[1])
    pos = np.abs(opts["pos"].astype(np.float64)).max() if opts.get("pos") is not None else 0.0
    step = 2.0 ** -8 if dtype == BF else U
    for x, y, src in ((dv.k, ref[0], new[0]),) + (((q_out, ref[6], opts["q"]),) if opts.get("q") is not None else ()):
        big = 2 * float(np.abs(f64(src) if torch.is_tensor(src) else src).max())
        assert np.all(np.abs(f64(x) - y) <= big * (2.0 ** -21 + pos * 2.0 ** -50) + step * np.abs(y))
    turned = opts.get("inv_freq") is not None
    if not turned:
        assert np.array_equal(f64(dv.k), ref[0])


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,d,before,ragged,page,rot,adjacent,sections,pos0", APPEND)
@pytest.mark.parametrize("in_place", [False, True])
def test_append_matches_the_oracle(ctx, dtype, B, T, Hq, Hkv, d, before, ragged, page, rot, adjacent, sections, pos0, in_place):
    seed = T * 100 + before
    r = np.random.default_rng(seed)
    c = Caches(dtype, lens_of(B, Hkv, before, ragged, seed), before + T + 3, d, page, seed)
    g = torch.Generator().manual_seed(seed + 1)
    fused = torch.randn(B, T, Hq + 2 * Hkv, d, generator=g).to(dtype)
    k, v = fused[:, :, Hq:Hq + Hkv], fused[:, :, Hq + Hkv:]
    fd = fused.to(DEV)
    n_new = r.integers(0, T + 1, B).astype(np.int32) if ragged else None
    kw, opts = {}, {"n_new": n_new}
    if rot:
        axes = len(sections) if sections else 1
        pos = (pos0 + r.integers(0, 50, (axes, B, T))).astype(np.int32)
        freq = (1e4 ** (-np.arange(rot // 2) / (rot // 2))).astype(np.float32)
        opts.update(pos=pos, inv_freq=freq.astype(np.float64), sections=sections, adjacent=adjacent)
        kw.update(pos=torch.from_numpy(pos if sections else pos[0]).to(DEV), inv_freq=torch.from_numpy(freq).to(DEV), sections=sections,
                  adjacent=adjacent)
    if Hq:
        q_out = torch.full((B, T, Hq, d), 7.0, dtype=dtype, device=DEV)
        opts.update(q=f64(fused[:, :, :Hq]), q_out=np.full((B, T, Hq, d), 7.0))
        if in_place:                                                        # the queries turn where they are
            q_out = fd[:, :, :Hq]
            opts["q_out"] = f64(fused[:, :, :Hq])
        kw.update(q=fd[:, :, :Hq], q_out=q_out)
    dv = c.dev()
    len_out, q_got = ctx.kv_append(fd[:, :, Hq:Hq + Hkv], fd[:, :, Hq + Hkv:], dv.k, dv.v, dv.len, pages=dv.pages, score=dv.score,
                                   kind=dv.kind, orig_pos=dv.pos, n_new=None if n_new is None else torch.from_numpy(n_new).to(DEV),
                                   length_out=dv.len if in_place else None, **kw)
    torch.cuda.synchronize()
    assert (len_out.data_ptr() == dv.len.data_ptr()) == in_place
    check_append(c, host(c.len), (k, v), opts, (dv, len_out, q_got), dtype)
    if not in_place:
        assert torch.equal(dv.len.cpu(), c.len)
    assert torch.equal(fd[:, :, Hq:].cpu(), fused[:, :, Hq:])               # the rows themselves stay


@pytest.mark.parametrize("in_place", [False, True])
def test_heads_that_are_full_and_pages_outside_the_pool(ctx, in_place):
    B, Hkv, d, T = 3, 2, 64, 40
    for page in (0, 16):
        c = Caches(BF, [[24, 25], [0, 64], [-1, 200]], 64, d, page, 31)
        if page:
            c.pages[0, 0, 2], c.pages[1, 0, 0] = -7, 10 ** 8
        new = torch.randn(2, B, T, Hkv, d, generator=torch.Generator().manual_seed(32)).to(BF)
        dv = c.dev()
        len_out, _ = ctx.kv_append(*new.to(DEV), dv.k, dv.v, dv.len, pages=dv.pages, score=dv.score, kind=dv.kind, orig_pos=dv.pos, new_kind=1,
                                   length_out=dv.len if in_place else None)
        torch.cuda.synchronize()
        check_append(c, host(c.len), new, {"new_kind": 1}, (dv, len_out, None), BF)
        assert len_out.tolist() == [[64, 25], [40, 64], [-1, 200]]


def test_append_of_nothing_copies_the_lengths(ctx):
    c = Caches(BF, [[3, 5]], 16, 64).dev()
    empty = torch.empty(1, 0, 2, 64, dtype=BF, device=DEV)
    out, _ = ctx.kv_append(empty, empty, c.k, c.v, c.len)
    assert torch.equal(out, c.len) and ctx.kv_append(empty, empty, c.k, c.v, c.len, length_out=c.len)[0] is c.len


@pytest.mark.parametrize("dtype,d,page", [(BF, 128, 64), (FP, 64, 16)])
def test_compressed_lists_go_into_pages_and_attend_alike(ctx, dtype, d, page):
    """The path of a compressed cache: kv_compress leaves every head a length of its own, kv_append packs the lists with their
    small arrays into pages, tree_attn reads either the same to the bit."""
    B, Hkv, G, N = 2, 3, 2, 200
    c = Caches(dtype, [[N] * Hkv] * B, N, d, 0, 41)
    c.score.copy_(torch.rand(c.score.shape, generator=torch.Generator().manual_seed(42)) ** 8)
    c.kind[:, :, 20:180] = lv.KIND_IMAGE
    dv = c.dev()
    ctx.kv_compress(dv.k, dv.v, dv.score, dv.kind, dv.pos, dv.len, mode=lv.KV_THRESHOLD, beta=0.9)
    p = Caches(dtype, [[0] * Hkv] * B, N, d, page, 43).dev()
    ctx.kv_append(dv.k.transpose(1, 2), dv.v.transpose(1, 2), p.k, p.v, p.len, n_new=dv.len, pages=p.pages, score=p.score, kind=p.kind,
                  orig_pos=p.pos, score_new=dv.score, kind_new=dv.kind, orig_new=dv.pos, length_out=p.len)
    q = torch.randn(B, 3, Hkv * G, d, device=DEV).to(dtype)
    a, _ = ctx.tree_attn(q, dv.k, dv.v, dv.len, len_bound=N)
    b, _ = ctx.tree_attn(q, p.k, p.v, p.len, pages=p.pages, len_bound=N)
    torch.cuda.synchronize()
    assert torch.equal(p.len, dv.len) and len(set(dv.len.flatten().tolist())) > 1
    for i in range(B):
        for g in range(Hkv):
            s = torch.arange(int(dv.len[i, g]), device=DEV)
            rows = p.pages[i, g, s // page].long() * page + s % page
            for x, y in ((dv.k, p.k), (dv.v, p.v), (dv.score, p.score), (dv.kind, p.kind), (dv.pos, p.pos)):
                assert torch.equal(x[i, g, :len(s)], y.flatten(0, 1)[rows])
    assert torch.equal(a, b)


# ---- commit ---------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,d,page", [(BF, 128, 0), (BF, 64, 16), (FP, 128, 32), (FP, 64, 0)])
def test_commit_matches_the_oracle(ctx, dtype, d, page, in_place):
    B, Hkv, P = 7, 2, 70
    lens = [[30, 7], [0, 0], [15, 16], [31, -2], [100, 128], [5, 90], [9, 11]]
    path = torch.zeros(B, P, dtype=torch.int32)
    r = np.random.default_rng(51)
    n_path = [12, 70, 1, 5, 60, 0, 99]
    for b, n in enumerate(n_path):
        m = min(n, P)
        path[b, :m] = torch.from_numpy(np.sort(r.choice(75 if m < 70 else 71, m, replace=False)).astype(np.int32))
    path[3, :5] = torch.tensor([0, 1, 2, 2, 9])             # stops ascending
    path[6, :3] = torch.tensor([2, -1, 5])                  # turns negative
    c = Caches(dtype, lens, 128, d, page, 52)
    if page:
        c.pages[0, 0, 2], c.pages[2, 1, 1] = -1, 10 ** 7
    dv = c.dev()
    out = ctx.tree_commit(dv.k, dv.v, dv.len, path.to(DEV), torch.tensor(n_path, dtype=torch.int32, device=DEV), pages=dv.pages,
                          score=dv.score, kind=dv.kind, orig_pos=dv.pos, length_out=dv.len if in_place else None)
    torch.cuda.synchronize()
    ref = O.tree_commit(f64(c.k), f64(c.v), host(c.len), path.numpy(), n_path, pages=host(c.pages), score=host(c.score), kind=host(c.kind),
                        orig_pos=host(c.pos))
    for x, y in zip((dv.k, dv.v, dv.score, dv.kind, dv.pos, out), ref):
        assert np.array_equal(host(x), y)


# ---- together -------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,page", [(FP, 16), (BF, 32), (BF, 0)])
def test_drafting_and_keeping_a_path_is_decoding_it_token_by_token(ctx, dtype, page):
    """append + tree attention + commit, captured into a graph and replayed over three rounds, against appending the accepted
    tokens one at a time: the caches are equal to the bit, and so are the rows of the accepted path to the roundings."""
    B, T, Hq, Hkv, d = 2, 6, 4, 2, 64
    parent = np.array([[-1, 0, 0, 1, 2, 3], [-1, 0, 1, 0, 3, 3]], dtype=np.int32)
    depth = np.array([[0, 1, 1, 2, 2, 3], [0, 1, 2, 1, 2, 2]])
    accepted = np.array([[0, 2, 4], [0, 3, 5]], dtype=np.int32)
    n_path = torch.tensor([3, 2], dtype=torch.int32, device=DEV)
    words, path = lv.tree_mask(torch.from_numpy(parent)).to(DEV), torch.from_numpy(accepted).to(DEV)
    freq = torch.from_numpy((1e4 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)).to(DEV)
    a = Caches(dtype, [[20, 33], [7, 0]], 96, d, page, 61).dev()
    b = Caches(dtype, [[20, 33], [7, 0]], 96, d, page, 61).dev()
    draft_len = torch.zeros_like(a.len)
    k, v = (torch.zeros(B, T, Hkv, d, dtype=dtype, device=DEV) for _ in range(2))
    q, turned, out = (torch.zeros(B, T, Hq, d, dtype=dtype, device=DEV) for _ in range(3))
    pos = torch.zeros(B, T, dtype=torch.int32, device=DEV)
    small = lambda c: dict(pages=c.pages, score=c.score, kind=c.kind, orig_pos=c.pos)       # noqa: E731

    def step():
        ctx.kv_append(k, v, a.k, a.v, a.len, pos=pos, inv_freq=freq, q=q, q_out=turned, length_out=draft_len, **small(a))
        ctx.tree_attn(turned, a.k, a.v, draft_len, mask=words, pages=a.pages, out=out, reserve=False)
        ctx.tree_commit(a.k, a.v, a.len, path, n_path, length_out=a.len, **small(a))

    ctx.reserve(1 << 24)
    keep = [x.clone() for x in (a.k, a.v, a.score, a.kind, a.pos, a.len)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, y in zip((a.k, a.v, a.score, a.kind, a.pos, a.len), keep):
        x.copy_(y)
    g = torch.Generator().manual_seed(62)
    base = 50
    for rnd in range(3):
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, generator=g).to(dtype))
        pos.copy_(torch.from_numpy((base + depth).astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        n = n_path.tolist()
        for i in range(3):                                                  # the other way: one accepted token at a time
            one = torch.tensor([1 if i < n[x] else 0 for x in range(B)], dtype=torch.int32, device=DEV)
            pick = torch.from_numpy(accepted[:, i]).long().to(DEV)
            at = torch.arange(B, device=DEV)
            row = [x[at, pick].unsqueeze(1) for x in (k, v, q, pos.unsqueeze(-1))]
            _, qt = ctx.kv_append(row[0], row[1], b.k, b.v, b.len, pos=row[3].squeeze(-1).contiguous(), inv_freq=freq, q=row[2], n_new=one,
                                  length_out=b.len, **small(b))
            ref, _ = ctx.tree_attn(qt, b.k, b.v, b.len, n_rows=one, pages=b.pages)
            torch.cuda.synchronize()
            for x in range(B):
                if i < n[x]:
                    diff = (out[x, accepted[x, i]].double() - ref[x, 0].double()).abs().max()
                    assert diff <= (2e-5 if dtype == FP else 4 * 2.0 ** -8), (rnd, i, x)
        assert torch.equal(a.len, b.len)
        for x in range(B):
            for h in range(Hkv):
                s = torch.arange(int(a.len[x, h]), device=DEV)
                for c1, c2 in ((a.k, b.k), (a.v, b.v), (a.kind, b.kind), (a.pos, b.pos), (a.score, b.score)):
                    rows = (a.pages[x, h, s // page].long() * page + s % page) if page else s + (x * Hkv + h) * 96
                    f1, f2 = ((y.reshape(-1, d) if y.shape[-1] == d and y.dim() == (3 if page else 4) else y.reshape(-1)) for y in (c1, c2))
                    assert torch.equal(f1[rows], f2[rows])
        base += 3


def test_two_graphs_share_a_workspace_and_follow_the_lengths(ctx):
    """Two captured calls, one of runs dealt out by the lengths and one of runs by the slots, replayed in turn while the lengths and
    the queries change, against eager calls."""
    long, short = (Caches(BF, [[4096] * 8] * 16, 4096, 128, 0, 73).dev(), Caches(BF, [[5000] * 2], 5000, 128, 0, 74).dev())
    q = [torch.zeros(16, 32, 32, 128, dtype=BF, device=DEV), torch.zeros(1, 3, 8, 128, dtype=BF, device=DEV)]
    out = [torch.zeros_like(x) for x in q]
    ctx.reserve(1 << 27)

    def call(i, o, **kw):
        c = (long, short)[i]
        return ctx.tree_attn(q[i], c.k, c.v, c.len, out=o, **kw)[0]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(0, out[0], reserve=False)
        call(1, out[1], reserve=False)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in q]
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            call(i, out[i], reserve=False)
    r = torch.Generator().manual_seed(75)
    for rnd in range(4):
        for x in q:
            x.copy_(torch.randn(x.shape, generator=r).to(BF))
        long.len.copy_((torch.rand(long.len.shape, generator=r) ** (1 + 2 * rnd) * 4064).to(torch.int32) + 32)
        short.len.copy_(torch.tensor([[5000 - 700 * rnd, 3 + rnd]], dtype=torch.int32))
        for g in (graphs if rnd % 2 else graphs[::-1]):
            g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(out[i], call(i, torch.empty_like(out[i]))), (rnd, i)
        torch.cuda.synchronize()


def test_another_stream_and_two_calls_in_a_row(ctx):
    """Calls on a stream of their own, back to back with one workspace, give what they give alone."""
    c = Caches(BF, [[900, 1200]], 1210, 128, 0, 71).dev()
    qs = [torch.randn(1, t, 8, 128, generator=torch.Generator().manual_seed(t)).to(BF).to(DEV) for t in (4, 60)]
    ref = [ctx.tree_attn(q, c.k, c.v, c.len)[0] for q in qs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [ctx.tree_attn(q, c.k, c.v, c.len)[0] for q in qs + qs]
    side.synchronize()
    for i, x in enumerate(got):
        assert torch.equal(x, ref[i % 2])


def test_entries_past_four_gigabytes(ctx):
    """A pool whose rows lie more than 2^32 bytes in: offsets are 64 bits."""
    d, page = 128, 65536
    n_pages = (5 << 30) // (page * d * 2)
    k = torch.zeros(n_pages, page, d, dtype=BF, device=DEV)
    v = torch.zeros(n_pages, page, d, dtype=BF, device=DEV)
    pages = torch.tensor([[[n_pages - 1]]], dtype=torch.int32, device=DEV)
    small = Caches(BF, [[100]], 128, d, 0, 81)
    length = torch.zeros(1, 1, dtype=torch.int32, device=DEV)
    s = small.dev()
    ctx.kv_append(s.k[:, :, :100].transpose(1, 2), s.v[:, :, :100].transpose(1, 2), k, v, length, pages=pages, length_out=length)
    q = torch.randn(1, 2, 4, d, generator=torch.Generator().manual_seed(82)).to(BF)
    big, _ = ctx.tree_attn(q.to(DEV), k, v, length, pages=pages, len_bound=128)
    ref, _ = check_attn(ctx, small, q, BF)
    torch.cuda.synchronize()
    assert torch.equal(big, ref) and torch.equal(k[n_pages - 1, :100], s.k[0, 0, :100]) and not bool(k[:n_pages - 1].any())
