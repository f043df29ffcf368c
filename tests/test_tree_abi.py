"""Refusals of the drafted-token calls, reported on the host before anything is launched (no GPU needed): the pointers
below are numbers that nothing reads."""
import ctypes as C

import pytest
import torch

import paper_2509_00419_amd as lv
from paper_2509_00419_amd import binding as bd

K, V, NEW, NEWV, Q, QO, POS, FREQ, LEN, LEN2, TAB, MASK = (x << 32 for x in range(1, 13))


def _cache(**kw):
    c = bd.Cache(K, V, None, None, None, None, 256, 0, 0, 0)
    for name, x in kw.items():
        setattr(c, name, x)
    return c


def _append(desc=(), src=(), cache=(), length=(LEN, LEN2)):
    d = bd.AppendDesc(bd.BF16, 2, 5, 8, 4, 128, 128, 0, 1, (C.c_int32 * 3)(64, 0, 0), 2, 0, 2560, 512, 128, 2560, 512, 128,
                      5120, 1024, 128, 5120, 1024, 128, 0, 0, 0, 0)
    s = bd.AppendSrc(NEW, NEWV, Q, QO, POS, FREQ, None, None, None, None)
    c = _cache()
    for obj, changes in ((d, desc), (s, src), (c, cache)):
        for name, x in dict(changes).items():
            setattr(obj, name, (C.c_int32 * 3)(*x) if name == "sections" else x)
    ctx = lv.Context(0)
    st = bd.lib.lvlm_kv_append(ctx._h, None, C.byref(d), C.byref(s), C.byref(c), *length)
    return st, bd.lib.lvlm_last_error(ctx._h).decode()


@pytest.mark.parametrize("kw,word", [
    (dict(desc={"dtype": 2}), "dtype"), (dict(desc={"hd": 96}), "head dimension"), (dict(desc={"B": 0}), "positive"),
    (dict(desc={"T": -1}), "positive"), (dict(desc={"Hkv": 0}), "positive"), (dict(desc={"Hq": 0}), "positive"),
    (dict(desc={"B": 65536}), "limits"), (dict(desc={"T": 1 << 23}), "limits"), (dict(desc={"Hkv": 1025}), "limits"),
    (dict(desc={"rot_dim": 24}), "rot_dim"), (dict(desc={"rot_dim": 144}), "rot_dim"), (dict(desc={"rot_dim": -16}), "rot_dim"),
    (dict(desc={"adjacent": 2}), "adjacent"), (dict(desc={"new_kind": 256}), "new_kind"), (dict(desc={"reserved": 1}), "reserved"),
    (dict(desc={"n_axes": 0}), "n_axes"), (dict(desc={"n_axes": 4}), "n_axes"), (dict(desc={"sections": (63, 0, 0)}), "sections"),
    (dict(desc={"n_axes": 2, "sections": (70, -6, 0)}), "sections"), (dict(src={"pos": None}), "pos"),
    (dict(src={"inv_freq": None}), "inv_freq"), (dict(src={"k": None}), "null"), (dict(src={"q_out": None}), "together"),
    (dict(desc={"rot_dim": 0}), "turned"), (dict(desc={"n_stride_h": 1}, src={"n_new": LEN}), "per sequence"),
    (dict(src={"k": NEW + 8}), "aligned"), (dict(src={"pos": POS + 2}), "aligned"), (dict(desc={"k_stride_t": 516}), "multiples"),
    (dict(desc={"v_stride_h": -128}), "multiples"), (dict(desc={"qo_stride_t": 512}), "overlap"),
    (dict(desc={"k_stride_b": 1 << 37}), "2^36"), (dict(desc={"m_stride_b": 1 << 37}), "2^36"), (dict(desc={"m_stride_b": -1}), "negative"),
    (dict(src={"k": K + 4096}), "overlap"), (dict(src={"q_out": Q + 256}), "overlaps q"), (dict(src={"q_out": V}), "overlaps the cache"),
    (dict(cache={"v": K + 256}), "overlap"), (dict(cache={"k": None}), "null"), (dict(cache={"score": 4098}), "aligned"),
    (dict(cache={"Lmax": 0}), "positive"), (dict(cache={"Lmax": (1 << 24) + 1}), "limits"), (dict(cache={"reserved": 1}), "reserved"),
    (dict(cache={"page_size": 16}), "need pages"), (dict(cache={"pages": TAB, "page_size": 48, "n_pages": 1}), "power of two"),
    (dict(cache={"pages": TAB, "page_size": 8, "n_pages": 1}), "power of two"),
    (dict(cache={"pages": TAB, "page_size": 0, "n_pages": 1}), "power of two"),
    (dict(cache={"pages": TAB, "page_size": 512, "n_pages": 1}), "multiple of page_size"),
    (dict(cache={"pages": TAB, "page_size": 64, "n_pages": 0}), "n_pages"),
    (dict(src={"n_new": LEN2}), "len_out overlaps n_new"), (dict(src={"pos": LEN2 + 8}), "len_out overlaps n_new or pos"),
    (dict(src={"orig_pos": 1 << 20}, cache={"orig_pos": (1 << 20) + 16}), "overlaps the cache's"),
    (dict(src={"kind": 1 << 20}, cache={"kind": 1 << 20}), "overlaps the cache's"),
    (dict(length=(None, LEN2)), "null"), (dict(length=(LEN, LEN + 4)), "overlaps len"), (dict(length=(LEN, LEN2 + 2)), "aligned"),
])
def test_append_refuses(kw, word):
    st, why = _append(**kw)
    assert st == 1 and word in why and why.startswith("kv_append: "), (st, why)


def test_an_append_of_nothing_in_place_launches_nothing():
    assert _append(desc={"T": 0}, src={"k": None, "v": None}, length=(LEN, LEN))[0] == 0


def _tree(desc=(), cache=(), q=Q, out=QO, length=LEN, n_rows=None, mask=MASK, lse=None):
    d = bd.TreeDesc(bd.BF16, 2, 5, 8, 4, 128, 256, 0, 0.09, 0, 5120, 1024, 128, 5120, 1024, 128)
    c = _cache()
    for obj, changes in ((d, desc), (c, cache)):
        for name, x in dict(changes).items():
            setattr(obj, name, x)
    ctx = lv.Context(0)
    st = bd.lib.lvlm_tree_attn(ctx._h, None, C.byref(d), q, C.byref(c), length, n_rows, mask, out, lse)
    return st, bd.lib.lvlm_last_error(ctx._h).decode()


@pytest.mark.parametrize("kw,word", [
    (dict(desc={"dtype": 2}), "dtype"), (dict(desc={"hd": 32}), "head dimension"), (dict(desc={"T": 0}), "T must"),
    (dict(desc={"T": 1025}), "T must"), (dict(desc={"Hq": 6}), "multiple of Hkv"), (dict(desc={"B": 65536}), "limits"),
    (dict(desc={"Hq": 1028}), "limits"), (dict(desc={"T": 1024, "Hq": 1024, "Hkv": 1}), "65536"),
    (dict(desc={"len_bound": 257}), "len_bound"), (dict(desc={"len_bound": -1}), "len_bound"), (dict(desc={"scale": 0.0}), "scale"),
    (dict(desc={"scale": float("nan")}), "scale"), (dict(desc={"scale": float("inf")}), "scale"), (dict(desc={"reserved": 3}), "reserved"),
    (dict(desc={"q_stride_t": 1023}), "multiples"), (dict(desc={"o_stride_h": 64}), "overlap"), (dict(desc={"o_stride_t": 0}), "overlap"),
    (dict(desc={"Lmax": 128}), "differ"), (dict(q=None), "null"), (dict(out=None), "null"), (dict(length=None), "null"),
    (dict(q=Q + 4), "aligned"), (dict(length=LEN + 1), "aligned"), (dict(mask=MASK + 2), "aligned"), (dict(out=Q + 1024), "overlap"),
    (dict(out=V + 1024), "overlap"), (dict(cache={"v": None}), "null"), (dict(lse=QO + 64), "row_lse overlaps"), (dict(lse=K), "row_lse overlaps"),
    (dict(cache={"pages": TAB, "page_size": 24, "n_pages": 3}), "power of two"),
])
def test_tree_attention_refuses(kw, word):
    st, why = _tree(**kw)
    assert st == 1 and word in why, (st, why)


def test_tree_attention_names_the_workspace_it_lacks():
    st, why = _tree(desc={"Lmax": 8192}, cache={"Lmax": 8192})      # (few rows over long lists: runs, whose sums lie there)
    assert st == 3 and "workspace" in why, (st, why)


@pytest.mark.parametrize("kw,word", [
    (dict(hd=96), "head dimension"), (dict(dtype=2), "dtype"), (dict(B=0), "positive"), (dict(Hkv=2000), "limits"), (dict(P=0), "P must"),
    (dict(P=65537), "P must"), (dict(B=8192, Hkv=1024), "2^23"), (dict(reserved=1), "reserved"), (dict(path=None), "null"), (dict(path=TAB + 1), "aligned"),
    (dict(len_out=None), "null"), (dict(len_out=LEN + 8), "overlaps len"), (dict(path=LEN2 + 16), "overlaps path"), (dict(len_out=MASK), "overlaps path or n_path"),
    (dict(cache={"k": None}), "null"),
])
def test_commit_refuses(kw, word):
    kw = dict(kw)
    path, len_out, cache = kw.pop("path", TAB), kw.pop("len_out", LEN2), _cache(**kw.pop("cache", {}))
    d = bd.CommitDesc(bd.BF16, 2, 4, 128, 5, 0)
    for name, x in kw.items():
        setattr(d, name, x)
    ctx = lv.Context(0)
    st = bd.lib.lvlm_tree_commit(ctx._h, None, C.byref(d), C.byref(cache), LEN, path, MASK, len_out)
    assert st == 1 and word in bd.lib.lvlm_last_error(ctx._h).decode()


def test_struct_sizes_match_the_header_layout():
    assert C.sizeof(bd.Cache) == 6 * 8 + 4 * 4
    assert C.sizeof(bd.AppendDesc) == 14 * 4 + 16 * 8
    assert C.sizeof(bd.AppendSrc) == 10 * 8
    assert C.sizeof(bd.TreeDesc) == 10 * 4 + 6 * 8
    assert C.sizeof(bd.CommitDesc) == 6 * 4


def _tree_ws(dtype, B, T, Hq, Hkv, Lmax, hd=128):
    return lv.Context(0).workspace_bytes(bd.OP_TREE_ATTN, bd.TreeDesc(dtype, B, T, Hq, Hkv, hd, Lmax, 0, 0.1, 0, T * Hq * hd, Hq * hd, hd,
                                                                      T * Hq * hd, Hq * hd, hd))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [bd.BF16, bd.F32])
def test_workspace_query_answers_at_the_limits_and_refuses_beyond(dtype, hd):
    for B, T, Hq, Hkv, Lmax in ((1, 1, 1, 1, 1), (1, 1024, 63, 1, 1 << 24), (65535, 1, 64, 64, 1 << 24), (8191, 1, 1024, 1024, 1 << 24),
                                (1023, 1024, 1024, 1024, 1 << 24), (65535, 128, 64, 2, 1 << 24)):
        assert _tree_ws(dtype, B, T, Hq, Hkv, Lmax, hd) >= 0
    assert _tree_ws(dtype, 65535, 1, 2, 2, 1 << 24, hd) == 0     # (more lists than the launch that folds takes: one run each)
    for B, T, Hq, Hkv, Lmax, word in ((65535, 1024, 1024, 1024, 1 << 24, "2\\^31"), (8192, 1, 1024, 1024, 1, "2\\^23"),
                                      (65535, 1, 1024, 256, 64, "2\\^23"), (1, 1, 1, 1, 1 << 25, "limits")):
        with pytest.raises(lv.LvlmError, match=word):
            _tree_ws(dtype, B, T, Hq, Hkv, Lmax, hd)


def test_tensors_of_another_device_type_or_layout_are_refused():
    """The torch side, on host tensors: nothing but the first check of each call can be reached without a GPU."""
    ctx = lv.Context(0)
    x = torch.zeros(1, 1, 4, 64)
    n = torch.zeros(1, 4, dtype=torch.int32)
    for call in (lambda: ctx.kv_append(x, x, x.transpose(1, 2), x.transpose(1, 2), n), lambda: ctx.tree_attn(x, x, x, n),
                 lambda: ctx.tree_commit(x, x, n, n, n[:, 0])):
        with pytest.raises(AssertionError, match="context's device"):
            call()
    for call in (lambda: ctx.kv_append(None, x, x, x, n), lambda: ctx.tree_attn(x, x, x), lambda: ctx.tree_commit(x, x, n, n, n, 1),
                 lambda: ctx.tree_attn(x, x, x, n, nonsense=1)):
        with pytest.raises(TypeError):
            call()
