"""Which memory the drafted-token calls may be given: what they refuse as overlapping, and what they must not refuse (no GPU needed).
The pointers are numbers that nothing reads.  A call that passes its checks goes to a device that does not exist and ends there: nothing is launched, with a GPU or without."""
import pytest

import paper_2509_00419_amd as lv
import test_tree_abi as abi
from test_tree_abi import FREQ, K, LEN, LEN2, MASK, NEW, NEWV, POS, Q, QO, TAB, V

NOWHERE = 99        # a device that no machine has


@pytest.fixture(autouse=True)
def no_device(monkeypatch):
    context = lv.Context
    monkeypatch.setattr(abi.lv, "Context", lambda device: context(NOWHERE))


def passes(result):
    st, why = result
    return st == 4 and "hipSetDevice(%d)" % NOWHERE in why


PLAIN = {"q": None, "q_out": None, "inv_freq": None}      # nothing turns


def test_the_calls_these_tests_change_pass():
    assert passes(abi._append()) and passes(abi._tree()) and passes(abi._append(desc={"rot_dim": 0}, src={**PLAIN, "pos": None}))


@pytest.mark.parametrize("n_axes", [-1, 0, 1, 3, 1 << 30])
def test_axes_are_not_read_where_nothing_turns(n_axes):
    desc = {"rot_dim": 0, "n_axes": n_axes}
    assert passes(abi._append(desc=desc, src={**PLAIN, "pos": None}))
    # positions given for the entries' sake: those of axis 0, whatever n_axes says
    assert passes(abi._append(desc=desc, src=PLAIN))
    st, why = abi._append(desc=desc, src={**PLAIN, "pos": LEN2 - 36})
    assert st == 1 and "len_out overlaps n_new or pos" in why
    assert passes(abi._append(desc=desc, src={**PLAIN, "pos": LEN2 - 40}))      # [2, 5] positions end where the lengths begin


def test_strides_of_counts_that_are_not_given_make_no_range():
    assert passes(abi._append(desc={"n_stride_b": 1 << 36, "n_stride_h": 1 << 36}))
    st, why = abi._append(desc={"n_stride_b": 1}, src={"n_new": LEN2 - 4})
    assert st == 1 and "len_out overlaps n_new" in why
    assert passes(abi._append(desc={"n_stride_b": 1}, src={"n_new": LEN2 - 8}))


def test_no_new_rows_read_nothing():
    """T = 0: positions and rows of such a call have no elements, and torch gives arrays without elements no address."""
    nothing = {"k": None, "v": None, "q": None, "q_out": None, "pos": None}
    assert abi._append(desc={"T": 0}, src=nothing, length=(LEN, LEN)) == (0, "")
    assert passes(abi._append(desc={"T": 0}, src=nothing))
    assert passes(abi._append(desc={"T": 0}, src={"k": K + 4096, "v": V, "q": K, "q_out": V}))
    assert passes(abi._append(desc={"T": 0}, src={"pos": LEN2}))
    for missing in ("pos", "inv_freq"):
        st, why = abi._append(src={missing: None})
        assert st == 1 and "pos and inv_freq" in why


# ---- outputs over what the call reads, or over each other ------------------------------------------------------------

SCORE, KIND, ORIG, NEW_SCORE, NEW_KIND, NEW_ORIG, COUNTS, PATH, N_PATH, LSE = (x << 32 for x in range(20, 30))
APPEND_READS = {"k": NEW, "v": NEWV, "q": Q, "pos": POS, "inv_freq": FREQ, "n_new": COUNTS, "score": NEW_SCORE, "kind": NEW_KIND, "orig_pos": NEW_ORIG}
CACHE = {"k": K, "v": V, "score": SCORE, "kind": KIND, "orig_pos": ORIG, "pages": TAB, "page_size": 64, "n_pages": 32}


def append(src=(), cache=(), length=(LEN, LEN2)):
    return abi._append(desc={"n_stride_b": 1, "m_stride_b": 20, "m_stride_h": 5}, src={**APPEND_READS, "q_out": QO, **dict(src)},
                       cache={**CACHE, **dict(cache)}, length=length)


def refused(result):
    st, why = result
    return st == 1 and "overlap" in why


def test_append_with_everything_given_passes():
    assert passes(append()) and passes(append(length=(LEN, LEN))) and passes(append(src={"q_out": Q}))


@pytest.mark.parametrize("read", [*APPEND_READS, "len", "pages"])
@pytest.mark.parametrize("written", ["k", "v", "score", "kind", "orig_pos", "q_out", "len_out"])
def test_append_refuses_an_output_over_what_it_reads(written, read):
    if (written, read) in (("q_out", "q"), ("len_out", "len")):
        pytest.skip("may be the same")
    at = LEN if read == "len" else TAB if read == "pages" else APPEND_READS[read]
    if written == "q_out":
        assert refused(append(src={"q_out": at}))
    elif written == "len_out":
        assert refused(append(length=(LEN, at)))
    else:
        assert refused(append(cache={written: at}))


@pytest.mark.parametrize("a,b", [(a, b) for i, a in enumerate(("k", "v", "score", "kind", "orig_pos")) for b in ("k", "v", "score", "kind", "orig_pos")[:i]])
def test_a_cache_of_arrays_that_overlap_is_refused(a, b):
    assert refused(append(cache={a: CACHE[b]}))
    assert refused(commit(cache={a: CACHE[b]}))


@pytest.mark.parametrize("a", ["k", "v", "score", "kind", "orig_pos"])
def test_queries_and_lengths_over_the_cache_are_refused(a):
    assert refused(append(src={"q_out": CACHE[a]})) and refused(append(length=(LEN, CACHE[a]))) and refused(commit(len_out=CACHE[a]))
    assert refused(append(length=(LEN, QO)))


def test_slices_of_one_buffer_do_not_overlap():
    """Rows of 1024 elements for q and 512 each for k and v, one after the other in a buffer: the ranges reach into each other, the rows do not."""
    row = 1024 + 512 + 512
    strides = {f"{x}_stride_{a}": n for x in ("q", "k", "v") for a, n in (("b", 5 * row), ("t", row))}
    qo = {"qo_stride_b": 5 * row, "qo_stride_t": row}
    src = {"q": Q, "k": Q + 2 * 1024, "v": Q + 2 * 1536}
    assert passes(abi._append(desc={**strides, **qo}, src={**src, "q_out": Q}))
    assert refused(abi._append(desc={**strides, **qo}, src={**src, "q_out": Q + 2 * 128}))            # reaches into k's rows
    assert refused(abi._append(desc={**strides, **qo}, src={**src, "q_out": Q + 2 * 1024}))
    # q turned into a slice of its own behind v's
    wide = {f"{x}_stride_{a}": n for x in ("q", "qo", "k", "v") for a, n in (("b", 5 * (row + 1024)), ("t", row + 1024))}
    assert passes(abi._append(desc=wide, src={**src, "q_out": Q + 2 * row}))
    assert refused(abi._append(desc=wide, src={**src, "q_out": Q + 2 * (row - 8)}))
    assert refused(abi._append(desc=wide, src={**src, "q_out": Q + 2 * (row + 8)}))                   # ... into the next row's q
    # heads before tokens, [B, heads, T, d]: the sequences' steps are what is left
    heads = {f"{x}_stride_{a}": n for x in ("q", "qo") for a, n in (("b", 16 * 5 * 128), ("t", 128), ("h", 5 * 128))}
    assert passes(abi._append(desc=heads, src={"q_out": Q + 2 * 8 * 5 * 128}))
    assert refused(abi._append(desc=heads, src={"q_out": Q + 2 * 7 * 5 * 128}))
    # the same for attention
    both = {f"{x}_stride_{a}": n for x in ("q", "o") for a, n in (("b", 5 * row), ("t", row))}
    assert passes(abi._tree(desc=both, out=Q + 2 * 1024)) and refused(abi._tree(desc=both, out=Q + 2 * 1016))


@pytest.mark.parametrize("read", [Q, K, V, LEN, COUNTS, MASK, TAB])
def test_attention_refuses_an_output_over_what_it_reads(read):
    pages = {"pages": TAB, "page_size": 64, "n_pages": 32}
    assert passes(abi._tree(cache=pages, n_rows=COUNTS, lse=LSE))
    assert refused(abi._tree(cache=pages, n_rows=COUNTS, lse=LSE, out=read)) and refused(abi._tree(cache=pages, n_rows=COUNTS, lse=read))


def commit(cache=(), path=PATH, n_path=N_PATH, length=LEN, len_out=LEN2):
    d = abi.bd.CommitDesc(abi.bd.BF16, 2, 4, 128, 5, 0)
    ctx, c = lv.Context(NOWHERE), abi._cache(**{**CACHE, **dict(cache)})
    st = abi.bd.lib.lvlm_tree_commit(ctx._h, None, abi.C.byref(d), abi.C.byref(c), length, path, n_path, len_out)
    return st, abi.bd.lib.lvlm_last_error(ctx._h).decode()


@pytest.mark.parametrize("read", [LEN, PATH, N_PATH, TAB])
@pytest.mark.parametrize("written", ["k", "v", "score", "kind", "orig_pos", "len_out"])
def test_commit_refuses_an_output_over_what_it_reads(written, read):
    assert passes(commit()) and passes(commit(len_out=LEN))
    if written == "len_out":
        assert read == LEN or refused(commit(len_out=read))
    else:
        assert refused(commit(cache={written: read})) and refused(commit(cache={written: read}, len_out=LEN))


def test_sizes_and_strides_at_their_limits():
    """Ranges of 2^60 bytes: whatever is said of them is said without overflow."""
    most = 1 << 36
    strides = {f"{x}_stride_{a}": most for x in ("k", "v", "q", "qo") for a in "bth"}
    small = {"n_stride_b": most, "n_stride_h": 0, "m_stride_b": most, "m_stride_h": most}
    for B, T, H in ((65535, 1 << 22, 1024), (1, 1 << 22, 1), (65535, 1, 1)):
        st, why = abi._append(desc={"B": B, "T": T, "Hq": H, "Hkv": H, **strides, **small}, src={"n_new": COUNTS, "kind": NEW_KIND},
                              cache={**CACHE, "Lmax": 1 << 24, "page_size": 65536, "n_pages": (1 << 31) - 1})
        assert st == 1 and "overlap" in why
    tree = {f"{x}_stride_{a}": most for x in "qo" for a in "bth"}
    assert refused(abi._tree(desc={"B": 65535, "T": 128, "Hq": 64, "Hkv": 2, **tree}))


@pytest.mark.parametrize("where", ["heads", "tokens", "sequences", "heads before tokens", "tokens before sequences"])
def test_parts_of_any_axis_do_not_overlap(where):
    """q, k and v of as many heads in one buffer, one part after the other along an axis; q turned in place, or into a fourth part."""
    B, T, H, d = 2, 5, 4, 128
    order = {"heads": "bth", "tokens": "bth", "sequences": "bth", "heads before tokens": "bht", "tokens before sequences": "tbh"}[where]
    axis = {"heads": 3, "tokens": 2, "sequences": 0, "heads before tokens": 1, "tokens before sequences": 2}[where]
    sizes = [{"b": B, "t": T, "h": H}[a] for a in order] + [d]
    sizes.insert(axis, 4)                                               # q, k, v and q_out: a place of the parts' own among the axes
    stride = [1] * 5
    for i in range(3, -1, -1):
        stride[i] = stride[i + 1] * sizes[i + 1]
    part, stride = stride[axis], stride[:axis] + stride[axis + 1:]
    step = {a: stride[order.index(a)] for a in "bth"}
    desc = {f"{x}_stride_{a}": step[a] for x in ("q", "k", "v", "qo") for a in "bth"}
    src = {"q": Q, "k": Q + 2 * part, "v": Q + 4 * part}
    for at in range(4):
        got = abi._append(desc={"Hq": H, **desc}, src={**src, "q_out": Q + 2 * at * part})
        assert passes(got) if at in (0, 3) else refused(got), (at, got)
        if at and part > 8:
            got = abi._append(desc={"Hq": H, **desc}, src={**src, "q_out": Q + 2 * (at * part - 8)})
            assert refused(got), (at, got)
    tree = {f"{x}_stride_{a}": step[a] for x in "qo" for a in "bth"}
    assert passes(abi._tree(desc={"Hq": H, **tree}, out=Q + 2 * part)) and refused(abi._tree(desc={"Hq": H, **tree}, out=Q + 2 * (part - 8)))
