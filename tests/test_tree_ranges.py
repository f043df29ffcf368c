"""Which memory the drafted-token calls may be given: what they refuse as overlapping, and what they must not refuse (no GPU needed).
The pointers are numbers that nothing reads.  A call that passes its checks goes to a device that does not exist and ends there: nothing is launched, with a GPU or without."""
import pytest

import paper_2509_00419_amd as lv
import test_tree_abi as abi
from test_tree_abi import K, LEN, LEN2, V

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
