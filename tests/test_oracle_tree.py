"""Pins of the oracle's drafted-token operators: brute force, agreement with the definitions they extend, and the
packed visibility words of the library's host helper."""
import numpy as np
import pytest
import torch

import paper_2509_00419_amd as lv
from oracle import lvlm_oracle as O


def test_rotation_keeps_lengths_and_depends_on_the_difference_of_positions():
    r = np.random.default_rng(1)
    q, k = r.standard_normal((2, 64))
    freq = 1e4 ** (-np.arange(32) / 32)
    for adjacent in (False, True):
        def turn(x, p):
            return O.rotate(x, O.pair_angles([p], freq, [32]), adjacent)
        assert np.allclose(np.linalg.norm(turn(q, 77)), np.linalg.norm(q))
        assert np.allclose(turn(q, 19) @ turn(k, 7), turn(q, 1012) @ turn(k, 1000))
        assert np.array_equal(turn(q, 0), q)
    x = O.rotate(q, O.pair_angles([3], freq[:8], [8]))
    assert np.array_equal(x[16:], q[16:]) and not np.allclose(x[:16], q[:16])
    three = O.pair_angles([5, 6, 7], freq, [8, 12, 12])
    assert three[7] == 5 * freq[7] and three[8] == 6 * freq[8] and three[31] == 7 * freq[31]


def test_a_chain_is_causal_attention_and_one_row_is_decoding():
    r = np.random.default_rng(2)
    B, Hq, Hkv, d, N, T = 2, 4, 2, 8, 13, 5
    q, k, v = r.standard_normal((B, N, Hq, d)), r.standard_normal((B, N, Hkv, d)), r.standard_normal((B, N, Hkv, d))
    ref, lse = O.prefill_attn(q, k, v)
    kc, vc = k.transpose(0, 2, 1, 3), v.transpose(0, 2, 1, 3)
    length = np.full((B, Hkv), N)
    out, got, _ = O.tree_attn(q[:, N - T:], kc, vc, length)
    assert np.allclose(out, ref[:, N - T:], atol=1e-6) and np.allclose(got, lse[:, :, N - T:], atol=1e-6)
    one, _, _ = O.tree_attn(q[:, N - 1:], kc, vc, length, mask=np.ones((B, 1, 1), bool))
    assert np.allclose(one, ref[:, N - 1:], atol=1e-6)


def test_a_tree_row_is_its_own_chain():
    """Every row of a tree sees what it would see were its path alone in the cache."""
    r = np.random.default_rng(3)
    d, base, parent = 8, 6, [-1, 0, 0, 1, 2, 3, -1]
    T = len(parent)
    kc, vc = r.standard_normal((2, 1, 1, base + T, d))
    q = r.standard_normal((1, T, 2, d))
    out, lse, _ = O.tree_attn(q, kc, vc, np.array([[base + T]]), mask=O.tree_mask(parent)[None])
    for t in range(T):
        path = [t]
        while parent[path[0]] >= 0:
            path.insert(0, parent[path[0]])
        at = list(range(base)) + [base + i for i in path]
        ref, ref_lse, _ = O.tree_attn(q[:, [t] * len(path)], kc[:, :, at], vc[:, :, at], np.array([[len(at)]]))
        assert np.allclose(out[0, t], ref[0, -1]) and np.allclose(lse[0, :, t], ref_lse[0, :, -1])


def test_pages_are_only_another_place():
    r = np.random.default_rng(4)
    B, Hkv, d, size, T = 2, 2, 4, 16, 3
    length = np.array([[20, 0], [33, 15]])
    pages = np.array([[[5, 2, 9], [0, 7, -1]], [[3, 8, 1], [4, 6, -1]]])
    pool = r.standard_normal((2, 10, size, d))
    dense = np.zeros((2, B, Hkv, 48, d))
    for b in range(B):
        for g in range(Hkv):
            for s in range(48):
                page = pages[b, g, s // size]
                if page >= 0:
                    dense[:, b, g, s] = pool[:, page, s % size]
    new = r.standard_normal((2, B, T, Hkv, d))
    a = O.kv_append(*new, *pool, length, pages=pages)
    b_ = O.kv_append(*new, *dense, length)
    assert np.array_equal(a[5], b_[5])
    q = r.standard_normal((B, T, 4, d))
    x, y = O.tree_attn(q, a[0], a[1], a[5], pages=pages), O.tree_attn(q, b_[0], b_[1], b_[5])
    assert np.array_equal(x[0], y[0]) and np.array_equal(x[1], y[1])
    path, n_path = np.array([[0, 2, 9], [1, 0, 2]]), np.array([2, 3])
    c, e = O.tree_commit(a[0], a[1], length, path, n_path, pages=pages), O.tree_commit(b_[0], b_[1], length, path, n_path)
    assert np.array_equal(c[5], e[5]) and c[5].tolist() == [[22, 2], [34, 16]]
    assert np.array_equal(O.tree_attn(q, c[0], c[1], c[5], pages=pages)[0], O.tree_attn(q, e[0], e[1], e[5])[0])


def test_rows_that_see_nothing_and_entries_in_no_page():
    d = 4
    k = v = np.ones((1, 1, 8, d))
    out, lse, _ = O.tree_attn(np.ones((1, 2, 1, d)), k, v, np.array([[2]]), mask=np.array([[[1, 0], [0, 0]]], bool))
    assert np.array_equal(out[0, 1, 0], np.zeros(d)) and lse[0, 0, 1] == -np.inf and np.isfinite(lse[0, 0, 0])
    pool = np.ones((1, 16, d))
    out, lse, _ = O.tree_attn(np.ones((1, 1, 1, d)), pool, pool, np.array([[20]]), pages=np.array([[[7, 0]]]))
    assert np.allclose(lse, np.log(4 * np.exp(d ** 0.5)))
    assert O.kv_append(np.ones((1, 3, 1, d)), np.ones((1, 3, 1, d)), k * 0, v * 0, np.array([[6]]))[5][0, 0] == 6      # does not fit


@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64, 65, 300])
def test_visibility_words(T):
    r = np.random.default_rng(T)
    parent = np.array([r.integers(-1, t) if t else -1 for t in range(T)], dtype=np.int32)
    words = lv.tree_mask(torch.from_numpy(parent))
    assert words.shape == (T, (T + 31) // 32) and words.dtype == torch.int32
    bits = (words.numpy().view(np.uint32)[:, :, None] >> np.arange(32, dtype=np.uint32)) & 1
    assert np.array_equal(bits.reshape(T, -1)[:, :T].astype(bool), O.tree_mask(parent)) and bits.reshape(T, -1)[:, T:].sum() == 0
    two = lv.tree_mask(torch.from_numpy(np.stack([parent, np.arange(T) - 1])).long())
    assert torch.equal(two[0], words) and two.shape[0] == 2
    assert np.array_equal(O.tree_mask(np.arange(T) - 1), np.tril(np.ones((T, T), bool)))


@pytest.mark.parametrize("parent", [[0], [-2], [-1, 1], [-1, 0, 5], [-1, 2 ** 40]])
def test_parents_that_are_no_tree_are_refused(parent):
    with pytest.raises(lv.LvlmError):
        lv.tree_mask(torch.tensor(parent))
    with pytest.raises(ValueError):
        lv.tree_mask(torch.tensor(parent).float())
    with pytest.raises(lv.LvlmError):
        lv.tree_mask(torch.full((1025,), -1))
