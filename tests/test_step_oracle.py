"""Pins of the step's oracle (CPU): block tables by hand and by their invariants, the rotation against complex numbers, attention
against a brute-force softmax and its reductions."""
import numpy as np
import pytest

from oracle import ea_step as S


def test_block_tables_by_hand():
    table = np.array([[7, 3, -1, -1], [5, 1, 0, -1], [2, -1, -1, -1]], dtype=np.int32)
    free = np.array([4, 6, 8, -9, -9, -9], dtype=np.int32)
    # sequence 0 grows over a border of blocks of 16, 1 gives two blocks back, 2 grows inside its block
    t, f, n, lens, cu, slots, pos = S.block_tables(table, free, 3, [31, 48, 3], [34, 10, 5], 16, 8, seen=[100, 0, 50])
    assert list(t[0]) == [7, 3, 1, -1]                  # the first block given back (entry 1 of sequence 1)
    assert list(t[1]) == [5, 1, 0, -1] and list(t[2]) == [2, -1, -1, -1]
    assert n == 4 and list(f) == [4, 6, 8, 0, -9, -9]   # the other one on top of the list
    assert list(lens) == [34, 10, 5] and list(cu) == [0, 3, 3, 5]
    assert list(slots) == [3 * 16 + 15, 16, 17, 2 * 16 + 3, 2 * 16 + 4, -1, -1, -1]
    assert list(pos) == [100, 101, 102, 50, 51, -1, -1, -1]


def test_block_tables_without_room():
    table = np.full((3, 2), -1, dtype=np.int32)
    t, f, n, lens, cu, slots, pos = S.block_tables(table, np.array([9, 8], dtype=np.int32), 2, [0, 0, 0], [40, 20, 16], 16, 80)
    assert list(lens) == [0, 20, 0]                     # 40 rows do not fit the row of the table; the third finds the list empty
    assert n == 0 and list(t[1]) == [8, 9] and list(cu) == [0, 40, 60, 76]
    assert (slots[:40] == -1).all() and (slots[60:] == -1).all() and slots[40] == 8 * 16 and slots[56] == 9 * 16


@pytest.mark.parametrize("seed", range(6))
def test_growing_and_going_back_restores_the_list(seed):
    r = np.random.default_rng(seed)
    B, bs, mb = 7, 16, 9
    old = r.integers(0, 100, B)
    held = [-(-x // bs) for x in old]
    ids = r.permutation(80).astype(np.int32)
    table, at = np.full((B, mb), -1, dtype=np.int32), 0
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    free = np.full(80, -1, dtype=np.int32)
    free[:80 - at] = ids[at:]
    new = old + r.integers(0, 40, B)
    t1, f1, n1, l1, cu, slots, _ = S.block_tables(table, free, 80 - at, old, new, bs, int((new - old).sum()))
    assert (l1 == new).all() and len(set(slots.tolist())) == len(slots)
    used = [t1[b, j] for b in range(B) for j in range(-(-new[b] // bs))]
    assert sorted(used + f1[:n1].tolist()) == list(range(80))
    t2, f2, n2, l2, *_ = S.block_tables(t1, f1, n1, l1, old, bs, 0)
    assert n2 == 80 - at and (f2[:n2] == free[:n2]).all() and (l2 == old).all() and (t2 == t1).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product(interleaved):
    r = np.random.default_rng(1)
    x, pos, inv = r.standard_normal((5, 3, 8)), np.array([0, 1, 7, 1000, 2 ** 31 - 1]), 10.0 ** -np.arange(4)
    y = S.rotate(x, pos, inv, interleaved)
    z = x[..., 0::2] + 1j * x[..., 1::2] if interleaved else x[..., :4] + 1j * x[..., 4:]
    w = z * np.exp(1j * (pos[:, None] * inv))[:, None]
    got = y[..., 0::2] + 1j * y[..., 1::2] if interleaved else y[..., :4] + 1j * y[..., 4:]
    assert np.allclose(got, w, rtol=0, atol=1e-9)
    assert (y[0] == x[0]).all()


def test_attention_reductions():
    r = np.random.default_rng(2)
    q, k, v = r.standard_normal((3, 4)), r.standard_normal((9, 4)), r.standard_normal((9, 4))
    out, lse, spread, _ = S.attend_head(q, k, v, 9, 3)
    for i, n in enumerate((7, 8, 9)):
        e = np.exp(k[:n] @ q[i] / 2.0)
        assert np.allclose(out[i], (e[:, None] * v[:n]).sum(0) / e.sum()) and np.isclose(lse[i], np.log(e.sum()))
        assert (spread[i] >= np.abs(out[i]) - 1e-15).all()
    # equal keys: the mean; nothing to see: zeros and -inf
    out, lse, *_ = S.attend_head(q, np.ones((9, 4)), v, 9, 3)
    assert np.allclose(out[2], v.mean(0))
    out, lse, *_ = S.attend_head(q, k, v, 2, 3)
    assert (out[0] == 0).all() and lse[0] == -np.inf and np.allclose(out[1], v[0])
    # what stands behind the length does not matter
    k[5:], v[5:] = np.nan, np.inf
    assert np.isfinite(S.attend_head(q, k, v, 5, 3)[0]).all()
