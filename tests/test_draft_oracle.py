"""Pins of the oracle of quantised rows and drafted trees (CPU): the element formats against torch's own e4m3 and by hand, the least
power of two by brute force, trees against a walk and against the chain."""
import numpy as np
import pytest

from oracle import ea_draft as D
from oracle import ea_step as S


def test_grids_by_hand():
    assert D.E4M3[-1] == 448 and D.E4M3[1] == 2.0 ** -9 and D.E4M3[8] == 2.0 ** -6 and len(D.E4M3) == 127
    codes, e = D.quantise(np.array([6.0, -5.0, 2.5, 3.5, 0.25, 0.75, 1.25, -0.3] + [0.0] * 24), 4)
    assert e == [127] and list(codes[:8]) == [7, 14, 4, 6, 0, 2, 2, 9]      # halves to the even code
    assert list(D.values(codes, e, 4)[:8]) == [6, -4, 2, 4, 0, 1, 1, -0.5]
    assert list(D.packed(codes, 4)[:3]) == [7 | 14 << 4, 4 | 6 << 4, 0 | 2 << 4]
    assert np.array_equal(D.unpacked(D.packed(codes, 4), 4), codes)


@pytest.mark.parametrize("bits", [8, 4])
def test_elements_are_the_nearest_and_the_power_is_the_least(bits):
    import torch
    r = np.random.default_rng(bits)
    x = r.standard_normal((200, 64)) * 2.0 ** r.integers(-20, 20, (200, 1))
    x[3] = 0
    codes, e = D.quantise(x, bits)
    most, back = D.grid(bits)[-1], D.values(codes, e, bits)
    for i in range(200):
        for g in range(2):
            part = x[i, g * 32:(g + 1) * 32]
            by = 2.0 ** (int(e[i, g]) - 127)
            assert np.abs(part).max() <= most * by and (e[i, g] == 10 or np.abs(part).max() > most * by / 2)
            every = np.concatenate([D.grid(bits), -D.grid(bits)]) * by
            assert np.allclose(np.abs(every[None] - part[:, None]).min(1), np.abs(back[i, g * 32:(g + 1) * 32] - part), rtol=0, atol=0)
    if bits == 8:
        z = (x.reshape(200, 2, 32) / 2.0 ** (e[..., None] - 127.0)).reshape(200, 64)
        assert np.array_equal(torch.from_numpy(z).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy(), D.packed(codes, 8))
    again, e2 = D.quantise(back, bits)
    assert np.array_equal(D.values(again, e2, bits), back)


@pytest.mark.parametrize("bits", [8, 4])
def test_borders_of_the_range(bits):
    most = D.grid(bits)[-1]
    x = np.zeros((6, 32))
    x[0, 0] = D.BF16_MOST                      # not to infinity
    x[1, 0], x[1, 1] = np.inf, 1
    x[2, 5] = np.nan
    x[3, 0] = most                             # just fits
    x[4, 0] = most * (1 + 2.0 ** -20)          # just does not
    x[5, 0] = 2.0 ** -133                      # below what is resolved
    codes, e = D.quantise(x, bits)
    back = D.values(codes, e, bits)
    assert back[0, 0] == (1.875 if bits == 8 else 1.5) * 2.0 ** 127
    assert e[1] == 255 and e[2] == 255 and np.isnan(back[1:3]).all() and (codes[1:3] == 0).all()
    assert e[3] == 127 and back[3, 0] == most and e[4] == 128 and e[5] == 10 and back[5, 0] == 0


def test_trees_by_hand():
    #        0 -> 1, 2; 1 -> 3; 2 -> 4, 5; 6 alone | one token | none
    cu, parents = np.array([0, 7, 8, 8]), np.array([-1, 0, 0, 1, 2, 2, 9, 0])
    sees, pos = D.masks(parents, cu, seen=[10, 20, 30])
    assert [list(np.flatnonzero(x)) for x in sees] == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 2, 4], [0, 2, 5], [6], [0]]
    assert list(pos) == [10, 11, 11, 12, 12, 12, 10, 20]
    tokens, target = np.array([5, 8, 7, 1, 4, 4, 2, 3]), np.array([7, 0, 4, 0, 9, 6, 0, 1])
    assert D.accept(tokens, parents, target, cu) == ([[0, 2, 4], [0], []], [9, 1, -1])
    assert list(D.words_of(sees, 1)[:, 0]) == [1, 3, 5, 11, 21, 37, 64, 1]


def test_a_chain_is_the_step_itself():
    r = np.random.default_rng(2)
    cu, hq, d = np.array([0, 5, 6, 9]), 4, 16
    q = r.standard_normal((9, hq, d))
    lens = np.array([[9, 7], [3, 1], [2, 40]])                 # the third sequence's first head has fewer rows than tokens
    k, v = ([[r.standard_normal((n, d)) for n in x] for x in lens] for _ in range(2))
    parents = np.array([-1, 0, 1, 2, 3, -1, -1, 0, 1])
    sees, _ = D.masks(parents, cu)
    for a, b in zip(D.attend(q, cu, k, v, lens, sees), S.attend(q, cu, k, v, lens)):
        assert np.allclose(a, b, rtol=0, atol=1e-12)
