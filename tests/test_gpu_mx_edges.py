"""MX pools on the GPU where rows are not what the library writes, or calls are cut unusually: against the same call on clean rows, and
against the fp64 oracle with the tolerances of the pools' tests."""
import numpy as np
import pytest

from ea_inputs import widen
from oracle import ea_draft as D
import paper_2510_00636_amd as ea
from tests import test_gpu_mx as M
from tests import test_gpu_tree as T
from tests.test_gpu_mx import Mx, queries, sums
from tests.test_gpu_step import check_attend, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,hq,hkv,d", [(8, 8, 2, 128), (4, 8, 2, 128), (8, 6, 2, 64), (4, 6, 2, 64), (8, 4, 2, 256), (4, 4, 2, 256)])
@pytest.mark.parametrize("m", [2, 7, 40, 130])
@pytest.mark.parametrize("how", ["chain", "tree"])
def test_elements_past_the_end_of_bf16(bits, hq, hkv, d, m, how):
    """Elements that widen to 2^128 and more, in a row of the step: infinities to the tokens that see the row, nothing to the others.
    A sequence for each exponent that has such elements, and one for the last that has none."""
    exponents = range(246, 255) if bits == 8 else range(252, 255)
    r = np.random.default_rng(bits + d + m)
    B = len(exponents)
    lens = r.integers(m, m + 300, B)
    lens[0] = m
    c = Mx(hq * d, lens, hkv, d, 16, bits)
    cu = sums([m] * B)
    q = queries(d, int(cu[-1]), hq, d)
    if how == "tree":
        sees, words = D.masks(T.trees(r, [m] * B), cu)[0], -(-m // 64)
        call = lambda: T.run_mx(c, q, cu, sees, words, hq, hkv, d)    # noqa: E731
    else:
        sees = np.tril(np.ones((m, m), dtype=bool))[None].repeat(B, 0).reshape(B * m, m)
        call = lambda: M.run_mx(c, q, cu, hq, hkv, d)    # noqa: E731
    clean, clean_lse = call()
    bad = r.integers(1, m, B)                                  # the token whose row is spoiled: its second group of channels
    past = np.zeros((B, hkv, d), dtype=bool)
    top = 126 if bits == 8 else 7                              # the largest element's code
    for b, e in enumerate(exponents):
        least = (262 - e) * 8 if bits == 8 else 8 - 2 * (e - 252)      # the code of 2^(255 - e)
        row = lens[b] - m + bad[b]
        code = np.where(r.random((hkv, 32)) < 0.5, r.integers(0, min(least, top + 1), (hkv, 32)), r.integers(min(least, top), top + 1, (hkv, 32)))
        code[:, 0], code[:, 1] = min(least - 1, top), min(least, top)
        c.codes[1][b, :, row, 32:64] = code + 2 ** (bits - 1) * r.integers(0, 2, code.shape)
        c.e[1][b, :, row, 1] = e
        past[b] = np.abs(D.values(c.codes[1][b, :, row], c.e[1][b, :, row], bits)) >= 2.0 ** 128
    assert not past[0].any() and past[1:, :, 32:64].any(axis=(1, 2)).all()
    c.load()
    got, lse = call()
    got, clean = widen(got), widen(clean)
    assert np.array_equal(lse, clean_lse)
    for b in range(B):
        for i in range(m):
            t = cu[b] + i
            if not sees[t, bad[b]]:
                assert np.array_equal(got[t], clean[t])
                continue
            hit = past[b].repeat(hq // hkv, 0)
            assert not np.isfinite(got[t][hit]).any() and np.isfinite(got[t][~hit]).all()
            assert np.array_equal(got[t][:, :32], clean[t][:, :32]) and np.array_equal(got[t][:, 64:], clean[t][:, 64:])


# ------------------------------------------------------------------------- tiles of 256 rows, as bounds above 1024 keys have them
class Far(Mx):
    """The same rows under a bound above 1024: entries behind a sequence's blocks lead nowhere."""

    def load(self):
        super().load()
        t = np.full((len(self.lens), 1040 // self.bs + 1), -99, dtype=np.int32)
        t[:, :self.max_blocks] = self.table
        for b, n in enumerate(self.lens):
            t[b, -(-int(n) // self.bs):] = -99
        self.t = i32(t)
        self.pg = ea.make_paged(self.t, self.bs, self.nb)
        self.n = t.shape[1] * self.bs


SHAPES = [(8, 2, 128), (5, 1, 128), (16, 1, 64), (14, 2, 64), (4, 2, 256), (24, 1, 128), (64, 1, 64)]


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("m", [[33, 1, 0, 70], [9, 40, 300, 2], [129, 2, 130, 257]])
def test_stretches_in_tall_tiles(monkeypatch, hq, hkv, d, bits, m):
    monkeypatch.setattr(M, "Mx", Far)
    M.test_stretches(hq, hkv, d, bits, m)


@pytest.mark.parametrize("bits,hq,hkv,d,m", [(8, 8, 2, 128, [100, 1, 70]), (4, 6, 2, 64, [5, 2, 90]), (8, 6, 2, 64, [90, 2, 140]), (4, 8, 2, 128, [50, 130, 2]),
                                             (4, 4, 2, 256, [3, 200, 2])])
@pytest.mark.parametrize("where", ["values", "keys"])
def test_groups_that_are_not_numbers_in_tall_tiles(monkeypatch, bits, hq, hkv, d, m, where):
    monkeypatch.setattr(M, "Mx", Far)
    M.test_groups_that_are_not_numbers(bits, hq, hkv, d, m, where)


@pytest.mark.parametrize("bits,hq,hkv,d", [(8, 8, 2, 128), (8, 6, 2, 64), (4, 20, 1, 128), (4, 8, 2, 64), (4, 64, 1, 64)])
@pytest.mark.parametrize("m", [[64, 33, 2], [100, 1, 70], [256, 130, 17]])
@pytest.mark.parametrize("how", ["tree", "any"])
def test_trees_in_tall_tiles(monkeypatch, bits, hq, hkv, d, m, how):
    monkeypatch.setattr(T, "Mx", Far)
    T.test_trees_over_quantised_pools(bits, hq, hkv, d, m, how)


@pytest.mark.parametrize("bits,hq,hkv,d", [(8, 8, 2, 128), (4, 8, 2, 64), (8, 8, 2, 64), (4, 8, 2, 128)])
@pytest.mark.parametrize("m", [[30, 1, 2], [90, 3, 150]])
def test_lengths_that_make_no_sense_in_tall_tiles(bits, hq, hkv, d, m):
    """Negative lengths count as none, those over n as n."""
    c = Mx(5, [200, 160, 1100], hkv, d, 16, bits)
    cu = sums(m)
    q = queries(1, int(cu[-1]), hq, d)
    c.ld = i32([-7, 160, 1 << 30])
    got, lse = M.run_mx(c, q, cu, hq, hkv, d, n=1100)
    check_attend(got, lse, q, cu, c.val[0], c.val[1], np.array([[0] * hkv, [160] * hkv, [1100] * hkv]), "bf16")
    sees, words = T.some_masks(np.random.default_rng(3), m, "any"), -(-max(m) // 64)
    got, lse = T.run_mx(c, q, cu, sees, words, hq, hkv, d, n=1100)
    T.check(got, lse, q, cu, c.val[0], c.val[1], np.array([[0] * hkv, [160] * hkv, [1100] * hkv]),
            np.pad(sees, ((0, 0), (0, words * 64 - sees.shape[1]))), "bf16")


@pytest.mark.parametrize("bits,hq,hkv,d", [(4, 8, 2, 64), (8, 8, 2, 128)])
@pytest.mark.parametrize("m", [[60], [200, 1]])
def test_long_heads_in_tall_tiles(bits, hq, hkv, d, m):
    """Tiles that end inside a block, pieces of a head, and the same rows seen through masks of the chain."""
    lens = [4100, 1999][:len(m)]
    c = Mx(d + bits, lens, hkv, d, 32, bits)
    cu = sums(m)
    q = queries(d, int(cu[-1]), hq, d)
    L = np.repeat(c.lens[:, None], hkv, 1)
    got, lse = M.run_mx(c, q, cu, hq, hkv, d)
    check_attend(got, lse, q, cu, c.val[0], c.val[1], L, "bf16")
    sees, words = D.masks(T.trees(None, m, "chain"), cu)[0], -(-max(m) // 64)
    got, lse = T.run_mx(c, q, cu, sees, words, hq, hkv, d)
    check_attend(got, lse, q, cu, c.val[0], c.val[1], L, "bf16")


@pytest.mark.parametrize("bits,d", [(4, 64), (8, 64), (4, 128), (8, 128)])
def test_elements_past_the_end_of_bf16_in_tall_tiles(monkeypatch, bits, d):
    monkeypatch.setattr("tests.test_gpu_mx_edges.Mx", Far)
    for how in ("chain", "tree"):
        test_elements_past_the_end_of_bf16(bits, 8, 2, d, 70, how)
