"""MX pools on the GPU where rows are not what the library writes, or calls are cut unusually: against the same call on clean rows, and
against the fp64 oracle with the tolerances of the pools' tests."""
import numpy as np
import pytest

from ea_inputs import widen
from oracle import ea_draft as D
from tests import test_gpu_mx as M
from tests import test_gpu_tree as T
from tests.test_gpu_mx import Mx, queries, sums

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
