"""What a model's step makes of values at the ends of their types, far positions and loose bounds.

Tolerances, derived before the first run, stand at each test.  A rounding is off by at most half a step: bf16 2^-8, fp32 2^-24,
relative."""
import numpy as np
import pytest

from ea_inputs import inv_freq_table, widen
from ea_inputs.torch_io import to_dev, to_host
from oracle import ea_extensions as X
from oracle import ea_step as S
import paper_2510_00636_amd as ea
from tests.test_gpu_step import HALF, attend_bounds, attend_inputs, i32, kind, outputs, store

pytestmark = pytest.mark.gpu


def run_heads(q, cu, k, v, lens, dt, max_new=None, n=None, scales=(None, None)):
    """The attention over contiguous caches, as stored (dt: bf16, f32 or fp8); out as fp64 numbers."""
    import torch
    B, hkv, cap, d = k.shape
    st = "f32" if dt == "f32" else "bf16"
    p = ea.make_params(B, q.shape[1], hkv, d, kind(st))
    cud, n = i32(cu), cap if n is None else n
    step = ea.make_step(cud, q.shape[0], int(np.diff(cu).max()) if max_new is None else max_new)
    out, lse = outputs(q, st)
    ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
    qd, kd, vd, ld = to_dev(q), to_dev(k), to_dev(v), i32(lens)
    if dt == "fp8":
        ks, vs = (None if s is None else to_dev(s) for s in scales)
        ea.attend_fp8(p, qd, step, kd, vd, ks, vs, ld, n, cap, out, lse, ws)
    else:
        ea.attend(p, qd, step, kd, vd, ld, n, cap, out, lse, ws)
    torch.cuda.synchronize()
    return widen(to_host(out)), lse.cpu().numpy()


def tokens(cu, lens, g):
    """(token, query head, sequence, KV head, rows that it sees) of every result"""
    for b in range(len(cu) - 1):
        m = cu[b + 1] - cu[b]
        for i in range(m):
            for h in range(lens.shape[1]):
                for x in range(h * g, (h + 1) * g):
                    yield cu[b] + i, x, b, h, max(0, int(lens[b, h]) - (m - 1 - i))


# whole heads and heads that several workgroups share, few rows and stretches, every type
KERNELS = [("bf16", 8, 2, 128, [2, 1, 1], [40, 5000, 1]), ("bf16", 6, 2, 64, [3, 5, 2], [90, 5000, 1]), ("bf16", 4, 2, 256, [1, 4, 2], [70, 4000, 1]),
           ("bf16", 8, 2, 128, [100, 1, 70], [300, 20, 5000]), ("bf16", 16, 2, 64, [60, 3, 200], [61, 20, 3000]),
           ("bf16", 4, 2, 256, [90, 2, 70], [200, 20, 3000]), ("fp8", 8, 2, 128, [2, 1, 90], [40, 3000, 2500]),
           ("fp8", 4, 2, 256, [3, 60, 2], [5, 2000, 1]), ("f32", 4, 2, 64, [2, 30, 1], [40, 3000, 20]), ("f32", 8, 8, 64, [1500, 548, 2], [1500, 548, 1]),
           ("f32", 3, 3, 256, [2, 9, 70], [4, 900, 300])]


@pytest.mark.parametrize("what,dt,hq,hkv,d,m,lens", [(w, *x) for x in KERNELS for w in ("nan", "infinite logit")
                                                     if x[0] != "fp8" or w == "nan"])      # (these bytes have no infinities)
def test_a_sum_that_is_not_a_number_is_none_in_the_logarithm_either(what, dt, hq, hkv, d, m, lens):
    """lse is -inf where a token sees no row and nowhere else: a key of NaN, or one whose logit is +inf, makes a NaN of the sum.
    Tokens that do not see that key have what they have without it."""
    r = np.random.default_rng(d)
    st, g = "f32" if dt == "f32" else "bf16", hq // hkv
    lens = np.repeat(np.array(lens)[:, None], hkv, axis=1)
    q, cu, k, v, L = attend_inputs(d + hq, hq, hkv, d, st, lens, m)
    if dt == "fp8":
        k, v = (r.integers(0, 0x60, k.shape).astype(np.uint8) for _ in range(2))
    bad, row = k.copy(), lens[:, 0] - 1 - np.array(m) // 2
    put = {"bf16": (0x7FC0, 0x7F80), "f32": (np.nan, np.inf), "fp8": (0x7F, None)}[dt][what != "nan"]
    q[..., 3] = store(np.array([0.5]), st)[0]                  # so that an infinite key has an infinite logit, and no NaN
    for b in range(3):
        if row[b] >= 0:
            bad[b, :, row[b], 3] = put
    clean, clean_lse = run_heads(q, cu, k, v, L, dt)
    got, lse = run_heads(q, cu, bad, v, L, dt)
    for t, x, b, h, n in tokens(cu, L, g):
        if n == 0:
            assert (got[t, x] == 0).all() and lse[t, x] == -np.inf
        elif n > row[b] >= 0:
            assert np.isnan(got[t, x]).all() and np.isnan(lse[t, x]), (t, x, lse[t, x])
        else:
            assert np.isfinite(lse[t, x]) and np.isfinite(got[t, x]).all()
            if what == "nan":      # (an infinite logit moves the maximum that its neighbours' weights are taken against)
                assert np.array_equal(got[t, x], clean[t, x]) and lse[t, x] == clean_lse[t, x]


@pytest.mark.parametrize("dt,hq,hkv,d,m,lens", [x for x in KERNELS if x[0] != "fp8"])
def test_logits_that_are_all_minus_infinity(dt, hq, hkv, d, m, lens):
    """Such a token has zeros and -inf, like one that sees nothing; a logit of -inf among others weighs nothing."""
    st, g = "f32" if dt == "f32" else "bf16", hq // hkv
    lens = np.repeat(np.array(lens)[:, None], hkv, axis=1)
    q, cu, k, v, L = attend_inputs(d + hq, hq, hkv, d, st, lens, m)
    q[..., 3] = store(np.array([0.5]), st)[0]
    minus = 0xFF80 if dt == "bf16" else -np.inf
    k[0, :, :, 3] = minus
    last = np.maximum(lens[2, 0] - m[2] - 1, 0)                # of the third sequence one row that all its tokens see, if there is one
    k[2, :, last, 3] = minus
    got, lse = run_heads(q, cu, k, v, L, dt)
    for t, x, b, h, n in tokens(cu, L, g):
        if b == 0 or n == 0 or (b == 2 and last == 0 and n == 1):
            assert (got[t, x] == 0).all() and lse[t, x] == -np.inf
        else:
            assert np.isfinite(got[t, x]).all() and np.isfinite(lse[t, x])
    at = cu[2] + m[2] - 1                                      # the last token, by numbers
    n = int(lens[2, 0])
    for x in range(hq):
        keep = np.arange(n) != last
        if not keep.any():
            continue
        want = S.attend_head(widen(q[at:at + 1, x]), widen(k[2, x // g, :n][keep]), widen(v[2, x // g, :n][keep]), n - 1, 1)
        tol, tol_lse = attend_bounds(tuple(np.asarray(w) for w in want), dt, n, d)
        assert (np.abs(got[at, x] - want[0][0]) <= tol[0]).all() and abs(lse[at, x] - want[1][0]) <= tol_lse[0]


@pytest.mark.parametrize("dt,hq,hkv,d,m", [("bf16", 64, 64, 128, 1), ("bf16", 128, 64, 64, 2), ("bf16", 64, 64, 256, 1), ("bf16", 8, 4, 128, 60),
                                          ("bf16", 32, 4, 64, 90), ("bf16", 8, 4, 256, 70), ("f32", 8, 4, 64, 3), ("f32", 8, 4, 256, 30),
                                          ("f32", 16, 16, 64, 1100)])
@pytest.mark.parametrize("steps", [3.0, 7.5])
def test_large_values_weigh_at_most_once(dt, hq, hkv, d, m, steps):
    """One row of each head's 1600 has values of 2^126, and a logit that lies `steps` powers of two above the others', less than what moves
    the maximum that weights are taken against.  The result is below 2^126, so it has to be finite: no weight may pass one.

    The other values are zeros, so the result is 2^126 w / sum, where the exponent is off by the logit's error: d products and sums
    and two roundings of a logit of at most 8 ln 2 (d + 10) 2^-24 8, and 2^-22 of the power; the sum of at most 1600 weights 2^-24 * 1600 / 8
    + 64 2^-24; a weight's rounding to bf16 2^-8, and the result's."""
    n = 1600
    q, k, v = (store(np.zeros(s), dt) for s in ((m, hq, d), (1, hkv, n, d), (1, hkv, n, d)))
    q[..., 0] = store(np.ones(1), dt)[0]
    for h in range(hkv):                                       # all tokens see it, and some of whoever reads it have read others before
        k[0, h, n - m - 5 - h * 71 % 481, 0] = store(np.array([steps * np.log(2.0) * np.sqrt(d)]), dt)[0]
        v[0, h, n - m - 5 - h * 71 % 481] = store(np.array([2.0 ** 126]), dt)[0]
    cu, lens = np.array([0, m]), np.full((1, hkv), n)
    got, lse = run_heads(q, cu, k, v, lens, dt)
    logit = widen(k)[0, 0].max() / np.sqrt(d)
    seen = n - (m - 1 - np.arange(m))
    z = np.exp(logit) + seen - 1
    want = 2.0 ** 126 * np.exp(logit) / z
    assert np.isfinite(got).all()
    e = 8 * (d + 10) * 2.0 ** -24 + 2.0 ** -22 + 264 * 2.0 ** -24 + 2 * HALF[dt]
    assert (np.abs(got / want[:, None, None] - 1) <= e).all(), np.abs(got / want[:, None, None] - 1).max() / e
    assert (np.abs(lse - np.log(z)[:, None]) <= 8 * (d + 10) * 2.0 ** -24 + 2.0 ** -21 + 264 * 2.0 ** -24 + 2.0 ** -22 * np.log(z)[:, None]).all()


# --------------------------------------------------------------------------------------- weights as two numbers
def opposite_values(seed, hq, hkv, d, dt, lens, m):
    """Small logits, and values that take turns in sign: the result is small next to the values, so that what its own rounding
    may be off by does not cover what a weight's rounding to one bf16 number would make."""
    r = np.random.default_rng(seed)
    B, n = len(m), int(np.max(lens))
    cu = np.concatenate([[0], np.cumsum(m)])
    q = store(0.02 * r.standard_normal((int(cu[-1]), hq, d)), "bf16")
    k = r.standard_normal((B, hkv, n, d))
    v = (1.0 + r.random((B, hkv, 1, d))) * np.where(np.arange(n) % 2, -1.0, 1.0)[:, None]
    if dt == "fp8":
        k8, v8 = (torch_e4m3(x) for x in (k, v))
        return q, cu, k8, v8, X.fp8_e4m3_decode(k8), X.fp8_e4m3_decode(v8)
    ks, vs = store(k, "bf16"), store(v, "bf16")
    return q, cu, ks, vs, widen(ks), widen(vs)


def torch_e4m3(x):
    import torch
    return torch.from_numpy(x).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def two_number_bounds(want, n, d):
    """As attend_bounds, where a weight reaches the second product as the sum of two bf16 numbers: what the second one leaves is
    2^-8 of what the first one leaves, 2^-16 of the weight."""
    tol, tol_lse = attend_bounds(want, "bf16", n, d)
    return tol - (HALF["bf16"] - 2.0 ** -16) * want[2], tol_lse


@pytest.mark.parametrize("dt,hq,hkv,d,m,max_new", [
    ("bf16", 8, 2, 128, [1, 1, 1], 1), ("bf16", 8, 2, 128, [8, 3, 1], 8), ("bf16", 8, 2, 128, [16, 1, 9], 16), ("bf16", 14, 2, 64, [2, 1, 1], 2),
    ("bf16", 40, 1, 64, [1, 1, 1], 1), ("bf16", 4, 2, 256, [1, 8, 16], 16), ("bf16", 20, 1, 256, [1, 1, 1], 1), ("bf16", 24, 1, 128, [1, 1, 1], 300),
    ("fp8", 8, 2, 128, [1, 2, 4], 4), ("fp8", 8, 2, 128, [16, 3, 1], 16), ("fp8", 16, 8, 256, [1, 16, 3], 16), ("bf16", 8, 2, 128, [1], 1),
    # one sequence, with bounds as a captured step has them
    ("bf16", 8, 2, 128, [1], 500), ("bf16", 40, 8, 128, [3], 200), ("bf16", 4, 2, 256, [8], 64), ("fp8", 8, 2, 128, [4], 90)])
@pytest.mark.parametrize("n", [40, 900])
def test_few_tokens_have_weights_of_two_numbers(dt, hq, hkv, d, m, max_new, n):
    """Whatever the bounds say that there might be: with up to 16, 32 or 64 (token, head) rows per KV head a result is off by little
    more than its own rounding."""
    lens = np.array([[n - 2 * b] * hkv for b in range(len(m))])
    q, cu, k, v, kf, vf = opposite_values(n + d, hq, hkv, d, dt, lens, m)
    room = np.concatenate([q, np.zeros((max(0, max_new - len(q)), hq, d), dtype=q.dtype)])
    got, lse = run_heads(room, cu, k, v, lens, dt, max_new=max_new)
    t = len(q)
    want = S.attend(widen(q), cu, kf, vf, lens)
    tol, tol_lse = two_number_bounds(want, n, d)
    worst = np.abs(got[:t] - want[0]) / tol
    assert worst.max() <= 1, worst.max()
    assert (np.abs(lse[:t] - want[1]) <= tol_lse).all()
    assert (got[t:] == 7.0).all() and (lse[t:] == 7.0).all()


# ------------------------------------------------------------------------------------------- calls that are large
def test_many_heads_that_add_few_tokens():
    """131072 heads of up to four rows, under a bound of 16 tokens: no launch grows with heads times bound."""
    r = np.random.default_rng(4)
    B, hq, hkv, d, cap = 4096, 128, 32, 64, 4
    m = np.where(r.random(B) < 0.9, 1, r.integers(0, 4, B))
    lens = r.integers(0, cap + 1, (B, hkv))
    q, cu, k, v, L = attend_inputs(1, hq, hkv, d, "bf16", lens, m, cap=cap)
    got, lse = run_heads(q, cu, k, v, L, "bf16", max_new=16)
    assert (lse[:cu[-1]] != 7.0).all()
    some = np.unique(np.r_[0, 1, 2, r.integers(0, B, 12), B - 1])
    at = np.concatenate([np.arange(cu[b], cu[b + 1]) for b in some])
    part = np.concatenate([[0], np.cumsum(m[some])])
    want = S.attend(widen(q[at]), part, widen(k[some]), widen(v[some]), L[some])
    tol, tol_lse = attend_bounds(want, "bf16", cap, d)
    assert (np.abs(got[at] - want[0]) <= tol).all()
    none = want[1] == -np.inf
    assert (lse[at][none] == -np.inf).all() and (np.abs(lse[at][~none] - want[1][~none]) <= tol_lse[~none]).all()


def test_blocks_of_four_gib():
    """A block that has 4 GiB with its heads together: few tokens read it, stretches are refused."""
    import torch
    B, heads, d, bs, nb, n = 1, 128, 256, 65536, 2, 70
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    q, cu, k, v, L = attend_inputs(2, heads, heads, d, "bf16", [n], [1])
    pools = [torch.full((nb, heads, bs, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for pool, x in zip(pools, (k, v)):
        pool[1, :, :n] = to_dev(x[0])
    p, cud, table = ea.make_params(B, heads, heads, d, ea.EA_BF16), i32(cu), i32([[1]])
    pg, (out, lse), qd = ea.make_paged(table, bs, nb), outputs(q, "bf16"), to_dev(q)
    for bound in (1, 40):
        room = torch.zeros(bound, heads, d, dtype=torch.bfloat16, device="cuda")
        room[:1] = qd
        to = torch.zeros_like(room)
        step = ea.make_step(cud, bound, bound)
        ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda")
        if bound == 40:
            with pytest.raises(ea.EaError) as e:
                ea.attend_paged(p, room, step, pools[0], pools[1], pg, i32(L[:, 0]), n, to, None, ws)
            assert e.value.code == 2 and not to.any()
            continue
        ea.attend_paged(p, room, step, pools[0], pools[1], pg, i32(L[:, 0]), n, out, lse, ws)
        torch.cuda.synchronize()
        want = S.attend(widen(q), cu, widen(k), widen(v), L)
        tol, tol_lse = attend_bounds(want, "bf16", n, d)
        assert (np.abs(widen(to_host(out)) - want[0]) <= tol).all() and (np.abs(lse.cpu().numpy() - want[1]) <= tol_lse).all()
    pools.clear()
    torch.cuda.empty_cache()


# ----------------------------------------------------------------------------------------------- far positions
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("far", [1 << 12, 1 << 24, 1 << 31])
def test_angles_of_far_positions(d, inter, far):
    """Pairs (1, 0) become (cos, sin) of their angle, the fp64 product of position and frequency.  What the reduction leaves is rounded
    to fp32 with its remainder kept, sine and cosine of it are off by two steps at most (2 * 2^-24 below one), the remainder's sum by
    half a step."""
    import torch
    r = np.random.default_rng(far % 1000 + d)
    t = 3000
    pos = r.integers(far // 2, far, t)
    pos[0] = far - 1
    x = np.zeros((t, 2, d), dtype=np.float32)
    x[:, :, slice(0, None, 2) if inter else slice(0, d // 2)] = 1.0
    inv = inv_freq_table(d, 1e4)
    q, cache = torch.zeros(t, 1, d, device="cuda"), [torch.zeros(1, 1, t, d, device="cuda") for _ in range(2)]
    xd = to_dev(x)
    p = ea.make_params(1, 1, 1, d, ea.EA_F32, rope_layout=int(inter))
    rows = ea.make_new_rows(xd[:, :1], xd[:, 1:], xd[:, 1:], i32(pos), to_dev(inv))
    ea.append(p, rows, i32([0, t]), i32([[t]]), cache[0], cache[1], t, q)
    torch.cuda.synchronize()
    want = S.rotate(x.astype(np.float64), pos, inv, inter)
    tol = 2 * 2.0 ** -24 + 2.0 ** -25
    for got, w in ((to_host(q)[:, 0], want[:, 0]), (to_host(cache[0])[0, 0], want[:, 1])):
        assert np.abs(got - w).max() <= tol, np.abs(got - w).max() / tol


# ---------------------------------------------------------------------------------------------- small values
@pytest.mark.parametrize("dt,hq,hkv,d,m", [("bf16", 8, 2, 128, 1), ("bf16", 4, 2, 64, 1), ("bf16", 4, 2, 256, 2), ("bf16", 8, 2, 128, 60), ("bf16", 16, 2, 64, 90),
                                          ("bf16", 4, 2, 256, 70), ("f32", 4, 2, 64, 3), ("f32", 4, 2, 256, 30), ("f32", 8, 8, 64, 2100)])
def test_values_below_the_smallest_normal_number(dt, hq, hkv, d, m):
    """Values of 1 to 15 times 2^-130 that all weigh the same: in fp32 a token has the mean of those that it sees, in bf16 that or zero.

    A weight is 2^-8, or a number above that: products are whole multiples of 2^-138 and so are their sums, exact as long as they stay
    below 2^-126 and rounded to 24 bits above; the quotient is off by 2^-22 of itself and half of fp32's last step, 2^-150."""
    r = np.random.default_rng(d + m)
    n = 2400
    m = min(m, n)
    k, v = np.zeros((1, hkv, n, d)), r.integers(1, 16, (1, hkv, n, d)) * 2.0 ** -130
    qs, ks, vs = store(r.standard_normal((m, hq, d)), dt), store(k, dt), store(v, dt)
    assert np.array_equal(widen(vs), v)
    cu, lens = np.array([0, m]), np.full((1, hkv), n)
    got, lse = run_heads(qs, cu, ks, vs, lens, dt)
    seen = n - (m - 1 - np.arange(m))
    want = (np.cumsum(v[0], axis=1)[:, seen - 1] / seen[:, None]).transpose(1, 0, 2)      # [m, hkv, d]
    want = np.repeat(want, hq // hkv, axis=1)
    tol = 2.0 ** -22 * want + 2.0 ** -150 if dt == "f32" else 2.0 ** -126
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("m", [[1, 1], [2, 90], [100, 80]])
def test_a_scale_that_is_not_a_number(d, m):
    """What a head's scale makes of its keys reaches every token that sees one of them; a token that sees none has zeros and -inf."""
    r = np.random.default_rng(d)
    lens = np.array([[300, m[0] - 1], [700, 500]])
    cu = np.concatenate([[0], np.cumsum(m)])
    q = store(r.standard_normal((int(cu[-1]), 8, d)), "bf16")
    k, v = (r.integers(0, 0x60, (2, 2, 700, d)).astype(np.uint8) for _ in range(2))
    ks = np.array([[1.0, np.nan], [np.nan, 0.5]], dtype=np.float32)
    got, lse = run_heads(q, cu, k, v, lens, "fp8", scales=(ks, None))
    for t, x, b, h, n in tokens(cu, lens, 4):
        if n == 0:
            assert (got[t, x] == 0).all() and lse[t, x] == -np.inf
        elif np.isnan(ks[b, h]):
            assert np.isnan(got[t, x]).all() and np.isnan(lse[t, x])
        else:
            assert np.isfinite(got[t, x]).all() and np.isfinite(lse[t, x])
