"""A model's step over its cache on the GPU against its fp64 oracle: block tables, new rows, attention, and a loop of them.

Tolerances, derived before the first run.  A rounding is off by at most half a step: bf16 2^-8, fp16 2^-11, fp32 2^-24, e4m3 2^-4,
relative.  Rotated rows: angles keep 2^-31 of a turn, sine and cosine and three roundings of the products 2^-22 of the pair's
length, then the rounding to the stored type.  Attention: see `attend_bounds`."""
import numpy as np
import pytest

from ea_inputs import make_block_pools, widen, inv_freq_table, quantize_fp8, bf16_bits_from_f64
from ea_inputs.torch_io import to_dev, to_host
from oracle import ea_extensions as X
from oracle import ea_step as S
import paper_2510_00636_amd as ea

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
MARK = {"bf16": 0x7FC0, "f32": np.nan}          # what stands where nothing may look: NaN


def store(x, dt):
    return bf16_bits_from_f64(x) if dt == "bf16" else x.astype(np.float32)


def kind(dt):
    return ea.EA_BF16 if dt == "bf16" else ea.EA_F32


def i32(x):
    return to_dev(np.ascontiguousarray(np.asarray(x, dtype=np.int32)))


# ----------------------------------------------------------------------------------- block tables
def run_tables(table, free, count, old, new, bs, n_tokens, seen=None):
    import torch
    B, mb = table.shape
    p = ea.make_params(B, 2, 1, 64, ea.EA_BF16)
    t, f = i32(table), i32(free)
    pg = ea.make_paged(t, bs, len(free))
    out = [torch.full((x,), -7, dtype=torch.int32, device="cuda") for x in (B, 1, B + 1, max(n_tokens, 1))]
    slots = torch.full((max(n_tokens, 1),), -7, dtype=torch.int64, device="cuda")
    ea.block_tables(p, pg, i32(old), i32(new), f, i32([count]), out[0], out[1], out[2], n_tokens, slots, out[3],
                    None if seen is None else i32(seen))
    torch.cuda.synchronize()
    return to_host(t), to_host(f), int(out[1]), to_host(out[0]), to_host(out[2]), to_host(slots)[:n_tokens], to_host(out[3])[:n_tokens]


def check_tables(got, want, cu_end):
    for g, w in zip(got[:6], want[:6]):
        assert np.array_equal(g, w)
    n = min(cu_end, len(got[6]))
    assert np.array_equal(got[6][:n], want[6][:n]) and (got[6][n:] == -7).all()


@pytest.mark.parametrize("B,bs", [(1, 16), (3, 16), (64, 32), (65, 16), (257, 64), (1000, 16), (4096, 256)])
@pytest.mark.parametrize("kindof", ["one", "ragged", "cut", "both", "short"])
def test_block_tables(B, bs, kindof):
    r = np.random.default_rng(B * 7 + bs)
    mb = 40
    old = r.integers(0, mb * bs // 2, B)
    if kindof == "one":
        new = old + 1
    elif kindof == "ragged":
        new = old + np.where(r.random(B) < 0.2, r.integers(0, 9 * bs, B), r.integers(0, 3, B))
    elif kindof == "cut":
        new = (old * r.random(B)).astype(int)
    else:
        new = np.where(r.random(B) < 0.5, (old * r.random(B)).astype(int), old + r.integers(0, 2 * bs, B))
    if kindof == "short" and B > 2:
        new[1] = mb * bs + 1                                   # one that its row of the table has no room for
        old[2], new[2] = -5, -9                                # and lengths that make no sense
    held = [-(-max(int(x), 0) // bs) for x in old]
    spare = 4 * B if kindof != "short" else max(1, B // 8)     # too few blocks: some are not served
    nb = sum(held) + spare
    ids = r.permutation(nb).astype(np.int32)
    table, at = np.full((B, mb), -1, dtype=np.int32), 0
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    free = np.full(nb, -1, dtype=np.int32)
    free[:spare] = ids[at:]
    seen = r.integers(0, 1 << 20, B)
    total = int(np.maximum(0, np.maximum(new, 0) - np.maximum(old, 0)).sum())
    for n_tokens in sorted({0, total, total + 300}):
        for s in (None, seen):
            want = S.block_tables(table, free, spare, old, new, bs, n_tokens, s)
            check_tables(run_tables(table, free, spare, old, new, bs, n_tokens, s), want, total)
    # growing by a step and going back restores the list, the table's held entries and the count
    if kindof in ("one", "ragged"):
        t, f, n, lens, *_ = run_tables(table, free, spare, old, new, bs, 0)
        t2, f2, n2, lens2, *_ = run_tables(t, f, n, lens, old, bs, 0)
        assert n2 == spare and np.array_equal(f2[:n2], free[:spare]) and np.array_equal(lens2, old) and np.array_equal(t2, t)


# --------------------------------------------------------------------------------------- new rows
def pair_length(x, interleaved):
    h = x.shape[-1] // 2
    if interleaved:
        n = np.hypot(x[..., 0::2], x[..., 1::2])
        return np.repeat(n, 2, axis=-1)
    n = np.hypot(x[..., :h], x[..., h:])
    return np.concatenate([n, n], axis=-1)


def check_rotated(got, x, pos, inv, inter, dt):
    want = S.rotate(x, pos, inv, inter)
    tol = HALF[dt] * np.abs(want) + 2.0 ** -21 * pair_length(x, inter)
    assert bool((np.abs(got - want) <= tol).all())


@pytest.mark.parametrize("hq,hkv,d,bs,t", [(8, 2, 128, 16, 1), (5, 1, 64, 32, 37), (4, 4, 256, 16, 130), (6, 2, 128, 64, 2049),
                                          (40, 8, 128, 16, 48)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("form", ["dense", "strided", "in place", "no queries", "unturned"])
def test_append_paged(hq, hkv, d, bs, t, inter, form):
    import torch
    r = np.random.default_rng(t + d)
    nb = -(-t // bs) + 5
    inv = inv_freq_table(d, 5e5)
    x = store(r.standard_normal((t, hq + 2 * hkv, d)) * 3, "bf16")
    pos = r.integers(0, 1 << 20, t)
    pos[0] = 2 ** 31 - 1                                        # the farthest position there is
    slots = r.permutation(nb * bs)[:t].astype(np.int64)
    if t > 3:
        slots[2], slots[3] = -1, nb * bs                        # left out: nothing of them is written
    pools = [torch.full((nb, hkv, bs, d), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    xd = to_dev(x)
    parts = [xd[:, :hq], xd[:, hq:hq + hkv], xd[:, hq + hkv:]]
    if form != "strided":
        parts = [y.contiguous() for y in parts]
    q = None if form in ("no queries", "unturned") else parts[0]
    q_out = None if q is None else q if form == "in place" else torch.full((t, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    p = ea.make_params(1, hq, hkv, d, ea.EA_BF16, rope_layout=int(inter))
    rows = ea.make_new_rows(q, parts[1], parts[2], i32(pos), None if form == "unturned" else to_dev(inv))
    table = i32([[0]])
    ea.append_paged(p, rows, to_dev(slots), pools[0], pools[1], ea.make_paged(table, bs, nb), q_out)
    torch.cuda.synchronize()
    stored = (slots >= 0) & (slots < nb * bs)
    xf = widen(x)
    got = [widen(to_host(y)).transpose(0, 2, 1, 3).reshape(nb * bs, hkv, d) for y in pools]
    if form == "unturned":
        assert np.array_equal(got[0][slots[stored]], xf[stored, hq:hq + hkv])
    else:
        check_rotated(got[0][slots[stored]], xf[stored, hq:hq + hkv], pos[stored], inv, inter, "bf16")
    assert np.array_equal(got[1][slots[stored]], xf[stored, hq + hkv:])
    rest = np.setdiff1d(np.arange(nb * bs), slots[stored])
    assert (got[0][rest] == 5.0).all() and (got[1][rest] == 5.0).all()
    if q is not None:
        qo = widen(to_host(q_out))
        check_rotated(qo[stored], xf[stored, :hq], pos[stored], inv, inter, "bf16")
        assert np.array_equal(qo[~stored], xf[~stored, :hq] if form == "in place" else np.full_like(qo[~stored], 7.0))


@pytest.mark.parametrize("dt,d,hq,hkv", [("bf16", 128, 8, 2), ("bf16", 64, 4, 2), ("f32", 64, 4, 2), ("f32", 256, 3, 3), ("fp8", 128, 8, 2), ("fp8", 256, 2, 1)])
@pytest.mark.parametrize("inter", [False, True])
def test_append_to_heads_of_different_lengths(dt, d, hq, hkv, inter):
    import torch
    r = np.random.default_rng(d + hkv)
    B, cap = 4, 50
    m = np.array([1, 7, 0, 30])
    cu = np.concatenate([[0], np.cumsum(m)])
    t, room = int(cu[-1]), int(cu[-1]) + 9                      # rows behind the last sequence
    lens = np.stack([r.integers(mm, cap + 1, hkv) for mm in m])
    lens[1, 0] = 3                                              # fewer rows than new tokens: the first four have no row
    lens[3, -1] = cap + 2                                       # and the last two none here
    st = "f32" if dt == "f32" else "bf16"
    x = store(r.standard_normal((room, hq + 2 * hkv, d)) * 2, st)
    pos, inv = r.integers(0, 200000, room), inv_freq_table(d, 1e4)
    xd = to_dev(x)
    rows = ea.make_new_rows(xd[:, :hq], xd[:, hq:hq + hkv], xd[:, hq + hkv:], i32(pos), to_dev(inv))
    q_out = torch.full((room, hq, d), 7.0, dtype=xd.dtype, device="cuda")
    p = ea.make_params(B, hq, hkv, d, kind(st), rope_layout=int(inter))
    if dt == "fp8":
        cache = [torch.full((B, hkv, cap, d), 0x38, dtype=torch.uint8, device="cuda") for _ in range(2)]
        scale = [(r.random((B, hkv)) * 0.05 + 0.004).astype(np.float32) for _ in range(2)]     # some saturate
        ea.append_fp8(p, rows, i32(cu), i32(lens), cache[0], cache[1], to_dev(scale[0]), to_dev(scale[1]), cap, q_out)
        got = [X.fp8_e4m3_decode(to_host(c)) for c in cache]
        empty = X.fp8_e4m3_decode(np.array([0x38], dtype=np.uint8))[0]
    else:
        cache = [torch.full((B, hkv, cap, d), 5.0, dtype=xd.dtype, device="cuda") for _ in range(2)]
        ea.append(p, rows, i32(cu), i32(lens), cache[0], cache[1], cap, q_out)
        got, empty = [widen(to_host(c)) for c in cache], 5.0
    torch.cuda.synchronize()
    xf = widen(x)
    want_k, v = S.rotate(xf[:, hq:hq + hkv], pos, inv, inter), xf[:, hq + hkv:]
    slack = 2.0 ** -21 * pair_length(xf[:, hq:hq + hkv], inter)
    for b in range(B):
        for h in range(hkv):
            written = np.zeros(cap, dtype=bool)
            for i in range(m[b]):
                row, tok = lens[b, h] - m[b] + i, cu[b] + i
                if not 0 <= row < cap:
                    continue
                written[row] = True
                if dt == "fp8":
                    for c, w, s, more in ((got[0], want_k, scale[0], slack[tok, h]), (got[1], v, scale[1], 0.0)):
                        y = np.clip(w[tok, h] / float(s[b, h]), -448, 448)
                        # half a step: 2^-4 of a normal value, half of 2^-9 of those below 2^-6
                        tol = np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10) + more / float(s[b, h]) + 2.0 ** -22 * np.abs(y)
                        assert (np.abs(c[b, h, row] - y) <= tol).all()
                else:
                    assert (np.abs(got[0][b, h, row] - want_k[tok, h]) <= HALF[dt] * np.abs(want_k[tok, h]) + slack[tok, h]).all()
                    assert np.array_equal(got[1][b, h, row], v[tok, h])
            assert (got[0][b, h, ~written] == empty).all() and (got[1][b, h, ~written] == empty).all()
    qo = widen(to_host(q_out))
    check_rotated(qo[:t], xf[:t, :hq], pos[:t], inv, inter, st)
    assert (qo[t:] == 7.0).all()


# -------------------------------------------------------------------------------------- attention
def attend_bounds(want, dt, n, d):
    """Bounds of |out - exact| and |lse - exact|.

    A logit is a sum of d products in fp32, of which each and each sum rounds once: off by at most delta = (d + 8) 2^-24 max
    sum |q_c k_c| / sqrt(d), and two more roundings of it on the way to the exponent; a weight exp2f gives is off by 2^-22 more.
    A weight's relative error e reaches the weighted sum as e * spread (the weighted mean of |v|) and the sum of weights as e, so
    2 e * spread together.  Weights reach the second product rounded to the stored type: spread * HALF.  fp32 sums of n terms over
    four wavefronts' lanes and joined pieces: (n / 8 + 64) 2^-24 each.  The result is rounded once."""
    out, lse, spread, logit = want
    delta = (d + 8) * 2.0 ** -24 * logit + 2.0 ** -22 * (1 + logit)
    sums = (n / 8 + 64) * 2.0 ** -24
    e = 2 * (delta + sums)
    tol = (e[..., None] + (HALF[dt] if dt == "bf16" else 0.0)) * spread + HALF[dt] * np.abs(out) * 1.01 + 1e-37
    seen = np.isfinite(lse)
    return tol, delta + sums + 2.0 ** -22 * np.abs(np.where(seen, lse, 0.0)) + 2.0 ** -22


def make_heads(r, lens, d, dt, cap):
    """K, V [B, H, cap, d] with NaN from each head's length on, as stored and as fp64 lists."""
    B, H = lens.shape
    s, mu = np.exp(0.5 * r.standard_normal((H, d))), 1.4 * r.standard_normal((H, d))
    k = store(r.standard_normal((B, H, cap, d)) * s[None, :, None] + mu[None, :, None], dt)
    v = store(r.standard_normal((B, H, cap, d)) * np.exp(0.5 * r.standard_normal((B, H, cap, 1))), dt)
    for b in range(B):
        for h in range(H):
            k[b, h, lens[b, h]:] = v[b, h, lens[b, h]:] = MARK[dt]
    return k, v


def attend_inputs(seed, hq, hkv, d, dt, lens, m, room=0, cap=None):
    r = np.random.default_rng(seed)
    lens = np.asarray(lens)
    if lens.ndim == 1:
        lens = np.repeat(lens[:, None], hkv, axis=1)
    cap = int(max(lens.max(), 1)) if cap is None else cap
    k, v = make_heads(r, lens, d, dt, cap)
    cu = np.concatenate([[0], np.cumsum(m)])
    q = store(r.standard_normal((int(cu[-1]) + room, hq, d)), dt)
    return q, cu, k, v, lens


def check_attend(got, lse, q, cu, k, v, lens, dt):
    t, d = int(cu[-1]), q.shape[-1]
    kf, vf = widen(k) if k.dtype != np.float64 else k, widen(v) if v.dtype != np.float64 else v
    want = S.attend(widen(q), cu, kf, vf, lens)
    tol, tol_lse = attend_bounds(want, dt, int(lens.max()), d)
    out, ref = widen(got)[:t], want[0][:t]
    assert np.isfinite(out).all()
    worst = np.abs(out - ref) / tol[:t]
    assert worst.max() <= 1, worst.max()
    empty = ~np.isfinite(want[1][:t])
    assert (out[empty] == 0).all()
    if lse is not None:
        assert (lse[:t][empty] == -np.inf).all()
        assert (np.abs(lse[:t] - want[1][:t])[~empty] <= tol_lse[:t][~empty]).all()


def outputs(q, dt):
    import torch
    t, hq, d = q.shape
    out = torch.full((t, hq, d), 7.0, dtype=torch.bfloat16 if dt == "bf16" else torch.float32, device="cuda")
    return out, torch.full((t, hq), 7.0, dtype=torch.float32, device="cuda")


def run_paged(q, cu, k, v, lens, bs, n=None, max_new=None, seed=0, q_stride=0, with_lse=True):
    import torch
    B, hkv, cap, d = k.shape
    p = ea.make_params(B, q.shape[1], hkv, d, ea.EA_BF16)
    kp, vp, table, nb = make_block_pools(k, v, bs, seed)
    for b in range(B):                                         # entries behind a sequence's blocks lead nowhere
        table[b, -(-int(lens[b, 0]) // bs):] = -99
    t = i32(table)
    pg = ea.make_paged(t, bs, nb)
    n = table.shape[1] * bs if n is None else n
    step = ea.make_step(i32(cu), q.shape[0], int(np.diff(cu).max()) or 1 if max_new is None else max_new, q_stride)
    cud = i32(cu)
    step.cu_tokens = cud.data_ptr()
    out, lse = outputs(q, "bf16")
    ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
    ea.attend_paged(p, to_dev(q), step, to_dev(kp), to_dev(vp), pg, i32(lens[:, 0]), n, out, lse if with_lse else None, ws)
    torch.cuda.synchronize()
    return to_host(out), lse.cpu().numpy()


SHAPES = [(8, 2, 128), (5, 1, 128), (16, 1, 128), (14, 2, 64), (4, 2, 256), (24, 1, 128), (64, 1, 64), (40, 2, 256)]


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("bs", [16, 32, 256])
def test_single_tokens_over_pools(hq, hkv, d, bs):
    """Lengths on both sides of a tile's, a group's and a share's end, an empty cache and an absent sequence among them."""
    lens = [1, 15, 16, 17, 31, 33, 127, 128, 129, 0, 300, 1000, 1025, 40, 2500]
    m = [1] * len(lens)
    m[13] = 0
    q, cu, k, v, L = attend_inputs(hq + d, hq, hkv, d, "bf16", lens, m, room=3)
    got, lse = run_paged(q, cu, k, v, L, bs)
    check_attend(got, lse, q, cu, k, v, L, "bf16")
    assert (widen(got)[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("m", [[2, 3, 1, 4], [33, 1, 0, 70], [64, 64, 5, 200], [9, 40, 300, 2]])
def test_stretches_over_pools(hq, hkv, d, m):
    """Stretches of new tokens, with what came before or without, and one with fewer rows than tokens (the first see nothing)."""
    lens = [max(m[0] - 1, 0), 500 + m[1], 77, 1300]
    q, cu, k, v, L = attend_inputs(sum(m) + d, hq, hkv, d, "bf16", lens, m, room=2)
    got, lse = run_paged(q, cu, k, v, L, 16)
    check_attend(got, lse, q, cu, k, v, L, "bf16")
    assert (widen(got)[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("dt,hq,hkv,d", [("bf16", 8, 2, 128), ("bf16", 6, 2, 64), ("bf16", 4, 2, 256), ("f32", 4, 2, 64),
                                        ("f32", 7, 1, 128), ("f32", 3, 3, 256), ("f32", 64, 1, 64)])
@pytest.mark.parametrize("m", [[1, 1, 1], [3, 0, 1], [40, 1, 130]])
def test_heads_of_different_lengths(dt, hq, hkv, d, m):
    import torch
    r = np.random.default_rng(d + hq)
    lens = r.integers(0, 900, (3, hkv))
    lens[0, 0], lens[2, -1], lens[1, 0] = 0, 1500, 1
    cap = 1501                                                 # rows of 16 do not end with the tensor
    q, cu, k, v, L = attend_inputs(hq, hq, hkv, d, dt, lens, m, cap=cap)
    p = ea.make_params(3, hq, hkv, d, kind(dt))
    cud = i32(cu)
    for n, lse_too in ((cap, True), (1500, False)):
        step = ea.make_step(cud, q.shape[0], max(m))
        out, lse = outputs(q, dt)
        ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
        ea.attend(p, to_dev(q), step, to_dev(k), to_dev(v), i32(L), n, cap, out, lse if lse_too else None, ws)
        torch.cuda.synchronize()
        check_attend(to_host(out), lse.cpu().numpy() if lse_too else None, q, cu, k, v, L, dt)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (5, 1, 128), (24, 1, 128), (4, 2, 256), (20, 1, 256)])
@pytest.mark.parametrize("m", [[1, 1], [2, 6], [50, 200]])
@pytest.mark.parametrize("scaled", [True, False])
def test_fp8_caches(hq, hkv, d, m, scaled):
    import torch
    r = np.random.default_rng(d + hq)
    lens = r.integers(200, 1300, (2, hkv))
    lens[0, 0] = 33
    q, cu, k, v, L = attend_inputs(hq, hq, hkv, d, "f32", lens, m)
    q = store(q.astype(np.float64), "bf16")
    k8, ks = quantize_fp8(np.nan_to_num(k.astype(np.float64)))
    v8, vs = quantize_fp8(np.nan_to_num(v.astype(np.float64)))
    for b in range(2):
        for h in range(hkv):
            k8[b, h, L[b, h]:] = v8[b, h, L[b, h]:] = 0x7F     # NaN
    if not scaled:
        ks[:], vs[:] = 1.0, 1.0
        q = store(widen(q) * 0.05, "bf16")                     # bytes of up to 400: logits of the same size as with scales
    p = ea.make_params(2, hq, hkv, d, ea.EA_BF16)
    cud = i32(cu)
    step = ea.make_step(cud, q.shape[0], max(m))
    cap = k.shape[2]
    out, lse = outputs(q, "bf16")
    ws = torch.empty(ea.attend_workspace_bytes(p, step, cap), dtype=torch.uint8, device="cuda").fill_(0xFF)
    ea.attend_fp8(p, to_dev(q), step, to_dev(k8), to_dev(v8), to_dev(ks) if scaled else None, to_dev(vs) if scaled else None,
                  i32(L), cap, cap, out, lse, ws)
    torch.cuda.synchronize()
    kf, vf = (X.fp8_e4m3_decode(x) * s.astype(np.float64)[:, :, None, None] for x, s in ((k8, ks), (v8, vs)))
    check_attend(to_host(out), lse.cpu().numpy(), q, cu, kf, vf, L, "bf16")


# -------------------------------------------------------------------------------- they run together
class Loop:
    """A batch of sequences over block pools: steps of new tokens, and compress passes in between.  The oracle keeps every
    sequence's rows in numpy; the GPU's state is never corrected from it."""

    def __init__(self, B, hq, hkv, d, bs, max_blocks, num_blocks, seed):
        import torch
        self.r, self.B, self.hq, self.hkv, self.d, self.bs = np.random.default_rng(seed), B, hq, hkv, d, bs
        self.p = ea.make_params(B, hq, hkv, d, ea.EA_BF16)
        self.table = torch.full((B, max_blocks), -1, dtype=torch.int32, device="cuda")
        self.pg = ea.make_paged(self.table, bs, num_blocks)
        self.pools = [torch.full((num_blocks, hkv, bs, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        self.free = to_dev(self.r.permutation(num_blocks).astype(np.int32))
        self.count, self.lens = [i32([num_blocks]), i32([0])], [i32([0] * B), i32([0] * B)]
        self.inv = inv_freq_table(d, 5e5)
        self.invd = to_dev(self.inv)
        self.seen, self.rows = np.zeros(B, dtype=int), [[np.zeros((0, hkv, d)), np.zeros((0, hkv, d))] for _ in range(B)]
        self.n = max_blocks * bs

    def step(self, m, room=0):
        import torch
        m = np.asarray(m)
        t = int(m.sum()) + room
        qkv = store(self.r.standard_normal((t, self.hq + 2 * self.hkv, self.d)) * 1.5, "bf16")
        new = (self.lens[0].cpu().numpy() + m)
        cu, slots, pos = (torch.full(s, -5, dtype=x, device="cuda") for s, x in (((self.B + 1,), torch.int32), ((t,), torch.int64), ((t,), torch.int32)))
        pos.fill_(0)
        ea.block_tables(self.p, self.pg, self.lens[0], i32(new), self.free, self.count[0], self.lens[1], self.count[1], cu, t, slots, pos,
                        i32(self.seen))
        x = to_dev(qkv)
        rows = ea.make_new_rows(x[:, :self.hq], x[:, self.hq:self.hq + self.hkv], x[:, self.hq + self.hkv:], pos, self.invd)
        q = torch.zeros(t, self.hq, self.d, dtype=torch.bfloat16, device="cuda")
        ea.append_paged(self.p, rows, slots, self.pools[0], self.pools[1], self.pg, q)
        st = ea.make_step(cu, t, int(m.max()))
        out, lse = outputs(q, "bf16")
        ws = torch.empty(ea.attend_workspace_bytes(self.p, st, self.n), dtype=torch.uint8, device="cuda")
        ea.attend_paged(self.p, q, st, self.pools[0], self.pools[1], self.pg, self.lens[1], self.n, out, lse, ws)
        torch.cuda.synchronize()
        self.lens.reverse(), self.count.reverse()
        # the oracle: what stands in the cache is what the call stored, to within its own rounding
        xf, at = widen(qkv), np.concatenate([[0], np.cumsum(m)])
        assert np.array_equal(cu.cpu().numpy(), at) and np.array_equal(self.lens[0].cpu().numpy(), new)
        kp, vp, tab = (widen(to_host(y)) if y.dtype == torch.bfloat16 else to_host(y) for y in (*self.pools, self.table))
        used = []
        for b in range(self.B):
            s = slice(at[b], at[b + 1])
            k = S.rotate(xf[s, self.hq:self.hq + self.hkv], self.seen[b] + np.arange(m[b]), self.inv, False)
            blocks = tab[b, :-(-int(new[b]) // self.bs)]
            used += blocks.tolist()
            have = [X.paged_rows(z, blocks[None], int(new[b]))[0].transpose(1, 0, 2) if new[b] else np.zeros((0, self.hkv, self.d)) for z in (kp, vp)]
            old = len(self.rows[b][0])
            assert np.array_equal(have[0][:old], self.rows[b][0]) and np.array_equal(have[1][:old], self.rows[b][1])
            if m[b]:
                check_rotated(have[0][old:], xf[s, self.hq:self.hq + self.hkv], self.seen[b] + np.arange(m[b]), self.inv, False, "bf16")
                assert np.array_equal(have[1][old:], xf[s, self.hq + self.hkv:])
            self.rows[b] = have
        assert len(set(used)) == len(used) and len(used) + int(self.count[0]) == len(self.free)
        assert sorted(used + self.free[:int(self.count[0])].tolist()) == list(range(len(self.free)))
        self.seen += m
        L = np.repeat(new[:, None], self.hkv, axis=1)
        lists = [[[self.rows[b][i][:, h] for h in range(self.hkv)] for b in range(self.B)] for i in range(2)]
        want = S.attend(widen(to_host(q)), at, lists[0], lists[1], L)
        tol, tol_lse = attend_bounds(want, "bf16", int(new.max()), self.d)
        n = int(at[-1])
        assert bool((np.abs(widen(to_host(out)) - want[0])[:n] <= tol[:n]).all())
        assert bool((np.abs(lse.cpu().numpy() - want[1])[:n] <= tol_lse[:n]).all())
        return out

    def compress(self, n_keep):
        """All sequences hold as many rows as each other: a pass over the pools, then the blocks behind go back."""
        import torch
        n = int(self.lens[0][0])
        w = 16
        win = to_dev(store(self.r.standard_normal((self.B, self.hq, w, self.d)), "bf16"))
        ws = torch.empty(ea.workspace_bytes(self.p, n, w), dtype=torch.uint8, device="cuda")
        idx = torch.zeros(self.B, self.hkv, n_keep, dtype=torch.int32, device="cuda")
        ea.compress_layer_paged(self.p, win, w, int(self.seen[0]) - w, self.invd, int(self.seen[0]), self.pools[0], self.pools[1], self.pg, n, n_keep,
                                0, None, idx, None, ws)
        cu = torch.zeros(self.B + 1, dtype=torch.int32, device="cuda")
        ea.block_tables(self.p, self.pg, self.lens[0], i32([n_keep] * self.B), self.free, self.count[0], self.lens[1], self.count[1], cu)
        torch.cuda.synchronize()
        self.lens.reverse(), self.count.reverse()
        assert (self.lens[0] == n_keep).all() and (cu == 0).all()
        kept = idx.cpu().numpy()
        for b in range(self.B):
            self.rows[b] = [np.stack([z[kept[b, h], h] for h in range(self.hkv)], axis=1) for z in self.rows[b]]


@pytest.mark.parametrize("B,hq,hkv,d,bs", [(3, 8, 2, 128, 16), (2, 5, 1, 64, 32), (2, 4, 2, 256, 16)])
def test_a_loop_of_steps_and_compress_passes(B, hq, hkv, d, bs):
    s = Loop(B, hq, hkv, d, bs, max_blocks=40, num_blocks=B * 30 + 2, seed=d)
    s.step([200] * B)                          # the prompts
    for _ in range(3):
        s.step([1] * B, room=5)                # single tokens, with room behind them
    s.compress(90)                             # rows are no positions from here on
    s.step([3] * B)
    s.step([0] + [7] * (B - 1))                # one sequence waits
    s.step([41] + [34] * (B - 1))
    s.compress(64)
    s.step([1] * B)


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
def test_generation_over_an_adaptive_cache(dt):
    """compress_layer_adaptive leaves heads of different lengths; steps go on from there."""
    import torch
    r = np.random.default_rng(5)
    B, hq, hkv, d, n, cap, w = 2, 8, 4, 128, 600, 700, 16
    inv = inv_freq_table(d, 5e5)
    p = ea.make_params(B, hq, hkv, d, ea.EA_BF16)
    if dt == "bf16":
        k, v = (to_dev(store(r.standard_normal((B, hkv, cap, d)), "bf16")) for _ in range(2))
        win = to_dev(store(r.standard_normal((B, hq, w, d)), "bf16"))
        ws = torch.empty(ea.workspace_bytes(p, n, w), dtype=torch.uint8, device="cuda")
        idx, lens = torch.zeros(B, hkv, n, dtype=torch.int32, device="cuda"), torch.zeros(B, hkv, dtype=torch.int32, device="cuda")
        ea.compress_layer_adaptive(p, win, w, n - w, to_dev(inv), n, k, v, n, cap, 200, 20, None, idx, lens, ws)
        assert len(set(lens.flatten().tolist())) > 1
        scale = [None, None]
    else:
        k, v = (to_dev(r.integers(0, 0x77, (B, hkv, cap, d)).astype(np.uint8)) for _ in range(2))
        lens = i32(r.integers(100, 600, (B, hkv)))
        scale = [to_dev((r.random((B, hkv)) * 0.02 + 0.01).astype(np.float32)) for _ in range(2)]
    seen = n
    for m in ([1, 1], [5, 2], [1, 0], [40, 30]):
        t = sum(m)
        cu = i32(np.concatenate([[0], np.cumsum(m)]))
        lens = lens + i32(m)[:, None]
        x = to_dev(store(r.standard_normal((t, hq + 2 * hkv, d)), "bf16"))
        pos = i32(np.concatenate([seen + np.arange(a) for a in m]))
        q = torch.zeros(t, hq, d, dtype=torch.bfloat16, device="cuda")
        rows = ea.make_new_rows(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], pos, to_dev(inv))
        st = ea.make_step(cu, t, max(m))
        out, lse = outputs(q, "bf16")
        ws = torch.empty(ea.attend_workspace_bytes(p, st, cap), dtype=torch.uint8, device="cuda")
        if dt == "bf16":
            ea.append(p, rows, cu, lens, k, v, cap, q)
            ea.attend(p, q, st, k, v, lens, cap, cap, out, lse, ws)
        else:
            ea.append_fp8(p, rows, cu, lens, k, v, scale[0], scale[1], cap, q)
            ea.attend_fp8(p, q, st, k, v, scale[0], scale[1], lens, cap, cap, out, lse, ws)
        torch.cuda.synchronize()
        if dt == "bf16":
            kf, vf = widen(to_host(k)), widen(to_host(v))
        else:
            kf, vf = (X.fp8_e4m3_decode(to_host(z)) * to_host(s).astype(np.float64)[:, :, None, None] for z, s in ((k, scale[0]), (v, scale[1])))
        check_attend(to_host(out), lse.cpu().numpy(), to_host(q), cu.cpu().numpy(), kf, vf, lens.cpu().numpy(), "bf16")
        seen += max(m)


def test_a_step_in_a_graph_follows_the_lengths():
    """One captured step, replayed over lengths that grow on the device, against eager calls; eager work on the same workspace and
    other tensors in between."""
    import torch
    r = np.random.default_rng(11)
    B, hq, hkv, d, bs, mb = 5, 8, 2, 128, 16, 40
    nb = B * mb + 3
    p = ea.make_params(B, hq, hkv, d, ea.EA_BF16)
    inv = to_dev(inv_freq_table(d, 5e5))
    state = {}
    for name in ("graph", "eager"):
        g = np.random.default_rng(3)
        table = torch.full((B, mb), -1, dtype=torch.int32, device="cuda")
        state[name] = dict(table=table, pg=ea.make_paged(table, bs, nb), pools=[torch.zeros(nb, hkv, bs, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)],
                           free=to_dev(g.permutation(nb).astype(np.int32)), count=i32([nb]), lens=i32([0, 3, 100, 15, 400]) * 0, seen=i32([0] * B),
                           more=i32([1] * B), len_out=i32([0] * B), count_out=i32([0]), cu=i32([0] * (B + 1)), slots=torch.zeros(60, dtype=torch.int64, device="cuda"),
                           pos=torch.zeros(60, dtype=torch.int32, device="cuda"), x=torch.zeros(60, hq + 2 * hkv, d, dtype=torch.bfloat16, device="cuda"),
                           q=torch.zeros(60, hq, d, dtype=torch.bfloat16, device="cuda"), out=torch.zeros(60, hq, d, dtype=torch.bfloat16, device="cuda"),
                           lse=torch.zeros(60, hq, device="cuda"), want=i32([0] * B))

    def prepare(s, ws_of):
        st = ea.make_step(s["cu"], 60, 60)
        s["st"], s["ws"] = st, ws_of if ws_of is not None else torch.empty(ea.attend_workspace_bytes(p, st, mb * bs), dtype=torch.uint8, device="cuda")

    def go(s):
        torch.add(s["lens"], s["more"], out=s["want"])
        ea.block_tables(p, s["pg"], s["lens"], s["want"], s["free"], s["count"], s["len_out"], s["count_out"], s["cu"], 60, s["slots"], s["pos"], s["seen"])
        rows = ea.make_new_rows(s["x"][:, :hq], s["x"][:, hq:hq + hkv], s["x"][:, hq + hkv:], s["pos"], inv)
        ea.append_paged(p, rows, s["slots"], s["pools"][0], s["pools"][1], s["pg"], s["q"])
        ea.attend_paged(p, s["q"], s["st"], s["pools"][0], s["pools"][1], s["pg"], s["len_out"], mb * bs, s["out"], s["lse"], s["ws"])
        s["lens"].copy_(s["len_out"])
        s["count"].copy_(s["count_out"])
        s["seen"].add_(s["more"])

    prepare(state["graph"], None)
    prepare(state["eager"], state["graph"]["ws"])              # both use one workspace, one after the other
    side = torch.cuda.Stream()
    s = state["graph"]
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        go(s)
    torch.cuda.synchronize()
    for more in ([20, 3, 0, 30, 1], [1] * 5, [1] * 5, [0, 1, 50, 1, 1], [1] * 5, [2, 2, 2, 2, 2], [1] * 5):
        x = to_dev(store(r.standard_normal((60, hq + 2 * hkv, d)), "bf16"))
        for z in state.values():
            z["x"].copy_(x)
            z["more"].copy_(i32(more))
        state["graph"]["ws"].fill_(0xA5)                       # undefined between calls
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        go(state["eager"])
        torch.cuda.synchronize()
        n = sum(more)
        for key in ("table", "free", "count", "lens", "cu", "slots", "seen"):
            assert torch.equal(state["graph"][key], state["eager"][key]), key
        for key in ("q", "out", "lse"):
            assert torch.equal(state["graph"][key][:n], state["eager"][key][:n]), key


def test_calls_on_side_streams():
    """Two calls at once, each with a workspace of its own, give what they give alone."""
    import torch
    jobs = []
    for seed, m in ((1, [1, 1, 1]), (2, [30, 1, 64])):
        q, cu, k, v, L = attend_inputs(seed, 8, 2, 128, "bf16", [700, 1300, 90], m)
        jobs.append((run_paged(q, cu, k, v, L, 16, seed=seed), (q, cu, k, v, L)))
    p = ea.make_params(3, 8, 2, 128, ea.EA_BF16)
    streams, keep = [torch.cuda.Stream() for _ in range(2)], []
    for (_, (q, cu, k, v, L)), seed in zip(jobs, (1, 2)):
        kp, vp, table, nb = make_block_pools(k, v, 16, seed)
        t, cud, ld = i32(table), i32(cu), i32(L[:, 0])
        pg, st = ea.make_paged(t, 16, nb), ea.make_step(cud, q.shape[0], int(np.diff(cu).max()))
        out, lse = outputs(q, "bf16")
        n = table.shape[1] * 16
        ws = torch.empty(ea.attend_workspace_bytes(p, st, n), dtype=torch.uint8, device="cuda")
        keep.append((to_dev(q), st, to_dev(kp), to_dev(vp), pg, ld, n, out, lse, ws, t))
    torch.cuda.synchronize()
    for _ in range(3):
        for s, (q, st, kp, vp, pg, ld, n, out, lse, ws, _t) in zip(streams, keep):
            ea.attend_paged(p, q, st, kp, vp, pg, ld, n, out, lse, ws, stream=s)
    torch.cuda.synchronize()
    for ((want, want_lse), _), k in zip(jobs, keep):
        assert np.array_equal(to_host(k[7]), want) and np.array_equal(k[8].cpu().numpy(), want_lse)


# ------------------------------------------------------------------- values that are not finite, and what follows from them
def spoil(k, v, lens, m, dt, where):
    """Values that are not finite in rows of the step's own tokens: an infinity of either sign and a NaN, in different channels of
    different heads."""
    r = np.random.default_rng(8)
    k, v = k.copy(), v.copy()
    put = {"bf16": (0x7F80, 0xFF80, 0x7FC0), "f32": (np.inf, -np.inf, np.nan)}[dt]
    B, H = lens.shape
    for b in range(B):
        if m[b] < 2:
            continue
        for h in range(H):
            for x in put:
                row = lens[b, h] - m[b] + int(r.integers(0, m[b]))
                if row >= 0:
                    v[b, h, row, int(r.integers(0, v.shape[-1]))] = x
            if where == "keys":                      # a key that is not finite, of the last token: the others do not see it
                k[b, h, lens[b, h] - 1, 3] = put[2]
    return k, v


@pytest.mark.parametrize("dt,hq,hkv,d,m", [("bf16", 8, 2, 128, [2, 3, 1]), ("bf16", 24, 1, 128, [1, 2, 1]), ("bf16", 6, 2, 64, [5, 2, 40]),
                                          ("bf16", 8, 2, 128, [100, 1, 70]), ("bf16", 4, 2, 256, [3, 90, 2]), ("bf16", 16, 1, 64, [33, 200, 7]),
                                          ("f32", 4, 2, 64, [2, 30, 1]), ("f32", 6, 2, 128, [4, 1, 170]), ("f32", 256, 4, 256, [2, 9, 70]),
                                          ("fp8", 8, 2, 128, [3, 2, 1]), ("fp8", 4, 2, 256, [60, 150, 2])])
@pytest.mark.parametrize("where", ["values", "keys"])
def test_what_a_token_does_not_see_does_not_matter(dt, hq, hkv, d, m, where):
    """A value that is not finite reaches the tokens that see its row and no others: theirs are what they are without it."""
    import torch
    r = np.random.default_rng(hq)
    lens = r.integers(max(m), 400, (3, hkv))
    lens[2, -1] = m[2]
    q, cu, k, v, L = attend_inputs(hq + d, hq, hkv, d, "f32" if dt == "f32" else "bf16", lens, m)
    p = ea.make_params(3, hq, hkv, d, kind("f32" if dt == "f32" else "bf16"))
    cud, cap = i32(cu), k.shape[2]
    step = ea.make_step(cud, q.shape[0], max(m))

    def run(k, v):
        out, lse = outputs(q, "f32" if dt == "f32" else "bf16")
        ws = torch.empty(ea.attend_workspace_bytes(p, step, cap), dtype=torch.uint8, device="cuda").fill_(0xFF)
        if dt == "fp8":
            ea.attend_fp8(p, to_dev(q), step, to_dev(k), to_dev(v), None, None, i32(L), cap, cap, out, lse, ws)
        else:
            ea.attend(p, to_dev(q), step, to_dev(k), to_dev(v), i32(L), cap, cap, out, lse, ws)
        torch.cuda.synchronize()
        return widen(to_host(out)), lse.cpu().numpy()
    if dt == "fp8":
        k, v = (r.integers(0, 0x60, k.shape).astype(np.uint8) for _ in range(2))
        bad_k, bad_v = k.copy(), v.copy()
        for b in range(3):
            for h in range(hkv):
                if m[b] > 1:
                    bad_v[b, h, L[b, h] - 1 - int(r.integers(0, m[b])), 5] = 0x7F
                    if where == "keys":
                        bad_k[b, h, L[b, h] - 1, 3] = 0x7F
    else:
        bad_k, bad_v = spoil(k, v, L, m, dt, where)
    clean, clean_lse = run(k, v)
    got, lse = run(bad_k, bad_v)
    if dt == "fp8":
        no = (bad_v & 0x7F) == 0x7F
        vf = np.where(no, np.nan, X.fp8_e4m3_decode(np.where(no, 0, bad_v).astype(np.uint8)))
    else:
        vf = widen(bad_v)
    for b in range(3):
        for i in range(m[b]):
            for x in range(hq):
                h = x // (hq // hkv)
                n, t = L[b, h] - (m[b] - 1 - i), cu[b] + i
                seen = vf[b, h, :max(n, 0)]
                if where == "keys" and m[b] > 1 and i == m[b] - 1:
                    assert np.isnan(got[t, x]).all()
                    continue
                # an infinity times a weight whose lower part is zero is a NaN already: not finite is all that is promised
                fine = np.isfinite(seen).all(0)
                assert not np.isfinite(got[t, x][~fine]).any()
                assert np.array_equal(got[t, x][fine], clean[t, x][fine])
                assert lse[t, x] == clean_lse[t, x]
