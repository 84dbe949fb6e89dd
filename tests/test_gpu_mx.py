"""Pools of quantised rows on the GPU against their fp64 oracle: rows as they are written, read back and attended to.

Tolerances, derived before the first run.  A stored element is the nearest one to the exact key rounded to fp32, which is off by 2^-24
and as much again where the rounding goes the other way: elements of the key moved by 2^-23 either way are right, too.  Values are
not rotated: their bytes are the oracle's.  Reading back is exact but for numbers below 2^-126, which may be zeros.  Attention:
`attend_bounds` of the step's tests, on the values that the bytes stand for, since those reach the products exactly."""
import numpy as np
import pytest

from ea_inputs import bf16_bits_from_f64, inv_freq_table, widen
from ea_inputs.torch_io import to_dev, to_host
from oracle import ea_draft as D
from oracle import ea_step as S
import paper_2510_00636_amd as ea
from tests.test_gpu_step import attend_bounds, check_attend, check_rotated, i32, outputs, store

pytestmark = pytest.mark.gpu

BITS = {8: ea.EA_MXFP8, 4: ea.EA_MXFP4}


def as_pools(codes, e, bs, bits, table, nb):
    """codes [B, H, cap, d] and exponents [B, H, cap, d / 32] as pools behind a table; what belongs to nobody is NaN"""
    B, H, cap, d = codes.shape
    pool = np.full((nb, H, bs, d), 2 ** bits - 1, dtype=np.int64)
    scale = np.full((nb, H, bs, d // 32), 255, dtype=np.uint8)
    for b in range(B):
        for j in range(-(-cap // bs)):
            n = min(bs, cap - j * bs)
            pool[table[b, j], :, :n] = codes[b, :, j * bs:j * bs + n]
            scale[table[b, j], :, :n] = e[b, :, j * bs:j * bs + n]
    return D.packed(pool, bits), scale


class Mx:
    """Random rows, quantised, in pools: the handles of a call and the values that the bytes stand for."""

    def __init__(self, seed, lens, hkv, d, bs, bits, spread=0):
        r = np.random.default_rng(seed)
        self.lens, B, cap = np.asarray(lens), len(lens), int(max(max(lens), 1))
        self.max_blocks = -(-cap // bs)
        self.nb = B * self.max_blocks + 3
        table = r.permutation(self.nb)[:B * self.max_blocks].reshape(B, self.max_blocks).astype(np.int32)
        self.codes, self.e, self.val = [], [], []
        for i in range(2):
            mean = 1.4 * r.standard_normal((hkv, 1, d)) if i == 0 else 0.0
            x = r.standard_normal((B, hkv, cap, d)) * np.exp(0.5 * r.standard_normal((B, hkv, cap, 1))) + mean
            if spread:
                x = x * 2.0 ** r.integers(-spread, spread + 1, (B, hkv, cap, d // 32)).repeat(32, axis=-1)
            codes, e = D.quantise(x, bits)
            val = D.values(codes, e, bits)
            for b in range(B):                                 # rows behind a length are NaN, as stored
                codes[b, :, lens[b]:] = 2 ** bits - 1
                e[b, :, lens[b]:] = 255
            self.codes.append(codes)
            self.e.append(e)
            self.val.append(val)
        self.bits, self.bs, self.table = bits, bs, table
        self.load()

    def load(self):
        parts = [as_pools(c, e, self.bs, self.bits, self.table, self.nb) for c, e in zip(self.codes, self.e)]
        self.dev = [to_dev(parts[0][0]), to_dev(parts[1][0]), to_dev(parts[0][1]), to_dev(parts[1][1])]
        self.mx = ea.make_mx(*self.dev, BITS[self.bits])
        t = self.table.copy()
        for b, n in enumerate(self.lens):                      # entries behind a sequence's blocks lead nowhere
            t[b, -(-int(n) // self.bs):] = -99
        self.t = i32(t)
        self.pg = ea.make_paged(self.t, self.bs, self.nb)
        self.ld = i32(self.lens)
        self.n = self.max_blocks * self.bs


def run_mx(c, q, cu, hq, hkv, d, n=None, max_new=None, room=0):
    import torch
    p = ea.make_params(len(c.lens), hq, hkv, d, ea.EA_BF16)
    n = c.n if n is None else n
    step = ea.make_step(i32(cu), q.shape[0], max(1, int(np.diff(cu).max())) if max_new is None else max_new)
    out, lse = outputs(q, "bf16")
    ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
    ea.attend_mx(p, to_dev(q), step, c.mx, c.pg, c.ld, n, out, lse, ws)
    torch.cuda.synchronize()
    return to_host(out), lse.cpu().numpy()


def queries(seed, t, hq, d):
    return store(np.random.default_rng(seed).standard_normal((t, hq, d)), "bf16")


def sums(m):
    return np.concatenate([[0], np.cumsum(m)])


# --------------------------------------------------------------------------------------- writing
def written(pools, bits, bs, nb, hkv, d):
    """codes [rows, H, d] and exponents [rows, H, d / 32] of K and V"""
    k, v, ks, vs = (to_host(x) for x in pools)
    turn = lambda x: x.transpose(0, 2, 1, 3).reshape(nb * bs, hkv, -1)    # noqa: E731
    return [(D.unpacked(turn(x), bits), turn(s).astype(np.int64)) for x, s in ((k, ks), (v, vs))]


def empty_pools(nb, hkv, bs, d, bits):
    import torch
    return [torch.full((nb, hkv, bs, w), x, dtype=torch.uint8, device="cuda")
            for w, x in ((d * bits // 8, 0x11), (d * bits // 8, 0x22), (d // 32, 77), (d // 32, 88))]


@pytest.mark.parametrize("hq,hkv,d,bs,t", [(8, 2, 128, 16, 1), (5, 1, 64, 32, 37), (4, 4, 256, 16, 130), (6, 2, 128, 64, 700), (40, 8, 128, 16, 48)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("form", ["dense", "strided", "in place", "no queries", "unturned"])
def test_rows_as_they_are_written(hq, hkv, d, bs, t, inter, bits, form):
    import torch
    r = np.random.default_rng(t + d + bits)
    nb = -(-t // bs) + 5
    inv = inv_freq_table(d, 5e5)
    x = store(r.standard_normal((t, hq + 2 * hkv, d)) * np.exp2(r.integers(-6, 7, (t, hq + 2 * hkv, 1))), "bf16")
    pos = r.integers(0, 1 << 20, t)
    pos[0] = 2 ** 31 - 1
    slots = r.permutation(nb * bs)[:t].astype(np.int64)
    if t > 3:
        slots[2], slots[3] = -1, nb * bs                        # left out: nothing of them is written
    pools = empty_pools(nb, hkv, bs, d, bits)
    before = written(pools, bits, bs, nb, hkv, d)
    xd = to_dev(x)
    parts = [xd[:, :hq], xd[:, hq:hq + hkv], xd[:, hq + hkv:]]
    if form != "strided":
        parts = [y.contiguous() for y in parts]
    q = None if form in ("no queries", "unturned") else parts[0]
    q_out = None if q is None else q if form == "in place" else torch.full((t, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    p = ea.make_params(1, hq, hkv, d, ea.EA_BF16, rope_layout=int(inter))
    rows = ea.make_new_rows(q, parts[1], parts[2], i32(pos), None if form == "unturned" else to_dev(inv))
    table = i32([[0]])
    ea.append_mx(p, rows, to_dev(slots), ea.make_mx(*pools, BITS[bits]), ea.make_paged(table, bs, nb), q_out)
    torch.cuda.synchronize()
    got = written(pools, bits, bs, nb, hkv, d)
    stored = (slots >= 0) & (slots < nb * bs)
    xf = widen(x)
    key = xf[stored, hq:hq + hkv]
    if form == "unturned":
        want = [D.quantise(key, bits)]
    else:
        key = S.rotate(key, pos[stored], inv, inter)
        want = [D.quantise(key * (1 + s * 2.0 ** -23), bits) for s in (0, 1, -1)]
    k = (got[0][0][slots[stored]], got[0][1][slots[stored]])
    assert np.logical_or.reduce([k[1] == w[1] for w in want]).all()
    # (an element of a group whose exponent went the other way stands for the same number but for the smallest)
    same = np.logical_or.reduce([(k[0] == w[0]) | (np.abs(D.values(*k, bits) - D.values(*w, bits)) == 0) for w in want])
    assert same.all()
    val = D.quantise(xf[stored, hq + hkv:], bits)
    assert np.array_equal(got[1][0][slots[stored]], val[0]) and np.array_equal(got[1][1][slots[stored]], val[1])
    rest = np.setdiff1d(np.arange(nb * bs), slots[stored])
    for g, b in zip(got, before):
        assert np.array_equal(g[0][rest], b[0][rest]) and np.array_equal(g[1][rest], b[1][rest])
    if q is not None:
        qo = widen(to_host(q_out))
        check_rotated(qo[stored], xf[stored, :hq], pos[stored], inv, inter, "bf16")
        assert np.array_equal(qo[~stored], xf[~stored, :hq] if form == "in place" else np.full_like(qo[~stored], 7.0))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("inter", [False, True])
def test_numbers_at_the_borders_of_the_formats(bits, d, inter):
    """Not finite, at the largest element and one step above, where halves are rounded, below what is resolved, bf16's largest."""
    import torch
    r = np.random.default_rng(bits + d)
    most = 448.0 if bits == 8 else 6.0
    t, x = 24, np.zeros((24, 2, d))
    x[:] = r.standard_normal(x.shape) * 2.0 ** r.integers(-3, 4, x.shape)
    for g in range(d // 32):
        c = g * 32 + int(r.integers(0, 32))
        x[0, :, c] = np.nan
        x[1, :, c] = np.inf if g % 2 else -np.inf
        x[2, :, g * 32:g * 32 + 32] = 0.0
        x[3, :, c], x[4, :, c] = most * 2.0 ** g, most * 2.0 ** g * (1 + 2.0 ** -7)     # bf16's next number
        x[5, :, c] = -D.BF16_MOST
        x[6, :, g * 32:g * 32 + 32] *= 2.0 ** -126
        x[7, :, g * 32:g * 32 + 32] = 2.0 ** -133 * r.integers(-128, 128, 32)             # below the smallest normal number
        x[8, :, g * 32:g * 32 + 32] = D.BF16_MOST * r.choice([1, -1], 32) * 2.0 ** -r.integers(0, 4, 32)
        half = (np.arange(32) % 16 + 0.5) / 16 * 2.0 ** (np.arange(32) // 16)
        x[9, :, g * 32:g * 32 + 32] = half * most
        x[10, :, g * 32:g * 32 + 32] = half
        x[11, :, g * 32:g * 32 + 32] = np.append(half[:31], most) * 2.0 ** (g - 2)
    x[12, :, 5] = np.nan                                       # one group of the row only
    bits_x = bf16_bits_from_f64(np.where(np.isfinite(x), x, 0.0))
    bits_x = np.where(np.isnan(x), 0x7FC0, np.where(np.isposinf(x), 0x7F80, np.where(np.isneginf(x), 0xFF80, bits_x))).astype(np.uint16)
    xf = widen(bits_x)
    pools = empty_pools(2, 1, 16, d, bits)
    xd, table, slots = to_dev(bits_x), i32([[0, 1]]), to_dev(np.arange(t, dtype=np.int64))
    p = ea.make_params(1, 1, 1, d, ea.EA_BF16, rope_layout=int(inter))
    rows = ea.make_new_rows(None, xd[:, :1], xd[:, 1:])
    mx, pg = ea.make_mx(*pools, BITS[bits]), ea.make_paged(table, 16, 2)
    ea.append_mx(p, rows, slots, mx, pg)
    back = torch.zeros(2, 1, 1, 32, d, dtype=torch.bfloat16, device="cuda")
    ea.read_mx(p, mx, pg, i32([t]), 32, 32, back[0], back[1])
    torch.cuda.synchronize()
    for (codes, e), val, read in zip(written(pools, bits, 16, 2, 1, d), (xf[:, :1], xf[:, 1:]), back):
        want = D.quantise(val, bits)
        assert np.array_equal(e[:t], want[1])
        assert np.array_equal(codes[:t], want[0])
        ref, got = D.values(*want, bits)[:, 0], widen(to_host(read))[0, 0, :t]
        assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.isfinite(got[~np.isnan(ref)]).all()
        assert np.array_equal(got[~np.isnan(ref)], ref[~np.isnan(ref)])
        assert np.isnan(ref[12, :32]).all() and np.isfinite(ref[12, 32:]).all()


def test_a_rotation_that_passes_the_end_of_fp32():
    """A rotated channel of 2^128 and more is an infinity: its group reads back as NaN, the others do not."""
    import torch
    d, big = 128, D.BF16_MOST
    x = np.ones((1, 2, d))
    x[0, 0, 3] = x[0, 0, 67] = big                             # turned by 1/8 of a turn: one grows by sqrt(2)
    inv = np.zeros(64)
    inv[3] = np.pi / 4
    pools, xd = empty_pools(1, 1, 16, d, 8), to_dev(bf16_bits_from_f64(x))
    p = ea.make_params(1, 1, 1, d, ea.EA_BF16)
    rows = ea.make_new_rows(None, xd[:, :1], xd[:, 1:], i32([1]), to_dev(inv))
    ea.append_mx(p, rows, to_dev(np.zeros(1, dtype=np.int64)), ea.make_mx(*pools, ea.EA_MXFP8), ea.make_paged(i32([[0]]), 16, 1))
    torch.cuda.synchronize()
    codes, e = written(pools, 8, 16, 1, 1, d)[0]
    assert list(e[0, 0]) == [127 - 8, 127 - 8, 255, 127 - 8] or e[0, 0, 2] == 255 and e[0, 0, 1] != 255 and e[0, 0, 3] != 255


@pytest.mark.parametrize("bits", [8, 4])
def test_writing_what_was_read_changes_nothing(bits):
    import torch
    c = Mx(3, [100, 37], 2, 128, 16, bits, spread=6)
    p = ea.make_params(2, 4, 2, 128, ea.EA_BF16)
    out = torch.zeros(2, 2, 2, 100, 128, dtype=torch.bfloat16, device="cuda")
    ea.read_mx(p, c.mx, c.pg, c.ld, 100, 100, out[0], out[1])
    k, v = (torch.cat([out[i, 0].transpose(0, 1), out[i, 1, :, :37].transpose(0, 1)]).contiguous() for i in range(2))
    slots = np.concatenate([c.table[b][np.arange(n) // 16].astype(np.int64) * 16 + np.arange(n) % 16 for b, n in ((0, 100), (1, 37))])
    ea.append_mx(p, ea.make_new_rows(None, k, v), to_dev(slots), c.mx, c.pg)
    again = torch.zeros_like(out)
    ea.read_mx(p, c.mx, c.pg, c.ld, 100, 100, again[0], again[1])
    torch.cuda.synchronize()
    assert torch.equal(out, again)


# --------------------------------------------------------------------------------------- reading
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hkv,d,bs", [(2, 128, 16), (1, 64, 32), (3, 256, 16), (8, 128, 64)])
def test_rows_read_back(bits, hkv, d, bs):
    import torch
    lens = [133, 0, 1, 64, 500, 17]
    c = Mx(d + bits, lens, hkv, d, bs, bits, spread=20)
    p = ea.make_params(6, hkv, hkv, d, ea.EA_BF16)
    ld = i32([133, -4, 1, 64, 900, 17])                        # lengths that make no sense count as none, or as n
    for n, cap, which in ((500, 500, "kv"), (500, 531, "k"), (100, 120, "v")):
        out = [torch.full((6, hkv, cap, d), 7.0, dtype=torch.bfloat16, device="cuda") if x in which else None for x in "kv"]
        ea.read_mx(p, c.mx, c.pg, ld, n, cap, *out)
        torch.cuda.synchronize()
        for o, val in zip(out, c.val):
            if o is None:
                continue
            got = widen(to_host(o))
            for b in range(6):
                m = min(lens[b], n)
                assert np.array_equal(got[b, :, :m], val[b, :, :m]) and (got[b, :, m:] == 7.0).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_every_byte_and_every_exponent(bits):
    """Not only what the library writes: all codes under all exponents, 0 and 255 among them."""
    import torch
    d, bs, rows = 64, 16, 2048
    r = np.random.default_rng(1)
    e = r.integers(0, 256, (1, 1, rows, 2))
    e[0, 0, :512] = np.arange(512).reshape(512, 1) % 256
    codes = r.integers(0, 2 ** bits, (1, 1, rows, d))
    table = np.arange(rows // bs, dtype=np.int32)[None]
    b, s = as_pools(codes, e, bs, bits, table, rows // bs)
    dev = [to_dev(b), to_dev(b), to_dev(s), to_dev(s)]
    t = i32(table)
    out = torch.zeros(1, 1, rows, d, dtype=torch.bfloat16, device="cuda")
    ea.read_mx(ea.make_params(1, 1, 1, d, ea.EA_BF16), ea.make_mx(dev[0], dev[1], dev[2], dev[3], BITS[bits]), ea.make_paged(t, bs, rows // bs),
               i32([rows]), rows, rows, out, None)
    torch.cuda.synchronize()
    want, got = D.values(codes, e, bits)[0, 0], widen(to_host(out))[0, 0]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    # (numbers past bf16's largest one are infinities)
    want = np.where(np.abs(want) > D.BF16_MOST, np.sign(want) * np.inf, want)
    fine = ~np.isnan(want) & ((np.abs(want) >= 2.0 ** -126) | (want == 0))
    assert np.array_equal(got[fine], want[fine])
    small = ~np.isnan(want) & ~fine
    # bf16's numbers below 2^-126 are whole multiples of 2^-133, and an element of 2^-127 * 2^-9 is less than one: zeros, or half of that off
    assert ((got[small] == 0) | (np.abs(got[small] - want[small]) <= 2.0 ** -134)).all()


# ------------------------------------------------------------------------------------- attention
SHAPES = [(8, 2, 128), (5, 1, 128), (16, 1, 64), (14, 2, 64), (4, 2, 256), (24, 1, 128), (64, 1, 64), (40, 2, 256)]


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("bs", [16, 64])
def test_single_tokens(hq, hkv, d, bits, bs):
    lens = [1, 700, 64, 333, 16, 0, 129]
    c = Mx(hq + d, lens, hkv, d, bs, bits, spread=2)
    cu = sums([1] * 7)
    q = queries(d, 7, hq, d)
    got, lse = run_mx(c, q, cu, hq, hkv, d)
    check_attend(got, lse, q, cu, c.val[0], c.val[1], np.repeat(c.lens[:, None], hkv, 1), "bf16")


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("m", [[2, 3, 1, 4], [33, 1, 0, 70], [9, 40, 300, 2]])
def test_stretches(hq, hkv, d, bits, m):
    r = np.random.default_rng(sum(m))
    lens = r.integers(max(m), 600, 4)
    lens[3] = m[3]
    lens[0] = max(0, m[0] - 1)                                  # fewer rows than tokens: the first sees none
    c = Mx(hq + d, lens, hkv, d, 16, bits)
    cu = sums(m)
    q = queries(d, int(cu[-1]) + 5, hq, d)                      # rows behind the last sequence are left as they were
    got, lse = run_mx(c, q, cu, hq, hkv, d)
    check_attend(got, lse, q, cu, c.val[0], c.val[1], np.repeat(c.lens[:, None], hkv, 1), "bf16")
    assert (widen(got)[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("hq,hkv,d,bits", [(8, 2, 128, 8), (4, 2, 256, 4), (6, 2, 64, 8), (12, 4, 128, 4)])
@pytest.mark.parametrize("m,lens", [([1], [5000]), ([60], [4100]), ([300, 1], [3500, 4000])])
def test_long_heads_in_many_pieces(hq, hkv, d, bits, m, lens):
    c = Mx(d + bits, lens, hkv, d, 32, bits)
    cu = sums(m)
    q = queries(d, int(cu[-1]), hq, d)
    got, lse = run_mx(c, q, cu, hq, hkv, d)
    check_attend(got, lse, q, cu, c.val[0], c.val[1], np.repeat(c.lens[:, None], hkv, 1), "bf16")


@pytest.mark.parametrize("bits,d", [(8, 128), (4, 64), (8, 256)])
def test_many_sequences_and_loose_bounds(bits, d):
    r = np.random.default_rng(d)
    B = 150
    lens, m = r.integers(0, 90, B), r.integers(0, 4, B)
    c = Mx(d, lens, 2, d, 16, bits)
    cu = sums(m)
    q = queries(d, int(cu[-1]), 4, d)
    L = np.repeat(c.lens[:, None], 2, 1)
    for max_new in (3, 60, 500):
        got, lse = run_mx(c, q, cu, 4, 2, d, max_new=max_new)
        check_attend(got, lse, q, cu, c.val[0], c.val[1], L, "bf16")


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("m", [[1, 1, 1], [30, 1, 2], [90, 3, 150]])
def test_lengths_that_make_no_sense(bits, m):
    """Negative lengths count as none, those over n as n."""
    c = Mx(5, [200, 160, 200], 2, 128, 16, bits)
    cu = sums(m)
    q = queries(1, int(cu[-1]), 8, 128)
    c.ld = i32([-7, 160, 1 << 30])
    got, lse = run_mx(c, q, cu, 8, 2, 128, n=200)
    check_attend(got, lse, q, cu, c.val[0], c.val[1], np.array([[0, 0], [160, 160], [200, 200]]), "bf16")


@pytest.mark.parametrize("bits,hq,hkv,d,m", [(8, 8, 2, 128, [2, 3, 1]), (4, 6, 2, 64, [5, 2, 40]), (8, 8, 2, 128, [100, 1, 70]),
                                             (4, 4, 2, 256, [3, 90, 2]), (8, 4, 2, 256, [60, 150, 2]), (4, 8, 2, 128, [50, 130, 2])])
@pytest.mark.parametrize("where", ["values", "keys"])
def test_groups_that_are_not_numbers(bits, hq, hkv, d, m, where):
    """A group of exponent 255 in a row reaches the tokens that see that row, and no others."""
    r = np.random.default_rng(hq + d)
    lens = r.integers(max(m), 400, 3)
    lens[2] = m[2]
    c = Mx(hq * d, lens, hkv, d, 16, bits)
    cu = sums(m)
    q = queries(d, int(cu[-1]), hq, d)
    clean, clean_lse = run_mx(c, q, cu, hq, hkv, d)
    bad = np.full((3, hkv), -1)
    for b in range(3):
        if m[b] > 1:
            for h in range(hkv):
                bad[b, h] = lens[b] - 1 - (int(r.integers(0, m[b])) if where == "values" else 0)
                c.e[1][b, h, bad[b, h], 1] = 255
                if where == "keys":
                    c.e[0][b, h, lens[b] - 1, 0] = 255
    c.load()
    got, lse = run_mx(c, q, cu, hq, hkv, d)
    got, clean = widen(got), widen(clean)
    for b in range(3):
        for i in range(m[b]):
            for x in range(hq):
                h, t = x // (hq // hkv), cu[b] + i
                n = lens[b] - (m[b] - 1 - i)
                if where == "keys" and m[b] > 1 and i == m[b] - 1:
                    assert np.isnan(got[t, x]).all() and np.isnan(lse[t, x])
                    continue
                touched = np.zeros(d, dtype=bool)
                touched[32:64] = 0 <= bad[b, h] < n
                assert np.isnan(got[t, x][touched]).all()
                assert np.array_equal(got[t, x][~touched], clean[t, x][~touched]) and lse[t, x] == clean_lse[t, x]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("m", [[1, 1], [2, 90], [20, 70]])
def test_exponents_far_apart(bits, m):
    """Groups of a row whose powers of two lie up to 2^30 apart: each counts with its own."""
    c = Mx(9, [150, 270], 2, 128, 16, bits, spread=15)
    for b in range(2):      # keys that would leave one weight alone are brought down
        c.e[0] = np.where(c.e[0] == 255, 255, np.minimum(c.e[0], 121 if bits == 8 else 126))
    c.val[0] = D.values(np.where(c.e[0].repeat(32, -1) == 255, 0, c.codes[0]), np.where(c.e[0] == 255, 127, c.e[0]), bits)
    c.load()
    cu = sums(m)
    q = queries(4, int(cu[-1]), 8, 128)
    got, lse = run_mx(c, q, cu, 8, 2, 128)
    check_attend(got, lse, q, cu, c.val[0], c.val[1], np.repeat(c.lens[:, None], 2, 1), "bf16")


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("m", [1, 40])
def test_blocks_past_32_bits(bits, m):
    """The sequence's blocks lie past 2^32 bytes of the pool, its scales past 2^27."""
    import torch
    hq, hkv, d, bs = 4, 2, 128, 16
    n = 100
    row = d * bits // 8
    nb = (1 << 32) // (hkv * bs * row) + 40
    free = torch.cuda.mem_get_info()[0]
    if free < 3 * nb * hkv * bs * (row + 4):
        pytest.skip("not enough memory")
    c = Mx(2, [n], hkv, d, bs, bits)
    first = nb - 9
    big = []
    for x in c.dev:
        y = torch.zeros(nb, *x.shape[1:], dtype=torch.uint8, device="cuda")
        y[first:first + c.max_blocks] = x[c.table[0].astype(np.int64)]
        big.append(y)
    t = i32(np.arange(first, first + c.max_blocks)[None])
    c.mx, c.pg, c.t = ea.make_mx(*big, BITS[bits]), ea.make_paged(t, bs, nb), t
    cu, q = sums([m]), queries(3, m, hq, d)
    got, lse = run_mx(c, q, cu, hq, hkv, d)
    check_attend(got, lse, q, cu, c.val[0], c.val[1], np.array([[n] * hkv]), "bf16")
    p = ea.make_params(1, hq, hkv, d, ea.EA_BF16)
    back = torch.zeros(2, 1, hkv, n, d, dtype=torch.bfloat16, device="cuda")
    ea.read_mx(p, c.mx, c.pg, c.ld, n, n, back[0], back[1])
    xd = to_dev(store(np.random.default_rng(1).standard_normal((3, 2 * hkv, d)), "bf16"))
    slots = torch.arange(3, dtype=torch.int64, device="cuda") + (nb * bs - 3)
    ea.append_mx(p, ea.make_new_rows(None, xd[:, :hkv], xd[:, hkv:]), slots, c.mx, c.pg)
    torch.cuda.synchronize()
    for i in range(2):
        assert np.array_equal(widen(to_host(back[i]))[0], c.val[i][0])
        codes, e = D.quantise(widen(to_host(xd))[:, i * hkv:(i + 1) * hkv], bits)
        last = to_host(big[i][nb - 1])[:, -3:].transpose(1, 0, 2)
        assert np.array_equal(D.unpacked(last, bits), codes) and np.array_equal(to_host(big[2 + i][nb - 1])[:, -3:].transpose(1, 0, 2), e)


def test_the_library_writes_and_reads_what_it_attends_to():
    """Prompts rotated and stored, tokens generated behind them, in both formats: attention over the pools is that over the rows
    read back, and the compress pass takes those."""
    import torch
    hq, hkv, d, bs, B = 8, 2, 128, 16, 3
    r = np.random.default_rng(0)
    inv = to_dev(inv_freq_table(d, 1e4))
    p = ea.make_params(B, hq, hkv, d, ea.EA_BF16)
    for bits in (8, 4):
        nb, mb = 60, 20
        pools = empty_pools(nb, hkv, bs, d, bits)
        mx = ea.make_mx(*pools, BITS[bits])
        table, free = torch.full((B, mb), -1, dtype=torch.int32, device="cuda"), i32(r.permutation(nb))
        pg, count, lens = ea.make_paged(table, bs, nb), i32([nb]), i32([0] * B)
        for more in ([150, 77, 1], [1, 1, 1], [1, 0, 1], [40, 1, 2]):
            cu, t = sums(more), sum(more)
            new = lens + i32(more)
            len_out, count_out, cud = torch.zeros_like(lens), torch.zeros_like(count), i32([0] * (B + 1))
            slots, pos = torch.zeros(t, dtype=torch.int64, device="cuda"), i32([0] * t)
            ea.block_tables(p, pg, lens, new, free, count, len_out, count_out, cud, t, slots, pos)
            lens, count = len_out, count_out
            x = to_dev(store(r.standard_normal((t, hq + 2 * hkv, d)), "bf16"))
            rows = ea.make_new_rows(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], pos, inv)
            q, (out, lse) = torch.zeros(t, hq, d, dtype=torch.bfloat16, device="cuda"), outputs(np.zeros((t, hq, d)), "bf16")
            ea.append_mx(p, rows, slots, mx, pg, q)
            step, n = ea.make_step(cud, t, max(more)), mb * bs
            ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda")
            ea.attend_mx(p, q, step, mx, pg, lens, n, out, lse, ws)
            back = torch.full((2, B, hkv, n, d), float("nan"), dtype=torch.bfloat16, device="cuda")
            ea.read_mx(p, mx, pg, lens, n, n, back[0], back[1])
            torch.cuda.synchronize()
            L = np.repeat(to_host(lens)[:, None], hkv, 1)
            k, v = (np.nan_to_num(widen(to_host(y))) for y in back)
            check_attend(to_host(out), lse.cpu().numpy(), to_host(q), cu, k, v, L, "bf16")
        # a compress pass over the longest sequence: scored as read back, its best rows written again in front
        p1, m = ea.make_params(1, hq, hkv, d, ea.EA_BF16), int(lens[0])
        kb, vb = (back[i, :1].contiguous() for i in range(2))
        ws = torch.empty(ea.workspace_bytes(p1, m, 32), dtype=torch.uint8, device="cuda")
        keep = m // 2
        ea.compress_layer(p1, to_dev(store(r.standard_normal((1, hq, 32, d)), "bf16")), 32, m - 32, inv, m, kb, vb, m, n, keep, None, None, ws)
        at = torch.arange(keep, device="cuda")
        slots = table[0, at // bs].long() * bs + at % bs
        ea.append_mx(p1, ea.make_new_rows(None, kb[0, :, :keep].transpose(0, 1).contiguous(), vb[0, :, :keep].transpose(0, 1).contiguous()),
                     slots, mx, pg)
        again = torch.zeros(2, B, hkv, n, d, dtype=torch.bfloat16, device="cuda")
        ea.read_mx(p, mx, pg, i32([keep] + to_host(lens)[1:].tolist()), n, n, again[0], again[1])
        torch.cuda.synchronize()
        assert torch.equal(again[0, 0, :, :keep], kb[0, :, :keep]) and torch.equal(again[1, 0, :, :keep], vb[0, :, :keep])


def test_captured_and_replayed_on_other_lengths():
    """One captured step (store, attention, reading back) follows lengths and rows; every replay against the eager call."""
    import torch
    hq, hkv, d, bs, B = 8, 2, 128, 16, 3
    r = np.random.default_rng(4)
    c = Mx(8, [300, 400, 100], hkv, d, bs, 8)
    p, n = ea.make_params(B, hq, hkv, d, ea.EA_BF16), c.n
    t = i32(np.arange(c.nb)[None].repeat(B, 0)[:, :c.max_blocks])
    t.copy_(to_dev(c.table))
    pg, inv = ea.make_paged(t, bs, c.nb), to_dev(inv_freq_table(d, 1e4))
    lens, pos, slots = i32([200, 300, 50]), i32([0] * B), torch.zeros(B, dtype=torch.int64, device="cuda")
    x = torch.zeros(B, hq + 2 * hkv, d, dtype=torch.bfloat16, device="cuda")
    rows = ea.make_new_rows(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], pos, inv)
    q, (out, lse) = torch.zeros(B, hq, d, dtype=torch.bfloat16, device="cuda"), outputs(np.zeros((B, hq, d)), "bf16")
    cud = i32(range(B + 1))
    step = ea.make_step(cud, B, 1)
    ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda")
    back = torch.zeros(2, B, hkv, n, d, dtype=torch.bfloat16, device="cuda")

    def go(mx):
        ea.append_mx(p, rows, slots, mx, pg, q)
        ea.attend_mx(p, q, step, mx, pg, lens, n, out, lse, ws)
        ea.read_mx(p, mx, pg, lens, n, n, back[0], back[1])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        go(c.mx)
    torch.cuda.synchronize()
    other = [y.clone() for y in c.dev]
    mx2 = ea.make_mx(*other, ea.EA_MXFP8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        go(c.mx)
    for k in range(4):
        L = r.integers(1, [300, 400, 100])
        x.copy_(to_dev(store(r.standard_normal(x.shape), "bf16")))
        lens.copy_(i32(L))
        pos.copy_(i32(L + 5))
        slots.copy_(to_dev(np.array([c.table[b, (L[b] - 1) // bs] * bs + (L[b] - 1) % bs for b in range(B)], dtype=np.int64)))
        ws.fill_(0xA5)
        back.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [y.clone() for y in (q, out, lse, back, *c.dev)]
        back.zero_()
        go(mx2)
        torch.cuda.synchronize()
        for a, b in zip(got, (q, out, lse, back, *other)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_calls_on_side_streams():
    import torch
    cases = []
    for seed, m in ((1, [1, 1, 1]), (2, [30, 1, 64])):
        c = Mx(seed, [700, 1300, 90], 2, 128, 16, 8 if seed == 1 else 4)
        cu = sums(m)
        q = queries(seed, int(cu[-1]), 8, 128)
        cases.append((c, q, cu, run_mx(c, q, cu, 8, 2, 128)))
    p = ea.make_params(3, 8, 2, 128, ea.EA_BF16)
    streams, keep = [torch.cuda.Stream() for _ in range(2)], []
    for c, q, cu, _ in cases:
        step = ea.make_step(i32(cu), q.shape[0], int(np.diff(cu).max()))
        out, lse = outputs(q, "bf16")
        keep.append((to_dev(q), step, out, lse, torch.empty(ea.attend_workspace_bytes(p, step, c.n), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(3):
        for s, (c, *_), (q, step, out, lse, ws) in zip(streams, cases, keep):
            ea.attend_mx(p, q, step, c.mx, c.pg, c.ld, c.n, out, lse, ws, stream=s)
    torch.cuda.synchronize()
    for (*_, (want, want_lse)), (_, _, out, lse, _) in zip(cases, keep):
        assert np.array_equal(to_host(out), want) and np.array_equal(lse.cpu().numpy(), want_lse)
