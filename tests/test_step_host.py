"""Refusals of the step's entry points, before any launch (no GPU needed), and the plans of attention against their workspace."""
import ctypes

import pytest

import paper_2510_00636_amd as ea
from paper_2510_00636_amd.binding import EaNewRows, EaPaged, EaStep

VP, byref = ctypes.c_void_p, ctypes.byref
OK = 1 << 30            # fake, aligned addresses a GiB apart, never dereferenced: every call below fails its checks, or has nothing to do


def at(i):
    return VP((i + 1) * OK)


@pytest.fixture(scope="module")
def lib():
    return ea.load_library()


def bf16(**kw):
    return ea.make_params(kw.pop("batch", 2), kw.pop("hq", 4), kw.pop("hkv", 2), kw.pop("d", 128), kw.pop("dtype", ea.EA_BF16), **kw)


def test_block_tables_refusals(lib):
    def call(p=None, table=10 * OK, bs=16, mb=8, nb=100, args=(0, 1, 2, 3, 4, 5, 6), n=0, slots=None, pos=None, seen=None):
        pg = EaPaged(table, bs, mb, nb)
        ptr = [a if a is None else at(a) for a in args]
        return lib.ea_block_tables(byref(p or bf16()), byref(pg), *ptr, n, slots, pos, seen, None)
    for i in range(7):                                                       # a null pointer in each place
        assert call(args=tuple(None if j == i else j for j in range(7))) == 1
    assert call(table=0) == 1 and call(nb=0) == 1 and call(mb=0) == 1
    assert call(bs=24) == 2 and call(bs=8) == 2 and call(bs=1 << 17) == 2
    assert call(nb=1 << 31) == 2
    assert call(p=bf16(batch=4097)) == 2
    assert call(n=-1) == 1 and call(n=4) == 1 and call(n=4, slots=at(7)) == 1 and call(n=4, slots=VP(8 * OK + 4), pos=at(8)) == 1
    assert call(seen=VP(OK + 2)) == 1
    # what is written has to be apart from everything else
    assert call(args=(0, 1, 2, 3, 0, 5, 6)) == 1                             # len_out = len_old
    assert call(args=(0, 1, 2, 3, 4, 3, 6)) == 1                             # free_out = free_in
    assert call(table=OK) == 1                                               # the table over the old lengths
    assert call(args=(0, 1, 2, 3, 4, 5, 2)) == 1                             # prefix sums over the list
    assert call(n=4, slots=at(4), pos=at(8)) == 1                            # slots over len_out
    assert lib.ea_block_tables(byref(bf16()), None, at(0), at(1), at(2), at(3), at(4), at(5), at(6), 0, None, None, None, None) == 1


def test_append_refusals(lib):
    pg = EaPaged(10 * OK, 16, 8, 100)

    def rows(**kw):
        f = dict(q=3 * OK, k=4 * OK, v=5 * OK, n_tokens=8, pos=6 * OK, inv_freq=7 * OK)
        f.update(kw)
        return EaNewRows(**f)

    def paged(r, p=None, q_out=at(8), slots=at(9), k=at(11), v=at(12), g=pg):
        return lib.ea_append_paged(byref(p or bf16()), byref(r), slots, k, v, byref(g), q_out, None)
    for name in ("k", "v", "pos"):
        assert paged(rows(**{name: None})) == 1
    assert paged(rows(), q_out=None) == 1 and paged(rows(), slots=None) == 1 and paged(rows(), k=None) == 1
    assert paged(rows(), v=at(11)) == 1                                      # one pool for both
    assert paged(rows(inv_freq=None)) == 1                                   # queries without angles
    assert paged(rows(q=3 * OK + 8)) == 1 and paged(rows(k_stride=255)) == 1 and paged(rows(q_stride=4 * 128 + 4)) == 1
    assert paged(rows(v_stride=1 << 41)) == 1 and paged(rows(n_tokens=-1)) == 1
    assert paged(rows(n_tokens=(1 << 24) + 1)) == 2
    assert paged(rows(), p=bf16(dtype=ea.EA_F32)) == 2 and paged(rows(), g=EaPaged(10 * OK, 20, 8, 100)) == 2
    assert paged(rows(), q_out=VP(3 * OK + 8 + 16)) == 1                     # over the queries, but not the same place ...
    assert paged(rows(q=3 * OK), q_out=VP(3 * OK + 256)) == 1
    assert paged(rows(q_stride=8 * 128), q_out=VP(3 * OK)) == 1              # ... or the same place with another stride
    assert paged(rows(k=12 * OK)) == 1                                       # new rows inside the pool
    assert paged(rows(n_tokens=0)) == 0                                      # nothing to do

    def heads(r, p=None, cu=at(8), lens=at(9), cap=64, fp8=False, ks=None):
        if fp8:
            return lib.ea_append_fp8(byref(p or bf16()), byref(r), cu, lens, at(11), at(12), ks, None, cap, at(13), None)
        return lib.ea_append(byref(p or bf16()), byref(r), cu, lens, at(11), at(12), cap, at(13), None)
    assert heads(rows(), cu=None) == 1 and heads(rows(), lens=None) == 1 and heads(rows(), cap=0) == 1
    assert heads(rows(), fp8=True, p=bf16(d=64)) == 2 and heads(rows(), fp8=True, p=bf16(dtype=ea.EA_F32)) == 2
    assert heads(rows(), fp8=True, ks=VP(OK + 2)) == 1
    assert heads(rows(n_tokens=0)) == 0 and heads(rows(n_tokens=0), fp8=True) == 0


def test_attend_refusals(lib):
    def step(**kw):
        f = dict(cu_tokens=2 * OK, n_tokens=8, max_new=4, q_stride=0)
        f.update(kw)
        return EaStep(**f)

    def call(p=None, st=None, q=at(3), k=at(4), v=at(5), lens=at(6), n=64, cap=64, out=at(7), lse=None, ws=at(8), wsb=1 << 28):
        return lib.ea_attend(byref(p or bf16()), q, byref(st or step()), k, v, lens, n, cap, out, lse, ws, wsb, None)
    for name in ("q", "k", "v", "lens", "out", "ws"):
        assert call(**{name: None}) == 1
    assert call(ws=VP(8 * OK + 16)) == 1 and call(wsb=16) == 3 and call(lse=VP(OK + 2)) == 1
    assert call(st=step(cu_tokens=None)) == 1 and call(st=step(n_tokens=-1)) == 1 and call(st=step(max_new=0)) == 1
    assert call(st=step(n_tokens=(1 << 24) + 1)) == 2
    assert call(st=step(q_stride=4 * 128 - 8)) == 1 and call(st=step(q_stride=4 * 128 + 4)) == 1
    assert call(n=-1) == 1 and call(n=65) == 1 and call(n=1 << 27, cap=1 << 28) == 1
    assert call(out=at(3)) == 1 and call(out=VP(4 * OK + 256)) == 1          # out over q, out inside the cache
    assert call(p=bf16(d=96)) == 2 and call(p=bf16(dtype=ea.EA_FP8_E4M3)) == 2
    assert call(st=step(n_tokens=0)) == 0
    # paged and 8-bit
    def paged(pg, p=None, n=64):
        return lib.ea_attend_paged(byref(p or bf16()), at(3), byref(step()), at(4), at(5), byref(pg), at(6), n, at(7), None, at(8), 1 << 28, None)
    assert paged(EaPaged(9 * OK, 24, 8, 8)) == 2 and paged(EaPaged(9 * OK, 16, 3, 8)) == 1 and paged(EaPaged(0, 16, 8, 8)) == 1
    assert paged(EaPaged(9 * OK, 16, 8, 8), p=bf16(dtype=ea.EA_F32)) == 2
    def fp8(p):
        return lib.ea_attend_fp8(byref(p), at(3), byref(step()), at(4), at(5), None, None, at(6), 64, 64, at(7), None, at(8), 16, None)
    assert fp8(bf16(d=64)) == 2 and fp8(bf16(dtype=ea.EA_F32)) == 2 and fp8(bf16()) == 3
    # more workgroups than a launch has
    assert call(p=bf16(batch=1 << 14, hq=64, hkv=64), st=step(n_tokens=1 << 24, max_new=1 << 20), q=VP(1 << 50), out=VP(1 << 52)) == 2


def test_attend_workspace(lib):
    p = bf16(batch=3, hq=8, hkv=2)
    def size(n, t, m, p=p):
        return ea.attend_workspace_bytes(p, EaStep(OK, t, m, 0), n)
    assert size(0, 0, 1) >= 256 and size(4096, 3, 1) >= 256
    assert size(-1, 3, 1) == 0 and size(1 << 27, 3, 1) == 0 and size(64, 3, 0) == 0
    assert size(64, 3, 1, bf16(d=80)) == 0
    # partial results stay small next to the cache: no more than two per workgroup of the row kernel, or the splits of few tiles
    for n in (100, 5000, 131072, 1 << 26):
        for t, m in ((3, 1), (24, 8), (300, 100), (8192, 4096)):
            assert size(n, t, m) < (1 << 28)


def test_new_rows_take_views_of_one_projection():
    import torch
    qkv = torch.zeros(5, (4 + 2 + 2) * 64, dtype=torch.bfloat16)
    q, k, v = (x.unflatten(1, (-1, 64)) for x in qkv.split([256, 128, 128], dim=1))
    r = ea.make_new_rows(q, k, v)
    assert (r.q_stride, r.k_stride, r.v_stride, r.n_tokens) == (512, 512, 512, 5)
    assert r.k - r.q == 512 and r.v - r.k == 256
    with pytest.raises(ValueError):
        ea.make_new_rows(None, k.transpose(0, 1), v)
    with pytest.raises(ValueError):
        ea.make_new_rows(None, k[..., ::2], v)


def test_limits_come_before_the_workspace(lib):
    """What no workspace helps is said first, and what the launches of few rows do not need is no limit."""
    def call(p, t, new, hq, pg=None, wsb=16):
        st = EaStep(2 * OK, t, new, 0)
        f = (lib.ea_attend_paged, (byref(pg), at(6), 16)) if pg else (lib.ea_attend, (at(6), 16, 16))
        return f[0](byref(p), VP(1 << 50), byref(st), at(4), at(5), *f[1], VP(1 << 52), None, at(8), wsb, None)
    heads = bf16(batch=1 << 14, hq=64, hkv=64)
    assert call(heads, 1 << 24, 1 << 20, 64) == 2                            # stretches: too many tiles
    assert call(heads, 1 << 24, 16, 64) == 3                                 # few tokens each: no tiles
    assert call(bf16(batch=1 << 14, hq=64, hkv=64, dtype=ea.EA_F32), 1 << 24, 1, 64) == 2
    big = EaPaged(10 * OK, 65536, 1, 2)
    assert call(bf16(batch=1, hq=128, hkv=128, d=256), 4, 40, 128, big) == 3 # (no sequence adds more than 4 of 4 tokens)
    assert call(bf16(batch=1, hq=128, hkv=128, d=256), 40, 40, 128, big) == 2


def test_new_rows_that_are_not_there():
    """Tensors whose rows the library would read past: expanded ones, too few of q, v or the positions, other types."""
    import torch
    bf = dict(dtype=torch.bfloat16)
    q, k, v = (torch.zeros(6, h, 64, **bf) for h in (4, 2, 2))
    pos, inv = torch.zeros(6, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    assert ea.make_new_rows(q, k, v, pos, inv).n_tokens == 6
    one = torch.zeros(1, 2, 64, **bf)
    for bad in ((None, one.expand(6, 2, 64), v), (None, k, one.expand(6, 2, 64)), (torch.zeros(1, 4, 64, **bf).expand(6, 4, 64), k, v),
                (None, k.as_strided((6, 2, 64), (64, 64, 1)), v),               # tokens over one another
                (q[:5], k, v), (None, k, v[:5]), (None, k, torch.zeros(6, 3, 64, **bf)), (torch.zeros(6, 4, 128, **bf), k, v),
                (q.float(), k, v), (None, k, v.float()), (None, k.view(6, 128), v)):
        with pytest.raises(ValueError):
            ea.make_new_rows(*bad, pos, inv)
    for bad in ((pos[:5], inv), (None, inv), (pos.long(), inv), (pos, inv[:31]), (pos, inv.float()), (torch.zeros(12, dtype=torch.int32)[::2], inv)):
        with pytest.raises(ValueError):
            ea.make_new_rows(q, k, v, *bad)
    assert ea.make_new_rows(None, k, v, None, None).k_stride == 128             # stored as they are
    # one token is one place, whatever its stride; one head is contiguous, whatever the stride between heads
    assert ea.make_new_rows(None, one.expand(1, 2, 64), one).k_stride == 0
    thin = torch.zeros(1, 6, 64, **bf).transpose(0, 1)
    assert thin.stride(1) != 64 and ea.make_new_rows(None, thin, thin).k_stride == 64


def test_block_tables_of_more_entries_than_32_bits_count(lib):
    def call(batch, max_blocks):
        pg = EaPaged(1 << 50, 16, max_blocks, 100)
        # free_out lies over free_in: what passes the limit is turned away by the next check
        return lib.ea_block_tables(byref(bf16(batch=batch)), byref(pg), at(0), at(1), at(2), at(3), at(4), at(3), at(6), 0, None, None, None, None)
    assert call(4096, 1 << 19) == 2 and call(2, 1 << 30) == 2 and call(3, 0x7fffffff) == 2
    assert call(4096, (1 << 19) - 1) == 1 and call(1, 0x7fffffff) == 1
