"""Refusals of the entry points for quantised pools and drafted trees, before any launch (no GPU needed)."""
import ctypes

import pytest

import paper_2510_00636_amd as ea
from paper_2510_00636_amd.binding import EaMx, EaNewRows, EaPaged, EaStep, EaTree

VP, byref = ctypes.c_void_p, ctypes.byref
OK = 1 << 30            # fake, aligned addresses a GiB apart, never dereferenced: every call below fails its checks, or has nothing to do


def at(i):
    return VP((i + 1) * OK)


@pytest.fixture(scope="module")
def lib():
    return ea.load_library()


def params(**kw):
    return ea.make_params(kw.pop("batch", 2), kw.pop("hq", 4), kw.pop("hkv", 2), kw.pop("d", 128), kw.pop("dtype", ea.EA_BF16), **kw)


def pools(**kw):
    f = dict(k=20 * OK, v=21 * OK, k_scale=22 * OK, v_scale=23 * OK, format=ea.EA_MXFP8)
    f.update(kw)
    return EaMx(**f)


def step(**kw):
    f = dict(cu_tokens=2 * OK, n_tokens=8, max_new=4, q_stride=0)
    f.update(kw)
    return EaStep(**f)


PG = EaPaged(10 * OK, 16, 8, 100)
BAD_POOLS = [(dict(k=None), 1), (dict(v=None), 1), (dict(k_scale=None), 1), (dict(v_scale=23 * OK + 8), 1), (dict(k=20 * OK + 8), 1),
             (dict(format=2), 2), (dict(format=-1), 2), (dict(v=20 * OK), 1), (dict(k_scale=21 * OK + 256), 1), (dict(v_scale=22 * OK), 1)]


def test_append_refusals(lib):
    def rows(**kw):
        f = dict(q=3 * OK, k=4 * OK, v=5 * OK, n_tokens=8, pos=6 * OK, inv_freq=7 * OK)
        f.update(kw)
        return EaNewRows(**f)

    def call(r=None, p=None, mx=None, q_out=at(8), slots=at(9), g=PG):
        return lib.ea_append_mx(byref(p or params()), byref(r or rows()), slots, byref(mx or pools()), byref(g), q_out, None)
    for kw, code in BAD_POOLS:
        assert call(mx=pools(**kw)) == code, kw
    for name in ("k", "v", "pos"):
        assert call(rows(**{name: None})) == 1
    assert call(q_out=None) == 1 and call(slots=None) == 1 and call(slots=VP(9 * OK + 4)) == 1
    assert call(rows(inv_freq=None)) == 1                                    # queries without angles
    assert call(rows(q=3 * OK + 8)) == 1 and call(rows(k_stride=255)) == 1 and call(rows(n_tokens=-1)) == 1
    assert call(rows(n_tokens=(1 << 24) + 1)) == 2
    assert call(p=params(dtype=ea.EA_F32)) == 2 and call(p=params(dtype=ea.EA_FP8_E4M3)) == 2 and call(p=params(d=96)) == 2
    assert call(g=EaPaged(10 * OK, 20, 8, 100)) == 2 and call(g=EaPaged(0, 16, 8, 100)) == 1
    assert call(rows(k=21 * OK)) == 1 and call(rows(v=22 * OK)) == 1         # new rows inside the pools
    assert call(q_out=VP(23 * OK)) == 1                                      # queries over the scales
    assert call(rows(q=3 * OK), q_out=VP(3 * OK + 256)) == 1
    assert lib.ea_append_mx(byref(params()), None, at(9), byref(pools()), byref(PG), at(8), None) == 1
    assert lib.ea_append_mx(byref(params()), byref(rows()), at(9), None, byref(PG), at(8), None) == 1
    assert call(rows(n_tokens=0)) == 0 and call(rows(n_tokens=0), mx=pools(k=None)) == 1


def test_read_refusals(lib):
    def call(p=None, mx=None, g=PG, lens=at(3), n=64, cap=64, k=at(4), v=at(5)):
        return lib.ea_read_mx(byref(p or params()), byref(mx or pools()), byref(g), lens, n, cap, k, v, None)
    for kw, code in BAD_POOLS:
        assert call(mx=pools(**kw)) == code, kw
    assert call(lens=None) == 1 and call(k=VP(4 * OK + 2)) == 1 and call(v=VP(4 * OK + 2)) == 1
    assert call(n=-1) == 1 and call(n=65) == 1 and call(cap=0, n=0) == 1 and call(n=200, cap=200) == 1      # more than the table has
    assert call(v=at(4)) == 1 and call(k=VP(20 * OK + 512)) == 1 and call(v=VP(23 * OK)) == 1
    assert call(p=params(dtype=ea.EA_F32)) == 2
    assert call(n=0) == 0 and call(k=None, v=None) == 0


def test_attend_refusals(lib):
    p = params()

    def mx(pool=None, st=None, q=at(3), lens=at(6), n=64, out=at(7), ws=at(8), wsb=1 << 28, pp=None, tree=None):
        if tree is None:
            return lib.ea_attend_mx(byref(pp or p), q, byref(st or step()), byref(pool or pools()), byref(PG), lens, n, out, None, ws, wsb, None)
        return lib.ea_attend_tree_mx(byref(pp or p), q, byref(st or step()), byref(tree), byref(pool or pools()), byref(PG), lens, n,
                                     out, None, ws, wsb, None)
    tr = EaTree(30 * OK, 1)
    for t in (None, tr):
        for kw, code in BAD_POOLS:
            assert mx(pools(**kw), tree=t) == code, kw
        assert mx(q=None, tree=t) == 1 and mx(lens=None, tree=t) == 1 and mx(out=None, tree=t) == 1 and mx(ws=None, tree=t) == 1
        assert mx(wsb=16, tree=t) == 3 and mx(n=1000, tree=t) == 1 and mx(pp=params(dtype=ea.EA_F32), tree=t) == 2
        assert mx(out=VP(20 * OK + 4096), tree=t) == 1 and mx(out=VP(22 * OK), tree=t) == 1 and mx(out=at(3), tree=t) == 1
        assert mx(st=step(n_tokens=0), tree=t) == 0
    assert lib.ea_attend_mx(byref(p), at(3), byref(step()), None, byref(PG), at(6), 64, at(7), None, at(8), 1 << 28, None) == 1

    # masks, in all three forms
    def forms(tree, st=None, out=at(7)):
        s, t = byref(st or step()), byref(tree) if tree is not None else None
        return [lib.ea_attend_tree(byref(p), at(3), s, t, at(4), at(5), at(6), 64, 64, out, None, at(8), 1 << 28, None),
                lib.ea_attend_tree_paged(byref(p), at(3), s, t, at(4), at(5), byref(PG), at(6), 64, out, None, at(8), 1 << 28, None),
                lib.ea_attend_tree_mx(byref(p), at(3), s, t, byref(pools()), byref(PG), at(6), 64, out, None, at(8), 1 << 28, None)]
    assert forms(None) == [1] * 3
    assert forms(EaTree(None, 1)) == [1] * 3 and forms(EaTree(30 * OK + 4, 1)) == [1] * 3
    assert forms(EaTree(30 * OK, 0)) == [1] * 3 and forms(EaTree(30 * OK, 5)) == [2] * 3
    assert forms(tr, step(max_new=65)) == [1] * 3 and forms(EaTree(30 * OK, 4), step(n_tokens=300, max_new=257)) == [1] * 3
    assert forms(tr, out=VP(30 * OK)) == [1] * 3                             # out over the masks
    assert forms(tr, step(n_tokens=0)) == [0] * 3
    assert lib.ea_attend_tree(byref(p), at(3), byref(step()), byref(tr), at(4), at(5), at(6), 65, 64, at(7), None, at(8), 1 << 28, None) == 1
    assert lib.ea_attend_tree(byref(params(dtype=ea.EA_FP8_E4M3)), at(3), byref(step()), byref(tr), at(4), at(5), at(6), 64, 64, at(7), None,
                              at(8), 1 << 28, None) == 2


def test_refusals_over_scaled_bytes(lib):
    tr = EaTree(30 * OK, 1)

    def call(p=None, st=None, tree=tr, q=at(3), k=at(4), v=at(5), ks=at(11), vs=at(12), lens=at(6), n=64, cap=64, out=at(7), ws=at(8), wsb=1 << 28):
        return lib.ea_attend_tree_fp8(byref(p or params()), q, byref(st or step()), byref(tree) if tree else None, k, v, ks, vs, lens, n, cap, out,
                                      None, ws, wsb, None)
    assert call(p=params(d=64)) == 2 and call(p=params(dtype=ea.EA_F32)) == 2 and call(p=params(dtype=ea.EA_FP8_E4M3)) == 2
    assert call(tree=None) == 1 and call(tree=EaTree(None, 1)) == 1 and call(tree=EaTree(30 * OK, 5)) == 2 and call(st=step(max_new=65)) == 1
    for name in ("q", "k", "v", "lens", "out", "ws"):
        assert call(**{name: None}) == 1, name
    assert call(ks=VP(OK + 2)) == 1 and call(vs=VP(OK + 2)) == 1 and call(n=65) == 1 and call(cap=0, n=0) == 1 and call(wsb=16) == 3
    assert call(out=at(3)) == 1 and call(out=VP(5 * OK + 4096)) == 1 and call(out=at(29)) == 1
    assert call(st=step(n_tokens=0)) == 0 and call(st=step(n_tokens=0), ks=None, vs=None) == 0


def test_mask_refusals(lib):
    def call(st=None, parents=at(3), tree=EaTree(30 * OK, 1), seen=at(4), pos=at(5)):
        return lib.ea_tree_masks(byref(params()), byref(st or step()), parents, byref(tree), seen, pos, None)
    assert call(parents=None) == 1 and call(parents=VP(OK + 2)) == 1 and call(seen=VP(OK + 2)) == 1 and call(pos=VP(OK + 2)) == 1
    assert call(tree=EaTree(None, 1)) == 1 and call(tree=EaTree(30 * OK, 0)) == 1 and call(tree=EaTree(30 * OK, 5)) == 2
    assert call(step(max_new=65)) == 1 and call(step(cu_tokens=None)) == 1 and call(step(n_tokens=-1)) == 1
    assert call(parents=at(29)) == 1 and call(pos=at(3)) == 1 and call(pos=at(29)) == 1 and call(seen=at(5)) == 1
    assert call(pos=at(1)) == 1                                              # positions over the prefix sums
    assert call(step(n_tokens=0)) == 0


def test_accept_refusals(lib):
    def call(st=None, args=(3, 4, 5, 6, 7, 8)):
        return lib.ea_tree_accept(byref(params()), byref(st or step()), *[a if a is None else at(a) for a in args], None)
    for i in range(6):
        assert call(args=tuple(None if j == i else a for j, a in enumerate((3, 4, 5, 6, 7, 8)))) == 1
    for bad in ((3, 4, 5, 3, 7, 8), (3, 4, 5, 6, 4, 8), (3, 4, 5, 6, 7, 5), (3, 4, 5, 6, 6, 8), (3, 4, 5, 6, 7, 7), (3, 4, 5, 1, 7, 8)):
        assert call(args=bad) == 1, bad
    assert call(step(max_new=257)) == 2 and call(step(max_new=0)) == 1


def test_keep_refusals(lib):
    def forms(st=None, path=at(3), n_path=at(4), lens=at(5), out=at(6), slots=None, k=at(11), v=at(12), mx=None, p=None):
        s, pp = byref(st or step()), byref(p or params())
        return [lib.ea_keep_path(pp, s, path, n_path, k, v, lens, 64, out, None),
                lib.ea_keep_path_paged(pp, s, path, n_path, k, v, byref(PG), slots, lens, out, None),
                lib.ea_keep_path_mx(pp, s, path, n_path, byref(mx or pools()), byref(PG), slots, lens, out, None)]
    assert forms(path=None) == [1] * 3 and forms(n_path=None) == [1] * 3 and forms(lens=None) == [1] * 3 and forms(out=None) == [1] * 3
    assert forms(out=at(5)) == [1] * 3 and forms(out=at(3)) == [1] * 3 and forms(out=at(1)) == [1] * 3
    assert forms(step(max_new=257)) == [2] * 3 and forms(step(cu_tokens=None)) == [1] * 3
    assert forms(k=None)[:2] == [1, 1] and forms(v=at(11))[:2] == [1, 1] and forms(k=at(4))[:2] == [1, 1] and forms(out=at(12))[:2] == [1, 1]
    assert forms(slots=VP(OK + 4))[1:] == [1, 1]
    assert forms(p=params(dtype=ea.EA_F32))[1:] == [2, 2] and forms(p=params(dtype=ea.EA_FP8_E4M3))[1:] == [2, 2]
    assert forms(out=VP(22 * OK))[2] == 1
    for kw, code in BAD_POOLS:
        assert forms(mx=pools(**kw))[2] == code, kw
    assert lib.ea_keep_path(byref(params()), byref(step()), at(3), at(4), at(11), at(12), at(5), 0, at(6), None) == 1


def test_handles_check_their_tensors():
    import torch
    k, s = torch.zeros(3, 2, 16, 128, dtype=torch.uint8), torch.zeros(3, 2, 16, 4, dtype=torch.uint8)
    ea.make_mx(k, k.clone(), s, s.clone(), ea.EA_MXFP8)
    ea.make_mx(k[..., :64].contiguous(), k[..., 64:].contiguous(), s, s.clone(), ea.EA_MXFP4)
    for bad in ((k, k, s[..., :2].contiguous(), s, ea.EA_MXFP8), (k, k, s, s, ea.EA_MXFP4), (k.float(), k, s, s, ea.EA_MXFP8),
                (k[:, :, ::2], k[:, :, ::2], s[:, :, ::2], s[:, :, ::2], ea.EA_MXFP8), (k, k[:2], s, s[:2], ea.EA_MXFP8)):
        with pytest.raises(ValueError):
            ea.make_mx(*bad)
    ea.make_tree(torch.zeros(5, 2, dtype=torch.int64))
    for bad in (torch.zeros(5, dtype=torch.int64), torch.zeros(5, 2, dtype=torch.int32), torch.zeros(5, 4, dtype=torch.int64)[:, ::2],
                torch.zeros(5, 2, dtype=torch.float64), torch.zeros(5, 2, dtype=torch.complex64)):
        with pytest.raises(ValueError):
            ea.make_tree(bad)
