"""Stretches that are cut along the keys and joined again, on the GPU: how many rows a group of threads joins follows from the room that a
call has for tokens, and changes no bit (but up to 4096 rows a workgroup joins a row, its pieces in another order); and against the fp64
oracle, with the tolerances of the step's tests."""
import numpy as np
import pytest

from ea_inputs import make_block_pools, quantize_fp8, widen
from ea_inputs.torch_io import to_dev, to_host
from oracle import ea_draft as D
from oracle import ea_step as S
import paper_2510_00636_amd as ea
from tests.test_gpu_mx import Mx, sums
from tests.test_gpu_step import attend_bounds, attend_inputs, i32, kind, outputs
from tests.test_gpu_tree import handle, some_masks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form,hq,hkv,d,m,lens", [
    ("heads", 32, 2, 128, [130, 1, 90], [900, 3000, 700]), ("paged", 16, 4, 64, [200, 70], [2100, 500]), ("paged", 8, 2, 256, [300, 2], [1500, 40]),
    ("f32", 16, 2, 64, [60, 1, 30], [1800, 3, 900]), ("f32", 8, 2, 256, [40], [2000]), ("fp8", 32, 4, 128, [130, 40], [1200, 900]), ("mx8", 16, 2, 128, [150, 3], [2000, 600]),
    ("mx4", 16, 2, 64, [150, 3], [2000, 600])])
@pytest.mark.parametrize("masks", [False, True])
def test_rows_joined_together_or_alone(form, hq, hkv, d, m, lens, masks):
    check(form, hq, hkv, d, m, lens, masks, True)


@pytest.mark.parametrize("form", ["heads", "paged", "mx8", "f32"])
@pytest.mark.parametrize("masks", [False, True])
def test_rows_of_many_sequences(form, masks):
    """More sequences than a wavefront has lanes, some of which add nothing and some a token."""
    r = np.random.default_rng(1)
    m = r.choice([0, 1, 1, 2, 40, 70], 90)
    check(form, 8, 2, 64, list(m), list(r.integers(300, 900, 90)), masks, False)


def check(form, hq, hkv, d, m, lens, masks, oracle):
    import torch
    dt, B = "f32" if form == "f32" else "bf16", len(m)
    lens = np.maximum(np.asarray(lens), m)
    cu = sums(m)
    t = int(cu[-1])
    q, _, k, v, L = attend_inputs(d + t, hq, hkv, d, dt, lens, m)
    sees, words = some_masks(np.random.default_rng(t), list(m), "tree"), -(-max(m) // 64)
    if max(m) > 256:
        masks = False
    some, many = max(t, 4096 // hq + 1), 32768 // hq + 100      # tokens that make more than 4096, and more than 32768 rows
    assert some * hq <= 32768
    p = ea.make_params(B, hq, hkv, d, kind(dt))
    vf = widen(v)
    kf = widen(k)
    if form.startswith("mx"):
        c = Mx(7, lens, hkv, d, 16, int(form[2:]))
        kf, vf = c.val
    elif form == "paged":
        kp, vp, table, nb = make_block_pools(k, v, 16, 1)
        kd, vd, td = to_dev(kp), to_dev(vp), i32(table)
        pg = ea.make_paged(td, 16, nb)
    elif form == "fp8":
        (k8, ks), (v8, vs) = (quantize_fp8(np.nan_to_num(widen(x))) for x in (k, v))
        kd, vd, ksd, vsd = to_dev(k8), to_dev(v8), to_dev(ks), to_dev(vs)
    else:
        kd, vd = to_dev(k), to_dev(v)
    got = []
    for room in (t, some, many):
        x = np.concatenate([q, np.zeros((room - t, hq, d), dtype=q.dtype)])
        step, (out, lse), qd = ea.make_step(i32(cu), room, int(max(m))), outputs(x, dt), to_dev(x)
        tree = ea.make_tree(handle(sees, room, words)) if masks else None
        n = c.n if form.startswith("mx") else table.shape[1] * 16 if form == "paged" else k.shape[2]
        ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
        tail = (out, lse, ws)
        if form.startswith("mx"):
            args = (c.mx, c.pg, c.ld, n)
            ea.attend_tree_mx(p, qd, step, tree, *args, *tail) if masks else ea.attend_mx(p, qd, step, *args, *tail)
        elif form == "paged":
            args = (kd, vd, pg, i32(lens), n)
            ea.attend_tree_paged(p, qd, step, tree, *args, *tail) if masks else ea.attend_paged(p, qd, step, *args, *tail)
        elif form == "fp8":
            args = (kd, vd, ksd, vsd, i32(L), n, n)
            ea.attend_tree_fp8(p, qd, step, tree, *args, *tail) if masks else ea.attend_fp8(p, qd, step, *args, *tail)
        else:
            args = (kd, vd, i32(L), n, n)
            ea.attend_tree(p, qd, step, tree, *args, *tail) if masks else ea.attend(p, qd, step, *args, *tail)
        torch.cuda.synchronize()
        got.append((to_host(out), lse.cpu().numpy()))
    (out, lse), (far, far_lse) = got[1:]
    if dt != "f32":                              # (whose rows of a workgroup, and so the cuts, follow from the room, too)
        assert np.array_equal(out[:t], far[:t]) and np.array_equal(lse[:t], far_lse[:t])
    assert (widen(far)[t:] == 7.0).all() and (far_lse[t:] == 7.0).all()
    if oracle and form != "fp8":
        qf, full = widen(q), np.pad(sees, ((0, 0), (0, words * 64 - sees.shape[1])))
        want = D.attend(qf, cu, kf, vf, L, full) if masks else S.attend(qf, cu, kf, vf, L)
        tol, tol_lse = attend_bounds(want, dt, int(lens.max()), d)
        for out, lse in got:
            assert (np.abs(widen(out)[:t] - want[0]) <= tol).all() and (np.abs(lse[:t] - want[1]) <= tol_lse).all()
