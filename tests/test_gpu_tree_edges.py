"""Attention of drafted trees on the GPU where a call's bounds say little of what it finds, against the fp64 oracle.

Tolerances are those of the step's tests: `two_number_bounds` where weights are the sum of two bf16 numbers, which weights of one pass."""
import numpy as np
import pytest

from ea_inputs import make_block_pools, widen
from ea_inputs.torch_io import to_dev, to_host
from oracle import ea_draft as D
import paper_2510_00636_amd as ea
from tests.test_gpu_mx import Mx, sums
from tests.test_gpu_step import i32, outputs, store
from tests.test_gpu_step_values import opposite_values, two_number_bounds
from tests.test_gpu_tree import handle, trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form,hq,hkv,d,m,most,n", [("paged", 8, 2, 128, [1, 1, 1], 32, 30000), ("paged", 8, 2, 128, [1], 100, 20000), ("paged", 16, 4, 64, [1, 2, 4, 1], 20, 16000),
                                                    ("paged", 4, 2, 256, [8, 1], 64, 50000), ("mx8", 8, 2, 128, [1, 3, 4], 32, 30000), ("mx4", 8, 2, 128, [1], 100, 20000),
                                                    ("mx8", 4, 2, 256, [1, 4], 40, 4128), ("mx4", 4, 2, 256, [8], 60, 9000),
                                                    ("heads", 8, 2, 128, [2, 1, 1], 32, 30000), ("fp8", 4, 2, 256, [1, 1, 8], 40, 3000)])
@pytest.mark.parametrize("more", [0, 1])
def test_room_for_tokens_is_not_taken_for_tokens(form, hq, hkv, d, m, most, n, more):
    """Sequences that add few tokens under bounds as a captured step has them, with room for as many as these allow: their weights are two
    bf16 numbers, as without that room."""
    import torch
    B, cu = len(m), sums(m)
    lens = np.array([900 - 3 * b for b in range(B)])
    sees = D.masks(trees(np.random.default_rng(d), m, "chain"), cu)[0]
    t, room, words = int(cu[-1]), B * most + more, -(-most // 64)
    q, _, k, v, kf, vf = opposite_values(n + d, hq, hkv, d, "fp8" if form == "fp8" else "bf16", lens, m)
    rooms = np.concatenate([q, np.zeros((room - t, hq, d), dtype=q.dtype)])
    p, step = ea.make_params(B, hq, hkv, d, ea.EA_BF16), ea.make_step(i32(cu), room, most)
    tree = ea.make_tree(handle(sees, room, words))
    out, lse = outputs(rooms, "bf16")
    ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
    qd, bs = to_dev(rooms), 16
    if form in ("heads", "fp8"):
        ld = i32(np.repeat(lens[:, None], hkv, 1))
        kd, vd = (torch.zeros((B, hkv, n, d), dtype=torch.uint8 if form == "fp8" else torch.bfloat16, device="cuda") for _ in range(2))
        for x, y in ((kd, k), (vd, v)):
            x[:, :, :y.shape[2]] = to_dev(y)
        call = ea.attend_tree_fp8 if form == "fp8" else ea.attend_tree
        call(p, qd, step, tree, kd, vd, *((None, None) if form == "fp8" else ()), ld, n, n, out, lse, ws)
    elif form == "paged":
        kp, vp, table, nb = make_block_pools(k, v, bs, 1)
        wide = np.full((B, -(-n // bs)), -99)
        wide[:, :table.shape[1]] = table
        td = i32(wide)
        ea.attend_tree_paged(p, qd, step, tree, to_dev(kp), to_dev(vp), ea.make_paged(td, bs, nb), i32(lens), n, out, lse, ws)
    else:
        bits = int(form[2:])
        c = Mx(1, lens, hkv, d, bs, bits)
        for i, x in ((0, kf), (1, vf)):
            c.codes[i], c.e[i] = D.quantise(x, bits)
        kf, vf = (D.values(c.codes[i], c.e[i], bits) for i in (0, 1))
        c.load()
        wide = np.full((B, -(-n // bs)), -99)
        wide[:, :c.table.shape[1]] = c.table
        td = i32(wide)
        ea.attend_tree_mx(p, qd, step, tree, c.mx, ea.make_paged(td, bs, c.nb), c.ld, n, out, lse, ws)
    torch.cuda.synchronize()
    want = D.attend(widen(q), cu, kf, vf, np.repeat(lens[:, None], hkv, 1), np.pad(sees, ((0, 0), (0, words * 64 - sees.shape[1]))))
    tol, tol_lse = two_number_bounds(want, int(lens.max()), d)
    got = widen(to_host(out))
    worst = np.abs(got[:t] - want[0]) / tol
    assert worst.max() <= 1, worst.max()
    assert (np.abs(lse.cpu().numpy()[:t] - want[1]) <= tol_lse).all()
    assert (got[t:] == 7.0).all()
