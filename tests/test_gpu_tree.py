"""Drafted trees on the GPU against their fp64 oracle: masks and positions, attention, the accepted branch and its rows.

Whole numbers and moved rows are exact.  Attention's tolerances are `attend_bounds` of the step's tests."""
import numpy as np
import pytest

from ea_inputs import inv_freq_table, make_block_pools, widen
from ea_inputs.torch_io import to_dev, to_host
from oracle import ea_draft as D
import paper_2510_00636_amd as ea
from tests.test_gpu_mx import BITS, Mx, empty_pools, queries, sums
from tests.test_gpu_step import HALF, attend_bounds, attend_inputs, i32, kind, outputs, store

pytestmark = pytest.mark.gpu


def trees(r, m, how="mixed"):
    """parents of all tokens: now and then a token without one, or one that makes no sense"""
    out = []
    for a in m:
        for i in range(a):
            x = i - 1 if how == "chain" else int(r.integers(max(0, i - 7), i)) if i else -1
            if how == "mixed" and i and r.random() < 0.1:
                x = int(r.choice([-1, -5, i, i + 3, 1 << 30]))
            out.append(x)
    return np.array(out, dtype=np.int64)


def handle(sees, t, words):
    """masks on the device, of t tokens"""
    w = np.zeros((t, words), dtype=np.uint64)
    w[:sees.shape[0]] = D.words_of(sees, words)
    w[sees.shape[0]:] = ~np.uint64(0)
    return to_dev(w.view(np.int64))


# ----------------------------------------------------------------------------------- bookkeeping
@pytest.mark.parametrize("m", [[1], [16], [0, 3, 64, 1], [65, 7, 128], [256, 1, 200, 0, 33]])
@pytest.mark.parametrize("how", ["mixed", "chain"])
def test_masks_and_positions(m, how):
    import torch
    r = np.random.default_rng(sum(m))
    cu, t = sums(m), sum(m)
    parents, seen = trees(r, m, how), r.integers(0, 1 << 20, len(m))
    least = -(-max(m) // 64)
    for words in sorted({least, 4}):
        for with_seen in (True, False):
            sees = torch.full((t + 3, words), -7, dtype=torch.int64, device="cuda")
            pos = torch.full((t + 3,), -7, dtype=torch.int32, device="cuda")
            p, step = ea.make_params(len(m), 2, 1, 64, ea.EA_BF16), ea.make_step(i32(cu), t + 3, max(m))
            ea.tree_masks(p, step, i32(list(parents) + [0] * 3), ea.make_tree(sees), pos, i32(seen) if with_seen else None)
            torch.cuda.synchronize()
            want, at = D.masks(parents, cu, seen if with_seen else None)
            assert np.array_equal(to_host(sees)[:t].view(np.uint64), D.words_of(want, words))
            assert np.array_equal(to_host(pos)[:t], at)
            assert (to_host(sees)[t:] == -7).all() and (to_host(pos)[t:] == -7).all()
    ea.tree_masks(p, step, i32(list(parents) + [0] * 3), ea.make_tree(sees))       # positions are not asked for
    torch.cuda.synchronize()


def test_masks_of_a_sequence_that_adds_more_than_there_are_words():
    import torch
    m = [100, 5]
    cu, parents = sums(m), trees(np.random.default_rng(1), m, "chain")
    sees = torch.full((105, 1), -7, dtype=torch.int64, device="cuda")
    ea.tree_masks(ea.make_params(2, 2, 1, 64, ea.EA_BF16), ea.make_step(i32(cu), 105, 64), i32(parents), ea.make_tree(sees))
    torch.cuda.synchronize()
    want = D.words_of(D.masks(parents, cu)[0], 1)
    got = to_host(sees).view(np.uint64)
    assert np.array_equal(got[:64], want[:64]) and np.array_equal(got[100:], want[100:]) and (to_host(sees)[64:100] == -7).all()


def drafted(r, m, few=6):
    """parents, drafted tokens of a small vocabulary (children with the same token among them) and the model's answers"""
    parents = trees(r, m)
    return parents, r.integers(0, few, sum(m)), r.integers(0, few, sum(m))


@pytest.mark.parametrize("m", [[1], [16], [0, 3, 64, 1], [65, 7, 128], [256, 1, 200, 0, 33], [256] * 9])
@pytest.mark.parametrize("few", [1, 3, 50])
def test_accepted_branches(m, few):
    import torch
    r = np.random.default_rng(few + sum(m))
    parents, tokens, target = drafted(r, m, few)
    cu, B, most = sums(m), len(m), max(m) + 2
    path = torch.full((B, most), -7, dtype=torch.int32, device="cuda")
    n_path, nxt = (torch.full((B,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    step = ea.make_step(i32(cu), sum(m), min(most, 256))
    path = path[:, :min(most, 256)].contiguous()
    ea.tree_accept(ea.make_params(B, 2, 1, 64, ea.EA_BF16), step, i32(tokens), i32(parents), i32(target), path, n_path, nxt)
    torch.cuda.synchronize()
    want, behind = D.accept(tokens, parents, target, cu)
    assert list(to_host(n_path)) == [len(x) for x in want] and list(to_host(nxt)) == behind
    for got, x in zip(to_host(path), want):
        assert list(got[:len(x)]) == x and (got[len(x):] == -7).all()


def test_a_chain_that_is_accepted_to_its_end():
    import torch
    m = [256, 64]
    cu, parents = sums(m), trees(None, m, "chain")
    tokens = np.arange(320)
    path = torch.full((2, 256), -7, dtype=torch.int32, device="cuda")
    n_path, nxt = i32([0, 0]), i32([0, 0])
    ea.tree_accept(ea.make_params(2, 2, 1, 64, ea.EA_BF16), ea.make_step(i32(cu), 320, 256), i32(tokens), i32(parents), i32(tokens + 1), path, n_path, nxt)
    torch.cuda.synchronize()
    assert list(to_host(n_path)) == m and list(to_host(nxt)) == [256, 320]
    assert np.array_equal(to_host(path)[0], np.arange(256)) and np.array_equal(to_host(path)[1, :64], np.arange(64))


def ways(r, m, B):
    """paths [B, most], their counts, and the part of them that counts"""
    most = max(max(m), 1)
    path, count, good = np.full((B, most), -9), np.zeros(B, dtype=int), []
    for b in range(B):
        a = m[b]
        if a == 0:
            good.append([])
            count[b] = 3                                       # more than there are tokens
            continue
        x = sorted(r.choice(a, int(r.integers(1, a + 1)), replace=False).tolist())
        path[b, :len(x)], count[b] = x, len(x)
        good.append(x)
    return path, count, good


@pytest.mark.parametrize("form,d", [("paged", 128), ("paged", 64), ("paged", 256), ("mx8", 128), ("mx8", 64), ("mx4", 256), ("mx4", 64),
                                    ("heads", 128), ("f32", 64), ("f32", 256), ("fp8", 128)])
@pytest.mark.parametrize("m", [[1, 1], [16, 0, 5, 1], [200, 64, 3, 256]])
def test_rows_of_the_branch(form, d, m):
    import torch
    r = np.random.default_rng(d + sum(m))
    B, hkv, bs, cu = len(m), 3, 16, sums(m)
    path, count, good = ways(r, m, B)
    if len(m) == 4 and m[0] > 8:                               # paths that end in front of what makes no sense
        path[0, :6], count[0], good[0] = [0, 2, 5, 5, 6, 7], 6, [0, 2, 5]
        path[2, :2], count[2], good[2] = [1, 3], 2, [x for x in (1, 3) if x < m[2]]
        path[3, :2], count[3], good[3] = [-1, 0], 300, []
    per_head = form in ("heads", "f32", "fp8")
    rows = {"paged": 2 * d, "mx8": d, "mx4": d // 2, "heads": 2 * d, "f32": 4 * d, "fp8": d}[form]
    cap = max(m) + 90
    lens = r.integers(max(m), cap - 5, (B, hkv))
    if not per_head:
        lens[:] = lens[:, :1]
    else:
        lens[-1, 0] = cap + 4                                  # rows that are not there
    if m[1] > 2:
        lens[1] = m[1] - 2                                     # the first two tokens have no row
    widths = [rows, rows] + ([d // 32, d // 32] if form.startswith("mx") else [])
    p = ea.make_params(B, hkv, hkv, d, ea.EA_F32 if form == "f32" else ea.EA_FP8_E4M3 if form == "fp8" else ea.EA_BF16)
    step = ea.make_step(i32(cu), sum(m) + 4, path.shape[1])
    if per_head:
        host = [r.integers(0, 256, (B, hkv, cap, w)).astype(np.uint8) for w in widths]
        where = lambda b, h, row: (b, h, row) if 0 <= row < cap else None    # noqa: E731
    else:
        mb = -(-cap // bs)
        nb = B * mb + 2
        table = r.permutation(nb)[:B * mb].reshape(B, mb)
        host = [r.integers(0, 256, (nb, hkv, bs, w)).astype(np.uint8) for w in widths]
        where = lambda b, h, row: (table[b, row // bs], h, row % bs) if 0 <= row < mb * bs else None    # noqa: E731
        t = i32(table)
        pg = ea.make_paged(t, bs, nb)
    for skipped in ((False,) if per_head else (False, True)):
        slots = np.arange(sum(m) + 4, dtype=np.int64)
        want, want_len = [x.copy() for x in host], lens.copy()
        if skipped:
            slots[cu[0]:cu[1]] = -1                            # the first sequence was not served
        for b in range(B):
            if m[b] == 0 or (skipped and b == 0):
                continue
            for h in range(hkv):
                base = lens[b, h] - m[b]
                want_len[b, h] = max(base + len(good[b]), 0)
                for j, x in enumerate(good[b]):
                    frm, to = where(b, h, base + x), where(b, h, base + j)
                    if frm is not None and to is not None:
                        for y in want:
                            y[to] = y[frm]
        dev = [to_dev(x) for x in host]
        out = torch.full((B, hkv) if per_head else (B,), -7, dtype=torch.int32, device="cuda")
        ld = i32(lens if per_head else lens[:, 0])
        if per_head:
            ea.keep_path(p, step, i32(path), i32(count), dev[0], dev[1], ld, cap, out)
        elif form == "paged":
            ea.keep_path_paged(p, step, i32(path), i32(count), dev[0], dev[1], pg, ld, out, to_dev(slots) if skipped else None)
        else:
            ea.keep_path_mx(p, step, i32(path), i32(count), ea.make_mx(*dev, BITS[8 if form == "mx8" else 4]), pg, ld, out, to_dev(slots) if skipped else None)
        torch.cuda.synchronize()
        assert np.array_equal(to_host(out), want_len if per_head else want_len[:, 0])
        for x, y in zip(dev, want):
            assert np.array_equal(to_host(x), y)


# ------------------------------------------------------------------------------------- attention
def check(got, lse, q, cu, k, v, lens, sees, dt):
    t, d = int(cu[-1]), q.shape[-1]
    want = D.attend(widen(q)[:t], cu, k, v, lens, sees)
    tol, tol_lse = attend_bounds(want, dt, int(lens.max()), d)
    out = widen(got)[:t]
    assert np.isfinite(out).all()
    worst = np.abs(out - want[0]) / tol
    assert worst.max() <= 1, worst.max()
    empty = ~np.isfinite(want[1])
    assert (out[empty] == 0).all() and (lse[:t][empty] == -np.inf).all()
    assert (np.abs(lse[:t] - want[1])[~empty] <= tol_lse[~empty]).all()


def some_masks(r, m, how):
    """what the tokens see: a tree's masks, or any: none of the new rows, all of them, a random half"""
    cu, most = sums(m), max(max(m), 1)
    if how == "tree":
        return D.masks(trees(r, m), cu)[0]
    sees = r.random((int(cu[-1]), most)) < r.choice([0.0, 0.5, 1.0], (int(cu[-1]), 1))
    for b, a in enumerate(m):                                  # bits of tokens that there are not, set
        sees[cu[b]:cu[b + 1], a:] = True
    return sees


def run(form, q, cu, masks, words, k, v, lens, n=None, max_new=None, bs=16):
    """over tensors [B, H, cap, d] as stored; pools are made of them for "paged" """
    import torch
    B, hkv, cap, d = k.shape
    dt = "f32" if form == "f32" else "bf16"
    p = ea.make_params(B, q.shape[1], hkv, d, kind(dt))
    step = ea.make_step(i32(cu), q.shape[0], max(1, int(np.diff(cu).max())) if max_new is None else max_new)
    sees = handle(masks, q.shape[0], words)
    tree = ea.make_tree(sees)
    out, lse = outputs(q, dt)
    if form == "paged":
        kp, vp, table, nb = make_block_pools(k, v, bs, 1)
        for b in range(B):
            table[b, -(-int(lens[b, 0]) // bs):] = -99
        t, n = i32(table), table.shape[1] * bs if n is None else n
        ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
        ea.attend_tree_paged(p, to_dev(q), step, tree, to_dev(kp), to_dev(vp), ea.make_paged(t, bs, nb), i32(lens[:, 0]), n, out, lse, ws)
    else:
        n = cap if n is None else n
        ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
        ea.attend_tree(p, to_dev(q), step, tree, to_dev(k), to_dev(v), i32(lens), n, cap, out, lse, ws)
    torch.cuda.synchronize()
    return to_host(out), lse.cpu().numpy()


def run_mx(c, q, cu, masks, words, hq, hkv, d, max_new=None, n=None):
    import torch
    p, n = ea.make_params(len(c.lens), hq, hkv, d, ea.EA_BF16), c.n if n is None else n
    step = ea.make_step(i32(cu), q.shape[0], max(1, int(np.diff(cu).max())) if max_new is None else max_new)
    sees = handle(masks, q.shape[0], words)
    out, lse = outputs(q, "bf16")
    ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
    ea.attend_tree_mx(p, to_dev(q), step, ea.make_tree(sees), c.mx, c.pg, c.ld, n, out, lse, ws)
    torch.cuda.synchronize()
    return to_host(out), lse.cpu().numpy()


STEPS = [[1, 1, 1], [16, 1, 5], [8, 0, 3], [64, 33, 2], [100, 1, 70], [256, 130, 17]]


@pytest.mark.parametrize("form,hq,hkv,d", [("paged", 8, 2, 128), ("paged", 6, 2, 64), ("paged", 4, 2, 256), ("paged", 20, 1, 128), ("paged", 16, 16, 64),
                                           ("heads", 8, 2, 128), ("heads", 4, 2, 256), ("f32", 4, 2, 64), ("f32", 4, 1, 128), ("f32", 256, 4, 256)])
@pytest.mark.parametrize("m", STEPS)
@pytest.mark.parametrize("how", ["tree", "any"])
def test_trees(form, hq, hkv, d, m, how):
    if form == "f32" and d == 256 and sum(m) > 200:
        m = [40, 3, 1]
    r = np.random.default_rng(d + sum(m) + hq)
    lens = r.integers(max(m), max(m) + 300, (3, hkv))
    lens[1] = m[1]                                             # nothing in front of the tree: rows that see nothing
    lens[2, -1] = max(0, m[2] - 2) if m[2] > 2 else lens[2, -1]      # fewer rows than tokens
    if form == "paged":
        lens[:] = lens[:, -1:]
    dt = "f32" if form == "f32" else "bf16"
    q, cu, k, v, L = attend_inputs(hq + d, hq, hkv, d, dt, lens, m, room=3)
    sees = some_masks(r, m, how)
    for words in sorted({-(-max(m) // 64), 4}):
        got, lse = run(form, q, cu, sees, words, k, v, L)
        full = np.pad(sees, ((0, 0), (0, words * 64 - sees.shape[1])))      # (bits behind a sequence's tokens name no row)
        check(got, lse, q, cu, widen(k), widen(v), L, full, dt)
        assert (widen(got)[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("bits,hq,hkv,d", [(8, 8, 2, 128), (8, 6, 2, 64), (4, 4, 2, 256), (4, 20, 1, 128), (4, 8, 4, 64)])
@pytest.mark.parametrize("m", STEPS)
@pytest.mark.parametrize("how", ["tree", "any"])
def test_trees_over_quantised_pools(bits, hq, hkv, d, m, how):
    r = np.random.default_rng(d + sum(m))
    lens = r.integers(max(m), max(m) + 300, 3)
    lens[1] = m[1]
    lens[2] = max(0, m[2] - 2) if m[2] > 2 else lens[2]
    c = Mx(hq + d, lens, hkv, d, 16, bits)
    cu = sums(m)
    q = queries(d, int(cu[-1]) + 2, hq, d)
    sees = some_masks(r, m, how)
    words = -(-max(m) // 64)
    got, lse = run_mx(c, q, cu, sees, words, hq, hkv, d)
    check(got, lse, q, cu, c.val[0], c.val[1], np.repeat(c.lens[:, None], hkv, 1), np.pad(sees, ((0, 0), (0, words * 64 - sees.shape[1]))), "bf16")
    assert (widen(got)[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("form,hq,hkv,d", [("paged", 8, 2, 128), ("heads", 6, 2, 64), ("paged", 4, 2, 256), ("f32", 4, 2, 64), ("mx8", 8, 2, 128), ("mx4", 4, 2, 256)])
@pytest.mark.parametrize("m,lens", [([16], [4500]), ([64], [4100]), ([200, 20], [3500, 4400])])
def test_trees_behind_long_heads(form, hq, hkv, d, m, lens):
    r = np.random.default_rng(d + sum(m))
    sees, words = some_masks(r, m, "tree"), -(-max(m) // 64)
    full, cu = np.pad(sees, ((0, 0), (0, words * 64 - sees.shape[1]))), sums(m)
    if form.startswith("mx"):
        c = Mx(hq + d, lens, hkv, d, 32, int(form[2:]))
        q = queries(d, int(cu[-1]), hq, d)
        got, lse = run_mx(c, q, cu, sees, words, hq, hkv, d)
        check(got, lse, q, cu, c.val[0], c.val[1], np.repeat(c.lens[:, None], hkv, 1), full, "bf16")
        return
    dt = "f32" if form == "f32" else "bf16"
    q, cu, k, v, L = attend_inputs(hq + d, hq, hkv, d, dt, lens, m)
    got, lse = run(form, q, cu, sees, words, k, v, L)
    check(got, lse, q, cu, widen(k), widen(v), L, full, dt)


@pytest.mark.parametrize("form", ["paged", "heads", "f32"])
@pytest.mark.parametrize("max_new", [9, 40, 200])
def test_many_sequences_and_loose_bounds(form, max_new):
    r = np.random.default_rng(max_new)
    B, d = 140, 64
    m = r.integers(0, 9, B)
    lens = np.maximum(r.integers(0, 60, (B, 2)), m[:, None])
    if form == "paged":
        lens[:] = lens[:, :1]
    dt = "f32" if form == "f32" else "bf16"
    q, cu, k, v, L = attend_inputs(3, 4, 2, d, dt, lens, m)
    sees, words = some_masks(r, list(m), "any"), -(-max_new // 64)
    got, lse = run(form, q, cu, sees, words, k, v, L, max_new=max_new)
    check(got, lse, q, cu, widen(k), widen(v), L, np.pad(sees, ((0, 0), (0, words * 64 - sees.shape[1]))), dt)


@pytest.mark.parametrize("form", ["paged", "heads", "f32"])
@pytest.mark.parametrize("m", [[5, 1, 9], [30, 90, 2]])
def test_lengths_that_make_no_sense(form, m):
    r = np.random.default_rng(7)
    q, cu, k, v, L = attend_inputs(3, 8, 2, 64, "f32" if form == "f32" else "bf16", [200, 160, 200], m)
    sees, words = some_masks(r, m, "any"), -(-max(m) // 64)
    wild = np.array([[-7, -7], [160, 160], [1 << 30, 1 << 30]])
    got, lse = run(form, q, cu, sees, words, k, v, wild, n=200)
    check(got, lse, q, cu, widen(k), widen(v), np.array([[0, 0], [160, 160], [200, 200]]),
          np.pad(sees, ((0, 0), (0, words * 64 - sees.shape[1]))), "f32" if form == "f32" else "bf16")


@pytest.mark.parametrize("form,hq,hkv,d", [("paged", 8, 2, 128), ("heads", 6, 2, 64), ("paged", 4, 2, 256), ("f32", 4, 2, 64), ("f32", 128, 2, 128),
                                           ("mx8", 8, 2, 128), ("mx4", 4, 2, 256)])
@pytest.mark.parametrize("m", [[5, 16, 3], [60, 1, 130]])
def test_rows_that_a_token_does_not_see_do_not_matter(form, hq, hkv, d, m):
    """Keys and values of the step's rows that are not finite reach the tokens that see them; the others' results keep their bits."""
    r = np.random.default_rng(d + sum(m))
    sees, words = some_masks(r, m, "tree"), -(-max(m) // 64)
    lens, cu = r.integers(max(m), max(m) + 200, 3), sums(m)
    lens[1] = m[1]
    bad = [int(r.integers(0, a)) for a in m]                   # the token of each sequence whose row is spoiled
    last = [a - 1 for a in m]                                  # and one whose key is
    if form.startswith("mx"):
        c = Mx(hq + d, lens, hkv, d, 16, int(form[2:]))
        q = queries(d, int(cu[-1]), hq, d)
        clean, clean_lse = run_mx(c, q, cu, sees, words, hq, hkv, d)
        for b in range(3):
            c.e[1][b, :, lens[b] - m[b] + bad[b], 0] = 255
            c.e[0][b, :, lens[b] - m[b] + last[b], 1] = 255
        c.load()
        got, lse = run_mx(c, q, cu, sees, words, hq, hkv, d)
        channels = np.arange(d) < 32
    else:
        dt = "f32" if form == "f32" else "bf16"
        q, cu, k, v, L = attend_inputs(hq + d, hq, hkv, d, dt, lens, m)
        clean, clean_lse = run(form, q, cu, sees, words, k, v, L)
        k, v = k.copy(), v.copy()
        inf, nan = ((0x7F80, 0x7FC0) if dt == "bf16" else (np.inf, np.nan))
        for b in range(3):
            v[b, :, lens[b] - m[b] + bad[b], 7], v[b, :, lens[b] - m[b] + bad[b], d - 1] = inf, nan
            k[b, :, lens[b] - m[b] + last[b], 3] = nan
        got, lse = run(form, q, cu, sees, words, k, v, L)
        channels = (np.arange(d) == 7) | (np.arange(d) == d - 1)
    got, clean = widen(got), widen(clean)
    hit = False
    for b in range(3):
        for i in range(m[b]):
            t = cu[b] + i
            if sees[t, last[b]]:
                assert np.isnan(got[t]).all() and np.isnan(lse[t]).all()
                continue
            touched = channels & sees[t, bad[b]]
            hit |= bool(touched.any())
            assert not np.isfinite(got[t][:, touched]).any()
            assert np.array_equal(got[t][:, ~touched], clean[t][:, ~touched]) and np.array_equal(lse[t], clean_lse[t])
    assert hit


@pytest.mark.parametrize("form,d,m", [("paged", 128, [1, 1, 1]), ("paged", 128, [7, 12, 1]), ("paged", 256, [90, 5, 64]), ("heads", 64, [100, 3, 40]),
                                      ("f32", 64, [30, 1, 100])])
def test_a_chain_is_what_the_step_does(form, d, m):
    """Masks that see every row up to the token's own give what attention without masks gives, to rounding."""
    r = np.random.default_rng(d)
    dt = "f32" if form == "f32" else "bf16"
    lens = r.integers(max(m), 400, (3, 2))
    if form == "paged":
        lens[:] = lens[:, :1]
    q, cu, k, v, L = attend_inputs(d, 8, 2, d, dt, lens, m)
    sees = D.masks(trees(r, m, "chain"), cu)[0]
    got, lse = run(form, q, cu, sees, 4, k, v, L)
    check(got, lse, q, cu, widen(k), widen(v), L, np.pad(sees, ((0, 0), (0, 256 - sees.shape[1]))), dt)


# -------------------------------------------------------------------------------- all of it, in turn
@pytest.mark.parametrize("form", ["paged", "mx8", "mx4"])
def test_a_loop_of_drafting_steps(form):
    """Blocks, tree positions, rows, attention, the accepted branch, blocks given back: four steps, captured once and replayed, each
    against the oracle."""
    import torch
    hq, hkv, d, bs, B, most, nb, mb = 8, 2, 128, 16, 3, 20, 40, 20
    r = np.random.default_rng(11)
    p, n, T = ea.make_params(B, hq, hkv, d, ea.EA_BF16), mb * bs, B * most
    dev = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype, device="cuda")    # noqa: E731
    bits = int(form[2:]) if form != "paged" else 0
    pools = empty_pools(nb, hkv, bs, d, bits) if bits else [dev(nb, hkv, bs, d, dtype=torch.bfloat16) for _ in range(2)]
    table = torch.full((B, mb), -1, dtype=torch.int32, device="cuda")
    pg = ea.make_paged(table, bs, nb)
    mx = ea.make_mx(*pools, BITS[bits]) if bits else None
    inv_host = inv_freq_table(d, 1e4)
    inv, free, count, lens, seen = to_dev(inv_host), i32(r.permutation(nb)), i32([nb]), i32([0] * B), i32([5, 0, 1000])
    more, wanted, len_new, count_mid, cu, slots, pos = dev(B), dev(B), dev(B), dev(1), dev(B + 1), dev(T, dtype=torch.int64), dev(T)
    parents, tokens, target, sees = dev(T), dev(T), dev(T), dev(T, 1, dtype=torch.int64)
    path, n_path, nxt, len_kept, len_end, count_end, cu_end = dev(B, most), dev(B), dev(B), dev(B), dev(B), dev(1), dev(B + 1)
    x, q = dev(T, hq + 2 * hkv, d, dtype=torch.bfloat16), dev(T, hq, d, dtype=torch.bfloat16)
    out, lse = dev(T, hq, d, dtype=torch.bfloat16), dev(T, hq, dtype=torch.float32)
    rows = ea.make_new_rows(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], pos, inv)
    step, tree = ea.make_step(cu, T, most), ea.make_tree(sees)
    ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda")

    def go():
        torch.add(lens, more, out=wanted)
        ea.block_tables(p, pg, lens, wanted, free, count, len_new, count_mid, cu, T, slots, pos, seen)
        ea.tree_masks(p, step, parents, tree, pos, seen)
        if bits:
            ea.append_mx(p, rows, slots, mx, pg, q)
            ea.attend_tree_mx(p, q, step, tree, mx, pg, len_new, n, out, lse, ws)
        else:
            ea.append_paged(p, rows, slots, *pools, pg, q)
            ea.attend_tree_paged(p, q, step, tree, *pools, pg, len_new, n, out, lse, ws)
        ea.tree_accept(p, step, tokens, parents, target, path, n_path, nxt)
        if bits:
            ea.keep_path_mx(p, step, path, n_path, mx, pg, len_new, len_kept, slots)
        else:
            ea.keep_path_paged(p, step, path, n_path, *pools, pg, len_new, len_kept, slots)
        ea.block_tables(p, pg, len_new, len_kept, free, count_mid, len_end, count_end, cu_end)
        lens.copy_(len_end)
        count.copy_(count_end)

    def rest():
        return [y.clone() for y in (table, free, count, lens, *pools)]
    keep = rest()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        go()                                                   # (no tokens: nothing happens)
    torch.cuda.synchronize()
    for a, b in zip(keep, rest()):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        go()
    torch.cuda.synchronize()

    def row_values():
        """the cache's rows as numbers: [nb, hkv, bs, d] of K and V"""
        if not bits:
            return [widen(to_host(y)) for y in pools]
        return [D.values(D.unpacked(to_host(pools[i]), bits), to_host(pools[2 + i]), bits) for i in range(2)]

    from oracle import ea_step as S
    kept = [[np.zeros((hkv, 0, d)) for _ in range(B)] for _ in range(2)]        # what the sequences hold, by the oracle
    length, place = np.zeros(B, dtype=int), np.array([5, 0, 1000])
    for m in ([20, 1, 7], [12, 20, 0], [1, 1, 1], [20, 20, 20]):
        add = np.array(m)
        par = np.concatenate([trees(r, [a], "tree") for a in m] + [np.zeros(0, dtype=int)])
        tok, tgt = r.integers(0, 3, sum(m)), r.integers(0, 3, sum(m))
        xs = store(r.standard_normal((T, hq + 2 * hkv, d)), "bf16")
        x.copy_(to_dev(xs))
        more.copy_(i32(add))
        seen.copy_(i32(place))
        for to, val in ((parents, par), (tokens, tok), (target, tgt)):
            to.zero_()
            to[:sum(m)] = i32(val)
        ws.fill_(0xA5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c = sums(m)
        masks, at = D.masks(par, c, place)
        assert np.array_equal(to_host(sees)[:sum(m), 0].view(np.uint64), D.words_of(masks, 1)[:, 0]) and np.array_equal(to_host(pos)[:sum(m)], at)
        paths, behind = D.accept(tok, par, tgt, c)
        assert list(to_host(n_path)) == [len(y) for y in paths] and list(to_host(nxt)) == behind
        xf = widen(xs)
        key = S.rotate(xf[:sum(m), hq:hq + hkv], at, inv_host, False)
        # rows as they stand in the cache, rounded as its type rounds (a bf16 key that lies next to a border: half a step of the other one)
        val = xf[:sum(m), hq + hkv:]
        if bits:
            key, val = (D.values(*D.quantise(y, bits), bits) for y in (key, val))
        ks = [np.concatenate([kept[0][b], key[c[b]:c[b + 1]].transpose(1, 0, 2)], axis=1) for b in range(B)]
        vs = [np.concatenate([kept[1][b], val[c[b]:c[b + 1]].transpose(1, 0, 2)], axis=1) for b in range(B)]
        full = np.repeat((length + add)[:, None], hkv, 1)
        qf = to_host(q)[:max(sum(m), 1)]
        want = D.attend(widen(qf)[:sum(m)], c, ks, vs, full, np.pad(masks, ((0, 0), (0, 64 - masks.shape[1]))))
        tol, tol_lse = attend_bounds(want, "bf16", int(full.max()), d)
        if not bits:       # keys are rounded to bf16 in the cache: each logit, and with it a weight, moves by up to that
            moved = HALF["bf16"] * want[3]
            tol, tol_lse = tol + (2 * moved)[..., None] * want[2], tol_lse + moved
        got = widen(to_host(out))[:sum(m)]
        assert (np.abs(got - want[0]) <= tol).all() and (np.abs(to_host(lse)[:sum(m)] - want[1]) <= tol_lse).all()
        length = length + np.array([len(y) for y in paths])
        assert np.array_equal(to_host(lens), length)
        for i, (old, new) in enumerate(((ks, key), (vs, val))):
            for b in range(B):
                k0 = old[b].shape[1] - m[b]
                kept[i][b] = np.concatenate([old[b][:, :k0], old[b][:, k0:][:, paths[b]]], axis=1) if m[b] else old[b]
        now, tab = row_values(), to_host(table)
        for i in range(2):
            for b in range(B):
                for j in range(length[b]):
                    cell = now[i][tab[b, j // bs], :, j % bs]
                    if i == 1 or bits:
                        assert np.array_equal(cell, kept[i][b][:, j])
                    else:
                        assert (np.abs(cell - kept[i][b][:, j]) <= HALF["bf16"] * np.abs(cell) * 1.01 + 1e-5).all()
        held = sorted(int(tab[b, j]) for b in range(B) for j in range(-(-length[b] // bs)))
        assert sorted(held + to_host(free)[:int(count[0])].tolist()) == list(range(nb))
        place = place + np.array([len(y) for y in paths])


def test_sequences_that_were_not_served_keep_their_rows():
    """Too few blocks for a tree: its tokens have no rows, and the branch that their masks would give moves none."""
    import torch
    hkv, d, bs, B, nb, mb = 2, 128, 16, 2, 3, 4
    p = ea.make_params(B, 4, hkv, d, ea.EA_BF16)
    table, free, count = i32([[0, -1, -1, -1], [1, -1, -1, -1]]), i32([2, -1, -1]), i32([1])
    pg, old, new = ea.make_paged(table, bs, nb), i32([10, 12]), i32([20, 22])
    len_out, count_out, cu = i32([0, 0]), i32([0]), i32([0, 0, 0])
    slots, pos = torch.zeros(20, dtype=torch.int64, device="cuda"), i32([0] * 20)
    ea.block_tables(p, pg, old, new, free, count, len_out, count_out, cu, 20, slots, pos)
    k = torch.arange(nb * hkv * bs * d, device="cuda").to(torch.bfloat16).view(nb, hkv, bs, d)
    v, before = k.clone(), k.clone()
    path, n_path, kept = i32([[0, 3, 9] + [0] * 7] * 2), i32([3, 3]), i32([-7, -7])
    ea.keep_path_paged(p, ea.make_step(cu, 20, 10), path, n_path, k, v, pg, len_out, kept, slots)
    torch.cuda.synchronize()
    assert list(to_host(kept)) == [13, 12]
    assert torch.equal(k[1], before[1]) and torch.equal(v[1], before[1])
    want = before.clone()
    want[0, :, 11], want[0, :, 12] = before[0, :, 13], before[2, :, 3]
    assert torch.equal(k, want) and torch.equal(v, want)
