"""Quantised pools and drafted trees where calls are cut unusually: many heads and sequences, both kernels and all widths of their
joining launches, caches past 32 bits, workspaces that calls share.

Tolerances are `attend_bounds` of the step's tests; moved rows are exact."""
import numpy as np
import pytest

from ea_inputs import make_block_pools, quantize_fp8, widen
from ea_inputs.torch_io import to_dev, to_host
from oracle import ea_draft as D
from oracle import ea_extensions as X
import paper_2510_00636_amd as ea
from tests.test_gpu_mx import Mx, queries, run_mx as run_mx_chain, sums
from tests.test_gpu_step import attend_inputs, check_attend, i32, kind, outputs, run_paged
from tests.test_gpu_tree import check, handle, run, run_mx, some_masks

pytestmark = pytest.mark.gpu


def padded(sees, words):
    return np.pad(sees, ((0, 0), (0, words * 64 - sees.shape[1])))


# ----------------------------------------------------------------------- e4m3 rows with a scale per head
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (20, 1, 128), (4, 2, 256), (3, 3, 256)])
@pytest.mark.parametrize("m", [[1, 1, 1], [16, 0, 5], [64, 33, 2], [256, 130, 17]])
@pytest.mark.parametrize("how,scaled", [("tree", True), ("any", True), ("any", False)])
def test_trees_over_scaled_bytes(hq, hkv, d, m, how, scaled):
    import torch
    r = np.random.default_rng(d + sum(m) + hq)
    lens = r.integers(max(m), max(m) + 300, (3, hkv))
    lens[1] = m[1]                                             # nothing in front of the tree
    lens[2, -1] = 4200 if m[0] == 64 else max(0, m[2] - 2)     # a head in many pieces, or one of fewer rows than tokens
    q, cu, k, v, L = attend_inputs(hq + d, hq, hkv, d, "bf16", lens, m, room=3)
    k8, ks = quantize_fp8(np.nan_to_num(widen(k)))
    v8, vs = quantize_fp8(np.nan_to_num(widen(v)))
    if not scaled:
        ks, vs = np.ones_like(ks), np.ones_like(vs)
    else:
        ks[0, 0] = -ks[0, 0]                                   # a scale may have any sign
    for b in range(3):
        for h in range(hkv):
            k8[b, h, L[b, h]:] = v8[b, h, L[b, h]:] = 0x7F
    sees, words = some_masks(r, m, how), -(-max(m) // 64)
    cap = k.shape[2]
    p = ea.make_params(3, hq, hkv, d, ea.EA_BF16)
    step = ea.make_step(i32(cu), q.shape[0], max(m))
    tree = ea.make_tree(handle(sees, q.shape[0], words))
    out, lse = outputs(q, "bf16")
    ws = torch.empty(ea.attend_workspace_bytes(p, step, cap), dtype=torch.uint8, device="cuda").fill_(0xFF)
    ea.attend_tree_fp8(p, to_dev(q), step, tree, to_dev(k8), to_dev(v8), to_dev(ks) if scaled else None, to_dev(vs) if scaled else None,
                       i32(L), cap, cap, out, lse, ws)
    torch.cuda.synchronize()
    live = np.arange(cap)[None, None, :, None] < L[:, :, None, None]
    kf, vf = (np.where(live, X.fp8_e4m3_decode(np.where(live, x, 0).astype(np.uint8)), 0) * s.astype(np.float64)[:, :, None, None]
              for x, s in ((k8, ks), (v8, vs)))
    check(to_host(out), lse.cpu().numpy(), q, cu, kf, vf, L, padded(sees, words), "bf16")
    assert (widen(to_host(out))[cu[-1]:] == 7.0).all() and (lse.cpu().numpy()[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("d,m", [(128, [5, 16, 3]), (128, [60, 1, 130]), (256, [90, 5, 64])])
def test_bytes_that_are_not_numbers(d, m):
    """Rows of e4m3 bytes that are NaN reach the tokens that see them, and no others."""
    import torch
    hq, hkv = 4, 2
    r = np.random.default_rng(d + sum(m))
    lens = r.integers(max(m), max(m) + 200, 3)
    q, cu, k, v, L = attend_inputs(5, hq, hkv, d, "bf16", lens, m)
    k8, _ = quantize_fp8(np.nan_to_num(widen(k)))
    v8, _ = quantize_fp8(np.nan_to_num(widen(v)))
    sees, words = some_masks(r, m, "tree"), -(-max(m) // 64)
    p, step, cap = ea.make_params(3, hq, hkv, d, ea.EA_BF16), ea.make_step(i32(cu), q.shape[0], max(m)), k.shape[2]
    tree = ea.make_tree(handle(sees, q.shape[0], words))
    ws = torch.empty(ea.attend_workspace_bytes(p, step, cap), dtype=torch.uint8, device="cuda")
    got = []
    bad = [int(r.integers(0, a)) for a in m]
    for spoilt in (False, True):
        if spoilt:
            for b in range(3):
                v8[b, :, lens[b] - m[b] + bad[b], 9] = 0xFF
        out, lse = outputs(q, "bf16")
        ea.attend_tree_fp8(p, to_dev(q), step, tree, to_dev(k8), to_dev(v8), None, None, i32(L), cap, cap, out, lse, ws)
        torch.cuda.synchronize()
        got.append((widen(to_host(out)), lse.cpu().numpy()))
    (clean, clean_lse), (now, now_lse) = got
    assert np.array_equal(clean_lse, now_lse) and np.isfinite(clean).all()
    other = np.arange(d) != 9
    assert np.array_equal(clean[:, :, other], now[:, :, other])
    for b in range(3):
        for i in range(m[b]):
            t = cu[b] + i
            if sees[t, bad[b]]:
                assert np.isnan(now[t, :, 9]).all()
            else:
                assert np.array_equal(now[t, :, 9], clean[t, :, 9])


# ------------------------------------------------------------------------------------ many heads, sequences, rows
@pytest.mark.parametrize("form", ["heads", "f32"])
@pytest.mark.parametrize("B,hkv", [(9, 8), (33, 8)])
def test_more_heads_than_lanes_and_than_are_cut_one_by_one(form, B, hkv):
    """72 heads of lengths of their own are cut each for itself, 264 by sequences; some are long, some empty, some of a single token."""
    r = np.random.default_rng(B)
    m = r.choice([1, 3, 70, 130], B, p=[0.4, 0.2, 0.2, 0.2])
    m[0], m[-1], m[B // 2] = 100, 100, 0
    lens = r.integers(0, 400, (B, hkv)) + m[:, None]
    lens[0, 3], lens[-1, 7], lens[1, 0] = 2900, 1500, m[1]
    dt = "f32" if form == "f32" else "bf16"
    q, cu, k, v, L = attend_inputs(B, 2 * hkv, hkv, 64, dt, lens, m)
    sees = some_masks(r, list(m), "any")
    words = -(-int(m.max()) // 64)
    got, lse = run(form, q, cu, sees, words, k, v, L)
    check(got, lse, q, cu, widen(k), widen(v), L, padded(sees, words), dt)


@pytest.mark.parametrize("form", ["paged", "mx8"])
@pytest.mark.parametrize("long", [1900, 2300])
def test_few_trees_among_many_single_tokens(form, long):
    """70 sequences, five of which add a tree: where all lengths are short one kernel takes all of them, else each its own."""
    r = np.random.default_rng(long)
    B, hq, hkv, d = 70, 4, 1, 128
    m = np.ones(B, dtype=int)
    m[[0, 20, 63, 64, 69]] = [65, 90, 40, 128, 20]
    lens = r.integers(0, 60, B) + m
    lens[64], lens[3] = long, long - 40
    sees = some_masks(r, list(m), "any")
    words = -(-int(m.max()) // 64)
    cu = sums(m)
    if form == "paged":
        q, cu, k, v, L = attend_inputs(3, hq, hkv, d, "bf16", lens, m)
        got, lse = run(form, q, cu, sees, words, k, v, L)
        check(got, lse, q, cu, widen(k), widen(v), L, padded(sees, words), "bf16")
        return
    c = Mx(5, lens, hkv, d, 16, 8)
    q = queries(4, int(cu[-1]), hq, d)
    got, lse = run_mx(c, q, cu, sees, words, hq, hkv, d)
    check(got, lse, q, cu, c.val[0], c.val[1], c.lens[:, None], padded(sees, words), "bf16")


@pytest.mark.parametrize("form,B", [("paged", 2), ("paged", 5), ("f32", 2), ("f32", 5), ("heads", 5)])
def test_many_rows_are_joined(form, B):
    """14k to 41k, and 28k to 82k (token, head) rows, the longest of them in pieces."""
    r = np.random.default_rng(B)
    hq, hkv, d = 64, 2, 64
    m = [256] * (B - 1) + [190]
    lens = np.array([2500] + [int(x) for x in r.integers(260, 500, B - 1)])[:, None].repeat(hkv, 1)
    if form == "heads":
        lens[1, 0] += 900
    dt = "f32" if form == "f32" else "bf16"
    q, cu, k, v, L = attend_inputs(B, hq, hkv, d, dt, lens, m)
    sees = some_masks(r, m, "tree")
    got, lse = run(form, q, cu, sees, 4, k, v, L)
    check(got, lse, q, cu, widen(k), widen(v), L, padded(sees, 4), dt)


@pytest.mark.parametrize("m,hq", [([400], 64), ([700, 500], 64), ([60], 64)])
def test_many_rows_of_chains_are_joined(m, hq):
    """25600, 76800 and 3840 rows without masks, one sequence in pieces."""
    lens = [3000] + [600] * (len(m) - 1)
    q, cu, k, v, L = attend_inputs(7, hq, 2, 64, "bf16", np.maximum(lens, m), m)
    got, lse = run_paged(q, cu, k, v, L, 16)
    check_attend(got, lse, q, cu, k, v, L, "bf16")


@pytest.mark.parametrize("bits", [8, 4])
def test_shares_that_end_between_short_heads(bits):
    """800 heads of none to three groups each: every way that a share can end in front of a head's first group."""
    r = np.random.default_rng(bits)
    B, hq, hkv, d = 100, 8, 8, 64
    lens = r.integers(0, 300, B)
    lens[7] = 900
    c = Mx(bits, lens, hkv, d, 16, bits)
    m = (r.random(B) < 0.9).astype(int)
    cu = sums(m)
    q = queries(2, int(cu[-1]), hq, d)
    got, lse = run_mx_chain(c, q, cu, hq, hkv, d)
    check_attend(got, lse, q, cu, c.val[0], c.val[1], np.repeat(c.lens[:, None], hkv, 1), "bf16")


@pytest.mark.parametrize("form,d", [("paged", 64), ("paged", 128), ("mx8", 128), ("mx4", 256), ("paged", 256)])
@pytest.mark.parametrize("m", [[1, 1], [1, 4]])
def test_64_query_heads_of_one_kv_head(form, d, m):
    r = np.random.default_rng(d)
    sees, cu = some_masks(r, m, "tree"), sums(m)
    if form == "paged":
        q, cu, k, v, L = attend_inputs(3, 64, 1, d, "bf16", [700, 90], m)
        got, lse = run(form, q, cu, sees, 1, k, v, L)
        check(got, lse, q, cu, widen(k), widen(v), L, padded(sees, 1), "bf16")
        return
    c = Mx(9, [700, 90], 1, d, 16, int(form[2:]))
    q = queries(4, int(cu[-1]), 64, d)
    got, lse = run_mx(c, q, cu, sees, 1, 64, 1, d)
    check(got, lse, q, cu, c.val[0], c.val[1], c.lens[:, None], padded(sees, 1), "bf16")


# ------------------------------------------------------------------------------------------ far away, and together
@pytest.mark.parametrize("m", [6, 70])
def test_trees_and_their_rows_past_32_bits(m):
    """The sequence's blocks lie past 2^32 bytes of the pool: attention over them, and the branch's rows moved."""
    import torch
    hq, hkv, d, bs, n = 4, 2, 128, 16, 100
    nb = (1 << 32) // (hkv * bs * d * 2) + 40
    if torch.cuda.mem_get_info()[0] < 6 * nb * hkv * bs * d * 2:
        pytest.skip("not enough memory")
    q, cu, k, v, L = attend_inputs(2, hq, hkv, d, "bf16", [n], [m])
    kp, vp, table, small = make_block_pools(k, v, bs, 1)
    first = nb - small - 2
    big = []
    for x in (kp, vp):
        y = torch.zeros(nb, hkv, bs, d, dtype=torch.bfloat16, device="cuda")
        y[first:first + small] = to_dev(x)
        big.append(y)
    pg_table = i32(table + first)
    pg = ea.make_paged(pg_table, bs, nb)
    sees = some_masks(np.random.default_rng(m), [m], "tree")
    words = -(-m // 64)
    p, step = ea.make_params(1, hq, hkv, d, ea.EA_BF16), ea.make_step(i32(cu), m, m)
    out, lse = outputs(q, "bf16")
    ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda")
    ea.attend_tree_paged(p, to_dev(q), step, ea.make_tree(handle(sees, m, words)), *big, pg, i32([n]), n, out, lse, ws)
    torch.cuda.synchronize()
    check(to_host(out), lse.cpu().numpy(), q, cu, widen(k), widen(v), L, padded(sees, words), "bf16")
    path, len_out = i32([[0, 2, m - 1] + [0] * (m - 3)]), i32([0])
    ea.keep_path_paged(p, step, path, i32([3]), *big, pg, i32([n]), len_out)
    torch.cuda.synchronize()
    assert list(to_host(len_out)) == [n - m + 3]
    at = lambda row: (table[0, row // bs], slice(None), row % bs)    # noqa: E731
    for x, y in ((kp, big[0]), (vp, big[1])):
        want = x.copy()
        for j, s in enumerate((0, 2, m - 1)):
            want[at(n - m + j)] = x[at(n - m + s)]
        assert np.array_equal(to_host(y[first:first + small]).view(np.uint16), want.view(np.uint16))


def test_graphs_that_share_a_workspace():
    """Attention of trees over bf16 rows and over MX rows, and of single tokens over those, captured into a graph each with one
    workspace, replayed in turns: every replay has the bits of the call by itself."""
    import torch
    r = np.random.default_rng(3)
    hq, hkv, d = 8, 2, 128
    calls, shared = [], 0
    c8, c4 = Mx(1, [900, 70, 3100], hkv, d, 16, 8), Mx(2, [5000, 40, 800], hkv, d, 16, 4)
    for name, m in (("bf16", [100, 9, 30]), ("mx8", [20, 70, 1]), ("mx4", [1, 1, 1])):
        cu = sums(m)
        p, step = ea.make_params(3, hq, hkv, d, ea.EA_BF16), ea.make_step(i32(cu), int(cu[-1]), max(m))
        words = -(-max(m) // 64)
        tree = ea.make_tree(handle(some_masks(r, m, "tree"), int(cu[-1]), words))
        if name == "bf16":
            q, cu, k, v, L = attend_inputs(1, hq, hkv, d, "bf16", [1200, 60, 400], m)
            kd, vd, ld, cap = to_dev(k), to_dev(v), i32(L), k.shape[2]
            call = lambda q, o, l, w, a=(p, step, tree, kd, vd, ld, cap): ea.attend_tree(a[0], q, a[1], a[2], a[3], a[4], a[5], a[6], a[6], o, l, w)    # noqa: E731
            n = cap
        else:
            c = c8 if name == "mx8" else c4
            q, n = queries(5, int(cu[-1]), hq, d), c.n
            if name == "mx8":
                call = lambda q, o, l, w, a=(p, step, tree, c): ea.attend_tree_mx(a[0], q, a[1], a[2], a[3].mx, a[3].pg, a[3].ld, a[3].n, o, l, w)    # noqa: E731
            else:
                call = lambda q, o, l, w, a=(p, step, c): ea.attend_mx(a[0], q, a[1], a[2].mx, a[2].pg, a[2].ld, a[2].n, o, l, w)    # noqa: E731
        shared = max(shared, ea.attend_workspace_bytes(p, step, n))
        calls.append((call, to_dev(q), *outputs(q, "bf16")))
    ws = torch.empty(shared, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    want, graphs = [], []
    for call, q, out, lse in calls:
        call(q, out, lse, ws)
        torch.cuda.synchronize()
        want.append((out.clone(), lse.clone()))
    for call, q, out, lse in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call(q, out, lse, ws)
        graphs.append(g)
    torch.cuda.synchronize()
    for turn in range(4):
        for i in r.permutation(3):
            graphs[i].replay()
        torch.cuda.synchronize()
        for (_, _, out, lse), (o, l) in zip(calls, want):
            assert torch.equal(out, o) and torch.equal(lse, l), turn
            out.zero_()
            lse.zero_()
        ws.fill_(0x5A + turn)
        torch.cuda.synchronize()


@pytest.mark.parametrize("hq,hkv,d,m,n", [(8, 2, 128, [1, 1], 4096), (8, 8, 64, [30, 200], 900), (4, 2, 256, [256, 3], 5000), (32, 2, 128, [2, 2], 70)])
def test_no_call_writes_behind_its_workspace(hq, hkv, d, m, n):
    import torch
    cu = sums(m)
    t = int(cu[-1])
    p, step = ea.make_params(2, hq, hkv, d, ea.EA_BF16), ea.make_step(i32(cu), t, max(m))
    size = ea.attend_workspace_bytes(p, step, n)
    room = torch.full((size + 65536,), 0x3C, dtype=torch.uint8, device="cuda")
    ws = room[:size]
    q = torch.randn(t, hq, d, device="cuda").to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(t, hq, device="cuda")
    k = torch.randn(2, 2, hkv, n, d, device="cuda").to(torch.bfloat16)
    lens = i32([[n] * hkv, [n // 3 + m[1]] * hkv])
    tree = ea.make_tree(handle(some_masks(np.random.default_rng(0), m, "tree"), t, 4))
    ea.attend_tree(p, q, step, tree, k[0], k[1], lens, n, n, out, lse, ws)
    bs = 16
    nb = 2 * -(-n // bs)
    table = torch.arange(nb, dtype=torch.int32, device="cuda").view(2, -1)
    pg = ea.make_paged(table, bs, nb)
    for fmt, width in ((ea.EA_MXFP8, d), (ea.EA_MXFP4, d // 2)):
        e = [torch.randint(0, 100, (nb, hkv, bs, width), device="cuda").to(torch.uint8) for _ in range(2)]
        s = [torch.randint(120, 130, (nb, hkv, bs, d // 32), device="cuda").to(torch.uint8) for _ in range(2)]
        mx = ea.make_mx(*e, *s, fmt)
        ea.attend_mx(p, q, step, mx, pg, lens[:, 0].contiguous(), n, out, lse, ws)
        ea.attend_tree_mx(p, q, step, tree, mx, pg, lens[:, 0].contiguous(), n, out, lse, ws)
        torch.cuda.synchronize()
    assert (room[size:] == 0x3C).all()


@pytest.mark.parametrize("hq,hkv,d,m,lens", [(18, 6, 128, [12, 3, 9], [2600, 1700, 40]), (16, 4, 64, [64, 1, 33], [3000, 900, 33]), (8, 2, 256, [16, 5, 30], [4100, 5, 1999]),
                                             (4, 1, 128, [256, 60, 17], [4500, 2000, 17]), (16, 4, 256, [70, 0, 2], [2300, 7, 1])])
def test_many_rows_of_a_wavefront_over_fp32(hq, hkv, d, m, lens):
    """Trees that have more than 16 rows to a KV head, over lengths at which a wavefront takes up to 64 (d = 256: 32) of them."""
    r = np.random.default_rng(d + sum(m))
    L = np.maximum(np.array(lens)[:, None] - r.integers(0, 60, (3, hkv)), 0)
    q, cu, k, v, L = attend_inputs(d, hq, hkv, d, "f32", L, m, room=2)
    for how in ("tree", "any"):
        sees = some_masks(r, m, how)
        words = -(-max(m) // 64)
        got, lse = run("f32", q, cu, sees, words, k, v, L)
        check(got, lse, q, cu, widen(k), widen(v), L, padded(sees, words), "f32")
        assert (got[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_values_that_are_not_finite_among_many_rows_of_a_wavefront(d):
    hq, hkv, m = 8, 2, [20, 7, 30]
    r = np.random.default_rng(d)
    lens = np.array([4100, 2000, 30])
    q, cu, k, v, L = attend_inputs(d, hq, hkv, d, "f32", lens, m)
    sees = some_masks(r, m, "tree")
    clean, clean_lse = run("f32", q, cu, sees, 1, k, v, L)
    v = v.copy()
    bad = [5, 2, 17]
    for b in range(3):
        v[b, :, lens[b] - m[b] + bad[b], 3] = np.inf
    got, lse = run("f32", q, cu, sees, 1, k, v, L)
    other = np.arange(d) != 3
    assert np.array_equal(lse, clean_lse) and np.array_equal(got[:, :, other], clean[:, :, other])
    for b in range(3):
        for i in range(m[b]):
            t = cu[b] + i
            if sees[t, bad[b]]:
                assert not np.isfinite(got[t, :, 3]).any()
            else:
                assert np.array_equal(got[t, :, 3], clean[t, :, 3])


@pytest.mark.parametrize("form", ["paged", "heads", "fp8", "f32", "mx8", "mx4"])
@pytest.mark.parametrize("m", [[3, 1, 2], [40, 90, 1]])
def test_strided_queries_and_no_log_sums(form, m):
    """Queries inside wider rows give the bits of queries by themselves, and so does a call that is not asked for log-sums."""
    import torch
    hq, hkv, d = 8, 2, 128
    lens, cu = [700, 130, 300], sums(m)
    dt = "f32" if form == "f32" else "bf16"
    q, cu, k, v, L = attend_inputs(4, hq, hkv, d, dt, lens, m)
    sees, words = some_masks(np.random.default_rng(1), m, "tree"), -(-max(m) // 64)
    t, p = q.shape[0], ea.make_params(3, hq, hkv, d, kind(dt))
    tree, cud = ea.make_tree(handle(sees, t, words)), i32(cu)
    wide = torch.full((t, hq + 3, d), float("nan"), dtype=torch.float32 if dt == "f32" else torch.bfloat16, device="cuda")
    wide[:, :hq] = to_dev(q)
    if form.startswith("mx"):
        c = Mx(7, lens, hkv, d, 32, int(form[2:]))
    elif form == "paged":
        kp, vp, table, nb = make_block_pools(k, v, 16, 1)
        kd, vd, td = to_dev(kp), to_dev(vp), i32(table)
        pg = ea.make_paged(td, 16, nb)
    elif form == "fp8":
        kd, vd = (to_dev(quantize_fp8(np.nan_to_num(widen(x)))[0]) for x in (k, v))
    else:
        kd, vd = to_dev(k), to_dev(v)
    got = []
    for qd, stride, with_lse in ((to_dev(q), 0, True), (wide, (hq + 3) * d, True), (to_dev(q), 0, False)):
        step = ea.make_step(cud, t, max(m), stride)
        out, lse = outputs(q, dt)
        if not with_lse:
            lse = None
        if form.startswith("mx"):
            args = (c.mx, c.pg, c.ld, c.n)
            ws = torch.empty(ea.attend_workspace_bytes(p, step, c.n), dtype=torch.uint8, device="cuda")
            ea.attend_tree_mx(p, qd, step, tree, *args, out, lse, ws)
            plain = torch.empty_like(out)
            ea.attend_mx(p, qd, step, *args, plain, lse, ws)
            torch.cuda.synchronize()
            got.append([out, plain, lse])
            continue
        n = table.shape[1] * 16 if form == "paged" else k.shape[2]
        ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda")
        if form == "paged":
            ea.attend_tree_paged(p, qd, step, tree, kd, vd, pg, i32(lens), n, out, lse, ws)
        elif form == "fp8":
            ea.attend_tree_fp8(p, qd, step, tree, kd, vd, None, None, i32(L), n, n, out, lse, ws)
        else:
            ea.attend_tree(p, qd, step, tree, kd, vd, i32(L), n, n, out, lse, ws)
        torch.cuda.synchronize()
        got.append([out, lse])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert b is None or torch.equal(a, b)
    assert torch.isfinite(got[0][0].float()).all()


@pytest.mark.parametrize("hq,hkv,d,m,n", [(8, 2, 128, [16, 5], 9000), (8, 2, 64, [60, 3], 9000), (8, 4, 256, [9, 30], 5000), (18, 6, 128, [200, 1], 4000),
                                          (8, 2, 128, [2, 1], 700), (4, 1, 64, [256, 256], 40000)])
def test_no_call_over_fp32_writes_behind_its_workspace(hq, hkv, d, m, n):
    """Trees of more than 16 rows in tiles of 32 and 64, cut along the keys, and of few."""
    import torch
    cu = sums(m)
    t = int(cu[-1])
    p, step = ea.make_params(2, hq, hkv, d, ea.EA_F32), ea.make_step(i32(cu), t, max(m))
    size = ea.attend_workspace_bytes(p, step, n)
    room = torch.full((size + 65536,), 0x3C, dtype=torch.uint8, device="cuda")
    q = torch.randn(t, hq, d, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(t, hq, device="cuda")
    k = torch.randn(2, 2, hkv, n, d, device="cuda")
    tree = ea.make_tree(handle(some_masks(np.random.default_rng(0), m, "tree"), t, 4))
    for lens in ([n, n], [n, n // 3 + m[1]], [max(m), max(m)]):
        ea.attend_tree(p, q, step, tree, k[0], k[1], i32([[x] * hkv for x in lens]), n, n, out, lse, room[:size])
        torch.cuda.synchronize()
        assert (room[size:] == 0x3C).all() and torch.isfinite(out).all()
