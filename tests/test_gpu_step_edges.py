"""The calls of a model's step at their edges: many sequences, bounds that are loose, views, scales of either sign, lengths that make
no sense, caches past 2^32 numbers, and two captured calls on one workspace.  Bounds as in test_gpu_step.py."""
import numpy as np
import pytest

from ea_inputs import inv_freq_table, quantize_fp8, widen
from ea_inputs.torch_io import to_dev, to_host
from oracle import ea_extensions as X
import paper_2510_00636_amd as ea
from tests.test_gpu_step import HALF, attend_inputs, check_attend, check_rotated, i32, kind, outputs, run_paged, store

pytestmark = pytest.mark.gpu


def attend_heads(q, cu, k, v, lens, dt, n, cap, max_new, n_tokens=None, q_stride=0):
    """Contiguous caches; q as it is given (numpy, or a view on the device)."""
    import torch
    hq, d = q.shape[-2:]
    p = ea.make_params(k.shape[0], hq, k.shape[1], d, kind(dt))
    cud = i32(cu)
    step = ea.make_step(cud, q.shape[0] if n_tokens is None else n_tokens, max_new, q_stride)
    out, lse = outputs(q, dt)
    ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
    dev = [to_dev(x) if isinstance(x, np.ndarray) else x for x in (q, k, v)]
    ea.attend(p, dev[0], step, dev[1], dev[2], i32(lens), n, cap, out, lse, ws)
    torch.cuda.synchronize()
    return to_host(out), lse.cpu().numpy()


# ------------------------------------------------------------------------------------------ many sequences
def many(r, B):
    """Mostly single tokens, some absent, some stretches; lengths from nothing to some hundred."""
    m = np.where(r.random(B) < 0.7, 1, r.integers(0, 6, B))
    m[r.integers(0, B, 6)] = 40
    return m, r.integers(0, 500, B)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 2, 256), (6, 2, 64)])
@pytest.mark.parametrize("B", [65, 130])
def test_many_sequences_over_pools(hq, hkv, d, B):
    m, lens = many(np.random.default_rng(B + d), B)
    q, cu, k, v, L = attend_inputs(B, hq, hkv, d, "bf16", lens, m, room=1)
    got, lse = run_paged(q, cu, k, v, L, 16)
    check_attend(got, lse, q, cu, k, v, L, "bf16")
    assert (widen(got)[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("dt,hq,hkv,d", [("bf16", 8, 2, 128), ("f32", 4, 4, 64)])
@pytest.mark.parametrize("single", [True, False])
def test_many_sequences_with_a_length_per_head(dt, hq, hkv, d, single):
    r = np.random.default_rng(d)
    B = 130
    m, _ = many(r, B)
    if single:
        m[:] = 1
    lens = r.integers(0, 300, (B, hkv))
    q, cu, k, v, L = attend_inputs(3, hq, hkv, d, dt, lens, m)
    cap = k.shape[2]
    got, lse = attend_heads(q, cu, k, v, L, dt, cap, cap, int(m.max()))
    check_attend(got, lse, q, cu, k, v, L, dt)


@pytest.mark.parametrize("hq,hkv,d,B", [(8, 2, 128, 300), (4, 4, 64, 150), (16, 8, 256, 70)])
@pytest.mark.parametrize("heads", [False, True])
def test_more_heads_than_workgroups(hq, hkv, d, B, heads):
    """Short heads by the dozen to a workgroup, and some long ones over several."""
    r = np.random.default_rng(B)
    lens = r.integers(0, 60, (B, hkv if heads else 1))
    for _ in range(4):
        lens[r.integers(0, B), r.integers(0, lens.shape[1])] = r.integers(400, 1200)
    m = np.where(r.random(B) < 0.9, 1, r.integers(0, 4, B))
    q, cu, k, v, L = attend_inputs(B, hq, hkv, d, "bf16", lens if heads else lens[:, 0], m, room=1)
    if heads:
        got, lse = attend_heads(q, cu, k, v, L, "bf16", k.shape[2], k.shape[2], 3)
    else:
        got, lse = run_paged(q, cu, k, v, L, 32)
    check_attend(got, lse, q, cu, k, v, L, "bf16")
    assert (widen(got)[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("dt,hq,hkv,d,m", [("bf16", 8, 2, 64, [5, 16, 1, 9]), ("bf16", 12, 4, 128, [5, 12, 1, 21]), ("bf16", 4, 2, 256, [5, 12, 1, 16]),
                                          ("bf16", 20, 1, 256, [1, 1, 0, 1]), ("bf16", 33, 1, 128, [1, 1, 1, 1]), ("fp8", 8, 2, 128, [5, 16, 1, 9]),
                                          ("fp8", 4, 2, 256, [5, 12, 1, 16]), ("fp8", 33, 1, 128, [1, 1, 0, 1])])
def test_rows_of_all_heights(dt, hq, hkv, d, m):
    """Two and four operands of 16 rows, over heads that are cut and heads that see less than they add."""
    import torch
    r = np.random.default_rng(hq + d)
    lens = r.integers(0, 800, (4, hkv))
    lens[1, 0], lens[3, -1] = 3000, max(m[3] - 1, 0)
    q, cu, k, v, L = attend_inputs(d, hq, hkv, d, "bf16" if dt == "bf16" else "f32", lens, m, room=1)
    cap = k.shape[2]
    if dt == "bf16":
        got, lse = attend_heads(q, cu, k, v, L, "bf16", cap, cap, max(m))
    else:
        q = store(q.astype(np.float64), "bf16")
        (k8, ks), (v8, vs) = (quantize_fp8(np.nan_to_num(x.astype(np.float64))) for x in (k, v))
        p = ea.make_params(4, hq, hkv, d, ea.EA_BF16)
        cud = i32(cu)
        step, (out, lse) = ea.make_step(cud, q.shape[0], max(m)), outputs(q, "bf16")
        ws = torch.empty(ea.attend_workspace_bytes(p, step, cap), dtype=torch.uint8, device="cuda").fill_(0xFF)
        ea.attend_fp8(p, to_dev(q), step, to_dev(k8), to_dev(v8), to_dev(ks), to_dev(vs), i32(L), cap, cap, out, lse, ws)
        torch.cuda.synchronize()
        got, lse = to_host(out), lse.cpu().numpy()
        k, v = (X.fp8_e4m3_decode(x) * s.astype(np.float64)[:, :, None, None] for x, s in ((k8, ks), (v8, vs)))
    check_attend(got, lse, q, cu, k, v, L, "bf16")
    assert (widen(got)[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()


def test_fp32_prompt():
    """Enough rows for the kernel whose wavefronts lie over the rows."""
    q, cu, k, v, L = attend_inputs(5, 8, 8, 64, "f32", [1100, 1000], [1100, 948])
    got, lse = attend_heads(q, cu, k, v, L, "f32", 1100, 1100, 1100)
    check_attend(got, lse, q, cu, k, v, L, "f32")


# ------------------------------------------------------------------------------------------ bounds and lengths
@pytest.mark.parametrize("dt,d", [("bf16", 128), ("bf16", 256), ("f32", 64)])
@pytest.mark.parametrize("m", [[1, 1, 1], [3, 1, 40]])
def test_bounds_that_are_loose(dt, d, m):
    """n, max_new and n_tokens far above what there is: no other result than to rounding, and nothing written behind the tokens."""
    q, cu, k, v, L = attend_inputs(d, 8, 2, d, dt, [300, 17, 250], m, room=600, cap=20000)
    got, lse = attend_heads(q, cu, k, v, L, dt, 20000, 20000, 500)
    check_attend(got, lse, q, cu, k, v, L, dt)
    assert (widen(got)[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("m", [[1, 1, 1], [30, 1, 2]])
def test_lengths_that_make_no_sense(dt, m):
    """Below zero they are zero, above n they are n."""
    q, cu, k, v, _ = attend_inputs(7, 8, 2, 128, dt, [90, 90, 90], m, cap=90)
    given = np.array([[-5, 90], [2 ** 31 - 1, 91], [-2 ** 31, 0]])
    got, lse = attend_heads(q, cu, k, v, given, dt, 90, 90, max(m))
    check_attend(got, lse, q, cu, k, v, np.clip(given, 0, 90), dt)
    got, lse = attend_heads(q, cu, k, v, given, dt, 0, 90, max(m))
    assert (widen(got) == 0).all() and (lse == -np.inf).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("cu", [[0, 5, 40], [0, 70, 71], [30, 33, 34], [0, 2, 1]])
def test_prefix_sums_that_make_no_sense(dt, cu):
    """Sums past the tokens there are, or not ascending from zero: whatever they stand for, nothing outside is written."""
    import torch
    q, _, k, v, L = attend_inputs(9, 8, 2, 128, dt, [90, 60], [10, 10])
    guard = torch.full((200, 8, 128), 7.0, dtype=torch.bfloat16 if dt == "bf16" else torch.float32, device="cuda")
    lse = torch.full((200, 8), 7.0, device="cuda")
    p = ea.make_params(2, 8, 2, 128, kind(dt))
    cud = i32(cu)
    for max_new in (1, 20):
        step = ea.make_step(cud, 20, max_new)
        ws = torch.empty(ea.attend_workspace_bytes(p, step, 90), dtype=torch.uint8, device="cuda").fill_(0xFF)
        ea.attend(p, to_dev(q), step, to_dev(k), to_dev(v), i32(L), 90, 90, guard[100:120], lse[100:120], ws)
        torch.cuda.synchronize()
        for x in (guard, lse):
            assert bool((x[:100] == 7.0).all()) and bool((x[120:] == 7.0).all())


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 2, 256), (20, 1, 64)])
def test_a_sequence_that_adds_more_than_it_was_said_to(hq, hkv, d):
    """Its tokens may be left out; the others' are what they are."""
    q, cu, k, v, L = attend_inputs(hq, hq, hkv, d, "bf16", [300, 70, 500, 260], [1, 2, 90, 1])
    got, lse = attend_heads(q, cu, k, v, L, "bf16", k.shape[2], k.shape[2], 2)
    keep = np.r_[0:3, cu[3]:cu[4]]
    few = [0, 1, 3]
    check_attend(got[keep], lse[keep], q[keep], np.array([0, 1, 3, 4]), k[few], v[few], L[few], "bf16")


def test_more_new_rows_than_a_launch_has():
    import torch
    t, hq, hkv, d, bs = (1 << 23) + 3, 1, 1, 64, 16
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GB")
    here = np.array([0, 77, (1 << 23) - 1, 1 << 23, t - 1])
    slots = torch.full((t,), -1, dtype=torch.int64, device="cuda")
    slots[to_dev(here)] = torch.arange(5, device="cuda") * 7
    x = torch.zeros(t, 2, d, dtype=torch.bfloat16, device="cuda")
    rows = store(np.random.default_rng(1).standard_normal((5, 2, d)), "bf16")
    x[to_dev(here)] = to_dev(rows)
    pools = [torch.full((4, hkv, bs, d), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = i32([[0]])
    ea.append_paged(ea.make_params(1, hq, hkv, d, ea.EA_BF16), ea.make_new_rows(None, x[:, :1], x[:, 1:]), slots, pools[0], pools[1],
                    ea.make_paged(table, bs, 4))
    torch.cuda.synchronize()
    for i, pool in enumerate(pools):
        want = np.full((64, d), 5.0)
        want[np.arange(5) * 7] = widen(rows)[:, i]
        assert np.array_equal(widen(to_host(pool)).reshape(64, d), want)


# ------------------------------------------------------------------------------------------ joins, views, scales
@pytest.mark.parametrize("hq,hkv,d,m", [(16, 2, 64, [300, 1]), (16, 4, 128, [290, 3]), (16, 8, 256, [260, 2])])
def test_long_rows_cut_and_joined(hq, hkv, d, m):
    """More (token, head) rows than have a joining workgroup each, over heads that are cut."""
    q, cu, k, v, L = attend_inputs(hq, hq, hkv, d, "bf16", [5000, 20], m)
    got, lse = run_paged(q, cu, k, v, L, 64)
    check_attend(got, lse, q, cu, k, v, L, "bf16")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("m", [[1, 1], [2, 50]])
def test_queries_in_a_projection(dt, m):
    import torch
    q, cu, k, v, L = attend_inputs(4, 6, 2, 64, dt, [400, 130], m)
    wide = torch.full((q.shape[0], 6 + 2 * 2, 64), float("nan"), dtype=torch.bfloat16 if dt == "bf16" else torch.float32, device="cuda")
    wide[:, :6] = to_dev(q)
    cap = k.shape[2]
    got, lse = attend_heads(wide[:, :6], cu, k, v, L, dt, cap, cap, max(m), q_stride=wide.stride(0))
    check_attend(got, lse, q, cu, k, v, L, dt)


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("m", [[1, 1], [2, 80]])
def test_scales_of_either_sign(d, m):
    """A head's scale may be negative or zero: keys of zeros weigh all rows alike, values of zeros give zeros."""
    import torch
    q, cu, k, v, L = attend_inputs(6, 8, 2, d, "f32", [700, 300], m)
    q = store(q.astype(np.float64), "bf16")
    (k8, ks), (v8, vs) = (quantize_fp8(np.nan_to_num(x.astype(np.float64))) for x in (k, v))
    ks[0, 0], ks[1, 0], vs[0, 1], vs[1, 1] = -ks[0, 0], 0.0, -vs[0, 1], 0.0
    p = ea.make_params(2, 8, 2, d, ea.EA_BF16)
    cud, cap = i32(cu), k.shape[2]
    step = ea.make_step(cud, q.shape[0], max(m))
    out, lse = outputs(q, "bf16")
    ws = torch.empty(ea.attend_workspace_bytes(p, step, cap), dtype=torch.uint8, device="cuda").fill_(0xFF)
    ea.attend_fp8(p, to_dev(q), step, to_dev(k8), to_dev(v8), to_dev(ks), to_dev(vs), i32(L), cap, cap, out, lse, ws)
    torch.cuda.synchronize()
    kf, vf = (X.fp8_e4m3_decode(x) * s.astype(np.float64)[:, :, None, None] for x, s in ((k8, ks), (v8, vs)))
    check_attend(to_host(out), lse.cpu().numpy(), q, cu, kf, vf, L, "bf16")


# ------------------------------------------------------------------------------------------ past 32 bits
@pytest.fixture(scope="module")
def large():
    """Two buffers of 2^33 bf16 numbers, zeros."""
    import torch
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB")
    x = [torch.zeros(1 << 33, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    yield x
    x.clear()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("m", [1, 40])
def test_a_head_past_32_bits(large, m):
    """The second head's rows start 2^32 numbers behind the first one's: stored and read there, and what stood around them stays."""
    import torch
    hq, hkv, d, cap, n = 4, 2, 64, 1 << 26, 700
    for x in large:
        x.zero_()
    kc, vc = (x.view(1, hkv, cap, d) for x in large)
    r = np.random.default_rng(m)
    q, cu, k, v, L = attend_inputs(m, hq, hkv, d, "bf16", [n], [m])
    for dst, src in ((kc, k), (vc, v)):
        dst[:, :, :n - m] = to_dev(src[:, :, :n - m])
    x = store(r.standard_normal((m, hq + 2 * hkv, d)), "bf16")
    xd, pos, inv = to_dev(x), r.integers(0, 1 << 20, m), inv_freq_table(d, 1e4)
    p = ea.make_params(1, hq, hkv, d, ea.EA_BF16)
    rows = ea.make_new_rows(xd[:, :hq], xd[:, hq:hq + hkv], xd[:, hq + hkv:], i32(pos), to_dev(inv))
    qd = torch.empty(m, hq, d, dtype=torch.bfloat16, device="cuda")
    ea.append(p, rows, i32(cu), i32(L), kc, vc, cap, qd)
    torch.cuda.synchronize()
    xf = widen(x)
    got_k, got_v = (widen(to_host(y[0, :, n - m:n + 20].contiguous())) for y in (kc, vc))
    check_rotated(got_k[:, :m].transpose(1, 0, 2), xf[:, hq:hq + hkv], pos, inv, False, "bf16")
    assert np.array_equal(got_v[:, :m].transpose(1, 0, 2), xf[:, hq + hkv:]) and not got_k[:, m:].any() and not got_v[:, m:].any()
    got, lse = attend_heads(qd, cu, kc, vc, L, "bf16", n, cap, m)
    kh, vh = (to_host(y[:, :, :n].contiguous()) for y in (kc, vc))
    check_attend(got, lse, to_host(qd), cu, kh, vh, L, "bf16")


@pytest.mark.parametrize("m", [1, 40])
def test_blocks_past_32_bits(large, m):
    import torch
    hq, hkv, d, bs, n = 4, 2, 128, 64, 900
    nb = (1 << 33) // (hkv * bs * d)
    for x in large:
        x.zero_()
    kp, vp = (x.view(nb, hkv, bs, d) for x in large)
    q, cu, k, v, L = attend_inputs(m + 1, hq, hkv, d, "bf16", [n], [m])
    ids = np.concatenate([np.random.default_rng(m).permutation(np.arange(nb - 40, nb))[:14], [3]])
    for j, i in enumerate(ids):
        for dst, src in ((kp, k), (vp, v)):
            part = src[0, :, j * bs:(j + 1) * bs]
            dst[int(i), :, :part.shape[1]] = to_dev(np.ascontiguousarray(part))
    table = i32([ids])
    p = ea.make_params(1, hq, hkv, d, ea.EA_BF16)
    cud = i32(cu)
    step, (out, lse) = ea.make_step(cud, m, m), outputs(q, "bf16")
    ws = torch.empty(ea.attend_workspace_bytes(p, step, 15 * bs), dtype=torch.uint8, device="cuda").fill_(0xFF)
    ea.attend_paged(p, to_dev(q), step, kp, vp, ea.make_paged(table, bs, nb), i32(L[:, 0]), 15 * bs, out, lse, ws)
    torch.cuda.synchronize()
    check_attend(to_host(out), lse.cpu().numpy(), q, cu, k, v, L, "bf16")


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("f32", 64), ("fp8", 128)])
@pytest.mark.parametrize("m", [1, 24])
def test_a_length_past_32_bits(large, dt, d, m):
    """2^26 rows of one head.  Keys of zeros weigh all rows alike and only the last 1000 rows have values, so the result is their sum
    over the rows seen: sums of at most 1000 numbers and zeros, in fp32, the rest exact."""
    import torch
    n, tail, st = 1 << 26, 1000, "f32" if dt == "f32" else "bf16"
    for x in large:
        x.zero_()
    typ = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.uint8}[dt]
    kc, vc = (x.view(typ)[:n * d].view(1, 1, n, d) for x in large)
    r = np.random.default_rng(m)
    if dt == "fp8":
        values = r.integers(0x20, 0x50, (tail, d)).astype(np.uint8)
        vf = X.fp8_e4m3_decode(values)
    else:
        values = store(np.abs(r.standard_normal((tail, d))), dt)
        vf = widen(values)
    vc[0, 0, n - tail:] = to_dev(values)
    q = store(r.standard_normal((m, 2, d)), st)
    p = ea.make_params(1, 2, 1, d, kind(st))
    cud, lens = i32([0, m]), i32([[n]])
    step, (out, lse) = ea.make_step(cud, m, m), outputs(q, st)
    ws = torch.empty(ea.attend_workspace_bytes(p, step, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
    if dt == "fp8":
        ea.attend_fp8(p, to_dev(q), step, kc, vc, None, None, lens, n, n, out, lse, ws)
    else:
        ea.attend(p, to_dev(q), step, kc, vc, lens, n, n, out, lse, ws)
    torch.cuda.synchronize()
    got, lse = widen(to_host(out)), lse.cpu().numpy()
    for i in range(m):
        seen = n - (m - 1 - i)
        want = vf[:tail - (m - 1 - i)].sum(axis=0) / seen
        # weights are one, so nothing rounds but 1000 sums, three operations of the pieces' joining each, and the result
        tol = (HALF[st] + 1100 * 2.0 ** -24) * want
        assert (np.abs(got[i] - want) <= tol).all()
        assert (np.abs(lse[i] - np.log(seen)) <= 2.0 ** -22 * 20).all()


# ------------------------------------------------------------------------------------------ one workspace
def test_two_captured_calls_on_one_workspace():
    """Replayed in turns, with eager work and lengths that change in between; each replay against the eager call."""
    import torch
    hq, hkv, d, cap = 8, 2, 128, 3000
    p = ea.make_params(3, hq, hkv, d, ea.EA_BF16)
    jobs = []
    for seed, m in ((1, [1, 1, 1]), (2, [70, 1, 200])):
        q, cu, k, v, L = attend_inputs(seed, hq, hkv, d, "bf16", [2500, 900, 2999], m, cap=cap)
        k, v = np.nan_to_num(widen(k)), np.nan_to_num(widen(v))
        cud = i32(cu)
        jobs.append(dict(q=to_dev(q), cu=cud, k=to_dev(store(k, "bf16")), v=to_dev(store(v, "bf16")), lens=i32(L), out=outputs(q, "bf16"),
                         ref=outputs(q, "bf16"), st=ea.make_step(cud, q.shape[0], max(m))))
    size = max(ea.attend_workspace_bytes(p, j["st"], cap) for j in jobs)
    ws, own = (torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2))

    def go(j, to, w):
        ea.attend(p, j["q"], j["st"], j["k"], j["v"], j["lens"], cap, cap, *j[to], w)
    side = torch.cuda.Stream()
    for j in jobs:
        torch.cuda.synchronize()
        j["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(j["graph"], stream=side):
            go(j, "out", ws)
    r = np.random.default_rng(0)
    for turn in range(4):
        for j in jobs:
            j["lens"].copy_(i32(r.integers(200, cap, (3, hkv))))
            for x in j["out"]:
                x.fill_(7.0)
        torch.cuda.synchronize()
        for j in jobs if turn % 2 else jobs[::-1]:
            j["graph"].replay()
        torch.cuda.synchronize()
        for j in jobs:
            go(j, "ref", own)
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(j["out"], j["ref"]))
