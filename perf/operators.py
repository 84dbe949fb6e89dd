"""The operators of a model's step over its cache, as measurable cases: block tables and slot maps from request lengths, the
store of new rows behind their rotary embedding, and the attention of new tokens over what is cached.

A case is a dict of plain values; `form` says which operator a pass runs:

  tables        block_tables twice: the step's blocks are taken, and given back as after a compress pass
  append        append_paged: q, k, v rows cut out of one projection's rows, rotated, stored through the slot map
  append_heads  append: the same into a contiguous cache whose heads have lengths of their own
  paged         attend_paged: new tokens over block pools
  heads         attend: new tokens over a contiguous cache whose heads have lengths of their own (bf16 or fp32)
  fp8           attend_fp8: the same over e4m3 bytes

`own` false computes the operators in their plain form; true calls the library.
"""
import math
import random

import torch

own = False
DEV = "cuda"


# ------------------------------------------------------------------------------------ the cases
def _case(form, dtype="bf16", batch=1, hq=32, hkv=8, d=128, n=4096, least=0, m=1, few=0, block=16, base=5e5, inter=False,
          shape=0, name=None):
    """Sequence lengths lie between `least` (0: all are n) and n rows, new tokens included; each sequence adds m tokens, with
    few > 0 every `few`-th one m and the others up to m, most of them one.  `shape` seeds the lengths."""
    c = dict(form=form, dtype=dtype, batch=batch, hq=hq, hkv=hkv, d=d, n=n, least=least, m=m, few=few, block=block, base=base,
             inter=inter, shape=shape)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one generated token over the 4096 pairs that the periodic compress pass leaves: latency
        _case("paged", hq=40, n=4097, base=1e6, name="decode_1x4k"),
        # a server's batch of generated tokens, contexts of all lengths up to the compress pass's limit
        _case("paged", batch=48, hq=40, n=4608, least=17, block=64, shape=1, name="decode_48_ragged"),
        # four long contexts: the cache is read once per token
        _case("paged", batch=4, n=131072, block=256, name="decode_4x131k"),
        # after a pass with one budget per layer: every KV head kept another number of pairs
        _case("heads", batch=2, n=50001, least=3000, shape=2, name="decode_adaptive_50k"),
        # a long context held in 8 bits
        _case("fp8", n=131072, name="decode_fp8_131k"),
        # a mixed step at head dimension 256: a few sequences read a stretch of their prompt, the others generate
        _case("paged", batch=12, hq=16, d=256, n=8192, least=300, m=700, few=4, block=32, base=1e6, shape=3,
              name="mixed_d256_8k"),
        # 2048 tokens of a long prompt over the 32k in front of them: the largest case
        _case("paged", n=34816, m=2048, block=16, name="chunk_2k_over_32k"),
        # a small fp32 cache, 64 new tokens
        _case("heads", "f32", hq=4, hkv=2, d=64, n=1024, m=64, base=1e4, name="f32_chunk_1k"),
        # the rows of one generated token per sequence
        _case("append", batch=48, hq=40, n=4608, least=17, block=64, base=1e6, shape=1, name="append_48"),
        # the rows of a prompt's stretch, two sequences
        _case("append", batch=2, n=40000, m=4096, block=16, name="append_8k"),
        # the bookkeeping of a generated token per sequence
        _case("tables", batch=48, n=4608, least=17, shape=1, name="tables_48"),
        # and of a step that reads long prompts next to many generating sequences
        _case("tables", batch=512, n=16384, least=1, m=4000, few=32, shape=4, name="tables_512"),
    ]


def _size(rng, lo, hi):
    """log-uniform in [lo, hi], one time in three a multiple of 64"""
    x = int(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    return max(lo, x // 64 * 64) if rng.random() < 0.33 else x


def draw(rng):
    form = rng.choice(["paged", "paged", "paged", "paged", "heads", "heads", "fp8", "append", "append_heads", "tables"])
    f32 = form in ("heads", "append_heads") and rng.random() < 0.35
    hq, hkv, d = rng.choice([(32, 8, 128), (40, 8, 128), (28, 4, 128), (64, 8, 128), (16, 8, 256), (16, 2, 256), (32, 4, 64),
                             (8, 8, 128), (24, 8, 128), (4, 2, 64)])
    if form == "fp8" and d == 64:
        d = 128
    kw = dict(hq=hq, hkv=hkv, d=d, block=rng.choice([16, 16, 32, 64, 256]), base=rng.choice([1e4, 5e5, 1e6]),
              inter=rng.random() < 0.3, shape=rng.randrange(1 << 30))
    batch = rng.choice([1, 1, 2, 4, 8, 16, 48, 100])
    n = _size(rng, 64, 131072)
    m = rng.choice([1, 1, 1, 2, 5, _size(rng, 8, 300), _size(rng, 64, 4096)])
    few = rng.choice([0, 0, 3, 7])
    if form == "tables":
        batch = _size(rng, 1, 1000)
        return _case(form, batch=batch, n=_size(rng, 16, 32768), least=1, m=max(1, min(m, 65536 // batch)), few=few, **kw)
    if form.startswith("append"):
        batch, n = min(batch, 48), min(n, 8192)
        m = max(1, min(m, n, 16384 // batch))
        return _case(form, "f32" if f32 else "bf16", batch=batch, n=n, least=m if rng.random() < 0.5 else 0, m=m, few=few, **kw)
    # no more bytes and products than the largest listed cases have
    row = hkv * d * 2 * (4 if f32 else 2)
    n = max(16, min(n, int(1.5e9 / (row * batch))))
    m = max(1, min(m, n, int(6e11 / (batch * 4 * hq * d * n)) if not f32 else int(2e10 / (batch * 4 * hq * d * n))))
    if few == 0 and batch * m > 8192:
        m = 8192 // batch
    return _case(form, "f32" if f32 else "bf16", batch=batch, n=n, least=rng.choice([0, 1, max(1, n // 20)]), m=m, few=few, **kw)


def _lengths(c):
    """Per sequence (old rows, new tokens), and per KV head the rows with the new ones in."""
    r = random.Random(c["shape"])
    add, rows, heads = [], [], []
    for b in range(c["batch"]):
        a = c["m"]
        if c["few"] and b % c["few"]:
            a = 1 if r.random() < 0.7 else r.randint(1, c["m"])

        def one():
            if not c["least"]:
                return max(c["n"], a)
            lo = max(c["least"], 1)
            return max(a, int(round(math.exp(r.uniform(math.log(lo), math.log(max(c["n"], lo)))))))
        rows.append(one())
        heads.append([one() for _ in range(c["hkv"])] if "heads" in c["form"] else [rows[-1]] * c["hkv"])
        add.append(a)
    return add, rows, heads


def _capacity(c, heads):
    return max(max(h) for h in heads) + 37


def work(c):
    add, rows, heads = _lengths(c)
    t, e = sum(add), {"bf16": 2, "f32": 4}[c["dtype"]]
    if c["form"] == "tables":
        took = sum(-(-r // c["block"]) - -(-(r - a) // c["block"]) for r, a in zip(rows, add))
        # lengths in and out, the prefix sums, taken entries read and written and put back, a slot and a position per token
        return {"bytes": 2 * (16 * c["batch"] + 4 * c["batch"]) + 16 * took + 12 * t, "flops": 0}
    if c["form"].startswith("append"):
        per = (2 * c["hq"] + 4 * c["hkv"]) * c["d"] * e
        return {"bytes": t * (per + (12 if c["form"] == "append" else 4)), "flops": 3 * t * (c["hq"] + c["hkv"]) * c["d"]}
    pairs = sum(sum(max(0, n - a + 1 + i) for i in range(a)) for h, a in zip(heads, add) for n in h)
    cached = sum(map(sum, heads)) * 2 * c["d"] * (1 if c["form"] == "fp8" else e)
    return {"bytes": cached + t * c["hq"] * (2 * c["d"] * e + 4), "flops": 4 * c["d"] * (c["hq"] // c["hkv"]) * pairs}


# ----------------------------------------------------------------------------------- the inputs
def _rows(gen, c, heads, shape, scale=1.0):
    """Rows [.., heads, .., d] with per-channel means and scales of each head and four strong channels, as keys and queries
    have them: heads stand at dimension 1."""
    s = torch.exp(0.5 * torch.randn(heads, c["d"], generator=gen, device=DEV))
    m = math.sqrt(2.0) * torch.randn(heads, c["d"], generator=gen, device=DEV)
    if c["dtype"] == "bf16":
        m[:, :: c["d"] // 4] += 8.0
    view = [1] * len(shape)
    view[1], view[-1] = heads, c["d"]
    return torch.randn(shape, generator=gen, device=DEV).mul_(s.view(view)).add_(m.view(view)).mul_(scale)


def prepare(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    add, rows, heads = _lengths(c)
    t, dt = sum(add), {"bf16": torch.bfloat16, "f32": torch.float32}[c["dtype"]]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)    # noqa: E731
    st = dict(c, seed=seed, n_tokens=t, max_new=max(add), cu=i32([sum(add[:b]) for b in range(len(add) + 1)]))
    B, hq, hkv, d, bs = c["batch"], c["hq"], c["hkv"], c["d"], c["block"]
    seq = torch.repeat_interleave(torch.arange(B, device=DEV), torch.tensor(add, device=DEV), output_size=t)
    st["seq"], st["nth"] = seq, torch.arange(t, device=DEV) - st["cu"][seq]
    pages = [-(-r // bs) for r in rows]
    st["max_blocks"] = max(pages) + 1
    # tokens seen so far: the cache has been cut back now and then, rows are no positions
    seen = torch.tensor(rows, device=DEV) + torch.randint(0, 100000, (B,), generator=gen, device=DEV)
    st["seen"] = seen.to(torch.int32)
    if c["form"] == "tables":
        st["num_blocks"] = sum(pages) + 1 + c["shape"] * 37 % 1000
        order = torch.randperm(st["num_blocks"], generator=gen, device=DEV).to(torch.int32)
        held = [-(-(r - a) // bs) for r, a in zip(rows, add)]
        table, at = torch.full((B, st["max_blocks"]), -1, dtype=torch.int32, device=DEV), 0
        for b, k in enumerate(held):
            table[b, :k] = order[at:at + k]
            at += k
        free = torch.full((st["num_blocks"],), -1, dtype=torch.int32, device=DEV)
        free[: st["num_blocks"] - at] = order[at:]
        st.update(table=table, free=free, count=i32([st["num_blocks"] - at]), len_old=i32([r - a for r, a in zip(rows, add)]),
                  len_new=i32(rows), len_mid=torch.zeros(B, dtype=torch.int32, device=DEV),
                  len_end=torch.zeros(B, dtype=torch.int32, device=DEV), count_mid=i32([0]), count_end=i32([0]),
                  cu_mid=torch.zeros(B + 1, dtype=torch.int32, device=DEV), cu_end=torch.zeros(B + 1, dtype=torch.int32, device=DEV),
                  slots=torch.zeros(t, dtype=torch.int64, device=DEV), pos=torch.zeros(t, dtype=torch.int32, device=DEV))
        return st
    paged = c["form"] in ("append", "paged")
    if paged:
        st["num_blocks"] = sum(pages) + 3
        order = torch.randperm(st["num_blocks"], generator=gen, device=DEV).to(torch.int32)
        table, at = torch.zeros((B, st["max_blocks"]), dtype=torch.int32, device=DEV), 0
        for b, k in enumerate(pages):
            table[b, :k] = order[at:at + k]
            at += k
        st.update(table=table, lens=i32(rows))
        shape = (st["num_blocks"], hkv, bs, d)
    else:
        st.update(cap=_capacity(c, heads), lens=i32(heads))
        shape = (B, hkv, st["cap"], d)
    if c["form"].startswith("append"):
        # one projection's rows: q, k and v of a token side by side
        qkv = torch.cat([_rows(gen, c, hq, (t, hq, d)).flatten(1), _rows(gen, c, hkv, (t, hkv, d)).flatten(1),
                         torch.randn(t, hkv * d, generator=gen, device=DEV)], dim=1).to(dt)
        st.update(qkv=qkv, pos=(seen[seq] + st["nth"]).to(torch.int32), q_out=torch.zeros(t, hq, d, dtype=dt, device=DEV),
                  inv_freq=torch.pow(torch.tensor(c["base"], dtype=torch.float64, device=DEV),
                                     -2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d),
                  k=torch.zeros(shape, dtype=dt, device=DEV), v=torch.zeros(shape, dtype=dt, device=DEV))
        if paged:
            row = (st["lens"][seq] - (st["cu"][seq + 1] - st["cu"][seq]) + st["nth"]).long()
            st["slots"] = st["table"][seq, row // bs].long() * bs + row % bs
        return st
    k, v = _rows(gen, c, hkv, shape), torch.randn(shape, generator=gen, device=DEV)
    v.mul_(torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=gen, device=DEV)))
    if c["form"] == "fp8":
        st["k_scale"], st["v_scale"] = (x.abs().amax(dim=(2, 3)) / 400.0 for x in (k, v))
        k, v = ((x / s[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8) for x, s in ((k, st["k_scale"]), (v, st["v_scale"])))
    else:
        k, v = k.to(dt), v.to(dt)
    st.update(k=k, v=v, q=_rows(gen, c, hq, (t, hq, d), 0.5).to(dt), out=torch.zeros(t, hq, d, dtype=dt, device=DEV),
              lse=torch.zeros(t, hq, dtype=torch.float32, device=DEV))
    return st


# -------------------------------------------------------------------------------- the plain forms
def _plain_tables(st, old, new, slots):
    """One call: the table and the list change in place; returns lengths, count, prefix sums (and slots, positions)."""
    B, bs, mb = st["batch"], st["block"], st["max_blocks"]
    count = st["count"] if slots else st["count_mid"]
    held, need = (old.long() + bs - 1) // bs, (new.long() + bs - 1) // bs
    back = (held - need).clamp(min=0)
    want = (need - held).clamp(min=0) * (need <= mb)
    there = count.long() + back.sum()
    served = ((want.cumsum(0) <= there) | (want == 0)) & (need <= mb)
    take = want * served
    j = torch.arange(mb, device=DEV)[None]
    given = ((j >= need[:, None]) & (j < held[:, None])).flatten()
    taken = ((j >= held[:, None]) & (j < (held + take)[:, None])).flatten()
    flat = st["table"].view(-1)
    # what is returned stands on the list's end, the first one on top, and the takes come off the top
    nth_back, nth_take = given.long().cumsum(0) - 1, taken.long().cumsum(0) - 1
    top = count.long() + back.sum() - 1
    # returned blocks are put where they belong before the takes are read: places behind the list's old end only
    last = st["free"].numel() - 1
    where = torch.where(given, top - nth_back, last + 1).clamp(max=last + 1)
    grown = torch.cat([st["free"], st["free"][:1]]).scatter(0, where, flat)
    flat.copy_(torch.where(taken, grown[(top - nth_take).clamp(0, last)], flat))
    count_out = (count.long() + back.sum() - take.sum()).to(torch.int32)
    at = torch.arange(last + 1, device=DEV)
    st["free"].copy_(torch.where((at >= count.long()) & (at < count_out.long()), grown[:-1], st["free"]))
    len_out = torch.where(served, new, old)
    more = (new - old).clamp(min=0).long()
    cu = torch.cat([more.new_zeros(1), more.cumsum(0)])
    if not slots:
        return len_out, count_out, cu.to(torch.int32)
    t = torch.arange(st["n_tokens"], device=DEV)
    b = torch.searchsorted(cu[1:], t, right=True).clamp(max=B - 1)
    i = t - cu[b]
    row = old[b].long() + i
    slot = st["table"][b, (row // bs).clamp(max=mb - 1)].long() * bs + row % bs
    return (len_out, count_out, cu.to(torch.int32), torch.where(served[b] & (t < cu[-1]), slot, -1),
            (st["seen"][b].long() + i).to(torch.int32))


def _rotated(st, x):
    """rotary embedding of x [tokens, heads, d], angles in 64 bits"""
    ang = st["pos"].double()[:, None] * st["inv_freq"][None]
    co, si = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    x = x.float()
    if st["inter"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * co - b * si, a * si + b * co], dim=-1).flatten(-2)
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * co - b * si, a * si + b * co], dim=-1)


def _split(st):
    hq, hkv, d = st["hq"], st["hkv"], st["d"]
    q, k, v = st["qkv"].split([hq * d, hkv * d, hkv * d], dim=1)
    return q.unflatten(1, (hq, d)), k.unflatten(1, (hkv, d)), v.unflatten(1, (hkv, d))


def _plain_append(st):
    q, k, v = _split(st)
    dt = st["qkv"].dtype
    q, k = _rotated(st, q).to(dt), _rotated(st, k).to(dt)
    if st["form"] == "append":
        blk, row = st["slots"] // st["block"], st["slots"] % st["block"]
        st["k"][blk, :, row], st["v"][blk, :, row] = k, v
    else:
        seq, hkv = st["seq"], st["hkv"]
        more = (st["cu"][1:] - st["cu"][:-1])[seq]
        row = (st["lens"][seq] - (more - st["nth"])[:, None]).long()
        h = torch.arange(hkv, device=DEV)[None]
        st["k"][seq[:, None], h, row], st["v"][seq[:, None], h, row] = k, v
    return q, st["k"], st["v"]


def _plain_attend(st):
    B, hq, hkv, d, seq, nth = (st[x] for x in ("batch", "hq", "hkv", "d", "seq", "nth"))
    g, m = hq // hkv, st["max_new"]
    if st["form"] == "paged":
        n = st["max_blocks"] * st["block"]
        k, v = (st[x][st["table"].long()].float().transpose(1, 2).reshape(B, hkv, n, d) for x in "kv")
        lens = st["lens"][:, None].expand(B, hkv)
    else:
        n, lens = st["cap"], st["lens"]
        k, v = st["k"], st["v"]
        if st["form"] == "fp8":
            k, v = (x.view(torch.float8_e4m3fn).float() * st[s][:, :, None, None] for x, s in ((k, "k_scale"), (v, "v_scale")))
        k, v = k.float(), v.float()
    # queries of a sequence and KV head together, short sequences padded
    q = torch.zeros(B, m, hq, d, device=DEV)
    q[seq, nth] = st["q"].float()
    q = q.view(B, m, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, m * g, d)
    s = (q @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(B, hkv, m, g, n)
    more = (st["cu"][1:] - st["cu"][:-1]).long()
    sees = lens.long()[:, :, None] - more[:, None, None] + 1 + torch.arange(m, device=DEV)
    hidden = torch.arange(n, device=DEV) >= sees[..., None]
    s.masked_fill_(hidden[:, :, :, None], -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = s.sub_(top).exp_()
    z = w.sum(dim=-1, keepdim=True)
    # rows that no query of the sequence sees count for nothing, whatever they hold
    v = torch.where((torch.arange(n, device=DEV) >= lens[:, :, None])[..., None], 0.0, v)
    o = (w.view(B, hkv, m * g, n) @ v).view(B, hkv, m, g, d)
    o = torch.where(z > 0, o / z, 0.0)
    lse = (top + torch.log(z)).squeeze(-1)
    back = lambda x: x.movedim(1, 2)[seq, nth].flatten(1, 2)    # noqa: E731
    return back(o).to(st["q"].dtype), back(lse)


# ------------------------------------------------------------------------------------- one pass
def _kept(st):
    """What a program keeps between its steps: the parameters, the pool's description, a workspace."""
    import paper_2510_00636_amd as ea
    if "p" not in st:
        st["ea"] = ea
        st["p"] = ea.make_params(st["batch"], st["hq"], st["hkv"], st["d"], ea.EA_F32 if st["dtype"] == "f32" else ea.EA_BF16,
                                 rope_layout=int(st["inter"]))
        if "table" in st:
            st["pg"] = ea.make_paged(st["table"], st["block"], st["num_blocks"])
        if "qkv" in st:
            st["new"] = ea.make_new_rows(*_split(st), pos=st["pos"], inv_freq=st["inv_freq"])
        if "q" in st:
            st["step"] = ea.make_step(st["cu"], st["n_tokens"], st["max_new"])
            st["most"] = st["max_blocks"] * st["block"] if st["form"] == "paged" else st["cap"]
            st["ws"] = torch.empty(ea.attend_workspace_bytes(st["p"], st["step"], st["most"]), dtype=torch.uint8, device=DEV)
    return st["ea"]


def run(st):
    form = st["form"]
    if form == "tables":
        if own:
            ea = _kept(st)
            ea.block_tables(st["p"], st["pg"], st["len_old"], st["len_new"], st["free"], st["count"], st["len_mid"], st["count_mid"],
                            st["cu_mid"], st["n_tokens"], st["slots"], st["pos"], st["seen"])
            ea.block_tables(st["p"], st["pg"], st["len_mid"], st["len_old"], st["free"], st["count_mid"], st["len_end"],
                            st["count_end"], st["cu_end"])
        else:
            st["len_mid"], st["count_mid"], st["cu_mid"], st["slots"], st["pos"] = \
                _plain_tables(st, st["len_old"], st["len_new"], True)
            st["len_end"], st["count_end"], st["cu_end"] = _plain_tables(st, st["len_mid"], st["len_old"], False)
        return {x: st[x] for x in ("table", "free", "len_mid", "count_mid", "cu_mid", "slots", "pos", "len_end", "count_end", "cu_end")}
    if form.startswith("append"):
        if own:
            ea = _kept(st)
            if form == "append":
                ea.append_paged(st["p"], st["new"], st["slots"], st["k"], st["v"], st["pg"], st["q_out"])
            else:
                ea.append(st["p"], st["new"], st["cu"], st["lens"], st["k"], st["v"], st["cap"], st["q_out"])
            return {"q": st["q_out"], "k": st["k"], "v": st["v"]}
        return dict(zip("qkv", _plain_append(st)))
    if own:
        ea = _kept(st)
        if form == "paged":
            ea.attend_paged(st["p"], st["q"], st["step"], st["k"], st["v"], st["pg"], st["lens"], st["most"], st["out"], st["lse"], st["ws"])
        elif form == "heads":
            ea.attend(st["p"], st["q"], st["step"], st["k"], st["v"], st["lens"], st["most"], st["cap"], st["out"], st["lse"], st["ws"])
        else:
            ea.attend_fp8(st["p"], st["q"], st["step"], st["k"], st["v"], st["k_scale"], st["v_scale"], st["lens"], st["most"],
                          st["cap"], st["out"], st["lse"], st["ws"])
        return {"out": st["out"], "lse": st["lse"]}
    out, lse = _plain_attend(st)
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------------------ in 64 bits, apart
def exact(c, seed):
    """From the definitions, a sequence (and a head) after the other."""
    if c["form"] == "tables":
        return None
    st = prepare(c, seed)
    d, hq, hkv, g = c["d"], c["hq"], c["hkv"], c["hq"] // c["hkv"]
    add, rows, heads = _lengths(c)
    first = [sum(add[:b]) for b in range(len(add))]
    if c["form"].startswith("append"):
        qkv = st["qkv"].double().view(-1, hq + 2 * hkv, d)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        ang = torch.outer(st["pos"].double(), st["inv_freq"])
        turn = torch.complex(torch.cos(ang), torch.sin(ang))[:, None]

        def turned(x):
            if c["inter"]:
                return torch.view_as_real(torch.view_as_complex(x.reshape(*x.shape[:-1], d // 2, 2).contiguous()) * turn).reshape(x.shape)
            z = torch.complex(x[..., : d // 2], x[..., d // 2:]) * turn
            return torch.cat([z.real, z.imag], dim=-1)
        kd, vd = torch.zeros_like(st["k"], dtype=torch.float64), torch.zeros_like(st["v"], dtype=torch.float64)
        tk = turned(k)
        if c["form"] == "append":
            at_block = torch.div(st["slots"], c["block"], rounding_mode="floor")
            kd[at_block, :, st["slots"] - at_block * c["block"]] = tk
            vd[at_block, :, st["slots"] - at_block * c["block"]] = v
        else:
            for b, (f, a) in enumerate(zip(first, add)):
                for h in range(hkv):
                    end = heads[b][h]
                    kd[b, h, end - a:end], vd[b, h, end - a:end] = tk[f:f + a, h], v[f:f + a, h]
        return {"q": turned(q), "k": kd, "v": vd}
    if work(c)["flops"] > 3e12:
        return None
    out = torch.zeros(st["n_tokens"], hq, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st["n_tokens"], hq, dtype=torch.float64, device=DEV)
    for b, (f, a) in enumerate(zip(first, add)):
        for h in range(hkv):
            n = heads[b][h]
            if c["form"] == "paged":
                ids = st["table"][b, : -(-n // c["block"])].long()
                k, v = (st[x][ids, h].reshape(-1, d)[:n].double() for x in "kv")
            else:
                k, v = (st[x][b, h, :n] for x in "kv")
                if c["form"] == "fp8":
                    k, v = (x.view(torch.float8_e4m3fn).double() * st[s][b, h].double() for x, s in ((k, "k_scale"), (v, "v_scale")))
                k, v = k.double(), v.double()
            i = torch.arange(a, device=DEV)
            seen = torch.arange(n, device=DEV)[None] < (n - a + 1 + i)[:, None]
            for gg in range(g):
                s = st["q"][f:f + a, h * g + gg].double() @ k.T.contiguous() / math.sqrt(d)
                s = torch.where(seen, s, -math.inf)
                z = torch.logsumexp(s, dim=1)
                lse[f:f + a, h * g + gg] = z
                out[f:f + a, h * g + gg] = torch.exp(s - z[:, None]) @ v
    return {"out": out, "lse": lse}
