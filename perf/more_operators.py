"""The operators of a drafting server's step over pools of quantised rows, as measurable cases: rows quantised as they are written
and read back, attention over them, attention of drafted trees, and what a step does with its tree besides.

A case is a dict of plain values; `form` says which operator a pass runs, `cache` over what:

  store    append_mx: q, k, v rows cut out of one projection's rows, rotated, quantised, stored through the slot map (cache mx8)
  fill     append_mx and read_mx: whole prompts quantised and read back as bf16 tensors, which the compress pass takes
  read     read_mx: sequences of pools read back as bf16 tensors
  attend   attend_mx: new tokens, one behind the other, over MX pools
  tree     attend_tree_paged, attend_tree_mx, attend_tree: new tokens that form a tree, over pools or per-head tensors
  verify   tree_masks, tree_accept and keep_path*: masks and positions, the accepted branch, and its rows moved together

  cache    mx8, mx4: pools of e4m3 / e2m1 elements, one power of two for 32 channels; bf16: pools;
           heads, f32: contiguous bf16 / fp32 tensors whose heads have lengths of their own

`own` false computes the operators in their plain form; true calls the library.
"""
import math
import random

import torch

own = False
DEV = "cuda"


# ------------------------------------------------------------------------------------ the cases
def _case(form, cache="mx8", batch=1, hq=32, hkv=8, d=128, n=4096, least=0, m=1, few=0, block=16, base=5e5, inter=False,
          shape=0, name=None):
    """Sequence lengths lie between `least` (0: all are n) and n rows, new tokens included; each sequence adds m tokens, with
    few > 0 every `few`-th one m and the others up to m, most of them one.  `shape` seeds the lengths and the trees."""
    c = dict(form=form, cache=cache, batch=batch, hq=hq, hkv=hkv, d=d, n=n, least=least, m=m, few=few, block=block, base=base,
             inter=inter, shape=shape)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a server's batch of generated tokens, a row each: latency
        _case("store", batch=48, hq=40, n=4608, least=17, block=64, base=1e6, shape=1, name="store_48"),
        # stretches of odd lengths at head dimension 256, interleaved pairs
        _case("store", batch=5, hq=16, d=256, n=9000, least=1500, m=1111, block=32, base=1e6, inter=True, shape=2, name="store_5k_d256"),
        # two prompts in 4 bits, then read back for a compress pass
        _case("fill", "mx4", batch=2, n=4099, m=4099, name="fill_mx4_8k"),
        # a long context read back for a compress pass
        _case("read", "mx8", n=131072, block=256, name="read_mx8_131k"),
        # a batch of generated tokens, contexts of all lengths up to the compress pass's limit
        _case("attend", "mx8", batch=48, hq=40, n=4608, least=17, block=64, shape=1, name="decode_mx8_48_ragged"),
        # four long contexts in 4 bits: the cache is read once per token
        _case("attend", "mx4", batch=4, n=131072, block=256, name="decode_mx4_4x131k"),
        # 2048 tokens of a long prompt over the 32k in front of them: the largest case
        _case("attend", "mx8", n=34816, m=2048, block=16, name="chunk_mx8_2k_over_32k"),
        # one drafted tree over the 4096 pairs that the periodic compress pass leaves: latency
        _case("tree", "bf16", hq=40, n=4112, m=16, base=1e6, shape=5, name="tree_16_over_4k"),
        # a server's batch of trees over 8-bit contexts of all lengths
        _case("tree", "mx8", batch=24, n=8192, least=300, m=32, block=64, shape=6, name="tree_mx8_24x32"),
        # larger trees after a pass with one budget per layer: every KV head kept another number of pairs
        _case("tree", "heads", batch=2, n=50000, least=6000, m=127, shape=7, name="tree_heads_127"),
        # one tree's bookkeeping
        _case("verify", "bf16", n=700, m=16, shape=8, name="verify_1"),
        # and that of a batch, 8-bit pools
        _case("verify", "mx8", batch=48, n=1500, least=100, m=61, block=32, shape=9, name="verify_48"),
    ]


def _size(rng, lo, hi):
    """log-uniform in [lo, hi], one time in three a multiple of 64"""
    x = int(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    return max(lo, x // 64 * 64) if rng.random() < 0.33 else x


def draw(rng):
    form = rng.choice(["store", "fill", "read", "attend", "attend", "attend", "tree", "tree", "tree", "verify"])
    cache = {"store": ["mx8"], "fill": ["mx8", "mx4"], "read": ["mx8", "mx4"], "attend": ["mx8", "mx8", "mx4"],
             "tree": ["bf16", "bf16", "mx8", "mx4", "heads", "f32"], "verify": ["bf16", "mx8", "heads", "f32"]}[form]
    cache = rng.choice(cache)
    hq, hkv, d = rng.choice([(32, 8, 128), (40, 8, 128), (28, 4, 128), (64, 8, 128), (16, 8, 256), (16, 2, 256), (32, 4, 64),
                             (8, 8, 128), (18, 6, 128), (4, 2, 64)])
    kw = dict(hq=hq, hkv=hkv, d=d, block=rng.choice([16, 16, 32, 64, 256]), base=rng.choice([1e4, 5e5, 1e6]),
              inter=rng.random() < 0.3, shape=rng.randrange(1 << 30))
    batch = rng.choice([1, 1, 2, 4, 8, 16, 48, 100])
    few = rng.choice([0, 0, 3, 7])
    if form == "store":
        n, batch = _size(rng, 64, 8192), min(batch, 48)
        m = max(1, min(rng.choice([1, 1, 2, 5, _size(rng, 8, 4096)]), n, 8192 // batch))
        return _case(form, cache, batch=batch, n=n, least=m if rng.random() < 0.5 else 0, m=m, few=few, **kw)
    if form == "fill":
        batch = min(batch, 8)
        n = _size(rng, 1, 8192 // batch)
        return _case(form, cache, batch=batch, n=n, m=n, **kw)
    if form == "read":
        n = _size(rng, 16, 131072 // batch)
        return _case(form, cache, batch=batch, n=n, least=rng.choice([0, 1, max(1, n // 20)]), **kw)
    if form == "verify":
        batch = min(batch, 48)
        m = _size(rng, 2, 200)
        n = m + _size(rng, 1, max(2, 100000 // batch // 8))
        return _case(form, cache, batch=batch, n=n, least=rng.choice([0, m]), m=m, few=few, **kw)
    n = _size(rng, 64, 131072)
    n = max(16, min(n, int(4e9 / (hkv * d * 8 * batch))))      # no more cached numbers than the largest listed case
    if form == "tree":
        m = min(n, rng.choice([2, 4, 8, 16, _size(rng, 2, 64), _size(rng, 17, 200)]))
        # nor more products than its share: fp32 ones are dear
        batch = max(1, min(batch, int((2e10 if cache == "f32" else 2e11) / (4 * hq * d * n * m))))
        return _case(form, cache, batch=batch, n=n, least=rng.choice([0, m, max(m, n // 20)]), m=m, few=few, **kw)
    m = rng.choice([1, 1, 1, 2, 5, _size(rng, 8, 300), _size(rng, 64, 4096)])
    m = max(1, min(m, n, int(6e11 / (batch * 4 * hq * d * n))))
    if few == 0 and batch * m > 8192:
        m = 8192 // batch
    return _case(form, cache, batch=batch, n=n, least=rng.choice([0, 1, max(1, n // 20)]), m=m, few=few, **kw)


def _per_head(c):
    return c["cache"] in ("heads", "f32")


def _lengths(c):
    """Per sequence the tokens that it adds and its rows, and per KV head the rows, the new ones among them."""
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
        heads.append([one() for _ in range(c["hkv"])] if _per_head(c) else [rows[-1]] * c["hkv"])
        add.append(a)
    return add, rows, heads


def _trees(c, add):
    """Per sequence the parents of its drafted tokens (the first is the last token that was accepted; the others hang under one of
    the few in front of them), and the branch that the model will confirm."""
    r = random.Random(c["shape"] + 1)
    parents, branches = [], []
    for a in add:
        p = [-1] + [r.randint(max(0, i - 6), i - 1) for i in range(1, a)]
        branch = [0]
        while r.random() < 0.75:
            below = [i for i in range(a) if p[i] == branch[-1]]
            if not below:
                break
            branch.append(r.choice(below))
        parents.append(p)
        branches.append(branch)
    return parents, branches


def _row_bytes(c):
    """of a cached row"""
    d = c["d"]
    return {"mx8": d + d // 32, "mx4": d // 2 + d // 32, "bf16": 2 * d, "heads": 2 * d, "f32": 4 * d}[c["cache"]]


def work(c):
    add, rows, heads = _lengths(c)
    t, e, d, hq, hkv = sum(add), 4 if c["cache"] == "f32" else 2, c["d"], c["hq"], c["hkv"]
    words = -(-max(add) // 64)
    if c["form"] in ("store", "fill"):
        per = (2 * hq + 2 * hkv) * d * 2 + 2 * hkv * _row_bytes(c) + 12
        if c["form"] == "fill":
            per += 2 * hkv * (_row_bytes(c) + 2 * d)
        return {"bytes": t * per, "flops": 3 * t * (hq + hkv) * d}
    if c["form"] == "read":
        return {"bytes": sum(rows) * 2 * hkv * (_row_bytes(c) + 2 * d), "flops": 0}
    if c["form"] == "verify":
        moved = sum(sum(x != i for i, x in enumerate(p)) for p in _trees(c, add)[1])
        return {"bytes": t * (12 + 8 * words + 4) + 8 * len(add) + moved * 4 * hkv * _row_bytes(c), "flops": 0}
    io = t * hq * (2 * d * e + 4)
    cached = sum(map(sum, heads)) * 2 * _row_bytes(c)
    if c["form"] == "attend":
        pairs = sum(sum(max(0, n - a + 1 + i) for i in range(a)) for h, a in zip(heads, add) for n in h)
        return {"bytes": cached + io, "flops": 4 * d * (hq // hkv) * pairs}
    pairs = 0
    for p, h, a in zip(_trees(c, add)[0], heads, add):
        depth = []
        for x in p:
            depth.append(1 if x < 0 else depth[x] + 1)
        pairs += sum((n - a) * a + sum(depth) for n in h)
    return {"bytes": cached + io + 8 * words * t, "flops": 4 * d * (hq // hkv) * pairs}


# ----------------------------------------------------------------------------------- the inputs
def _rows(gen, c, heads, shape, scale=1.0):
    """Rows [.., heads, .., d] with per-channel means and scales of each head and four strong channels, as keys and queries
    have them: heads stand at dimension 1."""
    s = torch.exp(0.5 * torch.randn(heads, c["d"], generator=gen, device=DEV))
    m = math.sqrt(2.0) * torch.randn(heads, c["d"], generator=gen, device=DEV)
    if c["cache"] != "f32":
        m[:, :: c["d"] // 4] += 8.0
    view = [1] * len(shape)
    view[1], view[-1] = heads, c["d"]
    return torch.randn(shape, generator=gen, device=DEV).mul_(s.view(view)).add_(m.view(view)).mul_(scale)


def _scaled(x, bits):
    """Of rows [.., d]: their 32-channel groups divided by the group's power of two, and its exponent: the least one, from -117 on,
    that leaves no element above the format's largest number (448, or 6)."""
    g = x.unflatten(-1, (x.shape[-1] // 32, 32))
    top = g.abs().amax(dim=-1)
    f, e = torch.frexp(top)
    e = e - 9 + (f > 0.875) if bits == 8 else e - 3 + (f > 0.75)
    e = torch.where(top == 0, -117, e).clamp(min=-117).to(torch.int32)
    return torch.ldexp(g, -e[..., None]).flatten(-2), e


def _quantised(x, bits):
    """rows [.., d] -> bytes [.., d * bits / 8], scale bytes [.., d / 32]"""
    z, e = _scaled(x, bits)
    scale = (e + 127).to(torch.uint8)
    if bits == 8:
        return z.float().to(torch.float8_e4m3fn).view(torch.uint8), scale
    # 0, 1/2, 1, 3/2, 2, 3, 4, 6, halves to the even code
    a = z.abs()
    code = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, torch.round(a) + 2, torch.round(a / 2) + 4))
    code = code.to(torch.uint8) + 8 * (z < 0).to(torch.uint8)
    return code[..., 0::2] + 16 * code[..., 1::2], scale


def _values(b, scale, bits):
    """the numbers that bytes and scale bytes stand for, in 32 bits"""
    if bits == 8:
        x = b.view(torch.float8_e4m3fn).float()
    else:
        code = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
        x = code[torch.stack([b & 15, b >> 4], dim=-1).flatten(-2).int()]
    return torch.ldexp(x.unflatten(-1, (-1, 32)), scale[..., None].int() - 127).flatten(-2)


def _bits(c):
    return {"mx8": 8, "mx4": 4}.get(c["cache"], 0)


def prepare(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    add, rows, heads = _lengths(c)
    t, dt, bits = sum(add), torch.float32 if c["cache"] == "f32" else torch.bfloat16, _bits(c)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)    # noqa: E731
    st = dict(c, seed=seed, n_tokens=t, max_new=max(add), cu=i32([sum(add[:b]) for b in range(len(add) + 1)]))
    B, hq, hkv, d, bs = c["batch"], c["hq"], c["hkv"], c["d"], c["block"]
    seq = torch.repeat_interleave(torch.arange(B, device=DEV), torch.tensor(add, device=DEV), output_size=t)
    st["seq"], st["nth"] = seq, torch.arange(t, device=DEV) - st["cu"][seq]
    # tokens seen so far: the cache has been cut back now and then, rows are no positions
    seen = torch.tensor(rows, device=DEV) + torch.randint(0, 100000, (B,), generator=gen, device=DEV)
    st["seen"] = seen.to(torch.int32)
    if _per_head(c):
        st.update(cap=max(max(h) for h in heads) + 37, lens=i32(heads))
        shape = (B, hkv, st["cap"])
    else:
        pages = [-(-r // bs) for r in rows]
        st["max_blocks"], st["num_blocks"] = max(pages) + 1, sum(pages) + 3
        order = torch.randperm(st["num_blocks"], generator=gen, device=DEV).to(torch.int32)
        table, at = torch.zeros((B, st["max_blocks"]), dtype=torch.int32, device=DEV), 0
        for b, k in enumerate(pages):
            table[b, :k] = order[at:at + k]
            at += k
        st.update(table=table, lens=i32(rows))
        shape = (st["num_blocks"], hkv, bs)
    if c["form"] in ("store", "fill"):
        # one projection's rows: q, k and v of a token side by side
        qkv = torch.cat([_rows(gen, c, hq, (t, hq, d)).flatten(1), _rows(gen, c, hkv, (t, hkv, d)).flatten(1),
                         torch.randn(t, hkv * d, generator=gen, device=DEV)], dim=1).to(dt)
        row = (st["lens"][seq] - (st["cu"][seq + 1] - st["cu"][seq]) + st["nth"]).long()
        st.update(qkv=qkv, pos=(seen[seq] + st["nth"]).to(torch.int32), q_out=torch.zeros(t, hq, d, dtype=dt, device=DEV),
                  inv_freq=torch.pow(torch.tensor(c["base"], dtype=torch.float64, device=DEV),
                                     -2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d),
                  slots=st["table"][seq, row // bs].long() * bs + row % bs)
        for x in "kv":
            st[x] = torch.zeros(shape + (d * bits // 8,), dtype=torch.uint8, device=DEV)
            st[x + "_scale"] = torch.full(shape + (d // 32,), 127, dtype=torch.uint8, device=DEV)
    else:
        k, v = _rows(gen, c, hkv, shape + (d,)), torch.randn(shape + (d,), generator=gen, device=DEV)
        v.mul_(torch.exp(0.5 * torch.randn(shape + (1,), generator=gen, device=DEV)))
        if bits:
            (st["k"], st["k_scale"]), (st["v"], st["v_scale"]) = _quantised(k, bits), _quantised(v, bits)
        else:
            st["k"], st["v"] = k.to(dt), v.to(dt)
        del k, v
    if c["form"] in ("fill", "read"):
        st["cap"] = max(rows) + 5
        st["k_out"], st["v_out"] = (torch.zeros(B, hkv, st["cap"], d, dtype=dt, device=DEV) for _ in "kv")
    if c["form"] in ("attend", "tree"):
        st.update(q=_rows(gen, c, hq, (t, hq, d), 0.5).to(dt), out=torch.zeros(t, hq, d, dtype=dt, device=DEV),
                  lse=torch.zeros(t, hq, dtype=torch.float32, device=DEV))
    if c["form"] in ("tree", "verify"):
        parents, branches = _trees(c, add)
        words = -(-max(add) // 64)
        masks = []
        for p in parents:
            here = []
            for i, x in enumerate(p):
                here.append(1 << i | (here[x] if x >= 0 else 0))
            masks += here
        signed = lambda x: x - (1 << 64) if x >> 63 else x    # noqa: E731
        masks = [[signed(x >> 64 * w & (1 << 64) - 1) for w in range(words)] for x in masks]
        st.update(words=words, parents=i32(sum(parents, [])), sees=torch.tensor(masks, dtype=torch.int64, device=DEV))
    if c["form"] == "verify":
        # the model answers a confirmed token's successor behind it, and something that was not drafted elsewhere
        tokens = torch.randperm(1 << 17, generator=gen, device=DEV)[:t]
        target = torch.randint(1 << 17, 1 << 18, (t,), generator=gen, device=DEV)
        first = [sum(add[:b]) for b in range(len(add))]
        pairs = [(f + x, f + y) for f, p in zip(first, branches) for x, y in zip(p, p[1:])]
        if pairs:
            at, nxt = (torch.tensor(x, device=DEV) for x in zip(*pairs))
            target[at] = tokens[nxt]
        st.update(tokens=tokens.to(torch.int32), target=target.to(torch.int32), sees=torch.zeros_like(st["sees"]),
                  pos=torch.zeros(t, dtype=torch.int32, device=DEV), path=torch.full((B, max(add)), -1, dtype=torch.int32, device=DEV),
                  n_path=torch.zeros(B, dtype=torch.int32, device=DEV), next=torch.zeros(B, dtype=torch.int32, device=DEV),
                  len_out=torch.zeros_like(st["lens"]))
    return st


# -------------------------------------------------------------------------------- the plain forms
def _rotated(st, x):
    """rotary embedding of x [tokens, heads, d] in 64 bits: what is quantised lies next to a border now and then"""
    ang = st["pos"].double()[:, None] * st["inv_freq"][None]
    co, si = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    x = x.double()
    if st["inter"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * co - b * si, a * si + b * co], dim=-1).flatten(-2)
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * co - b * si, a * si + b * co], dim=-1)


def _split(st):
    hq, hkv, d = st["hq"], st["hkv"], st["d"]
    q, k, v = st["qkv"].split([hq * d, hkv * d, hkv * d], dim=1)
    return q.unflatten(1, (hq, d)), k.unflatten(1, (hkv, d)), v.unflatten(1, (hkv, d))


def _plain_store(st):
    q, k, v = _split(st)
    blk, row, bits = st["slots"] // st["block"], st["slots"] % st["block"], _bits(st)
    st["k"][blk, :, row], st["k_scale"][blk, :, row] = _quantised(_rotated(st, k), bits)
    st["v"][blk, :, row], st["v_scale"][blk, :, row] = _quantised(v.double(), bits)
    return _rotated(st, q).to(st["qkv"].dtype)


def _whole(st, x):
    """[B, hkv, rows, ..] of a pool's sequences, by the table"""
    return st[x][st["table"].long()].transpose(1, 2).flatten(2, 3)


def _plain_read(st):
    at = torch.arange(min(st["cap"], st["max_blocks"] * st["block"]), device=DEV)
    there = (at < st["lens"][:, None])[:, None, :, None]
    out = []
    for x in "kv":
        val = _values(_whole(st, x)[:, :, : at.numel()], _whole(st, x + "_scale")[:, :, : at.numel()], _bits(st)).to(torch.bfloat16)
        to = st[x + "_out"][:, :, : at.numel()]
        to.copy_(torch.where(there, val, to))
        out.append(st[x + "_out"])
    return out


def _plain_attend(st):
    B, hq, hkv, d, seq, nth = (st[x] for x in ("batch", "hq", "hkv", "d", "seq", "nth"))
    g, m, bits = hq // hkv, st["max_new"], _bits(st)
    if _per_head(st):
        n, lens, k, v = st["cap"], st["lens"].long(), st["k"].float(), st["v"].float()
    else:
        n, lens = st["max_blocks"] * st["block"], st["lens"].long()[:, None].expand(B, hkv)
        k, v = (_values(_whole(st, x), _whole(st, x + "_scale"), bits) if bits else _whole(st, x).float() for x in "kv")
    # queries of a sequence and KV head together, short sequences padded
    q = torch.zeros(B, m, hq, d, device=DEV)
    q[seq, nth] = st["q"].float()
    q = q.view(B, m, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, m * g, d)
    s = (q @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(B, hkv, m, g, n)
    more = (st["cu"][1:] - st["cu"][:-1]).long()
    at = torch.arange(n, device=DEV)
    if st["form"] == "tree":
        bit = torch.arange(64, device=DEV)
        sees = torch.zeros(B, m, 64 * st["words"], dtype=torch.bool, device=DEV)
        sees[seq, nth] = ((st["sees"][:, :, None] >> bit) & 1).bool().flatten(1)
        j = at - (lens - more[:, None])[..., None]                       # the row as a new token's number
        new = sees[:, None].expand(B, hkv, m, -1).gather(3, j.clamp(0, 64 * st["words"] - 1)[:, :, None].expand(B, hkv, m, n))
        j = j[:, :, None]
        hidden = (j >= 0) & ~(new & (j < more[:, None, None, None]))
    else:
        hidden = at >= (lens[:, :, None] - more[:, None, None] + 1 + torch.arange(m, device=DEV))[..., None]
    s.masked_fill_(hidden[:, :, :, None], -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = s.sub_(top).exp_()
    z = w.sum(dim=-1, keepdim=True)
    # rows that no query of the sequence sees count for nothing, whatever they hold
    v = torch.where((at >= lens[:, :, None])[..., None], 0.0, v)
    o = (w.view(B, hkv, m * g, n) @ v).view(B, hkv, m, g, d)
    o = torch.where(z > 0, o / z, 0.0)
    lse = (top + torch.log(z)).squeeze(-1)
    back = lambda x: x.movedim(1, 2)[seq, nth].flatten(1, 2)    # noqa: E731
    return back(o).to(st["q"].dtype), back(lse)


def _padded(st, x, rest):
    out = torch.full((st["batch"], st["max_new"]), rest, dtype=torch.long, device=DEV)
    out[st["seq"], st["nth"]] = x.long()
    return out


def _plain_verify(st):
    B, m, seq, nth = st["batch"], st["max_new"], st["seq"], st["nth"]
    j = torch.arange(m, device=DEV)
    more = (st["cu"][1:] - st["cu"][:-1]).long()
    parent = _padded(st, st["parents"], -1)
    # ancestors, a token itself among them: the powers of "itself or its parent"
    up = ((parent[..., None] == j) | torch.eye(m, dtype=torch.bool, device=DEV)).float()
    for _ in range((m - 1).bit_length()):
        up = (up @ up).clamp_(max=1.0)
    up = up > 0.5
    bits = torch.zeros(B, m, 64 * st["words"], dtype=torch.int64, device=DEV)
    bits[:, :, :m] = up
    sees = (bits.unflatten(2, (st["words"], 64)) << torch.arange(64, device=DEV)).sum(dim=-1)
    st["sees"].copy_(sees[seq, nth])
    st["pos"].copy_(st["seen"][seq] + up.sum(dim=-1)[seq, nth] - 1)
    # confirmed: the model answers the token behind its parent, and no twin of it stands in front; accepted: it and all above it
    token, target = _padded(st, st["tokens"], -1), _padded(st, st["target"], -2)
    right = (parent >= 0) & (token == target.gather(1, parent.clamp(min=0)))
    twin = (parent[:, :, None] == parent[:, None]) & (token[:, :, None] == token[:, None]) & (j[:, None] > j)
    right &= ~twin.any(dim=-1)
    right[:, 0] = True
    accepted = (~up | right[:, None]).all(dim=-1) & up[:, :, 0] & (j < more[:, None])
    count = accepted.sum(dim=-1)
    nth_accepted = accepted.cumsum(dim=-1) - 1
    grown = torch.cat([st["path"].long(), torch.full((B, 1), -1, dtype=torch.long, device=DEV)], dim=1)
    grown.scatter_(1, torch.where(accepted, nth_accepted, m), j.expand(B, m))
    path = grown[:, :m]
    st["path"].copy_(path)
    st["n_path"].copy_(count)
    st["next"].copy_(target.gather(1, path.gather(1, (count - 1)[:, None])).squeeze(1))
    # the branch's rows move together; behind its end the first row onto itself
    valid = j < count[:, None]
    src, dst = torch.where(valid, path, 0), torch.where(valid, j, 0)
    b = torch.arange(B, device=DEV)[:, None]
    if _per_head(st):
        first = (st["lens"].long() - more[:, None])[..., None]
        h = torch.arange(st["hkv"], device=DEV)[None, :, None]
        for x in "kv":
            st[x][b[..., None], h, first + dst[:, None]] = st[x][b[..., None], h, first + src[:, None]]
        st["len_out"].copy_(st["lens"] - (more - count)[:, None])
    else:
        first, bs = (st["lens"].long() - more)[:, None], st["block"]
        src, dst = first + src, first + dst
        src_block, dst_block = st["table"][b, src // bs].long(), st["table"][b, dst // bs].long()
        for x in ("k", "v", "k_scale", "v_scale") if _bits(st) else ("k", "v"):
            st[x][dst_block, :, dst % bs] = st[x][src_block, :, src % bs]
        st["len_out"].copy_(st["lens"] - (more - count))


# ------------------------------------------------------------------------------------- one pass
def _kept(st):
    """What a program keeps between its steps: the parameters, the pools' description, a workspace."""
    import paper_2510_00636_amd as ea
    if "p" not in st:
        st["ea"] = ea
        st["p"] = ea.make_params(st["batch"], st["hq"], st["hkv"], st["d"], ea.EA_F32 if st["cache"] == "f32" else ea.EA_BF16,
                                 rope_layout=int(st["inter"]))
        if "table" in st:
            st["pg"] = ea.make_paged(st["table"], st["block"], st["num_blocks"])
        if _bits(st):
            st["mx"] = ea.make_mx(st["k"], st["v"], st["k_scale"], st["v_scale"], ea.EA_MXFP8 if _bits(st) == 8 else ea.EA_MXFP4)
        if "qkv" in st:
            st["new"] = ea.make_new_rows(*_split(st), pos=st["pos"], inv_freq=st["inv_freq"])
        st["step"] = ea.make_step(st["cu"], st["n_tokens"], st["max_new"])
        if "sees" in st:
            st["tree"] = ea.make_tree(st["sees"])
        st["most"] = st["cap"] if _per_head(st) else st["max_blocks"] * st["block"]
        if "q" in st:
            st["ws"] = torch.empty(ea.attend_workspace_bytes(st["p"], st["step"], st["most"]), dtype=torch.uint8, device=DEV)
    return st["ea"]


def _own_attend(st, ea):
    rest = (st["lens"], st["most"])
    end = (st["out"], st["lse"], st["ws"])
    if st["form"] == "attend":
        ea.attend_mx(st["p"], st["q"], st["step"], st["mx"], st["pg"], *rest, *end)
    elif _bits(st):
        ea.attend_tree_mx(st["p"], st["q"], st["step"], st["tree"], st["mx"], st["pg"], *rest, *end)
    elif _per_head(st):
        ea.attend_tree(st["p"], st["q"], st["step"], st["tree"], st["k"], st["v"], *rest, st["cap"], *end)
    else:
        ea.attend_tree_paged(st["p"], st["q"], st["step"], st["tree"], st["k"], st["v"], st["pg"], *rest, *end)


def _own_verify(st, ea):
    ea.tree_masks(st["p"], st["step"], st["parents"], st["tree"], st["pos"], st["seen"])
    ea.tree_accept(st["p"], st["step"], st["tokens"], st["parents"], st["target"], st["path"], st["n_path"], st["next"])
    if _bits(st):
        ea.keep_path_mx(st["p"], st["step"], st["path"], st["n_path"], st["mx"], st["pg"], st["lens"], st["len_out"])
    elif _per_head(st):
        ea.keep_path(st["p"], st["step"], st["path"], st["n_path"], st["k"], st["v"], st["lens"], st["cap"], st["len_out"])
    else:
        ea.keep_path_paged(st["p"], st["step"], st["path"], st["n_path"], st["k"], st["v"], st["pg"], st["lens"], st["len_out"])


def _held(st):
    """the cache as the numbers that it stands for"""
    if not _bits(st):
        return {"k": st["k"], "v": st["v"]}
    out = {x: st[x].view(torch.float8_e4m3fn) for x in "kv"}
    return dict(out, **{x: st[x].view(torch.float8_e8m0fnu) for x in ("k_scale", "v_scale")})


def run(st):
    form = st["form"]
    ea = _kept(st) if own else None
    if form in ("store", "fill"):
        if own:
            ea.append_mx(st["p"], st["new"], st["slots"], st["mx"], st["pg"], st["q_out"])
            q = st["q_out"]
        else:
            q = _plain_store(st)
        if form == "store":
            return dict(_held(st), q=q)
    if form in ("fill", "read"):
        if own:
            ea.read_mx(st["p"], st["mx"], st["pg"], st["lens"], min(st["most"], st["cap"]), st["cap"], st["k_out"], st["v_out"])
            k, v = st["k_out"], st["v_out"]
        else:
            k, v = _plain_read(st)
        return {"q": q, "k": k, "v": v} if form == "fill" else {"k": k, "v": v}
    if form == "verify":
        if own:
            _own_verify(st, ea)
        else:
            _plain_verify(st)
        return dict(_held(st), **{x: st[x] for x in ("sees", "pos", "path", "n_path", "next", "len_out")})
    if own:
        _own_attend(st, ea)
        return {"out": st["out"], "lse": st["lse"]}
    out, lse = _plain_attend(st)
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------------------ in 64 bits, apart
def _on_grid(x, bits):
    """x [rows, d] in 64 bits -> its elements on the format's grid, and the powers of two that they stand on"""
    digits, least, most = (3, -6, 448.0) if bits == 8 else (1, 0, 6.0)
    g = x.reshape(x.shape[0], -1, 32)
    top = g.abs().max(dim=2).values
    e = torch.ceil(torch.log2(top / most))
    e = torch.where(top > most * torch.exp2(e), e + 1, e)
    e = torch.where((top > 0) & (top <= most * torch.exp2(e - 1)), e - 1, e)
    by = torch.exp2(torch.where(top > 0, e.clamp(min=-117), -117.0))
    z = g / by[:, :, None]
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** least))) - digits)
    return (torch.round(z / step) * step).reshape(x.shape), by


def _from_bytes(b, scale, bits):
    """bytes [rows, ..] of one head -> 64 bits, from the fields of the format"""
    code = b.long() if bits == 8 else torch.stack([b.long() % 16, b.long() // 16], dim=2).reshape(b.shape[0], -1)
    digits, bias, fields = (3, 7, 16) if bits == 8 else (1, 1, 4)
    sign = 1.0 - 2.0 * (code >= 2 ** (bits - 1)).double()
    code = code % 2 ** (bits - 1)
    frac, e = (code % 2 ** digits).double() / 2 ** digits, code // 2 ** digits
    assert int(e.max() if e.numel() else 0) < fields
    x = torch.where(e > 0, (1 + frac) * torch.exp2((e - bias).double()), frac * 2.0 ** (1 - bias))
    return sign * x * torch.exp2(scale.double() - 127).repeat_interleave(32, dim=1)


def exact(c, seed):
    """From the definitions, a sequence (and a head) after the other."""
    if work(c)["flops"] > 3e12:
        return None
    st = prepare(c, seed)
    d, hq, hkv, g, bits, bs = c["d"], c["hq"], c["hkv"], c["hq"] // c["hkv"], _bits(c), c["block"]
    add, rows, heads = _lengths(c)
    first = [sum(add[:b]) for b in range(len(add))]

    def pooled(x, b, h, n):
        """the first n rows of a sequence and head"""
        return st[x][st["table"][b, : -(-n // bs)].long(), h].reshape(-1, st[x].shape[-1])[:n]
    if c["form"] == "verify":
        # the branch that the targets were made of, a row after the other; whole numbers have no value in 64 bits
        held, table = {x: y.double() for x, y in _held(st).items()}, None if _per_head(c) else st["table"].tolist()
        for b, branch in enumerate(_trees(c, add)[1]):
            for h in range(hkv):
                base = heads[b][h] - add[b]
                for to, frm in enumerate(branch):
                    for y in held.values():
                        if _per_head(c):
                            y[b, h, base + to] = y[b, h, base + frm]
                        else:
                            at = [(table[b][(base + i) // bs], (base + i) % bs) for i in (to, frm)]
                            y[at[0][0], h, at[0][1]] = y[at[1][0], h, at[1][1]]
        return dict(held, **{x: None for x in ("sees", "pos", "path", "n_path", "next", "len_out")})
    if c["form"] in ("store", "fill"):
        qkv = st["qkv"].double().view(-1, hq + 2 * hkv, d)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        ang = torch.outer(st["pos"].double(), st["inv_freq"])
        turn = torch.complex(torch.cos(ang), torch.sin(ang))[:, None]

        def turned(x):
            if c["inter"]:
                return torch.view_as_real(torch.view_as_complex(x.reshape(*x.shape[:-1], d // 2, 2).contiguous()) * turn).reshape(x.shape)
            z = torch.complex(x[..., : d // 2], x[..., d // 2:]) * turn
            return torch.cat([z.real, z.imag], dim=-1)
        out = {"q": turned(q)}
        for x, y in (("k", turned(k)), ("v", v)):
            on, by = _on_grid(y.reshape(-1, d), bits)
            if c["form"] == "fill":
                whole = torch.zeros_like(st[x + "_out"], dtype=torch.float64)
                val = (on.reshape(-1, 32) * by.reshape(-1, 1)).reshape(-1, hkv, d)
                for b, (f, a) in enumerate(zip(first, add)):
                    whole[b, :, :a] = val[f:f + a].transpose(0, 1)
                out[x] = whole
                continue
            pool, scales = torch.zeros_like(st[x], dtype=torch.float64), torch.ones_like(st[x + "_scale"], dtype=torch.float64)
            at_block = torch.div(st["slots"], bs, rounding_mode="floor")
            pool[at_block, :, st["slots"] - at_block * bs] = on.reshape(-1, hkv, d)
            scales[at_block, :, st["slots"] - at_block * bs] = by.reshape(-1, hkv, d // 32)
            out[x], out[x + "_scale"] = pool, scales
        return out
    if c["form"] == "read":
        out = {}
        for x in "kv":
            out[x] = torch.zeros_like(st[x + "_out"], dtype=torch.float64)
            for b, n in enumerate(rows):
                for h in range(hkv):
                    out[x][b, h, :n] = _from_bytes(pooled(x, b, h, n), pooled(x + "_scale", b, h, n), bits)
        return out
    out = torch.zeros(st["n_tokens"], hq, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st["n_tokens"], hq, dtype=torch.float64, device=DEV)
    parents = _trees(c, add)[0] if c["form"] == "tree" else None
    for b, (f, a) in enumerate(zip(first, add)):
        among = torch.ones(a, a, dtype=torch.bool).tril()
        if parents:
            among = torch.eye(a, dtype=torch.bool)
            for i, x in enumerate(parents[b]):
                if x >= 0:
                    among[i] |= among[x]
        among = among.to(DEV)
        for h in range(hkv):
            n = heads[b][h]
            if _per_head(c):
                k, v = (st[x][b, h, :n].double() for x in "kv")
            elif bits:
                k, v = (_from_bytes(pooled(x, b, h, n), pooled(x + "_scale", b, h, n), bits) for x in "kv")
            else:
                k, v = (pooled(x, b, h, n).double() for x in "kv")
            seen = torch.cat([torch.ones(a, n - a, dtype=torch.bool, device=DEV), among], dim=1)
            for gg in range(g):
                s = st["q"][f:f + a, h * g + gg].double() @ k.T.contiguous() / math.sqrt(d)
                s = torch.where(seen, s, -math.inf)
                z = torch.logsumexp(s, dim=1)
                lse[f:f + a, h * g + gg] = z
                out[f:f + a, h * g + gg] = torch.exp(s - z[:, None]) @ v
    return {"out": out, "lse": lse}
