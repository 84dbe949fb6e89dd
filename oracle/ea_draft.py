"""Rows quantised with a power of two for 32 channels, and steps whose tokens form trees, in fp64 numpy: the definitions of
include/ea.h, one group, sequence and head after the other."""
import numpy as np

# what an element can be: 0 and the positive numbers, by code
E4M3 = np.array([(m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BF16_MOST = (2 - 2.0 ** -7) * 2.0 ** 127


def grid(bits):
    return E4M3 if bits == 8 else E2M1


def nearest(x, bits, most):
    """codes (without a sign) of the elements nearest to |x| <= most, halves to the even code"""
    g = grid(bits)
    g = g[g <= most]
    hi = np.clip(np.searchsorted(g, x), 1, len(g) - 1)
    lo = hi - 1
    up, down = g[hi] - x, x - g[lo]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def quantise(x, bits):
    """x [.., d] -> (codes [.., d] with the sign in the highest bit, exponent bytes [.., d / 32])"""
    g = np.asarray(x, dtype=np.float64)
    g = g.reshape(g.shape[:-1] + (g.shape[-1] // 32, 32))
    fine = np.isfinite(g).all(-1)
    z = np.where(fine[..., None], g, 0.0)
    top, most = np.abs(z).max(-1), grid(bits)[-1]
    e = np.full(top.shape, 10)
    for _ in range(300):                      # the least one that is large enough
        e = np.where(top > most * 2.0 ** (e - 127.0), e + 1, e)
    by = 2.0 ** (e - 127.0)
    # no element stands for more than bf16's largest number
    cap = np.where(most * by > BF16_MOST, most / 2 if bits == 4 else 240.0, most)
    codes = np.zeros(z.shape, dtype=np.int64)
    for c in np.unique(cap):
        at = cap == c
        codes[at] = nearest(np.minimum(np.abs(z[at]) / by[at][..., None], c), bits, c)
    codes += np.signbit(z) * 2 ** (bits - 1)
    return codes.reshape(x.shape), np.where(fine, e, 255)


def packed(codes, bits):
    """bytes of codes: two to a byte where they have four bits, the even channel low"""
    c = codes.astype(np.uint8)
    return c if bits == 8 else c[..., 0::2] | c[..., 1::2] << 4


def unpacked(b, bits):
    return b.astype(np.int64) if bits == 8 else np.stack([b & 15, b >> 4], axis=-1).reshape(b.shape[:-1] + (-1,)).astype(np.int64)


def values(codes, e, bits):
    """what codes and exponent bytes stand for"""
    sign, c = np.where(codes >> (bits - 1), -1.0, 1.0), codes & (2 ** (bits - 1) - 1)
    g = np.append(E4M3, np.nan) if bits == 8 else E2M1
    with np.errstate(invalid="ignore"):
        by = np.where(np.asarray(e) == 255, np.nan, 2.0 ** (np.asarray(e, dtype=np.float64) - 127))
        return sign * g[c] * np.repeat(by, 32, axis=-1)


# --------------------------------------------------------------------------------------- trees
def masks(parents, cu, seen=None):
    """bool [tokens, most tokens of a sequence] of what a token sees, and positions"""
    t, most = int(cu[-1]), max(1, int(np.diff(cu).max()))
    sees, pos = np.zeros((t, most), dtype=bool), np.zeros(t, dtype=np.int64)
    for b in range(len(cu) - 1):
        for i in range(cu[b + 1] - cu[b]):
            x, above = i, -1
            while x >= 0:
                sees[cu[b] + i, x] = True
                above += 1
                up = int(parents[cu[b] + x])
                x = up if 0 <= up < x else -1
            pos[cu[b] + i] = (0 if seen is None else int(seen[b])) + above
    return sees, pos


def words_of(sees, words):
    """the masks as 64-bit words"""
    bits = np.zeros((sees.shape[0], words * 64), dtype=np.uint64)
    n = min(sees.shape[1], words * 64)
    bits[:, :n] = sees[:, :n]
    return (bits.reshape(-1, words, 64) << np.arange(64, dtype=np.uint64)).sum(-1, dtype=np.uint64)


def accept(tokens, parents, target, cu):
    """per sequence the path and the model's answer behind it"""
    paths, nxt = [], []
    for b in range(len(cu) - 1):
        m, at = cu[b + 1] - cu[b], cu[b]
        if m == 0:
            paths.append([])
            nxt.append(-1)
            continue
        path = [0]
        while True:
            here = path[-1]
            below = [j for j in range(here + 1, m) if parents[at + j] == here and tokens[at + j] == target[at + here]]
            if not below:
                break
            path.append(below[0])
        paths.append(path)
        nxt.append(int(target[at + path[-1]]))
    return paths, nxt


def attend(q, cu, k, v, lengths, sees):
    """As ea_step.attend, token i of a sequence with m tokens seeing the rows below len - m and row len - m + j where sees[token, j]."""
    t, hq, d = q.shape
    out, spread = np.zeros((t, hq, d)), np.zeros((t, hq, d))
    lse, logit = np.full((t, hq), -np.inf), np.zeros((t, hq))
    for b in range(len(cu) - 1):
        m, hkv = cu[b + 1] - cu[b], len(lengths[b])
        g = hq // hkv
        for h in range(hkv):
            n = int(lengths[b][h])
            row = np.arange(max(n, 0)) - (n - m)
            for i in range(m):
                there = (row < 0) | sees[cu[b] + i][np.clip(row, 0, sees.shape[1] - 1)] & (row < sees.shape[1])
                if not there.any():
                    continue
                kk, vv = k[b][h][:n][there], v[b][h][:n][there]
                x = slice(h * g, (h + 1) * g)
                s = q[cu[b] + i, x] @ kk.T / np.sqrt(d)
                top = s.max(-1, keepdims=True)
                w = np.exp(s - top)
                z = w.sum(-1, keepdims=True)
                out[cu[b] + i, x], lse[cu[b] + i, x] = w @ vv / z, (top + np.log(z))[:, 0]
                spread[cu[b] + i, x] = w @ np.abs(vv) / z
                logit[cu[b] + i, x] = (np.abs(q[cu[b] + i, x]) @ np.abs(kk).T).max(-1) / np.sqrt(d)
    return out, lse, spread, logit
