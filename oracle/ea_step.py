"""A model's step over its cache, in fp64 numpy: block tables and slot maps, the rotary store of new rows, attention.

The definitions of include/ea.h, one sequence (and head) after the other."""
import numpy as np


def _blocks(rows, block_size):
    return -(-max(int(rows), 0) // block_size)


def block_tables(table, free_list, free, len_old, len_new, block_size, n_tokens, seen=None):
    """Returns (table, free_list, free, len_out, cu_tokens, slots, pos); slots is -1 and pos None-like (-1) behind the tokens."""
    table, free_list = table.copy(), free_list.copy()
    B, max_blocks = table.shape
    stack = [int(x) for x in free_list[:free]]
    back = []
    for b in range(B):
        for j in range(_blocks(len_new[b], block_size), _blocks(len_old[b], block_size)):
            back.append(int(table[b, j]))
    # the first one given back is the first to be taken again
    stack += back[::-1]
    cu, len_out, slots, pos = [0], [], [], []
    left = len(stack)                  # what the sequences so far have not asked for
    for b in range(B):
        held, need = _blocks(len_old[b], block_size), _blocks(len_new[b], block_size)
        fits = need <= max_blocks
        ok = fits
        if fits and need > held:
            left -= need - held
            ok = left >= 0
        if ok and need > held:
            for j in range(held, need):
                table[b, j] = stack.pop()
        len_out.append(max(int(len_new[b]), 0) if ok else max(int(len_old[b]), 0))
        old = max(int(len_old[b]), 0)
        more = max(0, max(int(len_new[b]), 0) - old)
        cu.append(cu[-1] + more)
        for i in range(more):
            row = old + i
            slots.append(int(table[b, row // block_size]) * block_size + row % block_size if ok else -1)
            pos.append((old if seen is None else int(seen[b])) + i)
    # the list beyond its end is not written, but for blocks given back and not taken
    for i in range(min(free, len(stack)), len(stack)):
        free_list[i] = stack[i]
    slots = (slots + [-1] * n_tokens)[:n_tokens]
    pos = (pos + [-1] * n_tokens)[:n_tokens]
    return (table, free_list, len(stack), np.array(len_out), np.array(cu), np.array(slots, dtype=np.int64), np.array(pos))


def rotate(x, pos, inv_freq, interleaved):
    """Eq. 1 on x [tokens, heads, d] (fp64)."""
    ang = np.asarray(pos, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)[None]
    co, si = np.cos(ang)[:, None], np.sin(ang)[:, None]
    out = np.empty_like(x)
    h = x.shape[-1] // 2
    first, second = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, h), slice(h, None))
    out[..., first] = x[..., first] * co - x[..., second] * si
    out[..., second] = x[..., first] * si + x[..., second] * co
    return out


def attend_head(q, k, v, length, m):
    """q [m, d] of one query head, k, v [>= length, d] of its KV head -> (out [m, d], lse [m], spread [m, d], logit [m]): spread is
    the weighted mean of |v| and logit the largest sum |q_c k_c| / sqrt(d) of a row, which error bounds are made of."""
    d = q.shape[-1]
    out, lse, spread, logit = np.zeros((m, d)), np.full(m, -np.inf), np.zeros((m, d)), np.zeros(m)
    for i in range(m):
        n = length - (m - 1 - i)
        if n <= 0:
            continue
        s = k[:n] @ q[i] / np.sqrt(d)
        top = s.max()
        w = np.exp(s - top)
        z = w.sum()
        out[i], lse[i] = w @ v[:n] / z, top + np.log(z)
        spread[i] = w @ np.abs(v[:n]) / z
        logit[i] = (np.abs(k[:n]) @ np.abs(q[i])).max() / np.sqrt(d)
    return out, lse, spread, logit


def attend(q, cu, k, v, lengths):
    """q [tokens, Hq, d], k, v lists [b][h] of [rows, d], lengths [B][Hkv]; tokens behind cu[-1] are left zero.
    Returns (out, lse, spread, logit) as attend_head's, over [tokens, Hq]."""
    t, hq, d = q.shape
    out, spread = np.zeros((t, hq, d)), np.zeros((t, hq, d))
    lse, logit = np.zeros((t, hq)), np.zeros((t, hq))
    for b in range(len(cu) - 1):
        m = cu[b + 1] - cu[b]
        hkv = len(lengths[b])
        g = hq // hkv
        for h in range(hkv):
            for x in range(h * g, (h + 1) * g):
                at = slice(cu[b], cu[b + 1])
                out[at, x], lse[at, x], spread[at, x], logit[at, x] = attend_head(q[at, x], k[b][h], v[b][h], int(lengths[b][h]), m)
    return out, lse, spread, logit
