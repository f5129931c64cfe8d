"""The paged 8-bit KV cache and the log probabilities in 64 bits, from their definitions in include/relax_mi355.h: numpy, one sequence and
one token at a time.  A pool is {"k", "v": uint8 [pages, g, blocks, 16 * d], "ks", "vs": float32 [pages, g, blocks]}."""
import numpy as np

BLOCK = 16


def code_index(name, d):
    """[16, d] -> place of (token, element) among the codes of a block."""
    t, e = np.meshgrid(np.arange(BLOCK), np.arange(d), indexing="ij")
    if name == "k":
        return ((e // 16) * BLOCK + t) * 16 + e % 16
    return (((e // 64 * 4 + t // 4) * 16 + e % 16) * 4 + e // 16 % 4) * 4 + t % 4


def rope_angles(pos, d, base=10000.0):
    return pos * base ** (-2.0 * np.arange(d // 2, dtype=np.float64) / d)


def rotate(x, pos, d):
    """x [heads, d] at one position, in 64 bits."""
    a, b = x[:, :d // 2], x[:, d // 2:]
    cos, sin = np.cos(rope_angles(pos, d)), np.sin(rope_angles(pos, d))
    return np.concatenate([a * cos - b * sin, a * sin + b * cos], axis=1)


def storable(x):
    return np.clip(np.where(np.isnan(x), 0.0, x), -65504.0, 65504.0)


def page_of(pages, n_pages, slot, pos, page_size):
    p = int(pages[slot][pos // page_size])
    return p if 0 <= p < n_pages else -1


def sequences(q_lens, kv_lens, slots):
    row = 0
    for b, (ql, L) in enumerate(zip(q_lens, kv_lens)):
        yield row, ql, L, b if slots is None else slots[b]
        row += ql


def append(pool, pages, page_size, k, v, q_lens, kv_lens, slots, d, rope=True):
    """What the pool has to hold behind the call: for each touched (name, page, head, block) the scale, and the unrounded code and whether it
    is new or old of each of the sequence's tokens in it.  Yields dicts; k, v float64 [n, g, d]."""
    n_pages = pool["k"].shape[0]
    for row, ql, L, slot in sequences(q_lens, kv_lens, slots):
        for first in range((L - ql) // BLOCK * BLOCK, L, BLOCK):
            page = page_of(pages, n_pages, slot, first, page_size)
            if page < 0:
                continue
            low, high = max(L - ql - first, 0), min(L - first, BLOCK)
            blk = first % page_size // BLOCK
            new = {"k": [], "v": []}
            for t in range(low, high):
                i = row + first + t - (L - ql)
                new["k"].append(storable(rotate(k[i], first + t, d) if rope else k[i]))
                new["v"].append(storable(v[i]))
            for name in "kv":
                x = np.stack(new[name])                                  # [tokens, g, d]
                index = code_index(name, d)
                for head in range(x.shape[1]):
                    old = np.float64(pool[name + "s"][page, head, blk]) if low else 0.0
                    s = max(old, np.abs(x[:, head]).max() / 127.0)
                    codes = pool[name][page, head, blk][index].astype(np.float64) - 128.0          # [16, d]
                    yield {"name": name, "at": (page, head, blk), "low": low, "high": high, "scale": s, "grew": s > old and low > 0,
                           "old": codes[:low] * (old / s if s else 0.0), "new": x[:, head] / s if s else 0.0 * x[:, head]}


def values(pool, name, pages, page_size, slot, positions, d):
    """float64 [len(positions), g, d] of one slot; NaN where there is no page."""
    index = code_index(name, d)
    g = pool[name].shape[1]
    out = np.full((len(positions), g, d), np.nan)
    for j, pos in enumerate(positions):
        page = page_of(pages, pool[name].shape[0], slot, int(pos), page_size)
        if page < 0:
            continue
        blk, t = pos % page_size // BLOCK, pos % BLOCK
        out[j] = (pool[name][page, :, blk][:, index[t]].astype(np.float64) - 128.0) * pool[name + "s"][page, :, blk].astype(np.float64)[:, None]
    return out


def attention(q, pool, pages, page_size, q_lens, kv_lens, slots, g, d, heads=None):
    """(out, tolerance), float64 [n, h, d], of the given query heads (None: all).  The tolerance counts what the kernels round, each to nearest, so by half a step, 2^-11, at most:
      the output to fp16                                                       2^-11 |o|, 2^-25 below fp16's normal range
      the probabilities to fp16, p (1 + e), |e| <= 2^-11, with a sum of the rounded ones: o becomes sum p (1 + e) v / sum p (1 + e), which is off by
      sum p (e - mean of e) v                                                  2^-11 (sum p |v| + |o|)
      values below 2^-31 of the largest                                        2^-32 of the largest |v|
      scores in fp32, whose sum of d products and scaling is off by (d + 8) 2^-24 of the sum of magnitudes, which changes a probability by
      that factor, at once in numerator and denominator                        2 (d + 8) 2^-24 |q| |k| sum p |v|
      sums of probabilities and of O in fp32, 2^6 roundings in a row           2^-18 sum p |v|
      weights below 2^-24 of the largest weight's 2^11                         2^-36 of the largest |v| each"""
    h = q.shape[1]
    rep = h // g
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for row, ql, L, slot in sequences(q_lens, kv_lens, slots):
        k, v = (values(pool, name, pages, page_size, slot, np.arange(L), d) for name in "kv")
        there = ~np.isnan(k[:, 0, 0])
        for head in range(h) if heads is None else heads:
            kh, vh = k[there, head // rep], v[there, head // rep]
            if not len(kh):
                continue
            t = np.arange(L)[there]
            qh = q[row:row + ql, head]
            seen = t[None, :] <= np.arange(L - ql, L)[:, None]
            s = np.where(seen, qh @ kh.T / np.sqrt(d), -np.inf)
            mag = np.where(seen, np.abs(qh) @ np.abs(kh).T / np.sqrt(d), 0.0)
            some = seen.any(axis=1)
            p = np.exp(s - np.where(some, s.max(axis=1), 0.0)[:, None])
            p /= np.where(some, p.sum(axis=1), 1.0)[:, None]
            o, mean = p @ vh, p @ np.abs(vh)
            delta = ((d + 8) * 2.0 ** -24 * mag.max(axis=1))[:, None]
            out[row:row + ql, head] = o
            tol[row:row + ql, head] = np.where(some[:, None], 2.0 ** -10 * np.abs(o) + (2.0 ** -11 + 2 * delta + 2.0 ** -18) * mean + 2.0 ** -25 +
                                               (len(t) * 2.0 ** -36 + 2.0 ** -32) * np.abs(vh).max(), 0.0)
    return out, tol


def token_logprobs(logits, targets, top):
    """(logprobs, entropy, ids, top logprobs) of float64 [n, V], row by row."""
    n, V = logits.shape
    lp, ent, ids, tops = np.zeros(n), np.zeros(n), np.zeros((n, top), np.int64), np.zeros((n, top))
    for i, x in enumerate(logits):
        finite = x[x > -np.inf]
        key = np.where(np.isnan(x), -np.inf, x)
        ids[i] = np.lexsort((np.arange(V), np.isnan(x), -key))[:top]
        if finite.size == 0 and not np.isnan(x).any():
            logp, ent[i] = np.full(V, -np.inf), 0.0
        else:
            with np.errstate(invalid="ignore"):
                m = np.nanmax(x) if not np.isnan(x).all() else np.nan
                z = x - m
                rest = np.exp(z[z < 0]).sum() + (z == 0).sum() - 1 if not np.isnan(z).any() else np.nan
                logp = np.where((x == -np.inf) & ~np.isnan(rest) if np.isnan(x).any() else x == -np.inf, -np.inf, z - np.log1p(rest))
                if np.isnan(x).any():
                    logp = np.full(V, np.nan)
                p = np.exp(logp)
                ent[i] = np.nan if np.isnan(rest) else -(p[p > 0] * logp[p > 0]).sum()
        t = -1 if targets is None else targets[i]
        lp[i] = logp[t] if 0 <= t < V else (np.nan if np.isnan(x).any() else -np.inf)
        tops[i] = logp[ids[i]]
    return lp, ent, ids, tops
