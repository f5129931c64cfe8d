"""Heads, rotary tables and the paged 4-bit KV cache from their definitions in include/relax_mi355.h, in numpy.  What the definition rounds (prepared heads, scales, codes)
is rounded here the same way, in the same order, so that it can be compared bit by bit; attention is in 64 bits.  A pool is {"k", "v": uint8
[pages, g, blocks, 8 * d], "ks", "vs": float16 [pages, g, blocks, d / 2]}."""
import numpy as np

from paged_oracle import BLOCK, page_of, sequences, storable

GROUP = 32
F = np.float32


def code_place(name, d):
    """[16, d] -> (byte, shift in it) of (token, element) among the codes of a block."""
    t, e = np.meshgrid(np.arange(BLOCK), np.arange(d), indexing="ij")
    if name == "k":
        word, i = (e // 8 % 4 * 16 + t) * (d // 32) + e // 32, e % 8
        return 4 * word + i % 2 * 2 + i // 4, i // 2 % 2 * 4
    word = (t // 4 * 16 + e % 16) * (d // 32) + e // 32
    return 4 * word + t % 4 % 2 * 2 + t % 4 // 2, e // 16 % 2 * 4


def scale_place(d):
    """[16, d / 32] -> place of (token, group) among the scales of a block."""
    t, j = np.meshgrid(np.arange(BLOCK), np.arange(d // GROUP), indexing="ij")
    return (t // 4 * (d // GROUP) + j) * 4 + t % 4


def frequencies(R, base, scaling="plain", factor=1.0, trained=1.0, slow=1.0, fast=2.0):
    t = np.arange(R // 2, dtype=np.float64)
    f = base ** (-2.0 * t / R)
    if scaling == "plain":
        w = np.ones_like(f)
    elif scaling == "linear":
        w = np.zeros_like(f)
    elif scaling == "wavelength":
        w = np.clip((trained * f / (2 * np.pi) - slow) / (fast - slow), 0, 1)
    else:
        at = lambda b: R * np.log(trained / (2 * np.pi * b)) / (2 * np.log(base))
        first, last = max(np.floor(at(fast)), 0.0), min(np.ceil(at(slow)), R - 1.0)
        w = 1 - np.clip((t - first) / max(last - first, 0.001), 0, 1)
    return f * (w + (1 - w) / factor)


def prepare(x, w, eps, cs, R, pairs):
    """Heads x float32 [.., heads, d] as relax_head_prep has them; w float32 [d] or None, cs float32 [.., 1, R / 2, 2] or None.  fp32, each operation rounded once."""
    x = x.astype(F)
    if w is not None:
        ms = (x.astype(np.float64) ** 2).sum(axis=-1, keepdims=True) / x.shape[-1] + np.float64(F(eps))
        with np.errstate(divide="ignore"):
            r = np.where(ms == 0, 0.0, 1.0 / np.sqrt(ms)).astype(F)
        x = (x * r) * w
    if cs is None:
        return x
    c, s = cs[..., 0], cs[..., 1]
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if pairs else (x[..., :R // 2], x[..., R // 2:R])
    a, b = a * c - b * s, a * s + b * c
    out = x.copy()
    if pairs:
        out[..., 0:R:2], out[..., 1:R:2] = a, b
    else:
        out[..., :R // 2], out[..., R // 2:R] = a, b
    return out


def round8(x):
    """float32 to eight significant bits, ties to even."""
    u = x.astype(F).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + (u >> 16 & 1)) & 0xffff0000).astype(np.uint32).view(F)


def quantise(x):
    """(codes [.., d] in 0..15, scales float16 [.., d / 32]) of finite float32 [.., d]."""
    y = x.reshape(*x.shape[:-1], -1, GROUP)
    top, low = y.max(axis=-1), y.min(axis=-1)
    s = np.clip(round8(np.where(top >= -low, top, low) * F(-0.125)), F(-8160), F(8160)).astype(np.float16)
    s32 = s.astype(F)[..., None]
    q = np.where(s32 != 0, y / np.where(s32 != 0, s32, F(1)), F(0))
    return (np.clip(np.rint(q), -8, 7) + 8).astype(np.uint8).reshape(x.shape), s


def append(pool, pages, page_size, k, v, q_lens, kv_lens, slots, cap=None):
    """The pool behind the call; k (prepared) and v float32 [n, g, d]."""
    pool = {key: x.copy() for key, x in pool.items()}
    d = k.shape[2]
    codes = {name: quantise(x) for name, x in (("k", k), ("v", v))}
    for row, ql, L, slot in sequences(q_lens, kv_lens, slots):
        for i in range(ql):
            pos = L - ql + i
            page = page_of(pages, pool["k"].shape[0], slot, pos, page_size)
            if page < 0:
                continue
            blk, t = pos % page_size // BLOCK, pos % BLOCK
            for name in "kv":
                u, s = codes[name][0][row + i], codes[name][1][row + i]
                byte, shift = (x[t] for x in code_place(name, d))
                at = pool[name][page, :, blk]                            # a view, [g, 8 d]
                for half in (0, 4):
                    sel = shift == half
                    at[:, byte[sel]] = (at[:, byte[sel]] & (0xF0 if half == 0 else 0x0F)) | (u[:, sel] << half)
                pool[name + "s"][page, :, blk][:, scale_place(d)[t]] = s
    return pool


def values(pool, name, pages, page_size, slot, positions, d):
    """(codes - 8, scales) float64 [len(positions), g, d] of one slot; NaN where there is no page."""
    g = pool[name].shape[1]
    c, s = (np.full((len(positions), g, d), np.nan) for _ in "cs")
    byte, shift = code_place(name, d)
    for j, pos in enumerate(positions):
        page = page_of(pages, pool[name].shape[0], slot, int(pos), page_size)
        if page < 0:
            continue
        blk, t = pos % page_size // BLOCK, pos % BLOCK
        c[j] = (pool[name][page, :, blk][:, byte[t]] >> shift[t] & 15).astype(np.float64) - 8
        s[j] = np.repeat(pool[name + "s"][page, :, blk][:, scale_place(d)[t]].astype(np.float64), GROUP, axis=1)
    return c, s


def attention(q, pool, pages, page_size, q_lens, kv_lens, slots, g, d, heads=None):
    """(out, tolerance), float64 [n, h, d], of the given query heads (None: all).  The tolerance counts what the kernels round, each to nearest, so by half a step at most:
      the output to fp16                                        2^-11 |o|, 2^-25 below fp16's normal range
      the weights, or weights times scales, to fp16             2^-11 sum p |v|; with a sum of the rounded ones 2^-11 |o| more
      ... below fp16's normal range                             2^-26 of the largest weight per code unit (few pairs: the smallest weight at the reference is 2, a
                                                                quarter of the largest at most), 2^-36 of the largest |v| per token (many pairs)
      scores: per 32 elements 40 sums of at most 23 sum |q| (codes 0..15 against -8 sum q), then scales, 8 sum |q| each, or 136 sums of 8 |s| sum |q|:
      1100 2^-24 sum |s| |q| / sqrt d, which changes a probability by that factor, in numerator and denominator
      sums over T tokens in fp32: T / 4 + 64 roundings of at most 23 sum p |s| (codes 0..15 against -8 sum p s), of each operand's group"""
    h = q.shape[1]
    rep = h // g
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for row, ql, L, slot in sequences(q_lens, kv_lens, slots):
        (kc, ks), (vc, vs) = (values(pool, name, pages, page_size, slot, np.arange(L), d) for name in "kv")
        there = ~np.isnan(kc[:, 0, 0])
        for head in range(h) if heads is None else heads:
            j = head // rep
            k, k_s, v, v_c, v_s = (kc * ks)[there, j], ks[there, j], (vc * vs)[there, j], vc[there, j], vs[there, j]
            if not len(k):
                continue
            t = np.arange(L)[there]
            qh = q[row:row + ql, head]
            seen = t[None, :] <= np.arange(L - ql, L)[:, None]
            some = seen.any(axis=1)
            s = np.where(seen, qh @ k.T / np.sqrt(d), -np.inf)
            mag = np.where(seen, np.abs(qh) @ np.abs(k_s).T / np.sqrt(d), 0.0)
            p = np.exp(s - np.where(some, s.max(axis=1), 0.0)[:, None])
            p /= np.where(some, p.sum(axis=1), 1.0)[:, None]
            o = p @ v
            delta = (1100 * 2.0 ** -24 * mag.max(axis=1))[:, None]
            scale = p @ np.abs(v_s)
            mean = p @ np.abs(v)
            small = 2.0 ** -26 * p.max(axis=1)[:, None] * (seen.astype(np.float64) @ np.abs(v_c)) + len(t) * 2.0 ** -36 * np.abs(v).max()
            out[row:row + ql, head] = o
            tol[row:row + ql, head] = np.where(some[:, None], 2.0 ** -10 * np.abs(o) + (2.0 ** -11 + 2 * delta) * mean + 2.0 ** -25 + small +
                                               (len(t) / 4 + 64) * 23 * 2.0 ** -24 * scale, 0.0)
    return out, tol
