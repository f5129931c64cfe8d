"""Attention over the paged 4-bit KV cache where its tolerance can be narrow: scores that are exact in fp32, so that an output is held to a part of sum p |v| whatever the size of the values
and the length of the context."""
import numpy as np
import pytest

import paged4_oracle as po
from test_gpu_paged4 import Bench, half, rx, seed_of  # noqa: F401  (rx: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def exact_scores(b, rng, v_scale):
    """Key scales of +-1/8, so that with queries in multiples of 1/4 below 32 every product and sum of a score is exact; value scales v_scale(shape) of eight bits."""
    for key, make in (("ks", lambda shape: rng.choice([-0.125, 0.125], shape)), ("vs", lambda shape: v_scale(shape) * rng.choice([-1, 1], shape))):
        x = po.round8(make(b.pool[key].shape).astype(np.float32)).astype(np.float16)
        b.pool[key] = np.where(np.isnan(b.pool[key]), b.pool[key], x).astype(np.float16)
        b.dev[key].copy_(torch.from_numpy(b.pool[key]))


def narrow(q, b):
    """(out, tolerance), float64 [n, h, d].  What is rounded, each to nearest:
      the output to fp16                             2^-11 |o|, 2^-25 below fp16's normal range
      weights, or weights times scales, to fp16      2^-11 sum p |v|; with a sum of the rounded ones 2^-11 |o| more
      ... below fp16's normal range                  a step is 2^-24; the largest weight times the root of the sum of squares of a lane's scales, sixteen, is 2^12 at least, so times the largest of
                                                     them 2^10: 2^-35 of the largest p times scale, of a code of 8 at most, per token; many pairs: the largest weight is 2^11 at least: 2^-36
                                                     of the largest p |v| per token
      exponents                                      scores are exact; times c and minus the reference they are below 2^6 in size: c is off by 4 2^-24 of itself, the multiply-add by 2^-24, the
                                                     exponential by 2^-22 of itself: below 2^-15 of a weight, in numerator and denominator
      sums in fp32                                   a product of 32 tokens is off by 4 2^-24 of its terms, at most 23 |s| p each (codes 0..15 against -8 sum p s): T / 32 + 8 of them in a row"""
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    rep = b.h // b.g
    for row, ql, L, slot in po.sequences(b.q_lens, b.kv_lens, b.slots):
        (kc, ks), (vc, vs) = (po.values(b.pool, name, b.pages, b.page_size, slot, np.arange(L), b.d) for name in "kv")
        for i in range(ql):
            seen = L - ql + i + 1
            for head in range(b.h):
                j = head // rep
                s = (kc * ks)[:seen, j] @ q[row + i, head] / np.sqrt(b.d)
                p = np.exp(s - s.max())
                p /= p.sum()
                v, scale = (vc * vs)[:seen, j], np.abs(vs[:seen, j])
                o, mean, unit = p @ v, p @ np.abs(v), p @ scale
                small = seen * max(2.0 ** -32 * p.max() * scale.max(), 2.0 ** -36 * (p[:, None] * np.abs(v)).max())
                out[row + i, head] = o
                tol[row + i, head] = 2.0 ** -10 * np.abs(o) + 2.0 ** -25 + (2.0 ** -11 + 2.0 ** -14) * mean + small + (seen / 32 + 8) * 4 * 2.0 ** -24 * 23 * unit
    return out, tol


@pytest.mark.parametrize("exponent,spread", [(-12, 0), (-15, 0), (-10, 8), (0, 0), (12, 0)])
@pytest.mark.parametrize("shape,rows,L", [((8, 1, 128), 1, 20001), ((8, 1, 128), 1, 4099), ((8, 1, 128), 3, 4099), ((16, 2, 64), 1, 9000), ((2, 2, 64), 3, 2000), ((4, 4, 64), 1, 700)], ids=str)
def test_values_of_any_size(rx, shape, rows, L, exponent, spread):  # noqa: F811
    """Scores of standard deviation 3, so that thousands of tokens share a row, and values whose scales are 2^exponent to twice that, or that many powers of two smaller from group to group."""
    rng = np.random.default_rng(seed_of(shape, rows, L, exponent))
    b = Bench(rx, rng, *shape, 64, [rows], [L])
    exact_scores(b, rng, lambda s: np.minimum(2.0 ** (exponent + rng.uniform(0, 1, s) - rng.integers(0, spread + 1, s)), 8160))
    q = (np.clip(np.rint(rng.standard_normal((rows, b.h, b.d)) * 5.2 * 4), -127, 127) / 4).astype(np.float16)
    got = b.attention(q).astype(np.float64)
    want, tol = narrow(q.astype(np.float64), b)
    over = np.abs(got - want) / tol
    assert (over <= 1).all(), (float(over.max()), np.sqrt((got - want).var() / want.var()))


@pytest.mark.parametrize("at", [0, 0.5, 1])
@pytest.mark.parametrize("exponent", [-13, -3])
@pytest.mark.parametrize("shape,rows,L", [((8, 1, 128), 1, 20001), ((16, 2, 64), 1, 9000), ((2, 2, 128), 4, 3000), ((4, 4, 64), 1, 700), ((8, 2, 128), 9, 3000)], ids=str)
def test_a_tail_of_small_weights(rx, shape, rows, L, exponent, at):  # noqa: F811
    """One token, whose value is zero, with 2^18 (heads of 64: 2^13) times the weight of each of the others: what they add up to comes out, although each is little."""
    h, g, d = shape
    b = Bench(rx, np.random.default_rng(seed_of(shape, at)), *shape, 64, [rows], [L])
    exact_scores(b, np.random.default_rng(1), lambda s: np.full(s, 2.0 ** exponent))
    pos = int(at * (L - rows))
    page, blk = b.pages[0, pos // 64], pos % 64 // 16
    for name, rest, mine in (("k", 8, 15), ("v", 15, 8)):
        b.pool[name][:] = rest * 17
        byte, shift = (x[pos % 16] for x in po.code_place(name, d))
        for half_ in (0, 4):
            where = byte[shift == half_]
            b.pool[name][page, :, blk][:, where] = (b.pool[name][page, :, blk][:, where] & (0xF0 if half_ == 0 else 0x0F)) | mine << half_
        b.dev[name].copy_(torch.from_numpy(b.pool[name]))
    for key in ("ks", "vs"):                                   # of one sign, so that the tail adds up
        b.pool[key] = np.abs(b.pool[key])
        b.dev[key].copy_(torch.from_numpy(b.pool[key]))
    q = np.full((rows, h, d), 1.25, np.float16)                # a score of 7 / 8 * 1.25 * sqrt d, the others 0
    got = b.attention(q).astype(np.float64)
    want, tol = narrow(q.astype(np.float64), b)
    over = np.abs(got - want) / tol
    assert np.abs(want).min() > 2.0 ** -20 and (over <= 1).all(), (float(over.max()), float(np.abs(got).max()), float(np.abs(want).min()))


@pytest.mark.parametrize("shape,rows", [((8, 1, 128), 1), ((4, 4, 64), 3), ((8, 2, 64), 5)], ids=str)
def test_scores_far_from_zero(rx, shape, rows):  # noqa: F811
    """Every score of a row is far below or above zero, up to 2^25: whatever the weights are held against stays a number.  (Beyond that fp32 tells scores apart by four and more.)"""
    h, g, d = shape
    for sign, size in ((-1, 100.0), (-1, 30000.0), (1, 30000.0)):
        for key_scale in (0.125, 8.0) + ((4096.0,) if size == 100.0 else ()):
            b = Bench(rx, np.random.default_rng(seed_of(shape)), *shape, 32, [rows], [900])
            rng = np.random.default_rng(5)
            exact_scores(b, rng, lambda s: np.full(s, 0.25))
            b.pool["k"][:] = 0x22                              # codes of 2: -6
            b.pool["ks"] = np.where(np.isnan(b.pool["ks"]), b.pool["ks"], np.float16(key_scale)).astype(np.float16)
            for key in ("k", "ks"):
                b.dev[key].copy_(torch.from_numpy(b.pool[key]))
            q = np.full((rows, h, d), -sign * size, np.float16)      # equal scores: the mean of the values
            got = b.attention(q).astype(np.float64)
            want, tol = narrow(q.astype(np.float64), b)
            assert (np.abs(got - want) <= tol).all(), (sign, size, key_scale)
