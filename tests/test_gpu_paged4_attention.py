"""Attention over the paged 4-bit KV cache where its tolerance can be narrow: scores that are exact in fp32, so that an output is held to a part of sum p |v| whatever the size of the values
and the length of the context."""
import numpy as np
import pytest

import paged4_oracle as po
from test_gpu_paged4 import Bench, half, rx, seed_of  # noqa: F401  (rx: the fixture)

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu


def exact_scores(b, rng, v_scale):
    """Key scales of +-1/8, so that with queries in multiples of 1/4 below 32 every product and sum of a score is exact; value scales v_scale(shape) of eight bits."""
    for key, make in (("ks", lambda shape: rng.choice([-0.125, 0.125], shape)), ("vs", lambda shape: v_scale(shape) * rng.choice([-1, 1], shape))):
        x = po.round8(make(b.pool[key].shape).astype(np.float32)).astype(np.float16)
        b.pool[key] = np.where(np.isnan(b.pool[key]), b.pool[key], x).astype(np.float16)
        b.dev[key].copy_(torch.from_numpy(b.pool[key]))


def narrow(q, b, rows=None, heads=None):
    """(out, tolerance), float64 [n, h, d], of the given rows of a sequence and heads (None: all; of others the tolerance is infinite).  What is rounded, each to nearest:
      the output to fp16                             2^-11 |o|, 2^-25 below fp16's normal range
      weights, or weights times scales, to fp16      2^-11 sum p |v|; with a sum of the rounded ones 2^-11 |o| more
      ... below fp16's normal range                  a step is 2^-24; the largest weight times the root of the sum of squares of a lane's scales, sixteen, is 2^12 at least, so times the largest of
                                                     them 2^10: 2^-35 of the largest p times scale, of a code of 8 at most, per token; many pairs: the largest weight is 2^11 at least: 2^-36
                                                     of the largest p |v| per token
      exponents                                      scores are exact; times c and minus the reference they are below 2^6 in size: c is off by 4 2^-24 of itself, the multiply-add by 2^-24, the
                                                     exponential by 2^-22 of itself: below 2^-15 of a weight, in numerator and denominator
      sums in fp32                                   a product of 32 tokens is off by 4 2^-24 of its terms, at most 23 |s| p each (codes 0..15 against -8 sum p s): T / 32 + 8 of them in a row"""
    out, tol = np.zeros(q.shape), np.full(q.shape, np.inf)
    rep = b.h // b.g
    for row, ql, L, slot in po.sequences(b.q_lens, b.kv_lens, b.slots):
        (kc, ks), (vc, vs) = (po.values(b.pool, name, b.pages, b.page_size, slot, np.arange(L), b.d) for name in "kv")
        for i in range(ql) if rows is None else rows:
            seen = L - ql + i + 1
            for head in range(b.h) if heads is None else heads:
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


@gpu
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


@gpu
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


@gpu
@pytest.mark.parametrize("shape,rows", [((8, 1, 128), 1), ((4, 4, 64), 3), ((8, 2, 64), 5)], ids=str)
def test_scores_far_from_zero(rx, shape, rows):  # noqa: F811
    """Every score of a row is far below or above zero, up to 2.8e7, where fp32 tells scores apart by two: whatever the weights are held against stays a number."""
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


def held(b, name, slot, L):
    """(values, scales) of one slot's first L tokens, float32 [g, L, d] on the GPU."""
    byte, shift = (torch.from_numpy(x).cuda() for x in po.code_place(name, b.d))
    pages = torch.from_numpy(b.pages[slot, :-(-L // b.page_size)]).cuda().long()
    u = (b.dev[name][pages][..., byte.flatten()].int() >> shift.flatten().int()) & 15            # [pages, g, blocks, 16 d]
    s = b.dev[name + "s"][pages][..., torch.from_numpy(po.scale_place(b.d)).cuda().flatten()]
    lead = u.shape[:3]
    s = s.view(*lead, 16, b.d // 32).repeat_interleave(32, dim=4).float()
    x = (u.view(*lead, 16, b.d).float() - 8) * s
    order = lambda y: y.permute(1, 0, 2, 3, 4).reshape(b.g, -1, b.d)[:, :L].contiguous()
    return order(x), order(s)


def misses(out, v, s, mass):
    """Where an output is not the value it has to be.  One token has all the weight but `mass`: what is rounded is its weight, or weight times scale, and the output, 2^-11 each, 2^-25 below
    fp16's normal range, sums in fp32 of few terms that are not zero, below 2^-17 of a scale; and the others' values, 8 scales at most, on either side."""
    return (out - v).abs() > 2.0 ** -10 * v.abs() + 2.0 ** -25 + (2.0 ** -17 + 16.0 * mass) * s.amax()


EVERY = {  # (heads, KV heads, d), q_lens, kv_lens
    "long": ((64, 8, 128), [1], [120001]), "long_4": ((8, 2, 64), [2], [30011]), "drafts": ((64, 8, 128), [3], [30011]), "tiles": ((16, 2, 64), [7, 1], [9000, 700]),
    "ungrouped": ((40, 40, 128), [1], [3001]), "ragged": ((16, 2, 64), [1] * 7, [40, 3000, 1, 700, 16, 9000, 129]), "chunk": ((8, 1, 128), [40, 3], [5000, 1030]),
    "rows": ((200, 200, 64), [256], [8200]), "short": ((32, 32, 64), [1] * 70, [100 + 3 * i for i in range(70)]),
}


@gpu
@pytest.mark.parametrize("device_table", [False, True])
@pytest.mark.parametrize("kind", sorted(EVERY))
def test_every_token_counts(rx, kind, device_table):  # noqa: F811
    """For every token of every sequence and KV head a query that gives it all the weight, in the context's length and cut of the call: the answer is its value, at the first token and the last one and on
    either side of every border of steps, wavefronts, parts and lookups.  A lost token is an answer from another."""
    shape, q_lens, kv_lens = EVERY[kind]
    rng = np.random.default_rng(seed_of(kind))
    slots = [int(x) for x in rng.permutation(len(q_lens))]
    b = Bench(rx, rng, *shape, 64, q_lens, kv_lens, slots, device_table=device_table)
    exact_scores(b, rng, lambda s_: np.full(s_, 2.0 ** -11))
    h, g, d = shape
    rep = h // g
    seqs, (ws, ws_bytes) = b.seqs(), b.workspace()
    kv = [[held(b, name, slot, L) for name in "kv"] for slot, L in zip(slots, kv_lens)]
    starts = np.concatenate([[0], np.cumsum(q_lens)])
    calls = max(-(-L // (ql * rep)) for ql, L in zip(q_lens, kv_lens)) + 1
    chosen = []                                                # [calls, rows, rep]: the token of a row and head of the group, at most the row's own
    for ql, L in zip(q_lens, kv_lens):
        at = torch.arange(calls * ql * rep, device="cuda").view(calls, ql, rep)
        chosen.append(torch.minimum(at, torch.arange(L - ql, L, device="cuda")[None, :, None]))
        assert len(torch.unique(chosen[-1])) == L
    mass = 0.0                                                 # of all other tokens, at most: a score is 64 |k|^2 / sqrt d and theirs are 64 k . k' / sqrt d, exact in fp32
    for (k, _), _ in kv:
        for j in range(g):
            for first in range(0, k.shape[1], 8192):
                s = k[j, first:first + 8192] @ k[j].t().contiguous() * (64 / d ** 0.5)
                mine = s[torch.arange(s.shape[0]), first + torch.arange(s.shape[0])].clone()
                s[torch.arange(s.shape[0]), first + torch.arange(s.shape[0])] = -float("inf")
                mass = max(mass, float((s - mine[:, None]).exp_().sum(dim=1).max()))
    assert mass < 2.0 ** -12, mass
    step, wrong = max(1, (1 << 28) // (b.n * h * d)), 0
    for lo in range(0, calls, step):
        hi = min(calls, lo + step)
        q = torch.empty((hi - lo, b.n, g, rep, d), dtype=torch.float16, device="cuda")
        for i, ((k, _), _) in enumerate(kv):
            q[:, starts[i]:starts[i + 1]] = (64 * k[:, chosen[i][lo:hi]]).permute(1, 2, 0, 3, 4).half()
        out = torch.full_like(q, float("nan"))
        for c in range(hi - lo):
            rx.check(rx.relax_paged4_attention(q[c], b.cache, seqs, b.dims, out[c], b.n, ws, ws_bytes))
        for i, (_, (v, s)) in enumerate(kv):
            want = v[:, chosen[i][lo:hi]].permute(1, 2, 0, 3, 4)
            wrong += int(misses(out[:, starts[i]:starts[i + 1]].float(), want, s, mass).any(dim=4).sum()) + int(out[:, starts[i]:starts[i + 1]].isnan().sum())
        del q, out
    assert wrong == 0 and b.error() == 0


ONCE = {
    "few": ((64, 8, 128), [1], [3001]), "few_4": ((8, 2, 64), [2], [2500]), "drafts": ((64, 8, 128), [3], [30011]), "tiles": ((16, 2, 64), [7, 1], [9000, 700]),
    "ungrouped": ((40, 40, 128), [1], [3001]), "ragged": ((16, 2, 64), [1] * 7, [40, 3000, 1, 700, 16, 2900, 129]), "chunk": ((8, 1, 128), [40, 3], [5000, 1030]),
    "rows": ((200, 200, 64), [256], [8200]), "short": ((32, 32, 64), [1] * 70, [100 + 3 * i for i in range(70)]),
}


@gpu
@pytest.mark.parametrize("device_table", [False, True])
@pytest.mark.parametrize("kind", sorted(ONCE))
def test_every_token_counts_once(rx, kind, device_table):  # noqa: F811
    """Equal scores, and of each element of a head one token alone whose value is not zero: its part of the sum.  A token that two wavefronts or parts count is twice that.
    The product of weight and scale, the weight in the denominator and the output are rounded, 3 times 2^-11; sums in fp32 as in narrow()."""
    shape, q_lens, kv_lens = ONCE[kind]
    rng = np.random.default_rng(seed_of(kind))
    slots = [int(x) for x in rng.permutation(len(q_lens))]
    b = Bench(rx, rng, *shape, 64, q_lens, kv_lens, slots, device_table=device_table)
    exact_scores(b, rng, lambda s_: np.full(s_, 512.0))
    b.pool["vs"] = np.abs(b.pool["vs"])
    b.dev["vs"].copy_(torch.from_numpy(b.pool["vs"]))
    h, g, d = shape
    rep = h // g
    seqs, (ws, ws_bytes) = b.seqs(), b.workspace()
    byte, shift = (torch.from_numpy(x).cuda() for x in po.code_place("v", d))
    q, wrong = torch.zeros((b.n, h, d), dtype=torch.float16, device="cuda"), 0
    starts = np.concatenate([[0], np.cumsum(q_lens)])
    for call in range(-(-max(kv_lens) // (g * d))):
        b.dev["v"].fill_(0x88)
        token = ((call * g + torch.arange(g, device="cuda"))[:, None] * d + torch.arange(d, device="cuda")).expand(g, d)
        for slot, L in zip(slots, kv_lens):
            j, e = torch.nonzero(token < L, as_tuple=True)
            t = token[j, e]
            page, at, sh = torch.from_numpy(b.pages[slot]).cuda().long()[t // 64], byte[t % 16, e], shift[t % 16, e]
            b.dev["v"][page, j, t % 64 // 16, at] = torch.where(sh == 0, 0x8F, 0xF8).to(torch.uint8)
        out = torch.full_like(q, float("nan"))
        rx.check(rx.relax_paged4_attention(q, b.cache, seqs, b.dims, out, b.n, ws, ws_bytes))
        for i, (ql, L) in enumerate(zip(q_lens, kv_lens)):
            vis = torch.arange(L - ql, L, device="cuda")[:, None, None] + 1
            want = torch.where(token < vis, 7 * 512.0 / vis, 0.0)[:, :, None]              # [rows, g, 1, d]
            got = out[starts[i]:starts[i + 1]].view(ql, g, rep, d).float()
            few = 1 <= ql * rep % 32 <= 8                      # a tile of codes 0..15 against -8 sum p s: sums of 512 scales, whose terms cancel but for one
            tol = 3 * 2.0 ** -11 * want + (L / 32 + 8) * 4 * 2.0 ** -24 * (23 * 512.0 if few else want)
            assert bool((tol[want > 0] < want[want > 0] / 2).all())
            wrong += int((~((got - want).abs() <= tol)).sum())
    assert wrong == 0 and b.error() == 0


def test_a_lost_token_is_a_miss():
    """The check above on an oracle that leaves a token out: its answer is another token's value, which differs by codes, many tolerances."""
    torch.manual_seed(3)
    u, s = torch.randint(0, 16, (500, 64)), torch.full((500, 64), 2.0 ** -11)
    v = (u - 8) * s
    assert not misses(v.half().float(), v, s, 2.0 ** -12).any()
    assert misses(v.roll(1, 0).half().float(), v, s, 2.0 ** -12).any(dim=1).all() and misses(torch.zeros_like(v), v, s, 2.0 ** -12).any(dim=1).all()


@gpu
@pytest.mark.parametrize("size,rising", [(96.0, False), (30000.0, False), (96.0, True), (30000.0, True)])
@pytest.mark.parametrize("shape,rows,L", [((8, 1, 128), 1, 9000), ((8, 1, 128), 3, 9000), ((4, 4, 64), 9, 2000), ((2, 1, 128), 30, 2000), ((100, 100, 128), 257, 1000)], ids=str)
def test_large_scores_that_differ_little(rx, shape, rows, L, size, rising):  # noqa: F811
    """Scores of 600 to 250000 that differ by some units from token to token, exact in fp32: wavefronts and parts, whose references differ, agree on the weights, and so does a row whose reference moves."""
    h, g, d = shape
    rng = np.random.default_rng(seed_of(shape, rows, L))
    b = Bench(rx, rng, *shape, 64, [rows], [L])
    exact_scores(b, rng, lambda s: np.full(s, 0.25))
    b.pool["k"][:] = 0xEE                                      # codes of 14: 6 / 8
    codes = 16 * np.arange(L) // L if rising else rng.integers(0, 16, L)      # of element 5, which makes the difference
    byte, shift = po.code_place("k", d)
    for pos in range(L):
        at = b.pool["k"][b.pages[0, pos // 64], :, pos % 64 // 16]
        t = pos % 16
        at[:, byte[t, 5]] = (at[:, byte[t, 5]] & (0xF0 if shift[t, 5] == 0 else 0x0F)) | codes[pos] << shift[t, 5]
    b.pool["ks"] = np.abs(b.pool["ks"])
    for key in ("k", "ks"):
        b.dev[key].copy_(torch.from_numpy(b.pool[key]))
    q = np.full((rows, h, d), size, np.float16)
    q[:, :, 5] = 64
    got = b.attention(q).astype(np.float64)
    want, tol = narrow(q.astype(np.float64), b, sorted({0, rows // 2, rows - 1}), sorted({0, h - 1}))
    over = np.abs(got - want) / tol
    assert (over <= 1).all(), float(over.max())
