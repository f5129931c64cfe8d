"""Heads before attention, scaled rotary tables and the paged 4-bit KV cache on the GPU against their definitions in numpy (paged4_oracle.py), at the sizes,
layouts and page tables where they can go wrong.  What the definition rounds is compared bit by bit, attention with a derived tolerance."""
import zlib

import numpy as np
import pytest

import paged4_oracle as po
import paged_oracle as po8

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

SHAPES = [(4, 4, 64), (32, 32, 128), (8, 2, 64), (16, 2, 128), (6, 2, 128), (40, 2, 64), (7, 1, 128), (10, 5, 64)]
EPS = 2.0 ** -17


@pytest.fixture(scope="module")
def rx():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2311_02103_amd import binding
    binding.lib()
    return binding


def seed_of(*what):
    return zlib.crc32(repr(what).encode()) % 100000


def half(rng, shape, std=1.0):
    return (rng.standard_normal(shape) * std).astype(np.float16)


def same_bits(a, b):
    return np.array_equal(np.ascontiguousarray(a).view(np.uint8), np.ascontiguousarray(b).view(np.uint8))


class Prep:
    """Norm weights and a rotary table on both sides."""

    def __init__(self, rx, rng, d, cap, norm=(True, True), rotary=None, pairs=False, rope=True, eps=EPS, base=10000.0):
        self.R, self.pairs, self.eps = rotary or d, pairs, eps
        self.w = [half(rng, d, 0.2) + np.float16(1) if n else None for n in norm]
        self.dev_w = [None if w is None else torch.from_numpy(w).cuda() for w in self.w]
        self.table, self.host = None, None
        if rope:
            self.table = torch.empty((cap, self.R // 2, 2), dtype=torch.float32, device="cuda")
            rx.check(rx.relax_rope_table_scaled(rx.RopeScaling(rx.ROPE_PLAIN, self.R, base, 1.0, 0.0, 0.0, 0.0, 0.0), cap, self.table))
            torch.cuda.synchronize()
            self.host = self.table.cpu().numpy()
        self.c = rx.HeadPrep(*self.dev_w, eps, self.table, rotary or 0, rx.ROPE_PAIRS if pairs else rx.ROPE_HALVES)

    def heads(self, x, pos, which):
        """x float [n, heads, d] at positions, which: 0 queries, 1 keys; float32."""
        w = self.w[which]
        with np.errstate(invalid="ignore", over="ignore"):
            return po.prepare(x.astype(np.float32), None if w is None else w.astype(np.float32), self.eps, None if self.host is None else self.host[pos][:, None], self.R, self.pairs)


def positions(q_lens, kv_lens):
    return np.concatenate([np.arange(L - ql, L) for ql, L in zip(q_lens, kv_lens)])


class Bench:
    """A pool with random contents, its device copy, and the calls on it.  The scales of positions that no sequence has reached are NaN."""

    def __init__(self, rx, rng, h, g, d, page_size, q_lens, kv_lens, slots=None, prep=None, spare=2, device_table=False, scale=(0.02, 0.3), table_slack=40):
        self.rx, self.h, self.g, self.d, self.page_size = rx, h, g, d, page_size
        self.q_lens, self.kv_lens, self.slots, self.table_slack = q_lens, kv_lens, slots, table_slack
        self.n = sum(q_lens)
        n_slots = len(q_lens) if slots is None else max(slots) + 2
        self.per = max(-(-L // page_size) for L in kv_lens)
        used = [(i if slots is None else slots[i], -(-L // page_size)) for i, L in enumerate(kv_lens)]
        n_pages = sum(c for _, c in used) + spare
        order = rng.permutation(n_pages)
        self.pages = np.full((n_slots, self.per), -7, np.int32)       # entries that no sequence reaches name no page
        at = 0
        for slot, count in used:
            self.pages[slot, :count] = order[at:at + count]
            at += count
        blocks = page_size // 16
        self.pool = {}
        for name in "kv":
            self.pool[name] = rng.integers(0, 256, (n_pages, g, blocks, 8 * d)).astype(np.uint8)
            s = po.round8(rng.uniform(*scale, (n_pages, g, blocks, d // 2)).astype(np.float32) * rng.choice([-1, 1], (n_pages, g, blocks, d // 2)).astype(np.float32))
            s = s.astype(np.float16)
            held = np.full_like(s, np.nan)
            for slot, L in zip([u for u, _ in used], kv_lens):
                for pos in range(L):
                    where = (self.pages[slot, pos // page_size], slice(None), pos % page_size // 16)
                    held[where][:, po.scale_place(d)[pos % 16]] = s[where][:, po.scale_place(d)[pos % 16]]
            self.pool[name + "s"] = held
        self.cap = self.per * page_size
        self.dims = rx.make_dims(h * d, h, g, d, 64, self.cap, n_slots)
        self.dev = {key: torch.from_numpy(x.copy()).cuda() for key, x in self.pool.items()}
        self.dev_pages = torch.from_numpy(self.pages.copy()).cuda()
        self.cache = rx.Paged4Cache(self.dev["k"], self.dev["v"], self.dev["ks"], self.dev["vs"], self.dev_pages, n_pages, page_size, self.per)
        self.prep = Prep(rx, rng, d, self.cap, **prep) if isinstance(prep, dict) else prep
        self.ws_bytes = rx.relax_paged4_workspace_bytes(self.dims, self.n, max(kv_lens), len(q_lens))
        self.ws = torch.full((self.ws_bytes,), 0xFF, dtype=torch.uint8, device="cuda")
        rx.check(rx.relax_workspace_init(self.dims, self.ws, self.ws_bytes))
        self.dev_table = None
        if device_table:
            starts = np.concatenate([[0], np.cumsum(q_lens)[:-1]])
            rows = np.stack([starts, q_lens, kv_lens, np.arange(len(q_lens)) if slots is None else slots]).astype(np.int32)
            self.dev_table = torch.from_numpy(rows).cuda()

    def seqs(self):
        kv = self.kv_lens if self.dev_table is None else [min(self.cap, L + self.table_slack) for L in self.kv_lens]      # upper bounds
        return self.rx.Seqs(self.q_lens, kv, self.slots, self.dev_table)

    def workspace(self):
        bound = self.rx.relax_paged4_workspace_bytes(self.dims, self.n, self.cap, len(self.q_lens))
        if bound > self.ws_bytes:
            self.ws, self.ws_bytes = torch.full((bound,), 0xFF, dtype=torch.uint8, device="cuda"), bound
            self.rx.check(self.rx.relax_workspace_init(self.dims, self.ws, self.ws_bytes))
        return self.ws, self.ws_bytes

    def append(self, qkv, q=True, stream=None):
        """qkv: host fp16 [n, (h + 2 g) d]."""
        x = torch.from_numpy(qkv).cuda()
        base, row = x.data_ptr(), x.shape[1]
        q_out = torch.full((self.n, self.h, self.d), float("nan"), dtype=torch.float16, device="cuda") if q else None
        self.rx.check(self.rx.relax_paged4_append(base if q else None, row, base + 2 * self.h * self.d, base + 2 * (self.h + self.g) * self.d, row, q_out,
                                                  None if self.prep is None else self.prep.c, self.cache, self.seqs(), self.dims, self.n, *self.workspace(), stream))
        torch.cuda.synchronize()
        return q_out.cpu().numpy() if q else None

    def attention(self, q, stream=None):
        qd = torch.from_numpy(q).cuda()
        out = torch.full(qd.shape, float("nan"), dtype=torch.float16, device="cuda")
        self.rx.check(self.rx.relax_paged4_attention(qd, self.cache, self.seqs(), self.dims, out, self.n, *self.workspace(), stream))
        torch.cuda.synchronize()
        return out.cpu().numpy()

    def read(self):
        out = torch.full((2, self.n, self.g, self.d), float("nan"), dtype=torch.float16, device="cuda")
        self.rx.check(self.rx.relax_paged4_read(self.cache, self.seqs(), self.dims, out[0], out[1], self.n, *self.workspace()))
        torch.cuda.synchronize()
        return out.cpu().numpy()

    def host_pool(self):
        return {key: x.cpu().numpy() for key, x in self.dev.items()}

    def error(self):
        return self.rx.relax_workspace_error(self.dims, self.ws)

    def clear(self):
        self.rx.check(self.rx.relax_workspace_init(self.dims, self.ws, self.ws_bytes))


def check_append(b, qkv, q_out):
    """The whole pool and q, bit by bit."""
    h, g, d = b.h, b.g, b.d
    x = qkv.reshape(b.n, h + 2 * g, d)
    pos = positions(b.q_lens, b.kv_lens)
    prepare = (lambda y, which: y.astype(np.float32)) if b.prep is None else (lambda y, which: b.prep.heads(y, pos, which))
    if q_out is not None:
        with np.errstate(over="ignore"):
            assert same_bits(q_out, prepare(x[:, :h], 0).astype(np.float16))
    kept = po8.storable(x[:, h:].astype(np.float32)).astype(np.float32)
    want = po.append(b.pool, b.pages, b.page_size, prepare(kept[:, :g], 1), kept[:, g:], b.q_lens, b.kv_lens, b.slots)
    got = b.host_pool()
    for key in want:
        assert same_bits(got[key], want[key]), key
    return want


LENS = [
    ([1], [1]), ([1], [2231]), ([1], [16]), ([1], [17]), ([5], [5]), ([16], [16]), ([17], [40]), ([33], [300]),
    ([1, 1, 1], [1, 32, 77]), ([3, 1, 40, 2], [3, 100, 41, 18]), ([2, 2, 2], [17, 33, 16]),
]
lens_id = lambda v: "x".join(map(str, v[0])) + "_of_" + "x".join(map(str, v[1]))      # noqa: E731
PREPS = [None, dict(), dict(norm=(False, False)), dict(pairs=True), dict(norm=(False, True), rotary=16), dict(norm=(True, False), rotary=48, pairs=True),
         dict(rotary=32), dict(rope=False)]


# ---- rotary tables --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("scaling", ["plain", "linear", "index", "wavelength"])
@pytest.mark.parametrize("R,positions", [(2, 1), (16, 63), (64, 64), (96, 65), (128, 4097), (256, 131), (128, 131072)])
def test_rotary_tables(rx, scaling, R, positions):
    """Against 64 bits.  An entry is off by its rounding to fp32, 2^-25 of an amplitude below 2 (a step of 2^-24 below it), and by 64-bit arithmetic: a frequency
    within 2^-50 (exp, ramp) times a position below 2^17, an angle's rounding 2^-36 at most, and sums of angles: below 2^-31 in all."""
    kind = {"plain": rx.ROPE_PLAIN, "linear": rx.ROPE_LINEAR, "index": rx.ROPE_INDEX_RAMP, "wavelength": rx.ROPE_WAVELENGTH_RAMP}[scaling]
    for base, factor, trained, slow, fast, amplitude in ((10000.0, 4.0, 2048.0, 1.0, 32.0, 0.0), (500000.0, 7.25, 8192.0, 1.0, 4.0, 1.25), (1.5, 0.5, 1.0, 0.01, 0.02, 1.0),
                                                         (10000.0, 32.0, 64.0, 500.0, 1000.0, 1.9)):
        table = torch.full((positions + 1, R // 2, 2), float("nan"), dtype=torch.float32, device="cuda")
        rx.check(rx.relax_rope_table_scaled(rx.RopeScaling(kind, R, base, factor, trained, slow, fast, amplitude), positions, table))
        got = table.cpu().numpy().astype(np.float64)
        assert np.isnan(got[positions:]).all()
        angle = np.arange(positions)[:, None] * po.frequencies(R, base, scaling, factor, trained, slow, fast)
        want = (amplitude or 1.0) * np.stack([np.cos(angle), np.sin(angle)], axis=2)
        assert np.abs(got[:positions] - want).max() <= 2.0 ** -25 * max(1.0, 2.0 * (amplitude > 1.0)) + 2.0 ** -31


def test_a_plain_table_is_the_layers(rx):
    dims = rx.make_dims(128, 2, 2, 64, 64, 300, 1, rope_base=10000.0)
    a, b = (torch.empty((300, 32, 2), dtype=torch.float32, device="cuda") for _ in "ab")
    rx.check(rx.relax_rope_table_init(dims, a))
    rx.check(rx.relax_rope_table_scaled(rx.RopeScaling(rx.ROPE_PLAIN, 64, 10000.0, 0.0, 0.0, 0.0, 0.0, 0.0), 300, b))
    torch.cuda.synchronize()
    assert float((a - b).abs().max()) <= 2.0 ** -24


# ---- heads ----------------------------------------------------------------------------------------------------------
class Heads:
    def __init__(self, rx, rng, h, g, d, q_lens, kv_lens, prep, device_table=False, cap=None):
        self.rx, self.h, self.g, self.d, self.q_lens, self.kv_lens, self.n = rx, h, g, d, q_lens, kv_lens, sum(q_lens)
        self.cap = cap or max(kv_lens)
        self.prep = Prep(rx, rng, d, self.cap, **prep)
        self.dims = rx.make_dims(h * d, h, g, d, 64, self.cap, len(q_lens))
        self.ws_bytes = rx.relax_head_workspace_bytes(self.dims, len(q_lens))
        self.ws = torch.full((self.ws_bytes,), 0xFF, dtype=torch.uint8, device="cuda")
        rx.check(rx.relax_workspace_init(self.dims, self.ws, self.ws_bytes))
        self.table = None
        if device_table:
            starts = np.concatenate([[0], np.cumsum(q_lens)[:-1]])
            self.table = torch.from_numpy(np.stack([starts, q_lens, kv_lens, np.arange(len(q_lens))]).astype(np.int32)).cuda()

    def seqs(self):
        return self.rx.Seqs(self.q_lens, self.kv_lens if self.table is None else [self.cap] * len(self.q_lens), None, self.table)

    def run(self, x, which="qk", gap=0, stream=None):
        """x host fp16 [n, (h + g) d] -> outputs with `gap` elements between rows, filled with NaN in front."""
        h, g, d = self.h, self.g, self.d
        xd = torch.from_numpy(x).cuda()
        outs = [torch.full((self.n, w * d + gap), float("nan"), dtype=torch.float16, device="cuda") for w in (h, g)]
        q, k = ("q" in which), ("k" in which)
        at, row = xd.data_ptr(), x.shape[1]
        self.rx.check(self.rx.relax_head_norm_rope(at if q else None, row, at + 2 * h * d if k else None, row, outs[0] if q else None, h * d + gap, outs[1] if k else None, g * d + gap,
                                                   self.prep.c, self.seqs(), self.dims, self.n, self.ws, self.ws_bytes, stream))
        torch.cuda.synchronize()
        return [o.cpu().numpy() for o in outs]

    def want(self, x):
        pos = positions(self.q_lens, self.kv_lens)
        y = x.reshape(self.n, self.h + self.g, self.d)
        with np.errstate(over="ignore", invalid="ignore"):
            return [self.prep.heads(z, pos, i).astype(np.float16).reshape(self.n, -1) for i, z in enumerate((y[:, :self.h], y[:, self.h:]))]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("prep", PREPS[1:], ids=str)
def test_heads(rx, shape, prep):
    for lens in (([1], [1]), ([1], [1000]), ([70], [75]), ([1] * 5, [3, 1, 9, 40, 2]), ([3, 1, 40, 2], [3, 100, 41, 18])):
        rng = np.random.default_rng(seed_of(shape, prep, lens))
        t = Heads(rx, rng, *shape, *lens, prep)
        x = half(rng, (t.n, (t.h + t.g) * t.d), 3.0)
        for got, want in zip(t.run(x), t.want(x)):
            assert same_bits(got, want)


@pytest.mark.parametrize("count", [17, 129, 300])
@pytest.mark.parametrize("device_table", [False, True])
def test_heads_of_many_sequences(rx, count, device_table):
    rng = np.random.default_rng(count)
    q_lens = [1 if count == 129 else int(rng.integers(1, 9)) for _ in range(count)]
    t = Heads(rx, rng, 6, 2, 64, q_lens, [q + int(rng.integers(0, 50)) for q in q_lens], dict(), device_table, cap=70)
    x = half(rng, (t.n, 8 * 64))
    for got, want in zip(t.run(x), t.want(x)):
        assert same_bits(got, want)


def test_heads_one_side_gaps_and_in_place(rx):
    rng = np.random.default_rng(11)
    t = Heads(rx, rng, 8, 2, 128, [20, 3], [30, 9], dict(rotary=64))
    x = half(rng, (23, 10 * 128))
    want = t.want(x)
    q, k = t.run(x, gap=24)
    assert same_bits(q[:, :1024], want[0]) and same_bits(k[:, :256], want[1]) and np.isnan(q[:, 1024:]).all() and np.isnan(k[:, 256:]).all()
    q, k = t.run(x, "q")
    assert same_bits(q, want[0]) and np.isnan(k).all()
    q, k = t.run(x, "k")
    assert same_bits(k, want[1]) and np.isnan(q).all()
    xd = torch.from_numpy(x).cuda()                            # in place, in a matrix of both
    at = xd.data_ptr()
    rx.check(rx.relax_head_norm_rope(at, 1280, at + 2048, 1280, at, 1280, at + 2048, 1280, t.prep.c, t.seqs(), t.dims, 23, t.ws, t.ws_bytes))
    torch.cuda.synchronize()
    got = xd.cpu().numpy()
    assert same_bits(got[:, :1024], want[0]) and same_bits(got[:, 1024:], want[1])


def test_heads_that_are_not_finite_or_zero(rx):
    rng = np.random.default_rng(12)
    for prep in (dict(eps=0.0), dict(norm=(False, False), pairs=True, rotary=32)):
        t = Heads(rx, rng, 4, 2, 64, [6], [6], prep)
        x = half(rng, (6, 6 * 64))
        x[0, :64], x[1, 3], x[2, 70], x[3, 300], x[4, 64:128] = 0, np.inf, np.nan, -np.inf, 65504
        x[5] = np.float16(6e-8)
        got, want = t.run(x), t.want(x)
        for a, b in zip(got, want):
            nan = np.isnan(b)
            assert np.array_equal(np.isnan(a), nan) and np.array_equal(a[~nan], b[~nan])
        assert (got[0][0, :64] == 0).all()


@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1e-30, 1.0, 3.4e38])
def test_heads_with_any_eps(rx, eps):
    """Heads of zeros, whose factor is that of eps alone, and of ordinary and of the smallest numbers."""
    rng = np.random.default_rng(14)
    t = Heads(rx, rng, 4, 2, 128, [4], [9], dict(eps=eps))
    x = half(rng, (4, 6 * 128))
    x[0], x[1, :128], x[2, :256] = 0, 0, np.float16(6e-8)
    for got, want in zip(t.run(x), t.want(x)):
        assert same_bits(got, want)


def test_heads_beyond_the_capacity(rx):
    """A device table's positions outside the table of angles: the nearest row, and the flag."""
    rng = np.random.default_rng(13)
    t = Heads(rx, rng, 4, 2, 64, [2, 1, 3, 1], [10, 20, 7, 5], dict(), True, cap=32)
    x = half(rng, (7, 6 * 64))
    assert all(same_bits(a, b) for a, b in zip(t.run(x), t.want(x))) and rx.relax_workspace_error(t.dims, t.ws) == 0
    for bad, at in ((33, 31), (1 << 30, 31), ((1 << 31) - 1, 31), (-1, 0), (-(1 << 31), 0)):
        t.table[2, 1] = bad
        rx.check(rx.relax_workspace_init(t.dims, t.ws, t.ws_bytes))
        got = t.run(x)
        assert rx.relax_workspace_error(t.dims, t.ws) == 4
        keep = t.kv_lens
        t.kv_lens = [10, at + 1, 7, 5]
        assert all(same_bits(a, b) for a, b in zip(got, t.want(x)))
        t.kv_lens = keep


# ---- append and read ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("lens", LENS, ids=lens_id)
def test_append_and_read(rx, shape, lens):
    rng = np.random.default_rng(seed_of(shape, lens))
    page_size = [16, 32, 64, 128, 256][(shape[0] + sum(lens[1])) % 5]
    b = Bench(rx, rng, *shape, page_size, *lens, prep=PREPS[seed_of(lens, shape) % len(PREPS)])
    qkv = half(rng, (b.n, (b.h + 2 * b.g) * b.d), std=3.0)
    pool = check_append(b, qkv, b.append(qkv))
    assert b.error() == 0
    k, v = b.read()
    for row, ql, L, slot in po8.sequences(b.q_lens, b.kv_lens, b.slots):
        for name, got in (("k", k), ("v", v)):
            c, s = po.values(pool, name, b.pages, page_size, slot, np.arange(L - ql, L), b.d)
            assert np.array_equal(got[row:row + ql].astype(np.float64), c * s), name      # exact


@pytest.mark.parametrize("prep", PREPS, ids=str)
@pytest.mark.parametrize("shape", [(8, 2, 64), (6, 3, 128)], ids=str)
def test_append_prepares_heads(rx, shape, prep):
    for lens in (([1], [30]), ([50, 1, 2], [55, 9, 2])):
        rng = np.random.default_rng(seed_of(shape, prep, lens))
        b = Bench(rx, rng, *shape, 16, *lens, prep=prep)
        qkv = half(rng, (b.n, (b.h + 2 * b.g) * b.d), std=2.0)
        check_append(b, qkv, b.append(qkv))


@pytest.mark.parametrize("count", [17, 64, 200])
@pytest.mark.parametrize("device_table", [False, True])
def test_append_of_many_sequences(rx, count, device_table):
    rng = np.random.default_rng(count)
    q_lens = [1 if count == 64 else int(rng.integers(1, 20)) for _ in range(count)]
    kv_lens = [q + int(rng.integers(0, 60)) for q in q_lens]
    slots = [int(s) for s in rng.permutation(count + 3)[:count]]
    b = Bench(rx, rng, 8, 2, 64, 32, q_lens, kv_lens, slots, prep=dict(), device_table=device_table)
    qkv = half(rng, (b.n, 12 * 64))
    check_append(b, qkv, b.append(qkv))
    assert b.error() == 0


def test_a_long_append(rx):
    """More wavefronts than are launched one head each: several KV heads per wavefront."""
    for shape in ((40, 40, 64), (9, 9, 128)):
        rng = np.random.default_rng(31)
        b = Bench(rx, rng, *shape, 256, [1001, 1002], [1004, 1002], prep=dict(norm=(False, True)))
        qkv = half(rng, (b.n, (b.h + 2 * b.g) * b.d))
        check_append(b, qkv, b.append(qkv))


def test_append_without_queries_and_from_matrices_of_their_own(rx):
    """q and q_out NULL; and k, v rows of their own strides, q in place."""
    benches = [Bench(rx, np.random.default_rng(5), 8, 4, 128, 64, [20, 3], [37, 9], prep=dict()) for _ in range(2)]
    qkv = half(np.random.default_rng(6), (23, 16 * 128))
    benches[0].append(qkv, q=False)
    check_append(benches[0], qkv, None)
    b = benches[1]
    x = torch.from_numpy(qkv).cuda()
    k = torch.full((b.n, 4 * 128 + 24), float("nan"), dtype=torch.float16, device="cuda")
    v = k.clone()
    k[:, :512], v[:, :512] = x[:, 1024:1536], x[:, 1536:]
    q = x[:, :1024].contiguous()
    rx.check(rx.relax_paged4_append(q, 1024, k, v, 536, q, b.prep.c, b.cache, b.seqs(), b.dims, b.n, *b.workspace()))      # q_out is q
    torch.cuda.synchronize()
    check_append(b, qkv, q.cpu().numpy().reshape(b.n, 8, 128))


def test_values_that_are_not_finite_tiny_or_large(rx):
    rng = np.random.default_rng(3)
    b = Bench(rx, rng, 4, 4, 64, 16, [20], [20])
    qkv = half(rng, (20, 12 * 64))
    qkv[3, 256], qkv[3, 520], qkv[18, 300], qkv[18, 600] = np.inf, -np.inf, np.nan, np.nan
    qkv[5, 256:512] = np.float16(6e-8)                         # 2^-24: scales below the smallest fp16 number
    qkv[6, 256:512] = half(rng, 256, 1e-6)
    qkv[7, 512:576], qkv[8, 512:576] = 65504, -65504
    qkv[9, 512:576] = np.where(np.arange(64) % 2, 60000, -60000)
    qkv[10, 512:768] = 0
    qkv[11, 512:768] = np.where(np.arange(256) % 3, 1.5, -1.5)      # two of the largest magnitude: the positive one leads
    check_append(b, qkv, b.append(qkv))
    assert np.isfinite(b.attention(half(rng, (20, 4, 64)))).all()
    k, v = b.read()
    assert np.isfinite(k).all() and (k[5] == 0).all() and (v[10] == 0).all()
    assert v[7, 0].max() == v[7, 0].min() == 65280 and v[8, 0].max() == v[8, 0].min() == -65280
    assert v[11].max() == 1.5 and v[11].min() == -1.3125


def test_quantisation_at_every_border(rx):
    """Every fp16 number of a binade against scales of eight bits, the quotients' ties among them: codes as the correctly rounded division has them."""
    g, d, n = 16, 128, 512
    b = Bench(rx, np.random.default_rng(1), g, g, d, 64, [n], [n])
    rng = np.random.default_rng(2)
    x = np.zeros((n, 3 * g, d), np.float16)
    kv = x[:, g:].reshape(n * 2 * g, d // 32, 32)
    top = rng.uniform(1, 2, kv.shape[:2]).astype(np.float16)
    steps = po.round8(top.astype(np.float32) / np.float32(-8)).astype(np.float64)[..., None]
    kv[:] = ((rng.integers(-8, 8, kv.shape) + 0.5) * steps).astype(np.float16)      # ties, where fp16 has them, and next to them
    kv[:, :, 1:8] = np.nextafter(kv[:, :, 1:8], np.float16(0))
    kv[:, :, 8:16] = np.nextafter(kv[:, :, 8:16], np.float16(4))
    kv[:, :, 16:24] = rng.uniform(-1, 1, (*kv.shape[:2], 8)).astype(np.float16) * top[..., None]
    kv[:, :, 0] = top
    qkv = x.reshape(n, -1)
    check_append(b, qkv, b.append(qkv))


# ---- attention ------------------------------------------------------------------------------------------------------
def attention_case(rx, rng, shape, page_size, q_lens, kv_lens, slots=None, std=1.0, device_table=False, scale=(0.02, 0.3), edit=None, heads=None):
    b = Bench(rx, rng, *shape, page_size, q_lens, kv_lens, slots, device_table=device_table, scale=scale)
    if edit:
        edit(b)
    q = half(rng, (b.n, b.h, b.d), std)
    got = b.attention(q).astype(np.float64)
    want, tol = po.attention(q.astype(np.float64), b.pool, b.pages, page_size, q_lens, kv_lens, slots, b.g, b.d, heads)
    if heads is not None:
        got, want, tol = got[:, heads], want[:, heads], tol[:, heads]
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.abs(got - want)[bad][:5], tol[bad][:5])
    return b


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("lens", LENS + [([1, 1], [1500, 700]), ([7], [513]), ([130], [130]), ([64], [1030])], ids=lens_id)
def test_attention(rx, shape, lens):
    rng = np.random.default_rng(seed_of(shape, lens) + 7)
    if shape == (32, 32, 128) and sum(lens[0]) > 40:
        shape = (5, 5, 128)                                    # (the oracle's time)
    b = attention_case(rx, rng, shape, [16, 32, 64, 128, 256][(shape[0] + sum(lens[1])) % 5], *lens)
    assert b.error() == 0


@pytest.mark.parametrize("device_table", [False, True])
@pytest.mark.parametrize("q_most", [1, 6, 40])
def test_attention_of_many_sequences(rx, q_most, device_table):
    rng = np.random.default_rng(40 + q_most)
    q_lens = [int(rng.integers(1, q_most + 1)) for _ in range(23)]
    kv_lens = [q + int(rng.integers(0, 200)) for q in q_lens]
    slots = [int(s) for s in rng.permutation(30)[:23]]
    attention_case(rx, rng, (8, 2, 64), 16, q_lens, kv_lens, slots, device_table=device_table)


@pytest.mark.parametrize("device_table", [False, True])
@pytest.mark.parametrize("shape,count,q_most", [((32, 32, 128), 100, 1), ((16, 16, 64), 200, 1), ((32, 4, 64), 300, 1), ((16, 16, 128), 128, 7)], ids=str)
def test_attention_of_many_short_sequences(rx, shape, count, q_most, device_table):
    """More tiles than wavefronts at a time, with holes in some page tables."""
    rng = np.random.default_rng(count + q_most)
    q_lens = [int(rng.integers(1, q_most + 1)) for _ in range(count)]
    kv_lens = [q + int(rng.integers(0, 150)) for q in q_lens]
    kv_lens[3] = q_lens[3]

    def lose(b):
        for i in (5, 50, count - 1):
            b.pages[i, 0] = -1
        b.dev_pages.copy_(torch.from_numpy(b.pages))
    b = attention_case(rx, rng, shape, 16, q_lens, kv_lens, device_table=device_table, edit=lose, heads=[0, shape[0] - 1])
    assert b.error() == 4


def scaled(factors):
    """edit: scales times what factors(rng, shape) gives, still of eight bits."""
    def edit(b):
        for i, key in enumerate(("ks", "vs")):
            with np.errstate(over="ignore", invalid="ignore"):
                x = po.round8(b.pool[key].astype(np.float32) * factors(np.random.default_rng(4 + i), b.pool[key].shape).astype(np.float32))
                b.pool[key] = np.clip(x, -8160, 8160).astype(np.float16)
            b.dev[key].copy_(torch.from_numpy(b.pool[key]))
    return edit


def test_attention_on_large_scores_and_uneven_scales(rx):
    """Scores of hundreds, so that one token takes the row; tokens and groups whose values differ by 10^6; the smallest and largest scales."""
    attention_case(rx, np.random.default_rng(2), (8, 2, 128), 16, [30, 1], [30, 700], std=40.0)
    uneven = scaled(lambda rng, shape: 10.0 ** rng.uniform(-4, 2, shape))
    for q_lens, kv_lens in (([200], [200]), ([1], [900]), ([20], [300])):
        attention_case(rx, np.random.default_rng(3), (4, 2, 64), 16, q_lens, kv_lens, edit=uneven)

    def largest(b):
        scaled(lambda rng, shape: np.full(shape, 1e6))(b)
        b.pool["ks"] = (b.pool["ks"].astype(np.float32) * np.float32(2.0 ** -13)).astype(np.float16)      # +-0.996
        b.dev["ks"].copy_(torch.from_numpy(b.pool["ks"]))
    attention_case(rx, np.random.default_rng(5), (4, 2, 64), 16, [1, 9], [200, 60], edit=largest)
    attention_case(rx, np.random.default_rng(6), (4, 2, 64), 16, [1, 9], [200, 60], edit=scaled(lambda rng, shape: np.full(shape, 1e-5)))


@pytest.mark.parametrize("std", [2.0 ** -20, 2.0 ** -10, 1000.0])
def test_attention_on_queries_of_any_size(rx, std):
    """The power of two that a row of q is multiplied with; rows whose elements differ by 2^24; a row of zeros."""
    rng = np.random.default_rng(61)
    for lens in (([1, 3], [77, 40]), ([100], [120])):
        b = Bench(rx, rng, 8, 2, 64, 16, *lens, scale=(0.02, 0.3) if std < 100 else (1e-4, 1e-3))
        q = half(rng, (b.n, 8, 64), std)
        q[0, 1] = 0
        q[1, 2, ::3] = np.float16(6e-8)
        got = b.attention(q).astype(np.float64)
        want, tol = po.attention(q.astype(np.float64), b.pool, b.pages, 16, *lens, None, 2, 64)
        assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("lead", [0, 45])
@pytest.mark.parametrize("pairs", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 40, 41, 48, 49, 64, 65])
def test_attention_at_every_width_of_a_tile(rx, pairs, lead):
    """Rows whose last tile has that many (row, head) pairs, on as many tokens as rows and behind 45 more: plain, and with large scores, uneven scales, blocks of zeros and a hole."""
    rng = np.random.default_rng(100 * pairs + lead)
    for shape, rows in (((2, 2, 128), pairs), ((3, 1, 64), -(-pairs // 3))):
        attention_case(rx, rng, shape, 16, [rows], [rows + lead])

    def spoil(b):
        scaled(lambda r, s: 10.0 ** r.uniform(-4, 2, s))(b)
        for key in ("ks", "vs"):
            b.pool[key][:, :, :, 5:9] = np.where(np.isnan(b.pool[key][:, :, :, 5:9]), np.nan, 0.0).astype(np.float16)
            b.dev[key].copy_(torch.from_numpy(b.pool[key]))
        b.pages[0, 1] = -1
        b.dev_pages.copy_(torch.from_numpy(b.pages))
    if pairs + lead > 16:
        assert attention_case(rx, rng, (2, 2, 128), 16, [pairs], [pairs + lead], std=4.0, edit=spoil).error() == 4


@pytest.mark.parametrize("rows,L", [(1, 900), (8, 1030), (12, 1003), (25, 2000)])
def test_bad_rows_in_small_tiles_and_parts(rx, rows, L):
    """A NaN or an infinity of a query stays in its row and head, also where a row's parts are merged."""
    rng = np.random.default_rng(rows)
    b = Bench(rx, rng, 6, 2, 64, 32, [rows], [L])
    q = half(rng, (rows, 6, 64))
    clean = b.attention(q)
    same = np.ones((rows, 6), bool)
    for row, head, value in ((0, 4, np.nan), (rows // 2, 1, np.inf), (rows - 1, 2, -np.inf)):
        q[row, head, 7 * head] = value
        same[row, head] = False
    got = b.attention(q)
    assert np.array_equal(got[same], clean[same]) and not np.isfinite(got[~same]).all(axis=1).any()


@pytest.mark.parametrize("shape,q_lens,kv_lens", [((8, 2, 64), [1, 3, 20], [3000, 50, 700]), ((64, 8, 128), [1], [40]), ((100, 100, 64), [300, 1], [300, 900])], ids=str)
def test_attention_in_place(rx, shape, q_lens, kv_lens):
    """out may be q: a tile reads its rows before it writes them, and no other reads them."""
    rng = np.random.default_rng(17)
    b = Bench(rx, rng, *shape, 16, q_lens, kv_lens)
    q = half(rng, (b.n, b.h, b.d))
    want, x = b.attention(q), torch.from_numpy(q).cuda()
    rx.check(rx.relax_paged4_attention(x, b.cache, b.seqs(), b.dims, x, b.n, *b.workspace()))
    torch.cuda.synchronize()
    assert same_bits(x.cpu().numpy(), want)


def test_parts_of_many_lengths(rx):
    """Sequences of one and of many parts in one call, in no order of length: those that are merged are the first in the order of lengths, and have rows of any number."""
    rng = np.random.default_rng(81)
    for shape, q_lens, kv_lens in (((16, 2, 64), [1, 1, 1, 1, 1, 1, 1], [40, 3000, 1, 700, 16, 9000, 129]), ((4, 2, 128), [3, 1, 20, 1, 2], [50, 6000, 2200, 1, 4000]),
                                   ((8, 1, 128), [1, 1], [20000, 3])):
        for device_table in (False, True):
            attention_case(rx, rng, shape, 32, q_lens, kv_lens, list(range(len(q_lens)))[::-1], device_table=device_table)


# Calls whose sequences fill tiles of 256 (row, head) pairs, 160 to 200 of them and more over all KV heads: (heads, KV heads, d), q_lens, kv_lens, heads to check
MANY_ROWS = [
    ((80, 80, 64), [300], [300], [0, 41, 79]),
    ((80, 80, 128), [257], [1000], [0, 1, 40, 79]),
    ((64, 8, 128), [33, 60, 40, 32, 35, 47, 33, 64, 50, 45], [33, 61, 300, 32, 99, 47, 700, 64, 1050, 45], [0, 7, 8, 63]),
    ((40, 8, 128), [300, 1, 450, 3, 260], [310, 800, 450, 77, 900], [0, 5, 13, 39]),
    ((40, 8, 64), [1001], [1001], [0, 9, 39]),
    ((160, 160, 64), [256], [8200], [0, 77, 159]),                # more blocks than are in LDS at a time
    ((24, 8, 128), [2000], [2000], [2, 23]),
    ((100, 100, 64), [300], [300], [0, 41, 99]),
    ((100, 100, 128), [257], [1000], [0, 1, 99]),
    ((64, 8, 128), [33, 60, 40, 32, 35, 47, 33, 64, 50, 45, 70, 66, 100], [33, 61, 300, 32, 99, 47, 700, 64, 1050, 45, 70, 90, 333], [0, 7, 8, 63]),
    ((40, 8, 128), [300, 1, 450, 3, 260, 200], [310, 800, 450, 77, 900, 1200], [0, 5, 39]),
    ((40, 8, 64), [1300], [1300], [0, 9, 39]),
    ((200, 200, 64), [256], [8200], [0, 199]),                    # more blocks than are in LDS at a time
    ((24, 8, 128), [2150], [2150], [2, 23]),
]


@pytest.mark.parametrize("device_table", [False, True])
@pytest.mark.parametrize("case", MANY_ROWS, ids=lambda c: "%s_%d" % (c[0], sum(c[1])))
def test_attention_of_many_rows(rx, case, device_table):
    shape, q_lens, kv_lens, heads = case
    rng = np.random.default_rng(seed_of(shape, q_lens))
    attention_case(rx, rng, shape, [16, 64, 256][len(q_lens) % 3], q_lens, kv_lens, [len(q_lens) - i for i in range(len(q_lens))], device_table=device_table, heads=heads)


def test_many_rows_without_pages_with_bad_rows_and_uneven_scales(rx):
    q_lens, kv_lens, shape, heads = [300, 290, 256, 3], [400, 300, 280, 50], (40, 40, 128), [0, 17, 39]

    def spoil(b):
        scaled(lambda rng, s: 10.0 ** rng.uniform(-4, 2, s))(b)
        for key in ("ks", "vs"):
            b.pool[key][:, 17, 0] = np.where(np.isnan(b.pool[key][:, 17, 0]), np.nan, 0.0).astype(np.float16)      # blocks of zeros
            b.dev[key].copy_(torch.from_numpy(b.pool[key]))
        b.pages[0, 2], b.pages[2] = -5, b.pool["k"].shape[0]            # sequence 2 has no page at all
        b.dev_pages.copy_(torch.from_numpy(b.pages))
    b = attention_case(rx, np.random.default_rng(50), shape, 16, q_lens, kv_lens, edit=spoil, heads=heads)
    assert b.error() == 4
    q = half(np.random.default_rng(51), (b.n, 40, 128))
    clean = b.attention(q)
    assert (clean[590:846] == 0).all()
    q[7, 3, 5], q[100, 4, :] = np.nan, np.inf
    got = b.attention(q)
    same = np.ones((b.n, 40), bool)
    same[7, 3] = same[100, 4] = False
    assert np.isnan(got[7, 3]).all() and np.array_equal(got[same], clean[same])


def test_a_bad_query_row_stays_alone(rx):
    rng = np.random.default_rng(8)
    for q_lens, kv_lens in (([9], [50]), ([200], [200])):
        b = Bench(rx, rng, 8, 2, 64, 16, q_lens, kv_lens)
        q = half(rng, (b.n, 8, 64))
        clean = b.attention(q)
        q[4, 3, 7], q[5, 1, :] = np.nan, np.inf
        got = b.attention(q)
        assert np.isnan(got[4, 3]).all()
        same = np.ones((b.n, 8), bool)
        same[4, 3] = same[5, 1] = False
        assert np.array_equal(got[same], clean[same])


def test_pages_out_of_range(rx):
    """A block without a page: dropped by the append, left out by attention, zeros in a read, and flagged by each."""
    rng = np.random.default_rng(6)

    def lose(b):
        b.pages[0, 1], b.pages[1, 0], b.pages[1, 1] = b.pool["k"].shape[0], -1, 2 ** 31 - 1      # sequence 1 has no page at all
        b.dev_pages.copy_(torch.from_numpy(b.pages))
        for key in ("ks", "vs"):                                # block 0 of the pool, which is read in their place, may hold anything
            b.pool[key][0] = np.where(np.isin(0, b.pages[0]), b.pool[key][0], np.float16(np.nan))
            b.dev[key].copy_(torch.from_numpy(b.pool[key]))
    for q_lens, kv_lens in (([1, 1], [70, 20]), ([3, 20], [70, 20]), ([70, 20], [70, 20])):
        b = attention_case(rx, rng, (8, 2, 64), 16, q_lens, kv_lens, edit=lose)
        assert b.error() == 4
        out = b.attention(half(rng, (b.n, 8, 64)))
        assert (out[q_lens[0]:] == 0).all()
        b.clear()
        k, v = b.read()
        assert (k[q_lens[0]:] == 0).all() and (v[q_lens[0]:] == 0).all() and b.error() == 4
        b.clear()
        qkv = half(rng, (b.n, 12 * 64))
        check_append(b, qkv, b.append(qkv))
        assert b.error() == 4


def test_lengths_beyond_the_capacity(rx):
    """A device table's length that the capacity does not cover: no token is written or attended to, a read gives zeros, and each raises the flag."""
    rng = np.random.default_rng(64)
    for q_lens, kv_lens in (([1, 1], [40, 33]), ([30, 20], [40, 33])):
        for bad in (65, 1 << 30, (1 << 31) - 1, -1, -(1 << 31)):
            b = Bench(rx, rng, 8, 2, 64, 32, q_lens, kv_lens, device_table=True, prep=dict())
            b.dev_table[2, 1] = bad
            q = half(rng, (b.n, 8, 64))
            out = b.attention(q)
            assert b.error() == 4 and (out[q_lens[0]:] == 0).all() and (out[:q_lens[0]] != 0).any()
            b.clear()
            k, v = b.read()
            assert b.error() == 4 and (k[q_lens[0]:] == 0).all() and (v[q_lens[0]:] == 0).all()
            b.clear()
            qkv = half(rng, (b.n, 12 * 64))
            b.append(qkv)
            assert b.error() == 4
            x = po8.storable(qkv.reshape(b.n, 12, 64)[:, 8:].astype(np.float32)).astype(np.float32)[:q_lens[0]]
            want = po.append(b.pool, b.pages, 32, b.prep.heads(x[:, :2], positions(q_lens[:1], kv_lens[:1]), 1), x[:, 2:], q_lens[:1], kv_lens[:1], None)
            got = b.host_pool()
            assert all(same_bits(got[key], want[key]) for key in want)


def test_lengths_beyond_the_bounds_of_a_captured_call(rx):
    """Within the capacity, beyond what the host said: attended to in full."""
    rng = np.random.default_rng(65)
    b = Bench(rx, rng, 8, 2, 128, 64, [1, 2], [900, 700], device_table=True, table_slack=-500)
    q = half(rng, (b.n, 8, 128))
    got = b.attention(q).astype(np.float64)
    want, tol = po.attention(q.astype(np.float64), b.pool, b.pages, 64, [1, 2], [900, 700], None, 2, 128)
    assert (np.abs(got - want) <= tol).all()


DEVICE_LENGTHS = {"parts": ((4, 2, 64), 16, [1, 2, 1], [1100, 1500, 40]), "parts_128": ((8, 2, 128), 64, [3, 1], [900, 2000]), "wide_parts": ((8, 2, 128), 32, [9, 1], [900, 2000]),
                  "one_part": ((32, 32, 64), 16, [1] * 9, [30, 200, 77, 16, 100, 5, 64, 33, 90]), "rows": ((100, 100, 64), 16, [300, 270], [300, 296]),
                  "both_kernels": ((40, 40, 128), 16, [400, 2, 260, 300], [408, 70, 360, 300])}


@pytest.mark.parametrize("kind", sorted(DEVICE_LENGTHS))
def test_attention_on_lengths_of_a_device_table_beyond_the_capacity(rx, kind):
    """Known on the device only: such a sequence has no token, which gives zeros and the flag, and the others are what they are without it; with host bounds at the capacity and far
    below it."""
    shape, page, q_lens, kv_lens = DEVICE_LENGTHS[kind]
    b = Bench(rx, np.random.default_rng(76), *shape, page, q_lens, kv_lens, device_table=True)
    q = half(np.random.default_rng(77), (b.n, b.h, b.d))
    dev, (ws, ws_bytes) = torch.from_numpy(q).cuda(), b.workspace()
    starts = np.concatenate([[0], np.cumsum(q_lens)])
    for bounds in ([b.cap] * len(q_lens), kv_lens):
        out = torch.empty_like(dev)
        call = lambda: rx.check(rx.relax_paged4_attention(dev, b.cache, rx.Seqs(q_lens, bounds, None, b.dev_table), b.dims, out, b.n, ws, ws_bytes))
        rx.check(rx.relax_workspace_init(b.dims, ws, ws_bytes))
        b.dev_table[2] = torch.tensor(kv_lens, dtype=torch.int32)
        call()
        clean = out.clone()
        assert b.error() == 0
        for lost in {0, len(q_lens) - 1}:
            for length in (b.cap + 1, b.cap + 500, 2 ** 31 - 1, -1, -2 ** 31):
                b.dev_table[2, lost] = length
                out.fill_(float("nan"))
                call()
                rows = slice(int(starts[lost]), int(starts[lost + 1]))
                want = clean.clone()
                want[rows] = 0
                assert torch.equal(out, want) and b.error() == 4, (lost, length)
            b.dev_table[2] = torch.tensor(kv_lens, dtype=torch.int32)


@pytest.mark.parametrize("bound", [2, 130, 700])
def test_a_device_table_beyond_the_bounds_of_the_call(rx, bound):
    """Lengths of the table that the bounds of the host fall short of, within the capacity: all their tokens count, with the workspace of the bounds."""
    for q_lens, kv_lens, shape in (([1, 2], [3000, 41], (8, 2, 64)), ([1, 2], [3000, 41], (40, 2, 64))):
        b = Bench(rx, np.random.default_rng(78), *shape, 32, q_lens, kv_lens, device_table=True)
        q = half(np.random.default_rng(79), (b.n, b.h, 64))
        dev = torch.from_numpy(q).cuda()
        out = torch.empty_like(dev)
        ws_bytes = rx.relax_paged4_workspace_bytes(b.dims, b.n, bound, 2)
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
        rx.check(rx.relax_workspace_init(b.dims, ws, ws_bytes))
        rx.check(rx.relax_paged4_attention(dev, b.cache, rx.Seqs(q_lens, [bound, 41 if bound > 41 else 2], None, b.dev_table), b.dims, out, b.n, ws, ws_bytes))
        want, tol = po.attention(q.astype(np.float64), b.pool, b.pages, 32, q_lens, kv_lens, None, 2, 64)
        assert (np.abs(out.cpu().numpy().astype(np.float64) - want) <= tol).all()
        assert rx.relax_workspace_error(b.dims, ws) == 0


def test_append_and_read_on_device_lengths_next_to_the_end_of_their_type(rx):
    """Lengths whose last block ends behind 2^31, or below zero: no page, no row of another sequence touched."""
    rng = np.random.default_rng(83)
    b = Bench(rx, rng, 4, 2, 64, 16, [3, 20, 1], [20, 32, 9], device_table=True, prep=dict())
    qkv = half(rng, (b.n, 8 * 64))
    for length in (2 ** 31 - 1, 2 ** 31 - 5, 2 ** 31 - 16, 2 ** 31 - 17, -1, -1000, -2 ** 31 + 2, -2 ** 31):
        for lost, rows in ((0, slice(0, 3)), (1, slice(3, 23))):
            b.dev_table[2] = torch.tensor([20, 32, 9], dtype=torch.int32)
            b.clear()
            q = b.append(qkv)
            b.read()
            assert b.error() == 0
            b.dev_table[2, lost] = length
            held = b.host_pool()
            again_q = b.append(qkv)
            assert b.error() == 4
            keep = np.ones(b.n, bool)
            keep[rows] = False
            assert same_bits(again_q[keep], q[keep])
            again = b.host_pool()
            for key in held:
                assert same_bits(held[key], again[key]), (length, lost, key)
            got = b.read()
            assert (got[:, rows] == 0).all()


@pytest.mark.parametrize("by_address", [False, True])
def test_python_calls_on_a_stream_of_their_own(rx, by_address):
    """Table, heads, append, attention and read on a side stream that starts late, with nothing but what the calls allocate, against the same on the current stream; the current
    stream allocates and writes in between."""
    from paper_2311_02103_amd import runtime
    rng = np.random.default_rng(80)
    make = lambda: runtime.DevicePaged4Cache(n_heads=8, n_kv_heads=2, head_dim=64, kv_capacity=512, n_pages=16, page_size=32, n_max=500)
    here, there = make(), make()
    for layer in (here, there):
        layer.pages.copy_(torch.arange(16, dtype=torch.int32).view(1, 16))
    x = torch.from_numpy(half(rng, (500, 12 * 64))).cuda()
    seqs, scaling = rx.Seqs([500], [500]), rx.RopeScaling(rx.ROPE_LINEAR, 128, 10000.0, 2.0)

    def run(layer, stream):
        q = layer.append(x, seqs, stream=stream)
        return (q, layer.attention(q, seqs, stream=stream), *layer.read(seqs, 500, stream=stream), *layer.heads(x, seqs, stream=stream), runtime.rope_table(scaling, 5000, stream=stream))
    want = run(here, None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(20):
            late = torch.randn(2048, 2048, device="cuda") @ torch.randn(2048, 2048, device="cuda")
    for _ in range(3):
        got = run(there, side.cuda_stream if by_address else side)
        noise = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for size in (512, 4096, 65536, 1 << 20) for _ in range(4)]
    torch.cuda.synchronize()
    assert len(noise) == 16 and late.shape == (2048, 2048)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_shared_pages(rx):
    """Two sequences on the same first pages."""
    def share(b):
        b.pages[1, :4] = b.pages[0, :4]
        b.dev_pages.copy_(torch.from_numpy(b.pages))
    attention_case(rx, np.random.default_rng(12), (8, 2, 128), 16, [1, 30], [90, 111], edit=share)


def test_pool_beyond_32_bits(rx):
    """Blocks whose codes lie more than 4 GiB into the pool, scales more than 1 GiB."""
    rng = np.random.default_rng(13)
    g, d, page_size = 2, 128, 256
    per_page = g * page_size * d // 2
    n_pages = (1 << 32) // per_page + 40
    dims = rx.make_dims(4 * d, 4, g, d, 64, 2 * page_size, 1)
    k, v = (torch.empty(n_pages * per_page, dtype=torch.uint8, device="cuda") for _ in "kv")
    ks, vs = (torch.empty(n_pages * per_page // 16, dtype=torch.float16, device="cuda") for _ in "kv")
    ids = [n_pages - 2, n_pages - 31]
    pages = torch.tensor([ids], dtype=torch.int32, device="cuda")
    cache = rx.Paged4Cache(k, v, ks, vs, pages, n_pages, page_size, 2)
    ws_bytes = rx.relax_paged4_workspace_bytes(dims, 400, 400, 1)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    qkv = half(rng, (400, 8 * d))
    x = torch.from_numpy(qkv).cuda()
    q = torch.empty((400, 4, d), dtype=torch.float16, device="cuda")
    base = x.data_ptr()
    rx.check(rx.relax_paged4_append(base, 8 * d, base + 8 * d, base + 12 * d, 8 * d, q, None, cache, rx.Seqs([400], [400]), dims, 400, ws, ws_bytes))
    out = torch.empty((2, 4, d), dtype=torch.float16, device="cuda")
    rx.check(rx.relax_paged4_attention(q[-2:], cache, rx.Seqs([2], [400]), dims, out, 2, ws, ws_bytes))
    back = torch.empty((2, 400, g, d), dtype=torch.float16, device="cuda")
    rx.check(rx.relax_paged4_read(cache, rx.Seqs([400], [400]), dims, back[0], back[1], 400, ws, ws_bytes))
    full = torch.empty((400, 4, d), dtype=torch.float16, device="cuda")
    rx.check(rx.relax_paged4_attention(q, cache, rx.Seqs([400], [400]), dims, full, 400, ws, ws_bytes))
    torch.cuda.synchronize()
    blocks = page_size // 16
    pool = {name: t.view(n_pages, g, blocks, -1)[ids].cpu().numpy() for name, t in (("k", k), ("v", v), ("ks", ks), ("vs", vs))}
    local = np.array([[0, 1]], np.int32)
    y = qkv.astype(np.float32).reshape(400, 8, d)
    made = po.append({key: np.zeros_like(p) for key, p in pool.items()}, local, page_size, y[:, 4:6], y[:, 6:], [400], [400], None)
    for name, got in (("k", back[0]), ("v", back[1])):
        c, s = po.values(made, name, local, page_size, 0, np.arange(400), d)
        assert np.array_equal(got.cpu().numpy().astype(np.float64), c * s)
    want, tol = po.attention(qkv.astype(np.float64).reshape(400, 8, d)[:, :4], made, local, page_size, [400], [400], None, g, d)
    for got, rows in ((full, slice(0, 400)), (out, slice(398, 400))):
        assert (np.abs(got.cpu().numpy().astype(np.float64) - want[rows]) <= tol[rows]).all()


@pytest.mark.parametrize("shape,q_lens,heads", [((16, 1, 64), [1500] + [1] * 299, [0, 15]), ((64, 8, 64), [1] * 150 + [700] + [1] * 150, [0, 63]),
                                                ((8, 2, 64), [2, 31, 1, 1, 3] * 40, None)], ids=["small_tiles", "large_tiles", "ragged"])
@pytest.mark.parametrize("device_table", [False, True])
def test_one_prompt_among_many_sequences(rx, shape, q_lens, heads, device_table):
    rng = np.random.default_rng(71)
    attention_case(rx, rng, shape, 16, q_lens, [q + int(rng.integers(0, 60)) for q in q_lens], device_table=device_table, heads=heads)


# ---- together -------------------------------------------------------------------------------------------------------
def test_a_prompt_and_decode_steps_together(rx):
    """A serving program's run with normalised heads and half of each turned by neighbours: a prompt in two chunks, then tokens one by one, two sequences of
    different lengths, each step append and attention; attention meets what the pool holds, and stays near a dense fp16 cache's."""
    rng = np.random.default_rng(21)
    h, g, d, cap = 8, 2, 64, 128
    b = Bench(rx, rng, h, g, d, 32, [1, 1], [cap, cap], prep=dict(rotary=32, pairs=True))
    at = [0, 0]
    for step in [[37, 20], [21, 1]] + [[1, 1]] * 9:
        at = [a + s for a, s in zip(at, step)]
        b.q_lens, b.kv_lens, b.n = step, list(at), sum(step)
        b.pool = b.host_pool()
        qkv = half(rng, (b.n, (h + 2 * g) * d))
        q = b.append(qkv)
        check_append(b, qkv, q)
        got = b.attention(q).astype(np.float64)
        pool = b.host_pool()
        want, tol = po.attention(q.astype(np.float64), pool, b.pages, 32, step, at, None, g, d)
        assert (np.abs(got - want) <= tol).all()
        k, v = b.read()
        x = qkv.astype(np.float64).reshape(b.n, h + 2 * g, d)
        row = 0
        for i, ql in enumerate(step):
            sl = slice(row, row + ql)
            exact = b.prep.heads(qkv.reshape(b.n, -1, d)[sl, h:h + g], np.arange(at[i] - ql, at[i]), 1)
            for got_, true in ((k[sl], exact), (v[sl], x[sl, h + g:])):
                groups = true.reshape(ql, g, 2, 32)
                # off by most where an element is as far as the largest on the other side: code 15 holds 7 steps of it, and a step is max / 8 rounded to eight
                # bits, (max / 8)(1 - 2^-8) at least, so max - 7 (max / 8)(1 - 2^-8) = (max / 8)(1 + 7 2^-8)
                limit = np.abs(groups).max(axis=3, keepdims=True) / 8 * (1 + 7 * 2.0 ** -8)
                assert (np.abs(got_.astype(np.float64).reshape(groups.shape) - groups) <= limit).all()
            row += ql
    assert b.error() == 0


def test_prepared_heads_go_into_the_8_bit_cache(rx):
    """relax_head_norm_rope in front of relax_paged_append without a rotary table: heads that the 8-bit cache's own append cannot prepare."""
    rng = np.random.default_rng(22)
    h, g, d, n = 8, 2, 64, 21
    t = Heads(rx, rng, h, g, d, [n], [n], dict(rotary=32), cap=32)
    qkv = half(rng, (n, (h + 2 * g) * d))
    x = torch.from_numpy(qkv).cuda()
    at, row = x.data_ptr(), x.shape[1]
    rx.check(rx.relax_head_norm_rope(at, row, at + 2 * h * d, row, at, row, at + 2 * h * d, row, t.prep.c, t.seqs(), t.dims, n, t.ws, t.ws_bytes))
    k, v = (torch.empty((4, g, 1, 16 * d), dtype=torch.uint8, device="cuda") for _ in "kv")
    ks, vs = (torch.empty((4, g, 1), dtype=torch.float32, device="cuda") for _ in "kv")
    cache = rx.PagedCache(k, v, ks, vs, torch.tensor([[2, 0]], dtype=torch.int32, device="cuda"), None, 4, 16, 2)
    ws_bytes = rx.relax_paged_workspace_bytes(t.dims, n, n, 1)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    q, out = (torch.empty((n, h, d), dtype=torch.float16, device="cuda") for _ in "qo")
    rx.check(rx.relax_paged_append(at, row, at + 2 * h * d, at + 2 * (h + g) * d, row, q, cache, rx.Seqs([n], [n]), t.dims, n, ws, ws_bytes))
    rx.check(rx.relax_paged_attention(q, cache, rx.Seqs([n], [n]), t.dims, out, n, ws, ws_bytes))
    torch.cuda.synchronize()
    want_q, want_k = t.want(qkv[:, :(h + g) * d])
    assert same_bits(q.cpu().numpy().reshape(n, -1), want_q)
    pool = {"k": k.cpu().numpy(), "v": v.cpu().numpy(), "ks": ks.cpu().numpy(), "vs": vs.cpu().numpy()}
    pages = np.array([[2, 0]], np.int32)
    held = po8.values(pool, "k", pages, 16, 0, np.arange(n), d)
    assert np.abs(held - want_k.astype(np.float64).reshape(n, g, d)).max() <= 0.5001 * pool["ks"][[2, 0]].max()
    want, tol = po8.attention(q.cpu().numpy().astype(np.float64), pool, pages, 16, [n], [n], None, g, d)
    assert (np.abs(out.cpu().numpy().astype(np.float64) - want) <= tol).all()


def test_steps_in_a_graph_follow_the_table(rx):
    """Append and attention captured once with upper bounds, replayed while the device table counts up; every replay against an eager call on a second pool, other
    work in between."""
    rng = np.random.default_rng(30)
    h, g, d, page = 8, 2, 128, 16
    q_lens = [1, 1, 1]
    b, e = (Bench(rx, np.random.default_rng(31), h, g, d, page, q_lens, [640, 640, 640], device_table=True, prep=dict()) for _ in range(2))
    lens = [5, 300, 31]
    x = torch.zeros((3, (h + 2 * g) * d), dtype=torch.float16, device="cuda")
    outs = {name: [torch.empty((3, h, d), dtype=torch.float16, device="cuda") for _ in range(3)] for name in ("graph", "eager")}
    for bench in (b, e):
        bench.workspace()
    side = torch.cuda.Stream()

    def step(bench, name, stream):
        base, row = x.data_ptr(), x.shape[1]
        q, out, turned = outs[name]
        seqs = bench.seqs()
        rx.check(rx.relax_head_norm_rope(base, row, None, 0, turned, h * d, None, 0, bench.prep.c, seqs, bench.dims, 3, bench.ws, bench.ws_bytes, stream))
        rx.check(rx.relax_paged4_append(base, row, base + 2 * h * d, base + 2 * (h + g) * d, row, q, bench.prep.c, bench.cache, seqs, bench.dims, 3, bench.ws, bench.ws_bytes, stream))
        rx.check(rx.relax_paged4_attention(q, bench.cache, seqs, bench.dims, out, 3, bench.ws, bench.ws_bytes, stream))
    for bench in (b, e):
        bench.dev_table[2] = torch.tensor(lens, dtype=torch.int32)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(b, "graph", side)
    torch.cuda.synchronize()
    for _ in range(5):
        x.copy_(torch.from_numpy(half(rng, tuple(x.shape))))
        graph.replay()
        torch.cuda.synchronize()
        step(e, "eager", None)
        _ = (torch.randn(512, 512, device="cuda") @ torch.randn(512, 512, device="cuda")).sum()
        torch.cuda.synchronize()
        for a, c in zip(outs["graph"], outs["eager"]):
            assert torch.equal(a, c)
        assert torch.equal(outs["graph"][0], outs["graph"][2])      # the two calls prepare queries alike
        for key in b.dev:
            assert torch.equal(b.dev[key].view(torch.uint8), e.dev[key].view(torch.uint8)), key
        for bench in (b, e):
            bench.dev_table[2] += 1
        torch.cuda.synchronize()


def test_two_streams_with_workspaces_of_their_own(rx):
    rng = np.random.default_rng(33)
    b = [Bench(rx, rng, 8, 2, 128, 32, [1, 3], [900, 400]) for _ in range(2)]
    q = [half(rng, (4, 8, 128)) for _ in b]
    alone = [x.attention(y) for x, y in zip(b, q)]
    qd = [torch.from_numpy(y).cuda() for y in q]
    out = [torch.empty_like(y) for y in qd]
    streams = [torch.cuda.Stream() for _ in b]
    torch.cuda.synchronize()
    for _ in range(4):
        for i in (0, 1):
            rx.check(rx.relax_paged4_attention(qd[i], b[i].cache, b[i].seqs(), b[i].dims, out[i], 4, *b[i].workspace(), streams[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert np.array_equal(out[i].cpu().numpy(), alone[i])


def test_calls_repeat_bit_by_bit(rx):
    rng = np.random.default_rng(34)
    for shape, lens in (((8, 2, 128), ([1, 5], [700, 1300])), ((40, 40, 64), ([300], [333]))):
        b = Bench(rx, rng, *shape, 64, *lens)
        q = half(rng, (b.n, b.h, b.d))
        first = b.attention(q)
        assert all(same_bits(first, b.attention(q)) for _ in range(3))


def test_a_model_of_one_layer_with_normalised_heads(rx):
    """The Python classes as a program strings them together: projection, append, attention, the output product; requests of different ages, normalised heads of which part is
    turned at stretched positions.  Two layers share the tables.  Keys and values against the definition bit by bit, attention in 64 bits on what is held."""
    from paper_2311_02103_amd import runtime
    rng = np.random.default_rng(91)
    h, g, d, H, page = 8, 2, 64, 256, 16
    scaling = rx.RopeScaling(rx.ROPE_WAVELENGTH_RAMP, 32, 10000.0, 4.0, 64.0, 1.0, 4.0)
    mat = lambda m, k: torch.from_numpy(half(rng, (m, k), k ** -0.5)).cuda()
    norms = [torch.from_numpy(half(rng, d, 0.2) + np.float16(1)).cuda() for _ in "qk"]
    made = dict(n_heads=h, n_kv_heads=g, head_dim=d, kv_capacity=160, n_pages=30, page_size=page, kv_slots=3, n_max=200, q_norm=norms[0], k_norm=norms[1], eps=EPS, layout=rx.ROPE_PAIRS)
    first = runtime.DevicePaged4Cache(rope=scaling, **made)
    layers = [first, runtime.DevicePaged4Cache(share_from=first, **made)]
    first.pages.copy_(torch.from_numpy(rng.permutation(30).reshape(3, 10).astype(np.int32)))
    pages, table = first.pages.cpu().numpy(), first.rope.cpu().numpy()
    weights = [(mat((h + 2 * g) * d, H), mat(H, h * d)) for _ in layers]

    def product(x, w):
        y = torch.empty((x.shape[0], w.shape[0]), dtype=torch.float16, device="cuda")
        rx.check(rx.relax_half_matmul(x, w, y, x.shape[0], w.shape[0], w.shape[1]))
        return y
    held = [0, 0, 0]
    for slots, lens in (([1], [97]), ([2, 0, 1], [33, 60, 1]), ([0, 1, 2], [1, 1, 1]), ([2, 0], [1, 4])):
        for s_, ln in zip(slots, lens):
            held[s_] += ln
        kv_lens, n = [held[s_] for s_ in slots], sum(lens)
        seqs, pos = rx.Seqs(lens, kv_lens, slots), positions(lens, kv_lens)
        x = torch.from_numpy(half(rng, (n, H))).cuda()
        for layer, (wqkv, wo) in zip(layers, weights):
            before = {key: t.cpu().numpy() for key, t in (("k", layer.k), ("v", layer.v), ("ks", layer.k_scale), ("vs", layer.v_scale))}
            qkv = product(x, wqkv)
            q = layer.append(qkv, seqs)
            o = layer.attention(q, seqs)
            alone_q, alone_k = layer.heads(qkv, seqs)
            x = x + product(o.view(-1, h * d), wo)
            rows = qkv.cpu().numpy().reshape(n, h + 2 * g, d).astype(np.float32)
            w = [t.cpu().numpy().astype(np.float32) for t in norms]
            want_q, want_k = (po.prepare(rows[:, a:b], w_, np.float32(EPS), table[pos][:, None], 32, True) for a, b, w_ in ((0, h, w[0]), (h, h + g, w[1])))
            assert same_bits(q.cpu().numpy(), want_q.astype(np.float16)) and same_bits(alone_q.cpu().numpy(), want_q.astype(np.float16))
            assert same_bits(alone_k.cpu().numpy(), want_k.astype(np.float16))
            pool = po.append(before, pages, page, want_k, rows[:, h + g:], lens, kv_lens, slots)
            for key, t in (("k", layer.k), ("v", layer.v), ("ks", layer.k_scale), ("vs", layer.v_scale)):
                assert same_bits(t.cpu().numpy(), pool[key]), key
            want, tol = po.attention(q.cpu().numpy().astype(np.float64), pool, pages, page, lens, kv_lens, slots, g, d)
            assert (np.abs(o.cpu().numpy() - want) <= tol).all()
            for name, got in zip("kv", layer.read(seqs, n)):
                for row, ql, L, slot in po.sequences(lens, kv_lens, slots):
                    c, s_ = po.values(pool, name, pages, page, slot, np.arange(L - ql, L), d)
                    assert np.array_equal(got[row:row + ql].cpu().numpy().astype(np.float64), c * s_)
    assert rx.relax_workspace_error(first.dims, first.ws) == 0


def test_the_smallest_groups_that_are_held(rx):
    """A largest magnitude of 2^-22 is held as zeros, the next fp16 number above it as itself; 8 to 20 times 2^-24 by scales of one and two steps."""
    b = Bench(rx, np.random.default_rng(93), 4, 4, 64, 16, [9], [9])
    qkv = np.zeros((9, 12 * 64), np.float16)
    tops = [1, 3, 4, 5, 8, 11, 12, 20, -5]
    for row, top in enumerate(tops):
        qkv[row, 256:].reshape(-1, 32)[:, row] = np.float16(top * 2.0 ** -24)
    check_append(b, qkv, b.append(qkv))
    for got in b.read():
        for row, want in enumerate((0, 0, 0, 5, 8, 8, 12, 16, -5)):
            x = got[row].reshape(-1, 32).astype(np.float64)
            assert (x[:, row] == want * 2.0 ** -24).all() and (np.delete(x, row, axis=1) == 0).all(), tops[row]
