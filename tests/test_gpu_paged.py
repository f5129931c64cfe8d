"""The paged 8-bit KV cache on the GPU -- append with rotation and quantisation, read-back, attention -- against a plain implementation in
64 bits (paged_oracle.py), at the sizes, layouts and page tables where it can go wrong."""
import zlib

import numpy as np
import pytest

import paged_oracle as po

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

SHAPES = [(4, 4, 64), (32, 32, 128), (8, 2, 64), (16, 2, 128), (6, 2, 128), (40, 2, 64), (7, 1, 128)]


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


class Bench:
    """A pool with random contents, its device copy, and the calls on it."""

    def __init__(self, rx, rng, h, g, d, page_size, q_lens, kv_lens, slots=None, rope=True, spare=2, device_table=False, scale=(0.02, 0.05)):
        self.rx, self.h, self.g, self.d, self.page_size, self.rope = rx, h, g, d, page_size, rope
        self.q_lens, self.kv_lens, self.slots = q_lens, kv_lens, slots
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
            self.pool[name] = rng.integers(1, 256, (n_pages, g, blocks, 16 * d)).astype(np.uint8)
            s = rng.uniform(*scale, (n_pages, g, blocks)).astype(np.float32)
            self.pool[name + "s"] = s
        # scales of blocks that no sequence has reached: never written, so anything
        reached = np.zeros((n_pages, blocks), bool)
        for slot, L in zip([s for s, _ in used], kv_lens):
            for pos in range(0, L, 16):
                reached[self.pages[slot, pos // page_size], pos % page_size // 16] = True
        for name in "kv":
            self.pool[name + "s"][np.broadcast_to(~reached[:, None], self.pool[name + "s"].shape)] = np.nan
        self.cap = self.per * page_size
        self.dims = rx.make_dims(h * d, h, g, d, 64, self.cap, n_slots)
        self.dev = {key: torch.from_numpy(x.copy()).cuda() for key, x in self.pool.items()}
        self.dev_pages = torch.from_numpy(self.pages.copy()).cuda()
        self.table = None
        if rope:
            self.table = torch.empty(rx.relax_rope_table_bytes(self.dims) // 4, dtype=torch.float32, device="cuda")
            rx.check(rx.relax_rope_table_init(self.dims, self.table))
        self.cache = rx.PagedCache(self.dev["k"], self.dev["v"], self.dev["ks"], self.dev["vs"], self.dev_pages, self.table, n_pages, page_size, self.per)
        self.ws_bytes = rx.relax_paged_workspace_bytes(self.dims, self.n, max(kv_lens), len(q_lens))
        self.ws = torch.full((self.ws_bytes,), 0xFF, dtype=torch.uint8, device="cuda")
        rx.check(rx.relax_workspace_init(self.dims, self.ws, self.ws_bytes))
        self.dev_table = None
        if device_table:
            starts = np.concatenate([[0], np.cumsum(q_lens)[:-1]])
            rows = np.stack([starts, q_lens, kv_lens, np.arange(len(q_lens)) if slots is None else slots]).astype(np.int32)
            self.dev_table = torch.from_numpy(rows).cuda()

    def seqs(self, q_lens=None):
        kv = self.kv_lens if self.dev_table is None else [min(self.cap, L + 40) for L in self.kv_lens]      # upper bounds
        return self.rx.Seqs(q_lens or self.q_lens, kv, self.slots, self.dev_table)

    def workspace(self):
        bound = self.rx.relax_paged_workspace_bytes(self.dims, self.n, self.cap, len(self.q_lens))
        if bound > self.ws_bytes:
            self.ws, self.ws_bytes = torch.full((bound,), 0xFF, dtype=torch.uint8, device="cuda"), bound
            self.rx.check(self.rx.relax_workspace_init(self.dims, self.ws, self.ws_bytes))
        return self.ws, self.ws_bytes

    def append(self, qkv, q=True, stream=None):
        """qkv: host fp16 [n, (h + 2 g) d]."""
        x = torch.from_numpy(qkv).cuda()
        base, row = x.data_ptr(), x.shape[1]
        q_out = torch.full((self.n, self.h, self.d), float("nan"), dtype=torch.float16, device="cuda") if q else None
        self.rx.check(self.rx.relax_paged_append(base if q else None, row, base + 2 * self.h * self.d, base + 2 * (self.h + self.g) * self.d, row, q_out,
                                                 self.cache, self.seqs(), self.dims, self.n, *self.workspace(), stream))
        torch.cuda.synchronize()
        return q_out.cpu().numpy() if q else None

    def attention(self, q, stream=None):
        qd = torch.from_numpy(q).cuda()
        out = torch.full(qd.shape, float("nan"), dtype=torch.float16, device="cuda")
        self.rx.check(self.rx.relax_paged_attention(qd, self.cache, self.seqs(), self.dims, out, self.n, *self.workspace(), stream))
        torch.cuda.synchronize()
        return out.cpu().numpy()

    def read(self):
        out = torch.full((2, self.n, self.g, self.d), float("nan"), dtype=torch.float16, device="cuda")
        self.rx.check(self.rx.relax_paged_read(self.cache, self.seqs(), self.dims, out[0], out[1], self.n, *self.workspace()))
        torch.cuda.synchronize()
        return out.cpu().numpy()

    def host_pool(self):
        return {key: x.cpu().numpy() for key, x in self.dev.items()}

    def error(self):
        return self.rx.relax_workspace_error(self.dims, self.ws)


def check_append(b, qkv, q_out):
    h, g, d = b.h, b.g, b.d
    x = qkv.astype(np.float64).reshape(b.n, h + 2 * g, d)
    # q: one rounding to fp16 of two products and their sum in fp32, from a table entry of 2^-24
    if q_out is not None:
        want, tol = np.empty((b.n, h, d)), np.empty((b.n, h, d))
        for row, ql, L, slot in po.sequences(b.q_lens, b.kv_lens, b.slots):
            for i in range(ql):
                want[row + i] = po.rotate(x[row + i, :h], L - ql + i, d) if b.rope else x[row + i, :h]
                mag = np.abs(x[row + i, :h]).reshape(h, 2, d // 2).sum(axis=1)
                tol[row + i] = 2.0 ** -11 * np.abs(want[row + i]) + 2.0 ** -22 * np.concatenate([mag, mag], axis=1) + 2.0 ** -25
        assert (np.abs(q_out.astype(np.float64) - want) <= tol).all()
    # codes: |code - x / s| is half a step, and what fp32 adds at a border: rotation 3 roundings of 2^-24 of |a| + |b| <= 2 amax,
    # the scale and the quotient 2^-24 each: 127 * 8 * 2^-24 < 1e-4
    got, want = b.host_pool(), {key: v.copy() for key, v in b.pool.items()}
    for item in po.append(b.pool, b.pages, b.page_size, x[:, h:h + g], x[:, h + g:], b.q_lens, b.kv_lens, b.slots, d, b.rope):
        name, at = item["name"], item["at"]
        s = got[name + "s"][at]
        assert abs(s - item["scale"]) <= 2.0 ** -21 * item["scale"], (name, at, s, item["scale"])
        want[name + "s"][at] = s
        index = po.code_index(name, d)
        codes = got[name][at][index].astype(np.float64) - 128.0
        low, high = item["low"], item["high"]
        assert np.abs(codes[low:high] - item["new"]).max() <= 0.5 + 1e-4, (name, at)
        touched = index[low:high]
        if s > b.pool[name + "s"][at] and low > 0:
            assert np.abs(codes[:low] - item["old"]).max() <= 0.5 + 1e-4, (name, at)
            touched = index[:high]
        want[name][at][touched] = got[name][at][touched]
    for key in want:                                           # everything else as it was
        assert np.array_equal(got[key].view(np.uint8), want[key].view(np.uint8)), key


LENS = [
    ([1], [1]), ([1], [2231]), ([1], [16]), ([1], [17]), ([5], [5]), ([16], [16]), ([17], [40]), ([33], [300]),
    ([1, 1, 1], [1, 32, 77]), ([3, 1, 40, 2], [3, 100, 41, 18]), ([2, 2, 2], [17, 33, 16]),
]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("lens", LENS, ids=lambda v: "x".join(map(str, v[0])) + "_of_" + "x".join(map(str, v[1])))
def test_append_and_read(rx, shape, lens):
    rng = np.random.default_rng(seed_of(shape, lens))
    page_size = [16, 32, 64, 128, 256][(shape[0] + sum(lens[1])) % 5]
    b = Bench(rx, rng, *shape, page_size, *lens)
    qkv = half(rng, (b.n, (b.h + 2 * b.g) * b.d), std=3.0)
    q_out = b.append(qkv)
    check_append(b, qkv, q_out)
    assert b.error() == 0
    k, v = b.read()
    pool = b.host_pool()
    for row, ql, L, slot in po.sequences(b.q_lens, b.kv_lens, b.slots):
        for name, got in (("k", k), ("v", v)):
            want = po.values(pool, name, b.pages, page_size, slot, np.arange(L - ql, L), b.d)
            assert np.array_equal(got[row:row + ql], want.astype(np.float32).astype(np.float16)), name      # code * scale in fp32, one rounding


@pytest.mark.parametrize("count", [17, 64, 200])
@pytest.mark.parametrize("device_table", [False, True])
def test_append_of_many_sequences(rx, count, device_table):
    rng = np.random.default_rng(count)
    q_lens = [1 if count == 64 else int(rng.integers(1, 20)) for _ in range(count)]
    kv_lens = [q + int(rng.integers(0, 60)) for q in q_lens]
    slots = [int(s) for s in rng.permutation(count + 3)[:count]]
    b = Bench(rx, rng, 8, 2, 64, 32, q_lens, kv_lens, slots, device_table=device_table)
    qkv = half(rng, (b.n, 12 * 64))
    check_append(b, qkv, b.append(qkv))
    assert b.error() == 0


@pytest.mark.parametrize("rope", [False, True])
def test_append_without_queries_and_from_matrices_of_their_own(rx, rope):
    """q and q_out NULL; and k, v rows of their own strides, as a dense cache has them."""
    rng = np.random.default_rng(5)
    b = Bench(rx, rng, 8, 4, 128, 64, [20, 3], [37, 9], rope=rope)
    qkv = half(rng, (b.n, 16 * 128))
    b.append(qkv, q=False)
    check_append(b, qkv, None)
    first = b.host_pool()
    b2 = Bench(rx, np.random.default_rng(5), 8, 4, 128, 64, [20, 3], [37, 9], rope=rope)
    x = torch.from_numpy(qkv).cuda()
    k = torch.full((b.n, 4 * 128 + 24), float("nan"), dtype=torch.float16, device="cuda")
    v = k.clone()
    k[:, :512], v[:, :512] = x[:, 1024:1536], x[:, 1536:]
    q = x[:, :1024].contiguous()
    rx.check(rx.relax_paged_append(q, 1024, k, v, 536, q, b2.cache, b2.seqs(), b2.dims, b2.n, *b2.workspace()))      # q_out is q
    torch.cuda.synchronize()
    again = b2.host_pool()
    for key in first:
        assert np.array_equal(first[key].view(np.uint8), again[key].view(np.uint8)), key
    check_append(b2, qkv, q.cpu().numpy().reshape(b.n, 8, 128))


def test_token_by_token_scales_grow_and_old_codes_follow(rx):
    """Sixteen decode steps into one block, each larger than the one before: every step's scale is its own, and earlier tokens stay within
    the roundings that they have seen."""
    rng = np.random.default_rng(9)
    g, d = 2, 64
    b = Bench(rx, rng, 2, g, d, 16, [1], [16], rope=False)
    rows = []
    for t in range(16):
        b.kv_lens = [t + 1]
        b.pool = b.host_pool()
        qkv = half(rng, (1, (2 + 2 * g) * d), std=0.1 * 1.5 ** t)
        check_append(b, qkv, b.append(qkv))
        rows.append(qkv.astype(np.float64).reshape(6, d))
    pool = b.host_pool()
    got = po.values(pool, "v", b.pages, 16, 0, np.arange(16), d)
    for t in range(16):
        # half a step of every scale since: they grow by 1.5 in the mean; half a step of the last one per rounding bounds them all
        assert np.abs(got[t] - rows[t][4:]).max() <= pool["vs"][b.pages[0, 0], :, 0].max() * 0.5 * (16 - t) * 1.01


def test_values_that_are_not_finite(rx):
    rng = np.random.default_rng(3)
    b = Bench(rx, rng, 4, 4, 64, 16, [20], [20], rope=False)
    qkv = half(rng, (20, 12 * 64))
    qkv[3, 256], qkv[3, 520], qkv[18, 300], qkv[18, 600] = np.inf, -np.inf, np.nan, np.nan
    b.append(qkv)
    check_append(b, qkv, None)
    pool = b.host_pool()
    assert np.isfinite(pool["ks"][b.pages[0, 0]]).all() and pool["ks"][b.pages[0, 0], 0, 0] == np.float32(65504.0) / np.float32(127.0)
    out = b.attention(half(rng, (20, 4, 64)))
    assert np.isfinite(out).all()


def test_zeros(rx):
    b = Bench(rx, np.random.default_rng(1), 4, 4, 64, 16, [18], [18])
    qkv = np.zeros((18, 12 * 64), np.float16)
    q_out = b.append(qkv)
    check_append(b, qkv, q_out)
    assert (b.read() == 0).all() and (b.attention(q_out) == 0).all()


def attention_case(rx, rng, shape, page_size, q_lens, kv_lens, slots=None, std=1.0, device_table=False, scale=(0.02, 0.05), edit=None, heads=None):
    b = Bench(rx, rng, *shape, page_size, q_lens, kv_lens, slots, device_table=device_table, scale=scale)
    if edit:
        edit(b)
    q = half(rng, (b.n, b.h, b.d), std)
    got = b.attention(q).astype(np.float64)
    want, tol = po.attention(q.astype(np.float64), b.pool, b.pages, page_size, q_lens, kv_lens, slots, b.g, b.d, heads)
    bad = ~(np.abs(got - want) <= tol)
    if heads is not None:
        bad = bad[:, heads]
        got, want, tol = got[:, heads], want[:, heads], tol[:, heads]
    assert not bad.any(), (int(bad.sum()), np.abs(got - want)[bad][:5], tol[bad][:5])
    return b


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("lens", LENS + [([1, 1], [1500, 700]), ([7], [513]), ([130], [130]), ([64], [1030])],
                         ids=lambda v: "x".join(map(str, v[0])) + "_of_" + "x".join(map(str, v[1])))
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


def test_attention_on_large_scores_and_uneven_scales(rx):
    """Scores of hundreds, so that one token takes the row; blocks whose values differ by 10^6, the small ones alone visible to early rows."""
    attention_case(rx, np.random.default_rng(2), (8, 2, 128), 16, [30, 1], [30, 700], std=40.0)

    def uneven(b):
        for key in ("ks", "vs"):
            b.pool[key] *= (10.0 ** np.random.default_rng(4).uniform(-4, 2, b.pool[key].shape)).astype(np.float32)
            b.dev[key].copy_(torch.from_numpy(b.pool[key]))
    for q_lens, kv_lens in (([200], [200]), ([1], [900]), ([20], [300])):
        attention_case(rx, np.random.default_rng(3), (4, 2, 64), 16, q_lens, kv_lens, edit=uneven)


# Calls whose sequences fill tiles of 256 (row, head) pairs, 160 of them and more over all KV heads: (heads, KV heads, d), q_lens, kv_lens, heads to check
MANY_ROWS = [
    ((80, 80, 64), [300], [300], None),
    ((80, 80, 128), [257], [1000], [0, 1, 40, 79]),
    ((64, 8, 128), [33, 60, 40, 32, 35, 47, 33, 64, 50, 45], [33, 61, 300, 32, 99, 47, 700, 64, 1050, 45], None),
    ((40, 8, 128), [300, 1, 450, 3, 260], [310, 800, 450, 77, 900], [0, 5, 13, 39]),
    ((40, 8, 64), [1001], [1001], [0, 9, 39]),
    ((160, 160, 64), [256], [8200], [0, 77, 159]),                # more blocks than are in LDS at a time
    ((24, 8, 128), [2000], [2000], [2, 23]),
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
        for key in ("ks", "vs"):
            b.pool[key] *= (10.0 ** np.random.default_rng(4).uniform(-4, 2, b.pool[key].shape)).astype(np.float32)
            b.pool[key][:, 17, 0] = np.where(np.isnan(b.pool[key][:, 17, 0]), np.nan, 0.0).astype(np.float32)      # blocks of zeros
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
    for q_lens, kv_lens in (([1, 1], [70, 20]), ([3, 20], [70, 20]), ([70, 20], [70, 20])):
        b = attention_case(rx, rng, (8, 2, 64), 16, q_lens, kv_lens, edit=lose)
        assert b.error() == 4
        out = b.attention(half(rng, (b.n, 8, 64)))
        assert (out[q_lens[0]:] == 0).all()
        b.rx.check(rx.relax_workspace_init(b.dims, b.ws, b.ws_bytes))
        assert b.error() == 0
        k, v = b.read()
        assert (k[q_lens[0]:] == 0).all() and (v[q_lens[0]:] == 0).all() and b.error() == 4
        b.rx.check(rx.relax_workspace_init(b.dims, b.ws, b.ws_bytes))
        qkv = half(rng, (b.n, 12 * 64))
        check_append(b, qkv, b.append(qkv))
        assert b.error() == 4


def test_shared_pages(rx):
    """Two sequences on the same first pages."""
    def share(b):
        b.pages[1, :4] = b.pages[0, :4]
        b.dev_pages.copy_(torch.from_numpy(b.pages))
        for key in ("ks", "vs"):                                # (pages that sequence 1 no longer names were never reached)
            assert np.isfinite(b.pool[key][b.pages[0, :4]]).all()
    attention_case(rx, np.random.default_rng(12), (8, 2, 128), 16, [1, 30], [90, 111], edit=share)


def test_pool_beyond_32_bits(rx):
    """Blocks whose codes lie more than 4 GiB into the pool."""
    rng = np.random.default_rng(13)
    g, d, page_size = 2, 128, 256
    per_page = g * page_size * d
    n_pages = (1 << 32) // per_page + 40
    dims = rx.make_dims(4 * d, 4, g, d, 64, 2 * page_size, 1)
    k, v = (torch.empty(n_pages * per_page, dtype=torch.uint8, device="cuda") for _ in "kv")
    ks, vs = (torch.empty(n_pages * g * page_size // 16, dtype=torch.float32, device="cuda") for _ in "kv")
    ids = [n_pages - 2, n_pages - 31]
    pages = torch.tensor([ids], dtype=torch.int32, device="cuda")
    cache = rx.PagedCache(k, v, ks, vs, pages, None, n_pages, page_size, 2)
    ws_bytes = rx.relax_paged_workspace_bytes(dims, 400, 400, 1)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    x = torch.from_numpy(half(rng, (400, 8 * d))).cuda()
    q = torch.empty((400, 4, d), dtype=torch.float16, device="cuda")
    base = x.data_ptr()
    rx.check(rx.relax_paged_append(base, 8 * d, base + 8 * d, base + 12 * d, 8 * d, q, cache, rx.Seqs([400], [400]), dims, 400, ws, ws_bytes))
    out = torch.empty((2, 4, d), dtype=torch.float16, device="cuda")
    rx.check(rx.relax_paged_attention(q[-2:], cache, rx.Seqs([2], [400]), dims, out, 2, ws, ws_bytes))
    back = torch.empty((2, 400, g, d), dtype=torch.float16, device="cuda")
    rx.check(rx.relax_paged_read(cache, rx.Seqs([400], [400]), dims, back[0], back[1], 400, ws, ws_bytes))
    full = torch.empty((400, 4, d), dtype=torch.float16, device="cuda")
    rx.check(rx.relax_paged_attention(q, cache, rx.Seqs([400], [400]), dims, full, 400, ws, ws_bytes))
    torch.cuda.synchronize()
    pool = {name: t.view(n_pages, g, page_size // 16, -1)[ids].cpu().numpy() for name, t in (("k", k), ("v", v))}
    pool.update({name: t.view(n_pages, g, page_size // 16)[ids].cpu().numpy() for name, t in (("ks", ks), ("vs", vs))})
    local = np.array([[0, 1]], np.int32)
    want, tol = po.attention(q.cpu().numpy().astype(np.float64), pool, local, page_size, [400], [400], None, g, d)
    for got, rows in ((full, slice(0, 400)), (out, slice(398, 400))):
        assert (np.abs(got.cpu().numpy().astype(np.float64) - want[rows]) <= tol[rows]).all()
    for name, got in (("k", back[0]), ("v", back[1])):
        vals = po.values(pool, name, local, page_size, 0, np.arange(400), d)
        assert np.array_equal(got.cpu().numpy(), vals.astype(np.float32).astype(np.float16))
        assert np.abs(vals - x.cpu().numpy().astype(np.float64).reshape(400, 8, d)[:, 4 if name == "k" else 6:][:, :g]).max() < 0.02


def test_a_prompt_and_decode_steps_together(rx):
    """A serving program's run: a prompt in two chunks, then tokens one by one, two sequences of different lengths, each step append and attention;
    attention meets what the reads give, and stays near the dense fp16 cache's."""
    rng = np.random.default_rng(21)
    h, g, d, cap = 8, 2, 64, 128
    b = Bench(rx, rng, h, g, d, 32, [1, 1], [cap, cap])
    dense_dims = rx.make_dims(h * d, h, g, d, 64, cap, 2)
    dk, dv = (torch.zeros((2, cap, g, d), dtype=torch.float16, device="cuda") for _ in "kv")
    dense = rx.KVCache(dk, dv, b.table)
    dws_bytes = rx.relax_workspace_bytes(dense_dims, 64, cap, 2)
    dws = torch.empty(dws_bytes, dtype=torch.uint8, device="cuda")
    at = [0, 0]
    for step in [[37, 20], [21, 1]] + [[1, 1]] * 9:
        at = [a + s for a, s in zip(at, step)]
        b.q_lens, b.kv_lens, b.n = step, list(at), sum(step)
        qkv = half(rng, (b.n, (h + 2 * g) * d))
        q = b.append(qkv)
        got = b.attention(q).astype(np.float64)
        pool = b.host_pool()
        want, tol = po.attention(q.astype(np.float64), pool, b.pages, 32, step, at, None, g, d)
        assert (np.abs(got - want) <= tol).all()
        x = torch.from_numpy(qkv).cuda()
        rx.check(rx.relax_rmsnorm_rope(None, None, None, b.n, h * d, 1e-5, x, dense_dims, dense, rx.Seqs(step, at)))
        qd = x[:, :h * d].contiguous()
        out = torch.empty_like(qd)
        rx.check(rx.relax_attention(qd, dense, rx.Seqs(step, at), dense_dims, out, b.n, dws, dws_bytes))
        torch.cuda.synchronize()
        turned = qd.cpu().numpy().reshape(q.shape).astype(np.float64)
        assert (np.abs(turned - q) <= 2.0 ** -10 * np.abs(turned) + 2.0 ** -20).all()     # the same rotation, each rounded once
        # |x| < 5.5, so a scale is below 0.0433 and a value off by 0.022 per rounding, 0.04 with a scale that grew; scores by
        # sum |q| 0.04 / 8 < 64 * 0.8 * 0.02 / 8 = 0.13 in the mean of |q| and of the errors, weights by e^0.13, twice, on values near 1
        assert np.abs(got - out.cpu().numpy().astype(np.float64).reshape(got.shape)).max() < 0.04 + 2 * 0.13
    assert b.error() == 0


def test_steps_in_a_graph_follow_the_table(rx):
    """Append and attention captured once with upper bounds, replayed while the device table counts up; every replay against an eager call on a
    second pool, other work in between."""
    rng = np.random.default_rng(30)
    h, g, d, page = 8, 2, 128, 16
    q_lens = [1, 1, 1]
    b, e = (Bench(rx, np.random.default_rng(31), h, g, d, page, q_lens, [640, 640, 640], device_table=True) for _ in range(2))
    lens = [5, 300, 31]
    x = torch.zeros((3, (h + 2 * g) * d), dtype=torch.float16, device="cuda")
    outs = {}
    for name, bench in (("graph", b), ("eager", e)):
        outs[name] = [torch.empty((3, h, d), dtype=torch.float16, device="cuda") for _ in range(2)]
        bench.workspace()
    side = torch.cuda.Stream()

    def step(bench, name, stream):
        base, row = x.data_ptr(), x.shape[1]
        q, out = outs[name]
        seqs = bench.seqs()
        rx.check(rx.relax_paged_append(base, row, base + 2 * h * d, base + 2 * (h + g) * d, row, q, bench.cache, seqs, bench.dims, 3, bench.ws, bench.ws_bytes, stream))
        rx.check(rx.relax_paged_attention(q, bench.cache, seqs, bench.dims, out, 3, bench.ws, bench.ws_bytes, stream))
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
            rx.check(rx.relax_paged_attention(qd[i], b[i].cache, b[i].seqs(), b[i].dims, out[i], 4, *b[i].workspace(), streams[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert np.array_equal(out[i].cpu().numpy(), alone[i])


@pytest.mark.parametrize("shape,q_lens,heads", [((16, 1, 64), [1500] + [1] * 299, [0, 15]), ((64, 8, 64), [1] * 150 + [700] + [1] * 150, [0, 63]),
                                                ((8, 2, 64), [2, 31, 1, 1, 3] * 40, None)], ids=["small_tiles", "large_tiles", "ragged"])
@pytest.mark.parametrize("device_table", [False, True])
def test_one_prompt_among_many_sequences(rx, shape, q_lens, heads, device_table):
    """As many tiles for every sequence as the prompt has would be 450 000; and sequences that begin and end inside the search's groups of 64."""
    rng = np.random.default_rng(71)
    attention_case(rx, rng, shape, 16, q_lens, [q + int(rng.integers(0, 60)) for q in q_lens], device_table=device_table, heads=heads)


def test_queries_in_place(rx):
    rng = np.random.default_rng(72)
    b = Bench(rx, rng, 4, 2, 64, 16, [5, 1], [20, 3])
    x = torch.from_numpy(half(rng, (b.n, 8 * 64))).cuda()
    q, kv = x[:, :256].contiguous(), x[:, 256:].contiguous()
    at = kv.data_ptr()
    args = lambda q_ptr, stride, out: rx.relax_paged_append(q_ptr, stride, at, at + 256, 256, out, b.cache, b.seqs(), b.dims, b.n, *b.workspace())
    out = torch.empty_like(q)
    rx.check(args(q, 256, out))
    rx.check(args(q, 256, q))
    torch.cuda.synchronize()
    assert torch.equal(q, out)


def test_a_model_of_one_layer_from_prompt_to_log_probabilities(rx):
    """Matrices, append, attention, the head and the log probabilities as a program strings them together: three requests of different ages,
    a prompt scored token by token, then tokens picked with alternatives.  Attention against float64 on what the cache reads back as,
    log probabilities against float64 on the logits; the first alternative is the next token."""
    from paper_2311_02103_amd import runtime
    rng = np.random.default_rng(73)
    h, g, d, V, H = 8, 2, 64, 1000, 256
    mat = lambda m, k: torch.from_numpy(half(rng, (m, k), k ** -0.5)).cuda()
    emb, wqkv, wo, head = torch.from_numpy(half(rng, (V, H))).cuda(), mat((h + 2 * g) * d, H), mat(H, h * d), mat(V, H) * 4
    cache = runtime.DevicePagedCache(n_heads=h, n_kv_heads=g, head_dim=d, kv_capacity=160, n_pages=30, page_size=16, kv_slots=3, n_max=200)
    cache.pages.copy_(torch.from_numpy(rng.permutation(30).reshape(3, 10).astype(np.int32)))

    def product(x, w):
        y = torch.empty((x.shape[0], w.shape[0]), dtype=torch.float16, device="cuda")
        rx.check(rx.relax_half_matmul(x, w, y, x.shape[0], w.shape[0], w.shape[1]))
        return y
    held = [0, 0, 0]
    texts = [rng.integers(0, V, 120).astype(np.int32) for _ in range(3)]
    for slots, lens in (([1], [97]), ([2, 0, 1], [33, 60, 1]), ([0, 1, 2], [1, 1, 1]), ([2, 0], [1, 4]), ([1, 2, 0], [1, 1, 1])):
        for s, ln in zip(slots, lens):
            held[s] += ln
        ids = np.concatenate([texts[s][held[s] - ln:held[s]] for s, ln in zip(slots, lens)])
        targets = np.concatenate([texts[s][held[s] - ln + 1:held[s] + 1] for s, ln in zip(slots, lens)])
        kv_lens = [held[s] for s in slots]
        seqs = rx.Seqs(lens, kv_lens, slots)
        x = emb[torch.from_numpy(ids).cuda()]
        q = cache.append(product(x, wqkv), seqs)
        o = cache.attention(q, seqs)
        y = x + product(o.view(-1, h * d), wo)
        logits = product(y, head)
        lp, ent, top_ids, tops = runtime.token_logprobs(logits, torch.from_numpy(targets).cuda(), 5, True)
        pool = {key: t.cpu().numpy() for key, t in (("k", cache.k), ("v", cache.v), ("ks", cache.k_scale), ("vs", cache.v_scale))}
        want, tol = po.attention(q.cpu().numpy().astype(np.float64), pool, cache.pages.cpu().numpy(), 16, lens, kv_lens, slots, g, d)
        assert (np.abs(o.cpu().numpy() - want) <= tol).all()
        k, v = cache.read(seqs, len(ids))
        for row, ql, L, slot in po.sequences(lens, kv_lens, slots):
            for name, got in (("k", k), ("v", v)):
                vals = po.values(pool, name, cache.pages.cpu().numpy(), 16, slot, np.arange(L - ql, L), d)
                assert np.array_equal(got[row:row + ql].cpu().numpy(), vals.astype(np.float32).astype(np.float16))
        l64 = logits.cpu().numpy().astype(np.float64)
        wlp, went, wids, wtops = po.token_logprobs(l64, targets, 5)
        # a term e^z is off by 2^-23 |z| log2(e) and 2^-22, |z| weighted by e^z averages below log V + 1: log S by 2^-22 (log V + 4) = 2^-22 11, the entropy by log V + 2 < 9
        # times that, and the results' own rounding 2^-22 of less than 20: below 2^-22 128 together
        assert np.array_equal(top_ids.cpu().numpy(), wids)
        for got, ref in ((lp, wlp), (tops, wtops), (ent, went)):
            assert np.abs(got.cpu().numpy() - ref).max() <= 2.0 ** -15
        for s, row in zip(slots, np.cumsum(lens) - 1):
            texts[s][held[s]] = top_ids[row, 0].item()
    assert rx.relax_workspace_error(cache.dims, cache.ws) == 0


def test_lengths_of_a_device_table_beyond_the_capacity(rx):
    """Known on the device only: such a sequence has no pages, and the rotary table no rows for it."""
    rng = np.random.default_rng(74)
    b = Bench(rx, rng, 4, 2, 64, 16, [3, 20, 1], [20, 32, 9], device_table=True)
    b.dev_table[2, 1] = b.cap + 500
    qkv = half(rng, (b.n, 8 * 64))
    b.append(qkv)
    assert b.error() == 4
    got, blocks = b.host_pool(), b.pages[1][b.pages[1] >= 0]
    for key in got:                                            # nothing of its pages was touched, the others' rows are in
        assert np.array_equal(got[key][blocks].view(np.uint8), b.pool[key][blocks].view(np.uint8)), key
    others = np.r_[0:3, 23:24]
    k, v = b.read()
    assert (k[3:23] == 0).all() and (v[3:23] == 0).all()
    x = qkv.astype(np.float64).reshape(b.n, 8, 64)
    assert np.abs(v[others] - x[others, 6:]).max() <= np.abs(x).max() / 127 + 2.0 ** -9


def test_python_side_checks_and_layers_that_share_a_workspace(rx):
    from paper_2311_02103_amd import runtime
    rng = np.random.default_rng(75)
    first = runtime.DevicePagedCache(n_heads=4, n_kv_heads=2, head_dim=64, kv_capacity=64, n_pages=4, page_size=16, n_max=40, rope_base=None)
    second = runtime.DevicePagedCache(n_heads=4, n_kv_heads=2, head_dim=64, kv_capacity=64, n_pages=4, page_size=16, n_max=40, share_from=first)
    first.pages.copy_(torch.tensor([[2, 0, 3, 1]], dtype=torch.int32))
    seqs, x = rx.Seqs([40], [40]), [torch.from_numpy(half(rng, (40, 8 * 64))).cuda() for _ in range(2)]
    for layer, rows in zip((first, second), x):
        q = layer.append(rows, seqs)
        assert torch.equal(q.view(40, 256), rows[:, :256])                             # no rotary table: q as it is
    for layer, rows in zip((first, second), x):
        k, v = layer.read(seqs, 40)
        off = (torch.stack([k, v], 1) - rows[:, 256:].view(40, 2, 2, 64)).abs().max().item()
        assert off <= rows.abs().max().item() * (0.5 / 127 + 2.0 ** -10)               # half a step of a block's scale, and the rounding to fp16
        one = layer.append(rows[39:, :].as_strided((1, 512), (1, 1)), rx.Seqs([1], [41]))      # one row: any stride
        assert torch.equal(one.view(-1), rows[39, :256])
    with pytest.raises(ValueError):
        first.append(x[0].float(), seqs)
    with pytest.raises(ValueError):
        first.append(x[0][:, :-8], seqs)
    with pytest.raises(ValueError):
        first.attention(torch.empty((40, 64, 4), dtype=torch.float16, device="cuda").transpose(1, 2), seqs)
    with pytest.raises(rx.RelaxError):
        first.append(torch.empty((41, 512), dtype=torch.float16, device="cuda"), rx.Seqs([41], [64 + 1]))
    with pytest.raises(ValueError):
        runtime.token_logprobs(x[0], torch.zeros(40, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        runtime.token_logprobs(x[0].float())
    assert rx.relax_workspace_error(first.dims, first.ws) == 0


# (heads, KV heads, d), page, q_lens, kv_lens: calls of tiles of 16 pairs in several splits, in one, and of tiles of 256 pairs
DEVICE_LENGTHS = {"splits": ((4, 2, 64), 16, [1, 2, 1], [1100, 1500, 40]), "splits_128": ((8, 2, 128), 64, [3, 1], [900, 2000]),
                  "one_split": ((32, 32, 64), 16, [1] * 9, [30, 200, 77, 16, 100, 5, 64, 33, 90]), "rows": ((80, 80, 64), 16, [300, 270], [300, 296]),
                  "both_kernels": ((40, 40, 128), 16, [400, 2, 260, 300], [408, 70, 360, 300])}


@pytest.mark.parametrize("kind", sorted(DEVICE_LENGTHS))
def test_attention_on_lengths_of_a_device_table_beyond_the_capacity(rx, kind):
    """Known on the device only: such a sequence has no token, which gives zeros and the flag, and the others are what they are without it; with host
    bounds at the capacity and far below it."""
    shape, page, q_lens, kv_lens = DEVICE_LENGTHS[kind]
    b = Bench(rx, np.random.default_rng(76), *shape, page, q_lens, kv_lens, device_table=True)
    q = half(np.random.default_rng(77), (b.n, b.h, b.d))
    dev, (ws, ws_bytes) = torch.from_numpy(q).cuda(), b.workspace()
    starts = np.concatenate([[0], np.cumsum(q_lens)])
    for bounds in ([b.cap] * len(q_lens), kv_lens):
        out = torch.empty_like(dev)
        call = lambda: rx.check(rx.relax_paged_attention(dev, b.cache, rx.Seqs(q_lens, bounds, None, b.dev_table), b.dims, out, b.n, ws, ws_bytes))
        rx.check(rx.relax_workspace_init(b.dims, ws, ws_bytes))
        b.dev_table[2] = torch.tensor(kv_lens, dtype=torch.int32)
        call()
        clean = out.clone()
        assert b.error() == 0
        for lost in {0, len(q_lens) - 1}:
            for length in (b.cap + 1, b.cap + 500, 2 ** 31 - 1):
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
    """Lengths of the table that the bounds of the host fall short of, within the capacity: all their tokens count."""
    q_lens, kv_lens, shape = [1, 2], [3000, 41], (8, 2, 64)
    b = Bench(rx, np.random.default_rng(78), *shape, 32, q_lens, kv_lens, device_table=True)
    q = half(np.random.default_rng(79), (b.n, 8, 64))
    dev = torch.from_numpy(q).cuda()
    out = torch.empty_like(dev)
    ws_bytes = rx.relax_paged_workspace_bytes(b.dims, b.n, bound, 2)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    rx.check(rx.relax_workspace_init(b.dims, ws, ws_bytes))
    rx.check(rx.relax_paged_attention(dev, b.cache, rx.Seqs(q_lens, [bound, 41 if bound > 41 else 2], None, b.dev_table), b.dims, out, b.n, ws, ws_bytes))
    want, tol = po.attention(q.astype(np.float64), b.pool, b.pages, 32, q_lens, kv_lens, None, 2, 64)
    assert (np.abs(out.cpu().numpy().astype(np.float64) - want) <= tol).all()
    assert rx.relax_workspace_error(b.dims, ws) == 0


@pytest.mark.parametrize("by_address", [False, True])
def test_python_calls_on_a_stream_of_their_own(rx, by_address):
    """Append, attention, read and log probabilities on a side stream that starts late, with nothing but what the calls allocate, against the same on
    the current stream; the current stream allocates and writes in between."""
    from paper_2311_02103_amd import runtime
    rng = np.random.default_rng(80)
    make = lambda: runtime.DevicePagedCache(n_heads=8, n_kv_heads=2, head_dim=64, kv_capacity=512, n_pages=16, page_size=32, n_max=500)
    here, there = make(), make()
    for layer in (here, there):
        layer.pages.copy_(torch.arange(16, dtype=torch.int32).view(1, 16))
    x = torch.from_numpy(half(rng, (500, 12 * 64))).cuda()
    logits, targets = torch.from_numpy(half(rng, (3, 70001), 3)).cuda(), torch.tensor([5, 70000, 12345], dtype=torch.int32, device="cuda")
    seqs = rx.Seqs([500], [500])

    def run(layer, stream):
        q = layer.append(x, seqs, stream=stream)
        return (q, layer.attention(q, seqs, stream=stream), *layer.read(seqs, 500, stream=stream), *runtime.token_logprobs(logits, targets, 7, True, stream=stream))
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


@pytest.mark.parametrize("shape", [(4, 2, 64), (8, 4, 128)], ids=str)
def test_rotated_keys_that_are_not_finite_or_near_the_limit(rx, shape):
    """Infinities and NaNs are replaced in the inputs, so that a pair's other element is what its finite input gives, at position 0 too; a pair near
    fp16's limit is held as it is behind the rotation, up to 65504 * sqrt 2."""
    rng = np.random.default_rng(81)
    h, g, d = shape
    b = Bench(rx, rng, h, g, d, 16, [40], [40])
    qkv = half(rng, (40, (h + 2 * g) * d))
    k = qkv[:, h * d:(h + g) * d].reshape(40, g, d)
    k[0, 0, 3], k[0, 0, 5 + d // 2], k[0, 1, 7], k[17, 1, 2], k[18, 0, 9] = np.inf, -np.inf, np.nan, np.nan, -np.inf
    k[32:, 0, 1], k[32:, 0, 1 + d // 2] = 65504, -65504
    qkv[:, h * d:(h + g) * d] = k.reshape(40, g * d)
    b.append(qkv)
    pool = b.host_pool()
    want = np.stack([po.rotate(po.storable(k[t].astype(np.float64)), t, d) for t in range(40)])
    assert np.abs(want[32:]).max() > 80000
    index = po.code_index("k", d)
    for first in (0, 16, 32):
        page, block = b.pages[0, first // 16], want[first:first + 16]
        for head in range(g):
            s = pool["ks"][page, head, 0]
            # as check_append: the scale within 2^-21, a code within half a step and 1e-4, since |a| + |b| of a pair is at most twice the block's maximum
            assert abs(s - np.abs(block[:, head]).max() / 127) <= 2.0 ** -21 * s
            codes = pool["k"][page, head, 0][index].astype(np.float64) - 128
            assert np.abs(codes[:len(block)] - block[:, head] / np.abs(block[:, head]).max() * 127).max() <= 0.5 + 1e-4
    out, tol = po.attention(half(np.random.default_rng(82), (40, h, d)).astype(np.float64), pool, b.pages, 16, [40], [40], None, g, d)
    got = b.attention(half(np.random.default_rng(82), (40, h, d)))
    assert (np.abs(got - out) <= tol).all()
    back, vals = b.read()[0], po.values(pool, "k", b.pages, 16, 0, np.arange(40), d)
    with np.errstate(over="ignore"):
        assert np.array_equal(back, vals.astype(np.float32).astype(np.float16))


def test_append_and_read_on_device_lengths_next_to_the_end_of_their_type(rx):
    """Lengths whose last block ends behind 2^31: no page, no row of another sequence touched."""
    rng = np.random.default_rng(83)
    b = Bench(rx, rng, 4, 2, 64, 16, [3, 20, 1], [20, 32, 9], device_table=True)
    qkv = half(rng, (b.n, 8 * 64))
    for length in (2 ** 31 - 1, 2 ** 31 - 5, 2 ** 31 - 16, 2 ** 31 - 17):
        for lost, rows in ((0, slice(0, 3)), (1, slice(3, 23))):
            b.dev_table[2] = torch.tensor([20, 32, 9], dtype=torch.int32)
            rx.check(rx.relax_workspace_init(b.dims, b.ws, b.ws_bytes))
            b.append(qkv)
            k, v = b.read()
            assert b.error() == 0
            b.dev_table[2, lost] = length
            held = b.host_pool()
            b.append(qkv)
            assert b.error() == 4
            again = b.host_pool()
            for key in held:
                assert np.array_equal(held[key].view(np.uint8), again[key].view(np.uint8)), (length, lost, key)
            got = b.read()
            assert (got[:, rows] == 0).all()
            keep = np.ones(b.n, bool)
            keep[rows] = False
            assert np.array_equal(got[0][keep], k[keep]) and np.array_equal(got[1][keep], v[keep])


@pytest.mark.parametrize("kind", ["splits", "rows"])
def test_device_lengths_below_zero(rx, kind):
    """Not a length: nothing is read or written for it, whatever the other sequences do."""
    shape, page, q_lens, kv_lens = DEVICE_LENGTHS[kind]
    b = Bench(rx, np.random.default_rng(84), *shape, page, q_lens, kv_lens, device_table=True)
    qkv = half(np.random.default_rng(85), (b.n, (b.h + 2 * b.g) * b.d))
    q = b.append(qkv)
    clean, held = b.attention(q), b.host_pool()
    first = q_lens[0]
    for length in (-1, -1000, -2 ** 31, -2 ** 31 + 2):
        b.dev_table[2, 0] = length
        assert np.array_equal(b.append(qkv)[first:], q[first:])
        out, again = b.attention(q), b.host_pool()
        assert (out[:first] == 0).all() and np.array_equal(out[first:], clean[first:]), length
        for key in held:
            assert np.array_equal(held[key].view(np.uint8), again[key].view(np.uint8)), (length, key)
