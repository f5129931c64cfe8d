"""relax_token_logprobs on the GPU against a plain implementation in 64 bits."""
import numpy as np
import pytest

import paged_oracle as po

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def rx():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2311_02103_amd import binding
    binding.lib()
    return binding


def call(rx, x, targets, top, offset=0, pad=0, ws=True):
    """x: host fp16 [n, V], placed at `offset` elements into a buffer with rows V + pad apart."""
    n, V = x.shape
    buf = torch.full((offset + n * (V + pad) + 8,), 60000.0, dtype=torch.float16, device="cuda")      # logits of other rows must not count
    buf[offset:offset + n * (V + pad)].view(n, V + pad)[:, :V] = torch.from_numpy(x).cuda()
    t = None if targets is None else torch.from_numpy(targets.astype(np.int32)).cuda()
    lp = None if targets is None else torch.full((n,), 7.0, device="cuda")
    ent = torch.full((n,), 7.0, device="cuda")
    ids = torch.full((n, top), -5, dtype=torch.int32, device="cuda")
    tops = torch.full((n, top), 7.0, device="cuda")
    b = rx.relax_token_logprobs_workspace_bytes(n, V, top)
    w = torch.full((b,), 0xFF, dtype=torch.uint8, device="cuda") if ws else None
    rx.check(rx.relax_token_logprobs(buf.data_ptr() + 2 * offset, V + pad, t, lp, ent, ids if top else None, tops if top else None, n, V, top, w, b if ws else 0))
    torch.cuda.synchronize()
    return (None if lp is None else lp.cpu().numpy()), ent.cpu().numpy(), ids.cpu().numpy(), tops.cpu().numpy()


def check(x, targets, top, got):
    """A term e^z is off by 2^-23 of |z| log2(e) (its exponent's rounding) and 2^-22; weighted by e^z, |z| averages below log V + 1.  So log S is
    off by 2^-22 (log V + 4) at most, a log probability by that and its own rounding, the entropy by log V + 1 times as much."""
    lp, ent, ids, tops = po.token_logprobs(x.astype(np.float64), targets, top)
    slack = 2.0 ** -22 * (np.log(x.shape[1]) + 4)
    assert np.array_equal(got[2], ids)
    for name, a, b, tol in (("logprobs", got[0], lp, slack), ("entropy", got[1], ent, slack * (np.log(x.shape[1]) + 2)), ("top", got[3], tops, slack)):
        if a is None:
            continue
        same = (np.isnan(a) & np.isnan(b)) | (a == b)
        with np.errstate(invalid="ignore"):
            assert (same | (np.abs(a - b) <= tol + 2.0 ** -22 * np.abs(b))).all(), (name, a[~same][:5], b[~same][:5])


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("n,V,top", [(1, 1, 1), (1, 7, 7), (3, 33, 32), (2, 100, 0), (5, 688, 5), (1, 32000, 5), (4, 32000, 20), (2, 32761, 32), (2, 32762, 1),
                                     (1, 50257, 10), (2, 65530, 3), (2, 128256, 32), (1, 152064, 20), (2, 163833, 8), (2, 163834, 8), (1, 262144, 32), (256, 32762, 3), (3, 262016, 32), (2, 262017, 32)])
def test_rows(rx, n, V, top, ws):
    rng = np.random.default_rng(V)
    x = (rng.standard_normal((n, V)) * 2.5).astype(np.float16)
    t = rng.integers(0, V, n)
    check(x, t, top, call(rx, x, t, top, ws=ws))


@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5), (8, 8), (7, 1)])
@pytest.mark.parametrize("V", [1, 9, 1001, 33001, 64007])
def test_alignment_and_strides(rx, offset, pad, V):
    rng = np.random.default_rng(V + offset)
    x = (rng.standard_normal((3, V)) * 3).astype(np.float16)
    t = rng.integers(0, V, 3)
    check(x, t, min(V, 6), call(rx, x, t, min(V, 6), offset, pad))


ROWS = {
    "equal": lambda rng, V: np.full(V, 1.5),
    "two values": lambda rng, V: rng.integers(0, 2, V) * 2.0,
    "signed zeros": lambda rng, V: np.where(rng.integers(0, 2, V) == 0, 0.0, -0.0),
    "ascending": lambda rng, V: np.arange(V) * (20.0 / V),
    "descending": lambda rng, V: np.arange(V)[::-1] * (20.0 / V),
    "one certain": lambda rng, V: np.where(np.arange(V) == V // 3, 40.0, rng.standard_normal(V)),
    "masked but five": lambda rng, V: np.where(np.arange(V) % (V // 5 + 1) == 3, rng.standard_normal(V), -np.inf),
    "all masked": lambda rng, V: np.full(V, -np.inf),
    "lowest value": lambda rng, V: np.where(np.arange(V) == V - 1, 0.0, -65504.0),
    "all lowest": lambda rng, V: np.full(V, -65504.0),
    "large": lambda rng, V: rng.standard_normal(V) * 20000,
    "one NaN": lambda rng, V: np.where(np.arange(V) == 2, np.nan, rng.standard_normal(V)),
    "NaN and masked": lambda rng, V: np.where(np.arange(V) % 3 == 0, np.nan, -np.inf),
    "all NaN": lambda rng, V: np.full(V, np.nan),
    "one infinite": lambda rng, V: np.where(np.arange(V) == V // 2, np.inf, rng.standard_normal(V)),
    # the 2000 largest logits where a few thread groups own them: more than the candidate list holds
    "bunched": lambda rng, V: np.where(np.arange(V) // 8 % 64 < 3, 10.0 + rng.standard_normal(V), rng.standard_normal(V)),
}


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("kind", sorted(ROWS))
@pytest.mark.parametrize("V,top", [(40, 32), (32000, 20), (152064, 32), (200000, 5)])
def test_unusual_rows(rx, kind, V, top, ws):
    rng = np.random.default_rng(1)
    x = np.stack([ROWS[kind](rng, V), rng.standard_normal(V) * 2.5]).astype(np.float16)
    t = np.array([V // 3, 0])
    check(x, t, top, call(rx, x, t, top, ws=ws))


def test_targets_outside_and_no_targets(rx):
    rng = np.random.default_rng(4)
    x = rng.standard_normal((4, 500)).astype(np.float16)
    t = np.array([-1, 500, 2 ** 31 - 1, 499])
    got = call(rx, x, t, 3)
    check(x, t, 3, got)
    assert (got[0][:3] == -np.inf).all()
    check(x, None, 3, call(rx, x, None, 3))


def test_a_certain_token_keeps_its_digits(rx):
    """log p = -log1p(rest): about -1e-9 here, which 1 + rest in 32 bits has lost."""
    x = np.full((1, 1000), -9.0, np.float16)
    x[0, 17] = 18.5
    got = call(rx, x, np.array([17]), 1)
    want = -np.log1p(999 * np.exp(-27.5))
    assert abs(got[0][0] - want) <= 1e-4 * abs(want) and got[3][0, 0] == got[0][0]


def test_many_rows_do_not_touch_each_other(rx):
    rng = np.random.default_rng(6)
    x = (rng.standard_normal((700, 4099)) * 2).astype(np.float16)
    t = rng.integers(0, 4099, 700)
    got = call(rx, x, t, 4, offset=5, pad=2)
    check(x, t, 4, got)
    # the row by itself; it is aligned otherwise there, so its sums are taken in another order
    check(x[350:351], t[350:351], 4, call(rx, x[350:351], t[350:351], 4, ws=False))


def test_behind_a_head_and_in_a_graph(rx):
    """Hidden rows through the vocabulary projection, then their log probabilities: eagerly and replayed from a graph."""
    rng = np.random.default_rng(7)
    n, H, V, top = 9, 256, 2000, 8
    h = torch.from_numpy(rng.standard_normal((n, H)).astype(np.float16)).cuda()
    w = torch.from_numpy((rng.standard_normal((V, H)) * 0.1).astype(np.float16)).cuda()
    t = torch.from_numpy(rng.integers(0, V, n).astype(np.int32)).cuda()
    logits = torch.empty((n, V), dtype=torch.float16, device="cuda")
    out = [torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, top), dtype=torch.int32, device="cuda"), torch.empty((n, top), device="cuda")]
    b = rx.relax_token_logprobs_workspace_bytes(n, V, top)
    ws = torch.empty(b, dtype=torch.uint8, device="cuda")

    def step(stream=None):
        rx.check(rx.relax_half_matmul(h, w, logits, n, V, H, stream))
        rx.check(rx.relax_token_logprobs(logits, V, t, *out, n, V, top, ws, b, stream))
    step()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    for _ in range(4):
        h.copy_(torch.from_numpy(rng.standard_normal((n, H)).astype(np.float16)))
        graph.replay()
        torch.cuda.synchronize()
        x, got = logits.cpu().numpy(), [o.cpu().numpy() for o in out]
        check(x, t.cpu().numpy(), top, got)
        step()
        _ = torch.randn(300, 300, device="cuda").sum()
        torch.cuda.synchronize()
        for a, o in zip(got, out):
            assert np.array_equal(a, o.cpu().numpy())


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("V,top", [(9, 9), (40, 32), (32000, 20), (152064, 32), (200000, 5)])
def test_infinite_rows_with_masked_tokens(rx, V, top, ws):
    """A +inf leaves no log probability but that of a token at -inf, in the vocabulary or outside; a NaN leaves none."""
    rng = np.random.default_rng(9)
    x = (rng.standard_normal((12, V)) * 2.5).astype(np.float16)
    x[:, V // 4], x[:, V // 2], x[:, 0] = -np.inf, np.inf, 0.0
    x[4:8, 1:] = np.where(rng.integers(0, 3, (4, V - 1)) == 0, np.inf, -np.inf)
    x[8:, V - 1] = np.nan
    t = np.array([V // 4, V // 2, 0, V] * 3)
    x[4, t[4]], x[5, t[5]] = -np.inf, np.inf
    got = call(rx, x, t, top, ws=ws)
    check(x, t, top, got)
    assert got[0][0] == got[0][3] == got[0][4] == got[0][7] == -np.inf and np.isnan(np.r_[got[0][1:3], got[0][5:7], got[0][8:], got[1]]).all()


def test_more_rows_than_a_launch_has_threads_for(rx):
    """2^24 + 300 rows of two logits, a workgroup of 256 threads each; closed form in 64 bits, tolerances as in check()."""
    n, V = (1 << 24) + 300, 2
    x = torch.randn((n, V), device="cuda", generator=torch.Generator(device="cuda").manual_seed(10)).half()
    t = torch.randint(0, V, (n,), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(11))
    lp, ent, tops = (torch.full((n,), 7.0, device="cuda") for _ in range(3))
    ids = torch.full((n,), -5, dtype=torch.int32, device="cuda")
    rx.check(rx.relax_token_logprobs(x, V, t, lp, ent, ids, tops, n, V, 1))
    d = x.double()
    d = d[:, 1] - d[:, 0]
    want = torch.stack([-torch.log1p(torch.exp(d)), -torch.log1p(torch.exp(-d))], 1)
    slack = 2.0 ** -22 * (np.log(V) + 4)
    assert torch.equal(ids, (d > 0).to(torch.int32))
    for got, ref, tol in ((lp, want.gather(1, t.long()[:, None])[:, 0], slack), (tops, want.max(1).values, slack), (ent, -(want.exp() * want).sum(1), slack * (np.log(V) + 2))):
        assert bool(((got.double() - ref).abs() <= tol + 2.0 ** -22 * ref.abs()).all())
