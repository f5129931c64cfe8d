"""Host-side contract of the paged cache calls and of relax_token_logprobs: every refusal comes before anything is enqueued, and the plain
implementation that the GPU tests use is pinned to the layout's definition."""
import numpy as np

import paged_oracle as po
from paper_2311_02103_amd import binding as rx

P = 0x10000   # a non-null fake device address


def dims(**kw):
    base = dict(hidden=256, n_heads=4, n_kv_heads=4, head_dim=64, ffn=688, kv_capacity=64, kv_slots=2)
    base.update(kw)
    return rx.make_dims(**base)


def cache(**kw):
    a = dict(k=P, v=P, k_scale=P, v_scale=P, pages=P, rope=P, n_pages=10, page_size=16, pages_per_slot=4)
    a.update(kw)
    return rx.PagedCache(*[a[k] for k in ("k", "v", "k_scale", "v_scale", "pages", "rope", "n_pages", "page_size", "pages_per_slot")])


BIG = 1 << 26


def calls(c, s, d, n, ws=P, ws_bytes=BIG):
    return {rx.relax_paged_append(P, 256, P, P, 256, P, c, s, d, n, ws, ws_bytes), rx.relax_paged_attention(P, c, s, d, P, n, ws, ws_bytes),
            rx.relax_paged_read(c, s, d, P, P, n, ws, ws_bytes)}


def test_what_the_paged_calls_refuse_alike():
    d, s, ok = dims(), rx.Seqs([2], [5]), cache()
    for name in ("k", "v", "k_scale", "v_scale", "pages"):
        assert calls(cache(**{name: None}), s, d, 2) == {rx.ERR_NULL}, name
    assert calls(None, s, d, 2) == {rx.ERR_NULL}
    assert calls(ok, None, d, 2) == {rx.ERR_NULL}
    assert calls(ok, s, None, 2) == {rx.ERR_NULL}
    assert calls(ok, s, d, 2, ws=None) == {rx.ERR_NULL}
    for name, v in (("k", P + 8), ("v", P + 4), ("k_scale", P + 2), ("v_scale", P + 1), ("pages", P + 2), ("rope", P + 4), ("n_pages", 0), ("n_pages", -1),
                    ("pages_per_slot", 0)):
        assert calls(cache(**{name: v}), s, d, 2) == {rx.ERR_SHAPE}, (name, v)
    for size in (0, -16, 8, 24, 48, 512):
        assert calls(cache(page_size=size), s, d, 2) == {rx.ERR_UNSUPPORTED}, size
    assert calls(cache(n_pages=1 << 29), s, d, 2) == {rx.ERR_UNSUPPORTED}              # 2^31 blocks
    assert calls(cache(pages_per_slot=3), s, d, 2) == {rx.ERR_CAPACITY}                # 48 positions for a capacity of 64
    assert calls(ok, s, d, 3) == {rx.ERR_SHAPE}                                        # sum of q_lens
    assert calls(ok, s, d, 0) == {rx.ERR_SHAPE}
    assert calls(ok, rx.Seqs([2, 0], [5, 5]), d, 2) == {rx.ERR_SHAPE}
    assert calls(ok, rx.Seqs([2], [1]), d, 2) == {rx.ERR_SHAPE}
    assert calls(ok, rx.Seqs([2], [65]), d, 2) == {rx.ERR_CAPACITY}
    assert calls(ok, rx.Seqs([2], [5], [2]), d, 2) == {rx.ERR_CAPACITY}
    assert calls(ok, s, dims(head_dim=96), 2) == {rx.ERR_UNSUPPORTED}
    assert calls(ok, s, dims(n_heads=6), 2) == {rx.ERR_SHAPE}
    assert calls(ok, s, d, 2, ws=P + 128) == {rx.ERR_WORKSPACE}
    need = rx.relax_paged_workspace_bytes(d, 2, 5, 1)
    assert calls(ok, s, d, 2, ws_bytes=need - 1) == {rx.ERR_WORKSPACE}
    many = dims(kv_slots=70000)
    assert calls(ok, rx.Seqs([1] * 65536, [1] * 65536), many, 65536) == {rx.ERR_UNSUPPORTED}


def test_what_single_calls_refuse():
    d, s, c = dims(), rx.Seqs([2], [5]), cache()
    put = lambda q=P, qs=256, k=P, v=P, kvs=256, out=P: rx.relax_paged_append(q, qs, k, v, kvs, out, c, s, d, 2, P, BIG)
    assert {put(k=None), put(v=None), put(q=None), put(out=None)} == {rx.ERR_NULL}
    assert {put(q=P + 2), put(k=P + 8), put(v=P + 4), put(out=P + 8), put(qs=257), put(kvs=260), put(qs=248), put(kvs=248), put(kvs=-256)} == {rx.ERR_SHAPE}
    wide = lambda q_out, n: rx.relax_paged_append(P, 512, 2 * P, 2 * P, 512, q_out, c, rx.Seqs([n], [5]), d, n, P, BIG)
    assert wide(P, 2) == rx.ERR_SHAPE                                                  # in place with rows of another pitch: row 1 would land in row 0's keys
    assert rx.relax_paged_attention(None, c, s, d, P, 2, P, BIG) == rx.ERR_NULL
    assert rx.relax_paged_attention(P, c, s, d, None, 2, P, BIG) == rx.ERR_NULL
    assert rx.relax_paged_attention(P + 8, c, s, d, P, 2, P, BIG) == rx.ERR_SHAPE
    assert rx.relax_paged_attention(P, c, s, d, P + 8, 2, P, BIG) == rx.ERR_SHAPE
    assert rx.relax_paged_read(c, s, d, None, None, 2, P, BIG) == rx.ERR_NULL
    assert rx.relax_paged_read(c, s, d, P + 2, None, 2, P, BIG) == rx.ERR_SHAPE


def test_workspace_covers_every_smaller_call():
    assert rx.relax_paged_workspace_bytes(None, 1, 1, 1) == 0
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0)):
        assert rx.relax_paged_workspace_bytes(dims(), *bad) == 0
    for d in (dims(), dims(n_heads=64, n_kv_heads=8, head_dim=128), dims(n_heads=32, n_kv_heads=32, head_dim=128)):
        for n in (1, 2, 16, 100, 5000):
            for L in (1, 129, 4096, 100000):
                at = rx.relax_paged_workspace_bytes(d, n, L, 3)
                assert at <= rx.relax_paged_workspace_bytes(d, n + 1, L, 3) and at <= rx.relax_paged_workspace_bytes(d, n, L + 1, 3)
                assert at <= rx.relax_paged_workspace_bytes(d, n, L, 50)


def test_what_token_logprobs_refuses():
    f = lambda x=P, st=100, t=P, lp=P, e=P, i=P, tp=P, n=2, V=100, k=5: rx.relax_token_logprobs(x, st, t, lp, e, i, tp, n, V, k)
    assert {f(x=None), f(t=None), f(lp=None), f(i=None), f(tp=None), f(t=None, lp=None, e=None, k=0)} == {rx.ERR_NULL}
    assert {f(n=0), f(V=0, k=0), f(st=99), f(k=-1), f(V=4), f(x=P + 1), f(t=P + 2), f(lp=P + 2), f(e=P + 1), f(i=P + 2), f(tp=P + 2)} == {rx.ERR_SHAPE}
    assert {f(k=33), f(V=(1 << 30) + 1, st=1 << 31)} == {rx.ERR_UNSUPPORTED}
    assert rx.relax_token_logprobs_workspace_bytes(0, 10, 1) == 0 and rx.relax_token_logprobs_workspace_bytes(1, 10, 33) == 0


def test_layout_of_the_plain_implementation():
    """Every place of a block once, and the header's formulas at single tokens and elements."""
    for d in (64, 128):
        for name in "kv":
            index = po.code_index(name, d)
            assert sorted(index.ravel()) == list(range(16 * d))
        assert po.code_index("k", d)[5, 35] == (35 // 16 * 16 + 5) * 16 + 35 % 16
        assert po.code_index("v", d)[13, 35] == ((3 * 16 + 3) * 4 + 2) * 4 + 1


def test_plain_token_logprobs():
    x = np.log(np.array([[0.5, 0.25, 0.125, 0.125], [0.0625, 0.0625, 0.5, 0.375]]))
    lp, ent, ids, tops = po.token_logprobs(x, np.array([1, 9]), 4)
    assert np.allclose(lp[0], np.log(0.25)) and lp[1] == -np.inf
    assert np.allclose(ent[0], 1.75 * np.log(2))
    assert ids.tolist() == [[0, 1, 2, 3], [2, 3, 0, 1]] and np.allclose(np.exp(tops[1]), [0.5, 0.375, 0.0625, 0.0625])


def test_capacities_beyond_the_arithmetic_of_positions():
    """2^31 - 1 positions, rounded up to a split, are no 32-bit number: refused by every call, behind the workspace."""
    for cap in ((1 << 30) + 1, (1 << 31) - 1):
        d, c = dims(kv_capacity=cap), cache(rope=None, page_size=256, pages_per_slot=1 << 23)
        for L in (5, cap):
            assert calls(c, rx.Seqs([2], [L]), d, 2) == {rx.ERR_UNSUPPORTED}, (cap, L)
        assert calls(c, rx.Seqs([2], [cap]), d, 2, ws_bytes=256) == {rx.ERR_WORKSPACE}
    at = [rx.relax_paged_workspace_bytes(dims(kv_capacity=(1 << 31) - 1, n_heads=1, n_kv_heads=1), 1, L, 1) for L in (1, 128, 4096, 1 << 22, (1 << 23) + 1, 1 << 30, (1 << 31) - 1)]
    assert at == sorted(at) and at[0] > 0
