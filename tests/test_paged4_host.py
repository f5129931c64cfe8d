"""Host-side contract of the rotary tables, the heads and the paged 4-bit cache: every refusal comes before anything is enqueued, and the plain implementation that
the GPU tests use is pinned to the layout's definition."""
import math

import numpy as np

import paged4_oracle as po
from paper_2311_02103_amd import binding as rx

P = 0x10000   # a non-null fake device address
BIG = 1 << 26
NAN, INF = float("nan"), float("inf")


def dims(**kw):
    base = dict(hidden=256, n_heads=4, n_kv_heads=4, head_dim=64, ffn=688, kv_capacity=64, kv_slots=2)
    base.update(kw)
    return rx.make_dims(**base)


def cache(**kw):
    a = dict(k=P, v=P, k_scale=P, v_scale=P, pages=P, n_pages=10, page_size=16, pages_per_slot=4)
    a.update(kw)
    return rx.Paged4Cache(*[a[k] for k in ("k", "v", "k_scale", "v_scale", "pages", "n_pages", "page_size", "pages_per_slot")])


def prep(**kw):
    return rx.HeadPrep(**{**dict(q_norm=P, k_norm=P, eps=1e-6, rope=P), **kw})


def calls(c, s, d, n, ws=P, ws_bytes=BIG):
    return {rx.relax_paged4_append(P, 256, P, P, 256, P, prep(), c, s, d, n, ws, ws_bytes), rx.relax_paged4_attention(P, c, s, d, P, n, ws, ws_bytes),
            rx.relax_paged4_read(c, s, d, P, P, n, ws, ws_bytes)}


def heads(q=P, qs=256, k=P, ks=256, qo=2 * P, qos=256, ko=3 * P, kos=256, p=prep(), s=rx.Seqs([2], [5]), d=dims(), n=2, ws=P, ws_bytes=BIG):
    return rx.relax_head_norm_rope(q, qs, k, ks, qo, qos, ko, kos, p, s, d, n, ws, ws_bytes)


def test_what_the_paged_calls_refuse_alike():
    d, s, ok = dims(), rx.Seqs([2], [5]), cache()
    for name in ("k", "v", "k_scale", "v_scale", "pages"):
        assert calls(cache(**{name: None}), s, d, 2) == {rx.ERR_NULL}, name
    assert calls(None, s, d, 2) == calls(ok, None, d, 2) == calls(ok, s, None, 2) == calls(ok, s, d, 2, ws=None) == {rx.ERR_NULL}
    for name, v in (("k", P + 8), ("v", P + 4), ("k_scale", P + 8), ("v_scale", P + 2), ("pages", P + 2), ("n_pages", 0), ("n_pages", -1), ("pages_per_slot", 0)):
        assert calls(cache(**{name: v}), s, d, 2) == {rx.ERR_SHAPE}, (name, v)
    for size in (0, -16, 8, 24, 48, 512):
        assert calls(cache(page_size=size), s, d, 2) == {rx.ERR_UNSUPPORTED}, size
    assert calls(cache(n_pages=1 << 29), s, d, 2) == {rx.ERR_UNSUPPORTED}              # 2^31 blocks
    assert calls(cache(pages_per_slot=3), s, d, 2) == {rx.ERR_CAPACITY}                # 48 positions for a capacity of 64
    assert calls(ok, s, d, 3) == calls(ok, s, d, 0) == calls(ok, rx.Seqs([2, 0], [5, 5]), d, 2) == calls(ok, rx.Seqs([2], [1]), d, 2) == {rx.ERR_SHAPE}
    assert calls(ok, rx.Seqs([2], [65]), d, 2) == calls(ok, rx.Seqs([2], [5], [2]), d, 2) == {rx.ERR_CAPACITY}
    assert calls(ok, s, dims(head_dim=96), 2) == {rx.ERR_UNSUPPORTED} and calls(ok, s, dims(n_heads=6), 2) == {rx.ERR_SHAPE}
    assert calls(ok, s, d, 2, ws=P + 128) == {rx.ERR_WORKSPACE}
    assert calls(ok, s, d, 2, ws_bytes=rx.relax_paged4_workspace_bytes(d, 2, 5, 1) - 1) == {rx.ERR_WORKSPACE}
    assert calls(ok, rx.Seqs([1] * 65536, [1] * 65536), dims(kv_slots=70000), 65536) == {rx.ERR_UNSUPPORTED}
    for cap in ((1 << 30) + 1, (1 << 31) - 1):
        assert calls(cache(page_size=256, pages_per_slot=1 << 23), s, dims(kv_capacity=cap), 2) == {rx.ERR_UNSUPPORTED}


def test_what_single_calls_refuse():
    d, s, c = dims(), rx.Seqs([2], [5]), cache()
    put = lambda q=P, qs=256, k=P, v=P, kvs=256, out=P, p=prep(): rx.relax_paged4_append(q, qs, k, v, kvs, out, p, c, s, d, 2, P, BIG)
    assert {put(k=None), put(v=None), put(q=None), put(out=None)} == {rx.ERR_NULL}
    assert {put(q=P + 2), put(k=P + 8), put(v=P + 4), put(out=P + 8), put(qs=257), put(kvs=260), put(qs=248), put(kvs=248), put(kvs=-256)} == {rx.ERR_SHAPE}
    assert rx.relax_paged4_append(P, 512, 2 * P, 2 * P, 512, P, None, c, s, d, 2, P, BIG) == rx.ERR_SHAPE      # in place with rows of another pitch
    assert rx.relax_paged4_attention(None, c, s, d, P, 2, P, BIG) == rx.relax_paged4_attention(P, c, s, d, None, 2, P, BIG) == rx.ERR_NULL
    assert rx.relax_paged4_attention(P + 8, c, s, d, P, 2, P, BIG) == rx.relax_paged4_attention(P, c, s, d, P + 8, 2, P, BIG) == rx.ERR_SHAPE
    assert rx.relax_paged4_read(c, s, d, None, None, 2, P, BIG) == rx.ERR_NULL and rx.relax_paged4_read(c, s, d, P + 2, None, 2, P, BIG) == rx.ERR_SHAPE


def test_what_preparing_heads_refuses():
    put = lambda p: {heads(p=p), rx.relax_paged4_append(P, 256, P, P, 256, P, p, cache(), rx.Seqs([2], [5]), dims(), 2, P, BIG)}
    for name in ("q_norm", "k_norm", "rope"):
        assert put(prep(**{name: P + 8})) == {rx.ERR_SHAPE}
    for eps in (-1e-6, NAN, INF):
        assert put(prep(eps=eps)) == {rx.ERR_SHAPE}
    for bad in (dict(rotary_dim=-16), dict(rotary_dim=80), dict(rotary_dim=8), dict(rotary_dim=24), dict(layout=2), dict(layout=-1)):
        assert put(prep(**bad)) == {rx.ERR_UNSUPPORTED}, bad
    assert {heads(p=None), heads(ws=None), heads(q=None), heads(qo=None), heads(k=None), heads(ko=None), heads(q=None, qo=None, k=None, ko=None), heads(s=None),
            heads(d=None)} == {rx.ERR_NULL}
    assert {heads(q=P + 8), heads(k=P + 2), heads(qo=P + 8), heads(ko=P + 4), heads(qs=248), heads(ks=252), heads(qos=257), heads(kos=-256), heads(n=3),
            heads(qo=P, qos=512), heads(ko=P, kos=512), heads(s=rx.Seqs([2], [1]))} == {rx.ERR_SHAPE}
    assert heads(s=rx.Seqs([2], [65])) == rx.ERR_CAPACITY
    assert heads(d=dims(head_dim=96)) == rx.ERR_UNSUPPORTED and heads(d=dims(kv_capacity=(1 << 30) + 1)) == rx.ERR_UNSUPPORTED
    assert heads(ws=P + 64) == heads(ws_bytes=rx.relax_head_workspace_bytes(dims(), 1) - 1) == rx.ERR_WORKSPACE
    assert heads(s=rx.Seqs([1] * 65536, [1] * 65536), d=dims(kv_slots=70000), n=65536) == rx.ERR_UNSUPPORTED
    assert rx.relax_head_workspace_bytes(None, 1) == rx.relax_head_workspace_bytes(dims(), 0) == 0
    assert rx.relax_head_workspace_bytes(dims(), 1) <= rx.relax_head_workspace_bytes(dims(), 100)


def test_what_a_scaled_table_refuses():
    good = dict(scaling=rx.ROPE_WAVELENGTH_RAMP, rotary_dim=64, base=10000.0, factor=4.0, trained=2048.0, slow=1.0, fast=4.0, amplitude=1.0)
    f = lambda positions=10, table=P, **kw: rx.relax_rope_table_scaled(rx.RopeScaling(**{**good, **kw}), positions, table)
    assert rx.relax_rope_table_scaled(None, 10, P) == f(table=None) == rx.ERR_NULL
    assert {f(positions=0), f(positions=-1), f(rotary_dim=0), f(rotary_dim=-2), f(table=P + 8)} == {rx.ERR_SHAPE}
    assert {f(scaling=-1), f(scaling=4), f(rotary_dim=63), f(rotary_dim=258), f(positions=(1 << 30) + 1)} == {rx.ERR_UNSUPPORTED}
    for bad in (dict(base=1.0), dict(base=-5.0), dict(base=NAN), dict(base=INF), dict(factor=0.0), dict(factor=-1.0), dict(factor=NAN), dict(factor=INF), dict(trained=0.5),
                dict(trained=NAN), dict(trained=INF), dict(slow=0.0), dict(slow=4.0), dict(slow=NAN), dict(fast=NAN), dict(fast=INF), dict(amplitude=NAN), dict(amplitude=INF)):
        assert f(**bad) == rx.ERR_SHAPE, bad
        assert f(**bad, scaling=rx.ROPE_INDEX_RAMP) == rx.ERR_SHAPE, bad
        assert rx.relax_rope_scaled_bytes(rx.RopeScaling(**{**good, **bad}), 10) == 0
    assert rx.relax_rope_scaled_bytes(rx.RopeScaling(**good), 1 << 30) == (1 << 30) * 256
    assert rx.relax_rope_scaled_bytes(rx.RopeScaling(**good), 0) == rx.relax_rope_scaled_bytes(None, 5) == 0


def test_workspace_covers_every_smaller_call():
    assert rx.relax_paged4_workspace_bytes(None, 1, 1, 1) == 0
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0)):
        assert rx.relax_paged4_workspace_bytes(dims(), *bad) == 0
    for d in (dims(), dims(n_heads=64, n_kv_heads=8, head_dim=128)):
        for n in (1, 2, 16, 100, 5000):
            for L in (1, 129, 4096, 100000):
                at = rx.relax_paged4_workspace_bytes(d, n, L, 3)
                assert at <= rx.relax_paged4_workspace_bytes(d, n + 1, L, 3) and at <= rx.relax_paged4_workspace_bytes(d, n, L + 1, 3)
                assert at <= rx.relax_paged4_workspace_bytes(d, n, L, 50)


def test_layout_of_the_plain_implementation():
    """Every half byte of a block once, every scale once, and the header's formulas at single tokens and elements."""
    for d in (64, 128):
        for name in "kv":
            byte, shift = po.code_place(name, d)
            assert sorted((2 * byte + shift // 4).ravel()) == list(range(16 * d))
        assert sorted(po.scale_place(d).ravel()) == list(range(16 * d // 32))
        byte, shift = po.code_place("k", d)
        # element 46 of token 5: word [46 / 8 % 4 = 1][5][46 / 32 = 1], element 6 of eight = 4 (b % 2) + b / 2 + 2 with b = 1
        assert (byte[5, 46], shift[5, 46]) == (4 * ((1 * 16 + 5) * (d // 32) + 1) + 1, 4)
        assert (byte[5, 33], shift[5, 33]) == (4 * (5 * (d // 32) + 1) + 2, 0)             # element 1: b = 2
        byte, shift = po.code_place("v", d)
        # element 35 of token 13: word [13 / 4 = 3][35 % 16 = 3][35 / 32 = 1], token 13 % 4 = 1 = 2 (b % 2) + b / 2 with b = 2, low half; element 51 above it
        assert (byte[13, 35], shift[13, 35]) == (4 * ((3 * 16 + 3) * (d // 32) + 1) + 2, 0)
        assert (byte[13, 51], shift[13, 51]) == (byte[13, 35], 4)
        assert po.scale_place(d)[6, 1] == (1 * (d // 32) + 1) * 4 + 2


def test_plain_quantisation():
    x = np.zeros((4, 32), np.float32)
    x[0, :4] = [8, -8, 4.5, -7.6]
    x[1, :3] = [-8, 7.4, 7.6]
    x[2, :2] = [1e-8, -1e-8]
    x[3] = 65504
    u, s = po.quantise(x)
    assert s[:, 0].tolist() == [-1.0, 1.0, 0.0, -8160.0]
    assert u[0, :5].tolist() == [0, 15, 4, 15, 8]              # 8 -> -8, -8 -> 8 kept at 7, 4.5 -> -4 (a tie, to even), -7.6 -> 8 kept at 7, 0
    assert u[1, :4].tolist() == [0, 15, 15, 8] and (u[2] == 8).all() and (u[3] == 0).all()
    for v, want in ((1.0, 1.0), (1.00390625, 1.0), (1.01171875, 1.015625), (257.0, 256.0), (259.0, 260.0), (-1.004, -1.0078125)):
        assert po.round8(np.array([v], np.float32))[0] == want      # 1 + 2^-8 is a tie, to even
    # every scale of eight bits times every code is an fp16 number
    for e in (-14, 0, 11):
        s = (np.arange(128, 256) * 2.0 ** (e - 7))
        v = s[:, None] * np.arange(-8, 8)
        assert np.array_equal(v.astype(np.float16).astype(np.float64), v)
    assert float(np.float16(8160) * np.float16(8)) == 65280


def test_plain_frequencies():
    f = po.frequencies(64, 10000.0, "wavelength", 4.0, 2048.0, 1.0, 4.0)
    plain = po.frequencies(64, 10000.0)
    turns = 2048 * plain / (2 * math.pi)
    assert np.allclose(f[turns >= 4], plain[turns >= 4]) and np.allclose(f[turns <= 1], plain[turns <= 1] / 4) and ((turns > 1) & (turns < 4)).any()
    assert np.allclose(po.frequencies(64, 10000.0, "linear", 4.0), plain / 4)
    f = po.frequencies(64, 10000.0, "index", 4.0, 2048.0, 1.0, 32.0)
    first, last = math.floor(64 * math.log(2048 / (64 * math.pi)) / (2 * math.log(1e4))), math.ceil(64 * math.log(2048 / (2 * math.pi)) / (2 * math.log(1e4)))
    assert np.allclose(f[:first + 1], plain[:first + 1]) and np.allclose(f[last:], plain[last:] / 4) and first + 1 < last < 32


def test_plain_quantisation_of_the_smallest_groups():
    """What the header says of them: those of 2^-22 and less are zeros, 2^-25 being a tie between 0 and the smallest scale, and what eight bits round to that; beyond, the scale is a multiple of 2^-24."""
    tiny = 2.0 ** -24
    for largest, scale, held in ((1, 0, 0), (3, 0, 0), (4, 0, 0), (4 * (1 + 2.0 ** -8), 0, 0), (4 * (1 + 2.0 ** -7), -1, 4), (5, -1, 5), (8, -1, 8), (11, -1, 8), (12, -2, 12), (20, -2, 16), (-4, 0, 0), (-5, 1, -5), (-8, 1, -8)):
        x = np.zeros((1, 32), np.float32)
        x[0, 7] = largest * tiny
        u, s = po.quantise(x)
        assert float(s[0, 0]) == scale * tiny and (float(u[0, 7]) - 8) * float(s[0, 0]) == held * tiny, largest


def test_a_factor_whose_inverse_is_no_number_is_refused():
    """The smallest numbers of fp64: pairs that a ramp leaves as they are would be 0 * infinity."""
    for scaling in (rx.ROPE_LINEAR, rx.ROPE_INDEX_RAMP, rx.ROPE_WAVELENGTH_RAMP):
        make = lambda factor: rx.RopeScaling(scaling, 64, 10000.0, factor, 2048.0, 1.0, 4.0, 1.0)
        for factor in (5e-324, 1e-310, 5.5e-309):
            assert rx.relax_rope_table_scaled(make(factor), 10, P) == rx.ERR_SHAPE and rx.relax_rope_scaled_bytes(make(factor), 10) == 0
        assert rx.relax_rope_scaled_bytes(make(6e-309), 10) == rx.relax_rope_scaled_bytes(make(1e308), 10) == 10 * 64 * 4
    assert rx.relax_rope_scaled_bytes(rx.RopeScaling(rx.ROPE_PLAIN, 64, 10000.0, 1e-310), 10) == 10 * 64 * 4       # (not used there)
