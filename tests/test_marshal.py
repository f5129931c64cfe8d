"""Argument marshalling in C (csrc/marshal.c) against a recording C function, and against the same in Python."""
import ctypes as C
import gc
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2311_02103_amd import binding as rx

marshal = pytest.importorskip("paper_2311_02103_amd._marshal")


class Recorder:
    def __init__(self, count, result=0):
        self.got = []
        self.fn = C.CFUNCTYPE(C.c_int32, *[C.c_int64] * count)(lambda *a: self.got.append(a) or result)
        self.address = C.cast(self.fn, C.c_void_p).value


class At:
    def __init__(self, at):
        self._at = at


class Stream:
    def __init__(self, address):
        self.cuda_stream = address


def descriptor(seqs):
    c = seqs.c()
    take = lambda p: None if not p else [p[i] for i in range(c.B)]
    return c.B, take(c.q_lens), take(c.kv_lens), take(c.slots), c.device_table


def test_every_kind_of_argument():
    rec = Recorder(15, -3)
    call = marshal.Call(rec.address, "ppppiiiirrrrsss")
    t, seqs, dims = torch.zeros(7, dtype=torch.float16), rx.Seqs([1], [2]), rx.make_dims(64, 1, 1, 64, 64, 8)
    cache = rx.Paged4Cache(1, 2, 3, 4, 5, 1, 16, 1)
    args = (None, 0x7fffffff0000, t, 0, -5, 1 << 40, np.int64(7), True, None, seqs, dims, cache, 0x1230, Stream(0x4560), Stream(0))
    assert call(*args) == -3
    assert rec.got == [(0, 0x7fffffff0000, t.data_ptr(), 0, -5, 1 << 40, 7, 1, 0, seqs._at, C.addressof(dims), cache._at, 0x1230, 0x4560, 0)]
    assert marshal.Call(Recorder(0, 9).address, "")() == 9


def test_what_it_refuses():
    rec = Recorder(3)
    call = marshal.Call(rec.address, "pir")
    for args, error in (((None, 1), TypeError), ((None, 1, None, None), TypeError), ((None, 1.5, None), TypeError), ((None, "1", None), TypeError),
                        ((torch.zeros(4, 4)[:, :2], 1, None), ValueError), ((object(), 1, None), AttributeError), ((None, 1, object()), AttributeError),
                        ((None, 1 << 70, None), OverflowError), ((1 << 70, 1, None), OverflowError), ((None, 1, At("x")), TypeError)):
        with pytest.raises(error):
            call(*args)
    with pytest.raises(TypeError):
        call(None, 1, None, stream=None)
    assert not rec.got
    for bad in ((0, "p"), (rec.address, "x"), (rec.address, "p" * 17)):
        with pytest.raises(ValueError):
            marshal.Call(*bad)


def test_a_stream_of_none_asks_for_the_current_one():
    rec = Recorder(1)
    code = "import sys; sys.path.insert(0, %r)\nfrom paper_2311_02103_amd import _marshal as m\nimport ctypes as C\ngot = []\n" % rx._HERE.rsplit("/", 1)[0]
    code += "f = C.CFUNCTYPE(C.c_int32, C.c_int64)(lambda a: got.append(a) or 0)\ncall = m.Call(C.cast(f, C.c_void_p).value, 's')\n"
    code += "m.slow_stream(lambda s: 5 if s is None else 1)\ncall(None)\nm.slow_stream(lambda s: None)\ncall(None)\n"
    code += "m.use_streams(lambda: 3, lambda d: d * 16)\ncall(None)\nm.use_streams(lambda: 3, lambda d: 0)\ncall(None)\nassert got == [5, 0, 48, 0], got\n"
    import subprocess
    subprocess.run([sys.executable, "-c", code], check=True, timeout=120)
    del rec


@pytest.mark.parametrize("kind", [rx._PySeqs, rx.Seqs])
def test_descriptors(kind):
    take = descriptor if kind is rx.Seqs else lambda s: (s.c().B, list(s._q), list(s._kv)[:s.B], None if s._sl is None else list(s._sl), s.c().device_table)
    table = torch.zeros(8, dtype=torch.int32)
    assert take(kind([3, 1], [3, 900])) == (2, [3, 1], [3, 900], None, None)
    assert take(kind((3, 1), np.array([3, 900]), slots=[7, 2], device_table=table)) == (2, [3, 1], [3, 900], [7, 2], table.data_ptr())
    assert take(kind([True], [(1 << 32) + 5], None, 0x1000)) == (1, [1], [5], None, 0x1000)
    assert take(kind([], [])) == (0, [], [], None, None) and kind([1], [2]).B == 1
    assert take(kind([1], [2, 3], [4, 5]))[:3] == (1, [1], [2])
    for bad in (([1, 2], [1]), ([1, 2], [1, 2], [0])):
        with pytest.raises(ValueError):
            kind(*bad)
    for bad in (([1], 5), (["x"], [1]), ([1], [None])):
        with pytest.raises((TypeError, ValueError)):
            kind(*bad)


def test_descriptors_hold_their_memory_and_the_table():
    table = torch.zeros(8, dtype=torch.int32)
    before = sys.getrefcount(table)
    seqs = rx.Seqs(list(range(1, 50)), list(range(100, 149)), device_table=table)
    assert sys.getrefcount(table) == before + 1
    c = seqs.c()
    del seqs
    gc.collect()
    junk = [rx.Seqs([9] * 49, [9] * 49) for _ in range(100)]
    assert [c.q_lens[i] for i in range(49)] == list(range(1, 50)) and [c.kv_lens[i] for i in range(49)] == list(range(100, 149))
    del c, junk
    gc.collect()
    assert sys.getrefcount(table) == before
    with pytest.raises(ValueError):
        rx.Seqs([1], [1], None, torch.zeros(4, 4, dtype=torch.int32)[:, :2])
    assert sys.getrefcount(table) == before


def test_no_reference_is_lost():
    rec = Recorder(4)
    call = marshal.Call(rec.address, "ppsr")
    t, at, stream = torch.zeros(3), At(123456789), Stream(987654321)
    before = [sys.getrefcount(x) for x in (t, at, stream, None)]
    for _ in range(1000):
        call(t, t, stream, at)
    rec.got.clear()
    after = [sys.getrefcount(x) for x in (t, at, stream, None)]
    assert after[:3] == before[:3] and abs(after[3] - before[3]) < 100


def test_the_python_form_says_the_same(monkeypatch):
    """The library's own refusals through both."""
    dims, cache, prep, P = rx.make_dims(256, 4, 4, 64, 688, 64, 2), rx.Paged4Cache(*[0x10000] * 5, 10, 16, 4), rx.HeadPrep(0x10000, 0x10000, 1e-6, 0x10000), 0x10000
    t = torch.zeros(512, dtype=torch.float16)

    def codes():
        out = []
        for s in (rx.Seqs([2], [5]), rx.Seqs([2], [65]), None):
            for d in (dims, None):
                out += [rx.relax_paged4_append(P, 256, P, P, 256, P, prep, cache, s, d, 2, P, 8), rx.relax_paged4_attention(t.data_ptr() // 16 * 16, cache, s, d, P, 2, P, 8, stream=0),
                        rx.relax_paged4_read(cache, s, d, P, None, 2, P, 8, stream=Stream(0)), rx.relax_head_norm_rope(P, 256, None, 0, P, 256, None, 0, prep, s, d, 2, P, 8)]
        return out + [rx.relax_rope_table_scaled(rx.RopeScaling(7, 64), 4, P), rx.relax_rope_table_scaled(None, 4, P)]
    monkeypatch.setattr(rx, "_bound", {})
    fast = codes()
    monkeypatch.setattr(rx, "_bound", {})
    monkeypatch.setattr(rx, "_marshal", None)
    assert codes() == fast and len(set(fast)) >= 4
    with pytest.raises(TypeError):
        rx._bound["relax_paged4_read"](1, 2)


def struct_calls():
    """(name, its arguments, {place of a struct among them: what belongs there}) of each call with structs."""
    P, s, d, cache, prep, scaling = 0x10000, rx.Seqs([2], [5]), rx.make_dims(256, 4, 4, 64, 688, 64, 2), rx.Paged4Cache(*[0x10000] * 5, 10, 16, 4), rx.HeadPrep(), rx.RopeScaling(7, 64)
    return [("relax_rope_table_scaled", [scaling, 4, P, 0], {0: scaling}), ("relax_head_norm_rope", [P, 256, None, 0, P, 256, None, 0, prep, s, d, 2, P, 8, 0], {8: prep, 9: s, 10: d}),
            ("relax_paged4_append", [P, 256, P, P, 256, P, prep, cache, s, d, 2, P, 8, 0], {6: prep, 7: cache, 8: s, 9: d}),
            ("relax_paged4_attention", [P, cache, s, d, P, 2, P, 8, 0], {1: cache, 2: s, 3: d}), ("relax_paged4_read", [cache, s, d, P, None, 2, P, 8, 0], {0: cache, 1: s, 2: d})]


@pytest.mark.parametrize("in_c", [True, False])
@pytest.mark.parametrize("name,args,places", struct_calls(), ids=lambda x: x if isinstance(x, str) else "")
def test_structs_of_another_type_are_refused(monkeypatch, name, args, places, in_c):
    """Anything but None and the struct that an argument is for: the library would read it as that struct.  (Those here have 4 KB of zeros behind their addresses.)"""
    monkeypatch.setattr(rx, "_bound", {})
    if not in_c:
        monkeypatch.setattr(rx, "_marshal", None)
    room = (C.c_char * 4096)()
    wrong = [bytearray(4096), np.zeros(1024, np.int32), torch.zeros(1024, dtype=torch.int32), [2], "x", 0x10000, At(C.addressof(room)), room, object(), rx.KVCache(1, 2, 3)]
    wrong += list({id(x): x for _, _, p in struct_calls() for x in p.values()}.values())
    call = getattr(rx, name)
    right = call(*args)
    for at, mine in places.items():
        for other in wrong:
            if type(other) is type(mine):
                continue
            with pytest.raises(TypeError):
                call(*args[:at], other, *args[at + 1:])
        assert call(*args[:at], None, *args[at + 1:]) == (right if name == "relax_paged4_append" and at == 6 else rx.ERR_NULL)      # (no preparation)
        raw = mine.c() if hasattr(mine, "c") else mine             # the C struct itself, and a subclass
        assert call(*args[:at], raw, *args[at + 1:]) == right
    assert call(*args) == right


def test_types_of_a_call():
    rec = Recorder(3)
    call = marshal.Call(rec.address, "rir", (At, (rx.LayerDims, rx.Seqs)))
    dims, seqs = rx.make_dims(64, 1, 1, 64, 64, 8), rx.Seqs([1], [2])

    class Other(At):
        pass
    assert call(Other(5), 1, dims) == 0 and call(None, 2, seqs) == 0 and call(At(7), 3, None) == 0
    assert [a[:2] for a in rec.got] == [(5, 1), (0, 2), (7, 3)]
    for args in ((dims, 1, dims), (At(1), 1, At(1)), (At(1), 1, bytearray(64))):
        with pytest.raises(TypeError):
            call(*args)
    for types in ((At,), (At, At, At), (At, 5), [At, At], (At, (At, 5))):
        with pytest.raises((TypeError, ValueError)):
            marshal.Call(rec.address, "rir", types)


@pytest.mark.parametrize("kind", [rx._PySeqs, rx.Seqs])
def test_descriptors_are_copied(kind):
    """Equal lengths, in memory that lives as long as the twin; the table is shared by a copy, copied by a deepcopy."""
    import copy

    class Mine(kind):
        pass
    table = torch.arange(8, dtype=torch.int32)
    for cls in (kind, Mine):
        seqs = cls([3, 1], [3, 900], [7, 2], table)
        if cls is Mine:
            seqs.note = "kept"
        for twin, shared in ((copy.copy(seqs), True), (copy.deepcopy(seqs), False)):
            assert type(twin) is cls and getattr(twin, "note", None) == getattr(seqs, "note", None)
            a, b = descriptor(seqs), descriptor(twin)
            assert a[:4] == b[:4] == (2, [3, 1], [3, 900], [7, 2])
            assert (a[4] == b[4]) == shared and b[4]
        alone = copy.deepcopy(cls(list(range(1, 50)), list(range(100, 149))))
        gc.collect()
        assert descriptor(alone) == (49, list(range(1, 50)), list(range(100, 149)), None, None)
    assert descriptor(copy.copy(kind([], []))) == (0, [], [], None, None)


@pytest.mark.parametrize("kind", [rx._PySeqs, rx.Seqs])
def test_the_number_of_sequences_can_be_set(kind):
    """The first B of those that there are lengths for; more would be read behind the arrays."""
    import copy
    seqs = kind([3, 1, 2], [3, 900, 4, 5], [7, 2, 0])
    for B in (2, 3, 1, 0, -1, 3):
        seqs.B = B
        assert seqs.B == seqs.c().B == copy.copy(seqs).B == copy.deepcopy(seqs).c().B == B
        if B > 0:
            assert descriptor(copy.copy(seqs)) == descriptor(seqs) == (B, [3, 1, 2][:B], [3, 900, 4][:B], [7, 2, 0][:B], None)
    for bad in (4, 1 << 31, -(1 << 31) - 1, 1 << 70):
        with pytest.raises((ValueError, OverflowError)):
            seqs.B = bad
    for bad in ("2", None, 1.5):
        with pytest.raises(TypeError):
            seqs.B = bad
    with pytest.raises((TypeError, AttributeError)):
        del seqs.B
    twin = copy.deepcopy(seqs)
    seqs.B, twin.B = 1, 2
    assert descriptor(seqs)[0] == 1 and descriptor(twin)[:2] == (2, [3, 1])
    twin.B = 3
    assert descriptor(twin)[1] == [3, 1, 2]
    rec = Recorder(1)
    if kind is rx.Seqs:
        got = []
        fn = C.CFUNCTYPE(C.c_int32, C.POINTER(rx.SeqsC))(lambda p: got.append((p[0].B, [p[0].q_lens[i] for i in range(p[0].B)])) or 0)
        call = marshal.Call(C.cast(fn, C.c_void_p).value, "r")
        seqs.B = 2
        assert call(seqs) == 0 and call(twin) == 0 and got == [(2, [3, 1]), (3, [3, 1, 2])]
    del rec


@pytest.mark.parametrize("kind", [rx._PySeqs, rx.Seqs])
def test_the_tables_address_is_that_of_the_call(kind):
    """A tensor whose storage is exchanged, the old one freed: each call takes the address that it has then, and refuses one that is not contiguous."""
    table = torch.zeros(8, dtype=torch.int32)
    seqs = kind([3, 1], [3, 900], device_table=table)
    first = table.data_ptr()
    assert seqs.c().device_table == first
    other = torch.ones(64, dtype=torch.int32)
    for change in (lambda: setattr(table, "data", other), lambda: table.set_(other, 8, (8,), (1,))):
        change()
        assert table.data_ptr() != first and seqs.c().device_table == table.data_ptr()
        if kind is rx.Seqs:
            got = []
            fn = C.CFUNCTYPE(C.c_int32, C.POINTER(rx.SeqsC))(lambda p: got.append(p[0].device_table) or 0)
            assert marshal.Call(C.cast(fn, C.c_void_p).value, "r")(seqs) == 0 and got == [table.data_ptr()]
            assert rx.SeqsC.from_address(seqs._at).device_table == table.data_ptr()
    table.set_(other, 0, (4, 2), (1, 4))
    with pytest.raises(ValueError):
        seqs.c()
    if kind is rx.Seqs:
        with pytest.raises(ValueError):
            marshal.Call(Recorder(1).address, "r")(seqs)


def test_a_call_keeps_the_descriptor_it_was_made_with():
    """Lengths that are given anew while the call runs, as by another thread, do not reach it, and its arrays stay."""
    seqs, got = rx.Seqs(list(range(1, 50)), list(range(100, 149))), []

    def during(p):
        rx.Seqs.__init__(seqs, [7], [8])
        seqs.B = 0
        gc.collect()
        junk = [rx.Seqs([9] * 49, [9] * 49) for _ in range(100)]
        got.append((p[0].B, [p[0].q_lens[i] for i in range(49)], [p[0].kv_lens[i] for i in range(49)], len(junk)))
        return 0
    fn = C.CFUNCTYPE(C.c_int32, C.POINTER(rx.SeqsC))(during)
    assert marshal.Call(C.cast(fn, C.c_void_p).value, "r")(seqs) == 0
    assert got == [(49, list(range(1, 50)), list(range(100, 149)), 100)]
    assert descriptor(seqs) == (0, [], [], None, None)
