"""What the Python side of the paged 4-bit cache refuses before it reaches the library, and where it allocates.  Tensors are on the CPU and the calls that would
enqueue work are replaced: nothing runs on a GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_2311_02103_amd import binding as rx
from paper_2311_02103_amd import runtime

PLAIN = rx.RopeScaling(rx.ROPE_PLAIN, 64, 10000.0, 1.0)
STRETCHED = rx.RopeScaling(rx.ROPE_LINEAR, 64, 10000.0, 4.0)


@pytest.fixture
def calls(monkeypatch):
    """The library calls that were made, as (name, arguments); they succeed and do nothing."""
    made = []
    for name in ("relax_workspace_init", "relax_rope_table_scaled", "relax_paged4_append", "relax_paged4_attention", "relax_paged4_read", "relax_head_norm_rope"):
        monkeypatch.setattr(rx, name, lambda *args, name=name: made.append((name, args)) or 0)
    return made


def cache(**kw):
    base = dict(n_heads=4, n_kv_heads=2, head_dim=64, kv_capacity=100, n_pages=4, page_size=64, kv_slots=2, n_max=8, device="cpu")
    base.update(kw)
    return runtime.DevicePaged4Cache(**base)


def test_what_a_layer_holds(calls):
    layer = cache(rope=rx.RopeScaling(rx.ROPE_LINEAR, 32, 10000.0, 2.0), layout=rx.ROPE_PAIRS, q_norm=torch.ones(64, dtype=torch.float16))
    assert layer.k.numel() == layer.v.numel() == 4 * 2 * 64 * 64 // 2 and layer.k_scale.numel() == 4 * 2 * 64 * 64 // 32 and layer.k_scale.dtype == torch.float16
    assert layer.rope.shape == (100, 16, 2) and layer.pages.shape == (2, 2) and (layer.pages == -1).all()
    c = layer.prep.c()
    assert c.rotary_dim == 32 and c.layout == rx.ROPE_PAIRS and c.q_norm and not c.k_norm and c.rope == layer.rope.data_ptr()
    assert layer.ws.numel() == rx.relax_paged4_workspace_bytes(layer.dims, 8, 100, 2)
    bare = cache(rope=None)
    assert bare.rope is None and not bare.prep.c().rope
    assert cache().rope.shape == (100, 32, 2)
    with pytest.raises(ValueError):
        cache(rope=rx.RopeScaling(rx.ROPE_LINEAR, 33, 10000.0, 2.0))
    for w in (torch.ones(64), torch.ones(128, dtype=torch.float16), torch.ones(64, dtype=torch.float16, device="meta")):
        with pytest.raises(ValueError):
            cache(q_norm=w)
        with pytest.raises(ValueError):
            cache(k_norm=w)


@pytest.mark.parametrize("other", [dict(kv_slots=3), dict(kv_capacity=101), dict(kv_capacity=128), dict(page_size=32), dict(rope=None), dict(rope=STRETCHED), dict(device="meta")], ids=str)
def test_layers_share_only_tables_that_cover_them(calls, other):
    first = cache()
    with pytest.raises(ValueError):
        cache(share_from=first, **other)


def test_tables_that_are_shared(calls):
    first = cache(rope=STRETCHED)
    for kw in (dict(), dict(kv_slots=1), dict(kv_capacity=64), dict(rope=STRETCHED), dict(n_pages=9), dict(n_kv_heads=4), dict(layout=rx.ROPE_PAIRS)):
        second = cache(share_from=first, **kw)
        assert second.pages is first.pages and second.rope is first.rope and second.ws is first.ws and second.cache.c().pages_per_slot == 2
        assert second.prep.c().rotary_dim == 64 and second.prep.c().layout == kw.get("layout", rx.ROPE_HALVES)
    with pytest.raises(ValueError):
        cache(share_from=first, rope=PLAIN)
    with pytest.raises(ValueError):
        cache(share_from=cache(rope=None), rope=PLAIN)
    assert cache(share_from=cache(rope=None), rope=None, kv_capacity=128).rope is None
    with pytest.raises(ValueError):
        cache(share_from=first, head_dim=32)                   # turns 64 elements


class FakeStream:
    cuda_stream = 0x5000


def test_what_a_call_on_a_stream_allocates_belongs_to_it(calls, monkeypatch):
    """Memory of the current stream would be handed out again there while the call's kernels run."""
    seqs, here, made = rx.Seqs([3], [3]), [], []
    layer = cache()

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            here.append(self.stream.cuda_stream)

        def __exit__(self, *_):
            here.pop()
    monkeypatch.setattr(torch.cuda, "stream", On)
    for name in ("empty", "empty_like"):
        plain = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, plain=plain, **kw: made.append(here[-1] if here else None) or plain(*a, **kw))
    x = torch.zeros((3, 8 * 64), dtype=torch.float16)
    for stream, want in ((FakeStream(), FakeStream.cuda_stream), (None, None)):
        for call, count in ((lambda: layer.append(x, seqs, stream=stream), 1), (lambda: layer.attention(x[:, :256].contiguous(), seqs, stream=stream), 1),
                            (lambda: layer.read(seqs, 3, stream=stream), 2), (lambda: layer.heads(x, seqs, stream=stream), 2),
                            (lambda: runtime.rope_table(PLAIN, 7, "cpu", stream=stream), 1)):
            made.clear(), calls.clear()
            call()
            assert made == [want] * count and len(calls) == 1 and calls[0][1][-1] is stream and not here


def test_tensors_that_do_not_fit(calls):
    """Each would be read or written past its end, or from another device's address."""
    layer, seqs = cache(), rx.Seqs([3], [3])
    new = lambda *shape, dtype=torch.float16, device="cpu": torch.zeros(shape, dtype=dtype, device=device)
    calls.clear()
    for qkv in (new(3, 512, device="meta"), new(3, 8, 64), new(1536), new(3, 520), new(512, 3).t(), new(3, 512, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            layer.append(qkv, seqs)
        with pytest.raises(ValueError):
            layer.heads(qkv, seqs)
    for q_out in (new(2, 4, 64), new(3, 4, 64, dtype=torch.float32), new(3, 64, 4).transpose(1, 2), new(3, 4, 64, device="meta"), new(3, 4, 128)):
        with pytest.raises(ValueError):
            layer.append(new(3, 512), seqs, q_out)
    for q, out in ((new(3, 2, 64), None), (new(3, 4, 32), None), (new(3, 8, 64), None), (new(3, 4, 64, device="meta"), None), (new(3, 4, 64), new(3, 4, 32)),
                   (new(3, 4, 64), new(3, 4, 64, dtype=torch.float32)), (new(3, 4, 64), new(3, 4, 64, device="meta")), (new(3, 4, 64), new(3, 8, 64)[:, :4])):
        with pytest.raises(ValueError):
            layer.attention(q, seqs, out)
    assert not calls
    layer.append(new(3, 520)[:, :512], seqs, new(3, 256)), layer.attention(new(3, 256), seqs, new(3, 4, 64))
    assert [name for name, _ in calls] == ["relax_paged4_append", "relax_paged4_attention"]


def test_a_scaling_that_changes_does_not_change_a_layer(calls):
    """The program fills the struct anew for its next model: layers that share a table still turn what that table is for, and read no row past its end."""
    mine = rx.RopeScaling(rx.ROPE_LINEAR, 32, 10000.0, 4.0)
    first = cache(rope=mine)
    mine.rotary_dim, mine.factor = 64, 2.0
    assert first.rope.shape == (100, 16, 2) and first.rotary.rotary_dim == 32 and first.prep.c().rotary_dim == 32
    second = cache(share_from=first)
    assert second.prep.c().rotary_dim == 32 and second.rotary.rotary_dim == 32
    with pytest.raises(ValueError):
        cache(share_from=first, rope=mine)
    assert cache(share_from=first, rope=rx.RopeScaling(rx.ROPE_LINEAR, 32, 10000.0, 4.0)).prep.c().rotary_dim == 32
