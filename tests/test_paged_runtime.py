"""What the Python side of the paged cache and of the log probabilities refuses before it reaches the library, and where it allocates.  Tensors are
on the CPU and the calls that would enqueue work are replaced: nothing runs on a GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_2311_02103_amd import binding as rx
from paper_2311_02103_amd import runtime


@pytest.fixture
def calls(monkeypatch):
    """The library calls that were made, as (name, arguments); they succeed and do nothing."""
    made = []
    for name in ("relax_workspace_init", "relax_rope_table_init", "relax_paged_append", "relax_paged_attention", "relax_paged_read", "relax_token_logprobs"):
        monkeypatch.setattr(rx, name, lambda *args, name=name: made.append((name, args)) or 0)
    return made


def cache(**kw):
    base = dict(n_heads=4, n_kv_heads=2, head_dim=64, kv_capacity=100, n_pages=4, page_size=64, kv_slots=2, n_max=8, device="cpu")
    base.update(kw)
    return runtime.DevicePagedCache(**base)


@pytest.mark.parametrize("other", [dict(kv_slots=3), dict(kv_capacity=101), dict(kv_capacity=128), dict(page_size=32), dict(page_size=128, kv_capacity=100),
                                   dict(head_dim=128), dict(rope_base=None), dict(rope_base=500000.0), dict(kv_capacity=128, page_size=32)], ids=str)
def test_layers_share_only_tables_that_cover_them(calls, other):
    first = cache()
    with pytest.raises(ValueError):
        cache(share_from=first, **other)


def test_a_rotary_base_where_the_other_layer_has_none(calls):
    first = cache(rope_base=None)
    with pytest.raises(ValueError):
        cache(share_from=first, rope_base=10000.0)
    assert cache(share_from=first).rope is None and cache(share_from=first, head_dim=128, rope_base=None).rope is None


def test_tables_that_are_shared(calls):
    first = cache(rope_base=500000.0)
    for kw in (dict(), dict(kv_slots=1), dict(kv_capacity=64), dict(rope_base=500000.0), dict(n_pages=9), dict(n_kv_heads=4)):
        second = cache(share_from=first, **kw)
        assert second.pages is first.pages and second.rope is first.rope and second.ws is first.ws
        assert second.rope_base == 500000.0 and second.dims.rope_base == 500000.0 and second.cache.c().pages_per_slot == first.pages.shape[1]
    assert cache().rope_base == 10000.0
    assert cache(share_from=cache(share_from=first, kv_slots=1, kv_capacity=64)).pages is first.pages      # what counts is the tables' size
    assert cache(share_from=cache(rope_base=None), kv_capacity=128).rope is None


class FakeStream:
    cuda_stream = 0x5000


@pytest.mark.parametrize("by_address", [False, True])
def test_what_a_call_on_a_stream_allocates_belongs_to_it(calls, monkeypatch, by_address):
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

    class ExternalStream(FakeStream):
        def __init__(self, address):
            self.cuda_stream = address
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "ExternalStream", ExternalStream)
    for name in ("empty", "empty_like"):
        plain = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, plain=plain, **kw: made.append(here[-1] if here else None) or plain(*a, **kw))
    stream = FakeStream.cuda_stream if by_address else FakeStream()
    x, logits = torch.zeros((3, 8 * 64), dtype=torch.float16), torch.zeros((2, 70000), dtype=torch.float16)
    for stream, want in ((stream, FakeStream.cuda_stream), (None, None)):
        for call, count in ((lambda: layer.append(x, seqs, stream=stream), 1), (lambda: layer.attention(x[:, :256].contiguous(), seqs, stream=stream), 1),
                            (lambda: layer.read(seqs, 3, stream=stream), 2),
                            (lambda: runtime.token_logprobs(logits, torch.zeros(2, dtype=torch.int32), 4, True, stream=stream), 5)):
            made.clear(), calls.clear()
            call()
            assert made == [want] * count and len(calls) == 1 and calls[0][1][-1] is stream and not here


def test_tensors_that_do_not_fit(calls):
    """Each would be read or written past its end, or from another device's address."""
    layer, seqs = cache(), rx.Seqs([3], [3])
    new = lambda *shape, dtype=torch.float16, device="cpu": torch.zeros(shape, dtype=dtype, device=device)
    calls.clear()
    for qkv, q_out in ((new(3, 512, device="meta"), None), (new(3, 8, 64), None), (new(1536), None), (new(3, 520), None), (new(512, 3).t(), None), (new(3, 512, dtype=torch.bfloat16), None),
                       (new(3, 512), new(2, 4, 64)), (new(3, 512), new(3, 4, 64, dtype=torch.float32)), (new(3, 512), new(3, 64, 4).transpose(1, 2)),
                       (new(3, 512), new(3, 4, 64, device="meta")), (new(3, 512), new(3, 4, 128))):
        with pytest.raises(ValueError):
            layer.append(qkv, seqs, q_out)
    for q, out in ((new(3, 2, 64), None), (new(3, 4, 32), None), (new(3, 8, 64), None), (new(3, 4, 64, device="meta"), None), (new(3, 4, 64), new(3, 4, 32)),
                   (new(3, 4, 64), new(3, 4, 64, dtype=torch.float32)), (new(3, 4, 64), new(3, 4, 64, device="meta")), (new(3, 4, 64), new(3, 8, 64)[:, :4])):
        with pytest.raises(ValueError):
            layer.attention(q, seqs, out)
    logits = new(3, 100)
    for targets, ws in ((new(2, dtype=torch.int32), None), (new(3, dtype=torch.int64), None), (new(3, dtype=torch.int32, device="meta"), None),
                        (new(6, dtype=torch.int32)[::2], None), (None, new(64, dtype=torch.float32)), (None, new(64, dtype=torch.uint8, device="meta")),
                        (None, new(128, dtype=torch.uint8)[::2])):
        with pytest.raises(ValueError):
            runtime.token_logprobs(logits, targets, 3, ws=ws)
    assert not calls
    layer.append(new(3, 520)[:, :512], seqs, new(3, 256)), layer.attention(new(3, 256), seqs, new(3, 4, 64))
    runtime.token_logprobs(logits, new(3, dtype=torch.int32), 3, ws=new(512, dtype=torch.uint8))
    assert [name for name, _ in calls] == ["relax_paged_append", "relax_paged_attention", "relax_token_logprobs"]
