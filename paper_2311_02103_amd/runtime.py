"""Device-side bookkeeping around the C ABI: torch tensors that own the weights, the KV cache,
the rotary table and the workspace of one layer.  Allocation and host->device copies only."""
from __future__ import annotations

import contextlib
from typing import Dict, Optional, Sequence

import numpy as np
import torch

from . import binding as rx


def to_device(a: np.ndarray, device="cuda") -> torch.Tensor:
    """numpy uint16 (fp16 bits) -> torch.float16, uint32 -> int32 (same bits), others as is."""
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).to(device).view(torch.float16)
    if a.dtype == np.uint32:
        return torch.from_numpy(a.view(np.int32)).to(device)
    return torch.from_numpy(a).to(device)


def f16_bits(t: torch.Tensor) -> np.ndarray:
    """torch.float16 tensor -> numpy uint16 bit patterns on the host."""
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class DeviceLayer:
    """One decoder layer resident on the GPU, sized by upper bounds (n_max, L_max = kv_capacity, B_max)."""

    def __init__(self, host_weights: Dict[str, np.ndarray], *, hidden: int, n_heads: int, n_kv_heads: int, head_dim: int,
                 ffn: int, kv_capacity: int, kv_slots: int = 1, n_max: int = 1, B_max: Optional[int] = None,
                 rms_eps: float = 1e-5, rope_base: float = 10000.0, device="cuda", share_from: "DeviceLayer" = None, group: int = 32):
        self.device = device
        self.dims = rx.make_dims(hidden, n_heads, n_kv_heads, head_dim, ffn, kv_capacity, kv_slots, rms_eps, rope_base, group)
        mats = {"wqkv": ((n_heads + 2 * n_kv_heads) * head_dim, hidden), "wo": (hidden, n_heads * head_dim),
                "wgu": (2 * ffn, hidden), "wdown": (hidden, ffn)}
        self.t = {k: to_device(v, device) for k, v in host_weights.items()}
        self.weights = rx.LayerWeights(*(rx.QMat(self.t[n + ".q"], self.t[n + ".s"], *mats[n], group) for n in mats),
                                       self.t["norm_attn"], self.t["norm_ffn"])
        self.n_max, self.B_max = n_max, (B_max if B_max is not None else max(kv_slots, 1))
        if share_from is not None:          # layers of one model share cache geometry, rope table and workspace
            self.rope, self.ws, self.ws_bytes = share_from.rope, share_from.ws, share_from.ws_bytes
        else:
            self.rope = torch.empty(rx.relax_rope_table_bytes(self.dims) // 4, dtype=torch.float32, device=device)
            rx.check(rx.relax_rope_table_init(self.dims, self.rope), "relax_rope_table_init")
            self.ws_bytes = rx.relax_workspace_bytes(self.dims, n_max, kv_capacity, self.B_max)
            self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
            rx.check(rx.relax_workspace_init(self.dims, self.ws, self.ws_bytes), "relax_workspace_init")
        shape = (kv_slots, kv_capacity, n_kv_heads, head_dim)
        self.k = torch.zeros(shape, dtype=torch.float16, device=device)
        self.v = torch.zeros(shape, dtype=torch.float16, device=device)
        self.cache = rx.KVCache(self.k, self.v, self.rope)

    def load_cache(self, k_bits: np.ndarray, v_bits: np.ndarray) -> None:
        self.k.copy_(to_device(k_bits, self.device).view(self.k.shape))
        self.v.copy_(to_device(v_bits, self.device).view(self.v.shape))

    def forward(self, x: torch.Tensor, q_lens: Sequence[int], kv_lens: Sequence[int], slots=None,
                out: Optional[torch.Tensor] = None, device_table: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        n = x.shape[0]
        if out is None:
            out = torch.empty_like(x)
        seqs = rx.Seqs(q_lens, kv_lens, slots, device_table)
        rx.check(rx.relax_decoder_layer(self.dims, self.weights, x, self.cache, seqs, out, n, self.ws, self.ws_bytes, stream),
                 "relax_decoder_layer")
        return out

    def prepare(self, x: torch.Tensor, q_lens: Sequence[int], kv_lens: Sequence[int], slots=None,
                out: Optional[torch.Tensor] = None, stream=None):
        """Marshal one relax_decoder_layer call once; the returned closure only crosses the C boundary.
        The symbolic values (n, every L_b) are still plain arguments of that C call."""
        import ctypes as C
        n = x.shape[0]
        out = torch.empty_like(x) if out is None else out
        seqs = rx.Seqs(q_lens, kv_lens, slots)
        keep = (seqs, self.weights.c(), self.cache.c(), seqs.c(), x, out)
        fn = rx.lib().relax_decoder_layer
        args = (C.byref(self.dims), C.byref(keep[1]), x.data_ptr(), C.byref(keep[2]), C.byref(keep[3]), out.data_ptr(), n,
                self.ws.data_ptr(), self.ws_bytes)

        def call(stream_handle=None):
            rc = fn(*args, stream_handle if stream_handle is not None else rx._stream(stream))
            if rc != 0:
                raise rx.RelaxError(rc, "relax_decoder_layer")
            return out

        call.keep = keep
        return call


class DeviceModel:
    """A stack of decoder layers with embedding, final norm and fp16 LM head resident on the GPU.

    layer_weights: one host dict per layer (as DeviceLayer takes); a dict may appear several times in the list
    (weight sharing between layers keeps big synthetic models small on the host) -- its device copy is shared too,
    each layer still has its own KV cache."""

    def __init__(self, layer_weights: Sequence[Dict[str, np.ndarray]], embedding_bits: np.ndarray, norm_final_bits: np.ndarray,
                 lm_head_bits: np.ndarray, *, hidden: int, n_heads: int, n_kv_heads: int, head_dim: int, ffn: int,
                 kv_capacity: int, kv_slots: int = 1, n_max: int = 1, B_max: Optional[int] = None, rms_eps: float = 1e-5,
                 rope_base: float = 10000.0, device="cuda", group: int = 32):
        self.device = device
        self.dims = rx.make_dims(hidden, n_heads, n_kv_heads, head_dim, ffn, kv_capacity, kv_slots, rms_eps, rope_base, group)
        self.vocab = int(embedding_bits.shape[0])
        mats = {"wqkv": ((n_heads + 2 * n_kv_heads) * head_dim, hidden), "wo": (hidden, n_heads * head_dim),
                "wgu": (2 * ffn, hidden), "wdown": (hidden, ffn)}
        uploaded = {}
        self.layers = []
        for hw in layer_weights:
            if id(hw) not in uploaded:
                t = {k: to_device(v, device) for k, v in hw.items()}
                uploaded[id(hw)] = (t, rx.LayerWeights(*(rx.QMat(t[n + ".q"], t[n + ".s"], *mats[n], group) for n in mats),
                                                       t["norm_attn"], t["norm_ffn"]))
            self.layers.append(uploaded[id(hw)][1])
        self._tensors = uploaded
        self.embedding = to_device(embedding_bits, device)
        self.norm_final = to_device(norm_final_bits, device)
        self.lm_head = to_device(lm_head_bits, device)
        self.model = rx.Model(self.dims, self.layers, self.vocab, self.embedding, self.norm_final, self.lm_head)
        self.n_max, self.B_max = n_max, (B_max if B_max is not None else max(kv_slots, 1))
        self.rope = torch.empty(rx.relax_rope_table_bytes(self.dims) // 4, dtype=torch.float32, device=device)
        rx.check(rx.relax_rope_table_init(self.dims, self.rope), "relax_rope_table_init")
        self.ws_bytes = rx.relax_model_workspace_bytes(self.model, n_max, kv_capacity, self.B_max)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        rx.check(rx.relax_workspace_init(self.dims, self.ws, self.ws_bytes), "relax_workspace_init")
        shape = (kv_slots, kv_capacity, n_kv_heads, head_dim)
        self.k = [torch.zeros(shape, dtype=torch.float16, device=device) for _ in self.layers]
        self.v = [torch.zeros(shape, dtype=torch.float16, device=device) for _ in self.layers]
        self.caches = [rx.KVCache(k, v, self.rope) for k, v in zip(self.k, self.v)]

    def step(self, ids: torch.Tensor, q_lens: Sequence[int], kv_lens: Sequence[int], slots=None,
             logits: Optional[torch.Tensor] = None, next_ids: Optional[torch.Tensor] = None, stream=None,
             device_table: Optional[torch.Tensor] = None):
        """ids: int32 [n] on the device.  Returns (logits fp16 [B,V], next_ids int32 [B]).  With device_table (int32 [4][B] on
        the device: q_start, q_len, kv_len, slot) the kernels read positions there and kv_lens are upper bounds."""
        B = len(q_lens)
        if logits is None:
            logits = torch.empty((B, self.vocab), dtype=torch.float16, device=self.device)
        if next_ids is None:
            next_ids = torch.empty((B,), dtype=torch.int32, device=self.device)
        rx.check(rx.relax_model_step(self.model, ids, self.caches, rx.Seqs(q_lens, kv_lens, slots, device_table), logits, next_ids,
                                     int(ids.shape[0]), self.ws, self.ws_bytes, stream), "relax_model_step")
        return logits, next_ids


def _allocating_for(stream):
    """Context in which torch's new tensors belong to `stream` (as the calls take it: None, a torch stream or its address).  Memory of another stream
    could be handed out again while the kernels on this one still use it, or still be in use there."""
    if stream is None:
        return contextlib.nullcontext()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


def _check_tensor(t: torch.Tensor, dtype, count: int, device, what: str) -> None:
    """The calls take an address and count elements from there."""
    if t.dtype != dtype or t.numel() != count or not t.is_contiguous() or t.device != device:
        raise ValueError("%s: %d elements of %s, contiguous, on %s" % (what, count, dtype, device))


_NOT_GIVEN = object()


class DevicePagedCache:
    """The 8-bit paged KV cache of one layer: the pool, its scales, the page table `pages` (int32 [kv_slots, pages per slot], written by the caller, who
    hands out the pool's pages), the rotary table and the workspace, sized by upper bounds (n_max, L_max = kv_capacity, B_max).  rope_base: 10000 if not
    given, None: no rotation.  share_from: another layer's page table, rotary table and workspace, which have to cover this one's slots and positions;
    rope_base is then the other layer's.  Tensors that a call with `stream` returns belong to that stream, as under torch.cuda.stream."""

    def __init__(self, *, n_heads: int, n_kv_heads: int, head_dim: int, kv_capacity: int, n_pages: int, page_size: int = 64, kv_slots: int = 1,
                 n_max: int = 1, B_max: Optional[int] = None, rope_base: Optional[float] = _NOT_GIVEN, device="cuda", share_from: "DevicePagedCache" = None):
        self.device, self.page_size = device, page_size
        self.rope_base = rope_base if rope_base is not _NOT_GIVEN else 10000.0 if share_from is None else share_from.rope_base
        self.dims = rx.make_dims(n_heads * head_dim, n_heads, n_kv_heads, head_dim, 64, kv_capacity, kv_slots, rope_base=self.rope_base or 10000.0)
        self.n_max, self.B_max = n_max, (B_max if B_max is not None else max(kv_slots, 1))
        if share_from is not None:          # layers of one model share the page table, the rotary table and the workspace
            self._check_shared(share_from)
            self.pages, self.rope, self.ws, self.ws_bytes = share_from.pages, share_from.rope, share_from.ws, share_from.ws_bytes
        else:
            self.pages = torch.full((kv_slots, -(-kv_capacity // page_size)), -1, dtype=torch.int32, device=device)
            self.rope = None
            if self.rope_base is not None:
                self.rope = torch.empty(rx.relax_rope_table_bytes(self.dims) // 4, dtype=torch.float32, device=device)
                rx.check(rx.relax_rope_table_init(self.dims, self.rope), "relax_rope_table_init")
            self.ws_bytes = rx.relax_paged_workspace_bytes(self.dims, n_max, kv_capacity, self.B_max)
            self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
            rx.check(rx.relax_workspace_init(self.dims, self.ws, self.ws_bytes), "relax_workspace_init")
        shape = (n_pages, n_kv_heads, page_size // rx.RELAX_PAGED_BLOCK, rx.RELAX_PAGED_BLOCK * head_dim)
        self.k, self.v = (torch.empty(shape, dtype=torch.uint8, device=device) for _ in "kv")
        self.k_scale, self.v_scale = (torch.empty(shape[:3], dtype=torch.float32, device=device) for _ in "kv")
        self.cache = rx.PagedCache(self.k, self.v, self.k_scale, self.v_scale, self.pages, self.rope, n_pages, page_size, self.pages.shape[1])

    def _check_shared(self, other: "DevicePagedCache") -> None:
        """The kernels index the shared tables by this layer's sizes, which the C calls cannot compare with the tables'."""
        slots, positions = other.pages.shape[0], other.pages.shape[1] * other.page_size
        if other.rope is not None:          # [kv_capacity, d / 2, 2]
            positions = min(positions, other.rope.numel() // other.dims.head_dim)
        if self.page_size != other.page_size:
            raise ValueError("share_from: pages of %d tokens, the table's are of %d" % (self.page_size, other.page_size))
        if self.dims.kv_slots > slots or self.dims.kv_capacity > positions:
            raise ValueError("share_from: %d slots of %d positions on tables for %d of %d" % (self.dims.kv_slots, self.dims.kv_capacity, slots, positions))
        if self.rope_base != other.rope_base or (other.rope is not None and self.dims.head_dim != other.dims.head_dim):
            raise ValueError("share_from: the rotary table has another base or head_dim")
        if torch.empty(0, device=self.device).device != other.pages.device:
            raise ValueError("share_from: the tables are on another device")

    def append(self, qkv: torch.Tensor, seqs: "rx.Seqs", q_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """qkv: fp16 [n, (h + 2 g) d], rows contiguous (any stride between them).  Returns q, rotated, fp16 [n, h, d]."""
        h, g, d = self.dims.n_heads, self.dims.n_kv_heads, self.dims.head_dim
        if qkv.dtype != torch.float16 or qkv.dim() != 2 or qkv.shape[1] != (h + 2 * g) * d or qkv.stride(1) != 1 or qkv.device != self.pages.device:
            raise ValueError("qkv is fp16 [n, (h + 2 g) d] with contiguous rows, on the cache's device")
        n, at = qkv.shape[0], qkv.data_ptr()
        pitch = qkv.stride(0) if n > 1 else qkv.shape[1]
        if q_out is not None:
            _check_tensor(q_out, torch.float16, n * h * d, self.pages.device, "q_out [n, h, d]")
        else:
            with _allocating_for(stream):
                q_out = torch.empty((n, h, d), dtype=torch.float16, device=self.device)
        rx.check(rx.relax_paged_append(at, pitch, at + 2 * h * d, at + 2 * (h + g) * d, pitch, q_out, self.cache, seqs, self.dims, n,
                                       self.ws, self.ws_bytes, stream), "relax_paged_append")
        return q_out

    def attention(self, q: torch.Tensor, seqs: "rx.Seqs", out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        count = q.shape[0] * self.dims.n_heads * self.dims.head_dim
        _check_tensor(q, torch.float16, count, self.pages.device, "q [n, h, d]")
        if out is not None:
            _check_tensor(out, torch.float16, count, self.pages.device, "out [n, h, d]")
        else:
            with _allocating_for(stream):
                out = torch.empty_like(q)
        rx.check(rx.relax_paged_attention(q, self.cache, seqs, self.dims, out, q.shape[0], self.ws, self.ws_bytes, stream), "relax_paged_attention")
        return out

    def read(self, seqs: "rx.Seqs", n: int, stream=None):
        """(k, v) of the call's n rows as fp16 [n, g, d]."""
        with _allocating_for(stream):
            k, v = (torch.empty((n, self.dims.n_kv_heads, self.dims.head_dim), dtype=torch.float16, device=self.device) for _ in "kv")
        rx.check(rx.relax_paged_read(self.cache, seqs, self.dims, k, v, n, self.ws, self.ws_bytes, stream), "relax_paged_read")
        return k, v


def token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, top: int = 0, entropy: bool = False, ws: Optional[torch.Tensor] = None, stream=None):
    """relax_token_logprobs on fp16 logits [n, V], targets int32 [n]: (logprobs, entropy, top_ids, top_logprobs), None where not asked for.  ws: uint8, else made here.
    What is made here belongs to `stream`, as under torch.cuda.stream."""
    n, vocab = logits.shape
    if logits.dtype != torch.float16 or (vocab > 1 and logits.stride(1) != 1):
        raise ValueError("logits are fp16 [n, V] with contiguous rows")
    if targets is not None:
        _check_tensor(targets, torch.int32, n, logits.device, "targets [n]")
    if ws is not None:
        _check_tensor(ws, torch.uint8, ws.numel(), logits.device, "ws")
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=logits.device)
    with _allocating_for(stream):
        if ws is None:
            ws = new(rx.relax_token_logprobs_workspace_bytes(n, vocab, top), dtype=torch.uint8)
        lp, ent = new(n) if targets is not None else None, new(n) if entropy else None
        ids, tops = (new(n, top, dtype=torch.int32), new(n, top)) if top else (None, None)
    rx.check(rx.relax_token_logprobs(logits, logits.stride(0) if n > 1 else vocab, targets, lp, ent, ids, tops, n, vocab, top, ws, ws.numel(), stream), "relax_token_logprobs")
    return lp, ent, ids, tops


class DeviceLayerQ3:
    """One decoder layer on 3-bit weights resident on the GPU: the canonical matrices are uploaded, repacked once into the
    GPU-native layout (relax_repack_q3) and dropped; cache, rotary table and workspace as in DeviceLayer."""

    def __init__(self, host_weights: Dict[str, np.ndarray], *, hidden: int, n_heads: int, n_kv_heads: int, head_dim: int,
                 ffn: int, kv_capacity: int, kv_slots: int = 1, n_max: int = 1, B_max: Optional[int] = None,
                 rms_eps: float = 1e-5, rope_base: float = 10000.0, device="cuda"):
        self.device = device
        self.dims = rx.make_dims(hidden, n_heads, n_kv_heads, head_dim, ffn, kv_capacity, kv_slots, rms_eps, rope_base, 32)
        mats = {"wqkv": ((n_heads + 2 * n_kv_heads) * head_dim, hidden), "wo": (hidden, n_heads * head_dim),
                "wgu": (2 * ffn, hidden), "wdown": (hidden, ffn)}
        self.t = {}
        qm = []
        for name, (m, k) in mats.items():
            canon, sc = to_device(host_weights[name + ".q"], device), to_device(host_weights[name + ".s"], device)
            native = torch.empty_like(canon)
            rx.check(rx.relax_repack_q3(rx.QMat(canon, sc, m, k, 32), native), "relax_repack_q3")
            torch.cuda.synchronize()
            self.t[name + ".q"], self.t[name + ".s"] = native, sc
            qm.append(rx.QMat(native, sc, m, k, 32))
        self.t["norm_attn"], self.t["norm_ffn"] = to_device(host_weights["norm_attn"], device), to_device(host_weights["norm_ffn"], device)
        self.weights = rx.LayerWeights(*qm, self.t["norm_attn"], self.t["norm_ffn"])
        self.n_max, self.B_max = n_max, (B_max if B_max is not None else max(kv_slots, 1))
        self.rope = torch.empty(rx.relax_rope_table_bytes(self.dims) // 4, dtype=torch.float32, device=device)
        rx.check(rx.relax_rope_table_init(self.dims, self.rope), "relax_rope_table_init")
        self.ws_bytes = rx.relax_layer_q3_workspace_bytes(self.dims, n_max, kv_capacity, self.B_max)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        shape = (kv_slots, kv_capacity, n_kv_heads, head_dim)
        self.k = torch.zeros(shape, dtype=torch.float16, device=device)
        self.v = torch.zeros(shape, dtype=torch.float16, device=device)
        self.cache = rx.KVCache(self.k, self.v, self.rope)

    def load_cache(self, k_bits: np.ndarray, v_bits: np.ndarray) -> None:
        self.k.copy_(to_device(k_bits, self.device).view(self.k.shape))
        self.v.copy_(to_device(v_bits, self.device).view(self.v.shape))

    def forward(self, x: torch.Tensor, q_lens: Sequence[int], kv_lens: Sequence[int], slots=None,
                out: Optional[torch.Tensor] = None, device_table: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        n = x.shape[0]
        if out is None:
            out = torch.empty_like(x)
        seqs = rx.Seqs(q_lens, kv_lens, slots, device_table)
        rx.check(rx.relax_decoder_layer_q3(self.dims, self.weights, x, self.cache, seqs, out, n, self.ws, self.ws_bytes, stream),
                 "relax_decoder_layer_q3")
        return out


class DeviceLayerF16:
    """One decoder layer on plain fp16 weights resident on the GPU.  host_weights: 'wqkv', 'wo', 'wgu', 'wdown' as fp16 bit
    patterns [m,k] and the two norm vectors."""

    def __init__(self, host_weights: Dict[str, np.ndarray], *, hidden: int, n_heads: int, n_kv_heads: int, head_dim: int,
                 ffn: int, kv_capacity: int, kv_slots: int = 1, n_max: int = 1, B_max: Optional[int] = None,
                 rms_eps: float = 1e-5, rope_base: float = 10000.0, device="cuda"):
        self.device = device
        self.dims = rx.make_dims(hidden, n_heads, n_kv_heads, head_dim, ffn, kv_capacity, kv_slots, rms_eps, rope_base, 32)
        names = ("wqkv", "wo", "wgu", "wdown", "norm_attn", "norm_ffn")
        self.t = {k: to_device(host_weights[k], device) for k in names}
        self.weights = [self.t[k] for k in names]
        self.n_max, self.B_max = n_max, (B_max if B_max is not None else max(kv_slots, 1))
        self.rope = torch.empty(rx.relax_rope_table_bytes(self.dims) // 4, dtype=torch.float32, device=device)
        rx.check(rx.relax_rope_table_init(self.dims, self.rope), "relax_rope_table_init")
        self.ws_bytes = rx.relax_layer_f16_workspace_bytes(self.dims, n_max, kv_capacity, self.B_max)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        shape = (kv_slots, kv_capacity, n_kv_heads, head_dim)
        self.k = torch.zeros(shape, dtype=torch.float16, device=device)
        self.v = torch.zeros(shape, dtype=torch.float16, device=device)
        self.cache = rx.KVCache(self.k, self.v, self.rope)

    def load_cache(self, k_bits: np.ndarray, v_bits: np.ndarray) -> None:
        self.k.copy_(to_device(k_bits, self.device).view(self.k.shape))
        self.v.copy_(to_device(v_bits, self.device).view(self.v.shape))

    def forward(self, x: torch.Tensor, q_lens: Sequence[int], kv_lens: Sequence[int], slots=None,
                out: Optional[torch.Tensor] = None, device_table: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        n = x.shape[0]
        if out is None:
            out = torch.empty_like(x)
        seqs = rx.Seqs(q_lens, kv_lens, slots, device_table)
        rx.check(rx.relax_decoder_layer_f16(self.dims, self.weights, x, self.cache, seqs, out, n, self.ws, self.ws_bytes, stream),
                 "relax_decoder_layer_f16")
        return out
