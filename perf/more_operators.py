"""Operators of a serving step around a paged 4-bit KV cache, as they are measured: the calls, their plain form in elementary torch
operations, the work they cannot do without and their result in 64 bits.

  table       the rotary table of a model whose positions are stretched for long contexts (relax_rope_table_scaled)
  heads       queries and keys of a ragged call, normalised head by head and rotated in one pass (relax_head_norm_rope)
  append      the same on the way into the paged 4-bit cache, with the values (relax_paged4_append); what the cache then holds of the
              call's rows is read back (relax_paged4_read)
  attention   causal attention of a ragged call over the paged 4-bit cache (relax_paged4_attention)

Heads.  x' = x * w / sqrt(mean(x^2) + eps) over a head's elements where there are weights w, then the first `rotary` elements turn, in
pairs (e, e + rotary / 2) ("halves") or (2 e, 2 e + 1) ("pairs"), each product and sum rounded to 32 bits, the sum of squares in 64.

The cache.  Positions of a sequence are cut into pages of `page` tokens, a page into blocks of 16.  32 elements of a token are a group
with one scale s and codes u in 0..15 that stand for (u - 8) * s: s is the element of the largest magnitude (the positive one of two)
over -8, rounded to eight significant bits and at most 8160 in size, u = 8 + clamp(round(x / s), -8, 7).
  k codes  [pages][kv_heads][page / 16][4][16][d / 32][4 bytes]    byte b of token t: [e / 8 % 4][t][e / 32], element e % 8 = 4 (b % 2) + b / 2
                                                                   in its low half, that + 2 in its high half
  v codes  [pages][kv_heads][page / 16][4][16][d / 32][4 bytes]    [t / 4][e % 16][e / 32], token t % 4 = 2 (b % 2) + b / 2 in byte b, element
                                                                   e / 16 % 2 = 0 in its low half, 1 in its high half
  scales   [pages][kv_heads][page / 16][t / 4][e / 32][t % 4] fp16

The keys of a case:

  op          "table" | "heads" | "append" | "attention"
  heads, kv_heads, head_dim, page
  prompt, past                              rows of one sequence (0: no such sequence) on top of `past` cached tokens
  decodes, each, len_first, len_step        further sequences with `each` rows, lengths len_first + b * len_step
  norm, layout, rotary                      of "heads" and "append"
  positions, rotary, base, scaling, factor, trained      of a "table" case
"""
from __future__ import annotations

import math

import torch

own = False

ROPE_BASE = 10000.0
EPS = 2.0 ** -17
BLOCK, GROUP = 16, 32
SLOW, FAST = 1.0, 4.0                     # turns within the trained context, "wavelength"
INDEX_SLOW, INDEX_FAST = 1.0, 32.0        # "index"

TINY = dict(heads=4, kv_heads=4, head_dim=64)
B7 = dict(heads=32, kv_heads=32, head_dim=128)
B70 = dict(heads=64, kv_heads=8, head_dim=128)
GROUPED = dict(heads=32, kv_heads=8, head_dim=128)


def _call(op, shape, page=16, prompt=0, past=0, decodes=0, each=1, len_first=0, len_step=0, **more):
    return dict(op=op, page=page, prompt=prompt, past=past, decodes=decodes, each=each, len_first=len_first, len_step=len_step, **shape, **more)


def _prep(norm, layout, rotary):
    return dict(norm=norm, layout=layout, rotary=rotary)


def _table(positions, rotary, base, scaling, factor, trained):
    return dict(op="table", positions=positions, rotary=rotary, base=base, scaling=scaling, factor=factor, trained=trained)


def listed():
    return [
        # a context of 2048 stretched four times, part of the head
        dict(name="table_8192", **_table(8192, 64, 10000.0, "linear", 4.0, 2048)),
        # a long-document model: slow pairs are stretched, fast ones stay
        dict(name="table_131071", **_table(131071, 128, 500000.0, "wavelength", 8.0, 8192)),
        # one token of one user: nothing but latency
        dict(name="heads_1", **_call("heads", B70, decodes=1, len_first=2231, **_prep(True, "halves", 128))),
        # a prompt of odd length; half of each head turns, by neighbours
        dict(name="heads_prompt_2043", **_call("heads", GROUPED, prompt=2043, past=5, **_prep(True, "pairs", 64))),
        # one token of one user goes into the middle of a block
        dict(name="append_1", **_call("append", B7, decodes=1, len_first=2231, **_prep(False, "halves", 128))),
        # a batch of sixty-four decoding users with grouped heads and normalised queries and keys
        dict(name="append_64", **_call("append", B70, decodes=64, len_first=128, len_step=61, **_prep(True, "halves", 128))),
        # a prompt of odd length behind a cached beginning that ends inside a block
        dict(name="append_prompt_2043", **_call("append", B7, page=64, prompt=2043, past=5, **_prep(False, "halves", 128))),
        # the smallest model: one token on a short context
        dict(name="attention_tiny", **_call("attention", TINY, decodes=1, len_first=53)),
        # sixteen users between 100 and 8000 tokens with grouped heads
        dict(name="attention_16", **_call("attention", B70, page=32, decodes=16, len_first=100, len_step=526)),
        # one user with a very long document
        dict(name="attention_long", **_call("attention", B70, page=64, decodes=1, len_first=120001)),
        # drafted tokens of eight users are checked beside a chunk of a prompt
        dict(name="attention_drafts", **_call("attention", GROUPED, prompt=300, past=1201, decodes=8, each=5, len_first=700, len_step=391)),
        # a long prompt with grouped heads
        dict(name="attention_4096", **_call("attention", GROUPED, page=64, prompt=4096)),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _ragged(rng, count, each, longest):
    first = max(each, _log(rng, 1, max(2, longest // 2)))
    return dict(decodes=count, each=each, len_first=first, len_step=rng.randint(0, max(0, (longest - first) // max(1, count))))


def draw(rng):
    """One more case of the ranges above."""
    op = rng.choice(["table", "heads", "heads", "append", "append", "append", "attention", "attention", "attention", "attention", "attention"])
    if op == "table":
        trained = rng.choice([1024, 2048, 4096, 8192])
        return _table(_log(rng, 50, 131071), 16 * rng.randint(1, 8), rng.choice([10000.0, 500000.0]), rng.choice(["plain", "linear", "index", "wavelength"]),
                      round(rng.uniform(1.0, 32.0), 2), trained)
    shape, page = rng.choice([TINY, B7, B70, GROUPED, dict(heads=40, kv_heads=40, head_dim=128), dict(heads=16, kv_heads=2, head_dim=64)]), rng.choice([16, 32, 64, 128])
    wide = shape["kv_heads"] >= 32
    d = shape["head_dim"]
    more = {} if op == "attention" else _prep(rng.random() < 0.5, rng.choice(["halves", "pairs"]), rng.choice([d, d, d // 2, d // 4, 16 * rng.randint(1, d // 16)]))
    kind = rng.choice(["one", "batch", "batch", "drafts", "mixed", "prompt"])
    if kind == "one":
        return _call(op, shape, page, **_ragged(rng, 1, 1, 20000 if wide else 120000), **more)
    if kind == "batch":
        return _call(op, shape, page, **_ragged(rng, _log(rng, 2, 64), 1, 1000 if wide else rng.choice([600, 2000, 4000])), **more)
    if kind == "drafts":
        return _call(op, shape, page, **_ragged(rng, _log(rng, 1, 16), rng.randint(2, 17), 2000), **more)
    if kind == "mixed":
        return _call(op, shape, page, prompt=_log(rng, 2, 300), past=rng.randint(0, 1200), **_ragged(rng, _log(rng, 1, 20), 1, 1100), **more)
    return _call(op, shape, page, prompt=_log(rng, 2, 2043), past=rng.choice([0, rng.randint(1, 600)]), **more)


# ---- shapes of a call -----------------------------------------------------------------------------------------------
def _seqs(c):
    """(q_lens, kv_lens) of the call: the prompt first, then the other sequences."""
    q, kv = [], []
    if c["prompt"]:
        q, kv = [c["prompt"]], [c["past"] + c["prompt"]]
    return q + [c["each"]] * c["decodes"], kv + [c["len_first"] + b * c["len_step"] for b in range(c["decodes"])]


def _pages_per_slot(c):
    return max((L + c["page"] - 1) // c["page"] for L in _seqs(c)[1])


def _capacity(c):
    return _pages_per_slot(c) * c["page"]


def work(c):
    if c["op"] == "table":
        return {"bytes": c["positions"] * c["rotary"] * 4, "flops": 6 * c["positions"] * c["rotary"]}
    q, kv = _seqs(c)
    n, h, g, d = sum(q), c["heads"], c["kv_heads"], c["head_dim"]
    held = 2 * g * (d // 2 + 2 * d // GROUP)    # bytes of a token in the cache
    if c["op"] == "heads":                      # rows in and out, the angles of each row
        return {"bytes": 2 * n * (h + g) * d * 2 + n * c["rotary"] * 4, "flops": n * (h + g) * (4 * d * c["norm"] + 3 * c["rotary"])}
    if c["op"] == "append":                     # rows in, q out, codes out; codes in again, values out
        return {"bytes": n * (2 * h + 2 * g) * d * 2 + n * c["rotary"] * 4 + 2 * n * held + 2 * n * g * d * 2,
                "flops": n * (h + g) * (4 * d * c["norm"] + 3 * c["rotary"]) + 8 * n * g * d}
    pairs = sum(ql * (L - ql) + ql * (ql + 1) // 2 for ql, L in zip(q, kv))
    return {"bytes": sum(kv) * held + 2 * n * h * d * 2, "flops": 4 * pairs * h * d}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _gen(seed, tensor):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + tensor)
    return g


def _normal(seed, tensor, shape, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=_gen(seed, tensor))


def _pool(c, seed, tensor):
    """(codes [pages, kv_heads, blocks, 16, d] uint8, scales [pages, kv_heads, blocks, 16, d / 32] fp16) of N(0, 1) values, some of them in
    blocks that no sequence has reached yet."""
    pages, g, d, blocks = _pool_pages(c), c["kv_heads"], c["head_dim"], c["page"] // BLOCK
    x = _normal(seed, tensor, (pages, g, blocks, BLOCK, d // GROUP, GROUP))
    top, low = x.amax(dim=5), x.amin(dim=5)
    s = (torch.where(top >= -low, top, low) / -8.0).bfloat16().float()
    x /= s[..., None]
    return x.round_().clamp_(-8, 7).add_(8).to(torch.uint8).view(pages, g, blocks, BLOCK, d), s.half()


def _pool_pages(c):
    return len(_seqs(c)[0]) * _pages_per_slot(c) + 3


def _angle_table(positions, rotary):
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * ROPE_BASE ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / rotary)
    return torch.stack([angle.cos(), angle.sin()], dim=2).float()


def _page_table(c, seed):
    slots, per = len(_seqs(c)[0]), _pages_per_slot(c)
    order = torch.randperm(_pool_pages(c), device="cuda", generator=_gen(seed, 9))
    return order[:slots * per].view(slots, per).to(torch.int32)


def _rows_in(c, seed):
    return _normal(seed, 5, (sum(_seqs(c)[0]), (c["heads"] + 2 * c["kv_heads"]) * c["head_dim"])).half()


def _norms(c, seed):
    return [(1.0 + _normal(seed, t, (c["head_dim"],), 0.1)).half() for t in (6, 7)]


def prepare(c, seed):
    if c["op"] == "table":                      # bases of models differ a little from seed to seed
        return {"case": c, "base": _base(c, seed)}
    state = {"case": c}
    if c["op"] != "attention":
        state["qkv"] = _rows_in(c, seed)
        state["rope"] = _angle_table(_capacity(c), c["rotary"])
        state["norms"] = _norms(c, seed) if c["norm"] else None
    if c["op"] == "heads":
        return state
    d = c["head_dim"]
    state["pages"] = _page_table(c, seed)
    for name, tensor in (("k", 3), ("v", 4)):
        codes, scale = _pool(c, seed, tensor)
        state[name] = _packed(codes, name)
        lead = codes.shape[:3]
        state[name + "_scale"] = scale.view(*lead, 4, 4, d // GROUP).transpose(4, 5).contiguous()
    if c["op"] == "attention":
        state["q"] = _normal(seed, 5, (sum(_seqs(c)[0]), c["heads"], d)).half()
    return state


def _base(c, seed):
    return c["base"] * (1.0 + (seed % 1024) / 4096.0)


def _packed(codes, name):
    """codes [pages, kv_heads, blocks, 16, d] as the cache lays them out: [pages, kv_heads, blocks, 4, 16, d / 32, 4]."""
    lead, d = codes.shape[:3], codes.shape[4]
    if name == "k":
        x = codes.view(*lead, 16, d // 32, 4, 2, 2, 2).permute(0, 1, 2, 5, 3, 4, 8, 6, 7)      # [.., 4, 16, d / 32, byte / 2, byte % 2, half]
    else:
        x = codes.view(*lead, 4, 2, 2, d // 32, 2, 16).permute(0, 1, 2, 3, 8, 6, 5, 4, 7)
    return (x[..., 0] + 16 * x[..., 1]).reshape(*lead, 4, 16, d // 32, 4).contiguous()


# ---- the framework's calls ------------------------------------------------------------------------------------------
def _own_setup(state):
    """What a program makes once: the model's sizes, how its heads are prepared, the descriptor of the cache and a workspace."""
    from paper_2311_02103_amd import binding as rx

    c = state["case"]
    q, kv = _seqs(c)
    state["dims"] = rx.make_dims(c["heads"] * c["head_dim"], c["heads"], c["kv_heads"], c["head_dim"], 4 * c["heads"] * c["head_dim"], _capacity(c), len(q))
    if c["op"] != "attention":
        state["prep"] = rx.HeadPrep(*(state["norms"] or (None, None)), EPS, state["rope"], c["rotary"], rx.ROPE_HALVES if c["layout"] == "halves" else rx.ROPE_PAIRS)
    if c["op"] == "heads":
        state["ws_bytes"] = rx.relax_head_workspace_bytes(state["dims"], len(q))
    else:
        state["cache"] = rx.Paged4Cache(state["k"], state["v"], state["k_scale"], state["v_scale"], state["pages"], state["k"].shape[0], c["page"],
                                        state["pages"].shape[1])
        state["ws_bytes"] = rx.relax_paged4_workspace_bytes(state["dims"], sum(q), max(kv), len(q))
    state["ws"] = torch.empty(state["ws_bytes"], dtype=torch.uint8, device="cuda")
    state["lens"] = (q, kv)


def _run_own(state):
    from paper_2311_02103_amd import binding as rx

    c = state["case"]
    if c["op"] == "table":
        how = {"plain": rx.ROPE_PLAIN, "linear": rx.ROPE_LINEAR, "index": rx.ROPE_INDEX_RAMP, "wavelength": rx.ROPE_WAVELENGTH_RAMP}[c["scaling"]]
        slow, fast, amplitude = _ramp(c)
        out = torch.empty((c["positions"], c["rotary"] // 2, 2), dtype=torch.float32, device="cuda")
        rx.check(rx.relax_rope_table_scaled(rx.RopeScaling(how, c["rotary"], state["base"], c["factor"], c["trained"], slow, fast, amplitude), c["positions"], out),
                 "relax_rope_table_scaled")
        return [out]
    if "ws" not in state:
        _own_setup(state)
    h, g, d = c["heads"], c["kv_heads"], c["head_dim"]
    dims, ws = state["dims"], (state["ws"], state["ws_bytes"])
    seqs = rx.Seqs(*state["lens"])
    if c["op"] == "attention":
        out = torch.empty_like(state["q"])
        rx.check(rx.relax_paged4_attention(state["q"], state["cache"], seqs, dims, out, out.shape[0], *ws), "relax_paged4_attention")
        return [out]
    qkv = state["qkv"]
    n, row, base = qkv.shape[0], qkv.shape[1], qkv.data_ptr()
    q_out = torch.empty((n, h, d), dtype=torch.float16, device="cuda")
    if c["op"] == "heads":
        k_out = torch.empty((n, g, d), dtype=torch.float16, device="cuda")
        rx.check(rx.relax_head_norm_rope(base, row, base + 2 * h * d, row, q_out, h * d, k_out, g * d, state["prep"], seqs, dims, n, *ws), "relax_head_norm_rope")
        return [q_out, k_out]
    cache = state["cache"]
    rx.check(rx.relax_paged4_append(base, row, base + 2 * h * d, base + 2 * (h + g) * d, row, q_out, state["prep"], cache, seqs, dims, n, *ws), "relax_paged4_append")
    back = torch.empty((2, n, g, d), dtype=torch.float16, device="cuda")
    rx.check(rx.relax_paged4_read(cache, seqs, dims, back[0], back[1], n, *ws), "relax_paged4_read")
    return [q_out, back[0], back[1]]


# ---- the plain form -------------------------------------------------------------------------------------------------
def _ramp(c):
    """(slow, fast, amplitude) of a table case."""
    if c["scaling"] == "index":
        return INDEX_SLOW, INDEX_FAST, 1.0 + 0.1 * math.log(c["factor"])
    return SLOW, FAST, 1.0


def _table_plain(state):
    """Angles in 64 bits: a far position times a frequency has none left of its fraction in 32."""
    c = state["case"]
    R, base, factor = c["rotary"], state["base"], c["factor"]
    slow, fast, amplitude = _ramp(c)
    t = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    f = base ** (-2.0 * t / R)
    if c["scaling"] == "plain":
        keep = torch.ones_like(f)
    elif c["scaling"] == "linear":
        keep = torch.zeros_like(f)
    elif c["scaling"] == "wavelength":
        keep = ((c["trained"] * f / (2.0 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
    else:
        at = [R * math.log(c["trained"] / (2.0 * math.pi * turns)) / (2.0 * math.log(base)) for turns in (fast, slow)]
        first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), R - 1)
        keep = 1.0 - ((t - first) / max(last - first, 0.001)).clamp(0.0, 1.0)
    f = f * (keep + (1.0 - keep) / factor)
    angle = torch.arange(c["positions"], dtype=torch.float64, device="cuda")[:, None] * f
    return [(torch.stack([angle.cos(), angle.sin()], dim=2) * amplitude).float()]


def _rows(q_lens, kv_lens):
    """(sequence, position) of every row of a call, as tensors."""
    ql, kv = torch.tensor(q_lens), torch.tensor(kv_lens)
    seq = torch.repeat_interleave(torch.arange(len(q_lens)), ql)
    start = torch.cumsum(ql, 0) - ql
    pos = (kv - ql)[seq] + torch.arange(int(ql.sum())) - start[seq]
    return seq.cuda(), pos.cuda()


def _heads_plain(state, pos):
    """(q, k) of the call's rows in 32 bits, [n, h, d] and [n, g, d]; the sums of squares in 64 bits, because a quantised key lies next to a
    border now and then."""
    c = state["case"]
    h, g, d, R = c["heads"], c["kv_heads"], c["head_dim"], c["rotary"]
    x = state["qkv"].float().view(-1, h + 2 * g, d)[:, :h + g]
    if c["norm"]:
        r = (1.0 / torch.sqrt(x.double().square().mean(dim=2, keepdim=True) + EPS)).float()
        w = torch.cat([state["norms"][0].float().expand(h, d), state["norms"][1].float().expand(g, d)])
        x = x * r * w
    cos, sin = state["rope"][pos][:, None, :, 0], state["rope"][pos][:, None, :, 1]
    a, b = (x[:, :, :R // 2], x[:, :, R // 2:R]) if c["layout"] == "halves" else (x[:, :, 0:R:2], x[:, :, 1:R:2])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat([a, b], dim=2) if c["layout"] == "halves" else torch.stack([a, b], dim=3).flatten(2)
    x = torch.cat([turned, x[:, :, R:]], dim=2)
    return x[:, :h], x[:, h:]


def _put(state, name, x, seq, pos):
    """x [n, g, d] in 32 bits goes into the cache."""
    c = state["case"]
    n, g, d = x.shape
    page, block, tok = state["pages"][seq, pos // c["page"]].long(), pos % c["page"] // BLOCK, pos % BLOCK
    x = x.reshape(n, g, d // GROUP, GROUP)
    top, low = x.amax(dim=3), x.amin(dim=3)
    s = (torch.where(top >= -low, top, low) / -8.0).bfloat16().float().clamp(-8160.0, 8160.0).half()
    state[name + "_scale"][page, :, block, tok // 4, :, tok % 4] = s
    s = torch.where(s == 0, torch.ones_like(s), s).float()
    u = (x / s[..., None]).round().clamp(-8, 7).add(8).to(torch.uint8)
    if name == "k":
        u = u.view(n, g, d // 32, 4, 2, 2, 2).permute(0, 1, 3, 2, 6, 4, 5)           # [n, g, 4, d / 32, byte / 2, byte % 2, half]
        state[name][page, :, block, :, tok] = (u[..., 0] + 16 * u[..., 1]).reshape(n, g, 4, d // 32, 4)
    else:
        u = u.view(n, g, d // 32, 2, 16).transpose(2, 4)                             # [n, g, 16, half, d / 32]
        state[name][page, :, block, tok // 4, :, :, tok % 4 // 2 + tok % 2 * 2] = u[:, :, :, 0] + 16 * u[:, :, :, 1]


def _values(state, name, pages):
    """What the cache holds in whole pages (any shape of page numbers), [*pages.shape, g, blocks, 16, d] in 32 bits."""
    x = state[name][pages]
    d = x.shape[-2] * 32
    lead, n = x.shape[:-4], x.dim() - 4
    x = torch.stack([x & 15, x >> 4], dim=-1).view(*lead, 4, 16, d // 32, 2, 2, 2)    # [.., byte / 2, byte % 2, half]
    order = (1, 2, 0, 4, 5, 3) if name == "k" else (0, 4, 3, 2, 5, 1)
    x = x.permute(*range(n), *(n + i for i in order)).reshape(*lead, BLOCK, d // GROUP, GROUP)
    s = state[name + "_scale"][pages].transpose(-1, -2).reshape(*lead, BLOCK, d // GROUP)
    return ((x.float() - 8.0) * s.float()[..., None]).flatten(-2)


def _append_plain(state):
    c = state["case"]
    h, g, d, page = c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    seq, pos = _rows(*_seqs(c))
    q, k = _heads_plain(state, pos)
    _put(state, "k", k, seq, pos)
    _put(state, "v", state["qkv"].float().view(-1, h + 2 * g, d)[:, h + g:], seq, pos)
    place = seq * state["pages"].shape[1] + pos // page
    which, item = torch.unique(place, return_inverse=True)
    pages = state["pages"].view(-1)[which].long()
    back = [_values(state, name, pages)[item, :, pos % page // BLOCK, pos % BLOCK].half() for name in "kv"]
    return [q.half(), back[0], back[1]]


def _attention_plain(state):
    c = state["case"]
    h, g, d = c["heads"], c["kv_heads"], c["head_dim"]
    q_lens, kv_lens = _seqs(c)
    B, qm, rep = len(q_lens), max(q_lens), h // g
    seq, pos = _rows(q_lens, kv_lens)
    first = torch.tensor(kv_lens, device="cuda") - torch.tensor(q_lens, device="cuda")
    place = pos - first[seq]
    pages = state["pages"].long()
    T = pages.shape[1] * c["page"]
    limit = first[:, None] + torch.arange(qm, device="cuda")                     # rows behind a sequence's last one are dropped
    q = torch.zeros((B, qm, g, rep, d), device="cuda")
    q[seq, place] = state["q"].float().view(-1, g, rep, d)
    q = q.permute(0, 2, 1, 3, 4).reshape(B * g, qm * rep, d)
    k = _values(state, "k", pages).transpose(1, 2).reshape(B * g, T, d)           # [B, g, pages, blocks, 16, d]
    s = torch.matmul(q, k.transpose(1, 2).contiguous()).view(B, g, qm, rep, T) / math.sqrt(d)
    del k
    s.masked_fill_((torch.arange(T, device="cuda") > limit[:, :, None])[:, None, :, None], -math.inf)
    s -= s.amax(dim=4, keepdim=True)
    s.exp_()
    s /= s.sum(dim=4, keepdim=True)
    v = _values(state, "v", pages).transpose(1, 2).reshape(B * g, T, d)
    out = torch.matmul(s.view(B * g, qm * rep, T), v).view(B, g, qm, rep, d).permute(0, 2, 1, 3, 4)
    return [out[seq, place].reshape(-1, h, d).half()]


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    if c["op"] == "table":
        return _table_plain(state)
    if c["op"] == "heads":
        return [x.half() for x in _heads_plain(state, _rows(*_seqs(c))[1])]
    return _append_plain(state) if c["op"] == "append" else _attention_plain(state)


# ---- the same in 64 bits, sequence by sequence ----------------------------------------------------------------------
def _exact_table(c, seed):
    R, base = c["rotary"], _base(c, seed)
    slow, fast, amplitude = _ramp(c)
    freq = []
    for t in range(R // 2):
        f = math.exp(-2 * t / R * math.log(base))
        if c["scaling"] == "linear":
            f /= c["factor"]
        elif c["scaling"] == "wavelength":
            w = min(max((c["trained"] * f / math.tau - slow) / (fast - slow), 0.0), 1.0)
            f = w * f + (1 - w) * f / c["factor"]
        elif c["scaling"] == "index":
            turns_at = lambda b: R / 2 * math.log(c["trained"] / (b * math.tau), base)
            lo, hi = max(math.floor(turns_at(fast)), 0), min(math.ceil(turns_at(slow)), R - 1)
            w = 1 - min(max((t - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f = w * f + (1 - w) * f / c["factor"]
        freq.append(f)
    angle = torch.outer(torch.arange(c["positions"], dtype=torch.float64, device="cuda"), torch.tensor(freq, dtype=torch.float64, device="cuda"))
    return [torch.view_as_real(torch.polar(torch.full_like(angle, amplitude), angle))]


def _exact_heads(c, seed):
    """(q, k, v) of the call's rows in 64 bits."""
    h, g, d, R = c["heads"], c["kv_heads"], c["head_dim"], c["rotary"]
    q_lens, kv_lens = _seqs(c)
    x = _rows_in(c, seed).double().view(-1, h + 2 * g, d)
    freq = ROPE_BASE ** (-torch.arange(R // 2, dtype=torch.float64, device="cuda") * 2 / R)
    parts = [x[:, :h], x[:, h:h + g]]
    at = torch.cat([torch.arange(L - ql, L, dtype=torch.float64, device="cuda") for ql, L in zip(q_lens, kv_lens)])
    turn = torch.polar(torch.ones((len(at), 1, R // 2), dtype=torch.float64, device="cuda"), at[:, None, None] * freq)
    out = []
    for i, y in enumerate(parts):
        if c["norm"]:
            y = y / (torch.linalg.vector_norm(y, dim=2, keepdim=True) ** 2 / d + EPS).sqrt() * _norms(c, seed)[i].double()
        if c["layout"] == "halves":
            z = torch.complex(y[..., :R // 2].contiguous(), y[..., R // 2:R].contiguous()) * turn
            z = torch.cat([z.real, z.imag], dim=2)
        else:
            z = torch.view_as_real(torch.view_as_complex(y[..., :R].reshape(*y.shape[:2], R // 2, 2).contiguous()) * turn).flatten(2)
        out.append(torch.cat([z, y[..., R:]], dim=2))
    return out[0], out[1], x[:, h + g:]


def _exact_append(c, seed):
    q, k, v = _exact_heads(c, seed)
    back = []
    for x in (k, v):
        y = x.reshape(*x.shape[:2], -1, GROUP)
        far = torch.gather(y, 3, (y.abs() + (y > 0) * 1e-12).argmax(dim=3, keepdim=True))
        m, e = torch.frexp(far / -8)
        s = torch.ldexp((m * 256).round() / 256, e)
        back.append(((y / s).round().clamp(-8, 7) * s).flatten(2))
    return [q, back[0], back[1]]


def _exact_attention(c, seed):
    h, g, d = c["heads"], c["kv_heads"], c["head_dim"]
    rep = h // g
    q_lens, kv_lens = _seqs(c)
    q = _normal(seed, 5, (sum(q_lens), h, d)).half().double()
    (kc, ks), (vc, vs) = _pool(c, seed, 3), _pool(c, seed, 4)
    table = _page_table(c, seed).long()
    held = lambda code, scale, pages, j: ((code[pages, j].double() - 8) * scale[pages, j].double().repeat_interleave(GROUP, dim=3)).reshape(-1, d)
    out, row = torch.empty_like(q), 0
    for b, (ql, L) in enumerate(zip(q_lens, kv_lens)):
        pages = table[b, :(L + c["page"] - 1) // c["page"]]
        hidden = torch.arange(L, device="cuda")[None] > torch.arange(L - ql, L, device="cuda")[:, None]
        for j in range(g):
            kj, vj = held(kc, ks, pages, j)[:L], held(vc, vs, pages, j)[:L]
            for r in range(j * rep, (j + 1) * rep):
                s = (q[row:row + ql, r] @ kj.t().contiguous() * d ** -0.5).masked_fill(hidden, -math.inf)
                out[row:row + ql, r] = torch.softmax(s, dim=1) @ vj
        row += ql
    return [out]


def exact(c, seed):
    if c["op"] == "table":
        return _exact_table(c, seed)
    if c["op"] == "heads":
        return list(_exact_heads(c, seed)[:2])
    return _exact_append(c, seed) if c["op"] == "append" else _exact_attention(c, seed)
