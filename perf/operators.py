"""Operators of a serving step around the paged 8-bit KV cache and the logits, as they are measured: the calls, their plain form in
elementary torch operations, the work they cannot do without and their result in 64 bits.

  append      k and v of a ragged call go into the paged cache, q and k rotated on the way (relax_paged_append); what the cache then
              stands for from the first block that the call touched to the end of each sequence is read back (relax_paged_read)
  attention   causal attention of a ragged call over the paged cache (relax_paged_attention)
  logprobs    log probability of one given token per row of logits, the entropy of the row and its most likely alternatives
              (relax_token_logprobs)

The cache.  Positions of a sequence are cut into pages of `page` tokens, a page into blocks of 16.  Per block and KV head keys and
values have one scale each, s = max|x| / 127, and codes u in 1..255 that stand for (u - 128) * s.  A block that a later call appends to
keeps its scale unless the new tokens need a larger one: then the codes that are there become round(c * s_old / s_new).
  k codes  [pages][kv_heads][page / 16][d / 16][16 tokens][16]            element e of a token: chunk e / 16, place e % 16
  v codes  [pages][kv_heads][page / 16][d / 64][4][16][4][4]              element e of token t: [e / 64][t / 4][e % 16][e / 16 % 4][t % 4]
  scales   [pages][kv_heads][page / 16]
The keys of a case:

  op          "append" | "attention" | "logprobs"
  heads, kv_heads, head_dim, page
  prompt, past                              rows of one sequence (0: no such sequence) on top of `past` cached tokens
  decodes, each, len_first, len_step        further sequences with `each` rows, lengths len_first + b * len_step
  rows, vocab, top                          of a "logprobs" case
"""
from __future__ import annotations

import math

import torch

own = False

ROPE_BASE = 10000.0
BLOCK = 16

TINY = dict(heads=4, kv_heads=4, head_dim=64)
B7 = dict(heads=32, kv_heads=32, head_dim=128)
B70 = dict(heads=64, kv_heads=8, head_dim=128)
GROUPED = dict(heads=32, kv_heads=8, head_dim=128)


def _call(op, shape, page=16, prompt=0, past=0, decodes=0, each=1, len_first=0, len_step=0):
    return dict(op=op, page=page, prompt=prompt, past=past, decodes=decodes, each=each, len_first=len_first, len_step=len_step, **shape)


def _logprobs(rows, vocab, top):
    return dict(op="logprobs", rows=rows, vocab=vocab, top=top)


def listed():
    return [
        # one token of one user goes into the middle of a block: nothing but latency
        dict(name="append_1", **_call("append", B7, decodes=1, len_first=2231)),
        # a batch of sixty-four decoding users with grouped heads
        dict(name="append_64", **_call("append", B70, decodes=64, len_first=128, len_step=61)),
        # a prompt of odd length behind a cached beginning that ends inside a block
        dict(name="append_prompt_2043", **_call("append", B7, page=64, prompt=2043, past=5)),
        # the smallest model: one token on a short context
        dict(name="attention_tiny", **_call("attention", TINY, decodes=1, len_first=53)),
        # interactive chat: one token of one user, middle of a 4096-token context, one query head per KV head
        dict(name="attention_1", **_call("attention", B7, decodes=1, len_first=2231)),
        # sixteen users between 100 and 8000 tokens with grouped heads
        dict(name="attention_16", **_call("attention", B70, page=32, decodes=16, len_first=100, len_step=526)),
        # one user with a very long document
        dict(name="attention_long", **_call("attention", B70, page=64, decodes=1, len_first=120001)),
        # drafted tokens are checked: five rows of eight users at once
        dict(name="attention_drafts", **_call("attention", GROUPED, decodes=8, each=5, len_first=700, len_step=391)),
        # a chunk of one prompt beside the decode rows of other users
        dict(name="attention_mixed", **_call("attention", B7, prompt=300, past=1201, decodes=20, len_first=90, len_step=57)),
        # a long prompt with grouped heads
        dict(name="attention_4096", **_call("attention", GROUPED, page=64, prompt=4096)),
        # the token just picked, with five alternatives, for one user
        dict(name="logprobs_1", **_logprobs(1, 32000, 5)),
        # every token of a prompt is scored
        dict(name="logprobs_2047", **_logprobs(2047, 32000, 20)),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _ragged(rng, count, each, longest):
    first = max(each, _log(rng, 1, max(2, longest // 2)))
    return dict(decodes=count, each=each, len_first=first, len_step=rng.randint(0, max(0, (longest - first) // max(1, count))))


def draw(rng):
    """One more case of the ranges above."""
    op = rng.choice(["append", "append", "attention", "attention", "attention", "attention", "logprobs", "logprobs"])
    if op == "logprobs":
        vocab = _log(rng, 100, 152064)
        return _logprobs(_log(rng, 1, max(1, min(2047, 65504000 // vocab))), vocab, min(vocab, _log(rng, 1, 32)))
    shape, page = rng.choice([TINY, B7, B70, GROUPED, dict(heads=40, kv_heads=40, head_dim=128), dict(heads=16, kv_heads=2, head_dim=64)]), rng.choice([16, 32, 64, 128])
    wide = shape["kv_heads"] >= 32
    kind = rng.choice(["one", "batch", "batch", "drafts", "mixed", "prompt"])
    if kind == "one":
        return _call(op, shape, page, **_ragged(rng, 1, 1, 20000 if wide else 120000))
    if kind == "batch":
        return _call(op, shape, page, **_ragged(rng, _log(rng, 2, 64), 1, 1000 if wide else rng.choice([600, 2000, 4000])))
    if kind == "drafts":
        return _call(op, shape, page, **_ragged(rng, _log(rng, 1, 16), rng.randint(2, 17), 2000))
    if kind == "mixed":
        return _call(op, shape, page, prompt=_log(rng, 2, 300), past=rng.randint(0, 1200), **_ragged(rng, _log(rng, 1, 20), 1, 1100))
    return _call(op, shape, page, prompt=_log(rng, 2, 2047), past=rng.choice([0, rng.randint(1, 600)]))


# ---- shapes of a call -----------------------------------------------------------------------------------------------
def _seqs(c):
    """(q_lens, kv_lens) of the call: the prompt first, then the other sequences."""
    q, kv = [], []
    if c["prompt"]:
        q, kv = [c["prompt"]], [c["past"] + c["prompt"]]
    return q + [c["each"]] * c["decodes"], kv + [c["len_first"] + b * c["len_step"] for b in range(c["decodes"])]


def _touched(c):
    """q_lens of the read-back: from the first block that the call appends to."""
    return [ql + (L - ql) % BLOCK for ql, L in zip(*_seqs(c))]


def _pages_per_slot(c):
    return max((L + c["page"] - 1) // c["page"] for L in _seqs(c)[1])


def work(c):
    if c["op"] == "logprobs":
        n, V, k = c["rows"], c["vocab"], c["top"]
        return {"bytes": n * V * 2 + n * 4 + n * 8 + n * k * 8, "flops": 6 * n * V}
    q, kv = _seqs(c)
    n, h, g, d = sum(q), c["heads"], c["kv_heads"], c["head_dim"]
    if c["op"] == "append":                     # rows in, q out, codes out; codes of the touched blocks in again, values out
        back = sum(_touched(c))
        return {"bytes": n * (2 * h + 2 * g) * d * 2 + 2 * n * g * d + 2 * back * g * d * 3, "flops": 6 * n * (h + g) * d + 8 * n * g * d}
    pairs = sum(ql * (L - ql) + ql * (ql + 1) // 2 for ql, L in zip(q, kv))
    return {"bytes": sum(kv) * 2 * g * (d + 4 / BLOCK) + 2 * n * h * d * 2, "flops": 4 * pairs * h * d}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _gen(seed, tensor):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + tensor)
    return g


def _normal(seed, tensor, shape, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=_gen(seed, tensor))


def _pool(c, seed, tensor):
    """(codes [pages, kv_heads, blocks, tokens, d] uint8, scales [pages, kv_heads, blocks]) of N(0, 1) values, some of them in blocks
    that no sequence has reached yet."""
    pages, g, d, blocks = _pool_pages(c), c["kv_heads"], c["head_dim"], c["page"] // BLOCK
    x = _normal(seed, tensor, (pages, g, blocks, BLOCK * d))
    s = x.abs().amax(dim=3) / 127.0
    x /= s[..., None]
    return x.round_().clamp_(-127, 127).add_(128).to(torch.uint8).view(pages, g, blocks, BLOCK, d), s


def _pool_pages(c):
    return len(_seqs(c)[0]) * _pages_per_slot(c) + 3


def _rope_table(positions, d):
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * ROPE_BASE ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    return torch.stack([angle.cos(), angle.sin()], dim=2).float()


def _page_table(c, seed):
    slots, per = len(_seqs(c)[0]), _pages_per_slot(c)
    order = torch.randperm(_pool_pages(c), device="cuda", generator=_gen(seed, 9))
    return order[:slots * per].view(slots, per).to(torch.int32)


def _logits(c, seed):
    return _normal(seed, 1, (c["rows"], c["vocab"]), 2.5).half()


def _targets(c, seed):
    return torch.randint(0, c["vocab"], (c["rows"],), dtype=torch.int32, device="cuda", generator=_gen(seed, 2))


def prepare(c, seed):
    if c["op"] == "logprobs":
        return {"case": c, "logits": _logits(c, seed), "targets": _targets(c, seed)}
    g, d = c["kv_heads"], c["head_dim"]
    state = {"case": c, "pages": _page_table(c, seed)}
    for name, tensor in (("k", 3), ("v", 4)):
        codes, state[name + "_scale"] = _pool(c, seed, tensor)
        lead = codes.shape[:3]
        if name == "k":
            state["k"] = codes.view(*lead, BLOCK, d // 16, 16).transpose(3, 4).contiguous()
        else:
            state["v"] = codes.view(*lead, 4, 4, d // 64, 4, 16).permute(0, 1, 2, 5, 3, 7, 6, 4).contiguous()
    n = sum(_seqs(c)[0])
    if c["op"] == "append":
        state["qkv"] = _normal(seed, 5, (n, (c["heads"] + 2 * g) * d)).half()
        state["rope"] = _rope_table(_pages_per_slot(c) * c["page"], d)
    else:
        state["q"] = _normal(seed, 5, (n, c["heads"], d)).half()
    return state


# ---- the framework's calls ------------------------------------------------------------------------------------------
def _own_setup(state):
    """What a program makes once: the descriptor of the cache, the model's sizes and a workspace."""
    from paper_2311_02103_amd import binding as rx

    c = state["case"]
    q, kv = _seqs(c)
    state["dims"] = rx.make_dims(c["heads"] * c["head_dim"], c["heads"], c["kv_heads"], c["head_dim"], 4 * c["heads"] * c["head_dim"],
                                 _pages_per_slot(c) * c["page"], len(q))
    state["cache"] = rx.PagedCache(state["k"], state["v"], state["k_scale"], state["v_scale"], state["pages"], state.get("rope"),
                                   state["k"].shape[0], c["page"], state["pages"].shape[1])
    rows = sum(_touched(c)) if c["op"] == "append" else sum(q)
    state["ws_bytes"] = rx.relax_paged_workspace_bytes(state["dims"], rows, max(kv), len(q))
    state["ws"] = torch.empty(state["ws_bytes"], dtype=torch.uint8, device="cuda")
    state["lens"] = (q, kv, _touched(c))
    return rx


def _run_own(state):
    from paper_2311_02103_amd import binding as rx

    c = state["case"]
    if c["op"] == "logprobs":
        n, V, k = c["rows"], c["vocab"], c["top"]
        if "ws" not in state:
            state["ws_bytes"] = rx.relax_token_logprobs_workspace_bytes(n, V, k)
            state["ws"] = torch.empty(state["ws_bytes"], dtype=torch.uint8, device="cuda")
        out = torch.empty((2, n), dtype=torch.float32, device="cuda")
        ids = torch.empty((n, k), dtype=torch.int32, device="cuda")
        top = torch.empty((n, k), dtype=torch.float32, device="cuda")
        rx.check(rx.relax_token_logprobs(state["logits"], V, state["targets"], out[0], out[1], ids, top, n, V, k, state["ws"], state["ws_bytes"]),
                 "relax_token_logprobs")
        return [out[0], out[1], ids, top]
    if "ws" not in state:
        _own_setup(state)
    q_lens, kv_lens, touched = state["lens"]
    h, g, d = c["heads"], c["kv_heads"], c["head_dim"]
    dims, cache, ws = state["dims"], state["cache"], (state["ws"], state["ws_bytes"])
    seqs = rx.Seqs(q_lens, kv_lens)
    if c["op"] == "attention":
        out = torch.empty_like(state["q"])
        rx.check(rx.relax_paged_attention(state["q"], cache, seqs, dims, out, out.shape[0], *ws), "relax_paged_attention")
        return [out]
    qkv = state["qkv"]
    n, row, base = qkv.shape[0], qkv.shape[1], qkv.data_ptr()
    q_out = torch.empty((n, h, d), dtype=torch.float16, device="cuda")
    rx.check(rx.relax_paged_append(base, row, base + 2 * h * d, base + 2 * (h + g) * d, row, q_out, cache, seqs, dims, n, *ws), "relax_paged_append")
    back = torch.empty((2, sum(touched), g, d), dtype=torch.float16, device="cuda")
    rx.check(rx.relax_paged_read(cache, rx.Seqs(touched, kv_lens), dims, back[0], back[1], back.shape[1], *ws), "relax_paged_read")
    return [q_out, back[0], back[1]]


# ---- the plain form -------------------------------------------------------------------------------------------------
def _rows(q_lens, kv_lens):
    """(sequence, position) of every row of a call, as tensors."""
    ql, kv = torch.tensor(q_lens), torch.tensor(kv_lens)
    seq = torch.repeat_interleave(torch.arange(len(q_lens)), ql)
    start = torch.cumsum(ql, 0) - ql
    pos = (kv - ql)[seq] + torch.arange(int(ql.sum())) - start[seq]
    return seq.cuda(), pos.cuda()


def _place(state, seq, pos):
    """(page, block of the page) of positions."""
    page = state["case"]["page"]
    return state["pages"][seq, pos // page].long(), pos % page // BLOCK


def _rotate(x, table):
    """Half-split rotary embedding of x [n, heads, d] in 32 bits; table [n, d / 2, 2]."""
    half = x.shape[2] // 2
    cos, sin = table[:, None, :, 0], table[:, None, :, 1]
    a, b = x[:, :, :half], x[:, :, half:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=2)


def _to_layout(name, x):
    """[.., g, d] of single tokens -> as indexing of the codes by (page, block, token) returns it."""
    n, g, d = x.shape
    return x.view(n, g, d // 16, 16) if name == "k" else x.view(n, g, d // 64, 4, 16).transpose(3, 4)


def _tokens(state, name, page, block, tok):
    codes = state[name]
    if name == "k":
        return codes[page, :, block, :, tok].flatten(2)
    return codes[page, :, block, :, tok // 4, :, :, tok % 4].transpose(3, 4).flatten(2)


def _put(state, name, x, seq, pos):
    """x [n, g, d] in 32 bits goes into the cache."""
    codes, scale = state[name], state[name + "_scale"]
    page, block = _place(state, seq, pos)
    key = page * scale.shape[2] + block
    items, item = torch.unique(key, return_inverse=True)
    ipage, iblock = items // scale.shape[2], items % scale.shape[2]
    g = x.shape[1]
    first = torch.full((items.numel(),), BLOCK, device=x.device).scatter_reduce(0, item, pos % BLOCK, "amin")
    need = torch.zeros((items.numel(), g), device=x.device).scatter_reduce(0, item[:, None].expand(-1, g), x.abs().amax(dim=2), "amax") / 127.0
    old = torch.where((first > 0)[:, None], scale[ipage, :, iblock], torch.zeros_like(need))
    new = torch.maximum(old, need)
    safe = torch.where(new > 0, new, torch.ones_like(new))
    there = codes[ipage, :, iblock]
    ratio = (old / safe).view(items.numel(), g, *([1] * (there.dim() - 2)))
    codes[ipage, :, iblock] = ((there.float() - 128.0) * ratio).round().add(128.0).to(torch.uint8)
    scale[ipage, :, iblock] = new
    c = (x / safe[item][:, :, None]).round().clamp(-127, 127).add(128.0).to(torch.uint8)
    tok = pos % BLOCK
    if name == "k":
        codes[page, :, block, :, tok] = _to_layout(name, c)
    else:
        codes[page, :, block, :, tok // 4, :, :, tok % 4] = _to_layout(name, c)


def _values(state, name, seq, pos):
    """What the cache holds at positions, [n, g, d] in 32 bits."""
    page, block = _place(state, seq, pos)
    return (_tokens(state, name, page, block, pos % BLOCK).float() - 128.0) * state[name + "_scale"][page, :, block][:, :, None]


def _append_plain(state):
    c = state["case"]
    h, g, d = c["heads"], c["kv_heads"], c["head_dim"]
    q_lens, kv_lens = _seqs(c)
    seq, pos = _rows(q_lens, kv_lens)
    x = state["qkv"].float().view(-1, h + 2 * g, d)
    table = state["rope"][pos]
    rotated = _rotate(x[:, :h + g], table)
    _put(state, "k", rotated[:, h:], seq, pos)
    _put(state, "v", x[:, h + g:], seq, pos)
    seq, pos = _rows(_touched(c), kv_lens)
    return [rotated[:, :h].half(), _values(state, "k", seq, pos).half(), _values(state, "v", seq, pos).half()]


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
    k = state["k"][pages].transpose(5, 4)                                       # [B, pages, g, blocks, 16 tokens, d / 16, 16]
    k = ((k.flatten(5).float() - 128.0) * state["k_scale"][pages][..., None, None]).transpose(1, 2).reshape(B * g, T, d)
    q = torch.zeros((B, qm, g, rep, d), device="cuda")
    q[seq, place] = state["q"].float().view(-1, g, rep, d)
    q = q.permute(0, 2, 1, 3, 4).reshape(B * g, qm * rep, d)
    s = torch.matmul(q, k.transpose(1, 2).contiguous()).view(B, g, qm, rep, T) / math.sqrt(d)
    del k
    limit = first[:, None] + torch.arange(qm, device="cuda")                     # rows behind a sequence's last one are dropped
    s.masked_fill_((torch.arange(T, device="cuda") > limit[:, :, None])[:, None, :, None], -math.inf)
    s -= s.amax(dim=4, keepdim=True)
    s.exp_()
    s /= s.sum(dim=4, keepdim=True)
    v = state["v"][pages].permute(0, 2, 1, 3, 5, 8, 4, 7, 6)                     # [B, g, pages, blocks, 4, 4, d / 64, 4, 16]
    v = (v.reshape(B, g, pages.shape[1], -1, BLOCK, d).float() - 128.0) * state["v_scale"][pages].transpose(1, 2)[..., None, None]
    out = torch.matmul(s.view(B * g, qm * rep, T), v.view(B * g, T, d)).view(B, g, qm, rep, d).permute(0, 2, 1, 3, 4)
    return [out[seq, place].reshape(-1, h, d).half()]


def _logprobs_plain(state):
    c = state["case"]
    x = state["logits"].float()
    s, ids = torch.sort(x, dim=1, descending=True, stable=True)                  # ties: the lowest index first
    z = x - s[:, :1]
    e = torch.exp(z)
    total = e.sum(dim=1)
    log_total = torch.log(total)
    logp = torch.gather(z, 1, state["targets"].long()[:, None])[:, 0] - log_total
    entropy = log_total - (e * z).sum(dim=1) / total
    return [logp, entropy, ids[:, :c["top"]].to(torch.int32), s[:, :c["top"]] - s[:, :1] - log_total[:, None]]


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    return _append_plain(state) if op == "append" else _attention_plain(state) if op == "attention" else _logprobs_plain(state)


# ---- the same in 64 bits, sequence by sequence ----------------------------------------------------------------------
def _exact_pool(c, seed, tensor):
    """The pool as values [pages, page, g, d], and its scales [pages, g, blocks]."""
    codes, s = _pool(c, seed, tensor)
    v = (codes.to(torch.int16) - 128).double() * s.double()[..., None, None]
    return v.permute(0, 2, 3, 1, 4).reshape(v.shape[0], c["page"], c["kv_heads"], c["head_dim"]), s.double()


def _exact_append(c, seed):
    h, g, d = c["heads"], c["kv_heads"], c["head_dim"]
    q_lens, kv_lens = _seqs(c)
    x = _normal(seed, 5, (sum(q_lens), (h + 2 * g) * d)).half().double().view(-1, h + 2 * g, d)
    table = _page_table(c, seed).long()
    freq = ROPE_BASE ** (-torch.arange(d // 2, dtype=torch.float64, device="cuda") * 2 / d)
    pools = [_exact_pool(c, seed, 3), _exact_pool(c, seed, 4)]
    q_out, back, row = [], [[], []], 0
    for b, (ql, L) in enumerate(zip(q_lens, kv_lens)):
        ang = torch.arange(L - ql, L, dtype=torch.float64, device="cuda")[:, None, None] * freq
        turned = torch.complex(x[row:row + ql, :h + g, :d // 2], x[row:row + ql, :h + g, d // 2:]) * torch.complex(ang.cos(), ang.sin())
        turned = torch.cat([turned.real, turned.imag], dim=2)
        q_out.append(turned[:, :h])
        low = (L - ql) // BLOCK * BLOCK
        at = torch.arange(low, L, device="cuda")
        for j, new in enumerate((turned[:, h:], x[row:row + ql, h + g:])):
            values, scales = pools[j]
            page, place = table[b, at // c["page"]], at % c["page"]
            held = L - ql - low                                        # tokens of the first block that were there
            t = torch.cat([values[page[:held], place[:held]], new])    # [L - low, g, d]
            full = (t.shape[0] + BLOCK - 1) // BLOCK
            pad = torch.cat([t, t.new_zeros(full * BLOCK - t.shape[0], g, d)]).view(full, BLOCK, g, d)
            fresh = torch.cat([t.new_zeros(held, g, d), new, t.new_zeros(full * BLOCK - t.shape[0], g, d)]).view(full, BLOCK, g, d)
            s = fresh.abs().amax(dim=(1, 3)) / 127
            if held:
                s[0] = torch.maximum(s[0], scales[page[0], :, place[0] // BLOCK])
            s = s[:, None, :, None]
            back[j].append(((pad / s).round() * s).view(full * BLOCK, g, d)[:t.shape[0]])
        row += ql
    return [torch.cat(q_out), torch.cat(back[0]), torch.cat(back[1])]


def _exact_attention(c, seed):
    h, g, d = c["heads"], c["kv_heads"], c["head_dim"]
    rep = h // g
    q_lens, kv_lens = _seqs(c)
    q = _normal(seed, 5, (sum(q_lens), h, d)).half().double()
    (kc, ks), (vc, vs) = _pool(c, seed, 3), _pool(c, seed, 4)
    table = _page_table(c, seed).long()
    out, row = torch.empty_like(q), 0
    for b, (ql, L) in enumerate(zip(q_lens, kv_lens)):
        pages = table[b, :(L + c["page"] - 1) // c["page"]]
        hidden = torch.arange(L, device="cuda")[None] > torch.arange(L - ql, L, device="cuda")[:, None]
        for j in range(g):
            kj = ((kc[pages, j].double() - 128) * ks[pages, j].double()[..., None, None]).reshape(-1, d)[:L]
            vj = ((vc[pages, j].double() - 128) * vs[pages, j].double()[..., None, None]).reshape(-1, d)[:L]
            for r in range(j * rep, (j + 1) * rep):
                s = (q[row:row + ql, r] @ kj.t().contiguous() * d ** -0.5).masked_fill(hidden, -math.inf)
                out[row:row + ql, r] = torch.softmax(s, dim=1) @ vj
        row += ql
    return [out]


def exact(c, seed):
    if c["op"] == "append":
        return _exact_append(c, seed)
    if c["op"] == "attention":
        return _exact_attention(c, seed)
    logp = torch.log_softmax(_logits(c, seed).double(), dim=1)
    entropy = -(logp.exp() * logp).sum(dim=1)
    given = logp[torch.arange(c["rows"], device="cuda"), _targets(c, seed).long()]
    return [given, entropy, None, torch.topk(logp, c["top"], dim=1).values]
