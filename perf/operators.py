"""The paged 4-bit key/value cache of the softmax layers: what is measured, and the same in plain tensor operations.

Two operators of ``arl2.Cache``: ``append`` (keys rotated on the way, both held in 4 bits) and ``attend`` (softmax attention of
new queries over what is held).  ``own`` says which side ``run`` computes: the library's, or elementary torch operations in 32 bits.

The format, for each token, key head and group of 64 channels: ``minimum`` and ``step`` in fp16, and a 4-bit code per channel that
stands for ``minimum + step * code``.  A page is [kv_heads] units of [K codes | V codes | K parameters | V parameters] for
``page_tokens`` tokens, the even channel of a pair of codes in the low half of its byte.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 64            # channels that share a minimum and a step
LIMIT = 61440.0       # magnitudes that are held: minimum + 15 steps stays inside fp16
FIFTEENTH = 1.0 / 15.0


def _append(name, streams, kv_heads, tokens, dtype="bf16", dim=128, page=64, start=0):
    return {"name": name, "op": "append", "streams": streams, "heads": kv_heads, "kv_heads": kv_heads, "dim": dim,
            "tokens": tokens, "start": start, "page": page, "dtype": dtype}


def _attend(name, streams, heads, kv_heads, queries, cached, dtype="bf16", dim=128, page=64, causal=False, ragged=False, rotate=True):
    return {"name": name, "op": "attend", "streams": streams, "heads": heads, "kv_heads": kv_heads, "dim": dim, "queries": queries,
            "cached": cached, "page": page, "dtype": dtype, "causal": causal, "ragged": ragged, "rotate": rotate}


def listed():
    return [
        # one new token in each of a few streams, the step of token-by-token generation: latency alone
        _append("append_token", 4, 12, 1, start=4680),
        # the clean latent of a one-frame block of the base model
        _append("append_frame", 1, 12, 1560, start=1560),
        # three-frame blocks of the wider model, four streams served together: bandwidth alone
        _append("append_wide", 4, 40, 4680, start=4680),
        # single precision, narrow heads, small pages, an odd length that begins inside a page
        _append("append_odd_fp32", 3, 2, 333, dtype="fp32", dim=64, page=16, start=77),
        # one query of one stream over a short cache: latency alone
        _attend("token_short", 1, 12, 12, 1, 500),
        # one query in each of a few streams over sixteen cached blocks: every byte of the cache once
        _attend("token_long", 4, 12, 12, 1, 74880),
        # one query per stream, five query heads to a key head, streams of different lengths
        _attend("token_groups", 8, 40, 8, 1, 9360, ragged=True),
        # a few new tokens at once, each seeing those before it, three query heads to a key head
        _attend("few_causal", 2, 12, 4, 7, 3001, causal=True),
        # a denoise pass of a one-frame block over six cached frames
        _attend("frame", 1, 12, 12, 1560, 9360),
        # prompts of several streams, each token seeing those before it, of different and odd lengths
        _attend("prompts_causal", 4, 12, 12, 701, 1399, causal=True, ragged=True, page=16),
        # a denoise pass of a three-frame block over four cached blocks
        _attend("block", 1, 12, 12, 4680, 18720, page=128),
        # single precision, narrow heads, a 16 x 16 latent frame over three of them
        _attend("frame_fp32", 1, 2, 2, 256, 768, dtype="fp32", dim=64, page=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _pairs(case):
    """Visible (query, key) pairs of one head, over the streams."""
    total, n = 0, case["queries"]
    for have in _lengths(case):
        if not case["causal"]:
            total += n * have
        else:   # query i of n sees have - n + i + 1 keys
            first = max(0, n - have)
            total += (n - first) * (have - n) + (n * (n + 1) - first * (first + 1)) // 2
    return total


def draw(rng):
    top = listed()
    most = {k: max(work(c)[k] for c in top) for k in ("bytes", "flops")}
    most_bytes = {op: max(work(c)["bytes"] for c in top if c["op"] == op) for op in ("append", "attend")}
    while True:
        streams, page = rng.choice((1, 1, 2, 3, 4, 8)), rng.choice((16, 32, 64, 128))
        dtype = rng.choice(("bf16", "bf16", "bf16", "fp32"))
        dim = rng.choice((128, 128, 128, 64))
        heads, kv_heads = rng.choice(((12, 12), (12, 12), (40, 40), (2, 2), (12, 4), (40, 8), (12, 2), (5, 1)))
        if rng.random() < 0.35:
            c = _append("", streams, kv_heads, _log_int(rng, 1, 4680), dtype, dim, page, start=rng.randint(0, 9360))
        else:
            # from one token to a few, or a block
            queries = rng.choice((1, _log_int(rng, 1, 64), _log_int(rng, 64, 4680)))
            c = _attend("", streams, heads, kv_heads, queries, _log_int(rng, 1, 74880), dtype, dim, page, causal=rng.random() < 0.3,
                        ragged=rng.random() < 0.4, rotate=rng.random() < 0.7)
        del c["name"]
        w = work(c)
        if w["bytes"] > most_bytes[c["op"]] or w["flops"] > most["flops"]:
            continue
        if c["op"] == "attend" and c["heads"] * c["streams"] * c["queries"] * c["cached"] > 1.1e9:   # the plain form's scores
            continue
        return c


# ------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[case["dtype"]]


def _lengths(case):
    """Tokens that each stream holds: all the same, or shorter from stream to stream."""
    have, streams = case["cached"], case["streams"]
    return [have - (b * have) // (2 * streams) if case["ragged"] else have for b in range(streams)]


def _unit_bytes(case):
    return case["page"] * (case["dim"] + case["dim"] // GROUP * 8)


def _tables(case, rows, device):
    """Rotary tables of one row per position."""
    half = case["dim"] // 2
    freq = 10000.0 ** (-torch.arange(half, device=device, dtype=torch.float32) / half)
    angle = torch.arange(rows, device=device, dtype=torch.float32)[:, None] * freq
    return angle.cos().contiguous(), angle.sin().contiguous()


def _pool(case, per_stream, gen, device):
    """Pages in which anything may stand, handed out in no order."""
    streams, width = case["streams"], -(-per_stream // case["page"])
    count = streams * width + 3
    pages = torch.randint(0, 256, (count, case["kv_heads"] * _unit_bytes(case)), generator=gen, device=device, dtype=torch.uint8)
    table = torch.randperm(count, generator=gen, device=device)[: streams * width].to(torch.int32).view(streams, width)
    return pages, table.contiguous()


def prepare(case, seed):
    device = "cuda"
    gen = torch.Generator(device=device).manual_seed(seed)
    streams, kv_heads, dim = case["streams"], case["kv_heads"], case["dim"]
    state = {"case": case}

    def values(tokens, heads):   # channels with an offset and a size of their own, as keys have them
        x = torch.randn(streams, tokens, heads, dim, generator=gen, device=device)
        size = 0.5 + torch.rand(heads, dim, generator=gen, device=device)
        return (x * size + 0.3 * torch.randn(heads, dim, generator=gen, device=device)).to(_dtype(case))

    if case["op"] == "append":
        n = case["start"] + case["tokens"]
        state["pages"], state["table"] = _pool(case, n, gen, device)
        state["k"], state["v"] = values(case["tokens"], kv_heads), values(case["tokens"], kv_heads)
        state["start"] = torch.full((streams,), case["start"], dtype=torch.int32, device=device)
        state["cos"], state["sin"] = _tables(case, n, device)
        queries = case["tokens"]
    else:
        n = max(case["cached"], case["queries"])
        state["pages"], state["table"] = _pool(case, case["cached"], gen, device)
        for first in range(0, case["cached"], 4096):   # (a part at a time: the plain form takes several times the room)
            tokens = min(4096, case["cached"] - first)
            at = torch.arange(first, first + tokens, device=device).expand(streams, tokens)
            _store(case, state, at, *(_hold(values(tokens, kv_heads).float()) for _ in range(2)))
        state["q"] = values(case["queries"], case["heads"])
        state["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device=device)
        state["cos"], state["sin"] = _tables(case, n, device) if case["rotate"] else (None, None)
        queries = case["queries"]
    if own:
        from paper_2605_16579_b200 import arl2

        layer = arl2.Layer(streams, case["heads"], queries, dim, case["dtype"], device="cuda:0")
        state["layer"] = layer
        state["cache"] = arl2.Cache(layer, state["pages"].shape[0], state["table"].shape[1], kv_heads=kv_heads, page_tokens=case["page"],
                                    rope_cos=state["cos"], rope_sin=state["sin"], pages=state["pages"], page_table=state["table"])
    return state


# -------------------------------------------------------------------------------- the plain form
def _rotate(x, cos, sin, at):
    """Adjacent channels of x [B, T, H, D] turned by the angles of positions at [B, T]."""
    c, s = cos[at][:, :, None, :], sin[at][:, :, None, :]
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack((x0 * c - x1 * s, x0 * s + x1 * c), dim=-1).flatten(-2)


def _hold(x):
    """fp32 rows [B, T, H, D] -> codes, parameters, and the values that these stand for."""
    g = x.clamp(-LIMIT, LIMIT).unflatten(-1, (-1, GROUP))
    low = g.amin(-1, keepdim=True)
    step = ((g.amax(-1, keepdim=True) - low) * FIFTEENTH).half().float()
    low = low.half().float()
    inverse = torch.where(step > 0, torch.reciprocal(step), torch.zeros_like(step))
    code = ((g - low) * inverse).round().clamp(0, 15)
    held = low + step * code
    params = torch.cat((low, step), -1).half()     # [B, T, H, groups, 2]
    return code.to(torch.uint8).flatten(-2), params, held.flatten(-2)


def _views(case, pages):
    """Codes [page, head, token, D / 2] and parameters [page, head, token, groups, 2] of keys and values, in the pages."""
    p, d = case["page"], case["dim"]
    unit = pages.view(pages.shape[0], case["kv_heads"], -1)
    codes, params = p * d // 2, p * d // GROUP * 4
    at = [0, codes, 2 * codes, 2 * codes + params, 2 * codes + 2 * params]
    k, v, kp, vp = (unit[:, :, a:b] for a, b in zip(at, at[1:]))
    half = lambda t: t.unflatten(-1, (p, d // GROUP, 4)).view(torch.float16)  # noqa: E731
    return k.unflatten(-1, (p, d // 2)), v.unflatten(-1, (p, d // 2)), half(kp), half(vp)


def _store(case, state, at, keys, values):
    """Writes what _hold made of the tokens at positions at [B, T] into the pages."""
    page = torch.gather(state["table"].long(), 1, at // case["page"])[:, :, None]
    slot = (at % case["page"])[:, :, None]
    head = torch.arange(case["kv_heads"], device=at.device)[None, None, :]
    kc, vc, kp, vp = _views(case, state["pages"])
    for (code, params, _), c, p in ((keys, kc, kp), (values, vc, vp)):
        c[page, head, slot] = code[..., 0::2] | (code[..., 1::2] << 4)
        p[page, head, slot] = params


def _values(codes, params, table, rows):
    """What the first `rows` places of each stream hold, fp32 [B, H, rows, D]."""
    b, width = table.shape
    page = table.long()
    byte = codes[page].transpose(1, 2).flatten(2, 3)[:, :, :rows]            # [B, H, rows, D / 2]
    par = params[page].transpose(1, 2).flatten(2, 3)[:, :, :rows].float()    # [B, H, rows, groups, 2]
    code = torch.stack((byte & 15, byte >> 4), -1).flatten(-2).float().unflatten(-1, (-1, GROUP))
    return (par[..., 0:1] + par[..., 1:2] * code).flatten(-2)


def _plain_append(case, s):
    at = s["start"].long()[:, None] + torch.arange(case["tokens"], device=s["start"].device)
    keys, values = _hold(_rotate(s["k"].float(), s["cos"], s["sin"], at)), _hold(s["v"].float())
    _store(case, s, at, keys, values)
    return keys[2].to(_dtype(case)), values[2].to(_dtype(case))


def _plain_attend(case, s):
    n, have, rep = case["queries"], case["cached"], case["heads"] // case["kv_heads"]
    lengths = s["lengths"].long()
    place = torch.arange(have, device=lengths.device)
    at = lengths[:, None] - n + torch.arange(n, device=lengths.device)        # positions of the queries [B, n]
    seen = (place < lengths[:, None])[:, None, :].expand(-1, n, -1)
    if case["causal"]:
        seen = seen & (place <= at[:, :, None])
    q = s["q"].float()
    if case["rotate"]:
        q = _rotate(q, s["cos"], s["sin"], at.clamp(min=0))
    # [B, kv head, group, n, D]
    q = q.transpose(1, 2).unflatten(1, (case["kv_heads"], rep)) / math.sqrt(case["dim"])
    kc, vc, kp, vp = _views(case, s["pages"])
    inside = (place < lengths[:, None])[:, None, :, None]
    k = torch.where(inside, _values(kc, kp, s["table"], have), 0.0)
    v = torch.where(inside, _values(vc, vp, s["table"], have), 0.0)
    scores = q.flatten(2, 3) @ k.transpose(-1, -2)                            # [B, kv head, group * n, have]
    scores = scores.unflatten(2, (rep, n)).masked_fill_(~seen[:, None, None], -math.inf)
    weight = (scores - scores.amax(-1, keepdim=True).clamp_(min=-3e38)).exp_()
    total = weight.sum(-1, keepdim=True)
    out = weight.flatten(2, 3) @ v
    out = out.unflatten(2, (rep, n)) / torch.where(total > 0, total, 1.0)
    return out.flatten(1, 2).transpose(1, 2).to(_dtype(case)).contiguous()


def run(state):
    case = state["case"]
    if own and case["op"] == "append":
        return state["cache"].append(state["k"], state["v"], state["start"], held=True)
    if own:
        return state["cache"].attend(state["q"], state["lengths"], causal=case["causal"])
    return (_plain_append if case["op"] == "append" else _plain_attend)(case, state)


# ------------------------------------------------------------------------------ what it cannot do without
def work(case):
    size, dim = (4 if case["dtype"] == "fp32" else 2), case["dim"]
    held = dim + dim // GROUP * 8                       # bytes of a token and key head: codes and parameters of both
    if case["op"] == "append":
        rows = case["streams"] * case["tokens"] * case["kv_heads"]
        # both inputs, what is held, its values, the rotary tables; rotating, rounding and packing a value: about ten operations
        return {"bytes": rows * (2 * dim * size + held + 2 * dim * size) + case["tokens"] * dim * 4, "flops": rows * 2 * dim * 10}
    q = case["streams"] * case["queries"] * case["heads"] * dim * size
    return {"bytes": sum(_lengths(case)) * case["kv_heads"] * held + 2 * q, "flops": 4 * dim * case["heads"] * _pairs(case)}


# ------------------------------------------------------------------------------------- in 64 bits
def _turned64(x, cos, sin, at):
    """Row x [T, H, D] as complex numbers, times the unit numbers of positions at [T]."""
    z = torch.view_as_complex(x.double().unflatten(-1, (-1, 2)).contiguous())
    return torch.view_as_real(z * torch.complex(cos[at].double(), sin[at].double())[:, None, :]).flatten(-2)


def _held64(x):
    parts = []
    for part in x.split(GROUP, dim=-1):
        part = part.clamp(-LIMIT, LIMIT)
        low, high = part.min(-1, keepdim=True).values, part.max(-1, keepdim=True).values
        step, base = ((high - low) / 15).half().double(), low.half().double()
        nearest = torch.round((part - base) / torch.where(step > 0, step, 1.0)).clamp(0, 15)
        parts.append(base + step * nearest)
    return torch.cat(parts, -1)


def _stream64(case, state, b, have, which):
    """Keys (which = 0) or values (1) of stream b, read page by page: [H, have, D]."""
    p, d, h = case["page"], case["dim"], case["kv_heads"]
    pages = state["pages"][state["table"][b, : -(-have // p)].long()].view(-1, h, _unit_bytes(case))
    half = p * d // 2
    byte = pages[:, :, which * half:(which + 1) * half].reshape(-1, h, p, d // 2).int()
    words = p * (d // GROUP) * 4
    par = pages[:, :, p * d + which * words:p * d + (which + 1) * words].contiguous().view(torch.float16).reshape(-1, h, p, d // GROUP, 2).double()
    out = torch.empty(byte.shape[0], h, p, d, dtype=torch.float64, device=byte.device)
    for g in range(d // GROUP):
        cols = byte[..., g * GROUP // 2:(g + 1) * GROUP // 2]
        out[..., g * GROUP:(g + 1) * GROUP:2] = par[..., g, 0:1] + par[..., g, 1:2] * (cols % 16)
        out[..., g * GROUP + 1:(g + 1) * GROUP:2] = par[..., g, 0:1] + par[..., g, 1:2] * torch.div(cols, 16, rounding_mode="floor")
    return out.transpose(0, 1).reshape(h, -1, d)[:, :have]


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "append":
        at = torch.arange(case["start"], case["start"] + case["tokens"], device="cuda")
        keys = torch.stack([_held64(_turned64(k, s["cos"], s["sin"], at)) for k in s["k"]])
        return keys, torch.stack([_held64(v.double()) for v in s["v"]])
    n, rep = case["queries"], case["heads"] // case["kv_heads"]
    out = torch.zeros(case["streams"], n, case["heads"], case["dim"], dtype=torch.float64, device="cuda")
    for b, have in enumerate(_lengths(case)):
        keys, values = (_stream64(case, s, b, have, w) for w in (0, 1))
        at = torch.arange(have - n, have, device="cuda")
        q = s["q"][b].double()
        if case["rotate"]:
            q = _turned64(q, s["cos"], s["sin"], at.clamp(min=0))
        hidden = torch.arange(have, device="cuda") > at[:, None] if case["causal"] else None
        for h in range(case["heads"]):
            e = torch.einsum("id,jd->ij", q[:, h], keys[h // rep]) * case["dim"] ** -0.5
            if hidden is not None:
                e.masked_fill_(hidden, -math.inf)
            out[b, :, h] = torch.softmax(e, -1).nan_to_num_(0.0) @ values[h // rep]
    return out
