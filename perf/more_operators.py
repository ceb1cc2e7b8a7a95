"""What stands around the layer's core in a block of the model, and its memory over a whole video: what is measured, and the same in
plain tensor operations.

Three operators, each with its backward pass:

``Modulation``  the norm before a block and what comes after the one before it: r = x + gate * P(y), n = N(r) * w * (1 + scale) + shift,
                N and P a LayerNorm or an RMSNorm over the row (P may be absent), gate, scale and shift one row for the tokens of a frame.
``Rotation``    queries and keys on their way to the attention: a norm (over the token, over the head, or to length one), then the
                rotation of adjacent channels by positions along several axes, a range of the pairs for each.
``Recurrence``  the state over the blocks of a sequence: o_i = q_i S_n for the tokens i of block n, S_{n+1} = sigmoid(a_n) S_n + K_n^T V_n.

``own`` says which side ``run`` computes: the library's, or elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

AXES = {128: (22, 21, 21), 64: (12, 10, 10)}     # pairs that turn with the frame, the row and the column


def _modulate(name, streams, tokens, frame, heads, dim=128, dtype="bf16", wide=False, norm="layer", post="", back=False):
    return {"name": name, "op": "modulate", "back": back, "streams": streams, "tokens": tokens, "frame": frame, "heads": heads, "dim": dim,
            "dtype": dtype, "wide": wide, "norm": norm, "post": post}


def _rotate(name, streams, tokens, heads, kv_heads, dim=128, dtype="bf16", norm="token", rows=30, columns=52, first=0, given=False, back=False):
    return {"name": name, "op": "rotate", "back": back, "streams": streams, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "norm": norm, "rows": rows, "columns": columns, "first": first, "given": given}


def _recur(name, streams, tokens, block, heads, dim=128, dtype="bf16", begun=False, back=False):
    return {"name": name, "op": "recur", "back": back, "streams": streams, "tokens": tokens, "block": block, "heads": heads, "dim": dim,
            "dtype": dtype, "begun": begun}


def listed():
    return [
        # one new token in each of a few streams, a modulation of its own each: latency alone
        _modulate("modulate_token", 4, 1, 1, 12),
        # two three-frame blocks of the wider model, the residual stream in 32 bits: bandwidth alone
        _modulate("modulate_wide", 1, 9360, 1560, 40, wide=True),
        # a training step over two three-frame blocks of the base model, a modulation per frame
        _modulate("modulate_back", 1, 9360, 1560, 12, back=True),
        # single precision, norms before and after, narrow rows, frames of an odd length
        _modulate("modulate_back_odd_fp32", 3, 333, 77, 2, dim=64, dtype="fp32", norm="rms", post="rms", back=True),
        # queries and keys of one new token in each of a few streams, late in a video: latency alone
        _rotate("rotate_token", 4, 1, 12, 12, first=920),
        # a three-frame block of the wider model
        _rotate("rotate_wide", 1, 4680, 40, 40, first=27),
        # a training step over two blocks of the base model
        _rotate("rotate_back", 1, 9360, 12, 12, back=True),
        # single precision, a norm per head, fewer key heads, positions given one by one
        _rotate("rotate_back_odd_fp32", 3, 333, 5, 1, dim=64, dtype="fp32", norm="head", given=True, rows=9, columns=11, back=True),
        # the first blocks of a video of the wider model, gone through at once
        _recur("recur_wide", 1, 14040, 4680, 40),
        # small latent frames in single precision, one after the other
        _recur("recur_small_fp32", 2, 1000, 64, 2, dim=64, dtype="fp32", begun=True),
        # a training step over an 81-frame video of the base model (21 latent frames in blocks of three)
        _recur("recur_back", 1, 32760, 4680, 12, back=True),
        # short blocks of an odd length, the last one cut, narrow heads
        _recur("recur_back_odd", 2, 2003, 100, 5, dim=64, begun=True, back=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w, m = work(c), most.setdefault((c["op"], c["back"]), {"bytes": 0, "flops": 0})
        for k in m:
            m[k] = max(m[k], w[k])
    while True:
        streams = rng.choice((1, 1, 1, 2, 3, 4, 8))
        dtype = rng.choice(("bf16", "bf16", "bf16", "fp32"))
        dim = rng.choice((128, 128, 128, 64))
        heads, kv_heads = rng.choice(((12, 12), (12, 12), (40, 40), (2, 2), (16, 4), (40, 8), (8, 2), (5, 1)))
        back = rng.random() < 0.5
        op = rng.choice(("modulate", "rotate", "recur"))
        if op == "modulate":
            frame = rng.choice((1, _log_int(rng, 16, 1560), 1560))
            c = _modulate("", streams, _log_int(rng, 1, 14040), frame, heads, dim, dtype, dtype == "bf16" and rng.random() < 0.3,
                          rng.choice(("layer", "layer", "rms")), rng.choice(("", "", "layer", "rms")), back)
            if streams * c["tokens"] / frame > 4096:    # a modulation for each token is for single tokens
                continue
        elif op == "rotate":
            c = _rotate("", streams, _log_int(rng, 1, 14040), heads, kv_heads, dim, dtype, rng.choice(("token", "token", "head", "l2", "")),
                        rng.randint(4, 30), rng.randint(4, 52), rng.randint(0, 1000), rng.random() < 0.3, back)
        else:
            block = rng.choice((_log_int(rng, 16, 4680), 1560, 4680))
            tokens = max(1, min(40000, round(block * rng.uniform(0.5, 30))))
            c = _recur("", streams, tokens, block, heads, dim, dtype, rng.random() < 0.5, back)
        del c["name"]
        w, m = work(c), most[(c["op"], c["back"])]
        if w["bytes"] <= m["bytes"] and w["flops"] <= m["flops"]:
            return c


# ------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[case["dtype"]]


def _wide(case):
    return torch.float32 if case["wide"] else _dtype(case)


def _frames(case):
    return -(-case["tokens"] // case["frame"])


def _rows(case):
    """Rows of the rotary tables: one more than the last position along any axis."""
    return max(case["first"] + case["streams"] + -(-case["tokens"] // (case["rows"] * case["columns"])), case["rows"], case["columns"])


def _tables(case, device):
    """cos and sin of position * frequency of the pair within its axis, in 64 bits first: far positions."""
    columns = []
    for pairs in AXES[case["dim"]]:
        columns.append(10000.0 ** (-torch.arange(pairs, device=device, dtype=torch.float64) / pairs))
    angle = torch.arange(_rows(case), device=device, dtype=torch.float64)[:, None] * torch.cat(columns)
    return angle.cos().float().contiguous(), angle.sin().float().contiguous()


def prepare(case, seed):
    device = "cuda"
    gen = torch.Generator(device=device).manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device=device)  # noqa: E731
    streams, tokens, heads, dim = case["streams"], case["tokens"], case["heads"], case["dim"]
    width, kind = heads * dim, _dtype(case)
    s = {"case": case}
    if case["op"] == "modulate":
        # the residual stream has channels with an offset of their own; gates and scales are small; one buffer of three rows per frame
        x = randn(streams, tokens, width) * (0.5 + torch.rand(width, generator=gen, device=device)) + 0.3 * randn(width)
        y = randn(streams, tokens, width)
        mod = 0.3 * randn(streams, _frames(case), 3, width)
        s["gate"], s["scale"], s["shift"] = mod.unbind(2)
        s["weight"] = 1 + 0.1 * randn(width) if case["norm"] == "rms" else None
        s["post_weight"] = 1 + 0.1 * randn(width) if case["post"] else None
        s["y"] = y.to(kind)
        if case["back"]:
            s["r"] = x.to(_wide(case))
            s["dn"], s["dr"] = randn(streams, tokens, width).to(kind), randn(streams, tokens, width).to(_wide(case))
        else:
            s["x"] = x.to(_wide(case))
    elif case["op"] == "rotate":
        # keys have channels with an offset of their own
        s["q"] = randn(streams, tokens, heads, dim).to(kind)
        s["k"] = (randn(streams, tokens, case["kv_heads"], dim) + 0.3 * randn(case["kv_heads"], dim)).to(kind)
        s["cos"], s["sin"] = _tables(case, device)
        for x, n in (("q", heads), ("k", case["kv_heads"])):
            shape = {"token": (n * dim,), "head": (dim,)}.get(case["norm"])
            s[x + "_weight"] = None if shape is None else 1 + 0.2 * randn(*shape)
        s["start"] = (case["first"] + torch.arange(streams, device=device)).to(torch.int32)
        s["positions"] = _positions(case, s["start"]) if case["given"] else None
        if case["back"]:
            s["dq"], s["dk"] = randn(streams, tokens, heads, dim).to(kind), randn(streams, tokens, case["kv_heads"], dim).to(kind)
    else:
        # rows of queries and keys of length one, as the layer's features are; gates that forget a little per block
        unit = lambda x: (x / x.norm(dim=-1, keepdim=True)).to(kind)  # noqa: E731
        s["q"], s["k"] = unit(randn(streams, tokens, heads, dim)), unit(randn(streams, tokens, heads, dim))
        s["v"] = randn(streams, tokens, heads, dim).to(kind)
        blocks = -(-tokens // case["block"])
        s["decay"] = 2 + randn(streams, blocks, heads)
        s["state"] = randn(streams, heads, dim, dim) * math.sqrt(case["block"] / dim) if case["begun"] else None
        if case["back"]:
            s["do"] = randn(streams, tokens, heads, dim).to(kind)
            s["dstate"] = randn(streams, heads, dim, dim) if case["begun"] else None
    if own:
        from paper_2605_16579_b200 import arl2

        layer = arl2.Layer(streams, heads, min(tokens, 4680), dim, case["dtype"], device="cuda:0")
        if case["op"] == "modulate":
            s["own"] = arl2.Modulation(layer, case["frame"], norm=case["norm"], post=case["post"] or None,
                                       residual=torch.float32 if case["wide"] else None)
        elif case["op"] == "rotate":
            s["own"] = arl2.Rotation(layer, s["cos"], s["sin"], AXES[dim], grid=(case["rows"], case["columns"]), norm=case["norm"] or None,
                                     kv_heads=case["kv_heads"])
        else:
            s["own"] = arl2.Recurrence(layer, case["block"])
    return s


def _positions(case, start):
    """Frame, row and column of every token, [B, T, 3]."""
    l, area = torch.arange(case["tokens"], device=start.device), case["rows"] * case["columns"]
    frame = start[:, None].long() + l // area
    row, column = (l % area) // case["columns"], l % case["columns"]
    return torch.stack((frame, row.expand_as(frame), column.expand_as(frame)), -1).to(torch.int32)


# -------------------------------------------------------------------------------- the plain form
EPS = 1e-6


def _per_token(case, rows):
    """A row per frame [B, F, d] -> a row per token."""
    return rows.repeat_interleave(case["frame"], 1)[:, : case["tokens"]]


def _per_frame(case, x):
    """Sums of the tokens' rows over the frames, [B, F, d]."""
    frames = _frames(case)
    pad = frames * case["frame"] - case["tokens"]
    if pad:
        x = torch.cat((x, x.new_zeros(x.shape[0], pad, x.shape[2])), 1)
    return x.view(x.shape[0], frames, case["frame"], -1).sum(2)


def _normed(x, kind):
    """The rows of x normalised, and one over their deviation."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    inverse = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * inverse, inverse


def _norm_back(g, hat, inverse, kind):
    out = g - hat * (g * hat).mean(-1, keepdim=True)
    if kind == "layer":
        out = out - g.mean(-1, keepdim=True)
    return out * inverse


def _plain_modulate(case, s):
    y = s["y"].float()
    if case["post"]:
        y = _normed(y, case["post"])[0] * s["post_weight"]
    r = s["x"].float() + _per_token(case, s["gate"]) * y
    r = r.to(_wide(case))      # (what the norm reads is what the stream holds)
    hat = _normed(r.float(), case["norm"])[0]
    if s["weight"] is not None:
        hat = hat * s["weight"]
    n = hat * (1 + _per_token(case, s["scale"])) + _per_token(case, s["shift"])
    return r, n.to(_dtype(case))


def _plain_modulate_back(case, s):
    dn, y, gate, one = s["dn"].float(), s["y"].float(), _per_token(case, s["gate"]), 1 + _per_token(case, s["scale"])
    hat, inverse = _normed(s["r"].float(), case["norm"])
    w = 1.0 if s["weight"] is None else s["weight"]
    dshift, dscale = _per_frame(case, dn), _per_frame(case, dn * hat * w)
    dweight = None if s["weight"] is None else (dn * hat * one).sum((0, 1))
    dr = s["dr"].float() + _norm_back(dn * one * w, hat, inverse, case["norm"])
    dpost = None
    if case["post"]:
        hat, inverse = _normed(y, case["post"])
        y = hat * s["post_weight"]
        g = dr * gate
        dpost = (g * hat).sum((0, 1))
        dy = _norm_back(g * s["post_weight"], hat, inverse, case["post"])
    else:
        dy = dr * gate
    out = [dr.to(_wide(case)), dy.to(_dtype(case)), _per_frame(case, dr * y), dscale, dshift]
    return out + [t for t in (dweight, dpost) if t is not None]


def _angles(case, s):
    """cos and sin for every token, [B, T, 1, D / 2]."""
    at = (_positions(case, s["start"]) if s["positions"] is None else s["positions"]).long()
    axis = torch.repeat_interleave(torch.arange(3, device=at.device), torch.tensor(AXES[case["dim"]], device=at.device))
    rows = at[..., axis]
    return (torch.gather(t.expand(at.shape[0], -1, -1), 1, rows)[:, :, None] for t in (s["cos"], s["sin"]))


def _turn(x, c, sn):
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * c - b * sn, a * sn + b * c), -1).flatten(-2)


def _inverse_length(case, x):
    if case["norm"] == "l2":
        return torch.rsqrt((x * x).sum(-1, keepdim=True) + EPS)
    over = (-1,) if case["norm"] == "head" else (-2, -1)
    return torch.rsqrt((x * x).mean(over, keepdim=True) + EPS)


def _as_heads(weight, x):
    return 1.0 if weight is None else weight if weight.numel() == x.shape[-1] else weight.view(x.shape[2:])


def _plain_rotate(case, s):
    c, sn = _angles(case, s)
    out = []
    for name in ("q", "k"):
        x = s[name].float()
        if case["norm"]:
            x = x * _inverse_length(case, x) * _as_heads(s[name + "_weight"], x)
        out.append(_turn(x, c, sn).to(_dtype(case)))
    return out


def _plain_rotate_back(case, s):
    c, sn = _angles(case, s)
    out, weights = [], []
    for name in ("q", "k"):
        g = _turn(s["d" + name].float(), c, -sn)
        if case["norm"]:
            x, w = s[name].float(), s[name + "_weight"]
            inverse = _inverse_length(case, x)
            hat = x * inverse
            if w is not None:
                weights.append((g * hat).sum((0, 1) if case["norm"] == "token" else (0, 1, 2)).view(w.shape))
                g = g * _as_heads(w, x)
            over = (-2, -1) if case["norm"] == "token" else (-1,)
            mean = (g * hat).sum(over, keepdim=True) if case["norm"] == "l2" else (g * hat).mean(over, keepdim=True)
            g = (g - hat * mean) * inverse
        out.append(g.to(_dtype(case)))
    return out + weights


def _blocks(case, x):
    """[B, T, H, D] -> the blocks, [B, H, tokens, D] each, in 32 bits."""
    return [p.float().transpose(1, 2) for p in x.split(case["block"], 1)]


def _plain_recur(case, s):
    alpha = torch.sigmoid(s["decay"])
    state = torch.zeros_like(s["decay"][:, 0, :, None, None]).expand(-1, -1, case["dim"], case["dim"]) if s["state"] is None else s["state"]
    out = []
    for n, (q, k, v) in enumerate(zip(*(_blocks(case, s[x]) for x in "qkv"))):
        out.append((q @ state).transpose(1, 2).to(_dtype(case)))
        state = alpha[:, n, :, None, None] * state + k.transpose(2, 3) @ v
    return torch.cat(out, 1), state


def _plain_recur_back(case, s):
    alpha = torch.sigmoid(s["decay"])
    q, k, v, do = (_blocks(case, s[x]) for x in ("q", "k", "v", "do"))
    shape = (case["streams"], case["heads"], case["dim"], case["dim"])
    states = [alpha.new_zeros(shape) if s["state"] is None else s["state"]]
    for n in range(len(q) - 1):
        states.append(alpha[:, n, :, None, None] * states[n] + k[n].transpose(2, 3) @ v[n])
    d = alpha.new_zeros(shape) if s["dstate"] is None else s["dstate"]
    dq, dk, dv, da = [], [], [], []
    for n in range(len(q) - 1, -1, -1):
        dq.append(do[n] @ states[n].transpose(2, 3))
        dk.append(v[n] @ d.transpose(2, 3))
        dv.append(k[n] @ d)
        da.append((d * states[n]).sum((2, 3)))
        d = alpha[:, n, :, None, None] * d + q[n].transpose(2, 3) @ do[n]
    whole = lambda parts: torch.cat([p.transpose(1, 2) for p in parts[::-1]], 1).to(_dtype(case))  # noqa: E731
    return whole(dq), whole(dk), whole(dv), torch.stack(da[::-1], 1) * alpha * (1 - alpha), d


_PLAIN = {("modulate", False): _plain_modulate, ("modulate", True): _plain_modulate_back, ("rotate", False): _plain_rotate,
          ("rotate", True): _plain_rotate_back, ("recur", False): _plain_recur, ("recur", True): _plain_recur_back}


def run(state):
    case, s = state["case"], state
    if not own:
        return _PLAIN[case["op"], case["back"]](case, s)
    op = s["own"]
    if case["op"] == "modulate":
        if not case["back"]:
            return op.forward(s["x"], s["y"], gate=s["gate"], scale=s["scale"], shift=s["shift"], weight=s["weight"], post_weight=s["post_weight"])
        out = op.backward(s["r"], s["dn"], s["dr"], s["y"], gate=s["gate"], scale=s["scale"], shift=s["shift"], weight=s["weight"],
                          post_weight=s["post_weight"])
    elif case["op"] == "rotate":
        where = {"positions": s["positions"]} if case["given"] else {"start": s["start"]}
        if not case["back"]:
            return op.forward(s["q"], s["k"], q_weight=s["q_weight"], k_weight=s["k_weight"], **where)
        out = op.backward(s["dq"], s["dk"], s["q"], s["k"], q_weight=s["q_weight"], k_weight=s["k_weight"], **where)
    elif not case["back"]:
        return op.forward(s["q"], s["k"], s["v"], s["decay"], state=s["state"])
    else:
        return op.backward(s["do"], s["q"], s["k"], s["v"], s["decay"], state=s["state"], dstate=s["dstate"])
    return [t for t in out if t is not None]


# ------------------------------------------------------------------------------ what it cannot do without
def work(case):
    size, rows, dim = (4 if case["dtype"] == "fp32" else 2), case["streams"] * case["tokens"], case["dim"]
    if case["op"] == "modulate":
        width, wide = case["heads"] * dim, 4 if case["wide"] else size
        frames = 3 * 4 * case["streams"] * _frames(case) * width
        if not case["back"]:
            # x and y in, r and n out
            return {"bytes": rows * width * (2 * wide + 2 * size) + frames, "flops": rows * width * (14 if case["post"] else 9)}
        # r, y and both gradients in, two out; gate and scale in, three gradients of rows per frame out
        return {"bytes": rows * width * (3 * wide + 3 * size) + frames * 5 // 3, "flops": rows * width * (34 if case["post"] else 22)}
    if case["op"] == "rotate":
        channels = rows * (case["heads"] + case["kv_heads"]) * dim
        moved = 2 if not case["back"] or not case["norm"] else 3
        return {"bytes": channels * size * moved, "flops": channels * (3 + (4 if case["norm"] else 0)) * (2 if case["back"] else 1)}
    states = case["streams"] * case["heads"] * dim * dim * 4
    if not case["back"]:
        return {"bytes": rows * case["heads"] * dim * size * 4 + states * (2 if case["begun"] else 1), "flops": rows * case["heads"] * 4 * dim * dim}
    return {"bytes": rows * case["heads"] * dim * size * 7 + states * (3 if case["begun"] else 1), "flops": rows * case["heads"] * 10 * dim * dim}


# ------------------------------------------------------------------------------------- in 64 bits
def _norm64(x, kind):
    if kind == "layer":
        return torch.nn.functional.layer_norm(x, x.shape[-1:], eps=EPS)
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)


def _modulate64(case, x, y, gate, scale, shift, weight, post_weight):
    """Residual and normed rows, frame by frame."""
    r, n = [], []
    for f in range(_frames(case)):
        a, b = f * case["frame"], min(case["tokens"], (f + 1) * case["frame"])
        add = y[:, a:b]
        if case["post"]:
            add = _norm64(add, case["post"]) * post_weight
        here = x[:, a:b] + add * gate[:, f:f + 1]
        r.append(here)
        here = here if case["back"] else here.to(_wide(case)).double()
        here = _norm64(here, case["norm"])
        if weight is not None:
            here = here * weight
        n.append(here * (1 + scale[:, f:f + 1]) + shift[:, f:f + 1])
    return torch.cat(r, 1), torch.cat(n, 1)


def _rotate64(case, s, x, weight):
    if case["norm"] == "token":
        x = (_norm64(x.flatten(2), "rms") * weight).view(x.shape)
    elif case["norm"] == "head":
        x = _norm64(x, "rms") * weight
    elif case["norm"] == "l2":
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) + EPS)
    at, first = _positions(case, s["start"]).long(), 0
    unit = torch.complex(s["cos"].double(), s["sin"].double())
    z, parts = torch.view_as_complex(x.unflatten(-1, (-1, 2)).contiguous()), []
    for axis, pairs in enumerate(AXES[case["dim"]]):
        parts.append(z[..., first:first + pairs] * unit[at[..., axis], first:first + pairs][:, :, None])
        first += pairs
    return torch.view_as_real(torch.cat(parts, -1)).flatten(-2)


def _recur64(case, q, k, v, decay, state):
    out = []
    for n in range(-(-case["tokens"] // case["block"])):
        part = slice(n * case["block"], (n + 1) * case["block"])
        out.append(torch.einsum("bthi,bhij->bthj", q[:, part], state))
        state = torch.einsum("bthi,bthj->bhij", k[:, part], v[:, part]) + state / (1 + torch.exp(-decay[:, n]))[:, :, None, None]
    return torch.cat(out, 1), state


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    leaf = lambda name: None if s.get(name) is None else s[name].double().detach().clone().requires_grad_(case["back"])  # noqa: E731
    if case["op"] == "modulate":
        names = ("y", "gate", "scale", "shift", "weight", "post_weight")
        v = {n: leaf(n) for n in names}
        if not case["back"]:
            return _modulate64(case, s["x"].double(), *(v[n] for n in names))
        # the backward pass is given r: the x it came from is r less what was added
        with torch.no_grad():
            x = s["r"].double() - (_modulate64(case, torch.zeros_like(s["r"], dtype=torch.float64), *(v[n] for n in names))[0])
        x.requires_grad_(True)
        r, n = _modulate64(case, x, *(v[n] for n in names))
        wanted = [x] + [v[n] for n in names if v[n] is not None]
        return torch.autograd.grad((r, n), wanted, (s["dr"].double(), s["dn"].double()))
    if case["op"] == "rotate":
        v = {n: leaf(n) for n in ("q", "k", "q_weight", "k_weight")}
        out = [_rotate64(case, s, v[n], v[n + "_weight"]) for n in ("q", "k")]
        if not case["back"]:
            return out
        return torch.autograd.grad(out, [t for t in v.values() if t is not None], [s["dq"].double(), s["dk"].double()])
    v = {n: leaf(n) for n in ("q", "k", "v", "decay")}
    shape = (case["streams"], case["heads"], case["dim"], case["dim"])
    state = torch.zeros(shape, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()
    state.requires_grad_(case["back"])
    out, last = _recur64(case, *v.values(), state)
    if not case["back"]:
        return out, last
    dlast = torch.zeros_like(last) if s["dstate"] is None else s["dstate"].double()
    return torch.autograd.grad((out, last), list(v.values()) + [state], (s["do"].double(), dlast))
