"""Definitions in 64 bits of what stands around the core in a block, and how far a result may be off.

A rounding to type t is off by at most u(t) = eps / 2 relative to the value.  What is computed before it is fp32 sums over a row: a tree
of shuffles, at most 8 + 5 + 5 additions deep per sum, and about ten operations per element, so 64 fp32 roundings of the largest
magnitude that enters are more than an element can have.  A sum over n tokens is off by at most (n + 64) roundings of the sum of
its terms' magnitudes, whatever the order.
"""
import torch

U32 = 2.0 ** -24


def u(dtype):
    return torch.finfo(dtype).eps / 2


def near(got, want, slack, what=""):
    """|got - want| <= u(type) |want| (1 + tiny) + slack, slack a number or a tensor; got is not NaN where want is not."""
    got64 = got.double()
    bound = u(got.dtype) * want.abs() * 1.001 + slack + 1e-300
    off = (got64 - want).abs() / bound
    assert not torch.isnan(off).any(), what
    worst = float(off.detach().max())
    assert worst <= 1.0, f"{what}: {worst:.3g} times the tolerance"


def norm64(x, kind, eps=1e-6):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)


def per_token(rows, frame, tokens):
    return rows.repeat_interleave(frame, 1)[:, :tokens]


def modulate64(x, y, gate, scale, shift, weight, post_weight, frame, norm, post, hold=lambda r: r):
    """r and n in the inputs' 64 bits; hold: what the stream makes of r before the norm reads it."""
    tokens = x.shape[1]
    r = x
    if y is not None:
        add = y
        if post is not None:
            add = norm64(add, post)
            add = add if post_weight is None else add * post_weight
        r = r + (add if gate is None else add * per_token(gate, frame, tokens))
    n = norm64(hold(r), norm)
    if weight is not None:
        n = n * weight
    if scale is not None:
        n = n * (1 + per_token(scale, frame, tokens))
    if shift is not None:
        n = n + per_token(shift, frame, tokens)
    return r, n


def angles64(cos, sin, axes, at):
    """Unit numbers [B, T, 1, D / 2] of positions at [B, T, 3]; positions outside count as the first or last row."""
    at = at.long().clamp(0, cos.shape[0] - 1)
    z = torch.complex(cos.double(), sin.double())
    out, first = [], 0
    for axis, pairs in enumerate(axes):
        out.append(z[at[..., axis], first:first + pairs])
        first += pairs
    out.append(torch.ones(*at.shape[:2], cos.shape[1] - first, dtype=z.dtype, device=z.device))
    return torch.cat(out, -1)[:, :, None]


def rotate64(x, unit, norm, weight, eps=1e-6):
    if norm == "token":
        x = norm64(x.flatten(2), "rms", eps).view(x.shape)
        x = x if weight is None else x * weight.view(x.shape[2:])
    elif norm == "head":
        x = norm64(x, "rms", eps)
        x = x if weight is None else x * weight
    elif norm == "l2":
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) + eps)
    z = torch.view_as_complex(x.unflatten(-1, (-1, 2)).contiguous()) * unit
    return torch.view_as_real(z).flatten(-2)


def grid_positions(start, tokens, rows, columns):
    l = torch.arange(tokens, device=start.device)
    frame = start[:, None].long() + l // (rows * columns)
    return torch.stack((frame, (l // columns % rows).expand_as(frame), (l % columns).expand_as(frame)), -1)


def tables(rows, dim, device="cuda"):
    half = dim // 2
    angle = torch.arange(rows, device=device, dtype=torch.float64)[:, None] * 1000.0 ** (-torch.arange(half, device=device, dtype=torch.float64) / half)
    return angle.cos().float().contiguous(), angle.sin().float().contiguous()


def leaves(*tensors):
    return [None if t is None else t.double().detach().clone().requires_grad_(True) for t in tensors]
