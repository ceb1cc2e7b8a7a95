"""Training the remembering branch of a block over a whole video at once, against a teacher that attends to all earlier blocks.

    python examples/train_memory.py [--blocks 4] [--tokens 240] [--heads 4] [--steps 20] [--fp32]

One block of the model: the norm before it, modulated per frame; projections; queries and keys as rows of length one, turned by frame,
row and column; the recurrence over the blocks of the video; a gate per token and head; the projection back, added to the residual stream
with the frame's gate.  Modulation, rotation and recurrence are the library's kernels in both directions (autograd functions around their
forward and backward calls), the matrix products between them are torch's.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2605_16579_b200 import arl2  # noqa: E402


class Modulate(torch.autograd.Function):
    """(x, y, gate, scale, shift) -> (r, n); y and gate may be None."""

    @staticmethod
    def forward(ctx, op, x, y, gate, scale, shift):
        r, n = op.forward(x, y, gate=gate, scale=scale, shift=shift)
        ctx.op = op
        ctx.save_for_backward(r, y, gate, scale, shift)
        return (r if y is not None else r.view_as(r)), n

    @staticmethod
    def backward(ctx, dr, dn):
        r, y, gate, scale, shift = ctx.saved_tensors
        dx, dy, dgate, dscale, dshift, _, _ = ctx.op.backward(r, dn.contiguous(), dr.contiguous(), y, gate=gate, scale=scale, shift=shift)
        return None, dx, dy, dgate, dscale, dshift


class Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, op, q, k):
        ctx.op = op
        ctx.save_for_backward(q, k)
        return op.forward(q, k)

    @staticmethod
    def backward(ctx, dq, dk):
        q, k = ctx.saved_tensors
        dq, dk, _, _ = ctx.op.backward(dq.contiguous(), dk.contiguous(), q, k)
        return None, dq, dk


class Remember(torch.autograd.Function):
    @staticmethod
    def forward(ctx, op, q, k, v, decay):
        ctx.op = op
        ctx.save_for_backward(q, k, v, decay)
        return op.forward(q, k, v, decay, final=False)[0]

    @staticmethod
    def backward(ctx, dout):
        q, k, v, decay = ctx.saved_tensors
        return (None,) + ctx.op.backward(dout.contiguous(), q, k, v, decay, initial=False)[:4]


class Block(torch.nn.Module):
    def __init__(self, heads, dim, blocks, frames, rows, columns, dtype, device):
        super().__init__()
        self.heads, self.dim, self.block = heads, dim, frames * rows * columns
        d, tokens = heads * dim, blocks * self.block
        layer = arl2.Layer(1, heads, min(tokens, 4680), dim, dtype, device=device)
        half = dim // 2
        axes = (half - 2 * (half // 3), half // 3, half // 3)
        freq = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) for n in axes])
        angle = torch.arange(max(blocks * frames, rows, columns), dtype=torch.float64)[:, None] * freq
        cos, sin = (t.float().contiguous().to(device) for t in (angle.cos(), angle.sin()))
        self.before = arl2.Modulation(layer, rows * columns)
        self.after = arl2.Modulation(layer, rows * columns)
        self.turn = arl2.Rotation(layer, cos, sin, axes, grid=(rows, columns), norm="l2")
        self.memory = arl2.Recurrence(layer, self.block)
        self.layer, n_frames = layer, blocks * frames
        small = lambda *shape: torch.nn.Parameter(torch.randn(*shape, device=device) / d ** 0.5)  # noqa: E731
        self.w_qkv, self.w_gate, self.w_out = small(d, 3 * d), small(d, heads), small(d, d)
        self.modulation = torch.nn.Parameter(0.1 * torch.randn(1, n_frames, 3, d, device=device))
        self.decay = torch.nn.Parameter(torch.full((1, blocks, heads), 2.0, device=device))

    def forward(self, x):
        shift, scale, gate = self.modulation.unbind(2)
        _, n = Modulate.apply(self.before, x, None, None, scale, shift)
        w = [p.to(n.dtype) for p in (self.w_qkv, self.w_gate, self.w_out)]
        q, k, v = (n @ w[0]).unflatten(-1, (3, self.heads, self.dim)).unbind(2)     # parts of one row: no copies
        q, k = Rotate.apply(self.turn, q, k)
        o = Remember.apply(self.memory, q, k, v, self.decay) * torch.sigmoid(n @ w[1])[..., None]
        y = o.flatten(2) @ w[2]
        r, _ = Modulate.apply(self.after, x, y, gate, None, None)
        return r


def teacher(x, heads, dim, block):
    """Softmax attention of each block over the blocks before it, of x itself."""
    b, t, _ = x.shape
    q = x.float().view(b, t, heads, dim).transpose(1, 2)
    s = q @ q.transpose(2, 3) / dim ** 0.5
    at = torch.arange(t, device=x.device) // block
    s = s.masked_fill(at[:, None] <= at[None, :], -3e38)
    out = torch.where((at > 0)[:, None], s.softmax(-1) @ q, torch.zeros_like(q))
    return x.float() + out.transpose(1, 2).flatten(2)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=240, help="of a latent frame: a multiple of 8")
    ap.add_argument("--heads", type=int, default=4)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--fp32", action="store_true")
    a = ap.parse_args(argv)
    torch.manual_seed(1)
    dev, dtype = torch.device("cuda:0"), torch.float32 if a.fp32 else torch.bfloat16
    model = Block(a.heads, a.dim, a.blocks, 1, 8, a.tokens // 8, "fp32" if a.fp32 else "bf16", dev)
    x = torch.randn(1, a.blocks * a.tokens, a.heads * a.dim, device=dev).to(dtype)
    target = teacher(x, a.heads, a.dim, model.block)
    optimizer = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses = []
    for step in range(a.steps):
        optimizer.zero_grad(set_to_none=True)
        loss = (model(x).float() - target).square().mean()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    model.layer.sync_status()
    losses = [float(v) for v in losses]
    print(f"{a.blocks} blocks of {model.block} tokens, {a.heads} heads: loss {losses[0]:.4f} at first, {losses[-1]:.4f} after {a.steps} steps")
    return model, x, target, losses


if __name__ == "__main__":
    main()
