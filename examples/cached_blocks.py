"""A softmax layer of the stack over a growing cache held in 4 bits: blocks of a video are denoised one after the other.

    python examples/cached_blocks.py [--blocks 6] [--tokens 1560] [--heads 12] [--steps 4]

At every denoising step the block's keys and values are written to their places in the cache (over those of the step before), rotated
to their positions on the way, and the block's queries read all tokens so far; the clean pass writes them for good.  Then a few
tokens are generated one by one over the same cache.  Beside it runs the same layer over a contiguous bf16 cache
(``Layer.teacher_step``): the outputs' distance is what 4 bits cost, and both caches' sizes are printed, with the scratch that the 4-bit
cache's calls need: one for all caches whose calls follow one another, here those of the blocks and of the single tokens.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2605_16579_b200 import arl2, workload  # noqa: E402


def rotated(x, cos, sin, first):
    """What the 4-bit cache does on the way, for the bf16 one."""
    c, s = (t[first:first + x.shape[1], None, :] for t in (cos, sin))
    a, b = x.float()[..., 0::2], x.float()[..., 1::2]
    return torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2).to(torch.bfloat16)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--blocks", type=int, default=6)
    ap.add_argument("--tokens", type=int, default=1560)
    ap.add_argument("--heads", type=int, default=12)
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--page", type=int, default=64)
    a = ap.parse_args(argv)
    dev, L, H, D = torch.device("cuda:0"), a.tokens, a.heads, 128
    d, most = H * D, a.blocks * a.tokens + 8
    gen = torch.Generator(device=dev).manual_seed(1)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device=dev)  # noqa: E731

    layer = arl2.Layer(1, H, L, D, "bf16", device=dev)
    layer.set_projections(*(((randn(d, d) / d ** 0.5).to(torch.bfloat16)) for _ in range(3)), (randn(d, H) / d ** 0.5).to(torch.bfloat16),
                          (randn(d, d) / d ** 0.5).to(torch.bfloat16))
    cos, sin = (t.to(dev) for t in workload.rope_tables(most, D))
    # pages of the pool in no order, as a pool that other streams share hands them out
    width = -(-most // a.page)
    cache = arl2.Cache(layer, width + 5, width, page_tokens=a.page, rope_cos=cos, rope_sin=sin)
    cache.page_table.copy_(torch.randperm(width + 5, generator=gen, device=dev)[:width].to(torch.int32).view(1, width))
    wide_k, wide_v = (torch.zeros(1, most, H, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
    start, lengths = (torch.zeros(1, dtype=torch.int32, device=dev) for _ in range(2))

    worst = 0.0
    for block in range(a.blocks):
        first = block * L
        start.fill_(first)
        lengths.fill_(first + L)
        clean = randn(1, L, d)
        for step in range(a.steps + 1):              # the last one is the clean pass
            noise = 1.0 - step / a.steps
            x = (clean + noise * randn(1, L, d)).to(torch.bfloat16)
            q, k, v, _ = layer.project_in(x)
            cache.append(k, v, start)
            y = layer.project_out(cache.attend(q, lengths))
            wide_k[:, first:first + L], wide_v[:, first:first + L] = rotated(k, cos, sin, first), v
            other = layer.project_out(layer.teacher_step(rotated(q, cos, sin, first), wide_k[:, :first + L].contiguous(), wide_v[:, :first + L].contiguous()))
            far = float((y.float() - other.float()).norm() / other.float().norm())
            worst = max(worst, far)
        print(f"block {block}: {first + L} tokens cached, output of the clean pass {far:.3f} from bf16's")

    # tokens one by one over the same cache
    single = arl2.Layer(1, H, 1, D, "bf16", device=dev)
    follow = arl2.Cache(single, cache.cfg.num_pages, width, page_tokens=a.page, rope_cos=cos, rope_sin=sin, pages=cache.pages, page_table=cache.page_table,
                        workspace=cache.workspace)
    for i in range(8):
        start.fill_(a.blocks * L + i)
        lengths.fill_(a.blocks * L + i + 1)
        q, k, v = (randn(1, 1, H, D).to(torch.bfloat16) for _ in range(3))
        follow.append(k, v, start)
        out = follow.attend(q, lengths)
    layer.sync_status()
    single.sync_status()
    held, wide = int(width * cache.page_bytes), width * a.page * H * D * 4       # (of the same number of tokens)
    scratch = cache.workspace.numel()
    print(f"cache: {held / 1e6:.1f} MB in 4 bits, {wide / 1e6:.1f} MB in bf16 ({wide / held:.2f} times), and {scratch / 1e6:.1f} MB of scratch for "
          f"all layers that run one after the other; outputs at most {worst:.3f} apart")
    return {"worst": worst, "held": held, "wide": wide, "scratch": scratch, "last": out}


if __name__ == "__main__":
    main()
