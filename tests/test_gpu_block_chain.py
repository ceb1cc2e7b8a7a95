"""Modulation, rotation and recurrence together, as a block of the model uses them: with the layer's projections, and in training."""
import importlib.util
import os

import pytest
import torch

from block_util import angles64, grid_positions, modulate64, rotate64, tables

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_memory", os.path.join(ROOT, "examples", "train_memory.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("captured", [False, True])
def test_a_block_of_the_model(captured):
    """Norm, projections, rotation with lengths of one, recurrence, projection, residual and the next norm, bf16, against 64 bits.

    Each of the stages rounds its output to bf16 (2^-9 of it, rms), and a state or a sum of D terms averages what came before: a few
    roundings in all; 2e-2 of the largest value, which the layer's own parity tests allow, is five of the largest single ones."""
    from paper_2605_16579_b200 import arl2

    B, H, D, rows, columns, frames, blocks = 2, 3, 128, 7, 9, 2, 3
    L, d = frames * rows * columns, H * D
    T, F = L * blocks, frames * blocks
    g = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    layer = arl2.Layer(B, H, T, D, "bf16")
    weights = [(randn(d, d) / d ** 0.5).bfloat16() for _ in range(3)] + [(randn(d, H) / d ** 0.5).bfloat16(), (randn(d, d) / d ** 0.5).bfloat16()]
    layer.set_projections(*weights)
    cos, sin = tables(40, D)
    axes = (22, 21, 21)
    before, after = arl2.Modulation(layer, rows * columns), arl2.Modulation(layer, rows * columns, post="rms")
    turn, memory = arl2.Rotation(layer, cos, sin, axes, grid=(rows, columns), norm="l2"), arl2.Recurrence(layer, L)
    x, mod, decay = randn(B, T, d).bfloat16(), 0.3 * randn(B, F, 5, d), 2 + randn(B, blocks, H)
    start = torch.tensor([0, 11], device="cuda", dtype=torch.int32)
    shift, scale, gate, shift2, scale2 = mod.unbind(2)

    def run():
        _, n = before.forward(x, scale=scale, shift=shift)
        q, k, v, _ = layer.project_in(n)
        q, k = turn.forward(q, k, start=start)
        o, last = memory.forward(q, k, v, decay)
        return after.forward(x, layer.project_out(o), gate=gate, scale=scale2, shift=shift2) + (last,)

    r, n2, last = run()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = run()
        x.copy_(x.flip(1))
        graph.replay()
        r, n2, last = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, (r, n2, last)))
    layer.sync_status()

    w = [t.double() for t in weights]
    m = [t.double() for t in mod.unbind(2)]
    _, n = modulate64(x.double(), None, None, m[1], m[0], None, None, rows * columns, "layer", None)
    q, k, v = ((n @ w[i]).view(B, T, H, D) for i in range(3))
    unit = angles64(cos, sin, axes, grid_positions(start, T, rows, columns))
    q, k = rotate64(q, unit, "l2", None), rotate64(k, unit, "l2", None)
    state, out = torch.zeros(B, H, D, D, dtype=torch.float64, device="cuda"), []
    for i in range(blocks):
        part = slice(i * L, (i + 1) * L)
        out.append(torch.einsum("bthi,bhij->bthj", q[:, part], state))
        state = torch.sigmoid(decay[:, i].double())[:, :, None, None] * state + torch.einsum("bthi,bthj->bhij", k[:, part], v[:, part])
    y = torch.cat(out, 1).flatten(2) @ w[4]
    # (the first block reads an empty state: its rows of y are zero, and a norm of zeros is zero)
    want_r, want_n = modulate64(x.double(), y, m[2], m[4], m[3], None, None, rows * columns, "layer", "rms")
    for name, a, b in (("r", r, want_r), ("n", n2, want_n), ("state", last, state)):
        assert float((a.double() - b).abs().max() / b.abs().max()) < 2e-2, name
    assert torch.equal(r[:, :L], x[:, :L])


def test_the_example_trains():
    model, _, _, losses = example().main(["--blocks", "3", "--tokens", "40", "--heads", "2", "--steps", "3"])
    assert all(torch.isfinite(torch.tensor(losses))) and all(torch.isfinite(p.grad).all() for p in model.parameters())


def test_the_example_gradients():
    """<gradient, direction> of the whole block against central differences, fp32 (no TF32 in torch's products).

    The loss is of order 1; its outputs are off by some 2^-20 of themselves, the mean of their squares by 2^-20 at most, the
    difference by 2^-20 / h; third derivatives leave h^2 times the gradient's size."""
    model, x, target, _ = example().main(["--blocks", "3", "--tokens", "24", "--heads", "2", "--dim", "64", "--steps", "1", "--fp32"])
    loss = lambda: (model(x).double() - target).square().mean()  # noqa: E731
    model.zero_grad(set_to_none=True)
    loss().backward()
    g = torch.Generator(device="cuda").manual_seed(2)
    h = 2.0 ** -6
    for name, p in model.named_parameters():
        way = torch.randn(p.shape, generator=g, device="cuda")
        way /= way.norm()
        told, size = float((p.grad.double() * way.double()).sum()), float(p.grad.double().norm())
        with torch.no_grad():
            p.add_(way, alpha=h)
            up = float(loss())
            p.add_(way, alpha=-2 * h)
            down = float(loss())
            p.add_(way, alpha=h)
        assert abs((up - down) / (2 * h) - told) <= 2.0 ** -20 / h * 4 + h * h * max(size, 1.0), (name, (up - down) / (2 * h), told, size)


def test_calls_on_two_streams_at_once():
    """They share no scratch: each call has its own."""
    from paper_2605_16579_b200 import arl2

    layer = arl2.Layer(1, 12, 16, 128, "bf16")
    g = torch.Generator(device="cuda").manual_seed(3)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    T = 3000
    memory, mod = arl2.Recurrence(layer, 700), arl2.Modulation(layer, 500, norm="rms")
    q, k, v, do = (randn(1, T, 12, 128).bfloat16() / 11 for _ in range(4))
    decay, w = randn(1, 5, 12), 1 + 0.1 * randn(1536)
    calls = [lambda: memory.backward(do, q, k, v, decay), lambda: mod.backward(q.flatten(2), do.flatten(2), v.flatten(2), k.flatten(2), weight=w)]
    want = [c() for c in calls]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(4):
        for i, (s, c) in enumerate(zip(streams, calls)):
            with torch.cuda.stream(s):
                got[i].append(c())
    torch.cuda.synchronize()
    for w_, runs in zip(want, got):
        for out in runs:
            assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(out, w_))
    layer.sync_status()


def test_nothing_is_written_beside_the_outputs():
    """Outputs and workspaces inside larger buffers of known bytes."""
    from paper_2605_16579_b200 import arl2

    B, T, H, D = 2, 77, 5, 64
    d = H * D
    layer = arl2.Layer(B, H, 16, D, "bf16")
    g = torch.Generator(device="cuda").manual_seed(4)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    guards = []

    def inside(shape, dtype):
        n = torch.Size(shape).numel() * torch.tensor([], dtype=dtype).element_size()
        buffer = torch.full((n + 2048,), 0xA5, dtype=torch.uint8, device="cuda")
        guards.append((buffer, n))
        return buffer[1024:1024 + n].view(dtype).view(shape)

    x, y = randn(B, T, d).bfloat16(), randn(B, T, d).bfloat16()
    mod = arl2.Modulation(layer, 10, norm="layer", post="layer")
    w, pw = 1 + 0.1 * randn(d), 1 + 0.1 * randn(d)
    mod.forward(x, y, post_weight=pw, r=inside((B, T, d), torch.bfloat16), n=inside((B, T, d), torch.bfloat16))
    mod.backward(x, y, y, y, weight=w, post_weight=pw, workspace=inside((mod.workspace_bytes(T),), torch.uint8))
    cos, sin = tables(100, D)
    turn = arl2.Rotation(layer, cos, sin, (12, 10, 10), grid=(4, 5), norm="head", kv_heads=2)
    q, k, hw = x.view(B, T, H, D), randn(B, T, 2, D).bfloat16(), 1 + 0.1 * randn(D)
    turn.forward(q, k, q_out=inside((B, T, H, D), torch.bfloat16), k_out=inside((B, T, 2, D), torch.bfloat16))
    turn.backward(q, k, q, k, q_weight=hw, k_weight=hw, workspace=inside((turn.workspace_bytes(T),), torch.uint8))
    memory = arl2.Recurrence(layer, 30)
    decay = randn(B, 3, H)
    memory.forward(q, q, q, decay, out=inside((B, T, H, D), torch.bfloat16), workspace=inside((memory.workspace_bytes(T),), torch.uint8))
    memory.backward(q, q, q, q, decay, workspace=inside((memory.workspace_bytes(T, True),), torch.uint8))
    layer.sync_status()
    for buffer, n in guards:
        assert (buffer[:1024] == 0xA5).all() and (buffer[1024 + n:] == 0xA5).all()
