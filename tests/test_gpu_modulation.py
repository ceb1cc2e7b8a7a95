"""The modulation on the GPU: both directions against the definition in 64 bits, its refusals, streams and graphs."""
import pytest
import torch

from block_util import U32, leaves, modulate64, near, per_token, u

pytestmark = pytest.mark.gpu


def op(B, H, D, dtype, frame, **kw):
    from paper_2605_16579_b200 import arl2

    layer = arl2.Layer(B, H, 16, D, dtype)
    return arl2, arl2.Modulation(layer, frame, **kw)


def inputs(B, T, frame, d, dtype, wide, seed, offset=0.3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    F = -(-T // frame)
    x = (randn(B, T, d) + offset * randn(d)).to(torch.float32 if wide else dtype)
    y = randn(B, T, d).to(dtype)
    gate, scale, shift = (0.3 * randn(B, F, 3, d)).unbind(2)
    weight, post = 1 + 0.1 * randn(d), 1 + 0.1 * randn(d)
    return x, y, gate, scale, shift, weight, post, randn


CASES = [
    # B, T, frame, H, D, dtype, fp32 residual, norm, post
    (1, 1, 1, 1, 64, torch.bfloat16, False, "layer", None),
    (3, 5, 2, 1, 64, torch.float32, False, "rms", "layer"),
    (2, 333, 77, 2, 64, torch.float32, False, "rms", "rms"),
    (2, 130, 1, 3, 64, torch.bfloat16, True, "layer", "rms"),
    (1, 700, 300, 12, 128, torch.bfloat16, False, "layer", None),
    (4, 1, 1560, 12, 128, torch.bfloat16, False, "layer", "layer"),
    (1, 1201, 4, 12, 128, torch.bfloat16, False, "rms", None),
    (2, 257, 100, 17, 128, torch.bfloat16, True, "layer", None),
    (1, 150, 64, 40, 128, torch.bfloat16, True, "layer", "layer"),
    (1, 90, 50, 40, 128, torch.float32, False, "layer", "rms"),
    (1, 37, 10, 64, 128, torch.bfloat16, False, "rms", "layer"),
    (1, 3001, 4, 12, 128, torch.bfloat16, False, "layer", "rms"),
    (1, 20000, 7000, 1, 128, torch.bfloat16, False, "layer", None),
]


def slack_n(r, inverse_of, factor):
    """64 fp32 roundings of the largest magnitude that enters an element of a norm's output."""
    return 64 * U32 * (r.abs().amax(-1, keepdim=True) * inverse_of + 1) * factor


def inverse(x, kind):
    c = x - x.mean(-1, keepdim=True) if kind == "layer" else x
    return 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-6)


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    B, T, frame, H, D, dtype, wide, norm, post = case
    _, m = op(B, H, D, dtype, frame, norm=norm, post=post, residual=torch.float32 if wide else None)
    x, y, gate, scale, shift, weight, pw, _ = inputs(B, T, frame, H * D, dtype, wide, 1)
    pw = pw if post else None
    r, n = m.forward(x, y, gate=gate, scale=scale, shift=shift, weight=weight, post_weight=pw)
    w = [None if t is None else t.double() for t in (x, y, gate, scale, shift, weight, pw)]
    # the norm reads r as it is stored: the kernel's own r
    want_r, want_n = modulate64(*w, frame, norm, post, hold=lambda _: r.double())
    g = per_token(w[2], frame, T).abs()
    near(r, want_r, 64 * U32 * (w[0].abs() + g * (slack_n(w[1], inverse(w[1], post), 1) / (64 * U32) * 1.5 if post else w[1].abs())), "r")
    factor = (per_token(w[3], frame, T).abs() + 1) * w[5].abs().max()
    near(n, want_n, slack_n(r.double(), inverse(r.double(), norm), factor) + 4 * U32 * per_token(w[4], frame, T).abs(), "n")


@pytest.mark.parametrize("case", CASES)
def test_backward(case):
    B, T, frame, H, D, dtype, wide, norm, post = case
    _, m = op(B, H, D, dtype, frame, norm=norm, post=post, residual=torch.float32 if wide else None)
    x, y, gate, scale, shift, weight, pw, randn = inputs(B, T, frame, H * D, dtype, wide, 2)
    pw = pw if post else None
    dn, dr = randn(*x.shape).to(dtype), randn(*x.shape).to(x.dtype)
    got = m.backward(x, dn, dr, y, gate=gate, scale=scale, shift=shift, weight=weight, post_weight=pw)
    # x stands for r: what is added to it is taken off the 64-bit input again
    v = leaves(y, gate, scale, shift, weight, pw)
    with torch.no_grad():
        x64 = x.double() - modulate64(torch.zeros_like(x, dtype=torch.float64), *v, frame, norm, post)[0]
    x64.requires_grad_(True)
    r64, n64 = modulate64(x64, *v, frame, norm, post)
    wanted = [x64] + [t for t in v if t is not None]
    want = torch.autograd.grad((r64, n64), wanted, (dr.double(), dn.double()))
    got = [t for t in got if t is not None]
    assert len(got) == len(want)
    names = ["dx", "dy", "dgate", "dscale", "dshift", "dweight"] + (["dpost"] if post else [])
    # magnitudes that enter an element of dx and dy
    with torch.no_grad():
        big = lambda t: t.abs().amax(-1, keepdim=True)  # noqa: E731
        inv = inverse(x.double(), norm)
        hat = big(x.double()) * inv + 1
        g = big(dn.double() * (per_token(v[2], frame, T) + 1) * v[4])
        mag_x = dr.double().abs() + inv * g * (1 + hat * hat)
        mag_y = big(mag_x) * big(per_token(v[1], frame, T))
        u_mag = y.double().abs()
        if post:
            inv_y = inverse(y.double(), post)
            hat_y = big(y.double()) * inv_y + 1
            mag_y = mag_y * big(v[5]) * inv_y * (1 + hat_y * hat_y)
            u_mag = hat_y * big(v[5])
        per_frame = lambda t: torch.stack([p.sum(1) for p in t.expand(x.shape).split(frame, 1)], 1)  # noqa: E731
        count = min(frame, T) + 64 + 64
        slack = {"dx": 64 * U32 * mag_x, "dy": 64 * U32 * mag_y,
                 "dgate": count * U32 * per_frame(mag_x * u_mag),
                 "dscale": count * U32 * per_frame(dn.double().abs() * hat * v[4].abs()),
                 "dshift": count * U32 * per_frame(dn.double().abs())}
        slack["dweight"] = (B * T + 128) * U32 * (dn.double().abs() * hat * (1 + per_token(v[2], frame, T).abs())).sum((0, 1))
        slack["dpost"] = (B * T + 128) * U32 * (mag_x * u_mag * per_token(v[1], frame, T).abs()).sum((0, 1)) if post else 0
    for name, a, b in zip(names, got, want):
        near(a, b, slack[name], name)


def test_backward_against_differences():
    """<gradient, direction> against central differences of the kernel's own forward pass, fp32.

    The loss sum(r dr + n dn) is summed in 64 bits.  Outputs are off by some 2^-22 of their size s each, at random: the loss by 2^-22 s
    sqrt(count) |d|, its difference by that over h; h = 2^-6 makes it 2^-16 sqrt(count), and the third derivatives leave some h^2 of it."""
    B, T, frame, H, D = 2, 9, 4, 2, 64
    _, m = op(B, H, D, torch.float32, frame, norm="layer", post="rms")
    x, y, gate, scale, shift, weight, pw, randn = inputs(B, T, frame, H * D, torch.float32, False, 3)
    dn, dr = randn(*x.shape), randn(*x.shape)
    vals = [x, y, gate.contiguous(), scale.contiguous(), shift.contiguous(), weight, pw]

    def loss(v):
        r, n = m.forward(v[0], v[1], gate=v[2], scale=v[3], shift=v[4], weight=v[5], post_weight=v[6])
        return float((r.double() * dr).sum() + (n.double() * dn).sum())

    r, _ = m.forward(vals[0], vals[1], gate=vals[2], scale=vals[3], shift=vals[4], weight=vals[5], post_weight=vals[6])
    grads = m.backward(r, dn, dr, vals[1], gate=vals[2], scale=vals[3], shift=vals[4], weight=vals[5], post_weight=vals[6])
    h = 2.0 ** -6
    for i, g in enumerate(grads):
        way = randn(*vals[i].shape)
        way /= way.norm()
        plus, minus = ([v + s * h * way if j == i else v for j, v in enumerate(vals)] for s in (1, -1))
        measured = (loss(plus) - loss(minus)) / (2 * h)
        told = float((g.double() * way.double()).sum())
        size = float(g.double().norm())
        assert abs(measured - told) <= h * h * size + 2.0 ** -16 * x.numel() ** 0.5, (i, measured, told, size)


def test_parts_that_may_be_absent():
    B, T, frame, H, D = 2, 50, 7, 3, 128
    _, m = op(B, H, D, torch.bfloat16, frame)
    x, y, gate, scale, shift, weight, _, randn = inputs(B, T, frame, H * D, torch.bfloat16, False, 4)
    r, n = m.forward(x)
    assert r is x
    near(n, modulate64(x.double(), *[None] * 6, frame, "layer", None)[1], 64 * U32 * 30, "plain norm")
    r, n = m.forward(x, y, normed=False)
    assert n is None
    near(r, x.double() + y.double(), U32 * 16, "plain residual")
    # gradients: n alone, r alone
    dn, dr = randn(*x.shape).to(x.dtype), randn(*x.shape).to(x.dtype)
    dx, dy, *rest = m.backward(x, dn, shift=shift)
    assert dy is None and rest[0] is None and rest[1] is None and rest[2] is not None
    (v,) = leaves(x)
    want, = torch.autograd.grad(modulate64(v, *[None] * 6, frame, "layer", None)[1], v, dn.double())
    near(dx, want, 64 * U32 * 300, "dx of n alone")
    dx, dy, dgate, *rest = m.backward(None, None, dr, y, gate=gate, scale=scale)
    assert torch.equal(dx, dr) and rest == [None] * 4
    near(dy, dr.double() * per_token(gate.double(), frame, T), 0, "dy of r alone")
    near(dgate, torch.stack([p.sum(1) for p in (dr.double() * y.double()).split(frame, 1)], 1), 80 * U32 * 7 * 30, "dgate of r alone")


def test_in_place_and_expanded_rows():
    B, T, frame, H, D = 2, 64, 16, 5, 64
    _, m = op(B, H, D, torch.bfloat16, frame)
    x, y, gate, scale, shift, *_ = inputs(B, T, frame, H * D, torch.bfloat16, False, 5)
    one = [t[:1, :1].expand(B, T // frame, -1) for t in (gate, scale, shift)]
    want = m.forward(x, y, *(t.contiguous() for t in one))
    got = m.forward(x, y, *one)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    r, n = m.forward(x, y, *one, r=x, n=y)
    assert r is x and n is y and torch.equal(x, want[0]) and torch.equal(y, want[1])


def test_backward_in_place():
    """The C call: dx may be dr, and dy may be y or dn."""
    import ctypes

    B, T, frame, H, D = 2, 333, 50, 12, 128
    arl2, m = op(B, H, D, torch.bfloat16, frame)
    x, y, gate, scale, shift, weight, _, randn = inputs(B, T, frame, H * D, torch.bfloat16, False, 10)
    dn, dr = randn(*x.shape).to(x.dtype), randn(*x.shape).to(x.dtype)
    want = m.backward(x, dn, dr, y, gate=gate, scale=scale)
    ws = torch.empty(m.workspace_bytes(T), dtype=torch.uint8, device="cuda")
    rows = [ctypes.byref(arl2.arl2_rows(t.data_ptr(), t.stride(0), t.stride(1))) for t in (gate, scale)]

    def call(dn, dr, y, dx, dy):
        return arl2.load().arl2_modulate_backward(m.layer._ctx, ctypes.byref(m.cfg), T, x.data_ptr(), dn.data_ptr(), dr.data_ptr(), y.data_ptr(), *rows, None, None,
                                                  dx.data_ptr(), dy.data_ptr(), *[None] * 5, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)

    for over in ("y", "dn"):
        t = {"dn": dn.clone(), "dr": dr.clone(), "y": y.clone()}
        assert call(t["dn"], t["dr"], t["y"], t["dr"], t[over]) == 0
        assert torch.equal(t["dr"], want[0]) and torch.equal(t[over], want[1])
    assert call(dn, dr, y, dn, torch.empty_like(y)) == -1 and call(dn, dr, y, torch.empty_like(x), dr) == -1
    other = torch.empty_like(x)
    assert call(dn, dr, y, other, other) == -1


def test_a_large_mean_keeps_its_digits():
    """Rows of mean 1000 and deviation 1: each input is off by its own rounding alone, which the definition sees too."""
    B, T, H, D = 1, 40, 12, 128
    _, m = op(B, H, D, torch.float32, T)
    g = torch.Generator(device="cuda").manual_seed(6)
    x = 1000 + torch.randn(B, T, H * D, generator=g, device="cuda")
    _, n = m.forward(x)
    # the mean, a sum of some 18 levels, is off by a few roundings of 1000: against a deviation of 1
    near(n, modulate64(x.double(), *[None] * 6, T, "layer", None)[1], 24 * U32 * 1000, "n")


def test_what_is_not_finite_stays_in_its_row():
    B, T, H, D = 1, 30, 3, 128
    _, m = op(B, H, D, torch.bfloat16, 10)
    x, y, gate, scale, shift, *_ = inputs(B, T, 10, H * D, torch.bfloat16, False, 7)
    want = m.forward(x, y, gate, scale, shift)
    x2, y2 = x.clone(), y.clone()
    x2[0, 3, 5] = float("nan")
    y2[0, 17, 200] = float("inf")
    got = m.forward(x2, y2, gate, scale, shift)
    rows = [i for i in range(T) if i not in (3, 17)]
    for a, b in zip(got, want):
        assert torch.equal(a[0, rows], b[0, rows])
    assert torch.isnan(got[1][0, 3]).all() and torch.isnan(got[1][0, 17]).any()


def test_same_bits_again_and_on_another_stream_and_in_a_graph():
    B, T, frame, H, D = 1, 3001, 700, 12, 128
    _, m = op(B, H, D, torch.bfloat16, frame, norm="rms", post="rms")
    x, y, gate, scale, shift, weight, pw, randn = inputs(B, T, frame, H * D, torch.bfloat16, False, 8)
    dn, dr = randn(*x.shape).to(x.dtype), randn(*x.shape).to(x.dtype)

    def both():
        r, n = m.forward(x, y, gate, scale, shift, weight, pw)
        return (r, n) + m.backward(r, dn, dr, y, gate, scale, shift, weight, pw)

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for _ in range(3):
        eager = both()      # an eager call between replays
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(c, b) for a, b, c in zip(held, want, eager))
    # other inputs in the same places
    x.copy_(x.flip(1)), dn.copy_(dn.flip(1))
    graph.replay()
    want = both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_wrong_tensors_are_refused():
    arl2, m = op(2, 3, 128, torch.bfloat16, 4)
    x, y, gate, scale, shift, weight, pw, randn = inputs(2, 8, 4, 384, torch.bfloat16, False, 9)
    bad = [
        lambda: m.forward(x.float(), y), lambda: m.forward(x[:, :, :128], y), lambda: m.forward(x, y[:, :4]), lambda: m.forward(x.cpu()),
        lambda: m.forward(x, y, gate=gate[:, :1]), lambda: m.forward(x, y, gate=gate.bfloat16()), lambda: m.forward(x, gate=gate),
        lambda: m.forward(x, y, post_weight=pw), lambda: m.forward(x, y, weight=weight[:128]), lambda: m.forward(x, normed=False),
        lambda: m.forward(x.transpose(0, 1)), lambda: m.forward(x, y, r=y), lambda: m.forward(x, n=x), lambda: m.forward(x, r=x),
        lambda: m.forward(x, y, gate=gate.transpose(1, 2).contiguous().transpose(1, 2)),
        lambda: m.backward(x), lambda: m.backward(None, x), lambda: m.backward(x, x, gate=gate),
        lambda: m.backward(x, x, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
        lambda: arl2.Modulation(m.layer, 0), lambda: arl2.Modulation(m.layer, 4, norm="batch"), lambda: arl2.Modulation(m.layer, 4, residual=torch.float16),
        lambda: arl2.Modulation(arl2.Layer(1, 65, 4, 128, "bf16"), 4),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(arl2.Arl2Error):
            call()
            pytest.fail(f"call {i} was not refused")
    m.forward(x, y)
    m.layer.sync_status()
