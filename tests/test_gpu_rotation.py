"""The rotation on the GPU: both directions against the definition in 64 bits, positions, its refusals, streams and graphs."""
import pytest
import torch

from block_util import U32, angles64, grid_positions, leaves, near, rotate64, tables

pytestmark = pytest.mark.gpu

CASES = [
    # B, T, H, kv_heads, D, dtype, norm, axes, grid
    (1, 1, 1, 1, 64, torch.bfloat16, "token", (12, 10, 10), (3, 5)),
    (4, 1, 12, 12, 128, torch.bfloat16, "token", (22, 21, 21), (30, 52)),
    (3, 333, 5, 1, 64, torch.float32, "head", (12, 10, 10), (9, 11)),
    (1, 700, 12, 12, 128, torch.bfloat16, "token", (22, 21, 21), (15, 26)),
    (2, 301, 40, 8, 128, torch.bfloat16, "token", (22, 21, 21), (10, 10)),
    (1, 120, 40, 40, 128, torch.float32, "token", (1, 2, 1), (7, 9)),
    (2, 65, 8, 2, 128, torch.bfloat16, "head", (64,), (1, 1)),
    (1, 99, 3, 3, 64, torch.float32, "l2", (0, 17, 2), (4, 8)),
    (2, 77, 2, 2, 128, torch.bfloat16, None, (20, 3, 40), (5, 5)),
    (1, 41, 64, 64, 128, torch.bfloat16, "token", (22, 21, 21), (4, 4)),
    (1, 4001, 2, 1, 64, torch.bfloat16, "token", (10, 11, 11), (13, 17)),
]


def op(case, rows=400, **kw):
    from paper_2605_16579_b200 import arl2

    B, _, H, kv, D, dtype, norm, axes, grid = case
    cos, sin = tables(rows, D)
    layer = arl2.Layer(B, H, 16, D, dtype)
    return arl2, arl2.Rotation(layer, cos, sin, axes, grid=grid, norm=norm, kv_heads=kv, **kw), cos, sin


def inputs(case, seed):
    B, T, H, kv, D, dtype, norm, _, _ = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    # queries and keys as parts of one projection's rows
    both = randn(B, T, (H + kv) * D).to(dtype)
    q, k = both[..., : H * D].unflatten(-1, (H, D)), both[..., H * D:].unflatten(-1, (kv, D))
    shape = lambda n: (n * D,) if norm == "token" else (D,)  # noqa: E731
    w = [1 + 0.2 * randn(*shape(n)) if norm in ("token", "head") else None for n in (H, kv)]
    start = torch.arange(B, device="cuda", dtype=torch.int32) * 3 + 1
    return q, k, w, start, randn


def inverse(x, norm):
    if norm == "token":
        return 1 / torch.sqrt((x * x).mean((2, 3), keepdim=True) + 1e-6)
    if norm is None:
        return torch.ones_like(x[..., :1])
    return 1 / torch.sqrt(((x * x).sum(-1, keepdim=True) if norm == "l2" else (x * x).mean(-1, keepdim=True)) + 1e-6)


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("given", [False, True])
def test_forward(case, given):
    B, T, H, kv, D, dtype, norm, axes, grid = case
    _, r, cos, sin = op(case)
    q, k, (qw, kw), start, _ = inputs(case, 1)
    at = grid_positions(start, T, *grid)
    if given:
        g = torch.Generator(device="cuda").manual_seed(5)
        at = torch.randint(-3, cos.shape[0], (B, T, 3), generator=g, device="cuda")
    where = {"positions": at.int()} if given else {"start": start}
    got = r.forward(q, k, q_weight=qw, k_weight=kw, **where)
    unit = angles64(cos, sin, axes, at)
    for name, x, w, o in (("q", q, qw, got[0]), ("k", k, kw, got[1])):
        x = x.double()
        big = x.abs().amax((2, 3), keepdim=True) * inverse(x, norm) * (1 if w is None else float(w.abs().max()))
        near(o, rotate64(x, unit, norm, None if w is None else w.double()), 64 * U32 * big, name)
    # queries alone are other lanes' work, whose sums of squares are added in another order: the same bound, not the same bits
    alone, none = r.forward(q, q_weight=qw, **where)
    x = q.double()
    big = x.abs().amax((2, 3), keepdim=True) * inverse(x, norm) * (1 if qw is None else float(qw.abs().max()))
    near(alone, rotate64(x, unit, norm, None if qw is None else qw.double()), 64 * U32 * big, "q alone")
    assert none is None
    r.layer.sync_status()


@pytest.mark.parametrize("case", CASES)
def test_backward(case):
    B, T, H, kv, D, dtype, norm, axes, grid = case
    _, r, cos, sin = op(case)
    q, k, (qw, kw), start, randn = inputs(case, 2)
    dq, dk = randn(*q.shape).to(dtype), randn(*k.shape).to(dtype)
    got = r.backward(dq, dk, q, k, start=start, q_weight=qw, k_weight=kw)
    unit = angles64(cos, sin, axes, grid_positions(start, T, *grid))
    alone = r.backward(dq, None, q, start=start, q_weight=qw)
    assert alone[1] is None and alone[3] is None
    for name, x, w, d, dx, dw in (("q", q, qw, dq, got[0], got[2]), ("k", k, kw, dk, got[1], got[3]), ("q alone", q, qw, dq, alone[0], alone[2])):
        v = leaves(x, w)
        out = rotate64(v[0], unit, norm, v[1])
        want = torch.autograd.grad(out, [t for t in v if t is not None], d.double())
        with torch.no_grad():
            inv = inverse(v[0], norm)
            over = (2, 3) if norm == "token" else (3,)
            hat = v[0].abs().amax(over, keepdim=True) * inv
            g = d.double().abs().amax((2, 3), keepdim=True) * 2 * (1 if w is None else float(w.abs().max()))
            # the mean of G hat (a sum, for rows of length one, of D terms)
            mag = inv * g * (1 + hat * hat * (D if norm == "l2" else 1)) if norm else g
            near(dx, want[0], 64 * U32 * mag, "d" + name)
            if w is not None:
                terms = (d.double().abs() * 2 * hat)
                total = terms.sum((0, 1)).flatten() if norm == "token" else terms.expand(d.shape).sum((0, 1, 2))
                near(dw, want[1], (B * T * (1 if norm == "token" else x.shape[2]) + 128) * U32 * total.max(), "weight of " + name)


def test_backward_against_differences():
    """<gradient, direction> against central differences of the kernel's own forward pass in fp32; bounds as for the modulation."""
    case = (1, 7, 3, 2, 64, torch.float32, "token", (12, 10, 10), (2, 2))
    _, r, _, _ = op(case)
    q, k, (qw, kw), start, randn = inputs(case, 3)
    dq, dk = randn(*q.shape), randn(*k.shape)
    vals = [q.contiguous(), k.contiguous(), qw, kw]

    def loss(v):
        a, b = r.forward(v[0], v[1], start=start, q_weight=v[2], k_weight=v[3])
        return float((a.double() * dq).sum() + (b.double() * dk).sum())

    grads = r.backward(dq, dk, vals[0], vals[1], start=start, q_weight=qw, k_weight=kw)
    h = 2.0 ** -6
    for i, g in enumerate(grads):
        way = randn(*vals[i].shape)
        way /= way.norm()
        plus, minus = ([v + s * h * way if j == i else v for j, v in enumerate(vals)] for s in (1, -1))
        measured = (loss(plus) - loss(minus)) / (2 * h)
        told, size = float((g.double() * way.double()).sum()), float(g.double().norm())
        assert abs(measured - told) <= h * h * size + 2.0 ** -16 * q.numel() ** 0.5, (i, measured, told)


def test_length_one_is_what_the_layer_makes():
    """Rows of length one, turned: the recurrence's features; their length is 1 up to eps and roundings."""
    case = (1, 50, 4, 4, 128, torch.float32, "l2", (22, 21, 21), (5, 5))
    _, r, _, _ = op(case)
    q, k, _, start, _ = inputs(case, 4)
    a, b = r.forward(q, k, start=start)
    for t in (a, b):
        assert float((t.double().norm(dim=-1) - 1).abs().max()) < 1e-5


def test_positions_outside_of_the_tables():
    """Before them: the first row, silently; behind them: the last row, which is reported and then forgotten."""
    case = (2, 6, 2, 2, 64, torch.float32, None, (12, 10, 10), (1, 1))
    arl2, r, cos, sin = op(case, rows=9)
    q, k, _, _, _ = inputs(case, 5)
    at = torch.tensor([[-5, 0, 8], [2, -2 ** 31, 3], [0, 0, 0], [8, 8, 8], [1, 2, 3], [7, -1, 0]], device="cuda", dtype=torch.int32).expand(2, -1, -1).contiguous()
    a, _ = r.forward(q, k, positions=at)
    near(a, rotate64(q.double(), angles64(cos, sin, case[7], at), None, None), 16 * U32 * 5, "inside")
    r.layer.sync_status()
    at[1, 3, 1] = 2 ** 31 - 1
    a, _ = r.forward(q, k, positions=at)
    near(a, rotate64(q.double(), angles64(cos, sin, case[7], at), None, None), 16 * U32 * 5, "behind")
    with pytest.raises(arl2.Arl2Error, match="rotary tables"):
        r.layer.sync_status()
    r.layer.sync_status()
    start = torch.tensor([2 ** 31 - 2, 0], device="cuda", dtype=torch.int32)
    a, _ = r.forward(q, k, start=start)
    near(a[:1], rotate64(q[:1].double(), angles64(cos, sin, case[7], torch.tensor([8, 0, 0], device="cuda").expand(1, 6, 3)), None, None), 16 * U32 * 5, "far")
    with pytest.raises(arl2.Arl2Error):
        r.layer.sync_status()


def test_in_place():
    case = (2, 33, 6, 3, 64, torch.bfloat16, "head", (12, 10, 10), (3, 3))
    arl2, r, _, _ = op(case)
    q, k, (qw, kw), start, _ = inputs(case, 6)
    want = r.forward(q, k, start=start, q_weight=qw, k_weight=kw)
    a, b = q.contiguous(), k.contiguous()
    got = r.forward(a, b, start=start, q_weight=qw, k_weight=kw, q_out=a, k_out=b)
    assert got[0] is a and got[1] is b and torch.equal(a, want[0]) and torch.equal(b, want[1])


def test_same_bits_again_and_on_another_stream_and_in_a_graph():
    case = (1, 2500, 12, 12, 128, torch.bfloat16, "token", (22, 21, 21), (30, 52))
    _, r, _, _ = op(case)
    q, k, (qw, kw), start, randn = inputs(case, 7)
    dq, dk = randn(*q.shape).to(q.dtype), randn(*k.shape).to(k.dtype)

    def both():
        return r.forward(q, k, start=start, q_weight=qw, k_weight=kw) + r.backward(dq, dk, q, k, start=start, q_weight=qw, k_weight=kw)

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
    start.add_(5)
    for _ in range(2):
        graph.replay()
    want = both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_wrong_tensors_are_refused():
    case = (2, 8, 4, 2, 128, torch.bfloat16, "token", (22, 21, 21), (2, 2))
    arl2, r, cos, sin = op(case)
    q, k, (qw, kw), start, _ = inputs(case, 8)
    plain = arl2.Rotation(r.layer, cos, sin, (22, 21, 21))
    qc = q.contiguous()
    bad = [
        lambda: r.forward(q.float(), k), lambda: r.forward(q, k[:, :4]), lambda: r.forward(q[:, :, :2], k), lambda: r.forward(q.cpu(), k),
        lambda: r.forward(q, k, start=start.long()), lambda: r.forward(q, k, start=start[:1]), lambda: r.forward(q, k, positions=start),
        lambda: r.forward(q, k, q_weight=qw[:128]), lambda: r.forward(q, k, q_weight=qw.double()), lambda: plain.forward(q, q, q_weight=qw[:128].contiguous()),
        lambda: r.forward(q.transpose(2, 3), k), lambda: r.forward(q, k, q_out=q), lambda: r.forward(qc, k, k_out=qc[:, :, :2].contiguous(), q_out=qc[:1]),
        lambda: r.backward(qc, k), lambda: r.backward(qc, k.contiguous(), q), lambda: r.backward(q, None, q),
        lambda: r.backward(qc, None, q, q_weight=qw, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
        lambda: arl2.Rotation(r.layer, cos, sin, (30, 30, 30)), lambda: arl2.Rotation(r.layer, cos, sin, (-1, 2, 3)), lambda: arl2.Rotation(r.layer, cos, sin, (1, 1, 1, 1)),
        lambda: arl2.Rotation(r.layer, cos, sin, (22,), grid=(0, 1)), lambda: arl2.Rotation(r.layer, cos, sin, (22,), norm="batch"),
        lambda: arl2.Rotation(r.layer, cos, sin[:5], (22,)), lambda: arl2.Rotation(r.layer, cos, sin, (22,), kv_heads=0),
        lambda: arl2.Rotation(r.layer, cos, sin, (22,), kv_heads=200),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(arl2.Arl2Error):
            call()
            pytest.fail(f"call {i} was not refused")
    r.forward(q, k)
    r.layer.sync_status()


@pytest.mark.parametrize("H,kv,norm", [(64, 8, "token"), (64, 1, "head"), (3, 40, "token"), (40, 3, "head"), (1, 64, None)])
def test_queries_and_keys_of_very_different_widths(H, kv, norm):
    """A thread's share of a row goes by the wider of the two."""
    case = (1, 333, H, kv, 128, torch.bfloat16, norm, (22, 21, 21), (7, 9))
    test_forward(case, False)
    test_backward(case)
