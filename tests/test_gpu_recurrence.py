"""The recurrence over the blocks of a sequence on the GPU: both directions against the definition in 64 bits.

A sum of n terms in fp32 is off by at most n roundings (2^-23: tensor cores may cut instead of rounding) of the sum of their
magnitudes, whatever the order; the magnitudes come from the same recurrence over absolute values.  bf16 products are exact, a
state as two bf16 numbers is off by 2^-17 of itself; fp32 products of two TF32 numbers each are off by 2^-21.
"""
import pytest
import torch

from block_util import leaves, near

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
CASES = [
    # B, T, block, H, D, dtype, state given
    (1, 1, 1, 1, 64, BF, False),
    (1, 1, 1, 1, 128, FP, True),
    (2, 5, 1, 3, 128, BF, True),
    (2, 77, 7, 2, 64, FP, True),
    (1, 100, 300, 3, 64, BF, True),
    (2, 2003, 100, 5, 64, BF, True),
    (2, 1000, 64, 2, 64, FP, True),
    (1, 1560, 128, 2, 128, BF, False),
    (1, 1000, 129, 2, 128, FP, False),
    (3, 700, 250, 3, 128, BF, True),
    (1, 4680, 1560, 12, 128, BF, True),
    (1, 9000, 4680, 3, 128, BF, False),
    (2, 3333, 1111, 1, 64, BF, False),
    (1, 640, 16, 12, 128, BF, True),
    (1, 1500, 400, 4, 128, FP, True),
]


def op(B, H, D, dtype, block, flags=0):
    from paper_2605_16579_b200 import arl2

    return arl2, arl2.Recurrence(arl2.Layer(B, H, 16, D, dtype, flags=flags), block)


def inputs(case, seed, strided=False):
    B, T, block, H, D, dtype, begun = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    q, k, v = unit(randn(B, T, H, D)).to(dtype), unit(randn(B, T, H, D)).to(dtype), randn(B, T, H, D).to(dtype)
    if strided:   # parts of one row, as a joint projection leaves them
        q, k, v = torch.cat((q, k, v), 2).unflatten(2, (3, H)).unbind(2)
    decay = 2 + 2 * randn(B, -(-T // block), H)
    return q, k, v, decay, (randn(B, H, D, D) if begun else None), randn


def recur64(q, k, v, alpha, state, block):
    out = []
    for n in range(alpha.shape[1]):
        part = slice(n * block, (n + 1) * block)
        out.append(torch.einsum("bthi,bhij->bthj", q[:, part], state))
        state = alpha[:, n, :, None, None] * state + torch.einsum("bthi,bthj->bhij", k[:, part], v[:, part])
    return torch.cat(out, 1), state


def zeros_like_state(q):
    return torch.zeros(q.shape[0], q.shape[2], q.shape[3], q.shape[3], dtype=torch.float64, device=q.device)


def parts_of(case):
    """(relative error of a product with a state, of a state's terms and sums)"""
    _, T, block, _, D, dtype, _ = case
    sums = (min(block, T) + D + -(-T // block) + 64) * 2.0 ** -23
    return (2.0 ** -16 if dtype == BF else 2.0 ** -20) + sums, (0 if dtype == BF else 2.0 ** -20) + sums


def check(case, flags=0, strided=False):
    B, T, block, H, D, dtype, begun = case
    _, r = op(B, H, D, dtype, block, flags)
    q, k, v, decay, state, randn = inputs(case, 1, strided)
    do, dstate = randn(B, T, H, D).to(dtype), randn(B, H, D, D) if begun else None
    out, last = r.forward(q, k, v, decay, state=state)
    grads = r.backward(do, q, k, v, decay, state=state, dstate=dstate)
    r.layer.sync_status()

    x = leaves(q, k, v, decay)
    s0 = (zeros_like_state(q) if state is None else state.double()).requires_grad_(True)
    want, want_last = recur64(x[0], x[1], x[2], torch.sigmoid(x[3]), s0, block)
    want_grads = torch.autograd.grad((want, want_last), x + [s0], (do.double(), torch.zeros_like(want_last) if dstate is None else dstate.double()))

    with torch.no_grad():   # magnitudes: the same over absolute values
        rows, sums = parts_of(case)
        mag = [t.double().abs() for t in (q, k, v)]
        alpha = torch.sigmoid(decay.double())
        y = leaves(*mag, decay)
        with torch.enable_grad():
            m0 = s0.detach().abs().requires_grad_(True)
            m_out, m_last = recur64(y[0], y[1], y[2], torch.sigmoid(y[3]), m0, block)
            m_grads = torch.autograd.grad((m_out, m_last), y + [m0], (do.double().abs(), torch.zeros_like(m_last) if dstate is None else dstate.double().abs()))
        near(out, want, rows * m_out, "out")
        near(last, want_last, sums * m_last, "state")
        for name, a, b, m in zip(("dq", "dk", "dv"), grads, want_grads, m_grads):
            near(a, b, rows * m, name)
        near(grads[3], want_grads[3], 2 * rows * m_grads[3].abs(), "ddecay")
        near(grads[4], want_grads[4], sums * m_grads[4], "dstate")
        assert alpha.shape == grads[3].shape
    # without what may be left out: the sums are cut elsewhere, so other bits within the same bounds
    alone, none = r.forward(q, k, v, decay, state=state, final=False)
    assert none is None
    near(alone, want, rows * m_out, "out without the last state")
    again = r.backward(do, q, k, v, decay, state=state, dstate=dstate, initial=False)
    assert again[4] is None
    for a, b, m in zip(again, want_grads[:4], m_grads):
        near(a, b, 2 * rows * m.abs(), "without the first state's gradient")


@pytest.mark.parametrize("case", CASES)
def test_both_directions(case):
    check(case)


@pytest.mark.parametrize("case", [CASES[2], CASES[5], CASES[9]])
def test_plain_kernels_with_bf16(case):
    from paper_2605_16579_b200 import arl2

    check(case, flags=arl2.ARL2_FLAG_FORCE_SIMT)


@pytest.mark.parametrize("case", [CASES[3], CASES[8], CASES[14]])
def test_plain_kernels_with_fp32(case):
    from paper_2605_16579_b200 import arl2

    check(case, flags=arl2.ARL2_FLAG_FORCE_SIMT)


@pytest.mark.parametrize("case", [
    (1, 4000, 40, 5, 64, FP, True),       # several units for each CTA, a head without a neighbour
    (2, 6000, 131, 4, 128, FP, True),     # ... and a tile that has three rows
    (1, 3000, 1500, 3, 64, FP, False),
    (2, 3000, 1433, 3, 64, FP, True),
    (1, 2000, 2000, 1, 128, FP, True),
    (3, 65, 33, 1, 64, FP, True),
])
@pytest.mark.parametrize("strided", [False, True])
def test_fp32_rows(case, strided):
    check(case, strided=strided)


@pytest.mark.parametrize("case", [CASES[5], CASES[8], CASES[9]])
def test_strided_rows(case):
    check(case, strided=True)


@pytest.mark.parametrize("case", [
    (1, 900, 3, 2, 64, BF, True),
    (1, 512, 2, 1, 128, BF, False),
    (1, 1300, 5, 2, 64, FP, True),
    (2, 257, 1, 1, 64, FP, True),
    (1, 1541, 6, 1, 128, FP, False),
])
def test_hundreds_of_blocks(case):
    """More than a list of the scan has."""
    check(case)


def test_one_stream_for_all():
    """Rows that a stride of zero repeats over the streams."""
    B, T, block, H, D = 3, 300, 130, 2, 128
    _, r = op(B, H, D, BF, block)
    q, k, v, decay, _, _ = inputs((B, T, block, H, D, BF, False), 2)
    one = [t[:1].expand(B, -1, -1, -1) for t in (q, k, v)]
    got = r.forward(*one, decay)
    want = r.forward(*(t.contiguous() for t in one), decay)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # ... or over the tokens, which tiled copies cannot do: the plain kernels take them, off by as much
    one[1] = k[:, :1].expand(-1, T, -1, -1)
    case = (B, T, block, H, D, BF, False)
    out, last = r.forward(*one, decay)
    x = [t.double() for t in one]
    want, want_last = recur64(*x, torch.sigmoid(decay.double()), zeros_like_state(q), block)
    mag, mag_last = recur64(*(t.abs() for t in x), torch.sigmoid(decay.double()), zeros_like_state(q), block)
    near(out, want, parts_of(case)[0] * mag, "out")
    near(last, want_last, parts_of(case)[1] * mag_last, "state")
    do = v.contiguous()
    for a, b in zip(r.backward(do, *one, decay), r.backward(do, *(t.contiguous() for t in one), decay)):
        assert float((a.double() - b.double()).abs().max()) <= 2.0 ** -7 * float(b.double().abs().max())


def test_states_in_place():
    """The C calls: a state may be replaced by the one behind the last block, and its gradient by that of the one before the first."""
    import ctypes

    B, T, block, H, D = 2, 50, 20, 3, 64
    arl2, r = op(B, H, D, BF, block)
    q, k, v, decay, state, randn = inputs((B, T, block, H, D, BF, True), 9)
    want, want_last = r.forward(q, k, v, decay, state=state)
    do, dstate = randn(B, T, H, D).to(BF), randn(B, H, D, D)
    grads = r.backward(do, q, k, v, decay, state=state, dstate=dstate)
    lib, stream = arl2.load(), torch.cuda.current_stream().cuda_stream
    rows = [ctypes.byref(arl2.arl2_rows(t.data_ptr(), T * H * D, H * D)) for t in (q, k, v)]
    ws = torch.empty(r.workspace_bytes(T, True), dtype=torch.uint8, device="cuda")
    s, ds, out = state.clone(), dstate.clone(), [torch.empty_like(q) for _ in range(4)]
    args = (r.layer._ctx, ctypes.byref(r.cfg), T)
    assert lib.arl2_recur(*args, *rows, decay.data_ptr(), s.data_ptr(), out[0].data_ptr(), s.data_ptr(), ws.data_ptr(), ws.numel(), stream) == 0
    assert torch.equal(out[0], want) and torch.equal(s, want_last)
    assert lib.arl2_recur_backward(*args, do.data_ptr(), *rows, decay.data_ptr(), state.data_ptr(), ds.data_ptr(), *(t.data_ptr() for t in out[1:]), None,
                                   ds.data_ptr(), ws.data_ptr(), ws.numel(), stream) == 0
    assert torch.equal(ds, grads[4]) and all(torch.equal(a, b) for a, b in zip(out[1:], grads[:3]))
    # and what may not be the same memory
    assert lib.arl2_recur(*args, *rows, decay.data_ptr(), None, q.data_ptr(), None, ws.data_ptr(), ws.numel(), stream) == -1
    assert lib.arl2_recur_backward(*args, do.data_ptr(), *rows, decay.data_ptr(), None, None, do.data_ptr(), out[1].data_ptr(), out[2].data_ptr(), None, None,
                                   ws.data_ptr(), ws.numel(), stream) == -1


def test_block_after_block_is_the_layer():
    """The readout and the commit of the layer itself: queries and keys of length one, no feature maps.

    The layer reads its state as bf16 (2^-9 of it) and makes lengths of one again (2^-8 of a bf16 row): a few hundredths of the outputs'
    size, as its own parity tests allow."""
    B, L, N, H, D = 1, 200, 3, 2, 128
    arl2, r = op(B, H, D, BF, L)
    q, k, v, decay, _, _ = inputs((B, L * N, L, H, D, BF, False), 3)
    out, last = r.forward(q, k, v, decay)
    layer = arl2.Layer(B, H, L, D, "bf16")
    layer.set_params()
    big = torch.full((B, L, H), 50.0, device="cuda")
    for n in range(N):
        part = slice(n * L, (n + 1) * L)
        a, b, c = (t[:, part].contiguous() for t in (q, k, v))
        # gate 1 less gate 0: the readout alone
        got = layer.denoise_step(a, b, c, big).float() - layer.denoise_step(a, b, c, -big).float()
        if n > 0:
            assert float((got - out[:, part].float()).abs().max() / out[:, part].float().abs().max()) < 4e-2
        layer.commit(b, c, decay[:, n].contiguous())
    assert float((layer.get_state().cuda() - last).abs().max() / last.abs().max()) < 2e-2


def test_gates_at_their_ends():
    """Gates of zero (the state is forgotten) and one, and what they are the gradients of."""
    B, T, block, H, D = 1, 256, 64, 1, 64
    _, r = op(B, H, D, FP, block)
    q, k, v, decay, state, randn = inputs((B, T, block, H, D, FP, True), 4)
    decay[:, 1], decay[:, 2] = -float("inf"), float("inf")
    out, last = r.forward(q, k, v, decay, state=state)
    want, want_last = recur64(q.double(), k.double(), v.double(), torch.sigmoid(decay.double()), state.double(), block)
    near(out, want, 1e-5 * want.abs().max(), "out")
    near(last, want_last, 1e-5 * want_last.abs().max(), "state")
    dq, dk, dv, dd, ds = r.backward(randn(*out.shape), q, k, v, decay, state=state)
    assert dd[:, 1].abs().max() == 0 and dd[:, 2].abs().max() == 0 and all(torch.isfinite(t).all() for t in (dq, dk, dv, dd, ds))


def test_backward_against_differences():
    """<gradient, direction> against central differences of the kernel's own forward pass in fp32 (bounds as for the modulation; the
    recurrence is linear in each of q, k, v and the state, and its products are off by 2^-21)."""
    case = (1, 90, 25, 2, 64, FP, True)
    B, T, block, H, D, _, _ = case
    _, r = op(B, H, D, FP, block)
    q, k, v, decay, state, randn = inputs(case, 5)
    do, dstate = randn(B, T, H, D), randn(B, H, D, D)
    vals = [q.contiguous(), k.contiguous(), v.contiguous(), decay, state]

    def loss(x):
        out, last = r.forward(*x[:4], state=x[4])
        return float((out.double() * do).sum() + (last.double() * dstate).sum())

    grads = r.backward(do, *vals[:4], state=state, dstate=dstate)
    size = (float(r.forward(*vals[:4], state=state)[0].double().norm()) + float(state.norm())) * 2.0 ** -20
    h = 2.0 ** -4
    for i, g in enumerate(grads):
        way = randn(*vals[i].shape)
        way /= way.norm()
        plus, minus = ([x + s * h * way if j == i else x for j, x in enumerate(vals)] for s in (1, -1))
        measured = (loss(plus) - loss(minus)) / (2 * h)
        told = float((g.double() * way.double()).sum())
        assert abs(measured - told) <= h * h * float(g.double().norm()) * (1 if i == 3 else 0) + size / h, (i, measured, told)


def test_same_bits_again_and_on_another_stream_and_in_a_graph():
    case = (1, 5000, 700, 12, 128, BF, True)
    B, T, block, H, D, _, _ = case
    _, r = op(B, H, D, BF, block)
    q, k, v, decay, state, randn = inputs(case, 6)
    do, dstate = randn(B, T, H, D).to(BF), randn(B, H, D, D)

    def both():
        return r.forward(q, k, v, decay, state=state) + r.backward(do, q, k, v, decay, state=state, dstate=dstate)

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
    v.copy_(v.flip(1))
    for _ in range(2):
        eager = both()
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, eager))
    r.layer.sync_status()


def test_a_wait_that_expires_is_reported():
    """The output is undefined then, the layer stays usable."""
    case = (1, 600, 300, 2, 128, BF, False)
    arl2, r = op(1, 2, 128, BF, 300)
    q, k, v, decay, _, _ = inputs(case, 7)
    want = r.forward(q, k, v, decay)
    r.layer.debug_set_wait_limit(0)
    r.forward(q, k, v, decay)
    with pytest.raises(arl2.Arl2Error, match="expired"):
        r.layer.sync_status()
    r.layer.debug_set_wait_limit(-1)
    got = r.forward(q, k, v, decay)
    r.layer.sync_status()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("D", [64, 128])
def test_a_wait_that_expires_is_reported_fp32(D):
    arl2, r = op(1, 3, D, FP, 100)
    q, k, v, decay, _, randn = inputs((1, 2950, 100, 3, D, FP, False), 7)
    do = randn(1, 2950, 3, D)
    want = r.forward(q, k, v, decay)[0], *r.backward(do, q, k, v, decay)[:4]
    for call in (lambda: r.forward(q, k, v, decay), lambda: r.backward(do, q, k, v, decay)):
        r.layer.debug_set_wait_limit(0)
        call()
        with pytest.raises(arl2.Arl2Error, match="expired"):
            r.layer.sync_status()
        r.layer.debug_set_wait_limit(-1)
    got = r.forward(q, k, v, decay)[0], *r.backward(do, q, k, v, decay)[:4]
    r.layer.sync_status()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_wrong_tensors_are_refused():
    case = (2, 20, 8, 2, 128, BF, True)
    arl2, r = op(2, 2, 128, BF, 8)
    q, k, v, decay, state, randn = inputs(case, 8)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    bad = [
        lambda: r.forward(q.float(), k, v, decay), lambda: r.forward(q, k[:, :8], v, decay), lambda: r.forward(q, k, v.cpu(), decay),
        lambda: r.forward(q, k, v, decay[:, :2]), lambda: r.forward(q, k, v, decay.bfloat16()), lambda: r.forward(q, k, v, decay, state=state[:1]),
        lambda: r.forward(q.transpose(2, 3), k, v, decay), lambda: r.forward(q, k, v, decay, out=q), lambda: r.forward(q, k, v, decay, workspace=small),
        lambda: r.forward(q, k, v, decay, workspace=torch.empty(10)), lambda: r.backward(q[:, :8], q, k, v, decay), lambda: r.backward(q, q, k, v, decay, dstate=state.bfloat16()),
        lambda: r.backward(q, q, k, v, decay, workspace=small), lambda: arl2.Recurrence(r.layer, 0), lambda: r.forward(q[:, :0], k[:, :0], v[:, :0], decay[:, :0]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(arl2.Arl2Error):
            call()
            pytest.fail(f"call {i} was not refused")
    r.forward(q, k, v, decay)
    r.layer.sync_status()
