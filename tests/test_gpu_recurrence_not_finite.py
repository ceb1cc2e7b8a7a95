"""NaN and infinities in the recurrence's inputs, on each of its paths: what the definition makes not finite is not finite, and nothing else changes.

A NaN is planted as the GPU's own arithmetic writes it, all bits of the mantissa set, and with the last one alone (bf16: its own last one).  An infinity may come out as an infinity or as a NaN: the products
are made of parts of the numbers, and an infinity times a part that is zero is NaN."""
import pytest
import torch

import test_gpu_recurrence as recurrence

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
PATHS = [
    # B, T, block, H, D, dtype, state given; plain kernels asked for; keys that a stride of zero repeats
    ((1, 90, 25, 2, 64, FP, True), False, False),          # few tiles
    ((2, 300, 130, 2, 128, FP, True), True, False),
    ((2, 300, 130, 3, 64, BF, True), True, False),
    ((1, 300, 130, 2, 128, BF, False), False, True),
    ((1, 300, 130, 2, 64, FP, False), False, True),
    ((1, 1500, 400, 3, 128, FP, True), False, False),      # tensor memory from here on
    ((1, 4000, 40, 3, 64, FP, True), False, False),
    ((2, 700, 250, 3, 64, BF, True), False, False),
    ((1, 1000, 300, 2, 128, BF, False), False, False),
]
WORDS = {"nan": 0x7FFFFFFF, "negative nan": -1, "nan of one bit": 0x7F800001, "infinity": 0x7F800000, "negative infinity": -0x800000}


def plant(t, at, word):
    """Writes a number, given as the bits of a fp32 one, into a copy of t."""
    t = t.clone()
    if t.dtype == FP:
        t.view(torch.int32)[at] = word
    else:
        t.view(torch.int16)[at] = word >> 16 | (word & 1)
    return t


def definition(q, k, v, decay, state, do, dstate, block):
    x = [t.double().detach().requires_grad_(True) for t in (q, k, v, decay)]
    s0 = (recurrence.zeros_like_state(q) if state is None else state.double()).detach().requires_grad_(True)
    out, last = recurrence.recur64(x[0], x[1], x[2], torch.sigmoid(x[3]), s0, block)
    grads = torch.autograd.grad((out, last), x + [s0], (do.double(), torch.zeros_like(last) if dstate is None else dstate.double()))
    return [out.detach(), last.detach(), *grads]


@pytest.mark.parametrize("what", WORDS)
@pytest.mark.parametrize("path", range(len(PATHS)))
def test_planted(path, what):
    case, plain, repeated = PATHS[path]
    B, T, block, H, D, dtype, begun = case
    arl2, r = recurrence.op(B, H, D, dtype, block, 0)
    if plain:
        _, r = recurrence.op(B, H, D, dtype, block, arl2.ARL2_FLAG_FORCE_SIMT)
    q, k, v, decay, state, randn = recurrence.inputs(case, 11)
    do, dstate = randn(B, T, H, D).to(dtype), randn(B, H, D, D) if begun else None
    t = {"q": q, "k": k[:, :1].contiguous() if repeated else k, "v": v, "decay": decay, "state": state, "do": do, "dstate": dstate}

    def run(t):
        t = dict(t, k=t["k"].expand(-1, T, -1, -1))
        args = (t["q"], t["k"], t["v"], t["decay"])
        got = [*r.forward(*args, state=t["state"]), *r.backward(t["do"], *args, state=t["state"], dstate=t["dstate"])]
        return got, definition(*args, t["state"], t["do"], t["dstate"], block)

    clean, _ = run(t)
    assert all(torch.isfinite(c).all() for c in clean)
    b, h = B - 1, H - 1
    where = {"q": (b, T // 2, h, 5), "k": (b, 0 if repeated else T // 2, h, D - 1), "v": (b, T // 2 + 1, h, 17), "do": (b, T // 2 + 2, 0, 9),
             "state": (b, h, 3, D - 2), "dstate": (b, 0, D - 5, 6)}
    for name, at in where.items():
        if t[name] is None:
            continue
        got, want = run(dict(t, **{name: plant(t[name], at, WORDS[what])}))
        for o, g, w, c in zip(("out", "state", "dq", "dk", "dv", "ddecay", "dstate"), got, want, clean):
            finite = torch.isfinite(w)
            assert torch.equal(torch.isfinite(g), finite), f"{what} in {name}: {o}, {int((torch.isfinite(g) != finite).sum())} of {g.numel()}"
            assert torch.equal(g[finite], c[finite]), f"{what} in {name}: {o} elsewhere"
            if "nan" in what:
                assert torch.isnan(g[~finite]).all(), f"{what} in {name}: {o}"
    r.layer.sync_status()
