"""The modulation's backward pass over narrow rows, of which a tile has many, and with short frames, which end inside a tile."""
import pytest
import torch

import test_gpu_modulation as modulation
from block_util import U32, leaves, modulate64, near, per_token

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


@pytest.mark.parametrize("case", [
    # B, T, frame, H, D, dtype, fp32 residual, norm, post: 13 to 24 rows of a tile
    (1, 9360, 1560, 2, 128, BF, False, "layer", "layer"),
    (1, 9360, 7, 2, 128, BF, False, "rms", "rms"),
    (2, 4680, 100, 4, 128, BF, False, "layer", "rms"),
    (1, 9360, 11, 5, 64, BF, True, "layer", "layer"),
    (2, 6001, 300, 2, 128, BF, True, "rms", "rms"),
    (3, 3333, 5, 1, 128, FP, False, "rms", "layer"),
    (1, 8001, 50, 2, 128, FP, False, "layer", "rms"),
    (1, 20000, 13, 1, 64, BF, False, "layer", "layer"),
    (1, 20000, 1, 1, 64, FP, False, "rms", "rms"),
    (1, 9360, 9, 2, 128, BF, False, "layer", None),
    # twelve rows and fewer
    (1, 6000, 17, 5, 128, BF, False, "layer", "rms"),
    (1, 6000, 1, 12, 64, FP, False, "layer", "layer"),
])
def test_narrow_rows(case):
    modulation.test_backward(case)


@pytest.mark.parametrize("case", [
    (1, 9360, 9, 2, 128, BF, False), (2, 6001, 300, 5, 64, BF, True), (1, 20000, 13, 1, 128, FP, False), (1, 9360, 1560, 4, 128, BF, False),
])
def test_narrow_rows_without_weights(case):
    """dn, dr and y, no second norm and no weight: bounds as for the general form."""
    B, T, frame, H, D, dtype, wide = case
    _, m = modulation.op(B, H, D, dtype, frame, residual=torch.float32 if wide else None)
    x, y, gate, scale, shift, _, _, randn = modulation.inputs(B, T, frame, H * D, dtype, wide, 12)
    dn, dr = randn(*x.shape).to(dtype), randn(*x.shape).to(x.dtype)
    got = m.backward(x, dn, dr, y, gate=gate, scale=scale, shift=shift)
    v = leaves(y, gate, scale, shift)
    with torch.no_grad():
        x64 = x.double() - per_token(v[1], frame, T) * v[0]
    x64.requires_grad_(True)
    want = torch.autograd.grad(modulate64(x64, *v, None, None, frame, "layer", None), [x64] + v, (dr.double(), dn.double()))
    with torch.no_grad():
        big = lambda t: t.abs().amax(-1, keepdim=True)  # noqa: E731
        inv = modulation.inverse(x.double(), "layer")
        hat = big(x.double()) * inv + 1
        mag_x = dr.double().abs() + inv * big(dn.double() * (per_token(v[2], frame, T) + 1)) * (1 + hat * hat)
        per_frame = lambda t: torch.stack([p.sum(1) for p in t.expand(x.shape).split(frame, 1)], 1)  # noqa: E731
        count = min(frame, T) + 128
        slack = (64 * U32 * mag_x, 64 * U32 * big(mag_x) * big(per_token(v[1], frame, T)), count * U32 * per_frame(mag_x * y.double().abs()),
                 count * U32 * per_frame(dn.double().abs() * hat), count * U32 * per_frame(dn.double().abs()))
    for name, a, b, s in zip(("dx", "dy", "dgate", "dscale", "dshift"), got, want, slack):
        near(a, b, s, name)
