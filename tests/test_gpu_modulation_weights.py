"""The modulation's backward pass from C: gradients of weights that were not given, which count as ones."""
import ctypes

import pytest
import torch

import test_gpu_modulation as modulation
from block_util import U32, near, per_token

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,D,dtype,wide", [(3, 64, torch.bfloat16, False), (12, 128, torch.bfloat16, True), (40, 128, torch.bfloat16, False), (2, 128, torch.float32, False)])
@pytest.mark.parametrize("with_dr,with_y,scaled", [(True, True, True), (True, True, False), (False, True, True), (True, False, True)])
def test_weight_gradient_without_a_weight(H, D, dtype, wide, with_dr, with_y, scaled):
    """dweight = sum over the tokens of dn N(r) (1 + scale), whatever else is given; the workspace holds NaN before the call."""
    B, T, frame = 2, 333, 50
    arl2, m = modulation.op(B, H, D, dtype, frame, residual=torch.float32 if wide else None)
    x, y, gate, scale, shift, weight, _, randn = modulation.inputs(B, T, frame, H * D, dtype, wide, 11)
    dn, dr = randn(*x.shape).to(dtype), randn(*x.shape).to(x.dtype)
    ws = torch.full((m.workspace_bytes(T) // 4,), float("nan"), device="cuda")
    dx, dy, dweight = torch.empty_like(x), torch.empty_like(y), torch.full((H * D,), float("nan"), device="cuda")
    rows = lambda t: ctypes.byref(arl2.arl2_rows(t.data_ptr(), t.stride(0), t.stride(1)))  # noqa: E731
    status = arl2.load().arl2_modulate_backward(
        m.layer._ctx, ctypes.byref(m.cfg), T, x.data_ptr(), dn.data_ptr(), dr.data_ptr() if with_dr else None, y.data_ptr() if with_y else None,
        rows(gate) if with_y else None, rows(scale) if scaled else None, None, None, dx.data_ptr(), dy.data_ptr() if with_y else None, None, None, None,
        dweight.data_ptr(), None, ws.data_ptr(), 4 * ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert status == 0
    x64 = x.double()
    c = x64 - x64.mean(-1, keepdim=True)
    inverse = modulation.inverse(x64, "layer")
    one = 1 + per_token(scale.double(), frame, T) if scaled else torch.ones_like(x64)
    terms = dn.double() * c * inverse * one
    # hat is off by 64 roundings of the row's largest magnitude, the sum by one for each term
    mag = (dn.double().abs() * (x64.abs().amax(-1, keepdim=True) * inverse + 1) * one.abs()).sum((0, 1))
    near(dweight, terms.sum((0, 1)), (B * T + 128) * U32 * mag, "dweight")
    want = m.backward(x, dn, dr if with_dr else None, y if with_y else None, gate=gate if with_y else None, scale=scale if scaled else None,
                      weight=torch.ones(H * D, device="cuda"))
    assert torch.equal(dweight, want[5]) and torch.equal(dx, want[0]) and (not with_y or torch.equal(dy, want[1]))
