"""CPU-side checks of modulation, rotation and recurrence: sizes, and what is refused before any CUDA call."""
import ctypes

import pytest
import torch

from paper_2605_16579_b200 import arl2


@pytest.fixture(scope="module")
def lib():
    return arl2.load(build_if_missing=True)


def layer_config(B=2, H=12, L=16, D=128, dtype="bf16", flags=0):
    return arl2.make_config(B, H, L, D, dtype, flags=flags)


def modulation(**kw):
    v = dict(frame_tokens=100, norm=arl2.ARL2_NORM_LAYER, post_norm=arl2.ARL2_NORM_NONE, eps=0.0, flags=0)
    v.update(kw)
    return arl2.arl2_modulation_config(ctypes.sizeof(arl2.arl2_modulation_config), *v.values())


def rotation(**kw):
    v = dict(kv_heads=4, rope_rows=100, axis_pairs=(22, 21, 21), grid_rows=3, grid_columns=5, norm=arl2.ARL2_NORM_TOKEN, eps=0.0)
    v.update(kw)
    return arl2.arl2_rotation_config(ctypes.sizeof(arl2.arl2_rotation_config), *v.values())


def recurrence(block=100):
    return arl2.arl2_recurrence_config(ctypes.sizeof(arl2.arl2_recurrence_config), block)


def sizes(lib, cfg, tokens, m=None, t=None, e=None):
    r = ctypes.byref
    return [lib.arl2_modulation_workspace_bytes(r(cfg), r(m), tokens) if m else 0, lib.arl2_rotation_workspace_bytes(r(cfg), r(t), tokens) if t else 0,
            lib.arl2_recurrence_workspace_bytes(r(cfg), r(e), tokens, 0) if e else 0, lib.arl2_recurrence_workspace_bytes(r(cfg), r(e), tokens, 1) if e else 0]


def test_structs_match_the_header():
    assert [ctypes.sizeof(s) for s in (arl2.arl2_rows, arl2.arl2_modulation_config, arl2.arl2_rotation_config, arl2.arl2_recurrence_config)] == [24, 24, 40, 8]


def test_workspaces(lib):
    cfg = layer_config()
    small, large = (sizes(lib, cfg, n, modulation(), rotation(), recurrence()) for n in (1, 20000))
    assert all(0 < a <= b and a % 256 == 0 and b % 256 == 0 for a, b in zip(small, large))
    # sums over tokens: bounded, whatever the length; states: one of 4 D^2 bytes for each block and head at least
    assert large[:2] == sizes(lib, cfg, 10 ** 6, modulation(), rotation())[:2] and large[0] < 64 << 20
    states = 2 * 12 * 200 * 128 * 128 * 4
    assert states < large[2] < large[3]
    # a block longer than the sequence is one block
    assert sizes(lib, cfg, 50, e=recurrence(10 ** 6)) == sizes(lib, cfg, 50, e=recurrence(50))


@pytest.mark.parametrize("bad", [dict(frame_tokens=0), dict(norm=0), dict(norm=arl2.ARL2_NORM_TOKEN), dict(post_norm=arl2.ARL2_NORM_HEAD), dict(post_norm=-1),
                                 dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(flags=2)])
def test_modulations_that_are_refused(lib, bad):
    assert sizes(lib, layer_config(), 10, modulation(**bad))[0] == 0 and lib.arl2_last_error() != b""


@pytest.mark.parametrize("bad", [dict(kv_heads=0), dict(kv_heads=65), dict(rope_rows=0), dict(axis_pairs=(22, 21, 22)), dict(axis_pairs=(-1, 0, 0)),
                                 dict(axis_pairs=(2 ** 31 - 1, 2 ** 31 - 1, 2)), dict(grid_rows=0), dict(grid_columns=-3), dict(grid_rows=65536, grid_columns=65536),
                                 dict(norm=arl2.ARL2_NORM_LAYER), dict(norm=9), dict(eps=float("nan"))])
def test_rotations_that_are_refused(lib, bad):
    assert sizes(lib, layer_config(), 10, t=rotation(**bad))[1] == 0 and lib.arl2_last_error() != b""


def test_sizes_that_are_refused(lib):
    cfg = layer_config()
    for tokens in (0, -1, 2 ** 30):
        assert sizes(lib, cfg, tokens, modulation(), rotation(), recurrence()) == [0] * 4
    assert sizes(lib, cfg, 10, e=recurrence(0))[2:] == [0, 0]
    assert sizes(lib, layer_config(B=8, H=40), 2 ** 27, e=recurrence(1))[2:] == [0, 0]         # too many blocks
    wide = layer_config(H=65)
    assert sizes(lib, wide, 10, modulation(), rotation())[:2] == [0, 0]
    for c, f in ((modulation(), lib.arl2_modulation_workspace_bytes), (rotation(), lib.arl2_rotation_workspace_bytes)):
        c.struct_size -= 4
        assert f(ctypes.byref(cfg), ctypes.byref(c), 10) == 0
        assert f(ctypes.byref(cfg), None, 10) == 0 and f(None, ctypes.byref(c), 10) == 0
    c = recurrence()
    c.struct_size += 4
    assert lib.arl2_recurrence_workspace_bytes(ctypes.byref(cfg), ctypes.byref(c), 10, 1) == 0


def test_no_context_is_refused(lib):
    r, n = ctypes.byref, None
    rows = r(arl2.arl2_rows(16, 0, 0))
    assert lib.arl2_modulate(n, r(modulation()), 1, 16, n, n, n, n, n, n, n, 32, n) == -1
    assert lib.arl2_modulate_backward(n, r(modulation()), 1, 16, 32, n, n, n, n, *[n] * 10, 0, n) == -1
    assert lib.arl2_rotate(n, r(rotation()), 16, 32, 1, rows, n, n, n, n, n, 48, n, n) == -1
    assert lib.arl2_rotate_backward(n, r(rotation()), 16, 32, 1, 48, n, rows, n, *[n] * 9, 0, n) == -1
    assert lib.arl2_recur(n, r(recurrence()), 1, rows, rows, rows, 16, n, 32, n, n, 0, n) == -1
    assert lib.arl2_recur_backward(n, r(recurrence()), 1, 16, rows, rows, rows, *[n] * 9, 0, n) == -1


class OnGpu(torch.Tensor):
    """A host tensor that names a GPU as its device."""

    number = 0
    is_cuda = True

    @property
    def device(self):
        return torch.device("cuda", self.number)

    def get_device(self):
        return self.number


def on_gpu(number, shape, dtype=torch.bfloat16):
    t = torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)
    t.number = number
    return t


def test_tensors_of_another_gpu_are_refused():
    """The binding, on the host: an op of a layer on the second GPU, and no library call."""
    layer = arl2.Layer.__new__(arl2.Layer)
    layer.B, layer.H, layer.L, layer.D = 2, 4, 3, 64
    layer.device, layer._index, layer.dtype, layer._ctx, layer._lib = torch.device("cuda:1"), 1, torch.bfloat16, None, None
    op = arl2._BlockOp(layer)
    shape = (2, 5, 4, 64)
    assert op._strided(on_gpu(1, shape), shape, torch.bfloat16, "q", 2).row_stride == 256
    for number in (0, 2):
        with pytest.raises(arl2.Arl2Error, match="q: expected .* on cuda:1"):
            op._strided(on_gpu(number, shape), shape, torch.bfloat16, "q", 2)
    with pytest.raises(arl2.Arl2Error, match="workspace"):
        op._scratch(10, on_gpu(0, (10,), torch.uint8))
    with pytest.raises(arl2.Arl2Error, match="closed"):
        op._run(test_tensors_of_another_gpu_are_refused)
