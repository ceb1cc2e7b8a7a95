"""The binding refuses tensors of another GPU than the layer's.  On the host: tensors that say they are on a GPU, and no library call."""
import pytest
import torch

from paper_2605_16579_b200 import arl2


class OnGpu(torch.Tensor):
    """A host tensor that names a GPU as its device."""

    number = 0
    is_cuda = True

    @property
    def device(self):
        return torch.device("cpu") if self.number < 0 else torch.device("cuda", self.number)

    def get_device(self):
        return self.number


def on_gpu(number, shape, dtype):
    t = torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)
    t.number = number
    return t


@pytest.fixture
def layer():
    layer = arl2.Layer.__new__(arl2.Layer)
    layer.B, layer.H, layer.L, layer.D = 2, 4, 3, 64
    layer.device, layer._index, layer.dtype, layer._ctx = torch.device("cuda:1"), 1, torch.bfloat16, None
    return layer


@pytest.fixture
def cache(layer):
    cache = arl2.Cache.__new__(arl2.Cache)
    cache.layer, cache.device, cache.dtype, cache._index, cache._cache = layer, layer.device, layer.dtype, layer._index, None
    cache._B, cache._H, cache._D, cache.kv_heads = 2, 4, 64, 2
    cache._append = cache._attend = "call"
    cache.calls = []
    cache._run = lambda *args: cache.calls.append(args)
    return cache


def test_layer_wants_tensors_of_its_own_gpu(layer):
    layer._want(on_gpu(1, (2, 3), torch.float32), (2, 3), torch.float32, "x")
    for number in (0, 2, -1):
        with pytest.raises(arl2.Arl2Error, match="x: expected .* on cuda:1"):
            layer._want(on_gpu(number, (2, 3), torch.float32), (2, 3), torch.float32, "x")
    with pytest.raises(arl2.Arl2Error):
        layer._want(torch.zeros(2, 3), (2, 3), torch.float32, "x")


@pytest.mark.parametrize("at", range(6))
def test_append_takes_tensors_of_its_own_gpu(cache, at):
    number = [1] * 6
    if at < 5:
        number[at] = 0
    rows = (2, 3, 2, 64)
    k, v, kh, vh = (on_gpu(number[i], rows, torch.bfloat16) for i in (0, 1, 3, 4))
    start = on_gpu(number[2], (2,), torch.int32)
    if at == 5:
        cache.append(k, v, start, held=(kh, vh))
        assert len(cache.calls) == 1
        return
    with pytest.raises(arl2.Arl2Error):
        cache.append(k, v, start, held=(kh, vh))
    assert cache.calls == []


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("at", range(5))
def test_attend_takes_tensors_of_its_own_gpu(cache, at, strided):
    number = [1] * 5
    if at < 4:
        number[at] = 0
    q = on_gpu(number[0], (2, 3, 2, 4, 64), torch.bfloat16)[:, :, 1] if strided else on_gpu(number[0], (2, 3, 4, 64), torch.bfloat16)
    q.number = number[0]
    lengths, q_start = (on_gpu(number[i], (2,), torch.int32) for i in (1, 2))
    out = on_gpu(number[3], (2, 3, 4, 64), torch.bfloat16)
    if at == 4:
        cache.attend(q, lengths, q_start=q_start, out=out)
        assert len(cache.calls) == 1
        return
    with pytest.raises(arl2.Arl2Error):
        cache.attend(q, lengths, q_start=q_start, out=out)
    assert cache.calls == []
