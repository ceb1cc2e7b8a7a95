"""The 4-bit cache where its inputs are at their edges: outliers of one sign, rows that see nothing, values that rows do not see, small weights."""
import numpy as np
import pytest
import torch

from cache_util import Pool, attend64, hold, tolerance
from test_gpu_cache import TORCH, check, draw, make, start_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# ------------------------------------------------------------------------------------------------ append
OUTLIERS = [-np.inf, -1e30, -1e5, -7e4, np.inf, 1e30, 1e5, 7e4]


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp32", 128), ("bf16", 64), ("fp32", 64)])
def test_append_of_one_outlier(dtype, D):
    """One value of a group beyond what is held, of one sign, in a call of its own (whose lanes all hold this row); and all such rows in one
    call.  Both bit for bit as the format has them."""
    rng = np.random.default_rng(7)
    rows = (rng.standard_normal((1, len(OUTLIERS), 1, D)) * 100).astype(np.float32)
    for i, x in enumerate(OUTLIERS):
        rows[0, i, 0, 5 + i] = x
        rows[0, i, 0, 6 + i] = 0.0
    t = torch.from_numpy(rows).to(TORCH[dtype])
    code, low, step, values = hold(t.float().numpy())
    pages = []
    for single in (True, False):
        layer, cache, pool, _, _ = make(1, 1, 1, D, dtype, 16, 16)
        if single:
            got = [cache.append(t[:, i:i + 1].to(DEV), t[:, i:i + 1].to(DEV), start_of((i,)), held=True) for i in range(len(OUTLIERS))]
            got = [torch.cat(x, 1) for x in zip(*got)]
        else:
            got = cache.append(t.to(DEV), t.to(DEV), start_of((0,)), held=True)
        layer.sync_status()
        split, page, n = pool.split(), pool.order[0, 0], len(OUTLIERS)
        for w in range(2):
            assert (split[w][page, 0, :n] == (code[..., 0::2] | (code[..., 1::2] << 4))[0, :, 0]).all()
            assert np.array_equal(split[2 + w][page, 0, :n], np.stack((low, step), -1)[0, :, 0])
            assert torch.equal(got[w].float().cpu(), torch.from_numpy(values).to(TORCH[dtype]).float())
        pages.append(pool.guard.t.clone())
    assert torch.equal(pages[0], pages[1])
    assert np.isfinite(values).all()
