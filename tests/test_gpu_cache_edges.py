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


# ---------------------------------------------------------------------------------------------- attention
def fill_streams(pool, k, v):
    pool.fill(k.astype(np.float32), v.astype(np.float32))


@pytest.mark.parametrize("dtype,D,H,kv,queries", [("bf16", 128, 2, 2, 1), ("bf16", 64, 2, 2, 1), ("bf16", 128, 6, 2, 4), ("bf16", 64, 2, 2, 12),
                                                  ("fp32", 128, 2, 2, 1), ("fp32", 64, 4, 2, 6), ("bf16", 128, 2, 2, 70)])
@pytest.mark.parametrize("first", [3, 11, 150])
def test_values_not_finite_beside_wide_ones(dtype, D, H, kv, queries, first):
    """Tokens whose values are NaN, hidden from some rows by causality, in the same tile of keys as visible values of a wide range."""
    n = first + queries + 9
    layer, cache, pool, _, _ = make(1, H, kv, D, dtype, 16, n)
    rng = np.random.default_rng(first)
    k, v = rng.standard_normal((1, n, kv, D)), 200.0 * rng.standard_normal((1, n, kv, D))
    v[0, first + 1:first + 3] = np.nan             # seen by the third and later rows (the second sees one of them)
    fill_streams(pool, k, v)
    q, qf = draw((1, queries, H, D), dtype, 41)
    out = cache.attend(q, start_of((n,)), q_start=start_of((first,)), causal=True)
    layer.sync_status()
    ref, weight_v, reach = attend64(qf, pool, (n,), (first,), True)
    got = out.double().cpu().numpy()
    assert np.isfinite(got[0, 0]).all() and np.isnan(got[0, 1:]).all()
    room = tolerance(ref, weight_v, reach, dtype, n)
    assert (np.abs(got - ref)[0, 0] <= room[0, 0]).all()


@pytest.mark.parametrize("dtype,D,H,kv", [("bf16", 128, 2, 2), ("bf16", 64, 10, 2), ("fp32", 128, 2, 2), ("fp32", 64, 4, 1)])
@pytest.mark.parametrize("first", [3, 11, 300])
def test_wide_values_that_no_row_sees(dtype, D, H, kv, first):
    """A token's queries before later tokens whose values have a range 2^29 times as wide: nothing of the visible values' accuracy is lost."""
    n = first + 20
    layer, cache, pool, _, _ = make(1, H, kv, D, dtype, 16, n)
    rng = np.random.default_rng(first)
    k, v = rng.standard_normal((1, n, kv, D)), 1e-4 * rng.standard_normal((1, n, kv, D))
    v[0, first + 1:] = 6e4 * np.sign(v[0, first + 1:])
    fill_streams(pool, k, v)
    q, qf = draw((1, 1, H, D), dtype, 41)
    out = cache.attend(q, start_of((n,)), q_start=start_of((first,)), causal=True)
    layer.sync_status()
    check(out, *attend64(qf, pool, (n,), (first,), True), dtype, n)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,T,n,route", [(1, 3, 290, 1), (1, 300, 290, 3), (2, 40, 500, 3), (65, 40, 290, 2), (1, 260, 40000, 3)])
def test_not_finite_queries_that_see_no_key(B, T, n, route, D):
    """Rows of infinities and NaN before the first key, and in streams without keys, are zero as all rows that see none are; the others
    are as without them.  Items of one CTA and of several, operands made ahead and on the way.  route: the launches of a call."""
    layer, cache, pool, _, _ = make(B, 2, 2, D, "bf16", 64, n, L=T)
    rng = np.random.default_rng(T)
    k, v = (rng.standard_normal((B, min(n, 300), 2, D)) for _ in range(2))
    fill_streams(pool, k, v)
    if n > 300:
        pool.table[:] = pool.table[:, :4].repeat(1, -(-pool.width // 4))[:, :pool.width]      # the same four pages over and over
    hidden = 2                                      # rows before the first key
    lengths, first = [n] * B, [-hidden] * B
    if B > 1:
        lengths[B - 1] = 0
    if n > T:
        first = [f + n - T for f in first]
        first[0] = -hidden
    q, _ = draw((B, T, 2, D), "bf16", 61)
    call = lambda x: cache.attend(x, start_of(lengths), q_start=start_of(first), causal=True)  # noqa: E731
    before = layer.launch_count
    plain = call(q)
    assert layer.launch_count - before == route
    bad = q.clone()
    bad[0, 0, :, 3], bad[0, 1, 0, D - 1] = float("nan"), float("-inf")
    if B > 1:
        bad[B - 1] = float("nan")
        bad[B - 1, 5, 1] = float("inf")
    out = call(bad)
    layer.sync_status()
    assert (plain[0, :hidden] == 0).all() and torch.isfinite(plain).all()
    assert torch.equal(out, plain)


@pytest.mark.parametrize("D,queries,n", [(128, 1, 120), (128, 1, 4000), (64, 12, 1000), (128, 300, 1000), (64, 50, 700)])
def test_small_weights_beside_large_ones(D, queries, n):
    """Weights of about 2^-26 of the largest, which alone bring values: every 16 keys one takes nearly all the weight, and its value is zero.

    Beyond `tolerance`: weights are fp16 numbers of up to 2^7 (few rows) or 2^15 (many) for the largest, so that one is rounded to a
    multiple of at least 2^-31 of it: off by at most 2^-32.
    """
    H = 2
    layer, cache, pool, _, _ = make(1, H, H, D, "bf16", 64, n, L=queries)
    rng = np.random.default_rng(n)
    sign = np.where(rng.random(D) < 0.5, -1.0, 1.0)
    k, v = 0.3 * rng.standard_normal((1, n, H, D)), 0.5 + rng.random((1, n, H, D))
    large = np.arange(n) % 16 == 5
    # <q, k> scale = 26 log 2 for q = sign
    k[0, large] = sign * 26 * np.log(2.0) / D ** 0.5
    v[0, large] = 0.0
    fill_streams(pool, k, v)
    qf = np.broadcast_to(sign, (1, queries, H, D)).astype(np.float32)
    q = torch.from_numpy(qf.copy()).to(torch.bfloat16).to(DEV)
    out = cache.attend(q, start_of((n,)))
    layer.sync_status()
    ref, weight_v, reach = attend64(qf, pool, (n,), None, False)
    values = np.abs(pool.values(0, n)[1]).sum(1)             # [H, D]
    room = tolerance(ref, weight_v, reach, "bf16", n) + 2.0 ** -32 * values / large.sum()
    assert (ref > 1e-7).all() and (np.abs(out.double().cpu().numpy() - ref) <= room).all()
