"""The ways an attention call over the 4-bit cache can go: few rows and many, operands made ahead or on the way, many streams, other
contexts and streams, waits that expire, and arguments that the C entry refuses."""
import ctypes

import numpy as np
import pytest
import torch

from cache_util import Pool, attend64
from parity_util import Guarded
from paper_2605_16579_b200 import arl2, workload
from test_gpu_cache import check, draw, fill_random, make, start_of, status_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def fill_streams(pool, lengths, seed=10):
    for b, n in enumerate(lengths):
        if n > 0:
            one = Pool.__new__(Pool)
            one.__dict__ = dict(pool.__dict__, B=1, order=pool.order[b:b + 1])
            fill_random(one, n, seed + b)


def reference(qf, pool, lengths, causal, cos, sin, q_start=None):
    return attend64(qf, pool, lengths, q_start, causal, cos=None if cos is None else cos.numpy(), sin=None if sin is None else sin.numpy())


@pytest.mark.parametrize("causal", [False, True])
def test_operands_ahead_and_on_the_way_agree(causal):
    """The same call where the workspace holds the operands for certain, where the lengths decide that it does, and where they decide
    that it does not."""
    B, H, kv, T, page = 2, 4, 2, 290, 64
    lengths = (700, 513)
    outs, launches = [], []
    # capacity of a stream: the tokens that there are; and so much more that all of it would not fit
    for capacity, L in ((704, T), (1 << 19, T)):
        layer, cache, pool, cos, sin = make(B, H, kv, 128, "bf16", page, 704, rope_rows=704, L=L)
        fill_streams(pool, lengths)
        if capacity > 704:
            wide = torch.full((B, capacity // page), -7, dtype=torch.int32, device=DEV)
            wide[:, :pool.width] = pool.table
            cache = arl2.Cache(layer, pool.count, capacity // page, kv_heads=kv, page_tokens=page, pages=pool.guard.t, page_table=wide,
                               rope_cos=cos.to(DEV), rope_sin=sin.to(DEV))
        q, qf = draw((B, T, H, 128), "bf16", 20)
        before = layer.launch_count
        outs.append(cache.attend(q, start_of(lengths), causal=causal))
        launches.append(layer.launch_count - before)
        layer.sync_status()
        check(outs[-1], *reference(qf, pool, lengths, causal, cos, sin), "bf16", 700)
    assert launches == [3, 4]                   # unpack, attend, join; and with the other kernel beside it
    assert torch.equal(outs[0], outs[1])


def test_operands_on_the_way_where_the_workspace_is_too_small():
    """More cached tokens than there is room for operand tiles: the converting kernel does the work, and agrees with the others."""
    B, H, T, page, n = 1, 2, 150, 256, 4096 * 128 // 2 + 3000
    layer = arl2.Layer(B, H, T, 128, "bf16", device=DEV)
    width = -(-n // page)
    cache = arl2.Cache(layer, width, width, page_tokens=page)
    cache.page_table.copy_(torch.randperm(width, device=DEV).to(torch.int32).view(1, width))
    k, v = (torch.randn(1, 8192, H, 128, device=DEV).to(torch.bfloat16) for _ in range(2))
    for first in range(0, n, 8192):
        m = min(8192, n - first)
        cache.append(k[:, :m] * 1.5, v[:, :m], start_of((first,)))
    q, _ = draw((B, T, H, 128), "bf16", 21)
    long = cache.attend(q, start_of((n,)))
    layer.sync_status()
    assert torch.isfinite(long).all()
    # against the few-row kernel, 16 queries at a time
    parts = [cache.attend(q[:, i:i + 16].contiguous(), start_of((n,)), q_start=start_of((n - T + i,))) for i in range(0, T, 16)]
    far = (long.float() - torch.cat(parts, 1).float()).abs().max() / long.float().abs().max()
    assert far <= 2.0 ** -6, far
    # and a length that has room: the same cache, the other kernel
    short = cache.attend(q, start_of((500,)))
    parts = [cache.attend(q[:, i:i + 16].contiguous(), start_of((500,)), q_start=start_of((500 - T + i,))) for i in range(0, T, 16)]
    layer.sync_status()
    assert (short.float() - torch.cat(parts, 1).float()).abs().max() <= 2.0 ** -6 * short.float().abs().max()


@pytest.mark.parametrize("B,H,kv,T,n", [(70, 24, 3, 33, 300), (66, 2, 1, 130, 700), (12, 12, 12, 264, 900)])
def test_items_of_both_tiles_after_items_of_one(B, H, kv, T, n):
    """Items whose second tile of rows is empty among others: whoever has nothing to do in one keeps step with the ring."""
    layer, cache, pool, _, _ = make(B, H, kv, 128, "bf16", 64, n, L=T)
    lengths = [n] * B
    fill_streams(pool, lengths[:1])
    pool.table[1:] = pool.table[:1]          # all streams over the same pages
    q, qf = draw((1, T, H, 128), "bf16", 64)
    q = q.expand(B, T, H, 128).contiguous()
    outs = [cache.attend(q, start_of(lengths)) for _ in range(3)]
    layer.sync_status()
    one = Pool.__new__(Pool)
    one.__dict__ = dict(pool.__dict__, B=1, order=pool.order[:1])
    ref = reference(qf, one, lengths[:1], False, None, None)
    for b in (0, B // 2, B - 1):
        check(outs[0][b:b + 1], *ref, "bf16", n)
    assert all(torch.equal(x, outs[0]) for x in outs)


@pytest.mark.parametrize("H,kv,page,T,lengths,seed", [(2, 2, 64, 7, (11,), 292), (4, 2, 256, 16, (58, 44), 256), (6, 3, 16, 16, (19, 1, 65, 65, 25), 350)])
def test_one_of_few_keys_has_nearly_all_the_weight(H, kv, page, T, lengths, seed):
    """... and a value near zero, as minimum + 8 steps: what the other keys add is not to be cut off beside the two parts."""
    layer, cache, pool, _, _ = make(len(lengths), H, kv, 128, "bf16", page, max(lengths))
    fill_streams(pool, lengths, seed=seed)
    q, qf = draw((len(lengths), T, H, 128), "bf16", seed)
    out = cache.attend(q, start_of(lengths))
    layer.sync_status()
    check(out, *reference(qf, pool, lengths, False, None, None), "bf16", max(lengths))


@pytest.mark.parametrize("D", [64, 128])
def test_operands_of_several_items_where_the_workspace_is_too_small(D):
    """Rows of several items over more cached tokens than there is room for operand tiles: both kernels go out, and the converting one
    does the work; over fewer tokens the other one."""
    B, H, T, page, n = 1, 2, 300, 256, 4096 * 128 // 2 + 3000
    layer = arl2.Layer(B, H, T, D, "bf16", device=DEV)
    width = -(-n // page)
    cache = arl2.Cache(layer, width, width, page_tokens=page)
    cache.page_table.copy_(torch.randperm(width, device=DEV).to(torch.int32).view(1, width))
    k, v = (torch.randn(1, 8192, H, D, device=DEV).to(torch.bfloat16) for _ in range(2))
    for first in range(0, n, 8192):
        m = min(8192, n - first)
        cache.append(k[:, :m] * 1.5, v[:, :m], start_of((first,)))
    q, _ = draw((B, T, H, D), "bf16", 21)
    for tokens in (n, 500):
        before = layer.launch_count
        out = cache.attend(q, start_of((tokens,)))
        assert layer.launch_count - before == 4
        parts = [cache.attend(q[:, i:i + 20].contiguous(), start_of((tokens,)), q_start=start_of((tokens - T + i,))) for i in range(0, T, 20)]
        layer.sync_status()
        far = (out.float() - torch.cat(parts, 1).float()).abs().max() / out.float().abs().max()
        assert far <= 2.0 ** -6, (tokens, far)


@pytest.mark.parametrize("B,H,T,n", [(3, 12, 40, 1500), (1, 6, 130, 9000)])
def test_one_item_per_head_converts_on_the_way(B, H, T, n):
    """More than two key tiles per SM for one item per key head: no operands are made ahead."""
    layer, cache, pool, cos, sin = make(B, H, H, 128, "bf16", 64, n, rope_rows=n, L=T)
    lengths = [n - 37 * b for b in range(B)]
    fill_streams(pool, lengths)
    q, qf = draw((B, T, H, 128), "bf16", 63)
    before = layer.launch_count
    out = cache.attend(q, start_of(lengths))
    assert layer.launch_count - before == 2
    layer.sync_status()
    check(out, *reference(qf, pool, lengths, False, cos, sin), "bf16", n)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,T,lengths,route", [(2, 150, (517, 260), 3), (1, 300, (1000,), 3), (65, 20, None, 2), (3, 40, (0, 129, 1), 3)])
def test_many_rows_of_64_channels(B, T, lengths, route, causal):
    """Heads of 64 channels on tcgen05: operands made ahead, on the way (many streams), empty streams and an unaligned tensor.
    route: the launches of a call."""
    rng = np.random.default_rng(T)
    if lengths is None:
        lengths = [int(x) for x in rng.integers(0, 300, B)]
    n = max(lengths)
    layer, cache, pool, cos, sin = make(B, 4, 2, 64, "bf16", 32, n, rope_rows=max(n, T), L=T)
    fill_streams(pool, lengths)
    flat, ff = draw((B * T * 4 * 64 + 1,), "bf16", 61)
    q, qf = flat[1:].view(B, T, 4, 64), ff[1:].reshape(B, T, 4, 64)          # rows on 2 bytes
    before = layer.launch_count
    out = cache.attend(q, start_of(lengths), causal=causal)
    assert layer.launch_count - before == route
    layer.sync_status()
    check(out, *reference(qf, pool, lengths, causal, cos, sin), "bf16", n)
    assert torch.equal(out, cache.attend(q.clone(), start_of(lengths), causal=causal))


def test_context_without_tcgen05_of_64_channels():
    layer = arl2.Layer(1, 2, 1, 64, "bf16", device=DEV, flags=arl2.ARL2_FLAG_FORCE_SIMT)
    pool = Pool(1, 2, 64, 32, 333, DEV)
    cache = arl2.Cache(layer, pool.count, pool.width, page_tokens=32, pages=pool.guard.t, page_table=pool.table)
    fill_random(pool, 333, 30)
    q, qf = draw((1, 100, 2, 64), "bf16", 31)
    before = layer.launch_count
    out = cache.attend(q, start_of((333,)), causal=True)
    assert layer.launch_count - before == 1
    layer.sync_status()
    check(out, *reference(qf, pool, (333,), True, None, None), "bf16", 333)


@pytest.mark.parametrize("B,T,causal", [(33, 1, False), (70, 2, True), (40, 40, False), (66, 36, True)])
def test_many_streams(B, T, causal):
    """More streams than a plan counts by lanes, than it keeps copies of, and than operands are made ahead for; of lengths that differ."""
    rng = np.random.default_rng(B)
    lengths = [int(x) for x in rng.integers(0, 150, B)]
    layer, cache, pool, cos, sin = make(B, 2, 1, 128, "bf16", 16, 150, rope_rows=256)
    fill_streams(pool, lengths)
    q, qf = draw((B, T, 2, 128), "bf16", 22)
    out = cache.attend(q, start_of(lengths), causal=causal)
    layer.sync_status()
    check(out, *reference(qf, pool, lengths, causal, cos, sin), "bf16", 150)


@pytest.mark.parametrize("queries", [3, 60, 260])
def test_context_without_tcgen05(queries):
    """A bf16 context of the plain-FMA kernels has its cache read by the warp-level kernel, whatever the rows."""
    B, H, n = 1, 2, 333
    layer = arl2.Layer(B, H, 1, 128, "bf16", device=DEV, flags=arl2.ARL2_FLAG_FORCE_SIMT)
    pool = Pool(B, H, 128, 32, n, DEV)
    cache = arl2.Cache(layer, pool.count, pool.width, page_tokens=32, pages=pool.guard.t, page_table=pool.table)
    fill_random(pool, n, 30)
    q, qf = draw((B, queries, H, 128), "bf16", 31)
    out = cache.attend(q, start_of((n,)), causal=True)
    layer.sync_status()
    check(out, *reference(qf, pool, (n,), True, None, None), "bf16", n)


def test_calls_on_another_stream():
    """Append and attention on a stream of the caller's, after work on it that makes their inputs."""
    layer, cache, pool, cos, sin = make(1, 4, 4, 128, "bf16", 16, 400, rope_rows=400, L=100)
    (k, _), (q, _) = draw((1, 400, 4, 128), "bf16", 40), draw((1, 100, 4, 128), "bf16", 41)
    cache.append(k, k, start_of((0,)))
    want = cache.attend(q, start_of((400,)))
    pool.guard.t.fill_(0xFF)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late_k, late_q = torch.zeros_like(k), torch.zeros_like(q)
        torch.cuda._sleep(20_000_000)
        late_k.copy_(k)
        late_q.copy_(q)
        start, lengths = start_of((0,)), start_of((400,))
        cache.append(late_k, late_k, start)
        out = cache.attend(late_q, lengths)
    side.synchronize()
    layer.sync_status()
    assert torch.equal(out, want)


def test_two_caches_may_share_a_context_and_follow_one_another():
    layer, one, pool, cos, sin = make(1, 2, 2, 128, "bf16", 64, 300, L=40)
    other = arl2.Cache(layer, pool.count, pool.width, page_tokens=64, pages=pool.guard.t, page_table=pool.table)
    fill_random(pool, 300, 50)
    q, _ = draw((1, 40, 2, 128), "bf16", 51)
    a = [c.attend(q, start_of((300,))) for c in (one, other, one, other)]
    layer.sync_status()
    assert all(torch.equal(x, a[0]) for x in a)


@pytest.mark.parametrize("route", ["ahead", "way"])
def test_waits_that_expire(route):
    """The tcgen05 kernel gives up at different points of its work: reported once, and the next call gives the bits of before."""
    B = 1 if route == "ahead" else 65           # (operands are made ahead for up to 64 streams)
    T, n = (300, 900) if B == 1 else (40, 200)
    layer, cache, pool, cos, sin = make(B, 2, 2, 128, "bf16", 64, n, L=T)
    fill_random(pool, n, 60)
    q, _ = draw((B, T, 2, 128), "bf16", 61)
    lengths = start_of([n] * B)
    want = cache.attend(q, lengths)
    layer.sync_status()
    expired = 0
    for polls in (0, 1, 2, 3, 5, 8, 16, 40, 100):
        layer.debug_set_wait_limit(polls)
        out = Guarded(tuple(q.shape), q.dtype, DEV)
        cache.attend(q, lengths, out=out.t)
        try:
            layer.sync_status()
            assert polls > 0 and torch.equal(out.t, want)
        except arl2.Arl2Error as e:
            assert "status -4" in str(e)
            expired += 1
        assert out.intact() and pool.guard.intact()
        layer.debug_set_wait_limit(-1)
        assert torch.equal(cache.attend(q, lengths), want)
        layer.sync_status()
    assert expired > 0


def test_workspace_is_not_left():
    """Nothing outside of the workspace's bounds is written, with either kernel."""
    B, H, n, T = 2, 2, 400, 300
    layer, cache, pool, cos, sin = make(B, H, H, 128, "bf16", 64, n, L=T)
    fill_random(pool, n, 70)
    size = cache._workspace.numel()
    guard = Guarded((size + 256,), torch.uint8, DEV)
    at = (-guard.t.data_ptr()) % 256
    guard.t[:at] = 0x5A
    guard.t[at + size:] = 0x5A
    handle = ctypes.c_void_p()
    lib = arl2.load()
    status = lib.arl2_cache_create(layer._ctx, ctypes.byref(cache.cfg), pool.guard.t.data_ptr(), pool.table.data_ptr(), None, None,
                                   guard.t.data_ptr() + at, size, torch.cuda.current_stream().cuda_stream, ctypes.byref(handle))
    assert status == 0, lib.arl2_last_error()
    for queries in (1, 16, T):
        q, _ = draw((B, queries, H, 128), "bf16", 71)
        want = cache.attend(q, start_of((n, n - 30)))
        out = torch.empty_like(want)
        status = lib.arl2_cache_attend(handle, q.data_ptr(), q.stride(0), q.stride(1), queries, start_of((n, n - 30)).data_ptr(), None, 0, out.data_ptr(),
                                       torch.cuda.current_stream().cuda_stream)
        assert status == 0
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert guard.intact() and (guard.t[:at] == 0x5A).all() and (guard.t[at + size:] == 0x5A).all()
    lib.arl2_cache_destroy(handle)


def test_c_entry_refusals():
    """Arguments that the C entry finds wrong: a status, a message, no launch."""
    layer, cache, pool, cos, sin = make(2, 4, 2, 128, "bf16", 16, 64)
    lib = arl2.load()
    x = torch.zeros(2 * 3 * 4 * 128 * 2, dtype=torch.bfloat16, device=DEV)
    y = torch.zeros_like(x)
    n = start_of((1, 1))
    p, o, s = x.data_ptr(), y.data_ptr(), n.data_ptr()
    h, row = cache._cache, 4 * 128
    before = layer.launch_count
    attend = lambda q=p, b=3 * row, t=row, m=3, lengths=s, first=None, flags=0, out=o: lib.arl2_cache_attend(h, q, b, t, m, lengths, first, flags, out, None)  # noqa: E731
    append = lambda k=p, b=3 * 256, t=256, v=p, m=3, start=s, kh=None, vh=None: lib.arl2_cache_append(h, k, b, t, v, b, t, m, start, kh, vh, None)  # noqa: E731
    for status in (attend(q=None), attend(lengths=None), attend(out=None), attend(out=p), attend(m=0), attend(m=-1), attend(flags=2), attend(t=row - 1),
                   attend(b=-1), attend(t=1 << 41), attend(q=p + 1), attend(lengths=s + 2), attend(first=s + 1),
                   append(k=None), append(v=None), append(start=None), append(m=0), append(t=255), append(b=-4), append(kh=p), append(vh=p),
                   append(kh=o, vh=o), append(k=p + 1), append(start=s + 1)):
        assert status == -1
        assert lib.arl2_last_error() != b""
    # creation
    out = ctypes.c_void_p()
    table, pages, work, size = pool.table.data_ptr(), pool.guard.t.data_ptr(), cache._workspace.data_ptr(), cache._workspace.numel()
    create = lambda pg=pages, tb=table, c=None, sn=None, w=work, n=size: lib.arl2_cache_create(  # noqa: E731
        layer._ctx, ctypes.byref(cache.cfg), pg, tb, c, sn, w, n, None, ctypes.byref(out))
    for status, want in ((create(pg=None), -1), (create(tb=None), -1), (create(w=None), -1), (create(c=pages), -1), (create(c=pages, sn=pages), -1),
                         (create(pg=pages + 16), -1), (create(n=size - 1), -5), (create(w=work + 16), -5)):
        assert status == want and out.value is None
    assert layer.launch_count == before
    layer.sync_status()
