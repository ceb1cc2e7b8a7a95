"""The 4-bit cache's scratch: any size from the least on, one for several caches, given after the cache is made, and what is refused."""
import ctypes

import pytest
import torch

from parity_util import Guarded
from paper_2605_16579_b200 import arl2
from test_gpu_cache import check, draw, fill_random, make, start_of
from test_gpu_cache_routes import fill_streams, reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def scratch(size):
    """`size` guarded bytes on 256, in which anything may stand."""
    guard = Guarded((size + 256,), torch.uint8, DEV)
    guard.t.fill_(0x5A)
    at = (-guard.t.data_ptr()) % 256
    return guard, guard.t[at:at + size], lambda: guard.intact() and bool((guard.t[:at] == 0x5A).all() and (guard.t[at + size:] == 0x5A).all())


SHAPES = [  # B, H, kv_heads, D, dtype, queries, lengths, causal
    (1, 12, 12, 128, "bf16", 1, (4000,), False),
    (2, 6, 2, 64, "bf16", 5, (900, 30), True),
    (1, 12, 12, 128, "fp32", 40, (700,), True),
    (2, 4, 4, 128, "bf16", 300, (900, 513), True),
    (1, 8, 4, 64, "bf16", 600, (1300,), False),
    (3, 12, 12, 128, "bf16", 40, (1500, 0, 1463), False),        # one item per key head
]


@pytest.mark.parametrize("B,H,kv,D,dtype,T,lengths,causal", SHAPES)
def test_any_size_from_the_least_on(B, H, kv, D, dtype, T, lengths, causal):
    n = max(lengths)
    layer, cache, pool, cos, sin = make(B, H, kv, D, dtype, 64, n, rope_rows=max(n, T), L=T)
    fill_streams(pool, lengths)
    q, qf = draw((B, T, H, D), dtype, 20)
    least, full = arl2.Cache.workspace_range(layer, pool.count, pool.width, kv_heads=kv, page_tokens=64)
    assert cache.workspace.numel() == full
    ref = reference(qf, pool, lengths, causal, cos, sin)
    rows = 2 * 148 * 256 * 4 * (D + 2) + 8192       # all partial rows
    sizes = sorted({least, (least + min(full, rows)) // 2, min(full, rows + (1 << 20)), (rows + full) // 2 if full > rows else full, full - 1, full})
    first = cache.attend(q, start_of(lengths), causal=causal)
    for size in sizes:
        guard, room, intact = scratch(size)
        cache.set_workspace(room)
        out = cache.attend(q, start_of(lengths), causal=causal)
        again = cache.attend(q, start_of(lengths), causal=causal)
        layer.sync_status()
        check(out, *ref, dtype, n)
        assert torch.equal(out, again) and intact(), size
        if size == full:
            assert torch.equal(out, first)


def test_one_scratch_for_several_caches():
    """Two contexts of different types and shapes, calls in turn, few rows and many: as with a scratch of their own."""
    caches, calls, want = [], [], []
    for D, dtype, H, T, n, seed in ((128, "bf16", 4, 290, 700, 1), (64, "fp32", 6, 3, 2000, 2), (64, "bf16", 2, 100, 500, 3)):
        layer, cache, pool, _, _ = make(2, H, 2, D, dtype, 32, n, L=T)
        fill_random(pool, n, seed)
        for queries in (1, T):
            q, _ = draw((2, queries, H, D), dtype, seed)
            calls.append((layer, cache, q, start_of((n, n - 77))))
        caches.append((layer, cache, pool))
    for layer, cache, q, lengths in calls:
        want.append(cache.attend(q, lengths))
        layer.sync_status()
    guard, room, intact = scratch(max(cache.workspace.numel() for _, cache, _ in caches))
    for _, cache, _ in caches:
        cache.set_workspace(room)
        assert cache.workspace is room
    for _ in range(3):
        outs = [cache.attend(q, lengths) for _, cache, q, lengths in calls]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)) and intact()
    for layer, _, _ in caches:
        layer.sync_status()
    # given when the cache is made
    layer, cache, pool = caches[0]
    other = arl2.Cache(layer, pool.count, pool.width, kv_heads=2, page_tokens=32, pages=pool.guard.t, page_table=pool.table, workspace=room)
    assert torch.equal(other.attend(calls[1][2], calls[1][3]), want[1]) and intact()


def test_workspace_after_the_cache_and_refusals():
    layer, cache, pool, _, _ = make(1, 2, 2, 128, "bf16", 64, 300)
    fill_random(pool, 300, 50)
    q, _ = draw((1, 1, 2, 128), "bf16", 51)
    want = cache.attend(q, start_of((300,)))
    lib, handle, out, lengths = arl2.load(), ctypes.c_void_p(), torch.empty_like(q), start_of((300,))
    stream = torch.cuda.current_stream().cuda_stream
    before = layer.launch_count
    create = lambda ws, n: lib.arl2_cache_create(layer._ctx, ctypes.byref(cache.cfg), pool.guard.t.data_ptr(), pool.table.data_ptr(),  # noqa: E731
                                                 None, None, ws, n, stream, ctypes.byref(handle))
    attend = lambda: lib.arl2_cache_attend(handle, q.data_ptr(), 256, 256, 1, lengths.data_ptr(), None, 0, out.data_ptr(), stream)  # noqa: E731
    assert create(None, 1) == -1 and create(None, 0) == 0
    assert attend() == -5 and b"workspace" in lib.arl2_last_error()
    least, full = arl2.Cache.workspace_range(layer, pool.count, pool.width)
    guard, room, intact = scratch(least)
    give = lambda ws, n: lib.arl2_cache_set_workspace(handle, ws, n, stream)  # noqa: E731
    assert give(None, least) == -1 and give(room.data_ptr(), least - 1) == -5 and give(room.data_ptr() + 16, full) == -5
    assert attend() == -5 and layer.launch_count == before
    assert give(room.data_ptr(), least) == 0 and attend() == 0
    torch.cuda.synchronize()
    assert torch.equal(out, want) and intact() and layer.launch_count == before + 2
    lib.arl2_cache_destroy(handle)
    for bad in (torch.empty(least - 1, dtype=torch.uint8, device=DEV), torch.empty(full, dtype=torch.uint8), torch.empty(full, dtype=torch.int32, device=DEV),
                torch.empty(2, full, dtype=torch.uint8, device=DEV)[:, ::2], None):
        with pytest.raises(arl2.Arl2Error):
            cache.set_workspace(bad)
    with pytest.raises(arl2.Arl2Error):
        arl2.Cache(layer, pool.count, pool.width, workspace=torch.empty(100, dtype=torch.uint8, device=DEV))
    assert torch.equal(cache.attend(q, lengths), want)


def test_append_needs_no_workspace():
    layer, cache, pool, _, _ = make(1, 2, 2, 128, "bf16", 64, 100)
    (k, _), (v, _) = draw((1, 100, 2, 128), "bf16", 1), draw((1, 100, 2, 128), "bf16", 2)
    cache.append(k, v, start_of((0,)))
    want = pool.guard.t.clone()
    pool.guard.t.fill_(0xFF)
    lib, handle = arl2.load(), ctypes.c_void_p()
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.arl2_cache_create(layer._ctx, ctypes.byref(cache.cfg), pool.guard.t.data_ptr(), pool.table.data_ptr(), None, None, None, 0, stream,
                                 ctypes.byref(handle)) == 0
    start = start_of((0,))
    assert lib.arl2_cache_append(handle, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), 100, start.data_ptr(), None, None,
                                 stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(pool.guard.t, want)
    lib.arl2_cache_destroy(handle)
