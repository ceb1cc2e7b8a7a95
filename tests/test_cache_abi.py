"""CPU-side checks of the cache entry points: sizes of pages and workspaces, and what is refused before any CUDA call."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2605_16579_b200 import arl2

    return arl2.load(build_if_missing=True)


def config(**kw):
    from paper_2605_16579_b200 import arl2

    v = dict(kv_heads=4, page_tokens=64, num_pages=10, max_pages=5, rope_rows=0)
    v.update(kw)
    return arl2.arl2_cache_config(ctypes.sizeof(arl2.arl2_cache_config), v["kv_heads"], v["page_tokens"], v["num_pages"], v["max_pages"], v["rope_rows"])


def layer_config(B=2, H=12, L=16, D=128, dtype="bf16"):
    from paper_2605_16579_b200 import arl2

    return arl2.make_config(B, H, L, D, dtype)


def test_struct_matches_the_header():
    from paper_2605_16579_b200 import arl2

    assert ctypes.sizeof(arl2.arl2_cache_config) == 24


@pytest.mark.parametrize("D,kv_heads,page", [(64, 1, 16), (128, 4, 64), (128, 12, 256)])
def test_page_bytes(lib, D, kv_heads, page):
    """Per token and key head: D / 2 bytes of codes and D / 64 (minimum, step) pairs of fp16, for K and for V."""
    cfg, cache = layer_config(D=D), config(kv_heads=kv_heads, page_tokens=page)
    assert lib.arl2_cache_page_bytes(ctypes.byref(cfg), ctypes.byref(cache)) == kv_heads * page * 2 * (D // 2 + D // 64 * 4)


def test_workspace_is_bounded(lib):
    """The scratch grows with the capacity up to its bound, and a plain-FMA or fp32 context has none for operand tiles."""
    sizes = [lib.arl2_cache_workspace_bytes(ctypes.byref(layer_config()), ctypes.byref(config(max_pages=n))) for n in (1, 100, 10000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and sizes[2] == sizes[3] < 512 << 20
    assert all(n % 256 == 0 for n in sizes)
    assert lib.arl2_cache_workspace_bytes(ctypes.byref(layer_config(dtype="fp32")), ctypes.byref(config(max_pages=1 << 20))) < 64 << 20


@pytest.mark.parametrize("bad", [dict(kv_heads=0), dict(kv_heads=5), dict(kv_heads=24), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=512),
                                 dict(num_pages=0), dict(max_pages=0), dict(max_pages=1 << 25), dict(rope_rows=-1)])
def test_configurations_that_are_refused(lib, bad):
    cfg, cache = layer_config(), config(**bad)
    assert lib.arl2_cache_page_bytes(ctypes.byref(cfg), ctypes.byref(cache)) == 0
    assert lib.arl2_cache_workspace_bytes(ctypes.byref(cfg), ctypes.byref(cache)) == 0
    assert lib.arl2_last_error() != b""


def test_struct_size_and_null_are_refused(lib):
    cfg, cache = layer_config(), config()
    cache.struct_size = 20
    assert lib.arl2_cache_page_bytes(ctypes.byref(cfg), ctypes.byref(cache)) == 0
    assert lib.arl2_cache_page_bytes(ctypes.byref(cfg), None) == 0
    assert lib.arl2_cache_page_bytes(None, ctypes.byref(config())) == 0
    out = ctypes.c_void_p()
    assert lib.arl2_cache_create(None, ctypes.byref(config()), None, None, None, None, None, 0, None, ctypes.byref(out)) == -1
    assert out.value is None
    assert lib.arl2_cache_create(None, ctypes.byref(config()), None, None, None, None, None, 0, None, None) == -1
    assert lib.arl2_cache_append(None, None, 0, 0, None, 0, 0, 1, None, None, None, None) == -1
    assert lib.arl2_cache_attend(None, None, 0, 0, 1, None, None, 0, None, None) == -1
    lib.arl2_cache_destroy(None)


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "bf16"), (64, "fp32"), (128, "fp32")])
def test_least_workspace(lib, D, dtype):
    """The least scratch: 14336 partial rows (28 SMs' of 256, two each) beside two small tables, whatever the capacity."""
    cfg = layer_config(D=D, dtype=dtype)
    sizes = [lib.arl2_cache_least_workspace_bytes(ctypes.byref(cfg), ctypes.byref(config(max_pages=n))) for n in (1, 100, 1 << 20)]
    assert len(set(sizes)) == 1 and sizes[0] % 256 == 0
    assert 0 <= sizes[0] - 14336 * 4 * (D + 2) <= 8192
    assert sizes[0] < lib.arl2_cache_workspace_bytes(ctypes.byref(cfg), ctypes.byref(config(max_pages=1)))
    assert lib.arl2_cache_least_workspace_bytes(ctypes.byref(cfg), ctypes.byref(config(kv_heads=5))) == 0


def test_set_workspace_of_no_cache(lib):
    assert lib.arl2_cache_set_workspace(None, None, 0, None) == -1
