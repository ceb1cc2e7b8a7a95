"""The paged 4-bit cache on the GPU: pages bit for bit against the format in fp32, attention against 64 bits, and what is refused."""
import numpy as np
import pytest
import torch

from cache_util import Pool, attend64, hold, rotate, tolerance
from parity_util import Guarded
from paper_2605_16579_b200 import arl2, workload

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}


def make(B, H, kv_heads, D, dtype, page, capacity, rope_rows=0, seed=0, L=1, scale=0.0, spare=2):
    layer = arl2.Layer(B, H, L, D, dtype, device=DEV, softmax_scale=scale)
    pool = Pool(B, kv_heads, D, page, capacity, DEV, seed, spare)
    cos = sin = None
    if rope_rows:
        cos, sin = workload.rope_tables(rope_rows, D)
    cache = arl2.Cache(layer, pool.count, pool.width, kv_heads=kv_heads, page_tokens=page, pages=pool.guard.t, page_table=pool.table,
                       rope_cos=None if cos is None else cos.to(DEV), rope_sin=None if sin is None else sin.to(DEV))
    return layer, cache, pool, cos, sin


def draw(shape, dtype, seed, spread=1.0):
    """Channels with an offset and a size of their own, rounded to the I/O type; also as fp32 on the host."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * (0.5 + rng.random(shape[-2:])) + 0.3 * rng.standard_normal(shape[-2:])
    t = torch.from_numpy((x * spread).astype(np.float32)).to(TORCH[dtype])
    return t.to(DEV), t.float().numpy()


def start_of(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------------ append
APPENDS = [  # B, kv_heads, D, dtype, page, tokens, start, rope
    (1, 1, 64, "fp32", 16, 1, (0,), False),
    (1, 2, 128, "bf16", 16, 1, (15,), True),
    (3, 2, 64, "fp32", 16, 37, (0, 5, 16), True),
    (2, 12, 128, "bf16", 64, 130, (63, 64), True),
    (2, 5, 128, "fp32", 128, 77, (100, 0), True),
    (4, 3, 64, "bf16", 32, 19, (0, -1, 40, 7), True),
    (1, 40, 128, "bf16", 256, 301, (255,), False),
    (2, 12, 128, "bf16", 64, 700, (0, 33), True),
]


@pytest.mark.parametrize("B,kv_heads,D,dtype,page,tokens,start,rope", APPENDS)
def test_append_writes_the_format(B, kv_heads, D, dtype, page, tokens, start, rope):
    top = max(start) + tokens
    layer, cache, pool, cos, sin = make(B, kv_heads, kv_heads, D, dtype, page, top, rope_rows=top if rope else 0)
    before = pool.guard.t.clone()
    (k, kf), (v, vf) = draw((B, tokens, kv_heads, D), dtype, 1), draw((B, tokens, kv_heads, D), dtype, 2)
    held = [Guarded((B, tokens, kv_heads, D), TORCH[dtype], DEV) for _ in range(2)]
    for h in held:
        h.t.fill_(float("nan"))
    got = cache.append(k, v, start_of(start), held=(held[0].t, held[1].t))
    layer.sync_status()
    assert pool.guard.intact() and held[0].intact() and held[1].intact()
    if rope:
        pos = np.clip(np.array(start), 0, None)[:, None] + np.arange(tokens)
        kf = rotate(kf, cos.numpy(), sin.numpy(), pos, np.float32)
    split = pool.split()
    untouched = np.ones((pool.count, page), bool)
    for w, x in enumerate((kf, vf)):
        code, low, step, values = hold(x)
        packed = code[..., 0::2] | (code[..., 1::2] << 4)
        for b in range(B):
            if start[b] < 0:
                assert (got[w][b] == 0).all()
                continue
            t = start[b] + np.arange(tokens)
            pages, slots = pool.order[b, t // page], t % page
            untouched[pages, slots] = False
            assert (split[w][pages, :, slots] == packed[b]).all()
            par = split[2 + w][pages, :, slots]
            assert (par[..., 0] == low[b]).all() and (par[..., 1] == step[b]).all()
            assert torch.equal(got[w][b].float().cpu(), torch.from_numpy(values[b]).to(TORCH[dtype]).float())
            # a value is off by half a step, and by what rounding minimum and step to fp16 adds
            span = step[b].astype(np.float64)[..., None]
            room = span * (0.5 + 15 * 2.0 ** -11 + 1e-5) + np.abs(low[b].astype(np.float64))[..., None] * 2.0 ** -11 + 2.0 ** -24
            x64 = x[b].astype(np.float64).reshape(tokens, kv_heads, -1, 64)
            assert (np.abs(values[b].reshape(x64.shape) - x64) <= room + 15 * 2.0 ** -25).all()
    # nothing but the tokens' places was written
    after = Pool.split(pool)
    pool.guard.t.copy_(before)
    for a, o in zip(after, Pool.split(pool)):
        same = (a.view(np.uint8) == o.view(np.uint8)).reshape(*a.shape[:3], -1).all(-1)
        assert same.transpose(0, 2, 1)[untouched].all()


def test_append_without_held_values_and_over_old_ones():
    layer, cache, pool, cos, sin = make(2, 4, 4, 128, "bf16", 32, 200, rope_rows=200)
    old, _ = draw((2, 90, 4, 128), "bf16", 3)
    assert cache.append(old, old, start_of((10, 20))) is None
    (k, kf), (v, vf) = draw((2, 90, 4, 128), "bf16", 4), draw((2, 90, 4, 128), "bf16", 5)
    cache.append(k, v, start_of((10, 20)))
    layer.sync_status()
    pos = np.array((10, 20))[:, None] + np.arange(90)
    want = hold(rotate(kf, cos.numpy(), sin.numpy(), pos, np.float32))[3], hold(vf)[3]
    for b in range(2):
        have = pool.values(b, pos[b, -1] + 1)
        for w in range(2):
            assert np.array_equal(have[w][:, pos[b]].transpose(1, 0, 2).astype(np.float32), want[w][b])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_of_special_values(dtype):
    """Constant groups, zeros, infinities, huge and tiny values, a NaN: as the formula has them."""
    D = 128
    layer, cache, pool, _, _ = make(1, 1, 1, D, dtype, 16, 16)
    x = np.zeros((1, 9, 1, D), np.float32)
    x[0, 1] = 3.25
    x[0, 2, 0, 5], x[0, 2, 0, 70] = np.inf, -np.inf
    x[0, 3, 0, :64], x[0, 3, 0, 64:] = 1e30, np.linspace(-1e5, 1e5, 64)
    x[0, 4] = np.linspace(0, 1e-7, D)
    x[0, 5, 0, 3] = np.nan
    x[0, 6] = np.linspace(-61440, 61440, D)
    x[0, 7] = np.linspace(1000, 1001, D)
    x[0, 8] = -0.0
    t = torch.from_numpy(x).to(TORCH[dtype])
    got = cache.append(t.to(DEV), t.to(DEV), start_of((0,)), held=True)
    layer.sync_status()
    code, low, step, values = hold(t.float().numpy())
    split = pool.split()
    page = pool.order[0, 0]
    for w in range(2):
        assert (split[w][page, 0, :9] == (code[..., 0::2] | (code[..., 1::2] << 4))[0, :, 0]).all()
        assert np.array_equal(split[2 + w][page, 0, :9], np.stack((low, step), -1)[0, :, 0], equal_nan=True)
        assert np.array_equal(got[w].float().cpu().numpy(), torch.from_numpy(values).to(TORCH[dtype]).float().numpy(), equal_nan=True)
    assert np.isfinite(values[0, 6]).all() and np.isnan(values[0, 5, 0, :64]).all() and np.isfinite(values[0, 5, 0, 64:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_of_strided_and_odd_tensors(dtype):
    """Keys and values as slices of one projection's output, and as tensors that start off any wide boundary."""
    B, T, H, D = 2, 33, 3, 64
    want = None
    (k, _), (v, _) = draw((B, T, H, D), dtype, 6), draw((B, T, H, D), dtype, 7)
    for how in ("plain", "packed", "odd"):
        layer, cache, pool, _, _ = make(B, H, H, D, dtype, 16, 50, rope_rows=64)
        if how == "packed":
            both = torch.empty(B, T, 2, H, D, dtype=TORCH[dtype], device=DEV)
            both[:, :, 0], both[:, :, 1] = k, v
            a, b = both[:, :, 0], both[:, :, 1]
        elif how == "odd":
            a, b = (torch.empty(x.numel() + 1, dtype=x.dtype, device=DEV)[1:].view(x.shape).copy_(x) for x in (k, v))
        else:
            a, b = k, v
        held = cache.append(a, b, start_of((3, 17)), held=True)
        layer.sync_status()
        now = (pool.guard.t.clone(), held[0], held[1])
        if want is None:
            want = now
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(now, want)), how


# ---------------------------------------------------------------------------------------------- attention
ATTENDS = [  # B, H, kv_heads, D, dtype, page, queries, lengths, causal, rope
    (1, 1, 1, 64, "fp32", 16, 1, (1,), False, False),
    (1, 1, 1, 128, "bf16", 16, 1, (1,), False, True),
    (1, 2, 2, 128, "bf16", 16, 1, (500,), False, True),
    (3, 12, 12, 128, "bf16", 64, 1, (0, 17, 1000), False, True),
    (2, 40, 8, 128, "bf16", 32, 1, (333, 64), False, True),
    (2, 5, 1, 64, "bf16", 128, 3, (129, 4000), False, True),
    (2, 12, 4, 128, "bf16", 64, 7, (300, 5), True, True),        # rows of the second stream see nothing
    (1, 2, 2, 64, "fp32", 32, 33, (100,), False, True),
    (2, 2, 2, 64, "fp32", 16, 70, (70, 131), True, True),
    (2, 3, 3, 128, "fp32", 256, 17, (515, 3), True, False),
    (1, 12, 12, 128, "fp32", 64, 1, (2000,), False, True),
    (2, 4, 4, 64, "bf16", 64, 100, (257, 31), True, True),
    (2, 3, 3, 128, "bf16", 64, 20, (1001, 0), False, True),
    (1, 2, 1, 128, "bf16", 128, 129, (385,), False, True),
    (2, 2, 2, 128, "bf16", 16, 300, (300, 777), True, True),
    (1, 4, 4, 128, "bf16", 32, 513, (129,), False, False),       # more queries than keys
    (3, 2, 2, 128, "bf16", 64, 257, (640, 1, 0), False, True),
    (1, 1, 1, 128, "bf16", 64, 64, (20000,), False, True),       # few rows over a long cache
    (1, 8, 1, 128, "bf16", 64, 40, (1500,), True, True),
]


def fill_random(pool, n, seed, spread=1.0):
    rng = np.random.default_rng(seed)
    shape = (pool.B, n, pool.H, pool.D)
    for_head = lambda: rng.standard_normal(shape) * (0.5 + rng.random(shape[-2:])) + 0.3 * rng.standard_normal(shape[-2:])  # noqa: E731
    pool.fill((for_head() * spread).astype(np.float32), (for_head() * spread).astype(np.float32))


def check(got, ref, weight_v, reach, dtype, keys, rows=None):
    got = got.double().cpu().numpy()
    far = np.abs(got - ref)
    room = tolerance(ref, weight_v, reach, dtype, keys)
    assert np.isfinite(got).all()
    worst = (far / room).max()
    assert worst <= 1.0, f"{worst:.3f} times the tolerance, at {np.unravel_index((far / room).argmax(), far.shape)}"


@pytest.mark.parametrize("B,H,kv_heads,D,dtype,page,queries,lengths,causal,rope", ATTENDS)
def test_attend_against_64_bits(B, H, kv_heads, D, dtype, page, queries, lengths, causal, rope):
    top = max(max(lengths), queries)
    layer, cache, pool, cos, sin = make(B, H, kv_heads, D, dtype, page, max(lengths), rope_rows=top if rope else 0)
    for b in range(B):     # (places past a stream's length keep their NaN parameters)
        one = Pool.__new__(Pool)
        one.__dict__ = dict(pool.__dict__, B=1, order=pool.order[b:b + 1])
        if lengths[b]:
            fill_random(one, lengths[b], 10 + b)
    q, qf = draw((B, queries, H, D), dtype, 20)
    out = Guarded((B, queries, H, D), TORCH[dtype], DEV)
    out.t.fill_(float("nan"))
    cache.attend(q, start_of(lengths), causal=causal, out=out.t)
    layer.sync_status()
    assert out.intact() and pool.guard.intact()
    ref = attend64(qf, pool, lengths, None, causal, cos=None if cos is None else cos.numpy(), sin=None if sin is None else sin.numpy())
    check(out.t, *ref, dtype, max(lengths))
    again = cache.attend(q, start_of(lengths), causal=causal)
    assert torch.equal(again.view(torch.uint8), out.t.view(torch.uint8))     # bitwise, and the tickets are back at zero


@pytest.mark.parametrize("dtype,D,queries", [("bf16", 128, 1), ("bf16", 128, 24), ("bf16", 128, 200), ("fp32", 64, 5), ("bf16", 64, 40)])
@pytest.mark.parametrize("spread", [1e-3, 30.0])
def test_attend_sizes_of_values(dtype, D, queries, spread):
    """Small and large keys, values and queries: flat and one-hot softmax."""
    B, H, n = 2, 2, 700
    layer, cache, pool, _, _ = make(B, H, H, D, dtype, 64, n)
    fill_random(pool, n, 30, spread)
    q, qf = draw((B, queries, H, D), dtype, 31, spread)
    out = cache.attend(q, start_of((n, n - 69)))
    layer.sync_status()
    check(out, *attend64(qf, pool, (n, n - 69), None, False), dtype, n)


@pytest.mark.parametrize("dtype,D,queries", [("bf16", 128, 1), ("bf16", 128, 12), ("bf16", 128, 150), ("fp32", 64, 9), ("bf16", 64, 70)])
def test_attend_values_that_are_not_seen(dtype, D, queries):
    """NaN and infinities past a length, and in tokens that causality hides, reach no row that does not see them."""
    B, H, n = 2, 2, 200
    layer, cache, pool, _, _ = make(B, H, H, D, dtype, 64, n)
    rng = np.random.default_rng(40)
    k, v = (rng.standard_normal((B, n, H, D)).astype(np.float32) for _ in range(2))
    k[0, 190:], v[0, 190:] = np.nan, np.nan         # past the length
    v[1, 187, :, 3] = np.nan                        # seen by some rows only
    pool.fill(k, v)
    q, qf = draw((B, queries, H, D), dtype, 41)
    lengths, first = (190, 200), (190 - queries, 187 - queries // 2)
    out = cache.attend(q, start_of(lengths), q_start=start_of(first), causal=True)
    layer.sync_status()
    ref, weight_v, reach = attend64(qf, pool, lengths, first, True)
    got = out.double().cpu().numpy()
    assert np.isfinite(got[0]).all()
    hidden = queries // 2 if queries > 1 else 0     # rows of stream 1 before token 187 is visible
    assert np.isfinite(got[1, :hidden]).all()
    assert np.isnan(got[1, hidden:, :, :64]).all() == (hidden < queries)
    room = tolerance(ref, weight_v, reach, dtype, n)
    fine = np.isfinite(ref)
    assert (np.isfinite(got) == fine).all()
    assert (np.abs(got - ref)[fine] <= room[fine]).all()


@pytest.mark.parametrize("dtype,queries", [("bf16", 1), ("bf16", 40), ("fp32", 3)])
def test_attend_not_finite_queries(dtype, queries):
    """A row of q with an infinity or a NaN is NaN; the others are as without it."""
    layer, cache, pool, _, _ = make(1, 2, 2, 128, dtype, 64, 300)
    fill_random(pool, 300, 50)
    q, _ = draw((1, queries, 2, 128), dtype, 51)
    plain = cache.attend(q, start_of((300,)))
    q[0, 0, 0, 7] = float("inf")
    q[0, queries - 1, 1, 9] = float("nan")
    out = cache.attend(q, start_of((300,)))
    layer.sync_status()
    assert torch.isnan(out[0, 0, 0]).all() and torch.isnan(out[0, queries - 1, 1]).all()
    plain[0, 0, 0] = plain[0, queries - 1, 1] = 0
    out[0, 0, 0] = out[0, queries - 1, 1] = 0
    assert torch.equal(out, plain)


def test_attend_explicit_positions_scale_and_strides():
    layer, cache, pool, cos, sin = make(2, 4, 2, 128, "bf16", 32, 260, rope_rows=400, scale=0.05)
    fill_random(pool, 260, 60)
    wide, _ = draw((2, 11, 3, 4, 128), "bf16", 61)
    q = wide[:, :, 1]
    lengths, first = (260, 200), (300, 10)
    for causal in (False, True):
        out = cache.attend(q, start_of(lengths), q_start=start_of(first), causal=causal)
        layer.sync_status()
        ref = attend64(q.float().cpu().numpy(), pool, lengths, first, causal, scale=0.05, cos=cos.numpy(), sin=sin.numpy())
        check(out, *ref, "bf16", 260)
    odd = torch.empty(q.numel() + 1, dtype=q.dtype, device=DEV)[1:].view(q.shape).copy_(q)
    to = torch.empty(q.numel() + 1, dtype=q.dtype, device=DEV)[1:].view(q.shape)
    assert torch.equal(cache.attend(odd, start_of(lengths), q_start=start_of(first), causal=True, out=to), out)


def test_shared_pages_and_long_offsets():
    """Streams that name the same pages, and pages whose offsets pass 32 bits."""
    H, D, page = 40, 128, 256
    page_bytes = H * page * 144
    count = (1 << 32) // page_bytes + 3
    layer = arl2.Layer(2, H, 1, D, "bf16", device=DEV)
    pages = torch.empty(count, page_bytes, dtype=torch.uint8, device=DEV)
    table = start_of((count - 1, count - 2, count - 1, count - 3)).view(2, 2)
    cache = arl2.Cache(layer, count, 2, page_tokens=page, pages=pages, page_table=table)
    (k, kf), (v, vf) = draw((2, 300, H, D), "bf16", 70), draw((2, 300, H, D), "bf16", 71)
    k[1, :256], v[1, :256] = k[0, :256], v[0, :256]
    held = cache.append(k, v, start_of((0, 0)), held=True)
    q, qf = draw((2, 1, H, D), "bf16", 72)
    out = cache.attend(q, start_of((300, 290)))
    layer.sync_status()
    for b, n in enumerate((300, 290)):
        x, y, z = (t.double() for t in (qf_t(qf[b]), held_row(cache, pages, table, b, n, 0, H, page), held_row(cache, pages, table, b, n, 1, H, page)))
        p = torch.softmax(torch.einsum("ihd,jhd->hij", x, y) * D ** -0.5, -1)
        ref = torch.einsum("hij,jhd->ihd", p, z)
        assert (out[b].double() - ref).abs().max() <= 2.0 ** -6 * ref.abs().max()
        assert (held[0][b, :n].double() - y).abs().max() <= 2.0 ** -8 * y.abs().max()


def qf_t(x):
    return torch.from_numpy(x).to(DEV)


def held_row(cache, pages, table, b, n, which, H, page):
    """Values of stream b's first n tokens read out of the pages with torch: [n, H, 128]."""
    unit = pages[table[b].long()].view(-1, H, page * 144)
    codes = unit[:, :, which * page * 64:(which + 1) * page * 64].reshape(-1, H, page, 64)
    par = unit[:, :, page * 128 + which * page * 8:page * 128 + (which + 1) * page * 8].reshape(-1, H, page, 2, 4).contiguous().view(torch.float16).double()
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).double().unflatten(-1, (2, 64))
    return (par[..., 0:1] + par[..., 1:2] * code).flatten(-2).transpose(1, 2).reshape(-1, H, 128)[:n]


# ------------------------------------------------------------------- appended and read, as it is used
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp32", 64)])
def test_tokens_one_at_a_time_are_the_block_at_once(dtype, D):
    """A block appended whole, and the same tokens appended one by one, leave the same pages and causal outputs."""
    B, H, T = 2, 4, 21
    outs, pages = [], []
    (k, _), (v, _), (q, _) = (draw((B, T, H, D), dtype, s) for s in (80, 81, 82))
    for single in (False, True):
        layer, cache, pool, _, _ = make(B, H, H, D, dtype, 16, 64, rope_rows=64)
        if single:
            rows = []
            for i in range(T):
                cache.append(k[:, i:i + 1], v[:, i:i + 1], start_of((i, i + 9)))
                rows.append(cache.attend(q[:, i:i + 1], start_of((i + 1, i + 10)), q_start=start_of((i, i + 9))))
            outs.append(torch.cat(rows, 1))
        else:
            cache.append(k, v, start_of((0, 9)))
            outs.append(cache.attend(q, start_of((T, T + 9)), q_start=start_of((0, 9)), causal=True))
        layer.sync_status()
        pages.append(pool.guard.t.clone())
    assert torch.equal(pages[0], pages[1])
    # stream 1's first 9 places are NaN in both: its rows are NaN, and stream 0's agree
    assert torch.isnan(outs[0][1]).all() and torch.isnan(outs[1][1]).all()
    far = (outs[0][0].double() - outs[1][0].double()).abs().max() / outs[0][0].double().abs().max()
    assert far <= (2.0 ** -7 if dtype == "bf16" else 1e-5)


def test_captured_calls_follow_the_lengths():
    """A captured append and attention, replayed with other lengths on the device."""
    layer, cache, pool, cos, sin = make(2, 4, 4, 128, "bf16", 16, 400, rope_rows=400)
    fill_random(pool, 400, 90)
    (k, _), (v, _), (q, _) = (draw((2, 1, 4, 128), "bf16", s) for s in (91, 92, 93))
    start, lengths = start_of((0, 0)), start_of((1, 1))
    out = torch.empty_like(q)
    cache.append(k, v, start)
    cache.attend(q, lengths, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.append(k, v, start)
        cache.attend(q, lengths, out=out)
    for at in ((5, 300), (399, 0), (17, 16)):
        start.copy_(torch.tensor(at))
        lengths.copy_(torch.tensor(at) + 1)
        graph.replay()
        got = out.clone()
        assert torch.equal(got, cache.attend(q, lengths))
        ref = attend64(q.float().cpu().numpy(), pool, [a + 1 for a in at], None, False, cos=cos.numpy(), sin=sin.numpy())
        check(got, *ref, "bf16", 400)
    layer.sync_status()


# ----------------------------------------------------------------------------------- errors on the device
def status_of(layer):
    with pytest.raises(arl2.Arl2Error) as e:
        layer.sync_status()
    layer.sync_status()     # (cleared)
    return str(e.value)


@pytest.mark.parametrize("queries", [1, 200])
def test_out_of_range_is_left_out_and_reported(queries):
    layer, cache, pool, cos, sin = make(2, 2, 2, 128, "bf16", 16, 64, rope_rows=50)
    fill_random(pool, 64, 100)
    keep = pool.guard.t.clone()
    k, _ = draw((2, 4, 2, 128), "bf16", 101)
    # past the table
    held = cache.append(k, k, start_of((62, -1)), held=True)
    assert "status -6" in status_of(layer)
    assert (held[0][0, 2:] == 0).all()
    # past the rotary tables: nothing of it is written
    pool.guard.t.copy_(keep)
    cache.append(k, k, start_of((50, 55)))
    assert "rotary" in status_of(layer)
    assert torch.equal(pool.guard.t, keep) and pool.guard.intact()
    # pages that the pool does not have
    table = pool.table.clone()
    pool.table[0, 1], pool.table[1, 0] = pool.count, -5
    cache.append(k, k, start_of((16, 0)))
    assert "page" in status_of(layer)
    assert torch.equal(pool.guard.t, keep) and pool.guard.intact()
    q, qf = draw((2, queries, 2, 128), "bf16", 102)
    first = start_of((1 - queries, 1 - queries))     # (no position past the rotary tables)
    out = cache.attend(q, start_of((48, 16)), q_start=first)
    assert "page" in status_of(layer)
    assert torch.isfinite(out).all() and (out[1] == 0).all()      # stream 1 has nothing that can be seen
    pool.table.copy_(table)
    # a length past the table counts as all there is
    out = cache.attend(q, start_of((64, 1 << 30)), q_start=first)
    assert "length" in status_of(layer)
    full = cache.attend(q, start_of((64, 64)), q_start=first)
    layer.sync_status()
    assert torch.equal(out, full)
    # a position past the rotary tables counts as the last
    out = cache.attend(q, start_of((64, 64)), q_start=start_of((1000, 1000)))
    assert "rotary" in status_of(layer)
    assert torch.isfinite(out).all()
    # none of this stops a commit, which looks at the time-out word
    cache.append(k, k, start_of((62, -1)))
    layer16 = layer
    a = torch.zeros(2, 2, device=DEV)
    kk, _ = draw((2, 1, 2, 128), "bf16", 103)
    layer16.commit(kk, kk, a)
    assert (layer16.get_state().abs().sum(dim=(-1, -2)) > 0).all()
    status_of(layer)


def test_python_refusals():
    layer, cache, pool, cos, sin = make(2, 4, 2, 128, "bf16", 16, 64, rope_rows=64)
    k = torch.zeros(2, 3, 2, 128, dtype=torch.bfloat16, device=DEV)
    q = torch.zeros(2, 3, 4, 128, dtype=torch.bfloat16, device=DEV)
    n = start_of((1, 1))
    launches = layer.launch_count
    for bad in (lambda: cache.append(k.float(), k, n), lambda: cache.append(k, k[:, :2], n), lambda: cache.append(k, k, n.long()),
                lambda: cache.append(k.transpose(1, 2).contiguous().transpose(1, 2), k, n), lambda: cache.append(k.cpu(), k, n),
                lambda: cache.append(k, k, n, held=(k.float(), k)), lambda: cache.append(k, k, n, held=(k, torch.empty_like(k))),
                lambda: cache.attend(q, n[:1]), lambda: cache.attend(k, n), lambda: cache.attend(q, n, out=q),
                lambda: cache.attend(q, n, out=torch.empty_like(k)), lambda: cache.attend(q[:, :0], n), lambda: cache.append(k[:, :0], k[:, :0], n),
                lambda: arl2.Cache(layer, 4, 4, kv_heads=3), lambda: arl2.Cache(layer, 4, 4, page_tokens=48), lambda: arl2.Cache(layer, 0, 4),
                lambda: arl2.Cache(layer, 4, 4, rope_cos=cos.to(DEV)), lambda: arl2.Cache(layer, 4, 4, pages=pool.guard.t[:, 1:])):
        with pytest.raises(arl2.Arl2Error):
            bad()
    assert layer.launch_count == launches
    assert k.abs().sum() == 0
    cache.close()
    with pytest.raises(arl2.Arl2Error):
        cache.attend(q, n)
