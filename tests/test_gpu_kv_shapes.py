"""The attention calls at the sizes where they change their way: more requests than one CTA's scan or sort holds,
segments that many warps share, few and many rows in one call, offsets that pass 32 bits, scales that a caller made."""

import numpy as np
import pytest

import kv_reference as ref
import test_gpu_attribute as base
from test_gpu_kv import _cached, _check_rows, _gather, _np, _t, _type

pytestmark = pytest.mark.gpu

lv = base.lv
ctx = base.ctx


def _attend(lv, ctx, rng, lens, new, B, hq, hkv, d, dtype, check, scales_of=None):
    import torch
    lens, new = np.asarray(lens, np.int64), np.asarray(new, np.int64)
    codes, scales, table = _cached(rng, lens, B, hkv, d)
    if scales_of is not None:
        scales = scales_of(scales)
    X = np.concatenate([[0], np.cumsum(new)])
    q = torch.as_tensor(rng.normal(size=(X[-1], hq, d))).to(_type(dtype)).cuda()
    nan = float("nan")  # of a row that is not written
    o, lse = torch.full_like(q, nan), torch.full((int(X[-1]), hq), nan, device="cuda")
    cache = lv.KVCache(*(_t(a, "uint8") for a in codes), *(_t(a, "float32") for a in scales))
    lv.lv_kv_attend(ctx, cache, q, _t(lens - new, "int32"), _t(table, "int32"), o, lse=lse,
                    token_offsets=None if (new == 1).all() else _t(X, "int64"))
    assert ctx.status() == lv.LV_OK
    q64, o64, l64 = _np(q), _np(o), _np(lse)
    assert not np.isnan(o64).any() and not np.isnan(l64).any()
    for i in check:
        n, rows = int(lens[i]), slice(X[i], X[i + 1])
        seen = np.arange(n)[None, :] <= (n - new[i] + np.arange(new[i]))[:, None]
        _check_rows(o64[rows], l64[rows], q64[rows], _gather(codes, scales, table, i, n, B), seen, d ** -0.5, dtype, hq,
                    hkv, f"request {i} of {n}")


@pytest.mark.parametrize("n, B, hq, hkv, d", [(1024, 16, 4, 1, 64), (1025, 32, 2, 2, 64), (2600, 16, 5, 1, 128)])
def test_many_requests(lv, ctx, n, B, hq, hkv, d):
    rng = np.random.default_rng(n)
    lens = np.where(rng.random(n) < 0.02, rng.integers(500, 1500, n), rng.integers(1, 40, n))
    _attend(lv, ctx, rng, lens, np.ones(n), B, hq, hkv, d, "f16", rng.choice(n, 60, replace=False))


@pytest.mark.parametrize("n", [3, 1100])
def test_few_and_many_rows_in_one_call(lv, ctx, n):
    """Single tokens, none, and chunks side by side: each kind has its kernel, and every row is written once."""
    rng = np.random.default_rng(n)
    lens = rng.integers(30, 400, n)
    new = np.where(rng.random(n) < 0.02, 30, rng.integers(0, 4, n))
    new[:3] = 1, 5, 29
    _attend(lv, ctx, rng, lens, new, 16, 4, 1, 64, "bf16", np.concatenate([[0, 1, 2], rng.choice(n, min(n, 50), replace=False)]))


@pytest.mark.parametrize("lens, new, hq, hkv, d, dtype", [
    ([70_001], [1], 8, 1, 128, "bf16"), ([40_000, 17], [1, 1], 16, 1, 64, "f16"), ([9000, 30], [60, 20], 4, 1, 128, "f16"),
    ([33_000], [2], 2, 2, 64, "bf16"), ([20_000], [9], 64, 8, 64, "bf16"),
])
def test_shared_segments(lv, ctx, lens, new, hq, hkv, d, dtype):
    """One long request: every warp or CTA has a share of it, and the parts are joined."""
    rng = np.random.default_rng(sum(lens))
    _attend(lv, ctx, rng, lens, new, 32, hq, hkv, d, dtype, range(len(lens)))


@pytest.mark.parametrize("new", [1, 40])
def test_scales_of_any_size(lv, ctx, new):
    """Scales that no append made: no powers of two, far apart, negative, zero."""
    rng = np.random.default_rng(new)

    def of(s):
        s = np.where(np.isnan(s), s, s * np.exp(6.0 * rng.normal(size=s.shape)))
        s[0] = np.clip(s[0], 0, 0.02)  # keys: scores of a few dozens at most
        s = np.where(rng.random(s.shape) < 0.2, -s, s)
        return np.where(rng.random(s.shape) < 0.1, 0.0, s).astype(np.float32).astype(np.float64)

    _attend(lv, ctx, rng, [500, 333, 40], [new] * 3, 16, 4, 1, 128, "f16", range(3), of)


def test_append_under_a_scale_of_the_callers(lv, ctx):
    """A block held under 0.3: larger values make it a power of two, smaller ones are divided by 0.3."""
    import torch
    rng = np.random.default_rng(3)
    B, d = 16, 64
    codes = rng.integers(0, 127, (2, 2, 1, B, d)).astype(np.uint8)
    scales = np.full((2, 2, 1), np.float32(0.3))
    cache = lv.KVCache(*(_t(a, "uint8") for a in codes), *(_t(a, "float32") for a in scales))
    x = torch.as_tensor(rng.normal(size=(2, 1, d)) * np.array([1.0, 5000.0])[:, None, None]).to(torch.bfloat16).cuda()
    slots = np.array([5, B + 7])
    lv.lv_kv_store(ctx, cache, x, x, _t(slots, "int64"))
    assert ctx.status() == lv.LV_OK
    want, ws = ref.store(ref.E4M3[codes[0]], scales[0].astype(np.float64), _np(x), slots, B)
    assert ws[0, 0] == np.float64(np.float32(0.3)) and ws[1, 0] == 2.0**np.round(np.log2(ws[1, 0])) and ws[1, 0] > 1
    assert np.array_equal(_np(cache.k_scale), ws)
    assert np.array_equal(ref.E4M3[cache.k.cpu().numpy()], want)


@pytest.mark.parametrize("n, most", [(512, 9), (513, 9), (1024, 5), (1500, 6), (300, 300)])
def test_many_prompts(lv, ctx, n, most):
    import torch
    rng = np.random.default_rng(n)
    hq, hkv, d = 4, 2, 64
    lens = rng.integers(0, most + 1, n)
    if most == 300:
        lens[rng.random(n) < 0.9] = 2
    X = np.concatenate([[0], np.cumsum(lens)])
    x = torch.as_tensor(rng.normal(size=(X[-1], hq + 2 * hkv, d))).to(torch.bfloat16).cuda()
    nan = float("nan")
    o, lse = torch.full((int(X[-1]), hq, d), nan, dtype=x.dtype, device="cuda"), torch.full((int(X[-1]), hq), nan, device="cuda")
    lv.lv_prompt_attend(ctx, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], _t(X, "int64"), o, lse=lse)
    assert ctx.status() == lv.LV_OK
    assert not torch.isnan(o).any() and not torch.isnan(lse).any()
    x64, o64, l64 = _np(x), _np(o), _np(lse)
    for i in rng.choice(n, 60, replace=False):
        a, b = X[i], X[i + 1]
        _check_rows(o64[a:b], l64[a:b], x64[a:b, :hq], (x64[a:b, hq:hq + hkv], x64[a:b, hq + hkv:]), np.tri(b - a, dtype=bool),
                    d ** -0.5, "bf16", hq, hkv, f"sequence {i}")


def test_long_prompt(lv, ctx):
    """3,000 tokens: whole blocks of both tiles, the last ones cut; rows all along the sequence."""
    import torch
    rng = np.random.default_rng(4)
    T, hq, hkv, d = 3001, 5, 1, 128
    x = torch.as_tensor(rng.normal(size=(T, hq + 2 * hkv, d))).to(torch.float16).cuda()
    o, lse = torch.empty(T, hq, d, dtype=x.dtype, device="cuda"), torch.empty(T, hq, device="cuda")
    lv.lv_prompt_attend(ctx, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], _t([0, T], "int64"), o, lse=lse)
    assert ctx.status() == lv.LV_OK
    x64, o64, l64 = _np(x), _np(o), _np(lse)
    rows = np.unique(np.concatenate([rng.choice(T, 60, replace=False), [0, 24, 25, 49, 50, 127, 128, 2999, 3000]]))
    seen = np.arange(T)[None, :] <= rows[:, None]
    _check_rows(o64[rows], l64[rows], x64[rows, :hq], (x64[:, hq:hq + hkv], x64[:, hq + hkv:]), seen, d ** -0.5, "f16", hq,
                hkv, "rows")


def test_growing_scores(lv, ctx):
    """Keys whose scores grow block by block, past what the weights absorb, and then fall: outputs are rescaled on the way."""
    import torch
    rng = np.random.default_rng(5)
    T, d = 900, 64
    q = np.abs(rng.normal(size=(T, 1, d))) + 0.5
    up = np.concatenate([np.linspace(-3.0, 3.0, 600), np.linspace(3.0, -3.0, 300)])
    k, v = np.abs(rng.normal(size=(T, 1, d))) * up[:, None, None], rng.normal(size=(T, 1, d))
    q, k, v = (torch.as_tensor(a).to(torch.bfloat16).cuda() for a in (q, k, v))
    o, lse = torch.empty_like(q), torch.empty(T, 1, device="cuda")
    lv.lv_prompt_attend(ctx, q, k, v, _t([0, T], "int64"), o, lse=lse)
    assert ctx.status() == lv.LV_OK
    rows = np.arange(0, T, 13)
    _check_rows(_np(o)[rows], _np(lse)[rows], _np(q)[rows], (_np(k), _np(v)), np.arange(T)[None, :] <= rows[:, None], d ** -0.5,
                "bf16", 1, 1, "rows")


def test_nothing_but_nan(lv, ctx):
    """Values or keys that are all NaN give NaN everywhere, without a walk over every row's keys."""
    import torch
    T, hq, d = 6000, 8, 128
    x = torch.randn(T, hq + 2, d, device="cuda").bfloat16()
    o = torch.zeros(T, hq, d, dtype=x.dtype, device="cuda")
    for at in (hq, hq + 1):
        y = x.clone()
        y[:, at] = float("nan")
        lv.lv_prompt_attend(ctx, y[:, :hq], y[:, hq:hq + 1], y[:, hq + 1:], _t([0, T], "int64"), o)
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        lv.lv_prompt_attend(ctx, y[:, :hq], y[:, hq:hq + 1], y[:, hq + 1:], _t([0, T], "int64"), o)
        end.record()
        assert ctx.status() == lv.LV_OK
        assert torch.isnan(o).all()
        assert begin.elapsed_time(end) < 500.0


def test_values_past_four_gigabytes(lv, ctx):
    """A block whose codes stand beyond 2^32 bytes of the cache."""
    import torch
    B, hkv, d = 128, 8, 128
    n = 2**32 // (hkv * B * d) + 3
    code = torch.zeros((n, hkv, B, d), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((n, hkv), device="cuda")
    cache = lv.KVCache(code, code.clone(), scale, scale.clone())
    rng = np.random.default_rng(6)
    x = torch.as_tensor(rng.normal(size=(40, 2, hkv, d))).to(torch.bfloat16).cuda()
    slots = (n - 1) * B + np.arange(40)
    lv.lv_kv_store(ctx, cache, x[:, 0], x[:, 1], _t(slots, "int64"))
    table = _t([[n - 1]], "int32")
    for new in (1, 40):
        q = torch.as_tensor(rng.normal(size=(new, hkv, d))).to(torch.bfloat16).cuda()
        o, lse = torch.empty_like(q), torch.empty(new, hkv, device="cuda")
        lv.lv_kv_attend(ctx, cache, q, _t([40 - new], "int32"), table, o, lse=lse, token_offsets=_t([0, new], "int64"))
        assert ctx.status() == lv.LV_OK
        K, V = (ref.E4M3[c[n - 1].cpu().numpy()].transpose(1, 0, 2)[:40] * s[n - 1].double().cpu().numpy()[None, :, None]
                for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        seen = np.arange(40)[None, :] <= (40 - new + np.arange(new))[:, None]
        _check_rows(_np(o), _np(lse), _np(q), (K, V), seen, d ** -0.5, "bf16", hkv, hkv, f"{new} new")


def test_a_graph_outlives_larger_calls(lv):
    """A captured call keeps its scratch when later calls of the context need more."""
    import torch
    ctx = lv.Context()
    rng = np.random.default_rng(7)
    lens = np.array([5000, 4000])
    codes, scales, table = _cached(rng, lens, 16, 1, 64)
    cache = lv.KVCache(*(_t(a, "uint8") for a in codes), *(_t(a, "float32") for a in scales))
    q = torch.as_tensor(rng.normal(size=(2, 4, 64))).to(torch.bfloat16).cuda()
    c, tb, o = _t(lens - 1, "int32"), _t(table, "int32"), torch.empty_like(q)
    cs = torch.cuda.Stream()
    with torch.cuda.stream(cs):
        lv.lv_kv_attend(ctx, cache, q, c, tb, o, stream=cs)
    cs.synchronize()
    want = o.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=cs):
        lv.lv_kv_attend(ctx, cache, q, c, tb, o, stream=cs)
    big = torch.randn(4000, 8, 128, device="cuda").bfloat16()
    wide = lv.KVCache.empty(600, 1, 16, 128)
    lv.lv_kv_attend(ctx, wide, big, _t(np.zeros(1), "int32"), _t(np.arange(250)[None, :], "int32"), torch.empty_like(big),
                    token_offsets=_t([0, 4000], "int64"))
    torch.cuda.synchronize()
    o.fill_(9.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, want) and ctx.status() == lv.LV_OK
