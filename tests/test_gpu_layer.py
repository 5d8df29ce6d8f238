"""A step's work for each token on a GPU against its plain forms in 64 bits: products with their epilogue, the gated half,
head norms with rotation, log probabilities; at sizes, strides and values where they can go wrong, and as one run."""

import numpy as np
import pytest

import kv_reference as kvref
import layer_reference as ref
import test_gpu_attribute as base

pytestmark = pytest.mark.gpu

lv = base.lv
ctx = base.ctx
GUARD = 77.0


def _type(dtype):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]


def _np(t):
    import torch
    return t.to(torch.float64).cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _rows(a, dtype, extra=0, lead=0):
    """a [n][d] as a slice of a wider tensor whose other elements are guards: the slice, the whole."""
    import torch
    n, d = a.shape
    whole = torch.full((n + 2, lead + -(-d // 8) * 8 + extra), GUARD, dtype=_type(dtype), device="cuda")
    part = whole[1:n + 1, lead:lead + d]
    part.copy_(torch.as_tensor(a))
    return part, whole


def _vec(a, dtype, lead=1):
    """A vector at an odd place."""
    import torch
    whole = torch.empty(lead + len(a), dtype=_type(dtype), device="cuda")
    whole[lead:].copy_(torch.as_tensor(a))
    return whole[lead:]


def _untouched(whole, n, lead, d):
    """Nothing but rows 1 .. n, elements lead .. lead + d - 1 was written."""
    w = _np(whole).copy()
    w[1:n + 1, lead:lead + d] = GUARD
    assert np.all(w == GUARD)


SIZES = [(1, 1, 1), (1, 8, 8), (2, 3, 5), (3, 17, 5), (16, 64, 128), (17, 100, 129), (15, 4096, 8), (33, 1001, 257),
         (64, 576, 64), (65, 63, 192), (128, 4096, 256), (129, 65, 640), (192, 1280, 1290), (255, 200, 130), (257, 72, 384),
         (300, 1280, 1000), (1, 5120, 3584), (700, 520, 1111), (1023, 2048, 320), (2100, 128, 384), (5, 10000, 40),
         (4097, 16, 24), (600, 4096, 2560)]


def _linear_case(rng, n, d_in, d_out, whole=False):
    """Inputs that the 16-bit types hold; whole: small whole numbers, whose sums fp32 holds exactly."""
    if whole:
        return tuple(rng.integers(-3, 4, s).astype(float) for s in ((n, d_in), (d_out, d_in), (d_out, d_in), d_out, d_out,
                                                                     (n, d_out)))
    return (rng.normal(size=(n, d_in)), rng.normal(size=(d_out, d_in)) * d_in**-0.5,
            rng.normal(size=(d_out, d_in)) * d_in**-0.5, rng.normal(size=d_out), rng.normal(size=d_out),
            rng.normal(size=(n, d_out)) * 2)


def _held(a, dtype):
    import torch
    return torch.as_tensor(a).to(_type(dtype)).double().numpy()


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("form", ["plain", "bias", "residual", "all", "in_place"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_linear(lv, ctx, size, form, dtype):
    import torch
    n, d_in, d_out = size
    rng = np.random.default_rng([n, d_in, d_out, len(form)])
    act = {"plain": "none", "bias": "silu", "residual": "none", "all": "gelu", "in_place": "relu"}[form]
    x, w, _, b, _, r = (_held(a, dtype) for a in _linear_case(rng, n, d_in, d_out))
    b = b if form in ("bias", "all") else None
    r = r if form in ("residual", "all", "in_place") else None
    want, tol = ref.linear(x, w, b, act, r, dtype)
    dx, dw = _rows(x, dtype, 8, 16)[0], _rows(w, dtype, 24)[0]
    dr = _rows(r, dtype, 16)[0] if r is not None else None
    y, whole = _rows(r if form == "in_place" else np.zeros((n, d_out)), dtype, 8, 8)
    lv.lv_linear(ctx, dx, dw, y, bias=None if b is None else _vec(b, dtype), act=act,
                 residual=y if form == "in_place" else dr)
    assert ctx.status() == lv.LV_OK
    kvref.close(_np(y), want, tol, "y")
    _untouched(whole, n, 8, d_out)
    torch.cuda.synchronize()


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("act, bias", [("silu", False), ("gelu_tanh", True), ("gelu", False), ("relu", True), ("none", True)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_gated(lv, ctx, size, act, bias, dtype):
    n, d_in, d_out = size
    rng = np.random.default_rng([n, d_in, d_out, len(act)])
    x, wg, wu, bg, bu, _ = (_held(a, dtype) for a in _linear_case(rng, n, d_in, d_out))
    if not bias:
        bg = bu = None
    want, tol = ref.gated(x, wg, wu, bg, bu, act, dtype)
    y, whole = _rows(np.zeros((n, d_out)), dtype, 8, 8)
    # the gate's weights after the other ones, in one tensor, as halves of it
    both = _rows(np.concatenate([wu, wg]), dtype, 8)[0]
    lv.lv_gated_linear(ctx, _rows(x, dtype)[0], both[d_out:], both[:d_out], y, bias_gate=None if bg is None else _vec(bg, dtype),
                       bias_up=None if bu is None else _vec(bu, dtype, 3), act=act)
    assert ctx.status() == lv.LV_OK
    kvref.close(_np(y), want, tol, "y")
    _untouched(whole, n, 8, d_out)


@pytest.mark.parametrize("size", SIZES + [(8200, 192, 520), (2050, 1024, 1100)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_products_of_whole_numbers(lv, ctx, size, dtype):
    """Sums that fp32 holds exactly, in whatever order: the outputs are the exact values rounded once, bit for bit."""
    import torch
    n, d_in, d_out = size
    rng = np.random.default_rng([n, d_in, d_out])
    x, wg, wu, bg, bu, r = _linear_case(rng, n, d_in, d_out, True)
    dx, dg, du, dr = (_rows(a, dtype)[0] for a in (x, wg, wu, r))
    y, whole = _rows(np.zeros((n, d_out)), dtype)
    lv.lv_linear(ctx, dx, dg, y, bias=_vec(bg, dtype), residual=dr)
    want = torch.as_tensor(np.float32(x @ wg.T + bg + r)).to(_type(dtype))
    assert torch.equal(y.cpu(), want)
    _untouched(whole, n, 0, d_out)
    lv.lv_gated_linear(ctx, dx, dg, du, y, bias_gate=_vec(bg, dtype), bias_up=_vec(bu, dtype), act="relu")
    product = np.maximum(x @ wg.T + bg, 0) * (x @ wu.T + bu)
    keep = np.abs(product) < 2**24
    assert torch.equal(y.cpu()[torch.as_tensor(keep)], torch.as_tensor(np.float32(product)).to(_type(dtype))[torch.as_tensor(keep)])
    _untouched(whole, n, 0, d_out)
    assert ctx.status() == lv.LV_OK


@pytest.mark.parametrize("n", [1, 20, 300, 1500])
def test_products_keep_a_nan_to_its_row(lv, ctx, n):
    """A NaN or infinity in a token reaches its outputs alone, one in a weight its output's alone; values past a row's
    width reach nothing."""
    import torch
    rng = np.random.default_rng(n)
    d_in, d_out = 333, 260
    x, w, _, _, _, _ = _linear_case(rng, n, d_in, d_out, True)
    t, o = n // 2, 199
    x[t, 300] = np.nan
    w[o, 7] = np.inf
    dx, wx = _rows(x, "bf16")
    dw, ww = _rows(w, "bf16")
    wx[:, d_in:] = float("nan")
    ww[:, d_in:] = float("nan")
    y, _ = _rows(np.zeros((n, d_out)), "bf16")
    with np.errstate(invalid="ignore"):
        want = x @ w.T
    for call in (lambda: lv.lv_linear(ctx, dx, dw, y), lambda: lv.lv_gated_linear(ctx, dx, dw, dw, y, act="none")):
        call()
        got = _np(y)
        other = np.isfinite(want)
        assert np.array_equal(np.isfinite(got), other)
        assert np.isnan(got[t]).all()
        keep = np.delete(np.arange(n), t)
        assert np.array_equal(np.isnan(got[keep, o]), x[keep, 7] == 0)
    assert np.array_equal(got[other], torch.as_tensor(np.float32(want * want)).bfloat16().double().numpy()[other])


def test_products_of_large_values(lv, ctx):
    """What leaves fp16's range is infinite, the activations stay finite far out, and sums are not cut to 16 bits."""
    import torch
    x = torch.full((2, 512), 16.0, dtype=torch.float16, device="cuda")
    x[1] *= -1
    w = torch.full((8, 512), 16.0, dtype=torch.float16, device="cuda")
    y = torch.zeros(2, 8, dtype=torch.float16, device="cuda")
    lv.lv_linear(ctx, x, w, y)
    assert torch.isposinf(y[0]).all() and torch.isneginf(y[1]).all()
    lv.lv_linear(ctx, x, w, y, residual=torch.tensor([[-65504.0], [65504.0]], device="cuda").half().expand(2, 8).contiguous())
    assert torch.equal(y, torch.tensor([[65568.0], [-65568.0]], device="cuda").half().expand(2, 8))
    for act in ("silu", "gelu", "gelu_tanh", "relu"):
        lv.lv_linear(ctx, x, w, y, act=act)
        assert torch.isposinf(y[0]).all() and (y[1] == 0).all()
    assert ctx.status() == lv.LV_OK


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_activations_far_to_the_left(lv, ctx, act):
    """Where the activation is small it keeps its size: within 2^-7 of itself down to the least normal number (an output's
    half step 2^-8, and 2^-13 for an exponential of an argument of at most 90 that is rounded to 2^-23 of itself, six
    times)."""
    x = _held(-np.concatenate([np.linspace(0.01, 14, 200), np.linspace(14, 95, 200)]), "bf16")[:, None]
    y, _ = _rows(np.zeros((len(x), 1)), "bf16")
    lv.lv_linear(ctx, _rows(x, "bf16")[0], _rows(np.ones((1, 1)), "bf16")[0], y, act=act)
    want, got = ref.act(x, act), _np(y)
    normal = np.abs(want) > 2.0**-126
    assert np.all(np.abs(got - want)[normal] <= 2.0**-7 * np.abs(want)[normal])
    assert np.all(np.abs(got)[~normal] <= 2.0**-125)


# ------------------------------------------------------------------ rotation

LAYOUTS = [(32, 8, 128), (20, 4, 128), (10, 2, 128), (12, 12, 64), (16, 1, 64), (8, 1, 128), (1, 1, 64), (3, 3, 128),
           (64, 1, 64)]


def _rotate(lv, ctx, dtype, layout, offsets, c, n, dim, order, norm, eps=1e-6, base=1e4, seed=0, in_place=False, values=None):
    import torch
    hq, hkv, d = layout
    rng = np.random.default_rng([seed, hq, n, dim])
    heads = hq + 2 * hkv
    qkv = rng.normal(size=(n, heads, d)) * np.exp(rng.normal(size=(n, heads, 1))) if values is None else values(rng, n, heads, d)
    qkv = _held(qkv, dtype)
    wq, wk = (_held(np.exp(0.3 * rng.normal(size=d)), dtype) for _ in range(2))
    freq = [base ** (-2.0 * j / dim) for j in range(dim // 2)]
    if dim:
        freq[-1] = -freq[-1]
    whole = torch.as_tensor(qkv).to(_type(dtype)).cuda()
    q, k = whole[:, :hq], whole[:, hq:hq + hkv]
    if in_place:
        qo, ko = q, k
    else:
        out = torch.full((n, heads, d), GUARD, dtype=_type(dtype), device="cuda")
        qo, ko = out[:, hkv:hkv + hq], out[:, hkv + hq:]
    i64, i32 = (lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int64, device="cuda"),
                lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int32, device="cuda"))
    lv.lv_qk_rotate(ctx, q, k, qo, ko, lv.Rope(freq, order == "neighbours"), c=None if c is None else i32(c),
                    token_offsets=None if offsets is None else i64(offsets),
                    q_weight=_vec(wq, dtype) if norm else None, k_weight=_vec(wk, dtype, 3) if norm else None, eps=eps)
    at = np.arange(n + 1) if offsets is None else np.asarray(offsets)
    pos = ref.positions(n, at, c)
    seen = pos >= 0
    for got, x, w, name in ((qo, qkv[:, :hq], wq, "q"), (ko, qkv[:, hq:hq + hkv], wk, "k")):
        want, tol = ref.rotate(x, w if norm else None, eps, np.maximum(pos, 0), freq, order == "neighbours", dtype)
        got = _np(got)
        kvref.close(got[seen], want[seen], tol[seen], name)
        assert np.array_equal(got[~seen], x[~seen] if in_place else np.full_like(got[~seen], GUARD)), name
    if in_place:
        assert np.array_equal(_np(whole[:, hq + hkv:]), qkv[:, hq + hkv:])
    else:
        assert np.all(_np(out[:, :hkv]) == GUARD)


@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("order", ["halves", "neighbours"])
@pytest.mark.parametrize("part", [1, 2, 0, -1])
@pytest.mark.parametrize("norm", [True, False])
def test_rotate_decode(lv, ctx, layout, order, part, norm):
    d = layout[2]
    dim = {1: d, 2: d // 2, 0: 0, -1: 16}[part]
    rng = np.random.default_rng(d)
    for n in (1, 7, 130):
        c = np.minimum(np.exp(rng.normal(8, 2, n)).astype(int), 2**20)
        _rotate(lv, ctx, "bf16" if norm else "f16", layout, None, c, n, dim, order, norm, base=5e5, in_place=n == 7)
    assert ctx.status() == lv.LV_OK


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("offsets, c, n", [
    ([0, 5], None, 5), ([0, 1, 1, 4, 4, 300], None, 300), ([0, 3, 3, 40], [5, 0, 1000], 40), ([2, 9, 30], [0, 7], 33),
    ([0, 0, 0], [1, 2], 4), ([0, 2049], None, 2049), ([0, 1], [2**31 - 1], 1),
], ids=str)
def test_rotate_requests(lv, ctx, dtype, offsets, c, n):
    """Positions from offsets and contexts; tokens before the first request and behind the last stay as they were."""
    for layout in ((20, 4, 128), (16, 1, 64)):
        for in_place in (False, True):
            _rotate(lv, ctx, dtype, layout, offsets, c, n, layout[2], "halves", True, in_place=in_place)
    assert ctx.status() == lv.LV_OK


def test_rotate_many_requests(lv, ctx):
    rng = np.random.default_rng(4)
    p = rng.integers(0, 4, 3000)
    at = np.concatenate([[0], np.cumsum(p)])
    _rotate(lv, ctx, "bf16", (8, 1, 128), at, rng.integers(0, 100_000, 3000), int(at[-1]) + 3, 128, "halves", True)
    assert ctx.status() == lv.LV_OK


@pytest.mark.parametrize("dtype, size", [("bf16", 1e30), ("bf16", 1e-30), ("bf16", 3e38), ("bf16", 1e-39), ("f16", 6e4),
                                         ("f16", 1e-7), ("bf16", 0.0)])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-30])
def test_norm_of_far_values(lv, ctx, dtype, size, eps):
    """Squares beyond fp32's range on either side, zeros, and eps that counts or does not."""
    if size == 0.0 and eps == 0.0:
        eps = 1e-38
    _rotate(lv, ctx, dtype, (4, 2, 64), None, [0, 3, 9], 3, 64, "halves", True, eps=eps,
            values=lambda rng, n, h, d: rng.uniform(0.3, 0.9, (n, h, d)) * rng.choice([-1, 1], (n, h, d)) * size)
    assert ctx.status() == lv.LV_OK


def test_rotate_keeps_a_nan_to_its_head(lv, ctx):
    def values(rng, n, h, d):
        v = rng.normal(size=(n, h, d))
        v[1, 2, 5] = np.nan
        v[2, 0, 0] = np.inf
        return v
    import torch
    n, hq, hkv, d = 4, 4, 2, 64
    x = torch.as_tensor(values(np.random.default_rng(1), n, hq + hkv, d)).bfloat16().cuda()
    y = torch.zeros_like(x)
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    lv.lv_qk_rotate(ctx, x[:, :hq], x[:, hq:], y[:, :hq], y[:, hq:], lv.Rope.geometric(d), c=torch.zeros(n, dtype=torch.int32,
                    device="cuda"), q_weight=w, k_weight=w)
    bad = ~torch.isfinite(y).all(2).cpu()
    assert bad.nonzero().tolist() == [[1, 2], [2, 0]] and torch.isnan(y[1, 2]).all()
    assert torch.isnan(y[2, 0, [0, 32]]).all() and (y[2, 0, 1:32] == 0).all()  # a finite value over infinity


@pytest.mark.parametrize("order", ["halves", "neighbours"])
def test_rotate_leaves_the_rest_of_a_head(lv, ctx, order):
    """Elements past the rotated ones are scaled alone: an infinite weight or value there is an infinity, not a NaN."""
    import torch
    d = 64
    x = torch.ones(2, 2, d, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    w[40] = float("inf")
    y = torch.zeros_like(x)
    rope, c = lv.Rope.geometric(16, neighbours=order == "neighbours"), torch.tensor([3, 4], dtype=torch.int32, device="cuda")
    lv.lv_qk_rotate(ctx, x[:, :1], x[:, 1:], y[:, :1], y[:, 1:], rope, c=c, q_weight=w, k_weight=w)
    assert torch.isposinf(y[..., 40]).all() and torch.isfinite(y).sum() == 4 * (d - 1)
    x[0, 0, 50] = float("-inf")
    lv.lv_qk_rotate(ctx, x[:, :1], x[:, 1:], y[:, :1], y[:, 1:], rope, c=c)
    assert torch.isneginf(y[0, 0, 50]) and torch.isfinite(y).sum() == 4 * d - 1
    assert ctx.status() == lv.LV_OK


def test_rotate_bad_data(lv, ctx):
    """A negative context counts as none; offsets that decrease or leave the call are said."""
    import torch
    n, d = 6, 64
    x = torch.randn(n, 3, d, device="cuda").bfloat16()
    rope = lv.Rope.geometric(d)

    def call(offsets, c):
        y = torch.full_like(x, GUARD)
        lv.lv_qk_rotate(ctx, x[:, :2], x[:, 2:], y[:, :2], y[:, 2:], rope,
                        c=torch.tensor(c, dtype=torch.int32, device="cuda"),
                        token_offsets=torch.tensor(offsets, device="cuda") if offsets else None)
        return y, ctx.status()

    good, st = call([0, 2, 6], [0, 5])
    assert st == lv.LV_OK
    y, st = call([0, 2, 6], [-1, 5])
    assert st == lv.LV_EDATA and torch.equal(y, good)
    for offsets in ([0, 4, 2, 6], [0, 9, 6], [-3, 2, 6], [0, 2, 7], [5, 1, 0]):
        assert call(offsets, [0] * (len(offsets) - 1))[1] == lv.LV_EDATA
    assert call(None, [3, 4, 5, -2**31, 0, 0])[1] == lv.LV_EDATA
    assert call(None, [3, 4, 5, 2**31 - 1, 0, 0])[1] == lv.LV_OK


# ------------------------------------------------------------------ log probabilities

def _lp_close(lv, ctx, x, ids, n_top, dtype, lead=0, extra=0):
    import torch
    n, V = x.shape
    x = _held(x, dtype) if dtype != "f32" else np.float32(x).astype(np.float64)
    whole = torch.full((n, lead + V + extra), float("nan"), dtype=_type(dtype), device="cuda")
    dx = whole[:, lead:lead + V]
    dx.copy_(torch.as_tensor(x))
    logp, ent, lse = (torch.full((n,), GUARD, device="cuda") for _ in range(3))
    top = dict(top_ids=torch.full((n, n_top), -7, dtype=torch.int32, device="cuda"),
               top_logp=torch.full((n, n_top), GUARD, device="cuda")) if n_top else {}
    lv.lv_token_logprobs(ctx, dx, ids=torch.as_tensor(ids, dtype=torch.int32, device="cuda"), logp=logp, entropy=ent, lse=lse,
                         **top)
    want = ref.logprobs(x, ids, n_top)
    # Sums of V terms by at least 128 threads, each term's exponential good to 2^-20 where it counts (an argument rounded
    # to 2^-24 of at most 17 nats on average, the function 2^-22); differences and the last sum rounded to 2^-24.
    with np.errstate(invalid="ignore"):
        top_x = np.nanmax(np.where(np.isfinite(x), x, -np.inf), axis=1)
        top_x = np.where(np.isfinite(top_x), top_x, 0)
        ds = (V / 128 + 64) * 2.0**-24 + 2.0**-18
        kvref.close(_np(lse), want[2], np.where(np.isfinite(want[2]), ds + 2.0**-22 * (np.abs(want[2]) + np.abs(top_x)), 0), "lse")
        kvref.close(_np(ent), want[1], 2 * ds * (2 + np.abs(want[1])) + 2.0**-22 * np.log(V + 1), "entropy")
        kvref.close(_np(logp), want[0], ds + 2.0**-22 * np.abs(want[0]), "logp")
    if n_top:
        assert np.array_equal(_np(top["top_ids"]), want[3])
        kvref.close(_np(top["top_logp"]), want[4], ds + 2.0**-22 * np.abs(want[4]), "top_logp")
    return logp, ent, lse, top


@pytest.mark.parametrize("n, V, n_top", [(1, 1, 0), (1, 1, 3), (3, 7, 7), (2, 31, 32), (5, 33, 32), (1, 100, 1), (4, 1000, 20),
                                         (300, 257, 2), (1, 50257, 20), (2, 128_000, 32), (37, 4097, 5), (9, 8192, 32),
                                         (1, 262_144, 20), (1200, 640, 1), (16, 32_000, 0), (3, 100_003, 8)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_logprobs(lv, ctx, n, V, n_top, dtype):
    rng = np.random.default_rng([n, V, n_top])
    x = rng.normal(size=(n, V)) * 3
    ids = np.where(rng.random(n) < 0.5, x.argmax(1), rng.integers(0, V, n))
    _lp_close(lv, ctx, x, ids, n_top, dtype, lead=int(rng.integers(0, 9)), extra=int(rng.integers(0, 5)))
    assert ctx.status() == lv.LV_OK


@pytest.mark.parametrize("law", ["equal", "rising", "falling", "two_values", "one_hot", "zeros", "first_lanes", "strided", "last"])
@pytest.mark.parametrize("V", [40, 1000, 20_011])
def test_logprobs_orders(lv, ctx, law, V):
    """Ties, and the largest where a way of looking for them could miss some or drown in them."""
    v = np.arange(V, dtype=float)
    x = {"equal": np.full(V, 2.5), "rising": v / V * 8, "falling": -v / V * 8, "two_values": np.where(v % 3 == 1, 1.0, -1.0),
         "one_hot": np.where(v == V - 1, 90.0, 0.0), "zeros": np.where(v % 2 == 0, -0.0, 0.0),
         "first_lanes": np.where(v < 64, 10 + v / 64, v / V), "strided": np.where(v % 8 == 3, 5 + v / V, -5),
         "last": np.where(v >= V - 33, 4 + (V - v) / 64, 0)}[law]
    x = np.stack([x, x[::-1], np.roll(x, V // 3)])
    for dtype in ("bf16", "f32"):
        for n_top in (1, 32):
            _lp_close(lv, ctx, x, np.array([0, V - 1, V // 2]), n_top, dtype)
    assert ctx.status() == lv.LV_OK


@pytest.mark.parametrize("n, V, every, first", [(320, 128_000, 256, 8), (2450, 100_000, 128, 4)])
def test_logprobs_with_the_largest_in_one_place(lv, ctx, n, V, every, first):
    """The largest logits of a row all where a few threads read, thousands of them: more candidates than there is room for."""
    import torch
    x = torch.randn(n, V, device="cuda").bfloat16()
    piece = torch.arange(V, device="cuda") // 8 % every
    x = torch.where(piece < first, x + 20, x)
    ids, lp = torch.empty(n, 32, dtype=torch.int32, device="cuda"), torch.empty(n, 32, device="cuda")
    lv.lv_token_logprobs(ctx, x, top_ids=ids, top_logp=lp)
    for a in range(0, n, 400):
        part = x[a:a + 400].float()
        v, i = torch.sort(part, dim=1, descending=True, stable=True)
        assert torch.equal(ids[a:a + 400], i[:, :32].int())
        want = v[:, :32].double() - torch.logsumexp(part.double(), 1, keepdim=True)
        assert (lp[a:a + 400].double() - want).abs().max() < 1e-4
    assert ctx.status() == lv.LV_OK


@pytest.mark.parametrize("V", [5, 3000, 70_001])
def test_logprobs_masks(lv, ctx, V):
    """Masked logits (-inf, the type's lowest value), rows that a mask leaves empty, infinities and NaNs."""
    rng = np.random.default_rng(V)
    low = {"bf16": -3.3895313892515355e38, "f16": -65504.0, "f32": -3.4028234663852886e38}
    for dtype in ("bf16", "f16", "f32"):
        x = rng.normal(size=(9, V))
        x[0, 1:] = -np.inf
        x[1] = -np.inf
        x[2, 2:] = low[dtype]
        x[3] = low[dtype]
        x[4, [1, V - 1]] = np.inf
        x[5, V // 2] = np.nan
        x[6, 0], x[6, V - 1] = np.nan, np.inf
        x[7, rng.random(V) < 0.9] = -np.inf
        x[8] = -low[dtype]
        x[8, 1] = low[dtype]
        for n_top in (0, 4, 32):
            _lp_close(lv, ctx, x, np.full(9, 1), n_top, dtype)
    assert ctx.status() == lv.LV_OK


def test_logprobs_far_above_many(lv, ctx):
    """One logit of 1e31 above 2^24 others, whose sum times that distance is beyond fp32: all of the probability is its."""
    import torch
    x = torch.full((1, 1 << 24), 7.9, device="cuda")
    x.view(8, -1)[:, :4096] = 0.0  # what each of eight shares of the row begins with, and its sums are relative to
    x[0, 9_000_000] = 1e31
    lse, ent, lp = (torch.full((1,), GUARD, device="cuda") for _ in range(3))
    ids, top = torch.zeros(1, 2, dtype=torch.int32, device="cuda"), torch.zeros(1, 2, device="cuda")
    lv.lv_token_logprobs(ctx, x, ids=torch.tensor([9_000_000], dtype=torch.int32, device="cuda"), logp=lp, entropy=ent, lse=lse,
                         top_ids=ids, top_logp=top)
    assert lse.item() == float(np.float32(1e31)) and ent.item() == 0 and lp.item() == 0
    assert ids.tolist() == [[9_000_000, 4096]] and top[0, 0] == 0 and top[0, 1] == float(np.float32(7.9) - np.float32(1e31))
    assert ctx.status() == lv.LV_OK


def test_logprobs_ids_and_what_is_left_out(lv, ctx):
    import torch
    x = torch.randn(4, 50, device="cuda")
    lp = torch.full((4,), GUARD, device="cuda")
    lv.lv_token_logprobs(ctx, x, ids=torch.tensor([0, -1, 49, -1], dtype=torch.int32, device="cuda"), logp=lp)
    assert ctx.status() == lv.LV_OK and torch.isnan(lp).tolist() == [False, True, False, True]
    for bad in (50, -2, 2**31 - 1, -2**31):
        lv.lv_token_logprobs(ctx, x, ids=torch.tensor([0, 1, bad, 3], dtype=torch.int32, device="cuda"), logp=lp)
        assert ctx.status() == lv.LV_EDATA and torch.isnan(lp).tolist() == [False, False, True, False]
    lse = torch.full((4,), GUARD, device="cuda")
    lv.lv_token_logprobs(ctx, x, lse=lse)
    assert torch.allclose(lse, torch.logsumexp(x, 1), atol=1e-5)
    lv.lv_token_logprobs(ctx, x)


# ------------------------------------------------------------------ arrays of more than 2^31 elements

def test_products_past_32_bits(lv, ctx):
    import torch
    n, d_in, d_out = 300_001, 64, 8192
    x = torch.randint(-3, 4, (n, d_in), device="cuda").bfloat16()
    w = torch.randint(-3, 4, (d_out, d_in), device="cuda").bfloat16()
    y = torch.empty(n, d_out, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 1, 262_143, 262_144, 270_000, n - 2, n - 1], device="cuda")
    want = x[rows].double() @ w.double().t()
    lv.lv_linear(ctx, x, w, y)
    assert torch.equal(y[rows], want.bfloat16())
    lv.lv_linear(ctx, x, w, y, residual=y)
    assert torch.equal(y[rows], (want + want.bfloat16().double()).bfloat16())
    lv.lv_gated_linear(ctx, x, w, w, y, act="none")
    assert torch.equal(y[rows], (want * want).bfloat16())
    assert ctx.status() == lv.LV_OK


def test_rotate_past_32_bits(lv, ctx):
    import torch
    n, hq, hkv, d = 620_003, 20, 4, 128
    qkv = torch.empty(n, hq + 2 * hkv, d, dtype=torch.bfloat16, device="cuda").normal_()
    rows = [0, 599_186, 599_187, n - 1]
    before = _np(qkv[rows])
    rope = lv.Rope.geometric(d, 1e6)
    w = torch.full((d,), 1.5, dtype=torch.bfloat16, device="cuda")
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    lv.lv_qk_rotate(ctx, q, k, q, k, rope, token_offsets=torch.tensor([0, n], device="cuda"), q_weight=w, k_weight=w)
    after = _np(qkv[rows])
    want, tol = ref.rotate(before[:, :hq + hkv], np.full(d, 1.5), 1e-6, np.array(rows), list(rope.s.freq), False, "bf16")
    kvref.close(after[:, :hq + hkv], want, tol, "q and k")
    assert np.array_equal(after[:, hq + hkv:], before[:, hq + hkv:]) and ctx.status() == lv.LV_OK


def test_logprobs_past_32_bits(lv, ctx):
    import torch
    n, V = 40_001, 64_000
    x = torch.empty(n, V, dtype=torch.bfloat16, device="cuda").normal_()
    ids = torch.randint(0, V, (n,), device="cuda").int()
    logp, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    top, tlp = torch.empty(n, 2, dtype=torch.int32, device="cuda"), torch.empty(n, 2, device="cuda")
    lv.lv_token_logprobs(ctx, x, ids=ids, logp=logp, lse=lse, top_ids=top, top_logp=tlp)
    rows = [0, 33_554, 33_555, n - 1]
    want = ref.logprobs(_np(x[rows]), ids[rows].tolist(), 2)
    assert np.array_equal(_np(top[rows]), want[3])
    for got, w in ((logp, want[0]), (lse, want[2]), (tlp, want[4])):
        kvref.close(_np(got[rows]), w, 1e-4, "rows")
    assert ctx.status() == lv.LV_OK


# ------------------------------------------------------------------ together

def _layer(lv, ctx, s):
    """One layer's step without its attention norms: projection, head norms and rotation, append, attention, output projection
    onto the residual stream, gated block onto it, logits, log probabilities."""
    hq, hkv, d = s["layout"]
    n = s["h"].shape[0]
    lv.lv_linear(ctx, s["h"], s["w_qkv"], s["qkv"].view(n, -1), bias=s["b_qkv"])
    q, k, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]
    lv.lv_qk_rotate(ctx, q, k, q, k, s["rope"], token_offsets=s["offsets"], q_weight=s["w_q"], k_weight=s["w_k"])
    lv.lv_kv_plan(ctx, s["p"], s["c"], 16, s["free"], s["table"], s["offsets_out"], s["slots"], s["counts"])
    lv.lv_kv_store(ctx, s["cache"], k, v, s["slots"])
    lv.lv_prompt_attend(ctx, q, k, v, s["offsets"], s["o"])
    lv.lv_linear(ctx, s["o"].view(n, -1), s["w_o"], s["h2"], residual=s["h"])
    lv.lv_gated_linear(ctx, s["h2"], s["w_gate"], s["w_up"], s["mid"])
    lv.lv_linear(ctx, s["mid"], s["w_down"], s["h2"], residual=s["h2"])
    lv.lv_linear(ctx, s["h2"], s["w_vocab"], s["logits"])
    lv.lv_token_logprobs(ctx, s["logits"], ids=s["ids"], logp=s["logp"], entropy=s["ent"], top_ids=s["top_ids"],
                         top_logp=s["top_logp"])


def _layer_state(lv, p, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv, d, dm, ff, V = 4, 2, 64, 320, 456, 1003
    n, t = int(sum(p)), torch.bfloat16

    def r(*shape, by=1.0):
        return (torch.randn(*shape, device="cuda", generator=g) * by).to(t)

    def e(*shape, dt=t):
        return torch.full(shape, 0, dtype=dt, device="cuda")

    at = np.concatenate([[0], np.cumsum(p)])
    nb = int(sum(-(-x // 16) for x in p))
    logits = torch.full((n, 1008), float("nan"), dtype=t, device="cuda")
    return dict(layout=(hq, hkv, d), h=r(n, dm), w_qkv=r((hq + 2 * hkv) * d, dm, by=dm**-0.5), b_qkv=r((hq + 2 * hkv) * d),
                qkv=e(n, hq + 2 * hkv, d), rope=lv.Rope.geometric(d), offsets=torch.as_tensor(at, device="cuda"),
                w_q=r(d, by=0.2) + 1, w_k=r(d, by=0.2) + 1, p=torch.as_tensor(p, dtype=torch.int32, device="cuda"),
                c=e(len(p), dt=torch.int32), free=torch.arange(nb, dtype=torch.int32, device="cuda"),
                table=torch.full((len(p), 20), -1, dtype=torch.int32, device="cuda"),
                offsets_out=e(len(p) + 1, dt=torch.int64), slots=e(n, dt=torch.int64), counts=e(2, dt=torch.int64),
                cache=lv.KVCache.empty(nb, hkv, 16, d), o=e(n, hq, d), w_o=r(dm, hq * d, by=(hq * d)**-0.5), h2=e(n, dm),
                w_gate=r(ff, dm, by=dm**-0.5), w_up=r(ff, dm, by=dm**-0.5), mid=e(n, ff), w_down=r(dm, ff, by=ff**-0.5),
                w_vocab=r(V, dm, by=dm**-0.5), logits=logits[:, :V], ids=torch.randint(0, V, (n,), device="cuda", generator=g).int(),
                logp=e(n, dt=torch.float32), ent=e(n, dt=torch.float32), top_ids=e(n, 3, dt=torch.int32),
                top_logp=e(n, 3, dt=torch.float32))


OUTPUTS = ("qkv", "o", "h2", "mid", "logits", "logp", "ent", "top_ids", "top_logp")


@pytest.mark.parametrize("p", [[1], [3, 40, 1], [200, 0, 90, 17]])
def test_layer(lv, ctx, p):
    """Every call of a run together, each against the plain form of what the one before left."""
    s = _layer_state(lv, p, sum(p))
    _layer(lv, ctx, s)
    assert ctx.status() == lv.LV_OK
    hq, hkv, d = s["layout"]
    n = sum(p)
    f = {k: _np(v) for k, v in s.items() if hasattr(v, "dtype")}
    qkv, tol = ref.linear(f["h"], f["w_qkv"], f["b_qkv"], "none", None, "bf16")
    qkv, tol = qkv.reshape(n, -1, d), tol.reshape(n, -1, d)
    kvref.close(f["qkv"][:, hq + hkv:], qkv[:, hq + hkv:], tol[:, hq + hkv:], "v")
    pos = ref.positions(n, f["offsets"], None)
    # queries and keys have been rounded once between: that moves their norm's input by half a step each
    for a, b, w in ((0, hq, "w_q"), (hq, hq + hkv, "w_k")):
        want, tol_r = ref.rotate(qkv[:, a:b], f[w], 1e-6, pos, list(s["rope"].s.freq)[:d // 2], False, "bf16")
        size = np.abs(want).max(-1, keepdims=True) + 1
        kvref.close(f["qkv"][:, a:b], want, tol_r + 2.0**-6 * size, "q and k")
    x = f["o"].reshape(n, -1)
    h1, t1 = ref.linear(x, f["w_o"], None, "none", f["h"], "bf16")
    import torch
    h1 = torch.as_tensor(h1).bfloat16().double().numpy()  # may be a step off where the sum is near a middle
    mid, tm = ref.gated(h1, f["w_gate"], f["w_up"], None, None, "silu", "bf16")
    kvref.close(f["mid"], mid, tm + 2.0**-6 * (np.abs(mid) + 1), "mid")
    h2, t2 = ref.linear(f["mid"], f["w_down"], None, "none", h1, "bf16")
    kvref.close(f["h2"], h2, t2 + t1 + 2.0**-8 * np.abs(h1), "h2")
    logits, tl = ref.linear(f["h2"], f["w_vocab"], None, "none", None, "bf16")
    kvref.close(f["logits"], logits, tl, "logits")
    lp, ent, _, ids, tlp = ref.logprobs(f["logits"], f["ids"], 3)
    assert np.array_equal(f["top_ids"], ids)
    kvref.close(f["logp"], lp, 1e-4, "logp")
    kvref.close(f["top_logp"], tlp, 1e-4, "top_logp")
    kvref.close(f["ent"], ent, 3e-4, "entropy")


def test_layer_captured(lv, ctx):
    """The run captured into a graph gives on other inputs what it gives uncaptured, and the same bits at every replay."""
    import torch
    s, other = _layer_state(lv, [200, 0, 90, 17], 5), _layer_state(lv, [200, 0, 90, 17], 6)
    _layer(lv, ctx, s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _layer(lv, ctx, s)
    want = []
    for src in (s, other):
        _layer(lv, ctx, src)
        want.append({k: src[k].clone() for k in OUTPUTS})
    for i, src in enumerate((s, other, s)):
        if i:
            first = _layer_state(lv, [200, 0, 90, 17], 5 + i % 2)
            for k, v in s.items():
                if hasattr(v, "copy_"):
                    v.copy_(first[k])
        g.replay()
        torch.cuda.synchronize()
        for k in OUTPUTS:
            assert torch.equal(s[k].nan_to_num(7.5), want[i % 2][k].nan_to_num(7.5)), (i, k)
    assert ctx.status() == lv.LV_OK


def test_two_streams_and_contexts(lv):
    """Two contexts at work at once on two streams: the same bits as one after the other."""
    import torch
    ctxs = [lv.Context(), lv.Context()]
    states = [_layer_state(lv, [150, 33], 8), _layer_state(lv, [64, 64, 64], 9)]
    want = []
    for c, s in zip(ctxs, states):
        _layer(lv, c, s)
        torch.cuda.synchronize()
        want.append({k: s[k].clone() for k in OUTPUTS})
        for k in OUTPUTS:
            s[k].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        for c, s, st in zip(ctxs, states, streams):
            with torch.cuda.stream(st):
                _layer(lv, c, s)
    torch.cuda.synchronize()
    for c, s, w in zip(ctxs, states, want):
        assert c.status() == lv.LV_OK
        for k in OUTPUTS:
            assert torch.equal(s[k], w[k]), k
