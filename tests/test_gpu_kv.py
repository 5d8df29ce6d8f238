"""The attention calls on a GPU against their plain forms in 64 bits: plan, append, attention over the cache and over
packed prompts, at lengths, layouts and masks where they can go wrong."""

import numpy as np
import pytest

import kv_reference as ref
import test_gpu_attribute as base

pytestmark = pytest.mark.gpu

lv = base.lv
ctx = base.ctx


def _t(a, dt):
    import torch
    return torch.as_tensor(np.ascontiguousarray(a), dtype=getattr(torch, dt), device="cuda")


def _np(t):
    import torch
    return t.to(torch.float64).cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _type(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float16


# ------------------------------------------------------------------ plan

def _plan_case(rng, p, c, B, spare, width=None):
    p, c = np.asarray(p, np.int64), np.asarray(c, np.int64)
    held, total = -(-c // B), -(-(c + p) // B)
    need = int((total - held).sum())
    width = int(total.max(initial=0)) + 1 if width is None else width
    ids = rng.permutation(int(held.sum()) + need + 64)
    table = np.full((len(p), width), -7, np.int64)
    at = 0
    for i in range(len(p)):
        n = min(int(held[i]), width)
        table[i, :n] = ids[at:at + n]
        at += n
    return table, ids[at:at + max(0, need + spare)], int(p.sum())


@pytest.mark.parametrize("n, law, B, spare, pad", [
    (1, "one", 16, 0, 0), (1, "zero", 16, 0, 3), (3, "mixed", 16, 2, 5), (128, "decode", 16, 0, 0),
    (257, "mixed", 1, 9, 1), (2047, "mixed", 16, -40, 0), (2048, "mixed", 32, 0, 7), (2049, "mixed", 64, -3, 0),
    (5000, "decode", 128, 0, 100), (4100, "mixed", 16, -500, 11), (40, "long", 16, 0, 1), (2050, "zero", 16, 0, 9),
])
def test_plan(lv, ctx, n, law, B, spare, pad):
    import torch
    rng = np.random.default_rng(n + B)
    p = {"one": [5], "zero": np.zeros(n), "decode": np.ones(n), "long": rng.integers(0, 9000, n),
         "mixed": np.where(rng.random(n) < 0.1, rng.integers(0, 200, n), rng.integers(0, 2, n))}[law]
    c = rng.integers(0, 300, n)
    c[rng.random(n) < 0.3] = 0
    p = np.asarray(p, np.int64)
    table, free, tok = _plan_case(rng, p, c, B, spare)
    want = ref.plan(p, c, B, free, table, tok + pad)
    # arrays at odd places: only their types' own alignment is asked for
    d_p, d_c = _t(np.concatenate([[0], p]), "int32")[1:], _t(np.concatenate([[0], c]), "int32")[1:]
    d_table, d_free = _t(table, "int32"), _t(free, "int32")
    off = torch.full((n + 1,), -9, dtype=torch.int64, device="cuda")
    slots = torch.full((tok + pad,), -9, dtype=torch.int64, device="cuda")
    counts = torch.full((2,), -9, dtype=torch.int64, device="cuda")
    lv.lv_kv_plan(ctx, d_p, d_c, B, d_free, d_table, off, slots, counts)
    assert ctx.status() == lv.LV_OK
    for got, w, name in zip((d_table, off, slots, counts), want, ("table", "offsets", "slots", "counts")):
        assert np.array_equal(got.cpu().numpy(), w), name


def test_plan_of_no_request(lv, ctx):
    import torch
    e32 = torch.empty(0, dtype=torch.int32, device="cuda")
    off = torch.full((1,), 5, dtype=torch.int64, device="cuda")
    slots = torch.full((4,), 5, dtype=torch.int64, device="cuda")
    counts = torch.full((2,), 5, dtype=torch.int64, device="cuda")
    lv.lv_kv_plan(ctx, e32, e32, 16, e32, e32.view(0, 0), off, slots, counts)
    assert ctx.status() == lv.LV_OK
    assert off.tolist() == [0] and slots.tolist() == [-1] * 4 and counts.tolist() == [0, 0]


def test_plan_offsets_past_32_bits(lv, ctx):
    """Three requests of 2^31 - 1 new tokens: the offsets and counts pass 32 bits, the slots given are written."""
    import torch
    n, B, big = 3, 1 << 16, 2**31 - 1
    need = -(-big // B)
    free = _t(np.arange(3 * need), "int32")
    table = torch.zeros((n, need), dtype=torch.int32, device="cuda")
    off = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
    slots = torch.zeros(70_000, dtype=torch.int64, device="cuda")
    counts = torch.zeros(2, dtype=torch.int64, device="cuda")
    lv.lv_kv_plan(ctx, _t([big] * n, "int32"), _t([0] * n, "int32"), B, free, table, off, slots, counts)
    assert ctx.status() == lv.LV_EDATA  # more tokens than slots
    assert off.tolist() == [0, big, 2 * big, 3 * big] and counts.tolist() == [3 * big, 3 * need]
    assert torch.equal(slots, torch.arange(70_000, device="cuda"))
    assert torch.equal(table.flatten(), free)


def test_plan_bad_data(lv, ctx):
    """A negative length counts as no request; a row too short for its blocks is not written past its end."""
    import torch
    B = 16
    table = torch.full((4, 3), -7, dtype=torch.int32, device="cuda")
    guard = torch.full((4,), -7, dtype=torch.int32, device="cuda")
    off = torch.zeros(5, dtype=torch.int64, device="cuda")
    slots = torch.zeros(100, dtype=torch.int64, device="cuda")
    counts = torch.zeros(2, dtype=torch.int64, device="cuda")
    lv.lv_kv_plan(ctx, _t([-3, 2, 70, 1], "int32"), _t([5, -1, 0, 0], "int32"), B, _t(np.arange(10), "int32"), table, off,
                  slots, counts)
    assert ctx.status() == lv.LV_EDATA
    assert off.tolist() == [0, 0, 0, 70, 71] and counts.tolist() == [71, 6]
    assert table.tolist() == [[-7] * 3, [-7] * 3, [0, 1, 2], [5, -7, -7]]
    assert slots.tolist() == list(range(48)) + [-1] * 22 + [80] + [-1] * 29 and guard.tolist() == [-7] * 4


# ------------------------------------------------------------------ append

def _codes(rng, shape):
    """Random codes, NaN among none."""
    x = rng.integers(0, 256, shape)
    return np.where(x & 127 == 127, x - 1, x).astype(np.uint8)


@pytest.mark.parametrize("B, h, d, dtype, runs", [
    (16, 2, 128, "bf16", "decode"), (16, 8, 128, "f16", "prompts"), (32, 1, 64, "bf16", "mixed"),
    (64, 3, 128, "bf16", "mixed"), (128, 4, 64, "f16", "mixed"), (16, 1, 64, "f16", "one"), (128, 1, 128, "bf16", "mixed"),
])
@pytest.mark.parametrize("sliced", [False, True])
def test_store(lv, ctx, B, h, d, dtype, runs, sliced):
    import torch
    rng = np.random.default_rng(B * 10 + h + d)
    p, c = {"decode": (np.ones(200), rng.integers(0, 100, 200)), "one": ([1], [0]),
            "prompts": (rng.integers(1, 150, 9), np.zeros(9)),
            "mixed": (rng.integers(0, 170, 30), rng.integers(0, 60, 30))}[runs]
    p, c = np.asarray(p, np.int64), np.asarray(c, np.int64)
    table, free, tok = _plan_case(rng, p, c, B, 0)
    _, _, slots, _ = ref.plan(p, c, B, free, table, tok + 3)  # three padding tokens
    nb = int(max(table.max(), free.max(initial=0))) + 2
    x = rng.normal(size=(tok + 3, 2, h, d)) * np.exp(2.0 * rng.normal(size=(tok + 3, 2, h, 1)))
    x[rng.random(x.shape) < 0.05] = 0.0
    if tok > 20:
        x[3] = 0.0                      # tokens of zeros: the least scale, or the block's own
        x[5, 0, 0, 1] = np.nan          # held as NaN, not part of the magnitude
        x[6, 1, 0, 2] = -np.inf
        x[7, :, h - 1] *= 1e-30 if dtype == "bf16" else 1e-7
        x[8, 0] *= 1e30 if dtype == "bf16" else 1e3
    x = torch.as_tensor(x).to(_type(dtype)).cuda()
    k, v = (x[:, 0], x[:, 1]) if sliced else (x[:, 0].contiguous(), x[:, 1].contiguous())
    codes = _codes(rng, (2, nb, h, B, d))
    scales = 2.0**rng.integers(-12, 4, (2, nb, h))
    cache = lv.KVCache(*(_t(a, "uint8") for a in codes), *(_t(a, "float32") for a in scales))
    lv.lv_kv_store(ctx, cache, k, v, _t(slots, "int64"))
    assert ctx.status() == lv.LV_OK
    for j, (code, scale) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
        want, ws = ref.store(ref.E4M3[codes[j]], scales[j], _np(x[:, j]), slots, B)
        assert np.array_equal(_np(scale), ws)
        got = ref.E4M3[code.cpu().numpy()]
        assert np.array_equal(got, want, equal_nan=True), np.argwhere(~((got == want) | np.isnan(got)))[:5]
    before = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    lv.lv_kv_store(ctx, cache, k, v, _t(slots, "int64"))  # again: nothing grows, the same codes
    assert all(torch.equal(a, b) for a, b in zip(before, (cache.k, cache.v, cache.k_scale, cache.v_scale)))


def test_store_outside_the_cache(lv, ctx):
    import torch
    cache = lv.KVCache.empty(2, 1, 16, 64)
    x = torch.ones(3, 1, 64, dtype=torch.bfloat16, device="cuda")
    lv.lv_kv_store(ctx, cache, x, x, _t([32, 17, 2**60], "int64"))
    assert ctx.status() == lv.LV_EDATA
    assert cache.k[1, 0, 1].unique().tolist() != [0] and int(cache.k.count_nonzero()) == 64


# ------------------------------------------------------------------ attention

def _check_rows(got_o, got_lse, q, keys, seen, scale, dtype, hq, hkv, what):
    """Tokens q [R][hq][d] of one request on keys (K, V) [n][hkv][d]; seen [R][n]."""
    d = q.shape[2]
    for h in range(hq):
        g = h * hkv // hq
        o, lse, to, tl = ref.attend_rows(q[:, h], keys[0][:, g], keys[1][:, g], seen, scale, dtype, d)
        ref.close(got_o[:, h], o, to, f"{what} o head {h}")
        ref.close(got_lse[:, h], lse, tl, f"{what} lse head {h}")


def _cached(rng, lens, B, hkv, d, spread=1.0):
    """A cache with requests of the given lengths in scattered blocks; whatever no token was written to is NaN."""
    nb = int((-(-lens // B)).sum()) + 3
    codes = np.full((2, nb, hkv, B, d), 127, np.uint8)
    scales = np.full((2, nb, hkv), np.nan)
    width = int((-(-lens // B)).max(initial=0)) + 2
    table = np.full((len(lens), width), nb + 5, np.int64)  # entries past a request's end are not to be followed
    ids = rng.permutation(nb)
    at = 0
    for i, n in enumerate(lens):
        for k in range(-(-int(n) // B)):
            b, m = ids[at], min(B, int(n) - k * B)
            at += 1
            table[i, k] = b
            x = rng.normal(size=(2, hkv, m, d))
            s = ref.need_scale(np.abs(x).max((2, 3))) * np.exp(spread * rng.normal(size=(2, hkv)))
            y = ref.round_e4m3(np.clip(x / s[:, :, None, None], -448, 448))
            codes[:, b, :, :m] = _encode(y)
            scales[:, b] = s.astype(np.float32)
    return codes, scales, table


def _encode(y):
    """Codes of values that e4m3 holds."""
    order = np.argsort(ref.E4M3[:127])
    return (np.searchsorted(ref.E4M3[:127][order], np.abs(y)) | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def _gather(codes, scales, table, i, n, B):
    """K, V [n][hkv][d] of request i."""
    pos = np.arange(n)
    b = table[i, pos // B]
    return [ref.E4M3[codes[j][b, :, pos % B]] * np.float64(np.float32(scales[j][b]))[:, :, None] for j in range(2)]


@pytest.mark.parametrize("lens, new, B, hq, hkv, d, dtype", [
    ([1], 1, 16, 8, 8, 128, "bf16"), ([1, 2, 15, 16, 17, 31, 33], 1, 16, 4, 1, 128, "f16"),
    ([64, 65, 127, 128, 129, 1, 300], 1, 16, 10, 2, 128, "bf16"), ([1000, 3, 517], 1, 32, 12, 12, 64, "f16"),
    ([4097], 1, 16, 32, 8, 128, "bf16"), ([5000, 1, 2500], 1, 64, 16, 1, 64, "bf16"),
    ([777, 1200], 1, 128, 8, 1, 128, "f16"), ([40, 200, 3], 3, 16, 20, 4, 128, "bf16"),
    ([400, 290, 64], 64, 32, 6, 2, 128, "f16"), ([130, 129], 129, 16, 5, 1, 128, "bf16"),
    ([300], 7, 16, 64, 1, 64, "bf16"), ([513, 200], 200, 64, 3, 1, 64, "f16"), ([2000], 1, 16, 64, 1, 128, "f16"),
    (list(range(1, 120)), 1, 16, 5, 1, 128, "bf16"),
])
def test_cache_attention(lv, ctx, lens, new, B, hq, hkv, d, dtype):
    import torch
    rng = np.random.default_rng(len(lens) + new + hq)
    lens = np.asarray(lens, np.int64)
    new = np.minimum(lens, new)
    codes, scales, table = _cached(rng, lens, B, hkv, d)
    X = np.concatenate([[0], np.cumsum(new)])
    q = torch.as_tensor(rng.normal(size=(X[-1], hq + 1, d)) * 1.5).to(_type(dtype)).cuda()[:, :hq]
    o = torch.full((X[-1], hq, d), 9.0, dtype=q.dtype, device="cuda")
    lse = torch.full((X[-1], hq), 9.0, device="cuda")
    cache = lv.KVCache(*(_t(a, "uint8") for a in codes), *(_t(a, "float32") for a in scales))
    lv.lv_kv_attend(ctx, cache, q, _t(lens - new, "int32"), _t(table, "int32"), o, lse=lse,
                    token_offsets=None if new.max() == 1 else _t(X, "int64"))
    assert ctx.status() == lv.LV_OK
    q64, o64, l64 = _np(q), _np(o), _np(lse)
    for i, n in enumerate(lens):
        rows = slice(X[i], X[i + 1])
        seen = np.arange(n)[None, :] <= (n - new[i] + np.arange(new[i]))[:, None]
        _check_rows(o64[rows], l64[rows], q64[rows], _gather(codes, scales, table, i, int(n), B), seen, d ** -0.5,
                    dtype, hq, hkv, f"request {i} of {n}")
    again = torch.empty_like(o)
    lv.lv_kv_attend(ctx, cache, q, _t(lens - new, "int32"), _t(table, "int32"), again,
                    token_offsets=None if new.max() == 1 else _t(X, "int64"))
    assert torch.equal(again, o)  # no lse asked for, and the same bits


def test_cache_attention_hidden_blocks_and_empty_rows(lv, ctx):
    """A table entry of -1 hides its block; a query that sees nothing gives zeros and -inf; request 2 has no query."""
    import torch
    rng = np.random.default_rng(5)
    lens, new, B, hq, hkv, d = np.array([70, 20, 50, 33]), np.array([2, 20, 0, 1]), 16, 4, 2, 128
    codes, scales, table = _cached(rng, lens, B, hkv, d)
    table[0, 1] = -1
    table[1, 0] = -1   # the first 16 of 20 queries see nothing
    table[3, :] = -1   # nothing at all
    X = np.concatenate([[0], np.cumsum(new)])
    q = torch.as_tensor(rng.normal(size=(X[-1], hq, d))).to(torch.bfloat16).cuda()
    o = torch.full((X[-1], hq, d), 9.0, dtype=q.dtype, device="cuda")
    lse = torch.full((X[-1], hq), 9.0, device="cuda")
    cache = lv.KVCache(*(_t(a, "uint8") for a in codes), *(_t(a, "float32") for a in scales))
    lv.lv_kv_attend(ctx, cache, q, _t(lens - new, "int32"), _t(table, "int32"), o, lse=lse, token_offsets=_t(X, "int64"))
    assert ctx.status() == lv.LV_OK
    for i, n in enumerate(lens):
        rows, pos = slice(X[i], X[i + 1]), np.arange(n)
        seen = (pos[None, :] <= (n - new[i] + np.arange(new[i]))[:, None]) & (table[i, pos // B] >= 0)[None, :]
        K, V = _gather(codes, scales, table, i, int(n), B)
        _check_rows(_np(o[rows]), _np(lse[rows]), _np(q[rows]), (K, V), seen, d ** -0.5, "bf16", hq, hkv, f"request {i}")
    assert torch.all(o[2:18] == 0) and torch.all(torch.isinf(lse[2:18])) and torch.all(o[22] == 0)


def test_cache_attention_nan_only_where_seen(lv, ctx):
    """A NaN key or value reaches the queries that see it and no other, in a chunk whose rows share a tile."""
    import torch
    rng = np.random.default_rng(6)
    lens, new, B, hq, hkv, d = np.array([150, 90]), np.array([80, 90]), 16, 4, 1, 128
    codes, scales, table = _cached(rng, lens, B, hkv, d)
    codes[1, table[0, 100 // B], 0, 100 % B, 7] = 127   # a value at position 100 of request 0
    codes[0, table[1, 40 // B], 0, 40 % B, 3] = 127     # a key at position 40 of request 1
    X = np.concatenate([[0], np.cumsum(new)])
    q = torch.as_tensor(rng.normal(size=(X[-1], hq, d))).to(torch.float16).cuda()
    o = torch.empty_like(q)
    lse = torch.empty((X[-1], hq), device="cuda")
    cache = lv.KVCache(*(_t(a, "uint8") for a in codes), *(_t(a, "float32") for a in scales))
    lv.lv_kv_attend(ctx, cache, q, _t(lens - new, "int32"), _t(table, "int32"), o, lse=lse, token_offsets=_t(X, "int64"))
    assert ctx.status() == lv.LV_OK
    bad = torch.isnan(o)
    assert not bad[:30].any() and bad[30:80, :, 7].all()  # rows 70 .. 99 do not see position 100
    assert not bad[30:80, :, :7].any() and not bad[30:80, :, 8:].any() and not torch.isnan(lse[:80]).any()
    assert not bad[80:120].any() and bad[120:].all() and torch.isnan(lse[120:]).all()


def test_cache_attention_bad_data(lv, ctx):
    """Ids outside the cache are hidden, a negative context sees nothing, offsets out of range are no queries."""
    import torch
    rng = np.random.default_rng(7)
    lens, B, hq, hkv, d = np.array([40, 40, 40]), 16, 2, 1, 64
    codes, scales, table = _cached(rng, lens, B, hkv, d)
    good = table.copy()
    table[0, 1] = codes.shape[1]
    table[1, 0] = -2
    q = torch.as_tensor(rng.normal(size=(3, hq, d))).to(torch.bfloat16).cuda()
    o, lse = torch.full_like(q, 9.0), torch.full((3, hq), 9.0, device="cuda")
    cache = lv.KVCache(*(_t(a, "uint8") for a in codes), *(_t(a, "float32") for a in scales))
    lv.lv_kv_attend(ctx, cache, q, _t([39, 39, -1], "int32"), _t(table, "int32"), o, lse=lse)
    assert ctx.status() == lv.LV_EDATA
    for i, hide in ((0, 1), (1, 0)):
        pos = np.arange(40)
        _check_rows(_np(o[i:i + 1]), _np(lse[i:i + 1]), _np(q[i:i + 1]), _gather(codes, scales, good, i, 40, B),
                    (pos // B != hide)[None, :], d ** -0.5, "bf16", hq, hkv, f"request {i}")
    assert torch.all(o[2] == 0) and torch.all(lse[2] == float("-inf"))
    o.fill_(9.0)
    lv.lv_kv_attend(ctx, cache, q, _t([39, 39, 39], "int32"), _t(good, "int32"), o, token_offsets=_t([0, 5, 2, 3], "int64"))
    assert ctx.status() == lv.LV_EDATA
    assert torch.all(o[:2] == 9.0) and not torch.any(o[2] == 9.0)


@pytest.mark.parametrize("lens, hq, hkv, d, dtype", [
    ([1], 4, 4, 128, "bf16"), ([2, 1, 3], 32, 8, 128, "bf16"), ([63, 64, 65], 5, 1, 128, "f16"),
    ([127, 0, 128, 129], 10, 2, 128, "bf16"), ([255, 256, 257], 3, 3, 64, "bf16"), ([700], 8, 2, 64, "f16"),
    ([1000, 1, 130], 4, 1, 128, "f16"), ([31, 33, 384, 385, 0, 0, 12], 16, 1, 64, "bf16"), ([300, 90], 64, 1, 128, "bf16"),
    ([20] * 40, 7, 7, 64, "f16"), ([513], 20, 4, 128, "bf16"), ([200, 311], 33, 1, 128, "f16"), ([1100], 2, 1, 128, "bf16"),
])
@pytest.mark.parametrize("sliced", [False, True])
def test_prompt_attention(lv, ctx, lens, hq, hkv, d, dtype, sliced):
    import torch
    rng = np.random.default_rng(sum(lens) + hq)
    lens = np.asarray(lens, np.int64)
    X = 3 + np.concatenate([[0], np.cumsum(lens)])  # tokens before and after the sequences belong to none
    T = int(X[-1]) + 2
    x = torch.as_tensor(rng.normal(size=(T, hq + 2 * hkv, d)) * 1.5).to(_type(dtype)).cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if not sliced:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    x[:3] = float("nan")
    x[-2:] = float("nan")
    o = torch.full((T, hq, d), 9.0, dtype=q.dtype, device="cuda")
    lse = torch.full((T, hq), 9.0, device="cuda")
    lv.lv_prompt_attend(ctx, q, k, v, _t(X, "int64"), o, lse=lse)
    assert ctx.status() == lv.LV_OK
    assert torch.all(o[:3] == 9.0) and torch.all(o[-2:] == 9.0) and torch.all(lse[:3] == 9.0) and torch.all(lse[-2:] == 9.0)
    q64, k64, v64, o64, l64 = (_np(t) for t in (q, k, v, o, lse))
    for a, b in zip(X, X[1:]):
        _check_rows(o64[a:b], l64[a:b], q64[a:b], (k64[a:b], v64[a:b]), np.tri(b - a, dtype=bool), d ** -0.5, dtype, hq,
                    hkv, f"sequence at {a}")
    again = torch.full_like(o, 9.0)
    lv.lv_prompt_attend(ctx, q, k, v, _t(X, "int64"), again)
    assert torch.equal(again, o)


def test_prompt_attention_nan_only_where_seen(lv, ctx):
    import torch
    rng = np.random.default_rng(8)
    T, hq, d = 400, 2, 128
    q, k, v = (torch.as_tensor(rng.normal(size=(T, h, d))).to(torch.bfloat16).cuda() for h in (hq, 1, 1))
    v[150, 0, 9] = float("nan")
    v[350, 0, 5] = float("inf")
    o, lse = torch.empty_like(q), torch.empty(T, hq, device="cuda")
    lv.lv_prompt_attend(ctx, q, k, v, _t([0, 300, T], "int64"), o, lse=lse)
    assert ctx.status() == lv.LV_OK
    bad = ~torch.isfinite(o)
    assert not bad[:150].any() and bad[150:300, :, 9].all() and not bad[150:300, :, :9].any()
    assert not bad[300:350].any() and torch.all(torch.isposinf(o[350:, :, 5])) and torch.isfinite(lse).all()
    k[150, 0, 9] = float("nan")
    lv.lv_prompt_attend(ctx, q, k, v, _t([0, 300, T], "int64"), o, lse=lse)
    bad = torch.isnan(o)
    assert not bad[:150].any() and bad[150:300].all() and not bad[300:350].any()


def test_prompt_attention_large_scores(lv, ctx):
    """Scores of hundreds, and a scale of the caller's own."""
    import torch
    rng = np.random.default_rng(9)
    T, d = 200, 64
    q, k, v = (torch.as_tensor(rng.normal(size=(T, 1, d)) * a).to(torch.float16).cuda() for a in (12.0, 12.0, 1.0))
    o, lse = torch.empty_like(q), torch.empty(T, 1, device="cuda")
    for scale in (0.3, -0.02, 0.0):
        lv.lv_prompt_attend(ctx, q, k, v, _t([0, T], "int64"), o, lse=lse, scale=scale)
        _check_rows(_np(o), _np(lse), _np(q), (_np(k), _np(v)), np.tri(T, dtype=bool), float(np.float32(scale)), "f16", 1, 1,
                    f"scale {scale}")


def test_prompt_attention_bad_offsets(lv, ctx):
    import torch
    q = torch.ones(10, 1, 64, dtype=torch.bfloat16, device="cuda")
    o = torch.full_like(q, 9.0)
    lv.lv_prompt_attend(ctx, q, q, q, _t([0, 4, 2, 2, 11], "int64"), o)
    assert ctx.status() == lv.LV_EDATA
    assert torch.all(o[:4] == 1.0) and torch.all(o[4:] == 9.0)


# ------------------------------------------------------------------ together, and their refusals

def test_a_step_after_another(lv, ctx):
    """Prompts, then decode steps: plan, append and read; the cache's attention agrees with the prompts' own as far as
    8 bits hold the keys and values."""
    import torch
    rng = np.random.default_rng(10)
    n, B, hq, hkv, d = 5, 16, 8, 2, 128
    p = np.array([40, 1, 16, 33, 90])
    cache = lv.KVCache.empty(64, hkv, B, d)
    free, used = np.arange(64)[::-1].copy(), 0
    table = torch.full((n, 16), -1, dtype=torch.int32, device="cuda")
    c = np.zeros(n, np.int64)
    held = [np.zeros((0, 2, hkv, d)) for _ in range(n)]
    for step in range(6):
        X = np.concatenate([[0], np.cumsum(p)])
        x = torch.as_tensor(rng.normal(size=(X[-1], hq + 2 * hkv, d))).to(torch.bfloat16).cuda()
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        off = torch.empty(n + 1, dtype=torch.int64, device="cuda")
        slots = torch.empty(int(X[-1]), dtype=torch.int64, device="cuda")
        counts = torch.empty(2, dtype=torch.int64, device="cuda")
        d_c = _t(c, "int32")
        lv.lv_kv_plan(ctx, _t(p, "int32"), d_c, B, _t(free[used:], "int32"), table, off, slots, counts)
        lv.lv_kv_store(ctx, cache, k, v, slots)
        o, lse = torch.empty(int(X[-1]), hq, d, dtype=x.dtype, device="cuda"), torch.empty(int(X[-1]), hq, device="cuda")
        lv.lv_kv_attend(ctx, cache, q, d_c, table, o, lse=lse, token_offsets=off)
        used += int(counts[1])
        assert ctx.status() == lv.LV_OK and off.tolist() == X.tolist()
        if step == 0:
            o2 = torch.empty_like(o)
            lv.lv_prompt_attend(ctx, q, k, v, off, o2)
            assert float((o - o2).float().abs().max()) < 0.35  # e4m3 has 4 bits: 1/16 of values and scores of a few units
        kv = _np(torch.stack([k, v], 1))
        for i in range(n):
            held[i] = np.concatenate([held[i], kv[X[i]:X[i + 1]]])
            m = len(held[i])
            code = [np.stack([cache.k.cpu().numpy(), cache.v.cpu().numpy()])]
            K, V = _gather(code[0], np.stack([cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy()]),
                           table.cpu().numpy(), i, m, B)
            # what is held is within e4m3's half step (2^-4 relative, or half its least step) of what was stored; each
            # of a block's up to 15 growths may round a value held in the least steps once more
            sc = np.stack([cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy()])[:, table.cpu().numpy()[i, np.arange(m) // B]]
            for j, got in enumerate((K, V)):
                assert np.all(np.abs(got - held[i][:, j]) <= 2.0**-4 * np.abs(held[i][:, j]) + 16 * 2.0**-10 * sc[j][:, :, None])
            seen = np.arange(m)[None, :] <= (m - p[i] + np.arange(p[i]))[:, None]
            rows = slice(X[i], X[i + 1])
            _check_rows(_np(o[rows]), _np(lse[rows]), _np(q[rows]), (K, V), seen, d ** -0.5, "bf16", hq, hkv, f"step {step}")
        c = c + p
        p = np.ones(n, np.int64) if step != 2 else np.array([1, 0, 20, 1, 2])


def test_calls_on_another_stream_and_in_a_graph(lv, ctx):
    """On a stream of the caller's, and captured: the eager call's bits."""
    import torch
    rng = np.random.default_rng(11)
    lens, B, hq, hkv, d = rng.integers(1, 3000, 20), 16, 8, 2, 128
    codes, scales, table = _cached(rng, lens, B, hkv, d)
    cache = lv.KVCache(*(_t(a, "uint8") for a in codes), *(_t(a, "float32") for a in scales))
    q = torch.as_tensor(rng.normal(size=(20, hq, d))).to(torch.bfloat16).cuda()
    x = torch.as_tensor(rng.normal(size=(700, hq + 2 * hkv, d))).to(torch.bfloat16).cuda()
    d_c, d_table, X = _t(lens - 1, "int32"), _t(table, "int32"), _t([0, 450, 451, 700], "int64")
    outs = [torch.empty_like(q), torch.empty(700, hq, d, dtype=q.dtype, device="cuda")]

    def call(s):
        lv.lv_kv_attend(ctx, cache, q, d_c, d_table, outs[0], stream=s)
        lv.lv_prompt_attend(ctx, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], X, outs[1], stream=s)

    call(None)
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    cs = torch.cuda.Stream()
    for o in outs:
        o.fill_(7)
    torch.cuda.synchronize()
    with torch.cuda.stream(cs):
        call(cs)
    cs.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=cs):
        call(cs)
    for _ in range(3):
        for o in outs:
            o.fill_(7)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    assert ctx.status() == lv.LV_OK


def test_binding_refuses_what_the_c_call_cannot_see(lv, ctx):
    """Types, shapes and strides: the tensors of a call that do not fit are an invalid argument."""
    import torch
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    i32, i64, f32 = torch.int32, torch.int64, torch.float32
    cache = lv.KVCache.empty(4, 2, 16, 128)
    q, k, X = z(3, 4, 128), z(3, 2, 128), z(4, dt=i64)
    calls = [
        lambda: lv.KVCache(cache.k, cache.v[:3], cache.k_scale, cache.v_scale),
        lambda: lv.KVCache(cache.k.float(), cache.v, cache.k_scale, cache.v_scale),
        lambda: lv.KVCache(cache.k, cache.v, cache.k_scale.half(), cache.v_scale),
        lambda: lv.lv_kv_store(ctx, cache, k.float(), k.float(), z(3, dt=i64)),
        lambda: lv.lv_kv_store(ctx, cache, k, k.half(), z(3, dt=i64)),
        lambda: lv.lv_kv_store(ctx, cache, k, k, z(3, dt=i32)),
        lambda: lv.lv_kv_store(ctx, cache, k, k, z(2, dt=i64)),
        lambda: lv.lv_kv_store(ctx, cache, z(3, 2, 64), z(3, 2, 64), z(3, dt=i64)),
        lambda: lv.lv_kv_store(ctx, cache, k, z(3, 2, 256)[:, :, ::2], z(3, dt=i64)),
        lambda: lv.lv_kv_attend(ctx, cache, q, z(3, dt=i64), z(3, 2, dt=i32), q.clone()),
        lambda: lv.lv_kv_attend(ctx, cache, q, z(3, dt=i32), z(2, 2, dt=i32), q.clone()),
        lambda: lv.lv_kv_attend(ctx, cache, q, z(3, dt=i32), z(3, 2, dt=i32), q.half()),
        lambda: lv.lv_kv_attend(ctx, cache, q, z(3, dt=i32), z(3, 2, dt=i32), z(3, 5, 128)[:, :4]),
        lambda: lv.lv_kv_attend(ctx, cache, q, z(2, dt=i32), z(2, 2, dt=i32), q.clone()),  # three queries, two requests
        lambda: lv.lv_kv_attend(ctx, cache, z(3, 3, 128), z(3, dt=i32), z(3, 2, dt=i32), z(3, 3, 128)),
        lambda: lv.lv_kv_attend(ctx, cache, z(3, 4, 64), z(3, dt=i32), z(3, 2, dt=i32), z(3, 4, 64)),
        lambda: lv.lv_kv_attend(ctx, cache, q, z(3, dt=i32), z(3, 2, dt=i32), q.clone(), lse=z(3, 3, dt=f32)),
        lambda: lv.lv_kv_attend(ctx, cache, q, z(3, dt=i32), z(3, 2, dt=i32), q.clone(), scale=float("nan")),
        lambda: lv.lv_prompt_attend(ctx, q, k, k, z(4, dt=i32), q.clone()),
        lambda: lv.lv_prompt_attend(ctx, q, k, z(2, 2, 128), X, q.clone()),
        lambda: lv.lv_prompt_attend(ctx, q, k.half(), k, X, q.clone()),
        lambda: lv.lv_prompt_attend(ctx, q, z(3, 3, 128), z(3, 3, 128), X, q.clone()),
        lambda: lv.lv_prompt_attend(ctx, z(3, 4, 96), z(3, 2, 96), z(3, 2, 96), X, z(3, 4, 96)),
        lambda: lv.lv_prompt_attend(ctx, z(3, 65, 64), z(3, 1, 64), z(3, 1, 64), X, z(3, 65, 64)),
        lambda: lv.lv_prompt_attend(ctx, z(3 * 516)[4:].view(-1)[:3 * 512].view(3, 4, 128), k, k, X, q.clone()),
        lambda: lv.lv_kv_plan(ctx, z(3, dt=i32), z(3, dt=i32), 24, z(3, dt=i32), z(3, 2, dt=i32), X, z(3, dt=i64), z(2, dt=i64)),
        lambda: lv.lv_kv_plan(ctx, z(3, dt=i32), z(2, dt=i32), 16, z(3, dt=i32), z(3, 2, dt=i32), X, z(3, dt=i64), z(2, dt=i64)),
        lambda: lv.lv_kv_plan(ctx, z(3, dt=i32), z(3, dt=i32), 16, z(3, dt=i32), z(3, 2, dt=i32), z(3, dt=i64), z(3, dt=i64),
                              z(2, dt=i64)),
    ]
    for n, call in enumerate(calls):
        with pytest.raises(lv.LVError) as e:
            call()
        assert e.value.status == lv.LV_EINVAL, n
    assert ctx.status() == lv.LV_OK
    # nothing to do is no error
    none = z(0, dt=i32)
    lv.lv_kv_attend(ctx, cache, z(0, 4, 128), none, none.view(0, 0), z(0, 4, 128))
    lv.lv_prompt_attend(ctx, z(0, 4, 128), z(0, 2, 128), z(0, 2, 128), z(1, dt=i64), z(0, 4, 128))
    lv.lv_kv_store(ctx, cache, z(0, 2, 128), z(0, 2, 128), z(0, dt=i64))
    assert ctx.status() == lv.LV_OK
