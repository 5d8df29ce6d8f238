"""The attention calls where values that a query does not see, or scales far apart, could reach its output: every row is
its own keys' alone, whatever stands beside them."""

import numpy as np
import pytest

import kv_reference as ref
import test_gpu_attribute as base
from test_gpu_kv import _cached, _check_rows, _gather, _np, _t

pytestmark = pytest.mark.gpu

lv = base.lv
ctx = base.ctx


def _prompts(lv, ctx, q, k, v, X):
    import torch
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    lv.lv_prompt_attend(ctx, q, k, v, _t(X, "int64"), o, lse=lse)
    assert ctx.status() == lv.LV_OK
    return o, lse


@pytest.mark.parametrize("hq, d", [(5, 128), (3, 64), (33, 128)])
def test_prompt_rows_that_pad_a_tile(lv, ctx, hq, d):
    """Groups that do not divide a tile of 128 rows leave rows of it without a query: the outputs have the same bits
    whatever a call before left in shared memory there."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()  # noqa: E731
    q, k, v = rand(1500, hq, d), rand(1500, 1, d), rand(1500, 1, d)
    # tiles of whole groups on every SM before the call: rows of zeros, then large ones
    big = rand(20_000, 4, d)
    outs = []
    for size in (0.0, 100.0, 1e4):
        _prompts(lv, ctx, big * size, big[:, :1].contiguous(), big[:, :1].contiguous(), [0, 20_000])
        outs.append(_prompts(lv, ctx, q, k, v, [0, 1500]))
    for o, lse in outs[1:]:
        assert torch.equal(o, outs[0][0]) and torch.equal(lse, outs[0][1])


@pytest.mark.parametrize("len0", [1000, 1017, 530])
def test_prompt_rows_of_the_next_sequence(lv, ctx, len0):
    """A sequence's last tile holds queries of the next one: what these are changes no bit of its outputs."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g).half()  # noqa: E731
    T, d = len0 + 300, 64
    q, k, v = rand(T, 4, d), rand(T, 1, d), rand(T, 1, d)
    want = _prompts(lv, ctx, q, k, v, [0, len0, T])
    for size in (0.0, 50.0, float("nan")):
        q[len0:] = q[:300] * size
        o, lse = _prompts(lv, ctx, q, k, v, [0, len0, T])
        assert torch.equal(o[:len0], want[0][:len0]) and torch.equal(lse[:len0], want[1][:len0])


def _chunk_case(lv, ctx, rng, lens, new, B, hq, hkv, d, change, dtype="bfloat16"):
    """Requests over a cache whose codes and scales `change` has had; their outputs and what these are formed from."""
    import torch
    lens, new = np.asarray(lens, np.int64), np.asarray(new, np.int64)
    codes, scales, table = _cached(rng, lens, B, hkv, d)
    change(codes, scales, table)
    X = np.concatenate([[0], np.cumsum(new)])
    q = torch.as_tensor(rng.normal(size=(X[-1], hq, d))).to(getattr(torch, dtype)).cuda()
    o, lse = torch.full_like(q, 9.0), torch.full((int(X[-1]), hq), 9.0, device="cuda")
    cache = lv.KVCache(*(_t(a, "uint8") for a in codes), *(_t(a, "float32") for a in scales))
    lv.lv_kv_attend(ctx, cache, q, _t(lens - new, "int32"), _t(table, "int32"), o, lse=lse,
                    token_offsets=None if (new == 1).all() else _t(X, "int64"))
    assert ctx.status() == lv.LV_OK
    return X, _np(q), _np(o), _np(lse), codes, scales, table


def _check_own_keys(case, i, n, new, B, hq, hkv, d, rows, unit=1.0):
    """Rows of request i (n keys, the last `new` of them its queries') against the keys that they see and no other."""
    X, q, o, lse, codes, scales, table = case
    K, V = _gather(codes, scales, table, i, n, B)
    for j in rows:
        at, m = X[i] + j, n - new + j + 1
        _check_rows(o[at:at + 1] * unit, lse[at:at + 1], q[at:at + 1], (K[:m], V[:m] * unit), np.ones((1, m), bool), d ** -0.5,
                    "bf16", hq, hkv, f"row {j}")


@pytest.mark.parametrize("up", [2.0**28, 2.0**30, 2.0**90])
@pytest.mark.parametrize("n, new, hq, hkv", [(64, 64, 4, 1), (300, 64, 4, 1), (150, 150, 2, 2), (280, 64, 20, 1)])
def test_chunk_value_scales_of_later_tokens(lv, ctx, up, n, new, hq, hkv):
    """The last block's values are far larger than the others: rows before it keep their own values' weights."""
    B, d = 16, 128
    rng = np.random.default_rng(n)
    last = (n - 1) // B

    def change(codes, scales, table):
        scales[1, table[0, last]] *= up

    case = _chunk_case(lv, ctx, rng, [n], [new], B, hq, hkv, d, change)
    _check_own_keys(case, 0, n, new, B, hq, hkv, d, range(new - (n - last * B)))


@pytest.mark.parametrize("n, new, hq, hkv, d", [(64, 64, 4, 1, 128), (300, 64, 4, 1, 64), (150, 150, 2, 2, 128), (35, 5, 2, 1, 64)])
@pytest.mark.parametrize("which", [0, 1])
def test_nan_scales_of_later_tokens(lv, ctx, which, n, new, hq, hkv, d):
    """A NaN scale of the last block's keys or values is no matter of the rows before it."""
    B = 16
    rng = np.random.default_rng(n + which)
    last = (n - 1) // B
    before = max(0, new - (n - last * B))

    def change(codes, scales, table):
        scales[which, table[0, last]] = np.nan

    case = _chunk_case(lv, ctx, rng, [n], [new], B, hq, hkv, d, change)
    _check_own_keys(case, 0, n, new, B, hq, hkv, d, range(before))
    o, lse = case[2], case[3]
    assert np.isnan(o[before:]).all() and np.isnan(lse[before:]).all() == (which == 0)


def _quiet(codes, table, i, B, k0, k1):
    """Values of request i's keys k0 .. k1 - 1 to zero: their block's scale is another token's."""
    for j in range(k0, k1):
        codes[1, table[i, j // B], :, j % B] = 0


@pytest.mark.parametrize("up", [2.0**10, 2.0**40, 2.0**100])
@pytest.mark.parametrize("n, new, hq, hkv, d", [
    (64, 64, 4, 1, 128), (400, 60, 4, 1, 64), (3000, 40, 4, 1, 128),   # chunks, the last shared by many SMs
    (52, 3, 4, 2, 128), (900, 2, 5, 1, 64), (6000, 4, 4, 1, 128),      # few rows
])
def test_a_large_value_in_the_rows_own_block(lv, ctx, up, n, new, hq, hkv, d):
    """The largest value of a block stands for none of a row's keys, but its scale is theirs too: what they bring is
    zero, and the row's other keys keep their weights."""
    B = 16
    rng = np.random.default_rng(n)
    last = (n - 1) // B * B

    def change(codes, scales, table):
        scales[1, table[0, last // B]] *= up
        _quiet(codes, table, 0, B, last, n - 1)  # all but the last token's

    case = _chunk_case(lv, ctx, rng, [n], [new], B, hq, hkv, d, change)
    _check_own_keys(case, 0, n, new, B, hq, hkv, d, range(new - 1))


@pytest.mark.parametrize("n, new, hq", [(700, 1, 4), (700, 1, 10), (20_000, 1, 4), (500, 1, 40), (9000, 1, 40)])
@pytest.mark.parametrize("at", [0.0, 0.5])
def test_a_block_of_zeros_under_a_large_scale(lv, ctx, n, new, hq, at):
    """A block's values are zeros under a scale 2^60 above the others': it brings nothing, to blocks before and after."""
    B, d = 16, 128
    rng = np.random.default_rng(n + hq)
    b = int(at * n) // B

    def change(codes, scales, table):
        scales[1, table[0, b]] = 2.0**60
        _quiet(codes, table, 0, B, b * B, (b + 1) * B)

    case = _chunk_case(lv, ctx, rng, [n], [new], B, hq, 1, d, change)
    _check_own_keys(case, 0, n, new, B, hq, 1, d, range(new))


@pytest.mark.parametrize("n, new, hq", [(50, 3, 4), (50, 30, 4), (5000, 3, 4), (700, 1, 40)])
def test_values_a_hundred_binades_apart(lv, ctx, n, new, hq):
    """Values near 2^-80, and zeros under 2^100 in the last block: in units of 2^-80 the rows are as any other's."""
    B, d = 16, 128
    rng = np.random.default_rng(n + hq)
    last = (n - 1) // B * B

    def change(codes, scales, table):
        scales[1] *= 2.0**-80
        scales[1, table[0, last // B]] = 2.0**100
        _quiet(codes, table, 0, B, last, n)

    case = _chunk_case(lv, ctx, rng, [n], [new], B, hq, 1, d, change)
    _check_own_keys(case, 0, n, new, B, hq, 1, d, range(new), unit=2.0**80)


def test_f16_prompt_small_weights(lv, ctx):
    """Weights of 2^-26 under large values: 2^15 is the largest weight, so that they are held, and an infinity under one
    is an infinity.

    What is lost of a weight where it is rounded to f16 is half of the least step, 2^-25, where 2^7 stands for the
    largest: 2^-32 of it, which takes the place of 2^-24 in the bound."""
    import torch
    rng = np.random.default_rng(12)
    T, d, away = 2000, 64, -26 * np.log(2.0)
    q, k = np.zeros((T, 1, d)), np.zeros((T, 1, d))
    q[:, 0, 0] = 1.0
    k[1:, 0, 0] = away + 0.3 * rng.normal(size=T - 1)
    v = 20_000.0 + 5_000.0 * rng.normal(size=(T, 1, d))
    v[0] = 0.0
    v[700, 0, 7] = np.inf
    q, k, v = (torch.as_tensor(a).half().cuda() for a in (q, k, v))
    o, lse = torch.empty_like(q), torch.empty(T, 1, device="cuda")
    lv.lv_prompt_attend(ctx, q, k, v, _t([0, T], "int64"), o, lse=lse, scale=1.0)
    assert ctx.status() == lv.LV_OK
    assert torch.isposinf(o[700:, 0, 7]).all() and torch.isfinite(o[:700]).all()
    k64, v64, o64, l64 = _np(k)[:, 0], _np(v)[:, 0], _np(o)[:, 0], _np(lse)[:, 0]
    v64[700, 7] = 0.0
    for t in (0, 1, 50, 699, 700, 1500, T - 1):
        w = np.exp(k64[:t + 1, 0])
        want, a = w @ v64[:t + 1] / w.sum(), w @ np.abs(v64[:t + 1]) / w.sum()
        tol = 2.0**-11 * np.abs(want) + (1.01 * 2.0**-11 + 2.0**-16) * a + 2.0**-32 * np.abs(v64[:t + 1]).sum(0) / w.sum() + 2.0**-24
        fine = np.arange(d) != 7 if t >= 700 else np.ones(d, bool)
        ref.close(o64[t, fine], want[fine], tol[fine], f"row {t}")
        ref.close(l64[t], np.log(w.sum()), 2.0**-18, f"lse {t}")


def test_long_rows_done_again_in_a_prompt(lv, ctx):
    """127 rows of 150,000 keys each are done again alone, for the last token's value is NaN: the rest of the block
    waits for longer than its waits would last by themselves, and the call is good."""
    import torch
    T, d = 150_016, 64
    assert (T - 1) % 256 == 255 or T % 256 == 0  # the last tile is whole
    q = torch.zeros(T, 1, d, device="cuda").bfloat16()
    k = torch.randn(T, 1, d, device="cuda").bfloat16()
    v = torch.ones(T, 1, d, device="cuda").bfloat16()
    v[-1, 0, 3] = float("nan")
    o, lse = torch.empty_like(q), torch.empty(T, 1, device="cuda")
    lv.lv_prompt_attend(ctx, q, k, v, _t([0, T], "int64"), o, lse=lse)
    assert ctx.status() == lv.LV_OK
    assert torch.all(o[:-1] == 1.0) and torch.isnan(o[-1, 0, 3]) and torch.all(o[-1, 0, 4:] == 1.0)
    want = torch.log(torch.arange(1, T + 1, device="cuda", dtype=torch.float64))
    assert float((lse[:, 0] - want).abs().max()) < 1e-4


def test_long_rows_done_again_in_a_chunk(lv, ctx):
    """The same over the cache, where a block has an item of 140,000 keys to itself."""
    import torch
    B, h, d, n, new = 128, 160, 64, 140_000, 32
    nb = -(-n // B)
    one = torch.full((nb, h, B, d), 0x38, dtype=torch.uint8, device="cuda")  # 1.0
    value = one.clone()
    value[nb - 1, :, (n - 1) % B, 3] = 0x7f  # NaN
    scale = torch.ones(nb, h, device="cuda")
    cache = lv.KVCache(one, value, scale, scale.clone())
    q = torch.zeros(new, h, d, device="cuda").bfloat16()
    o, lse = torch.empty_like(q), torch.empty(new, h, device="cuda")
    lv.lv_kv_attend(ctx, cache, q, _t([n - new], "int32"), _t(np.arange(nb)[None], "int32"), o, lse=lse,
                    token_offsets=_t([0, new], "int64"))
    assert ctx.status() == lv.LV_OK
    assert torch.all(o[:-1] == 1.0) and torch.isnan(o[-1, :, 3]).all() and torch.all(o[-1, :, 4:] == 1.0)
    want = torch.log(torch.arange(n - new + 1, n + 1, device="cuda", dtype=torch.float64))
    assert float((lse - want[:, None]).abs().max()) < 1e-4


def test_chunks_far_apart_in_a_call(lv, ctx):
    """400,000 requests without a new token between two chunks: the block whose share has the end of one and the
    beginning of the other finds it without a walk over those between, which would outlast its waits at a few millions."""
    import torch
    n, B, hq, d, new, ctx_len = 400_000, 16, 4, 64, 40, 40_000
    rng = np.random.default_rng(13)
    total = ctx_len + new
    codes, scales, few = _cached(rng, np.array([total, total]), B, 1, d)
    table = torch.full((n, few.shape[1]), -1, dtype=torch.int32, device="cuda")
    table[0], table[-1] = _t(few[0], "int32"), _t(few[1], "int32")
    c = torch.zeros(n, dtype=torch.int32, device="cuda")
    c[0] = c[-1] = ctx_len
    X = torch.full((n + 1,), new, dtype=torch.int64, device="cuda")
    X[0], X[-1] = 0, 2 * new
    q = torch.as_tensor(rng.normal(size=(2 * new, hq, d))).bfloat16().cuda()
    o, lse = torch.empty_like(q), torch.empty(2 * new, hq, device="cuda")
    cache = lv.KVCache(*(_t(a, "uint8") for a in codes), *(_t(a, "float32") for a in scales))
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for _ in range(2):
        begin.record()
        lv.lv_kv_attend(ctx, cache, q, c, table, o, lse=lse, token_offsets=X)
        end.record()
    assert ctx.status() == lv.LV_OK
    for i in range(2):
        rows = slice(i * new, (i + 1) * new)
        seen = np.arange(total)[None, :] <= (ctx_len + np.arange(new))[:, None]
        _check_rows(_np(o[rows]), _np(lse[rows]), _np(q[rows]), _gather(codes, scales, few, i, total, B), seen, d ** -0.5,
                    "bf16", hq, 1, f"request {i}")
    assert begin.elapsed_time(end) < 50.0, begin.elapsed_time(end)


@pytest.mark.parametrize("n, new, hq", [(300, 1, 4), (300, 1, 10), (20_000, 1, 4), (300, 40, 4), (300, 3, 4)])
def test_value_scales_below_the_normal_range(lv, ctx, n, new, hq):
    """Value scales that have no reciprocal in fp32: their values are as good as zero, not infinite."""
    B, d = 16, 128
    rng = np.random.default_rng(n + new)

    def tiny(codes, scales, table):
        scales[1] = 1e-39

    case = _chunk_case(lv, ctx, rng, [n], [new], B, hq, 1, d, tiny)
    assert np.isfinite(case[2]).all() and np.abs(case[2]).max() <= 449 * 1e-39

    def some(codes, scales, table):
        scales[1, table[0, ::3][table[0, ::3] < len(codes[0])]] = 1e-42

    case = _chunk_case(lv, ctx, rng, [n], [new], B, hq, 1, d, some)
    _check_own_keys(case, 0, n, new, B, hq, 1, d, range(new))
