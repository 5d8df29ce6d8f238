"""Products of many tokens, tile after tile on one pair of CTAs: whole outputs against exact ones, bit for bit."""

import pytest

import layer_cases
import test_gpu_attribute as base

pytestmark = pytest.mark.gpu

lv = base.lv
ctx = base.ctx
GUARD = 77.0


def _rows(n, d, dtype, seed):
    """Whole numbers of -2 .. 2 as a slice of a wider tensor."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    whole = torch.full((n + 1, -(-d // 8) * 8 + 8), float("nan"), dtype=dtype, device="cuda")
    whole[:n, :d] = torch.randint(-2, 3, (n, d), device="cuda", generator=g).to(dtype)
    return whole[:n, :d]


def _product(x, w, bias):
    """Sums of at most 2^11 products of at most 4, and a bias: exact."""
    v = x.double() @ w.double().t()
    return v if bias is None else v + bias.double()


def _out(n, d, dtype):
    import torch
    whole = torch.full((n + 2, -(-d // 8) * 8 + 8), GUARD, dtype=dtype, device="cuda")
    return whole[1:n + 1, :d], whole


def _only_inside(whole, n, d):
    """Nothing was written but rows 1 .. n, elements 0 .. d - 1."""
    rest = whole.clone()
    rest[1:n + 1, :d] = GUARD
    assert (rest == GUARD).all()


def _gated(lv, ctx, n, d_in, d_out, dtype, seed):
    """All outputs of a call: relu(x wg^T + bg) (x wu^T + bu), a product of whole numbers below 2^24, rounded once."""
    import torch
    x, wg, wu = (_rows(m, d_in, dtype, seed + k) for k, m in enumerate((n, d_out, d_out)))
    bg, bu = (_rows(1, d_out, dtype, seed + k)[0] for k in (3, 4))
    y, whole = _out(n, d_out, dtype)
    lv.lv_gated_linear(ctx, x, wg, wu, y, bias_gate=bg, bias_up=bu, act="relu")
    want = _product(x, wg, bg).clamp(min=0) * _product(x, wu, bu)
    assert want.abs().max() < 2**24
    wrong = (y != want.to(dtype)).nonzero()
    assert len(wrong) == 0, (len(wrong), wrong[:4].tolist())
    _only_inside(whole, n, d_out)
    assert ctx.status() == lv.LV_OK


@pytest.mark.parametrize("case", layer_cases.GATED_AGAIN, ids=str)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_gated_exchange_from_tile_to_tile(lv, ctx, case, dtype):
    """Two warps exchange their sums once a turn, in places that they go through in turn: a tile's first exchange does not
    take the place of the last one of the tile before, which the other warp may still have to read."""
    import torch
    for seed in (1, 2, 3):
        _gated(lv, ctx, *case[1:4], getattr(torch, dtype), 10 * seed)


@pytest.mark.parametrize("case", layer_cases.GATED, ids=str)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_gated_of_other_widths(lv, ctx, case, dtype):
    import torch
    _gated(lv, ctx, *case[1:4], getattr(torch, dtype), 4)


def test_the_device_cuts_as_listed():
    """The sizes were looked out for the clusters that this device holds (the rule itself: test_layer_cut)."""
    import torch
    assert torch.cuda.get_device_properties(0).multi_processor_count == layer_cases.HOLD[1]


@pytest.mark.parametrize("case", layer_cases.LINEAR, ids=str)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_residual_from_tile_to_tile(lv, ctx, case, dtype):
    """All outputs of relu(x w^T + b) + r, r apart from the outputs and in their place: what is added is the tile's own."""
    import torch
    dt, (n, d_in, d_out) = getattr(torch, dtype), case[1:4]
    x, w, r = (_rows(m, k, dt, 7 + d) for m, k, d in ((n, d_in, 0), (d_out, d_in, 1), (n, d_out, 2)))
    b = _rows(1, d_out, dt, 10)[0]
    want = (_product(x, w, b).clamp(min=0) + r.double()).to(dt)
    for in_place in (False, True):
        y, whole = _out(n, d_out, dt)
        if in_place:
            y.copy_(r)
        lv.lv_linear(ctx, x, w, y, bias=b, act="relu", residual=y if in_place else r)
        wrong = (y != want).nonzero()
        assert len(wrong) == 0, (in_place, len(wrong), wrong[:4].tolist())
        _only_inside(whole, n, d_out)
    assert ctx.status() == lv.LV_OK
