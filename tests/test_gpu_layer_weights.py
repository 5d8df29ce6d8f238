"""Head norms whose weights are far from 1: an output has its own size, whatever its element's and its weight's."""

import numpy as np
import pytest

import kv_reference as kvref
import layer_reference as ref
import test_gpu_attribute as base

pytestmark = pytest.mark.gpu

lv = base.lv
ctx = base.ctx


def _held(a):
    import torch
    return torch.as_tensor(a).bfloat16().double().numpy()


@pytest.mark.parametrize("order", ["halves", "neighbours"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size, weight, eps", [
    (2.0**50, 2.0**80, 1e-6),    # each in range, their product is not
    (2.0**50, 2.0**80, 0.0), (1.0, 2.0**125, 1e-6), (2.0**-20, 2.0**120, 0.0), (2.0**100, 2.0**125, 1e-6),
    (2.0**-40, 2.0**-100, 0.0),  # the other way: their product is below the least normal number
    (2.0**-44, 2.0**-84, 1e-30), (2.0**-30, 2.0**-110, 1e-9), (1.0, 2.0**-120, 1e-6), (2.0**-100, 2.0**-60, 0.0),
    (1.0, 1.0, 1e-6), (2.0**-44, 2.0**-10, 0.0),
], ids=str)
def test_weights_of_any_size(lv, ctx, order, d, size, weight, eps):
    import torch
    rng = np.random.default_rng([d, len(order), int(np.log2(size)) + 200, int(np.log2(weight)) + 200])
    n, hq, hkv = 5, 6, 2
    x = _held(rng.uniform(0.3, 0.9, (n, hq + hkv, d)) * rng.choice([-1, 1], (n, hq + hkv, d)) * size)
    wq, wk = (_held(rng.uniform(0.5, 1.0, d) * weight * 2.0 ** -rng.integers(0, 3, d)) for _ in range(2))
    freq = [1e4 ** (-2.0 * j / d) for j in range(d // 2)]
    dx = torch.as_tensor(x).bfloat16().cuda()
    y = torch.zeros_like(dx)
    pos = np.array([0, 1, 7, 1000, 30_000])
    lv.lv_qk_rotate(ctx, dx[:, :hq], dx[:, hq:], y[:, :hq], y[:, hq:], lv.Rope(freq, order == "neighbours"),
                    c=torch.as_tensor(pos, dtype=torch.int32, device="cuda"),
                    q_weight=torch.as_tensor(wq).bfloat16().cuda(), k_weight=torch.as_tensor(wk).bfloat16().cuda(), eps=eps)
    got = y.double().cpu().numpy()
    for a, b, w in ((0, hq, wq), (hq, hq + hkv, wk)):
        want, tol = ref.rotate(x[:, a:b], w, eps, pos, freq, order == "neighbours", "bf16")
        kvref.close(got[:, a:b], want, tol, "q" if a == 0 else "k")
    assert ctx.status() == lv.LV_OK


def test_one_weight_far_from_the_others(lv, ctx):
    """An element that a tiny weight makes small keeps its size beside others of ordinary ones."""
    import torch
    d = 64
    x = torch.full((1, 2, d), 2.0**-40, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    w[40], w[41], w[42] = 2.0**-110, 2.0**120, 0.0
    y = torch.zeros_like(x)
    lv.lv_qk_rotate(ctx, x[:, :1], x[:, 1:], y[:, :1], y[:, 1:], lv.Rope.geometric(16), q_weight=w, k_weight=w, eps=0.0,
                    c=torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert torch.equal(y, w.expand_as(y))  # all elements alike: each is its weight
    assert ctx.status() == lv.LV_OK
