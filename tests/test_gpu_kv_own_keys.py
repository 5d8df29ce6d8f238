"""The attention calls where values that a query does not see, or scales far apart, could reach its output: every row is
its own keys' alone, whatever stands beside them."""

import pytest

import test_gpu_attribute as base
from test_gpu_kv import _t

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
