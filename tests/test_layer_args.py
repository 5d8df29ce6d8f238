"""A step's work for each token: refusals and struct layout on the host (no GPU needed), and the reference's own pins."""

import ctypes

import numpy as np
import pytest

import layer_reference as ref
from test_abi import lv  # noqa: F401

AT, ODD = 1 << 20, (1 << 20) + 8  # addresses that nothing reads: every call here ends before a launch


def _linear(lv, **kw):  # noqa: F811
    a = dict(ctx=AT, dtype=0, x=AT, xs=64, n=4, w=AT, ws=64, d_in=64, d_out=32, bias=AT, act=0, r=AT, rs=32, y=AT * 2, ys=32,
             stream=None)
    a.update(kw)
    return lv.lib().lv_linear(*a.values())


def _gated(lv, **kw):  # noqa: F811
    a = dict(ctx=AT, dtype=0, x=AT, xs=64, n=4, wg=AT, wu=AT, ws=64, d_in=64, d_out=32, bg=AT, bu=AT, act=1, y=AT * 2, ys=32,
             stream=None)
    a.update(kw)
    return lv.lib().lv_gated_linear(*a.values())


def _rope(lv, dim=128, order=0, freq=1.0):  # noqa: F811
    return lv.lv_rope(dim, order, (ctypes.c_double * 64)(*[freq] * 64))


def _rotate(lv, **kw):  # noqa: F811
    a = dict(ctx=AT, dtype=0, hq=8, hkv=2, d=128, q=AT, qs=1024, k=AT, ks=256, n=4, off=AT, c=AT, n_req=2, qw=AT, kw=AT,
             eps=1e-6, rope=ctypes.addressof(_rope(lv)), qo=AT, qos=1024, ko=AT, kos=256, stream=None)
    if "spec" in kw:
        kw["rope"] = ctypes.addressof(kw["spec"])
    keep = kw.pop("spec", None) or _rope(lv)
    if "rope" not in kw:
        kw["rope"] = ctypes.addressof(keep)
    a.update(kw)
    return lv.lib().lv_qk_rotate(*a.values())


def _logprobs(lv, **kw):  # noqa: F811
    a = dict(ctx=AT, dtype=0, x=AT, stride=100, n=4, vocab=100, ids=AT, logp=AT, ent=AT, lse=AT, top=3, ti=AT, tl=AT,
             stream=None)
    a.update(kw)
    return lv.lib().lv_token_logprobs(*a.values())


def test_struct_layout(lv):  # noqa: F811
    assert ctypes.sizeof(lv.lv_rope) == 8 + 64 * 8


@pytest.mark.parametrize("bad", [
    dict(ctx=None), dict(dtype=2), dict(dtype=-1), dict(x=None), dict(x=ODD), dict(xs=63), dict(xs=56), dict(xs=68),
    dict(n=-1), dict(n=2**30 + 1), dict(w=None), dict(w=ODD), dict(ws=56), dict(ws=60), dict(d_in=0), dict(d_in=2**24 + 1),
    dict(d_out=0), dict(d_out=-5), dict(d_out=2**24 + 1), dict(bias=AT + 1), dict(act=-1), dict(act=5), dict(r=ODD),
    dict(rs=24), dict(rs=36), dict(y=None), dict(y=ODD), dict(ys=24), dict(ys=33), dict(r=AT * 2, rs=40),
    dict(xs=2**38 + 8),
], ids=str)
def test_linear_refuses(lv, bad):  # noqa: F811
    assert _linear(lv, **bad) == lv.LV_EINVAL


@pytest.mark.parametrize("bad", [
    dict(ctx=None), dict(dtype=2), dict(x=None), dict(xs=56), dict(n=-1), dict(wg=None), dict(wu=None), dict(wu=ODD),
    dict(ws=60), dict(d_in=0), dict(d_out=0), dict(bg=AT + 1), dict(bu=AT + 1), dict(act=9), dict(y=None), dict(ys=30),
], ids=str)
def test_gated_refuses(lv, bad):  # noqa: F811
    assert _gated(lv, **bad) == lv.LV_EINVAL


@pytest.mark.parametrize("bad", [
    dict(ctx=None), dict(dtype=2), dict(hq=0), dict(hkv=0), dict(hq=7), dict(hq=130, hkv=2), dict(hkv=1025, hq=1025),
    dict(d=96), dict(d=256), dict(q=None), dict(q=ODD), dict(qs=1016), dict(qs=1028), dict(k=None), dict(ks=248), dict(n=-1),
    dict(n=2**30 + 1), dict(off=None), dict(off=AT + 4), dict(c=AT + 2), dict(n_req=-1), dict(n_req=2**24 + 1),
    dict(qw=AT + 1), dict(kw=AT + 1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(rope=None),
    dict(qo=None), dict(qo=ODD + AT), dict(qos=1016), dict(qos=1032), dict(ko=None), dict(kos=264), dict(kos=250),
], ids=str)
def test_rotate_refuses(lv, bad):  # noqa: F811
    assert _rotate(lv, **bad) == lv.LV_EINVAL


@pytest.mark.parametrize("spec", [(136, 0, 1.0), (-16, 0, 1.0), (24, 0, 1.0), (128, 2, 1.0), (128, 0, float("nan")),
                                  (128, 0, float("inf")), (64, 1, 8.5)], ids=str)
def test_rotate_refuses_frequencies(lv, spec):  # noqa: F811
    assert _rotate(lv, spec=_rope(lv, *spec)) == lv.LV_EINVAL
    if spec[0] == 136:
        assert _rotate(lv, d=64, spec=_rope(lv, 128), qs=512, ks=128, qos=512, kos=128) == lv.LV_EINVAL


@pytest.mark.parametrize("bad", [
    dict(ctx=None), dict(dtype=3), dict(dtype=-1), dict(x=None), dict(x=AT + 1), dict(dtype=2, x=AT + 2), dict(stride=99),
    dict(n=-1), dict(n=2**30 + 1), dict(vocab=0), dict(vocab=2**24 + 1, stride=2**25), dict(ids=None), dict(ids=AT + 2),
    dict(logp=AT + 2), dict(ent=AT + 2), dict(lse=AT + 1), dict(top=-1), dict(top=33), dict(ti=None), dict(tl=None),
    dict(ti=AT + 2), dict(tl=AT + 2),
], ids=str)
def test_logprobs_refuses(lv, bad):  # noqa: F811
    assert _logprobs(lv, **bad) == lv.LV_EINVAL


def test_nothing_to_do(lv):  # noqa: F811
    """No tokens: nothing is looked at, the arrays may be missing."""
    assert _linear(lv, n=0, x=None, y=None, r=None) == lv.LV_OK
    assert _gated(lv, n=0, x=None, y=None) == lv.LV_OK
    assert _rotate(lv, n=0, q=None, k=None, qo=None, ko=None) == lv.LV_OK
    assert _rotate(lv, n_req=0) == lv.LV_OK
    assert _logprobs(lv, n=0, x=None) == lv.LV_OK


def test_binding_refuses(lv):  # noqa: F811
    """Tensors of the wrong shape, type or place (these are on the host) never reach the library."""
    import torch

    class Ctx:
        h = AT

    def t(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype)

    refused = [
        lambda: lv.lv_linear(Ctx, t(4, 64), t(32, 64), t(4, 32)),
        lambda: lv.lv_linear(Ctx, t(4, 64), t(32), t(4, 32)),
        lambda: lv.lv_linear(Ctx, t(4, 64), t(32, 64, dtype=torch.float16), t(4, 32)),
        lambda: lv.lv_linear(Ctx, t(4, 64), t(32, 64), t(5, 32)),
        lambda: lv.lv_linear(Ctx, t(4, 64), t(32, 64), t(4, 32), act="swish"),
        lambda: lv.lv_gated_linear(Ctx, t(4, 64), t(32, 64), t(32, 64), t(4, 32)),
        lambda: lv.lv_gated_linear(Ctx, t(4, 64), t(32, 64), t(31, 64), t(4, 32)),
        lambda: lv.lv_qk_rotate(Ctx, t(4, 8, 64), t(4, 2, 64), t(4, 8, 64), t(4, 2, 64), lv.Rope([1.0] * 8)),
        lambda: lv.lv_qk_rotate(Ctx, t(4, 8, 64), t(4, 2), t(4, 8, 64), t(4, 2, 64), lv.Rope([1.0] * 8)),
        lambda: lv.lv_token_logprobs(Ctx, t(4, 64)),
        lambda: lv.lv_token_logprobs(Ctx, t(4)),
        lambda: lv.Rope([1.0] * 65),
        lambda: lv.Rope([1.0] * 9),
    ]
    for call in refused:
        with pytest.raises(lv.LVError) as e:
            call()
        assert e.value.status == lv.LV_EINVAL


def test_rope_frequencies(lv):  # noqa: F811
    r = lv.Rope.geometric(64, 500000.0, neighbours=True)
    assert r.s.dim == 64 and r.s.order == lv.LV_ROPE_NEIGHBOURS
    assert list(r.s.freq)[:32] == [500000.0 ** (-j / 32) for j in range(32)]


# ------------------------------------------------------------------ the reference's own pins

def test_reference_activations():
    v = np.array([-3.0, 0.0, 2.0])
    assert np.allclose(ref.act(v, "silu"), v / (1 + np.exp(-v)))
    assert np.allclose(ref.act(v, "gelu"), v * 0.5 * (1 + ref._erf(v / np.sqrt(2))))
    assert np.allclose(ref.act(v, "gelu_tanh"), 0.5 * v * (1 + np.tanh(np.sqrt(2 / np.pi) * (v + 0.044715 * v**3))))
    assert np.array_equal(ref.act(v, "relu"), [0, 0, 2]) and np.array_equal(ref.act(v, "none"), v)
    for name in ("silu", "gelu", "gelu_tanh"):  # the slopes that the bounds count with
        x = np.linspace(-8, 8, 20001)
        assert np.abs(np.diff(ref.act(x, name)) / np.diff(x)).max() < 1.13


def test_reference_rotation():
    """A quarter turn a token: (1, 0) goes to (0, 1) and on to (-1, 0); the norm of a head keeps its direction."""
    x = np.zeros((3, 1, 4))
    x[:, 0, 0] = 1
    y, _ = ref.rotate(x, None, 0.0, np.arange(3), [np.pi / 2], False, "f16")
    assert np.allclose(y[:, 0], [[1, 0, 0, 0], [0, 1, 0, 0], [-1, 0, 0, 0]])
    y, _ = ref.rotate(x, None, 0.0, np.arange(3), [np.pi / 2, 0], False, "f16")
    assert np.allclose(y[:, 0], [[1, 0, 0, 0], [0, 0, 1, 0], [-1, 0, 0, 0]])
    y, _ = ref.rotate(3 * x, np.array([2.0, 1, 1, 1]), 0.0, np.zeros(3), [], False, "f16")
    assert np.allclose(y[:, 0, 0], 4.0)
    assert ref.positions(7, [1, 3, 3, 6], [5, 9, 0]).tolist() == [-1, 5, 6, 0, 1, 2, -1]


def test_reference_logprobs():
    x = np.log(np.array([[0.25, 0.5, 0.25], [1.0, 1.0, 2.0]]))
    lp, ent, lse, ids, tlp = ref.logprobs(x, [2, -1], 2)
    assert np.allclose(lp[0], np.log(0.25)) and np.isnan(lp[1]) and np.allclose(lse, [0, np.log(4)])
    assert np.allclose(ent, 1.5 * np.log(2)) and ids.tolist() == [[1, 0], [2, 0]] and np.allclose(tlp[:, 0], np.log(0.5))
    lp, ent, lse, ids, tlp = ref.logprobs(np.full((1, 2), -np.inf), [1], 3)
    assert lp[0] == -np.inf and ent[0] == 0 and lse[0] == -np.inf and ids.tolist() == [[0, 1, -1]]
    lp, ent, lse, ids, tlp = ref.logprobs(np.array([[1.0, np.nan, np.inf, np.nan]]), [0], 4)
    assert np.isnan([lp[0], ent[0], lse[0]]).all() and ids.tolist() == [[1, 3, 2, 0]] and np.isnan(tlp).all()
