"""The attention calls' argument checks and struct layout (no GPU needed), and their reference's own pins."""

import ctypes

import numpy as np
import pytest

import kv_reference as ref
from test_abi import lv  # noqa: F401


def test_struct_layout(lv):  # noqa: F811
    assert ctypes.sizeof(lv.lv_kv_cache) == 4 * 8 + 8 + 4 * 4


def test_refused_without_a_context(lv):  # noqa: F811
    L, at = lv.lib(), ctypes.c_void_p(1 << 20)
    cache = lv.lv_kv_cache(at, at, at, at, 4, 16, 2, 128, 0)
    f = ctypes.c_float(1.0)
    assert L.lv_kv_plan(None, at, at, 1, 16, at, 1, at, 1, at, at, 1, at, None) == lv.LV_EINVAL
    assert L.lv_kv_store(None, ctypes.byref(cache), 0, at, 256, at, 256, at, 1, None) == lv.LV_EINVAL
    assert L.lv_kv_attend(None, ctypes.byref(cache), 0, 4, at, 512, 1, None, at, 1, at, 1, f, at, at, None) == lv.LV_EINVAL
    assert L.lv_prompt_attend(None, 0, 4, 2, 128, at, 512, at, 256, at, 256, 1, at, 1, f, at, at, None) == lv.LV_EINVAL


def test_reference_codes():
    """Every code's value rounds to itself, midpoints to the even neighbour, the largest is 448."""
    v = np.unique(ref.E4M3[np.isfinite(ref.E4M3)])
    assert v.max() == 448.0 and v.min() == -448.0 and len(v) == 253
    assert np.array_equal(ref.round_e4m3(v), v)
    code = {x: i for i, x in enumerate(v[v >= 0])}
    pos = v[v >= 0]
    mid = (pos[:-1] + pos[1:]) / 2
    assert all(code[x] % 2 == 0 for x in ref.round_e4m3(mid))
    assert np.isnan(ref.round_e4m3([np.nan, np.inf, -np.inf])).all()


@pytest.mark.parametrize("amax, want", [(448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (1.75, 2.0**-8), (1.76, 2.0**-7),
                                        (0.0, 2.0**-100), (1e-37, 2.0**-100), (3e38, 2.0**120)])
def test_reference_scale(amax, want):
    assert ref.need_scale(amax) == want
    assert amax <= 448 * want


def test_reference_attention_against_a_hand_case():
    """Two keys with scores 0 and ln 3: weights 1/4 and 3/4."""
    q, K, V = np.array([[1.0, 0.0]]), np.array([[0.0, 5.0], [np.log(3.0), 1.0]]), np.array([[4.0, 0.0], [8.0, 4.0]])
    o, lse, to, tl = ref.attend_rows(q, K, V, np.ones((1, 2), bool), 1.0, "f16", 2)
    assert np.allclose(o, [[7.0, 3.0]]) and np.allclose(lse, np.log(4.0)) and to.max() < 0.01
    o, lse, _, _ = ref.attend_rows(q, K, V, np.zeros((1, 2), bool), 1.0, "f16", 2)
    assert np.all(o == 0) and lse[0] == -np.inf


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [1, 2, 3, 10, 200])
def test_reference_bound_holds_for_its_own_roundings(dtype, n):
    """Weights rounded once, everything else in 64 bits, the output rounded once: within the bound that is derived for
    just that, at one key and at many."""
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float16
    rnd = lambda x: torch.as_tensor(x).to(t).double().numpy()  # noqa: E731
    rng = np.random.default_rng(n)
    for _ in range(200):
        q, K, V = rnd(rng.normal(size=(1, 8))), rnd(rng.normal(size=(n, 8))), rnd(rng.normal(size=(n, 8)))
        o, _, tol, _ = ref.attend_rows(q, K, V, np.ones((1, n), bool), 0.7, dtype, 8)
        s = 0.7 * (K @ q[0])
        w = np.exp(s - s.max())
        ref.close(rnd((rnd(w) @ V) / w.sum())[None], o, tol, "rounded")
