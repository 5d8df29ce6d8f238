"""The example that runs the attention calls together: its steps' attention agrees with a plain form over what the cache
holds, and its profile goes through the fit."""

import importlib.util
import os

import numpy as np
import pytest

import kv_reference as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("profile_steps", os.path.join(ROOT, "examples", "profile_steps.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_profile_and_fit(example):
    batches, y, engine = example.profile("32b-tp4", steps=60, seed=3, max_seqs=24, most=600)
    assert len(y) == 60 and (y > 0).all() and batches["offsets"][-1] == len(batches["p"])
    # a sequence's context is what its earlier steps brought
    assert engine.lens.sum() == batches["p"].sum()
    held = int((-(-engine.lens // example.BLOCK)).sum())
    assert engine.used == held and len(np.unique(engine.table.cpu().numpy()[:len(engine.lens)][engine.table.cpu().numpy()[:len(engine.lens)] >= 0])) == held
    model, report, accuracy, T, share, L = example.fit(batches, y, engine)
    assert sum(report["n"]) == 60 and accuracy["n"] == 60
    assert any(s == 0 for s in report["status"])
    assert np.isclose(float(share.sum()), float(T.sum()), rtol=1e-9)
    assert np.isclose(float(L.sum()), float(T.sum()), rtol=1e-9)
    assert engine.ctx.status() == engine.lv.LV_OK


def test_a_step_over_the_cache(example):
    """One decode step's outputs against the cache's own contents."""
    e = example.Engine("32b-tp4", 400, 8, 700, 5)
    e.step(0, np.array([300, 17, 64]))
    state = e.gen.get_state()
    c, o, _ = e.step(0, np.ones(3, np.int64))
    e.gen.set_state(state)
    q = e.torch.randn(3, e.hq + 2 * e.hkv, e.d, device="cuda", generator=e.gen).bfloat16()[:, :e.hq]
    q, o = (x.double().cpu().numpy() for x in (q, o))
    table = e.table.cpu().numpy()
    for i, n in enumerate(c + 1):
        pos = np.arange(n)
        b = table[i, pos // example.BLOCK]
        K, V = (ref.E4M3[code.cpu().numpy()[b, :, pos % example.BLOCK]] * scale.double().cpu().numpy()[b][:, :, None]
                for code, scale in ((e.cache.k, e.cache.k_scale), (e.cache.v, e.cache.v_scale)))
        for h in range(e.hq):
            g = h * e.hkv // e.hq
            want, _, tol, _ = ref.attend_rows(q[i:i + 1, h], K[:, g], V[:, g], np.ones((1, n), bool), e.d ** -0.5, "bf16", e.d)
            ref.close(o[i:i + 1, h], want, tol, f"sequence {i} head {h}")
