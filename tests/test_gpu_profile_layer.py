"""The example's whole-layer steps: they run, their outputs are those of the plain form of what the step's calls were given,
and their profile goes through the fit."""

import numpy as np
import pytest

import kv_reference as kvref
import layer_reference as ref
from test_gpu_profile_steps import example  # noqa: F401

pytestmark = pytest.mark.gpu


def _np(t):
    return t.double().cpu().numpy()


def test_a_whole_step(example):  # noqa: F811
    e = example.Engine("32b-tp4", 400, 8, 700, 5, whole=True)
    seen = {}
    before, after = e.layer.before, e.layer.after

    def watch_before(h, qkv, c, offsets):
        before(h, qkv, c, offsets)
        seen.update(h=h, qkv=qkv, c=c, offsets=offsets)

    def watch_after(h, o, last, ids, out):
        after(h, o, last, ids, out)
        seen.update(o=o, last=last, ids=ids, out=out)

    e.layer.before, e.layer.after = watch_before, watch_after
    for first, p in ((0, [60, 17, 1]), (0, [1, 1, 1]), (1, [1, 30])):
        e.step(first, np.array(p))
        s, L, f = seen, e.layer, {k: _np(v) for k, v in seen["out"].items()}
        h = _np(s["h"])
        qkv, tol = ref.linear(h, _np(L.w_qkv), _np(L.b_qkv), "none", None, "bf16")
        qkv, tol = (x.reshape(len(h), -1, e.d) for x in (qkv, tol))
        got = _np(s["qkv"])
        kvref.close(got[:, e.hq + e.hkv:], qkv[:, e.hq + e.hkv:], tol[:, e.hq + e.hkv:], "values")
        pos = ref.positions(len(h), s["offsets"].tolist(), s["c"].tolist())
        for a, b, w in ((0, e.hq, L.w_q), (e.hq, e.hq + e.hkv, L.w_k)):
            want, t = ref.rotate(qkv[:, a:b], _np(w), 1e-6, pos, list(L.rope.s.freq)[:e.d // 2], False, "bf16")
            # the projection was rounded before the norm: half a step of each of a pair
            kvref.close(got[:, a:b], want, t + 2.0**-6 * (np.abs(want).max(-1, keepdims=True) + 1), "queries and keys")
        # the last product and the scores, from what they were given
        x = f["h"][_np(s["last"]).astype(int)]
        logits, t = ref.linear(x, _np(L.w_vocab), None, "none", None, "bf16")
        kvref.close(f["logits"], logits, t, "logits")
        logp, _, _, ids, top = ref.logprobs(f["logits"], s["ids"].tolist(), 5)
        assert np.array_equal(f["top_ids"], ids)
        kvref.close(f["logp"], logp, 1e-4, "logp")
        kvref.close(f["top_logp"], top, 1e-4, "top_logp")
    assert e.ctx.status() == e.lv.LV_OK


def test_profile_and_fit_of_whole_steps(example):  # noqa: F811
    batches, y, engine = example.profile("32b-tp4", steps=40, seed=3, max_seqs=24, most=600, whole=True)
    assert len(y) == 40 and (y > 0).all()
    model, report, accuracy, T, share, L = example.fit(batches, y, engine)
    assert sum(report["n"]) == 40 and accuracy["n"] == 40
    assert np.isclose(float(share.sum()), float(T.sum()), rtol=1e-9)
    assert engine.ctx.status() == engine.lv.LV_OK
