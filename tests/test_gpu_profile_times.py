"""What the example's times are of: the GPU's work in steps of a context that is warm."""

import time

import numpy as np
import pytest

from test_gpu_profile_steps import example  # noqa: F401

pytestmark = pytest.mark.gpu


def test_profile_in_a_warm_context(example, monkeypatch):  # noqa: F811
    """The steps before the profile run in its context: no step that is timed sets the context's buffers up."""
    import paper_2608_08382_gb300 as lv
    made, real = [], lv.Context
    monkeypatch.setattr(lv, "Context", lambda: made.append(real()) or made[-1])
    _, y, engine = example.profile("32b-tp4", steps=8, seed=2, max_seqs=12, most=300)
    assert len(made) == 1 and engine.ctx is made[0] and len(y) == 8


def test_times_are_the_gpus(example, monkeypatch):  # noqa: F811
    """A call that takes the host 150 us longer does not make a small step longer."""
    import paper_2608_08382_gb300 as lv
    e = example.Engine("32b-tp4", 64, 4, 200, 6)
    e.step(0, np.array([30, 17, 64]))
    for _ in range(3):
        e.step(0, np.ones(3, np.int64))
    real = lv.lv_kv_store

    def slow(*a, **k):
        until = time.perf_counter() + 150e-6
        while time.perf_counter() < until:
            pass
        return real(*a, **k)

    monkeypatch.setattr(lv, "lv_kv_store", slow)
    ms = sorted(e.step(0, np.ones(3, np.int64))[2] for _ in range(9))
    assert ms[4] < 0.1, ms


def test_the_model_explains_the_times(example):  # noqa: F811
    """Half of the steps are explained to a fifth of their time or better (0.02 to 0.03 measured)."""
    batches, y, engine = example.profile("8b-tp1", steps=160, seed=4, max_seqs=96, most=2000)
    accuracy = example.fit(batches, y, engine)[2]
    assert accuracy["n"] == 160 and accuracy["p50"] < 0.2, accuracy
