"""The example's steps with the work around the attention time that work and no allocation."""

import numpy as np
import pytest

from test_gpu_profile_steps import example  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_step_allocates_nothing_between_its_events(example):  # noqa: F811
    import torch
    e = example.Engine("32b-tp4", 400, 8, 700, 5, whole=True)
    seen = []

    def count():
        return torch.cuda.memory_stats()["allocation.all.allocated"]

    def watch(call):
        def watched(*args):
            before = count()
            call(*args)
            seen.append(count() - before)
        return watched

    e.layer.before, e.layer.after = watch(e.layer.before), watch(e.layer.after)
    for first, p in ((0, [60, 17, 1]), (0, [1, 1, 1]), (1, [1, 30])):
        e.step(first, np.array(p))
        assert torch.equal(e.out["last"], e.out["h"][torch.as_tensor(np.cumsum(p) - 1, device="cuda")])
    assert seen == [0] * 6
