"""Tensors of a wrong number of dimensions are an invalid argument of the attention calls, like any other mismatch (no GPU
needed: the calls refuse them before anything else)."""

import pytest

from test_abi import lv  # noqa: F401


def test_wrong_number_of_dimensions(lv):  # noqa: F811
    torch = pytest.importorskip("torch")
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    i32, i64, u8, f32 = torch.int32, torch.int64, torch.uint8, torch.float32
    cache = lv.KVCache(z(4, 2, 16, 64, dt=u8), z(4, 2, 16, 64, dt=u8), z(4, 2, dt=f32), z(4, 2, dt=f32))
    q, k, X = z(3, 4, 64), z(3, 2, 64), z(4, dt=i64)
    calls = [
        lambda: lv.KVCache(z(4, 2, 16, dt=u8), z(4, 2, 16, dt=u8), z(4, 2, dt=f32), z(4, 2, dt=f32)),
        lambda: lv.lv_kv_store(None, cache, z(3), z(3), z(3, dt=i64)),
        lambda: lv.lv_kv_store(None, cache, torch.zeros((), dtype=torch.bfloat16), k, z(3, dt=i64)),
        lambda: lv.lv_kv_attend(None, cache, z(3, 256), z(3, dt=i32), z(3, 2, dt=i32), z(3, 256)),
        lambda: lv.lv_kv_attend(None, cache, q[None], z(3, dt=i32), z(3, 2, dt=i32), q[None]),
        lambda: lv.lv_prompt_attend(None, z(3, 256), k, k, X, z(3, 256)),
        lambda: lv.lv_prompt_attend(None, q, z(6), z(6), X, q),
    ]
    for n, call in enumerate(calls):
        with pytest.raises(lv.LVError) as e:
            call()
        assert e.value.status == lv.LV_EINVAL, n
