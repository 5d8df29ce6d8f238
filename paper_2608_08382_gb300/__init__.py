"""Python binding of the LLMVisor GB300 attribution library (``include/llmvisor.h``).

Argument marshalling only: every computation runs in the CUDA kernels of
``csrc/``.  Functions keep the C names (``lv_attribute``, ``lv_fit``, ...) and take
``torch`` CUDA tensors, passing their device pointers and the current CUDA stream.
There is no CPU fallback: importing this module fails loudly when the shared
library has not been built (``__graft_entry__.build()`` or
``python paper_2608_08382_gb300/build.py``).
"""

from __future__ import annotations

import ctypes
import dataclasses
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libllmvisor.so")

LV_OK, LV_EINVAL, LV_EOVERFLOW, LV_ENODATA, LV_ESINGULAR, LV_ECUDA, LV_EDATA, LV_ENOMEM, LV_ETIMEOUT = (
    0, -1, -2, -3, -4, -5, -6, -7, -8)
LV_ARITH_AUTO, LV_ARITH_FP64 = 0, 1
LV_TIME_TILES, LV_TIME_PAIRS = 1, 2
LV_STEP_RESET = 1
LV_BF16, LV_F16, LV_F32 = 0, 1, 2
LV_MAX_GROUP = 64
LV_ACT_NONE, LV_ACT_SILU, LV_ACT_GELU, LV_ACT_GELU_TANH, LV_ACT_RELU = range(5)
LV_ROPE_HALVES, LV_ROPE_NEIGHBOURS = 0, 1
LV_MAX_TOP = 32

EXPORTED = [
    "lv_status_string", "lv_arch_constants", "lv_ctx_create", "lv_ctx_destroy", "lv_ctx_set_arith", "lv_ctx_status",
    "lv_ctx_set_timing", "lv_ctx_kernel_time", "lv_ctx_selftest_barrier",
    "lv_features", "lv_batch_latency", "lv_attribute", "lv_attribute_f32", "lv_attribute_step",
    "lv_tenant_acc_create", "lv_tenant_acc_destroy",
    "lv_tenant_acc_reset", "lv_tenant_accumulate", "lv_tenant_totals", "lv_tenant_acc_state_bytes",
    "lv_tenant_acc_export", "lv_tenant_acc_import", "lv_fit", "lv_fit_vtc", "lv_accuracy", "lv_whatif",
    "lv_whatif_admit", "lv_attribute_noalloc", "lv_kv_plan", "lv_kv_store", "lv_kv_attend", "lv_prompt_attend",
    "lv_linear", "lv_gated_linear", "lv_qk_rotate", "lv_token_logprobs",
]


class LVError(RuntimeError):
    def __init__(self, status: int, where: str = ""):
        self.status = int(status)
        super().__init__(f"{where}: {lv_status_string(status)} ({status})")


class lv_arch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim",
                                              "ffn_dim", "weight_bytes", "kv_bytes", "tp")]


class lv_coef(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("beta", "a1", "a2", "a3", "a4")]


class lv_model(ctypes.Structure):
    _fields_ = [("seg", (lv_coef * 2) * 2), ("split", ctypes.c_int64 * 2)]


class lv_batches(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("c", ctypes.c_void_p), ("phase", ctypes.c_void_p),
                ("tenant", ctypes.c_void_p), ("offsets", ctypes.c_void_p), ("n_req", ctypes.c_int64),
                ("n_batch", ctypes.c_int64), ("n_tenants", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class lv_fit_report(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64 * 4), ("status", ctypes.c_int32 * 4), ("dropped", ctypes.c_int32 * 4),
                ("ssr", ctypes.c_double * 4), ("r2", ctypes.c_double * 4)]


class lv_accuracy_report(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("r2_ssr", ctypes.c_double), ("r2_corr", ctypes.c_double),
                ("mean_rel", ctypes.c_double), ("p50", ctypes.c_double), ("p90", ctypes.c_double),
                ("p99", ctypes.c_double)]


class lv_kv_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("n_blocks", ctypes.c_int64), ("block_tokens", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class lv_rope(ctypes.Structure):
    _fields_ = [("dim", ctypes.c_int32), ("order", ctypes.c_int32), ("freq", ctypes.c_double * 64)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"LLMVisor CUDA library not built: {LIB_PATH} is missing "
                          "(run __graft_entry__.build() or python paper_2608_08382_gb300/build.py)")
    L = ctypes.CDLL(LIB_PATH)
    P, I32, I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    sig = {
        "lv_status_string": ([I32], ctypes.c_char_p),
        "lv_arch_constants": ([P, P, P], I32),
        "lv_ctx_create": ([P], I32),
        "lv_ctx_destroy": ([P], None),
        "lv_ctx_set_arith": ([P, I32], I32),
        "lv_ctx_status": ([P, P], I32),
        "lv_ctx_set_timing": ([P, I32], I32),
        "lv_ctx_kernel_time": ([P, P, P], I32),
        "lv_ctx_selftest_barrier": ([P, P], I32),
        "lv_features": ([P, P, P, P, P, P, P, P], I32),
        "lv_batch_latency": ([P, P, P, P, I64, P, P], I32),
        "lv_attribute": ([P, P, P, P, P, P, P], I32),
        "lv_attribute_f32": ([P, P, P, P, P, P, P], I32),
        "lv_attribute_step": ([P, P, P, P, P, P, P, I32, P], I32),
        "lv_tenant_acc_create": ([P, I32, P], I32),
        "lv_tenant_acc_destroy": ([P], None),
        "lv_tenant_acc_reset": ([P, P], I32),
        "lv_tenant_accumulate": ([P, P, P, P, I64, P], I32),
        "lv_tenant_totals": ([P, P, P, P], I32),
        "lv_tenant_acc_state_bytes": ([P], I64),
        "lv_tenant_acc_export": ([P, P, I64, P], I32),
        "lv_tenant_acc_import": ([P, P, I64, P], I32),
        "lv_fit": ([P, P, P, I32, P, P, P], I32),
        "lv_fit_vtc": ([P, P, P, I32, P, P, P, P], I32),
        "lv_accuracy": ([P, P, P, I64, P, P], I32),
        "lv_whatif": ([P, P, P, P, P, P, I64, P, P, P], I32),
        "lv_whatif_admit": ([P, P, P, P, P, P, P, I64, P, P, I32, ctypes.c_double, P, P, P, P], I32),
        "lv_attribute_noalloc": ([P, P, P, P, P, P], I32),
        "lv_kv_plan": ([P, P, P, I64, I32, P, I64, P, I64, P, P, I64, P, P], I32),
        "lv_kv_store": ([P, P, I32, P, I64, P, I64, P, I64, P], I32),
        "lv_kv_attend": ([P, P, I32, I32, P, I64, I64, P, P, I64, P, I64, ctypes.c_float, P, P, P], I32),
        "lv_prompt_attend": ([P, I32, I32, I32, I32, P, I64, P, I64, P, I64, I64, P, I64, ctypes.c_float, P, P, P], I32),
        "lv_linear": ([P, I32, P, I64, I64, P, I64, I32, I32, P, I32, P, I64, P, I64, P], I32),
        "lv_gated_linear": ([P, I32, P, I64, I64, P, P, I64, I32, I32, P, P, I32, P, I64, P], I32),
        "lv_qk_rotate": ([P, I32, I32, I32, I32, P, I64, P, I64, I64, P, P, I64, P, P, ctypes.c_float, P, P, I64, P, I64, P],
                         I32),
        "lv_token_logprobs": ([P, I32, P, I64, I64, I32, P, P, P, P, I32, P, P, P], I32),
    }
    for name, (args, res) in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = res
    return L


_lib = _load()


def lib():
    return _lib


def lv_status_string(status: int) -> str:
    return _lib.lv_status_string(int(status)).decode()


def _check(status, where):
    if status != LV_OK:
        raise LVError(status, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = _device = None  # set once torch's CUDA state exists


def _stream(stream):
    """The stream's handle; None is torch's current stream.  A serving step's call is bound by its
    host side, so the current stream is taken as a bare handle, without a torch.cuda.Stream object,
    where torch has the two functions for that."""
    global _raw_stream, _device
    if stream is None:
        if _raw_stream is None:
            import torch
            torch.cuda.current_stream()
            raw, _device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
            if raw is None or _device is None:
                raw, _device = (lambda _: torch.cuda.current_stream().cuda_stream), (lambda: None)
            _raw_stream = raw
        return _raw_stream(_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


# ------------------------------------------------------------------ structs

def make_arch(arch) -> lv_arch:
    a = [int(v) for v in arch]
    return lv_arch(*a)


def make_model(coef, split) -> lv_model:
    """coef: (4, 5) array [phase*2 + regime][beta, a1, a2, a3, a4]; split: (2,) ints."""
    coef = np.asarray(coef, dtype=np.float64).reshape(4, 5)
    m = lv_model()
    for s in range(4):
        k = m.seg[s >> 1][s & 1]
        k.beta, k.a1, k.a2, k.a3, k.a4 = (float(v) for v in coef[s])
    m.split[0], m.split[1] = int(split[0]), int(split[1])
    return m


def model_coef(m: lv_model) -> np.ndarray:
    out = np.zeros((4, 5))
    for s in range(4):
        k = m.seg[s >> 1][s & 1]
        out[s] = (k.beta, k.a1, k.a2, k.a3, k.a4)
    return out


@dataclasses.dataclass
class Batches:
    """Device tensors of a batch set: int32 p, c, phase, tenant (or None), int64 offsets."""
    p: object
    c: object
    phase: object
    offsets: object
    tenant: object = None
    n_tenants: int = 0

    def struct(self) -> lv_batches:
        p, off = self.p, self.offsets
        return lv_batches(p.data_ptr(), _ptr(self.c), _ptr(self.phase), _ptr(self.tenant), off.data_ptr(), p.numel(),
                          off.numel() - 1, int(self.n_tenants), 0)

    @property
    def n_req(self):
        return int(self.p.numel())

    @property
    def n_batch(self):
        return int(self.offsets.numel()) - 1


def batches_to_device(p, c, phase, offsets, tenant=None, n_tenants=0, device="cuda"):
    import torch
    def t(a, dt):
        return torch.as_tensor(np.ascontiguousarray(a), dtype=dt).to(device)
    return Batches(p=t(p, torch.int32), c=t(c, torch.int32), phase=t(phase, torch.int32),
                   offsets=t(offsets, torch.int64), tenant=None if tenant is None else t(tenant, torch.int32),
                   n_tenants=int(n_tenants))


# ------------------------------------------------------------------ context

class Context:
    def __init__(self):
        h = ctypes.c_void_p()
        _check(_lib.lv_ctx_create(ctypes.byref(h)), "lv_ctx_create")
        self.h = h

    def set_arith(self, mode: int):
        _check(_lib.lv_ctx_set_arith(self.h, int(mode)), "lv_ctx_set_arith")

    def set_timing(self, mask):
        """mask: LV_TIME_TILES | LV_TIME_PAIRS, or 0 (True selects LV_TIME_TILES)."""
        _check(_lib.lv_ctx_set_timing(self.h, int(mask)), "lv_ctx_set_timing")

    def kernel_time(self):
        """(milliseconds, launches) of the timed kernels since the previous query."""
        ms, n = ctypes.c_double(), ctypes.c_int64()
        _check(_lib.lv_ctx_kernel_time(self.h, ctypes.byref(ms), ctypes.byref(n)), "lv_ctx_kernel_time")
        return float(ms.value), int(n.value)

    def selftest_barrier(self, stream=None) -> int:
        """Status of the grid-barrier self-test: LV_ETIMEOUT when the bounded wait works."""
        return int(_lib.lv_ctx_selftest_barrier(self.h, _stream(stream)))

    def status(self, stream=None) -> int:
        return int(_lib.lv_ctx_status(self.h, _stream(stream)))

    def close(self):
        if self.h:
            _lib.lv_ctx_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def lv_arch_constants(arch):
    a = make_arch(arch)
    phi = (ctypes.c_int64 * 3)()
    w = ctypes.c_int64()
    _check(_lib.lv_arch_constants(ctypes.byref(a), phi, ctypes.byref(w)), "lv_arch_constants")
    return np.array(list(phi), dtype=np.int64), int(w.value)


def lv_features(ctx: Context, b: Batches, arch=None, model: lv_model | None = None, req_feat=None, batch_feat=None,
                batch_seg=None, stream=None):
    a = make_arch(arch) if arch is not None else None
    bs = b.struct()
    _check(_lib.lv_features(ctx.h, ctypes.byref(a) if a is not None else None,
                            ctypes.byref(model) if model is not None else None, ctypes.byref(bs), _ptr(req_feat),
                            _ptr(batch_feat), _ptr(batch_seg), _stream(stream)), "lv_features")


def lv_batch_latency(ctx: Context, model: lv_model, batch_feat, batch_seg, T, stream=None):
    n = int(T.numel())
    _check(_lib.lv_batch_latency(ctx.h, ctypes.byref(model), _ptr(batch_feat), _ptr(batch_seg), n, _ptr(T),
                                 _stream(stream)), "lv_batch_latency")


def lv_attribute(ctx: Context, model: lv_model, b: Batches, T=None, share=None, acc: "TenantAcc | None" = None,
                 stream=None):
    bs = b.struct()
    _check(_lib.lv_attribute(ctx.h, ctypes.byref(model), ctypes.byref(bs), _ptr(T), _ptr(share),
                             acc.h if acc is not None else None, _stream(stream)), "lv_attribute")


def lv_attribute_step(ctx: Context, model: lv_model, b: Batches, T=None, share=None, acc: "TenantAcc | None" = None,
                      L=None, reset: bool = False, stream=None):
    """One serving step: lv_attribute, then (with acc) the tenant totals into L; reset starts acc from zero."""
    bs = b.struct()
    _check(_lib.lv_attribute_step(ctx.h, ctypes.byref(model), ctypes.byref(bs), _ptr(T), _ptr(share),
                                  acc.h if acc is not None else None, _ptr(L), LV_STEP_RESET if reset else 0,
                                  _stream(stream)), "lv_attribute_step")


def lv_attribute_f32(ctx: Context, model: lv_model, b: "Batches", T=None, share=None, acc: "TenantAcc | None" = None,
                     stream=None):
    bs = b.struct()
    _check(_lib.lv_attribute_f32(ctx.h, ctypes.byref(model), ctypes.byref(bs), _ptr(T), _ptr(share),
                                 acc.h if acc is not None else None, _stream(stream)), "lv_attribute_f32")


class TenantAcc:
    def __init__(self, ctx: Context, n_tenants: int):
        h = ctypes.c_void_p()
        _check(_lib.lv_tenant_acc_create(ctx.h, int(n_tenants), ctypes.byref(h)), "lv_tenant_acc_create")
        self.h, self.ctx, self.n_tenants = h, ctx, int(n_tenants)

    def reset(self, stream=None):
        _check(_lib.lv_tenant_acc_reset(self.h, _stream(stream)), "lv_tenant_acc_reset")

    def state_bytes(self) -> int:
        return int(_lib.lv_tenant_acc_state_bytes(self.h))

    def export(self, stream=None) -> bytes:
        n = self.state_bytes()
        buf = ctypes.create_string_buffer(n)
        _check(_lib.lv_tenant_acc_export(self.h, buf, n, _stream(stream)), "lv_tenant_acc_export")
        return buf.raw

    def import_(self, state: bytes, stream=None):
        buf = ctypes.create_string_buffer(bytes(state), len(state))
        _check(_lib.lv_tenant_acc_import(self.h, buf, len(state), _stream(stream)), "lv_tenant_acc_import")

    def close(self):
        if self.h:
            _lib.lv_tenant_acc_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def lv_tenant_accumulate(ctx: Context, acc: TenantAcc, share, tenant, stream=None):
    _check(_lib.lv_tenant_accumulate(ctx.h, acc.h, _ptr(share), _ptr(tenant), int(share.numel()), _stream(stream)),
           "lv_tenant_accumulate")


def lv_tenant_totals(ctx: Context, acc: TenantAcc, L, stream=None):
    _check(_lib.lv_tenant_totals(ctx.h, acc.h, _ptr(L), _stream(stream)), "lv_tenant_totals")


def lv_fit(ctx: Context, b: Batches, y, models: list, stream=None):
    """y: device float64 tensor [n_y, n_batch]; models: list of lv_model (split read, coefficients written).
    Returns a list of report dicts."""
    n_y = len(models)
    arr = (lv_model * n_y)(*models)
    reps = (lv_fit_report * n_y)()
    bs = b.struct()
    _check(_lib.lv_fit(ctx.h, ctypes.byref(bs), _ptr(y), n_y, arr, reps, _stream(stream)), "lv_fit")
    out = []
    for k in range(n_y):
        models[k] = arr[k]
        r = reps[k]
        out.append(dict(n=list(r.n), status=list(r.status), dropped=list(r.dropped), ssr=list(r.ssr),
                        r2=list(r.r2)))
    return out


def lv_fit_vtc(ctx: Context, b: Batches, y, stream=None):
    """y: device float64 tensor [n_y, n_batch].  Returns a list of (beta, a, status, count), one per y vector."""
    n_y = int(y.shape[0])
    coef = (ctypes.c_double * (2 * n_y))()
    st = (ctypes.c_int32 * n_y)()
    cnt = (ctypes.c_int64 * n_y)()
    bs = b.struct()
    _check(_lib.lv_fit_vtc(ctx.h, ctypes.byref(bs), _ptr(y), n_y, coef, st, cnt, _stream(stream)), "lv_fit_vtc")
    nan = float("nan")
    return [(coef[2 * k] if st[k] == 0 else nan, coef[2 * k + 1] if st[k] == 0 else nan, st[k], cnt[k])
            for k in range(n_y)]


def lv_accuracy(ctx: Context, y, T, stream=None) -> dict:
    """Accuracy of predictions T against measurements y (device float64 tensors of one length)."""
    r = lv_accuracy_report()
    _check(_lib.lv_accuracy(ctx.h, _ptr(y), _ptr(T), int(y.numel()), ctypes.byref(r), _stream(stream)),
           "lv_accuracy")
    return dict(n=r.n, r2_ssr=r.r2_ssr, r2_corr=r.r2_corr, mean_rel=r.mean_rel, p50=r.p50, p90=r.p90, p99=r.p99)


def lv_whatif(ctx: Context, model: lv_model, cand: Batches, p_new, c_new, phase_new, T_new=None, share_new=None,
              stream=None):
    bs = cand.struct()
    _check(_lib.lv_whatif(ctx.h, ctypes.byref(model), ctypes.byref(bs), _ptr(p_new), _ptr(c_new), _ptr(phase_new),
                          int(p_new.numel()), _ptr(T_new), _ptr(share_new), _stream(stream)), "lv_whatif")


def lv_whatif_admit(ctx: Context, model: lv_model, cand: Batches, p_new, c_new, phase_new, tenant_new, L, budget,
                    slo: float, admit, T_new=None, share_new=None, stream=None):
    bs = cand.struct()
    _check(_lib.lv_whatif_admit(ctx.h, ctypes.byref(model), ctypes.byref(bs), _ptr(p_new), _ptr(c_new),
                                _ptr(phase_new), _ptr(tenant_new), int(p_new.numel()), _ptr(L), _ptr(budget),
                                int(L.numel()), float(slo), _ptr(T_new), _ptr(share_new), _ptr(admit),
                                _stream(stream)), "lv_whatif_admit")


# ------------------------------------------------------------------ attention work of a step

_dtypes = {}  # torch dtype -> LV_BF16 / LV_F16, and the other types that the calls below check


def _types():
    import torch
    _dtypes.update({torch.bfloat16: LV_BF16, torch.float16: LV_F16, "i32": torch.int32, "i64": torch.int64,
                    "f32": torch.float32, "u8": torch.uint8})
    return _dtypes


def _want(ok, where):
    """The binding knows shapes, types and strides that the C call cannot see: a mismatch is an invalid argument."""
    if not ok:
        raise LVError(LV_EINVAL, where)


def _rows(x, where):
    """Token stride in elements of a [token][head][element] tensor whose tokens are without gaps inside."""
    st = x.stride()
    _want(x.dim() == 3 and st[2] == 1 and (st[1] == x.shape[2] or x.shape[1] == 1), where)
    return st[0] if x.shape[0] > 1 else x.shape[1] * x.shape[2]


def _sizes(x, dims, where):
    """The sizes of a tensor of that many dimensions."""
    _want(len(x.shape) == dims, where)
    return x.shape


class KVCache:
    """A paged key/value cache in e4m3: uint8 codes k, v [n_blocks][n_kv_heads][block_tokens][head_dim] and float32
    scales [n_blocks][n_kv_heads], all contiguous CUDA tensors, which it keeps."""

    def __init__(self, k, v, k_scale, v_scale):
        t = _dtypes or _types()
        n, h, b, d = _sizes(k, 4, "KVCache")
        _want(k.dtype == v.dtype == t["u8"] and v.shape == k.shape and k.is_contiguous() and v.is_contiguous()
              and k_scale.dtype == v_scale.dtype == t["f32"] and k_scale.shape == v_scale.shape == (n, h)
              and k_scale.is_contiguous() and v_scale.is_contiguous(), "KVCache")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.s = lv_kv_cache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), n, b, h, d, 0)

    @classmethod
    def empty(cls, n_blocks, n_kv_heads, block_tokens, head_dim, device="cuda"):
        """A cache of zeros: no block holds anything."""
        import torch
        shape = (n_blocks, n_kv_heads, block_tokens, head_dim)
        return cls(*(torch.zeros(shape, dtype=torch.uint8, device=device) for _ in "kv"),
                   *(torch.zeros(shape[:2], dtype=torch.float32, device=device) for _ in "kv"))


def lv_kv_plan(ctx: Context, p, c, block_tokens: int, free_blocks, table, token_offsets, slots, counts, stream=None):
    """Block tables and slot maps of a step.  int32 p, c [n_req], free_blocks [n_free], table [n_req][width]; int64
    token_offsets [n_req + 1], slots [n_slots], counts [2]; table's new entries and the last three are written."""
    t = _dtypes or _types()
    n = p.numel()
    _want(p.dtype == c.dtype == free_blocks.dtype == table.dtype == t["i32"] and c.numel() == n
          and token_offsets.dtype == slots.dtype == counts.dtype == t["i64"] and token_offsets.numel() == n + 1
          and counts.numel() == 2 and table.dim() == 2 and table.shape[0] == n and table.is_contiguous()
          and p.is_contiguous() and c.is_contiguous() and free_blocks.is_contiguous() and token_offsets.is_contiguous()
          and slots.is_contiguous() and counts.is_contiguous(), "lv_kv_plan")
    _check(_lib.lv_kv_plan(ctx.h, p.data_ptr(), c.data_ptr(), n, int(block_tokens), free_blocks.data_ptr(),
                           free_blocks.numel(), table.data_ptr(), table.shape[1], token_offsets.data_ptr(),
                           slots.data_ptr(), slots.numel(), counts.data_ptr(), _stream(stream)), "lv_kv_plan")


def lv_kv_store(ctx: Context, cache: KVCache, k, v, slots, stream=None):
    """Appends k, v [n_tok][n_kv_heads][head_dim] (slices of a wider tensor may be given) to the cache."""
    t = _dtypes or _types()
    s, n = cache.s, _sizes(k, 3, "lv_kv_store")[0]
    _want(k.dtype == v.dtype and k.dtype in t and k.shape == v.shape == (n, s.n_kv_heads, s.head_dim)
          and slots.dtype == t["i64"] and slots.numel() == n and slots.is_contiguous(), "lv_kv_store")
    _check(_lib.lv_kv_store(ctx.h, ctypes.byref(s), t[k.dtype], k.data_ptr(), _rows(k, "lv_kv_store"), v.data_ptr(),
                            _rows(v, "lv_kv_store"), slots.data_ptr(), n, _stream(stream)), "lv_kv_store")


def lv_kv_attend(ctx: Context, cache: KVCache, q, c, table, o, lse=None, token_offsets=None, scale=None, stream=None):
    """Attention of queries q [n_tok][n_q_heads][head_dim] over the cache into o (and lse); scale None: 1/sqrt(head_dim)."""
    t = _dtypes or _types()
    s, n, (n_tok, hq, d) = cache.s, c.numel(), _sizes(q, 3, "lv_kv_attend")
    _want(q.dtype in t and d == s.head_dim and o.dtype == q.dtype and o.shape == q.shape and o.is_contiguous()
          and c.dtype == table.dtype == t["i32"] and c.is_contiguous() and table.dim() == 2 and table.shape[0] == n
          and table.is_contiguous()
          and (lse is None or (lse.dtype == t["f32"] and lse.shape == (n_tok, hq) and lse.is_contiguous()))
          and (token_offsets is None or (token_offsets.dtype == t["i64"] and token_offsets.numel() == n + 1
                                         and token_offsets.is_contiguous())), "lv_kv_attend")
    _check(_lib.lv_kv_attend(ctx.h, ctypes.byref(s), t[q.dtype], hq, q.data_ptr(), _rows(q, "lv_kv_attend"), n_tok,
                             _ptr(token_offsets), c.data_ptr(), n, table.data_ptr(), table.shape[1],
                             d ** -0.5 if scale is None else scale, o.data_ptr(), _ptr(lse), _stream(stream)),
           "lv_kv_attend")


def lv_prompt_attend(ctx: Context, q, k, v, offsets, o, lse=None, scale=None, stream=None):
    """Causal attention over packed prompts: q [n_tok][n_q_heads][head_dim], k and v [n_tok][n_kv_heads][head_dim] (slices
    of a wider tensor may be given), int64 offsets [n_seq + 1]; scale None: 1/sqrt(head_dim)."""
    t = _dtypes or _types()
    (n_tok, hq, d), (_, hkv, _) = _sizes(q, 3, "lv_prompt_attend"), _sizes(k, 3, "lv_prompt_attend")
    _want(q.dtype in t and k.dtype == v.dtype == o.dtype == q.dtype and k.shape == v.shape == (n_tok, hkv, d)
          and o.shape == q.shape and o.is_contiguous() and offsets.dtype == t["i64"] and offsets.numel() >= 1
          and offsets.is_contiguous()
          and (lse is None or (lse.dtype == t["f32"] and lse.shape == (n_tok, hq) and lse.is_contiguous())),
          "lv_prompt_attend")
    w = "lv_prompt_attend"
    _check(_lib.lv_prompt_attend(ctx.h, t[q.dtype], hq, hkv, d, q.data_ptr(), _rows(q, w), k.data_ptr(), _rows(k, w),
                                 v.data_ptr(), _rows(v, w), n_tok, offsets.data_ptr(), offsets.numel() - 1,
                                 d ** -0.5 if scale is None else scale, o.data_ptr(), _ptr(lse), _stream(stream)), w)


# ------------------------------------------------------------------ a step's work for each new token

_acts = {"none": LV_ACT_NONE, "silu": LV_ACT_SILU, "gelu": LV_ACT_GELU, "gelu_tanh": LV_ACT_GELU_TANH,
         "relu": LV_ACT_RELU}


# What a call of these costs on the host is what a small step waits for: the checks below ask a tensor for each thing
# once, and raise in one place.

def _flat(x, shape, dtype, where):
    """Row stride in elements of a tensor of that shape and type on a GPU whose rows are without gaps inside."""
    if x.dtype != dtype or x.shape != shape or not x.is_cuda:
        raise LVError(LV_EINVAL, where)
    rows, one = x.stride()
    if one != 1 and shape[1] != 1:
        raise LVError(LV_EINVAL, where)
    return rows if shape[0] > 1 else -(-shape[1] // 8) * 8


def _heads(x, shape, dtype, where):
    """Token stride in elements of a [token][head][element] tensor of that shape and type on a GPU, without gaps inside a
    token."""
    if x.shape != shape or x.dtype != dtype or not x.is_cuda:
        raise LVError(LV_EINVAL, where)
    tokens, heads, one = x.stride()
    if one != 1 or (heads != shape[2] and shape[1] != 1):
        raise LVError(LV_EINVAL, where)
    return tokens if shape[0] > 1 else shape[1] * shape[2]


def _vector(v, n, dtype, where):
    """Address of a vector of n elements on a GPU, or None."""
    if v is None:
        return None
    if v.dtype != dtype or v.shape != (n,) or not v.is_cuda or (n > 1 and v.stride(0) != 1):
        raise LVError(LV_EINVAL, where)
    return v.data_ptr()


def lv_linear(ctx: Context, x, w, y, bias=None, act="none", residual=None, stream=None):
    """y = act(x w^T + bias) + residual: x [n_tok][d_in], w [d_out][d_in], y and residual [n_tok][d_out] (which may be the
    same tensor), bias [d_out]; rows may be slices of wider ones that begin at 16-byte boundaries.  act: "none", "silu",
    "gelu", "gelu_tanh" or "relu"."""
    t, at, dt = _dtypes or _types(), "lv_linear", x.dtype
    xs, ws, kind, act = x.shape, w.shape, t.get(dt), _acts.get(act)
    if len(xs) != 2 or len(ws) != 2 or ws[1] != xs[1] or kind is None or act is None:
        raise LVError(LV_EINVAL, at)
    out = (xs[0], ws[0])
    st = _lib.lv_linear(ctx.h, kind, x.data_ptr(), _flat(x, xs, dt, at), xs[0], w.data_ptr(), _flat(w, ws, dt, at), xs[1],
                        ws[0], None if bias is None else _vector(bias, ws[0], dt, at), act,
                        None if residual is None else residual.data_ptr(),
                        0 if residual is None else _flat(residual, out, dt, at), y.data_ptr(), _flat(y, out, dt, at),
                        _stream(stream))
    if st:
        raise LVError(st, at)


def lv_gated_linear(ctx: Context, x, w_gate, w_up, y, bias_gate=None, bias_up=None, act="silu", stream=None):
    """y = act(x w_gate^T + bias_gate) * (x w_up^T + bias_up): x [n_tok][d_in], w_gate and w_up [d_out][d_in] of one
    stride, y [n_tok][d_out], biases [d_out]; as lv_linear otherwise."""
    t, at, dt = _dtypes or _types(), "lv_gated_linear", x.dtype
    xs, ws, kind, act = x.shape, w_gate.shape, t.get(dt), _acts.get(act)
    if len(xs) != 2 or len(ws) != 2 or ws[1] != xs[1] or kind is None or act is None:
        raise LVError(LV_EINVAL, at)
    stride = _flat(w_gate, ws, dt, at)
    if _flat(w_up, ws, dt, at) != stride:
        raise LVError(LV_EINVAL, at)
    st = _lib.lv_gated_linear(ctx.h, kind, x.data_ptr(), _flat(x, xs, dt, at), xs[0], w_gate.data_ptr(), w_up.data_ptr(),
                              stride, xs[1], ws[0], _vector(bias_gate, ws[0], dt, at), _vector(bias_up, ws[0], dt, at), act,
                              y.data_ptr(), _flat(y, (xs[0], ws[0]), dt, at), _stream(stream))
    if st:
        raise LVError(st, at)


class Rope:
    """How positions turn heads: pair j of a token at position n by n * freq[j] radians.  freq: up to 64 numbers, a
    multiple of 8; pairs are elements j and j + len(freq), or with neighbours=True 2j and 2j + 1."""

    def __init__(self, freq, neighbours=False):
        freq = [float(f) for f in freq]
        _want(len(freq) <= 64 and len(freq) % 8 == 0, "Rope")
        self.s = lv_rope(2 * len(freq), LV_ROPE_NEIGHBOURS if neighbours else LV_ROPE_HALVES, (ctypes.c_double * 64)(*freq))
        self.at = ctypes.addressof(self.s)

    @classmethod
    def geometric(cls, dim, base=10000.0, neighbours=False):
        """Frequencies base^(-2j/dim) for the dim/2 pairs of a head's first dim elements."""
        return cls([base ** (-2.0 * j / dim) for j in range(dim // 2)], neighbours)


def lv_qk_rotate(ctx: Context, q, k, q_out, k_out, rope: Rope, c=None, token_offsets=None, q_weight=None, k_weight=None,
                 eps=1e-6, stream=None):
    """Norms (where weights [head_dim] are given) and rotation of q [n_tok][n_q_heads][head_dim] and
    k [n_tok][n_kv_heads][head_dim] into q_out and k_out (slices of wider tensors may be given; q_out may be q, k_out k).
    Positions as lv_kv_attend's: int32 c [n_req], int64 token_offsets [n_req + 1] or None for one token a request; c None
    with token_offsets: requests that start on an empty cache."""
    t, at, dt = _dtypes or _types(), "lv_qk_rotate", q.dtype
    qs, ks, kind = q.shape, k.shape, t.get(dt)
    if len(qs) != 3 or len(ks) != 3 or kind is None or ks[0] != qs[0] or ks[2] != qs[2]:
        raise LVError(LV_EINVAL, at)
    n, hq, d = qs
    n_req = n if token_offsets is None else token_offsets.numel() - 1
    if n_req < 0:
        raise LVError(LV_EINVAL, at)
    _check(_lib.lv_qk_rotate(ctx.h, kind, hq, ks[1], d, q.data_ptr(), _heads(q, qs, dt, at), k.data_ptr(),
                             _heads(k, ks, dt, at), n, _vector(token_offsets, n_req + 1, t["i64"], at),
                             _vector(c, n_req, t["i32"], at), n_req, _vector(q_weight, d, dt, at),
                             _vector(k_weight, d, dt, at), eps, rope.at, q_out.data_ptr(), _heads(q_out, qs, dt, at),
                             k_out.data_ptr(), _heads(k_out, ks, dt, at), _stream(stream)), at)


def lv_token_logprobs(ctx: Context, logits, ids=None, logp=None, entropy=None, lse=None, top_ids=None, top_logp=None,
                      stream=None):
    """Of each row of logits [n_tok][vocab] (bfloat16, float16 or float32, any row stride): log probabilities logp of the
    given int32 ids, entropy and lse [n_tok] float32, and the largest logits' ids and log probabilities, int32 top_ids and
    float32 top_logp [n_tok][n_top]; what is None is left out."""
    t, at, dt = _dtypes or _types(), "lv_token_logprobs", logits.dtype
    n, vocab = _sizes(logits, 2, at)
    n_top, f32 = 0 if top_ids is None else _sizes(top_ids, 2, at)[1], t["f32"]
    kind = LV_F32 if dt == f32 else t.get(dt)
    rows, one = logits.stride()
    if kind is None or not logits.is_cuda or (one != 1 and vocab != 1) or (top_ids is None) != (top_logp is None):
        raise LVError(LV_EINVAL, at)
    if top_ids is not None and not (top_ids.dtype == t["i32"] and top_logp.dtype == f32 and top_ids.is_cuda
                                    and top_logp.is_cuda and top_ids.shape == top_logp.shape == (n, n_top)
                                    and top_ids.is_contiguous() and top_logp.is_contiguous()):
        raise LVError(LV_EINVAL, at)
    _check(_lib.lv_token_logprobs(ctx.h, kind, logits.data_ptr(), rows if n > 1 else vocab, n, vocab,
                                  _vector(ids, n, t["i32"], at), _vector(logp, n, f32, at), _vector(entropy, n, f32, at),
                                  _vector(lse, n, f32, at), n_top, None if top_ids is None else top_ids.data_ptr(),
                                  None if top_logp is None else top_logp.data_ptr(), _stream(stream)), at)
