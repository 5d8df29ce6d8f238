"""Profiles the attention work of serving steps on this machine and fits the latency model to it.

    python examples/profile_steps.py [--layout 8b-tp1] [--steps 240] [--seed 1]

A small engine's loop: prompts arrive and are attended to whole, their keys and values appended to a paged 8-bit cache;
between arrivals every running sequence takes a token, and now and then one of them a chunk of 200 more.  Each step is a
plan (lv_kv_plan), the append (lv_kv_store) and the attention (lv_prompt_attend for prompts on an empty cache, else
lv_kv_attend), timed with CUDA events.  As in an engine the GPU is at other work while a step's calls are issued, so the
times are the GPU's and not those of the Python calls, and that work leaves nothing of the cache in L2.  The steps' requests and times are then what the library takes as profiled
batches: lv_fit gives the coefficients of Eq. 1, lv_accuracy says how well they explain the times, lv_attribute shares
the predicted times out to the requests.  One layer, random inputs.
"""

from __future__ import annotations

import argparse
import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

LAYOUTS = {"8b-tp1": (32, 8, 128), "14b-tp2": (20, 4, 128), "32b-tp4": (10, 2, 128)}  # query, key/value heads, head size
BLOCK = 16


class Engine:
    """The cache, the block tables and the running sequences of one layer's attention."""

    def __init__(self, layout, n_blocks, max_seqs, max_len, seed, ctx=None):
        import torch

        import paper_2608_08382_gb300 as lv
        self.lv, self.torch = lv, torch
        self.hq, self.hkv, self.d = LAYOUTS[layout]
        self.ctx = ctx or lv.Context()
        self.cache = lv.KVCache.empty(n_blocks, self.hkv, BLOCK, self.d)
        self.free = torch.randperm(n_blocks, device="cuda").int()
        self.used = 0
        self.table = torch.full((max_seqs, -(-max_len // BLOCK)), -1, dtype=torch.int32, device="cuda")
        self.lens = np.zeros(0, np.int64)  # tokens in the cache, of each running sequence
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.other = torch.empty(2 << 30, dtype=torch.uint8, device="cuda")  # what other work writes, a third of a millisecond

    def step(self, first, p):
        """Runs sequences first, first + 1, .. with p new tokens each; returns c, the step's outputs and its milliseconds."""
        lv, torch, n = self.lv, self.torch, len(p)
        if first + n > len(self.lens):
            self.lens = np.concatenate([self.lens, np.zeros(first + n - len(self.lens), np.int64)])
        c, tok = self.lens[first:first + n].copy(), int(p.sum())
        # what the layer's projection would leave, and the step's buffers
        qkv = torch.randn(tok, self.hq + 2 * self.hkv, self.d, device="cuda", generator=self.gen).bfloat16()
        q, k, v = qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv], qkv[:, self.hq + self.hkv:]
        o = torch.empty(tok, self.hq, self.d, dtype=qkv.dtype, device="cuda")
        d_p, d_c = (torch.as_tensor(x, dtype=torch.int32, device="cuda") for x in (p, c))
        offsets = torch.empty(n + 1, dtype=torch.int64, device="cuda")
        slots = torch.empty(tok, dtype=torch.int64, device="cuda")
        counts = torch.empty(2, dtype=torch.int64, device="cuda")
        table = self.table[first:first + n]
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        self.other.zero_()
        begin.record()
        lv.lv_kv_plan(self.ctx, d_p, d_c, BLOCK, self.free[self.used:], table, offsets, slots, counts)
        lv.lv_kv_store(self.ctx, self.cache, k, v, slots)
        if not c.any():
            lv.lv_prompt_attend(self.ctx, q, k, v, offsets, o)
        else:
            lv.lv_kv_attend(self.ctx, self.cache, q, d_c, table, o, token_offsets=None if tok == n else offsets)
        end.record()
        end.synchronize()
        tokens, blocks = counts.tolist()
        if blocks > self.free.numel() - self.used:
            raise RuntimeError(f"the cache is full: {blocks} blocks needed, {self.free.numel() - self.used} free")
        assert tokens == tok
        self.used += blocks
        self.lens[first:first + n] += p
        return c, o, begin.elapsed_time(end)


def profile(layout="8b-tp1", steps=240, seed=1, max_seqs=192, most=3000):
    """Runs the loop; returns the profiled batches (p, c, phase, tenant, offsets), their latencies in seconds, and the engine."""
    rng = np.random.default_rng(seed)
    # a step of each kind with as many sequences as there will be: the context has its scratch and its kernels then
    warm = Engine(layout, 3 * max_seqs + 200, max_seqs, 1000, seed)
    for longest in (700, 1, 200):
        p = np.ones(max_seqs, np.int64)
        p[0] = longest
        warm.step(0, p)
    e = Engine(layout, max_seqs * (most + steps * 8) // BLOCK, max_seqs, most + steps * 210, seed, warm.ctx)
    del warm
    rows, sizes, y = [], [], []
    for s in range(steps):
        n = len(e.lens)
        if n == 0 or (n < max_seqs and s % 2 == 0):
            k = min(max_seqs - n, int(rng.integers(1, 5)))
            first, p = n, np.clip(np.rint(np.exp(rng.normal(6.0, 1.0, k))), 1, most).astype(np.int64)
        else:
            # any stretch of the running sequences, one token each; in one step of eight a chunk among them
            first = int(rng.integers(0, n))
            p = np.ones(int(rng.integers(1, n - first + 1)), np.int64)
            if s % 8 == 1:
                p[rng.integers(len(p))] = 200
        c, _, ms = e.step(first, p)
        rows.append(np.stack([p, c, (p > 1).astype(np.int64), rng.integers(0, 4, len(p))]))
        sizes.append(len(p))
        y.append(ms * 1e-3)
    if e.ctx.status() != e.lv.LV_OK:
        raise RuntimeError("a step's kernels met invalid data")
    p, c, phase, tenant = np.concatenate(rows, 1)
    return dict(p=p, c=c, phase=phase, tenant=tenant, offsets=np.concatenate([[0], np.cumsum(sizes)])), np.array(y), e


def fit(batches, y, engine):
    """Eq. 1's coefficients from the profiled steps, how well they explain them, and the tenants' shares of the prediction."""
    import torch
    lv, ctx = engine.lv, engine.ctx
    b = lv.batches_to_device(batches["p"], batches["c"], batches["phase"], batches["offsets"], batches["tenant"], 4)
    d_y = torch.as_tensor(y, dtype=torch.float64, device="cuda")
    models = [lv.make_model(np.zeros((4, 5)), (256, 256))]
    report = lv.lv_fit(ctx, b, d_y[None], models)[0]
    T = torch.empty(b.n_batch, dtype=torch.float64, device="cuda")
    share = torch.empty(b.n_req, dtype=torch.float64, device="cuda")
    acc = lv.TenantAcc(ctx, 4)
    lv.lv_attribute(ctx, models[0], b, T, share, acc)
    L = torch.empty(4, dtype=torch.float64, device="cuda")
    lv.lv_tenant_totals(ctx, acc, L)
    return models[0], report, lv.lv_accuracy(ctx, d_y, T), T, share, L


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--layout", choices=sorted(LAYOUTS), default="8b-tp1")
    ap.add_argument("--steps", type=int, default=240)
    ap.add_argument("--seed", type=int, default=1)
    a = ap.parse_args()
    batches, y, engine = profile(a.layout, a.steps, a.seed)
    model, report, accuracy, T, _, L = fit(batches, y, engine)
    print(f"{a.steps} steps, {int(batches['p'].sum())} tokens, {1e3 * y.sum():.2f} ms in all")
    for g, (n, st, r2) in enumerate(zip(report["n"], report["status"], report["r2"])):
        name = ("decode", "prefill")[g >> 1] + ", " + ("memory", "compute")[g & 1]
        coef = engine.lv.model_coef(model)[g]
        print(f"  {name}-bound: {n} steps" + (f", R^2 {r2:.4f}, coefficients {np.array2string(coef, precision=3)}" if st == 0 else
                                              f": {engine.lv.lv_status_string(st)}"))
    print("accuracy:", {k: round(v, 4) for k, v in accuracy.items()})
    print("tenants' shares of the predicted time (ms):", np.round(1e3 * L.cpu().numpy(), 3))


if __name__ == "__main__":
    main()
