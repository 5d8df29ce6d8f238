"""Profiles the attention work of serving steps on this machine, or the layer around it too, and fits the latency model to it.

    python examples/profile_steps.py [--whole] [--layout 8b-tp1] [--steps 240] [--seed 1]

A small engine's loop: prompts arrive and are attended to whole, their keys and values appended to a paged 8-bit cache;
between arrivals every running sequence takes a token, and now and then one of them a chunk of 200 more.  Each step is a
plan (lv_kv_plan), the append (lv_kv_store) and the attention (lv_prompt_attend for prompts on an empty cache, else
lv_kv_attend), timed with CUDA events.  As in an engine the GPU is at other work while a step's calls are issued, so the
times are the GPU's and not those of the Python calls, and that work leaves nothing of the cache in L2.  The steps' requests and times are then what the library takes as profiled
batches: lv_fit gives the coefficients of Eq. 1, lv_accuracy says how well they explain the times, lv_attribute shares
the predicted times out to the requests.  One layer, random inputs.

With --whole a step is also what the library does for its tokens around that, the term of Eq. 1 that grows with their number:
the projection to queries, keys and values (lv_linear), the norm and rotation of their heads (lv_qk_rotate), the attention
as above, the output projection onto the residual stream (lv_linear), the feed-forward block (lv_gated_linear, lv_linear),
and for each sequence's last token the logits and the log probability of a next one with its alternatives (lv_linear,
lv_token_logprobs).  A layer's two norms of the residual stream are not among it: the library has no call for them.  The rows
of the sequences' last tokens are picked by torch, between begin and end as the rest is.
"""

from __future__ import annotations

import argparse
import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

LAYOUTS = {"8b-tp1": (32, 8, 128), "14b-tp2": (20, 4, 128), "32b-tp4": (10, 2, 128)}  # query, key/value heads, head size
WIDTHS = {"8b-tp1": (4096, 14336), "14b-tp2": (5120, 6912), "32b-tp4": (5120, 6912)}  # hidden state, a rank's feed-forward
VOCAB = 32_000
BLOCK = 16


class Layer:
    """The weights of a layer on one rank and the work on its tokens outside the attention."""

    def __init__(self, layout, ctx, gen):
        import torch

        import paper_2608_08382_gb300 as lv
        self.lv, self.torch, self.ctx, self.gen = lv, torch, ctx, gen
        self.hq, self.hkv, self.d = LAYOUTS[layout]
        self.width, ffn = WIDTHS[layout]
        heads = (self.hq + 2 * self.hkv) * self.d
        self.w_qkv, self.w_o = self._w(heads, self.width), self._w(self.width, self.hq * self.d)
        self.w_gate, self.w_up, self.w_down = self._w(ffn, self.width), self._w(ffn, self.width), self._w(self.width, ffn)
        self.w_vocab, self.b_qkv = self._w(VOCAB, self.width), self.random(1, heads)[0]
        self.w_q, self.w_k = self.random(1, self.d)[0] * 0.1 + 1, self.random(1, self.d)[0] * 0.1 + 1
        self.rope = lv.Rope.geometric(self.d, 1e6)

    def random(self, n, d):
        return self.torch.randn(n, d, device="cuda", generator=self.gen).bfloat16()

    def _w(self, d_out, d_in):
        return self.random(d_out, d_in) * d_in**-0.5

    def empty(self, *shape, dtype=None):
        return self.torch.empty(shape, dtype=dtype or self.torch.bfloat16, device="cuda")

    def before(self, h, qkv, c, offsets):
        """Queries, keys and values [token][head][element] of hidden states h, at their sequences' positions."""
        lv, n = self.lv, len(h)
        lv.lv_linear(self.ctx, h, self.w_qkv, qkv.view(n, -1), bias=self.b_qkv)
        q, k = qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv]
        lv.lv_qk_rotate(self.ctx, q, k, q, k, self.rope, c=c, token_offsets=offsets, q_weight=self.w_q, k_weight=self.w_k)

    def after(self, h, o, last, ids, out):
        """What follows the attention's outputs o: the block's hidden states out["h"], and of the tokens `last` the log
        probabilities of ids and the five most likely ones."""
        lv, ctx = self.lv, self.ctx
        lv.lv_linear(ctx, o.view(len(h), -1), self.w_o, out["h"], residual=h)
        lv.lv_gated_linear(ctx, out["h"], self.w_gate, self.w_up, out["mid"])
        lv.lv_linear(ctx, out["mid"], self.w_down, out["h"], residual=out["h"])
        self.torch.index_select(out["h"], 0, last, out=out["last"])
        lv.lv_linear(ctx, out["last"], self.w_vocab, out["logits"])
        lv.lv_token_logprobs(ctx, out["logits"], ids=ids, logp=out["logp"], top_ids=out["top_ids"], top_logp=out["top_logp"])

    def outputs(self, n_tok, n_seq):
        f32, i32 = self.torch.float32, self.torch.int32
        return dict(h=self.empty(n_tok, self.width), mid=self.empty(n_tok, len(self.w_gate)),
                    last=self.empty(n_seq, self.width), logits=self.empty(n_seq, VOCAB), logp=self.empty(n_seq, dtype=f32),
                    top_ids=self.empty(n_seq, 5, dtype=i32), top_logp=self.empty(n_seq, 5, dtype=f32))


class Engine:
    """The cache, the block tables and the running sequences of one layer's attention."""

    def __init__(self, layout, n_blocks, max_seqs, max_len, seed, ctx=None, whole=False):
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
        self.layer = Layer(layout, self.ctx, self.gen) if whole else None
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
        if self.layer:
            h, self.out = self.layer.random(tok, self.layer.width), self.layer.outputs(tok, n)
            last = torch.as_tensor(np.cumsum(p) - 1, device="cuda")
            ids = torch.randint(0, VOCAB, (n,), device="cuda", generator=self.gen).int()
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        self.other.zero_()
        begin.record()
        lv.lv_kv_plan(self.ctx, d_p, d_c, BLOCK, self.free[self.used:], table, offsets, slots, counts)
        if self.layer:
            self.layer.before(h, qkv, d_c, offsets)
        lv.lv_kv_store(self.ctx, self.cache, k, v, slots)
        if not c.any():
            lv.lv_prompt_attend(self.ctx, q, k, v, offsets, o)
        else:
            lv.lv_kv_attend(self.ctx, self.cache, q, d_c, table, o, token_offsets=None if tok == n else offsets)
        if self.layer:
            self.layer.after(h, o, last, ids, self.out)
        end.record()
        end.synchronize()
        tokens, blocks = counts.tolist()
        if blocks > self.free.numel() - self.used:
            raise RuntimeError(f"the cache is full: {blocks} blocks needed, {self.free.numel() - self.used} free")
        assert tokens == tok
        self.used += blocks
        self.lens[first:first + n] += p
        return c, o, begin.elapsed_time(end)


def profile(layout="8b-tp1", steps=240, seed=1, max_seqs=192, most=3000, whole=False):
    """Runs the loop; returns the profiled batches (p, c, phase, tenant, offsets), their latencies in seconds, and the engine."""
    rng = np.random.default_rng(seed)
    # a step of each kind with as many sequences as there will be: the context has its scratch and its kernels then
    warm = Engine(layout, 3 * max_seqs + 200, max_seqs, 1000, seed, whole=whole)
    for longest in (700, 1, 200):
        p = np.ones(max_seqs, np.int64)
        p[0] = longest
        warm.step(0, p)
    if whole:
        warm.step(0, np.ones(2, np.int64))  # torch picks rows by another kernel where they are few
    e = Engine(layout, max_seqs * (most + steps * 8) // BLOCK, max_seqs, most + steps * 210, seed, warm.ctx,
               whole)
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
    ap.add_argument("--whole", action="store_true", help="the layer's products, head norms and scores too, not its attention alone")
    ap.add_argument("--steps", type=int, default=240)
    ap.add_argument("--seed", type=int, default=1)
    a = ap.parse_args()
    batches, y, engine = profile(a.layout, a.steps, a.seed, whole=a.whole)
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
