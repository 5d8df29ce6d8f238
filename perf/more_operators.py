"""The work of a serving step outside its attention, as cases that can be timed and compared.

What a step does for each of its new tokens besides attending: the products with the layer's weights, with what follows
them in the same pass (bias, activation, residual); the gated first half of a feed-forward block; the norm of every
query and key head with the rotation by its position; and at the end of a step the log probabilities of given tokens
with the distribution's entropy and its top alternatives.

A case fixes the shapes; the seed draws every value, the order of lengths and the given tokens.  With `own` false, a pass
computes the plain form in torch; with `own` true, it calls the library.
"""

import math

import torch

own = False

# Head layouts (query heads, key/value heads, head size) of one rank: the 8B-class shape on one rank, the 14B-class
# shape on two, the 32B-class shape on four.
LAYOUTS = {"8b-tp1": (32, 8, 128), "14b-tp2": (20, 4, 128), "32b-tp4": (10, 2, 128), "mha-64": (12, 12, 64),
           "mqa-64": (16, 1, 64), "mqa-128": (8, 1, 128)}
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6


def listed():
    return [
        # one token through a query/key/value projection with bias: the weights' bytes and latency are all there is
        dict(name="linear-decode-1", kind="linear", n_tok=1, d_in=5120, d_out=3584, bias=True, residual=False, act="none",
             dtype="bf16"),
        # a decode batch through the projection that ends a feed-forward block, added to the residual stream
        dict(name="linear-decode-96", kind="linear", n_tok=96, d_in=6912, d_out=5120, bias=False, residual=True,
             act="none", dtype="bf16"),
        # continuous batching with a chunk: the attention's output projection on a rank of four
        dict(name="linear-mixed-1100", kind="linear", n_tok=1100, d_in=1280, d_out=5120, bias=False, residual=True,
             act="none", dtype="f16"),
        # a packed step of prompts through the query/key/value projection
        dict(name="linear-prompts-8192", kind="linear", n_tok=8192, d_in=4096, d_out=6144, bias=False, residual=False,
             act="none", dtype="bf16"),
        # a small decode batch through a feed-forward block's gated half
        dict(name="gated-decode-16", kind="gated", n_tok=16, d_in=4096, d_out=14336, bias=False, act="silu",
             dtype="bf16"),
        # a chunk of a prompt among decodes
        dict(name="gated-chunk-333", kind="gated", n_tok=333, d_in=5120, d_out=6912, bias=False, act="silu",
             dtype="bf16"),
        # packed prompts, an odd number of tokens
        dict(name="gated-prompts-4001", kind="gated", n_tok=4001, d_in=5120, d_out=6912, bias=True, act="gelu_tanh",
             dtype="f16"),
        # a decode step's queries and keys, each at the position where its sequence stands: latency
        dict(name="rotate-decode-128", kind="rotate", n_seq=128, n_tok=128, law="decode", layout="14b-tp2", norm=True,
             rot=128, base=1e6, order="halves", dtype="bf16"),
        # twelve packed prompts
        dict(name="rotate-prompts-8005", kind="rotate", n_seq=12, n_tok=8005, law="prompt", layout="8b-tp1", norm=True,
             rot=128, base=5e5, order="halves", dtype="bf16"),
        # the sampled token of one sequence: latency
        dict(name="logprobs-decode-1", kind="logprobs", n_tok=1, vocab=128_000, top=20, dtype="bf16"),
        # a decode batch whose logits are kept in 32 bits
        dict(name="logprobs-decode-256", kind="logprobs", n_tok=256, vocab=128_000, top=5, dtype="f32"),
        # a long prompt scored token by token
        dict(name="logprobs-prompt-4096", kind="logprobs", n_tok=4096, vocab=32_000, top=1, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "gated", "gated", "rotate", "logprobs"])
    dtype = rng.choice(["bf16", "f16"])
    if kind in ("linear", "gated"):
        # any sizes, or multiples of 64, as most models have them
        unit = rng.choice([1, 64, 64])
        d_in, d_out = (unit * _log_int(rng, max(1, 16 // unit), 16384 // unit) for _ in range(2))
        halves = 2 if kind == "gated" else 1
        n_tok = _log_int(rng, 1, max(1, min(8192, int(4e11 / (2 * d_in * d_out * halves)))))
        case = dict(kind=kind, n_tok=n_tok, d_in=d_in, d_out=d_out, bias=rng.random() < 0.5, dtype=dtype)
        if kind == "gated":
            return dict(case, act=rng.choice(["silu", "gelu", "gelu_tanh", "relu"]))
        return dict(case, residual=rng.random() < 0.5, act=rng.choice(["none", "none", "none", "silu", "gelu", "relu"]))
    if kind == "rotate":
        layout = rng.choice(sorted(LAYOUTS))
        d = LAYOUTS[layout][2]
        law = rng.choice(["decode", "prompt", "chunk"])
        n_tok = _log_int(rng, 1, 4096 if law == "decode" else 8000)
        n_seq = n_tok if law == "decode" else rng.randint(1, min(n_tok, 40))
        return dict(kind=kind, n_seq=n_seq, n_tok=n_tok, law=law, layout=layout, norm=rng.random() < 0.6,
                    rot=rng.choice([d, d, d // 2, 16]), base=rng.choice([1e4, 5e5, 1e6]),
                    order=rng.choice(["halves", "halves", "neighbours"]), dtype=dtype)
    vocab = _log_int(rng, 100, 262_144)
    return dict(kind=kind, n_tok=_log_int(rng, 1, min(4096, 130_000_000 // vocab)), vocab=vocab,
                top=rng.choice([0, 1, 5, 20, 32]), dtype=rng.choice(["bf16", "f16", "f32"]))


# ------------------------------------------------------------------ inputs

def _padded(n):
    return -(-n // 8) * 8


def _rows(g, n, d, dtype, spread=1.0):
    """n rows of d values, in a buffer whose rows begin at multiples of 16 bytes."""
    x = torch.empty(n, _padded(d), dtype=dtype, device="cuda")
    for at in range(0, n, 4096):
        x[at:at + 4096] = torch.randn(x[at:at + 4096].shape, device="cuda", generator=g) * spread
    return x[:, :d]


def _split(g, tokens, n):
    """n uneven lengths of at least 1 that add up to tokens."""
    w = torch.exp(torch.randn(n, generator=g, dtype=torch.float64))
    x = torch.clamp((w / w.sum() * (tokens - n)).floor().long(), min=0) + 1
    x[torch.argmax(x)] += tokens - int(x.sum())
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    s, kind, dtype = dict(case), case["kind"], TYPES[case["dtype"]]
    n = case["n_tok"]
    if kind in ("linear", "gated"):
        d_in, d_out = case["d_in"], case["d_out"]
        x = _rows(g, n, d_in, dtype)
        # as in a trained model, a few channels stand out
        x *= torch.where(torch.rand(d_in, device="cuda", generator=g) < 0.01, 4.0, 1.0).to(dtype)
        s.update(x=x, w=_rows(g, d_out, d_in, dtype, d_in**-0.5))
        if kind == "gated":
            s.update(w_up=_rows(g, d_out, d_in, dtype, d_in**-0.5))
        for name in ("bias", "bias_up")[:2 if kind == "gated" else 1]:
            s[name] = _rows(g, 1, d_out, dtype, 0.5)[0] if case["bias"] else None
        if kind == "linear":
            s["residual"] = _rows(g, n, d_out, dtype, 2.0) if case["residual"] else None
        return s
    if kind == "rotate":
        hq, hkv, d = LAYOUTS[case["layout"]]
        # as a projection leaves them: queries, keys and values of a token side by side
        qkv = torch.randn(n, hq + 2 * hkv, d, device="cuda", generator=g)
        qkv *= torch.exp(0.5 * torch.randn(n, hq + 2 * hkv, 1, device="cuda", generator=g))
        qkv = qkv.to(dtype)
        p = torch.ones(n, dtype=torch.long) if case["law"] == "decode" else _split(host, n, case["n_seq"])
        c = torch.clamp(torch.exp(8.0 + 1.5 * torch.randn(case["n_seq"], generator=host)).long(), max=1 << 20)
        s.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], c=None if case["law"] == "prompt" else c.int().cuda(),
                 offsets=torch.cat([torch.zeros(1, dtype=torch.long), p.cumsum(0)]).cuda(),
                 freq=[case["base"] ** (-2.0 * j / case["rot"]) for j in range(case["rot"] // 2)])
        for name in ("q_weight", "k_weight"):
            w = torch.exp(0.3 * torch.randn(d, device="cuda", generator=g)).to(dtype)
            s[name] = w if case["norm"] else None
        if own:
            lv, _ = _lib()
            s["rope"] = lv.Rope(s["freq"], neighbours=case["order"] == "neighbours")
        return s
    x = torch.empty(n, _padded(case["vocab"]), dtype=dtype, device="cuda")
    for at in range(0, n, 1024):
        part = x[at:at + 1024]
        part.copy_(torch.randn(part.shape, device="cuda", generator=g) * 2.0)
    x = x[:, :case["vocab"]]
    # four different tokens of a row stand out, and half of the given ones are among them
    likely = torch.randint(0, case["vocab"], (n, 1), device="cuda", generator=g)
    likely = (likely + torch.tensor([0, 7, 29, 53], device="cuda")) % case["vocab"]
    x.scatter_add_(1, likely, (4.0 + 3.0 * torch.rand(n, 4, device="cuda", generator=g)).to(dtype))
    other = torch.randint(0, case["vocab"], (n,), device="cuda", generator=g)
    ids = torch.where(torch.rand(n, device="cuda", generator=g) < 0.5, likely[:, 0], other)
    s.update(x=x, ids=ids.int())
    return s


# ------------------------------------------------------------------ a pass

def run(s):
    return {"linear": _linear, "gated": _gated, "rotate": _rotate, "logprobs": _logprobs}[s["kind"]](s)


_kept = {}


def _lib():
    """The library and the program's context, kept for the program's life."""
    if not _kept:
        import paper_2608_08382_gb300 as lv
        _kept["lv"], _kept["ctx"] = lv, lv.Context()
    return _kept["lv"], _kept["ctx"]


def _act(x, name):
    if name == "silu":
        return x / (1.0 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * torch.erfc(x * -math.sqrt(0.5))
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x**3)))
    return torch.clamp(x, min=0.0) if name == "relu" else x


def _out(s):
    """Where the outputs go: rows that begin at multiples of 16 bytes."""
    return torch.empty(s["n_tok"], _padded(s["d_out"]), dtype=s["x"].dtype, device="cuda")[:, :s["d_out"]]


def _product(x, w, bias):
    y = torch.matmul(x.float(), w.float().t())
    return y if bias is None else y + bias.float()


def _linear(s):
    if own:
        lv, ctx = _lib()
        y = _out(s)
        lv.lv_linear(ctx, s["x"], s["w"], y, bias=s["bias"], act=s["act"], residual=s["residual"])
        return y
    y = _act(_product(s["x"], s["w"], s["bias"]), s["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _gated(s):
    if own:
        lv, ctx = _lib()
        y = _out(s)
        lv.lv_gated_linear(ctx, s["x"], s["w"], s["w_up"], y, bias_gate=s["bias"], bias_up=s["bias_up"], act=s["act"])
        return y
    gate = _act(_product(s["x"], s["w"], s["bias"]), s["act"])
    return (gate * _product(s["x"], s["w_up"], s["bias_up"])).to(s["x"].dtype)


def _rotate(s):
    q, k = s["q"], s["k"]
    if own:
        lv, ctx = _lib()
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        lv.lv_qk_rotate(ctx, q, k, q_out, k_out, s["rope"], c=s["c"],
                        token_offsets=None if s["law"] == "decode" else s["offsets"], q_weight=s["q_weight"],
                        k_weight=s["k_weight"], eps=EPS)
        return dict(q=q_out, k=k_out)
    t = torch.arange(s["n_tok"], device="cuda")
    seq = torch.bucketize(t, s["offsets"], right=True) - 1
    pos = t - s["offsets"][seq]
    if s["c"] is not None:
        pos = pos + s["c"].long()[seq]
    angle = pos.double()[:, None] * torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    rot = s["rot"]

    def one(x, weight):
        x = x.float()
        if weight is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
        if s["order"] == "neighbours":
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        else:
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        return torch.cat([turned, x[..., rot:]], -1).to(q.dtype)

    return dict(q=one(q, s["q_weight"]), k=one(k, s["k_weight"]))


def _logprobs(s):
    x, ids, n, top = s["x"], s["ids"], s["n_tok"], min(s["top"], s["vocab"])
    if own:
        lv, ctx = _lib()
        logp, entropy, lse = (torch.empty(n, dtype=torch.float32, device="cuda") for _ in range(3))
        out = dict(logp=logp, entropy=entropy, lse=lse)
        if top:
            out["top_ids"] = torch.empty(n, top, dtype=torch.int32, device="cuda")
            out["top_logp"] = torch.empty(n, top, dtype=torch.float32, device="cuda")
        lv.lv_token_logprobs(ctx, x, ids=ids, **out)
        return out
    x = x.float()
    most = x.amax(1, keepdim=True)
    e = torch.exp(x - most)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    lse = (most + log_total)[:, 0]
    # -sum p log p with log p = (x - most) - log total
    entropy = log_total[:, 0] - (e * (x - most)).sum(1) / total[:, 0]
    out = dict(logp=x.gather(1, ids.long()[:, None])[:, 0] - most[:, 0] - log_total[:, 0], entropy=entropy, lse=lse)
    if top:
        value, index = torch.sort(x, dim=1, descending=True, stable=True)
        out["top_ids"] = index[:, :top].int()
        out["top_logp"] = value[:, :top] - most - log_total
    return out


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    kind, n = case["kind"], case["n_tok"]
    if kind in ("linear", "gated"):
        d_in, d_out, halves = case["d_in"], case["d_out"], 2 if kind == "gated" else 1
        extra = (halves * d_out if case["bias"] else 0) + (n * d_out if case.get("residual") else 0)
        return {"bytes": 2 * (n * d_in + halves * d_out * d_in + n * d_out + extra),
                "flops": 2 * n * d_in * d_out * halves}
    if kind == "rotate":
        hq, hkv, d = LAYOUTS[case["layout"]]
        heads = n * (hq + hkv)
        return {"bytes": heads * d * 4 + (4 * d if case["norm"] else 0) + 8 * case["n_seq"],
                "flops": heads * (3 * case["rot"] + (4 * d if case["norm"] else 0))}
    size = 4 if case["dtype"] == "f32" else 2
    return {"bytes": n * (case["vocab"] * size + 16 + 8 * min(case["top"], case["vocab"])), "flops": 5 * n * case["vocab"]}


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_products, "gated": _exact_products, "rotate": _exact_rotate,
            "logprobs": _exact_logprobs}[case["kind"]](s)


def _exact_act(v, name):
    if name == "silu":
        return v * torch.special.expit(v)
    if name == "gelu":
        return v * torch.special.ndtr(v)
    if name == "gelu_tanh":
        return v * torch.special.expit(2.0 * math.sqrt(2.0 / math.pi) * v * (1.0 + 0.044715 * v * v))
    return torch.where(v > 0, v, torch.zeros_like(v)) if name == "relu" else v


def _exact_products(s):
    """Block of tokens by block of tokens: act(W x + b), times the second product or plus the residual."""
    w, out = s["w"].double(), []
    up = s["w_up"].double() if s["kind"] == "gated" else None
    for at in range(0, s["n_tok"], 1024):
        x = s["x"][at:at + 1024].double().t()
        v = w @ x
        if s["bias"] is not None:
            v += s["bias"].double()[:, None]
        v = _exact_act(v, s["act"])
        if up is not None:
            u = up @ x
            v = v * (u if s["bias_up"] is None else u + s["bias_up"].double()[:, None])
        elif s["residual"] is not None:
            v = v + s["residual"][at:at + 1024].double().t()
        out.append(v.t())
    return torch.cat(out)


def _exact_rotate(s):
    """Each pair of elements as a complex number, turned by exp(i pos freq)."""
    at, c = s["offsets"].tolist(), None if s["c"] is None else s["c"].tolist()
    pos = torch.cat([torch.arange(b - a, dtype=torch.float64) + (c[i] if c else 0)
                     for i, (a, b) in enumerate(zip(at, at[1:]))]).cuda()
    freq = torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), torch.outer(pos, freq))[:, None]
    rot, half, out = s["rot"], s["rot"] // 2, {}
    j = torch.arange(half, device="cuda")
    first, second = (2 * j, 2 * j + 1) if s["order"] == "neighbours" else (j, j + half)
    for name in ("q", "k"):
        v, weight = s[name].double(), s[name + "_weight"]
        if weight is not None:
            v = v * torch.rsqrt(v.square().sum(-1, keepdim=True) / v.shape[-1] + EPS) * weight.double()
        z = torch.complex(v[..., first], v[..., second]) * turn
        v = v.clone()
        v[..., first], v[..., second] = z.real, z.imag
        out[name] = v
    return out


def _exact_logprobs(s):
    n, vocab, top = s["n_tok"], s["vocab"], min(s["top"], s["vocab"])
    parts = []
    for at in range(0, n, 256):
        v = s["x"][at:at + 256].double()
        logp = torch.log_softmax(v, 1)
        p = dict(logp=logp[torch.arange(len(v), device="cuda"), s["ids"][at:at + 256].long()],
                 entropy=-(torch.exp(logp) * logp).sum(1), lse=torch.logsumexp(v, 1))
        if top:
            picked, left = [], v.clone()
            index = torch.arange(vocab, device="cuda")
            for _ in range(top):
                best = left.amax(1, keepdim=True)
                first = torch.where(left == best, index, vocab).amin(1)
                picked.append(first)
                left.scatter_(1, first[:, None], float("-inf"))
            p["top_ids"] = torch.stack(picked, 1).int()
            p["top_logp"] = logp.gather(1, p["top_ids"].long())
        parts.append(p)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
