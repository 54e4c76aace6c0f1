"""The operators around attention in a serving step of ragged requests, as measurable cases.

A server of requests that differ in length, adapter and sampling settings needs, beside attention and its cache:
tokens drawn with a temperature, top-k, top-p and min-p of each row's own from given random numbers (kind "sample"),
projections whose shared weights are joined by the low-rank adapter of each request (kind "lora"), and the norms between
the blocks of a layer with the residual add (kind "norm").

``run`` computes each in elementary torch operations, in 32 bits (sampling in 64: a draw next to the border of two
tokens, or a cut next to the border of a nucleus, must not depend on rounding), or, where ``own`` is true, with the
framework's operators.  ``exact`` restates each from its definition in 64 bits.  Widths and vocabularies are those of the
presets in ``workloads``: tiny d 256, V 1024 (fp32); small 768, 32768; block 2048, 128000; posttrain 5376, 262144.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

# width, rows of the QKV projection, vocabulary, type of the activations
DIMS = {"tiny": (256, 768, 1024, "f32"), "small": (768, 2304, 32768, "bf16"), "block": (2048, 4096, 128000, "bf16"),
        "posttrain": (5376, 8192, 262144, "bf16")}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
PROMPTS = "512,33,300,1,127,480,64,211,512,95,402,17,256,350,129,512,5,444,190,63,371,288,500,12"


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # One request's next token, the usual settings of a chat server: the latency of a single draw.
        {"name": "sample_small_token", "kind": "sample", "vocab": 32768, "rows": 1, "type": "f32", "shape": "peaked",
         "settings": "nucleus", "mask": True},
        # The next tokens of 64 requests with settings of their own: greedy, top-k, nucleus, min-p, plain temperature.
        {"name": "sample_block_mixed", "kind": "sample", "vocab": 128000, "rows": 64, "type": "f32", "shape": "peaked",
         "settings": "mixed", "mask": True},
        # Canvas rows of the 27 B model early in a generation: bf16 logits near a flat distribution, with many ties and a
        # nucleus of most of the vocabulary.
        {"name": "sample_posttrain_flat", "kind": "sample", "vocab": 262144, "rows": 33, "type": "bf16", "shape": "flat",
         "settings": "nucleus", "mask": True},
        # Every canvas row of 16 sequences of 32, drawn at once with a nucleus: the bytes of the logits.
        {"name": "sample_block_canvas", "kind": "sample", "vocab": 128000, "rows": 512, "type": "f32", "shape": "peaked",
         "settings": "nucleus", "mask": True},
        # Four short prompts of the fp32 model, two adapters.
        {"name": "lora_tiny_f32", "kind": "lora", "n_in": 256, "n_out": 768, "type": "f32", "rank": 8, "adapters": 2,
         "rows": "32,7,128,61", "spare": 0},
        # The QKV projection of one new token for each of 64 requests with 40 adapters: weights and adapters are read once.
        {"name": "lora_block_tokens", "kind": "lora", "n_in": 2048, "n_out": 4096, "type": "bf16", "rank": 16,
         "adapters": 40, "rows": ",".join(["1"] * 64), "spare": 0},
        # The same projection over a prefill of 24 prompts with 6 adapters, in a buffer with a few rows to spare.
        {"name": "lora_block_prompts", "kind": "lora", "n_in": 2048, "n_out": 4096, "type": "bf16", "rank": 16,
         "adapters": 6, "rows": PROMPTS, "spare": 26},
        # A block step of the 27 B model, 8 requests of 32 rows with adapters of rank 64.
        {"name": "lora_posttrain_step", "kind": "lora", "n_in": 5376, "n_out": 8192, "type": "bf16", "rank": 64,
         "adapters": 7, "rows": ",".join(["32"] * 8), "spare": 0},
        # The norms around one token of the small model: latency.
        {"name": "norm_small_token", "kind": "norm", "d": 768, "x": "f32", "y": "f32", "type": "bf16", "rows": "1",
         "spare": 0, "post": True, "gate": False, "scale": 1.0},
        # A block step of 32 sequences with a gate of each sequence's own, the residual stream in bf16.
        {"name": "norm_block_step", "kind": "norm", "d": 2048, "x": "bf16", "y": "bf16", "type": "bf16",
         "rows": ",".join(["32"] * 32), "spare": 0, "post": False, "gate": True, "scale": 0.5},
        # Sandwich norms over a prefill of the 27 B model: fp32 residual stream, the block's output in bf16.
        {"name": "norm_posttrain_prompts", "kind": "norm", "d": 5376, "x": "f32", "y": "bf16", "type": "bf16",
         "rows": "8111,900,1,2500", "spare": 37, "post": True, "gate": False, "scale": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "sample", "lora", "lora", "norm"])
    if kind == "sample":
        vocab = rng.choice([rng.randint(2, 1024), 32768, _log(rng, 1000, 262144), 128000, 262144])
        return {"kind": kind, "vocab": vocab, "rows": _log(rng, 1, max(1, min(512, 60_000_000 // vocab))),
                "type": rng.choice(["f32", "f32", "bf16"]), "shape": rng.choice(["peaked", "peaked", "flat"]),
                "settings": rng.choice(["mixed", "mixed", "nucleus", "topk", "temperature", "minp", "greedy"]),
                "mask": rng.random() < 0.5}
    if kind == "lora":
        name = rng.choice(["tiny", "small", "block", "block", "posttrain"])
        d, qkv, _, kind_of = DIMS[name]
        n_in, n_out = rng.choice([(d, qkv), (d, d), (d, 8 * rng.randint(1, d // 4)), (8 * rng.randint(2, d // 8), d)])
        n = _log(rng, 1, 64)
        most = rng.choice([1, 1, 32, 500])
        rows = [most if most <= 32 and rng.random() < 0.7 else rng.randint(0, most) for _ in range(n)]
        while sum(rows) > (600 if name in ("tiny", "posttrain") else 6000):
            rows.pop()
        if not any(rows):
            rows = [most]
        return {"kind": kind, "n_in": n_in, "n_out": n_out, "type": kind_of, "rank": rng.choice([8, 16, 16, 24, 64, 128]),
                "adapters": _log(rng, 1, 64), "rows": ",".join(map(str, rows)), "spare": rng.choice([0, 0, 5, 100])}
    d = rng.choice([768, 2048, 5376, rng.randint(1, 6000)])
    rows = [_log(rng, 1, 2000) - 1 for _ in range(_log(rng, 1, 32))]
    while sum(rows) > 11000:
        rows.pop()
    if not any(rows):
        rows = [3]
    return {"kind": kind, "d": d, "x": rng.choice(["f32", "f32", "bf16"]), "y": rng.choice(["f32", "bf16"]),
            "type": rng.choice(["bf16", "bf16", "f32"]), "rows": ",".join(map(str, rows)), "spare": rng.choice([0, 0, 9]),
            "post": rng.random() < 0.5, "gate": rng.random() < 0.5, "scale": rng.choice([1.0, 0.5, 0.7071])}


# ------------------------------------------------------------------ inputs
def _ints(text):
    return [int(v) for v in str(text).split(",")]


def _cum(values):
    out = [0]
    for v in values:
        out.append(out[-1] + v)
    return out


def _of_rows(case):
    """First row of each sequence, and one past the last sequence's; rows of the buffers."""
    cu = _cum(_ints(case["rows"]))
    return cu, cu[-1] + case["spare"]


def _adapter(case, b):
    """Sequence b's adapter, -1 for none: every one has its turn."""
    return b % (case["adapters"] + 1) - 1


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _settings(kind, rows, g):
    """Per row: temperature, top-k (0: all), top-p and min-p (1 and 0: off)."""
    def pick(*of):
        return torch.tensor(of, device="cuda")[torch.randint(0, len(of), (rows,), generator=g, device="cuda")]

    one, none = torch.ones(rows, device="cuda"), torch.zeros(rows, device="cuda")
    off = torch.zeros(rows, dtype=torch.int32, device="cuda")
    if kind == "greedy":
        return none, off, one, none
    if kind == "temperature":
        return pick(0.7, 1.0, 1.3), off, one, none
    if kind == "topk":
        return pick(0.7, 1.0), pick(1, 20, 50, 1000).to(torch.int32), one, none
    if kind == "nucleus":
        return pick(0.8, 1.0), off, pick(0.8, 0.9, 0.95), none
    if kind == "minp":
        return pick(0.8, 1.0, 1.5), off, one, pick(0.02, 0.05, 0.1)
    return (pick(0.0, 0.6, 0.8, 1.0, 1.3), pick(0, 0, 1, 40, 200).to(torch.int32), pick(1.0, 1.0, 0.95, 0.9, 0.5),
            pick(0.0, 0.0, 0.05))


def prepare(case, seed):
    g = _gen(seed)
    s = SimpleNamespace(case=case)
    kind = case["kind"]

    def rand(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if kind == "sample":
        rows, vocab = case["rows"], case["vocab"]
        x = rand(rows, vocab)
        if case["shape"] == "peaked":          # a trained head's row: a long tail, and a few tokens far above it
            x.mul_(2.0)
            top = torch.randint(0, vocab, (rows, 12), generator=g, device="cuda")
            x.scatter_add_(1, top, 6.0 + 3.0 * rand(rows, 12))
        s.logits = x.to(TYPES[case["type"]])
        s.mask_id = vocab - 1 if case["mask"] else -1
        s.temperature, s.top_k, s.top_p, s.min_p = _settings(case["settings"], rows, g)
        s.u = torch.rand(rows, generator=g, device="cuda")
        s.tok = torch.empty(rows, dtype=torch.int32, device="cuda")
        s.prob = torch.empty(rows, dtype=torch.float32, device="cuda")
    elif kind == "lora":
        t, n_in, n_out, r, n = TYPES[case["type"]], case["n_in"], case["n_out"], case["rank"], case["adapters"]
        cu, total = _of_rows(case)
        s.x = rand(total, n_in).to(t)
        s.w = (rand(n_out, n_in) / math.sqrt(n_in)).to(t)
        s.a = (rand(n, r, n_in) / math.sqrt(n_in)).to(t)
        s.b = (0.5 * rand(n, n_out, r) / math.sqrt(r)).to(t)
        s.scale = torch.exp(0.3 * rand(n))
        s.y = torch.zeros((total, n_out), dtype=t, device="cuda")
        s.cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
        s.adapter = torch.tensor([_adapter(case, b) for b in range(len(cu) - 1)], dtype=torch.int32, device="cuda")
    else:
        d, t = case["d"], TYPES[case["type"]]
        cu, total = _of_rows(case)
        s.x = (2.0 * rand(total, d)).to(TYPES[case["x"]])
        s.y = (rand(total, d) * torch.exp(0.5 * rand(total, 1))).to(TYPES[case["y"]])
        s.post = (1 + 0.1 * rand(d)).to(t) if case["post"] else None
        s.pre = (1 + 0.1 * rand(d)).to(t)
        s.gate = rand(len(cu) - 1, d).to(t) if case["gate"] else None
        s.x_out, s.n_out = torch.zeros_like(s.x), torch.zeros((total, d), dtype=t, device="cuda")
        s.cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    if own:
        import paper_2609_37924_gb300.tadm as T
        s.T = T
        if kind == "lora":
            need = T.tadm_lora_scratch_size(s.cu.numel() - 1, s.x.shape[0], case["n_in"], case["n_out"], case["adapters"],
                                            case["rank"], 1 if case["type"] == "bf16" else 0)
            s.scratch = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ one pass
EPS = 1e-6


def run(s):
    kind = s.case["kind"]
    if not own:
        return {"sample": _plain_sample, "lora": _plain_lora, "norm": _plain_norm}[kind](s)
    T = s.T
    if kind == "sample":
        T.tadm_sample(s.logits, s.u, s.tok, temperature=s.temperature, top_k=s.top_k, top_p=s.top_p, min_p=s.min_p,
                      prob=s.prob, mask_id=s.mask_id)
        return s.tok, s.prob
    if kind == "lora":
        T.tadm_lora_project(s.x, s.w, s.y, s.cu, s.adapter, s.a, s.b, s.scale, s.scratch)
        return s.y
    T.tadm_residual_norm(s.x, s.y, s.x_out, s.n_out, cu_rows=s.cu, post_gain=s.post, gate=s.gate, pre_gain=s.pre,
                         residual_scale=s.case["scale"], eps=EPS)
    return s.x_out, s.n_out


def _plain_sample(s):
    """A row's ids in falling order of their logits (ties: rising id), of which top-k, min-p and top-p each keep a first
    part; then the first kept id, in the order of ids, whose cumulative weight exceeds u times the mass kept."""
    x = s.logits.double()
    if s.mask_id >= 0:
        x[:, s.mask_id] = -math.inf
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    x, ids = torch.sort(x, dim=1, descending=True, stable=True)
    t = s.temperature.double()[:, None]
    greedy = t <= 2.0 ** -100
    w = torch.exp((x - x[:, :1]) / torch.where(greedy, torch.ones_like(t), t))
    rank = torch.arange(x.shape[1], device=x.device)
    k = torch.where(s.top_k > 0, s.top_k, x.shape[1])[:, None]
    keep = (rank < torch.where(greedy, torch.ones_like(k), k)) & (w >= s.min_p.double()[:, None]) & (x > -math.inf)
    w = w * keep
    cum = torch.cumsum(w, 1)
    p = s.top_p.double()[:, None]
    w = w * ((cum - w < p * cum[:, -1:]) | (p >= 1) | (rank == 0))
    w = torch.zeros_like(w).scatter_(1, ids, w)
    cum = torch.cumsum(w, 1)
    past = cum > s.u.double()[:, None] * cum[:, -1:]
    tok = past.to(torch.uint8).argmax(1, keepdim=True)
    s.tok.copy_(tok[:, 0])
    s.prob.copy_((w.gather(1, tok) / cum[:, -1:])[:, 0])
    return s.tok, s.prob


def _plain_lora(s):
    """y = W x + scale_a B_a (A_a x), a the adapter of the row's sequence; rows behind the last sequence stay."""
    cu, _ = _of_rows(s.case)
    x = s.x[:cu[-1]].float()
    y = x @ s.w.float().T
    for a in range(s.case["adapters"]):
        rows = [torch.arange(cu[b], cu[b + 1], device=x.device) for b in range(len(cu) - 1) if _adapter(s.case, b) == a]
        if rows:
            at = torch.cat(rows)
            y[at] += (x[at] @ s.a[a].float().T) @ s.b[a].float().T * s.scale[a]
    s.y[:cu[-1]] = y.to(s.y.dtype)
    return s.y


def _plain_norm(s):
    """x' = scale x + gate u, u = y or its RMS norm times a gain; n = the RMS norm of x' times a gain."""
    cu, _ = _of_rows(s.case)
    n = cu[-1]
    u = s.y[:n].float()
    if s.post is not None:
        u = u * torch.rsqrt(u.square().mean(-1, keepdim=True) + EPS) * s.post.float()
    if s.gate is not None:
        seq = torch.searchsorted(s.cu[1:].contiguous(), torch.arange(n, dtype=torch.int32, device=u.device), right=True)
        u = u * s.gate.float()[seq]
    x = s.x[:n].float() * s.case["scale"] + u
    s.x_out[:n] = x.to(s.x_out.dtype)
    s.n_out[:n] = (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * s.pre.float()).to(s.n_out.dtype)
    return s.x_out, s.n_out


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size[case["type"]] + case["rows"] * 28, "flops": 4.0 * n}
    cu, _ = _of_rows(case)
    n, e = cu[-1], size[case["type"]]
    if case["kind"] == "lora":
        i, o, r = case["n_in"], case["n_out"], case["rank"]
        with_one = [b for b in range(len(cu) - 1) if _adapter(case, b) >= 0 and cu[b + 1] > cu[b]]
        adapted = sum(cu[b + 1] - cu[b] for b in with_one)
        used = len({_adapter(case, b) for b in with_one})
        return {"bytes": e * (n * (i + o) + i * o + used * r * (i + o)), "flops": 2.0 * n * i * o + 2.0 * adapted * r * (i + o)}
    d = case["d"]
    gates = (len(cu) - 1) * d * e if case["gate"] else 0
    return {"bytes": n * d * (2 * size[case["x"]] + size[case["y"]] + e) + gates + 2 * d * e, "flops": 12.0 * n * d}


# ------------------------------------------------------------------ exact
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(s)
    cu, total = _of_rows(case)
    if case["kind"] == "lora":
        y = torch.zeros((total, case["n_out"]), dtype=torch.float64, device="cuda")
        w = s.w.double()
        for b in range(len(cu) - 1):
            x, a = s.x[cu[b]:cu[b + 1]].double(), _adapter(case, b)
            out = torch.einsum("ti,oi->to", x, w)
            if a >= 0:
                out += torch.einsum("tr,or->to", torch.einsum("ti,ri->tr", x, s.a[a].double()), s.b[a].double()) * s.scale[a].double()
            y[cu[b]:cu[b + 1]] = out
        return y
    x_out = torch.zeros((total, case["d"]), dtype=torch.float64, device="cuda")
    n_out = torch.zeros_like(x_out)
    for b in range(len(cu) - 1):
        at = slice(cu[b], cu[b + 1])
        u = s.y[at].double()
        if s.post is not None:
            u = u / torch.sqrt((u * u).sum(-1, keepdim=True) / case["d"] + EPS) * s.post.double()
        if s.gate is not None:
            u = u * s.gate[b].double()
        x = case["scale"] * s.x[at].double() + u
        x_out[at] = x
        n_out[at] = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + EPS) * s.pre.double()
    return x_out, n_out


def _exact_sample(s):
    """Row by row on the host: thresholds found by a search over sorted weights, the draw by one over the kept ids' sums."""
    if s.logits.numel() > 70_000_000:
        return None
    logits = s.logits.float().cpu().numpy()
    t, k, p, m, u = (v.double().cpu().numpy() for v in (s.temperature, s.top_k, s.top_p, s.min_p, s.u))
    toks, probs = [], []
    for r in range(logits.shape[0]):
        ids = np.arange(logits.shape[1])
        ids = ids[(logits[r] > -np.inf) & (ids != s.mask_id)]
        x = logits[r][ids].astype(np.float64)
        if t[r] <= 2.0 ** -100:
            toks.append(int(ids[np.argmax(x)]))
            probs.append(1.0)
            continue
        w = np.exp((x - x.max()) / t[r])
        order = np.argsort(-x, kind="stable")
        n = len(order) if k[r] <= 0 else min(int(k[r]), len(order))
        n = max(1, min(n, int(np.count_nonzero(w >= m[r]))))
        sums = np.cumsum(w[order[:n]])
        if p[r] < 1:
            n = int(np.searchsorted(sums, p[r] * sums[-1], side="left")) + 1
        kept = np.sort(order[:n])
        sums = np.cumsum(w[kept])
        at = int(np.searchsorted(sums, u[r] * sums[-1], side="right"))
        at = min(at, len(kept) - 1)
        toks.append(int(ids[kept[at]]))
        probs.append(w[kept[at]] / sums[-1])
    return (torch.tensor(toks, dtype=torch.int32, device="cuda"),
            torch.tensor(probs, dtype=torch.float64, device="cuda"))
