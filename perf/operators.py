"""The operators around the attention backward that a policy update needs, as cases that can be timed: the embedding of a
batch's tokens and its gradient, the step between two blocks of a layer (a norm after the block, its gate, the scaled
residual sum, the norm before the next block) and its gradient, and the global gradient norm with clipping.  The embedding and
the step between blocks also run in a rollout, on the rows of a decode step.

`run` computes each operator in its plain form from elementary torch operations, or, where `own` is true, through
`paper_2609_35140_b200.binding`.  Model shapes are those of the package's workloads with the FFN widths that
`bench.py` uses.  Token ids are Zipf-distributed over a scrambled vocabulary, as those of text are.
"""
import math

import numpy as np
import torch

own = False

BF, F32 = torch.bfloat16, torch.float32
DTYPES = {"bf16": BF, "fp32": F32}

# query heads, KV heads, head dim, hidden, FFN intermediate, vocabulary
MODELS = {
    "tiny": (4, 1, 64, 256, 704, 2048),
    "1.5B": (12, 2, 128, 1536, 8960, 151936),
    "7B": (28, 4, 128, 3584, 18944, 152064),
    "long": (32, 8, 128, 4096, 12288, 151936),
    "32B": (64, 8, 128, 5120, 27648, 151936),
}
EPS = 1e-6


def listed():
    return [
        # the sampled tokens of a rollout step enter the model: latency only
        {"name": "embed_decode", "kind": "embed", "model": "7B", "rows": 64, "scaled": False},
        # a batch of prompts of odd total length, embeddings scaled by sqrt(hidden)
        {"name": "embed_prompts", "kind": "embed", "model": "long", "rows": 8191, "scaled": True},
        # the smallest update step
        {"name": "embed_grad_tiny", "kind": "embed_grad", "model": "tiny", "rows": 256, "micro": 1, "dtype": "bf16", "scaled": False},
        # an update micro-batch: the gradient of the whole table is written
        {"name": "embed_grad_update", "kind": "embed_grad", "model": "7B", "rows": 16001, "micro": 1, "dtype": "bf16", "scaled": False},
        # gradient accumulation in 32 bits: the second micro-batch adds to the rows that it meets
        {"name": "embed_grad_accumulate", "kind": "embed_grad", "model": "1.5B", "rows": 6007, "micro": 2, "dtype": "fp32", "scaled": True},
        # between attention and FFN in a rollout step: latency only
        {"name": "norm_decode", "kind": "norm", "model": "7B", "rows": 64, "post": True, "gate": "channel", "next": True, "branch_scale": 1.0},
        # the same over an update micro-batch of odd size, with one weight per token
        {"name": "norm_update", "kind": "norm", "model": "32B", "rows": 9001, "post": True, "gate": "token", "next": True, "branch_scale": 0.22},
        # the smallest update step's gradients
        {"name": "norm_grad_tiny", "kind": "norm_grad", "model": "tiny", "rows": 256, "post": True, "gate": "token", "next": True, "branch_scale": 0.22},
        # gradients of an update micro-batch
        {"name": "norm_grad_update", "kind": "norm_grad", "model": "7B", "rows": 16001, "post": True, "gate": "channel", "next": True, "branch_scale": 1.0},
        # one small layer's gradients, clipped: latency only
        {"name": "clip_tiny", "kind": "clip", "model": "tiny", "layers": 1, "dtype": "bf16", "table": False, "odd": False, "limit": 0.05, "clipped": True},
        # gradients in 32 bits, some at odd addresses, below the limit: nothing is written
        {"name": "clip_below", "kind": "clip", "model": "7B", "layers": 2, "dtype": "fp32", "table": False, "odd": True, "limit": 1000.0, "clipped": False},
        # a whole model's gradients, clipped on their way into the optimiser's buffer
        {"name": "clip_model", "kind": "clip", "model": "1.5B", "layers": 28, "dtype": "bf16", "table": True, "odd": False, "limit": 1.0, "clipped": True},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"]


def _draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm", "norm_grad", "norm_grad", "clip", "clip"])
    c = {"kind": kind, "model": rng.choice(["tiny", "1.5B", "7B", "long", "32B"])}
    if kind == "clip":
        c["layers"] = _log_uniform(rng, 1, 64)
        c["dtype"] = rng.choice(["bf16", "bf16", "fp32", "mixed"])
        c["table"], c["odd"], c["clipped"] = rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.6
        c["limit"] = rng.choice([0.01, 0.05]) if c["clipped"] else 1000.0
        return c
    c["rows"] = _log_uniform(rng, 1, 32768)
    if kind in ("embed", "embed_grad"):
        c["scaled"] = rng.random() < 0.5
        if kind == "embed_grad":
            c["dtype"] = rng.choice(["bf16", "fp32"])
            c["micro"] = rng.choice([1, 2, 3]) if c["dtype"] == "fp32" else 1
        return c
    c["post"], c["gate"] = rng.random() < 0.7, rng.choice(["none", "channel", "token"])
    c["next"], c["branch_scale"] = rng.random() < 0.85, rng.choice([1.0, 0.22, -0.5])
    return c


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most:
            return c


class _Tensors:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape, std=1.0, mean=0.0, dtype=BF):
        out = torch.empty(shape, dtype=dtype, device="cuda")
        step = max(1, (1 << 26) // max(1, math.prod(shape[1:])))
        for r in range(0, shape[0], step):
            part = torch.randn((min(step, shape[0] - r),) + shape[1:], generator=self.g, device="cuda")
            out[r:r + step] = part.mul_(std).add_(mean)
        return out

    def ids(self, n, V):
        """Rank r with probability log((r + 2) / (r + 1)) / log(V + 1), ranks scattered over the vocabulary."""
        u = torch.rand(n, generator=self.g, device="cuda", dtype=torch.float64)
        rank = (torch.exp(u * math.log(V + 1)) - 1).long().clamp_(0, V - 1)
        return ((rank * 40009 + 12345) % V).to(torch.int32)


def _distinct(n, V):
    """Expected number of distinct ids among n."""
    r = np.arange(1, V + 1, dtype=np.float64)
    p = np.log1p(1.0 / r) / math.log(V + 1)
    return float(-np.expm1(n * np.log1p(-p)).sum())


def _shapes(case):
    """(name, numbers of elements) of the gradients that a clip sees, and their types."""
    Hq, Hkv, d, H, inter, V = MODELS[case["model"]]
    sizes = []
    if case["table"]:
        sizes.append(V * H)
    for _ in range(case["layers"]):
        if case["odd"]:
            sizes.append(1)                            # a learned branch scale: what follows it loses its alignment
        sizes += [H, Hq * d * H, Hkv * d * H, Hkv * d * H, H * Hq * d, H, 2 * inter * H, H * inter]
    sizes.append(H)
    kinds = [("fp32" if i % 3 == 0 else "bf16") if case["dtype"] == "mixed" else case["dtype"] for i in range(len(sizes))]
    return sizes, kinds


def _flat_grads(case, t):
    """Gradients as views of one flat buffer per type, in the model's order."""
    sizes, kinds = _shapes(case)
    flats = {k: t.normal(max(1, sum(n for n, kk in zip(sizes, kinds) if kk == k)), std=1e-3, dtype=DTYPES[k])
             for k in sorted(set(kinds))}
    if case["table"]:                                  # most tokens of a vocabulary do not occur in a batch
        V, H = MODELS[case["model"]][5], MODELS[case["model"]][3]
        rows = torch.rand(V, generator=t.g, device="cuda") < 0.1
        flats[kinds[0]][:V * H].view(V, H).mul_(rows.to(DTYPES[kinds[0]])[:, None])
    return flats, _views(case, flats)


def _views(case, flats):
    sizes, kinds = _shapes(case)
    at, views = {k: 0 for k in flats}, []
    for n, k in zip(sizes, kinds):
        views.append(flats[k][at[k]:at[k] + n])
        at[k] += n
    return views


def prepare(case, seed):
    Hq, Hkv, d, H, inter, V = MODELS[case["model"]]
    t, kind = _Tensors(seed), case["kind"]
    s = {"kind": kind, "case": dict(case)}
    if kind == "clip":
        s["flats"], s["grads"] = _flat_grads(case, t)
        s["limit"] = case["limit"]
        if case["clipped"]:
            s["out_flats"] = {k: torch.empty_like(f) for k, f in s["flats"].items()}
            s["out"] = _views(case, s["out_flats"])
        return s
    T = case["rows"]
    if kind in ("embed", "embed_grad"):
        s["scale"] = math.sqrt(H) if case["scaled"] else 1.0
        if kind == "embed":
            s.update(ids=t.ids(T, V), table=t.normal(V, H, std=0.02))
        else:
            s.update(vocab=V, micro=[(t.normal(T, H, std=1e-3), t.ids(T, V)) for _ in range(case["micro"])],
                     d_table=torch.empty(V, H, dtype=DTYPES[case["dtype"]], device="cuda"))
        return s
    s.update(x=t.normal(T, H, std=2.0), branch_scale=case["branch_scale"], weight=None, post=None, gate=None)
    if case["next"]:
        s["weight"] = t.normal(H, std=0.2, mean=1.0)
    if case["post"]:
        s["post"] = t.normal(H, std=0.2, mean=1.0)
    if case["gate"] != "none":
        s["gate"] = t.normal(H, std=0.3, mean=0.5) if case["gate"] == "channel" else t.normal(T, 1, std=0.3, mean=0.5)
    if kind == "norm":
        s["residual"] = t.normal(T, H, std=4.0)
    else:
        s.update(stream=t.normal(T, H, std=4.0), d_stream=t.normal(T, H, std=1e-3),
                 d_y=t.normal(T, H, std=1e-3) if case["next"] else None)
    return s


# ---------------------------------------------------------------- plain forms

def _inv_rms(v):
    return torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS)


def _branch(s):
    """x after its norm, and the factor of the gate."""
    x = s["x"].float()
    n = x * _inv_rms(x) * s["post"].float() if s["post"] is not None else x
    return n, s["branch_scale"] * (s["gate"].float() if s["gate"] is not None else 1.0)


def _plain_norm(s):
    n, f = _branch(s)
    stream = (s["residual"].float() + f * n).to(BF)
    out = {"stream": stream}
    if s["weight"] is not None:
        v = stream.float()
        out["y"] = (v * _inv_rms(v) * s["weight"].float()).to(BF)
    return out


def _plain_norm_grad(s):
    out = {}
    G = s["d_stream"].float()
    if s["weight"] is not None:
        v, dy = s["stream"].float(), s["d_y"].float()
        r = _inv_rms(v)
        v = v * r
        out["d_weight"] = (dy * v).sum(0)
        q = dy * s["weight"].float()
        G = G + r * (q - v * (q * v).mean(-1, keepdim=True))
    n, f = _branch(s)
    dn = f * G
    if s["gate"] is not None:
        dg = s["branch_scale"] * (G * n)
        out["d_gate"] = dg.sum(0) if s["gate"].dim() == 1 else dg.sum(1, keepdim=True)
    out["d_residual"] = G.to(BF)
    if s["post"] is not None:
        x = s["x"].float()
        r = _inv_rms(x)
        x = x * r
        out["d_post_weight"] = (dn * x).sum(0)
        p = dn * s["post"].float()
        dn = r * (p - x * (p * x).mean(-1, keepdim=True))
    out["d_x"] = dn.to(BF)
    return out


def _plain_clip(s):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for g in s["grads"]:
        total += g.float().square().sum(dtype=torch.float64)
    norm = total.sqrt().float().reshape(1)
    if "out" in s:
        coef = torch.where(norm > s["limit"], s["limit"] / norm, torch.ones_like(norm))
        for g, o in zip(s["grads"], s["out"]):
            o.copy_(g.float() * coef)
        return {"norm": norm, "grads": s["out_flats"]}
    return {"norm": norm, "grads": s["flats"]}       # below the limit the gradients stay


def _plain_embed_grad(s):
    acc = torch.zeros(s["vocab"], s["micro"][0][0].shape[1], device="cuda")
    for dy, ids in s["micro"]:
        acc.index_add_(0, ids, dy.float())
    return s["d_table"].copy_(acc.mul_(s["scale"]))


# ---------------------------------------------------------------- one pass

def _own(s):
    from paper_2609_35140_b200 import binding as tik
    kind = s["kind"]
    if kind == "embed":
        return tik.tik_embedding(s["ids"], s["table"], s["scale"])
    if kind == "embed_grad":
        for i, (dy, ids) in enumerate(s["micro"]):
            tik.tik_embedding_bwd(dy, ids, s["vocab"], s["scale"], d_table=s["d_table"], accumulate=i > 0)
        return s["d_table"]
    if kind == "norm":
        y, stream = tik.tik_block_norm(s["x"], s["residual"], s["weight"], EPS, post_weight=s["post"], gate=s["gate"],
                                       branch_scale=s["branch_scale"])
        return {"stream": stream} if y is None else {"stream": stream, "y": y}
    if kind == "norm_grad":
        got = tik.tik_block_norm_bwd(s["d_y"], s["d_stream"], s["x"], s["stream"], s["weight"], EPS, post_weight=s["post"],
                                     gate=s["gate"], branch_scale=s["branch_scale"])
        names = ("d_x", "d_residual", "d_weight", "d_post_weight", "d_gate")
        return {k: v for k, v in zip(names, got) if v is not None}
    if "out" in s:
        return {"norm": tik.tik_grad_clip(s["grads"], s["limit"], out=s["out"]), "grads": s["out_flats"]}
    return {"norm": tik.tik_grad_clip(s["grads"], s["limit"]), "grads": s["flats"]}


def run(state):
    s = state
    if own:
        return _own(s)
    kind = s["kind"]
    if kind == "embed":
        return (s["table"][s["ids"]].float() * s["scale"]).to(BF)
    return {"embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "clip": _plain_clip}[kind](s)


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_norm_rows(v, w):
    return v / torch.sqrt((v * v).sum(1, keepdim=True) / v.shape[1] + EPS) * w


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    D = torch.float64
    if kind == "embed":
        return s["table"].index_select(0, s["ids"].long()).to(D) * s["scale"]
    if kind == "embed_grad":
        out = torch.zeros(s["vocab"], s["d_table"].shape[1], dtype=D, device="cuda")
        for dy, ids in s["micro"]:
            out.index_put_((ids.long(),), dy.to(D) * s["scale"], accumulate=True)
        return out
    if kind == "clip":
        total = sum(float((f[i:i + (1 << 26)].to(D) ** 2).sum()) for f in s["flats"].values() for i in range(0, f.numel(), 1 << 26))
        norm = math.sqrt(total)
        c = s["limit"] / norm if norm > s["limit"] else 1.0
        return {"norm": torch.tensor([norm], dtype=D, device="cuda"),
                "grads": {k: (f.to(D) * c if s["case"]["clipped"] else f) for k, f in s["flats"].items()}}
    a, x = s["branch_scale"], s["x"].to(D)
    g = torch.ones(1, 1, dtype=D, device="cuda") if s["gate"] is None else s["gate"].to(D).reshape(1, -1) if s["gate"].dim() == 1 else s["gate"].to(D)
    n = x if s["post"] is None else _exact_norm_rows(x, s["post"].to(D))
    if kind == "norm":
        stream = s["residual"].to(D) + a * g * n
        out = {"stream": stream}
        if s["weight"] is not None:
            out["y"] = _exact_norm_rows(stream.to(BF).to(D), s["weight"].to(D))
        return out
    # gradients: the Jacobian of v -> v / rms(v) o w, transposed
    def back(d, v, w):
        H = v.shape[1]
        rms = torch.sqrt((v * v).sum(1, keepdim=True) / H + EPS)
        return d * w / rms - v * ((d * w * v).sum(1, keepdim=True) / (H * rms ** 3)), (d * v / rms).sum(0)
    out, G = {}, s["d_stream"].to(D)
    if s["weight"] is not None:
        more, out["d_weight"] = back(s["d_y"].to(D), s["stream"].to(D), s["weight"].to(D))
        G = G + more
    out["d_residual"], dn = G, a * g * G
    if s["gate"] is not None:
        out["d_gate"] = (a * G * n).sum(0) if s["gate"].dim() == 1 else (a * G * n).sum(1, keepdim=True)
    if s["post"] is not None:
        out["d_x"], out["d_post_weight"] = back(dn, x, s["post"].to(D))
    else:
        out["d_x"] = dn
    return out


def work(case):
    Hq, Hkv, d, H, inter, V = MODELS[case["model"]]
    kind = case["kind"]
    if kind == "clip":
        sizes, kinds = _shapes(case)
        size = float(sum(n * (2 if k == "bf16" else 4) for n, k in zip(sizes, kinds)))
        # the norm has to be known before the first gradient is scaled: what is scaled is read again
        return {"bytes": size * (3 if case["clipped"] else 1), "flops": sum(sizes) * (3.0 if case["clipped"] else 2.0)}
    T = case["rows"]
    if kind == "embed":
        return {"bytes": 2.0 * H * (T + _distinct(T, V)) + 4.0 * T, "flops": float(T * H)}
    if kind == "embed_grad":
        e, m = (2.0 if case["dtype"] == "bf16" else 4.0), case["micro"]
        return {"bytes": m * (2.0 * T * H + 4.0 * T) + e * V * H + (m - 1) * 2 * e * H * _distinct(T, V), "flops": float(m * T * H)}
    planes = 4 if kind == "norm" else 6
    planes -= 0 if case["next"] else 1 if kind == "norm" else 2         # no y; no d_y and no stream to read
    return {"bytes": 2.0 * planes * T * H + 8.0 * H, "flops": (10.0 if kind == "norm" else 30.0) * T * H}
