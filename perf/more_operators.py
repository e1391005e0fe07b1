"""The two ends of a policy update's backward pass that a trainer brought along itself, as cases that can be timed: the clipped
policy loss with its KL term and its gradient, the gradient of the token log-probabilities (with respect to the hidden rows and
to lm_head), and the AdamW step over all of a model's tensors, with its states in 32 or in 8 bits.

`run` computes each operator in its plain form from elementary torch operations, or, where `own` is true, through
`paper_2609_35140_b200.binding`.  Model shapes are those of the package's workloads with the FFN widths that `bench.py` uses.
Log-probabilities are those of sampled tokens under a policy that has moved a little since; hidden rows lean towards their
target's row of lm_head, so that a target's probability is anything between nothing and one, as in a text.
"""
import math

import torch

own = False

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
FP8, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
DTYPES = {"bf16": BF, "fp32": F32}

# query heads, KV heads, head dim, hidden, FFN intermediate, vocabulary
MODELS = {
    "tiny": (4, 1, 64, 256, 704, 2048),
    "1.5B": (12, 2, 128, 1536, 8960, 151936),
    "7B": (28, 4, 128, 3584, 18944, 152064),
    "long": (32, 8, 128, 4096, 12288, 151936),
    "32B": (64, 8, 128, 5120, 27648, 151936),
}
BETA1, BETA2, ADAM_EPS, DECAY = 0.9, 0.999, 1e-8, 0.1
BLOCK = 32                                             # elements that share a scale of an 8-bit state


def listed():
    return [
        # one short response per prompt of a small update step: latency only
        {"name": "loss_tiny", "kind": "loss", "tokens": 256, "seqs": 4, "reduction": "token", "per_seq": False, "weight": False,
         "ref": False, "dual": False},
        # a group-relative update: an advantage per response, prompts masked, a KL term, the mean over responses of their means
        {"name": "loss_group", "kind": "loss", "tokens": 60013, "seqs": 64, "reduction": "sequence", "per_seq": True, "weight": True,
         "ref": True, "dual": False},
        # a whole batch at once, advantages per token, importance weights, three thresholds
        {"name": "loss_batch", "kind": "loss", "tokens": 1000003, "seqs": 1024, "reduction": "token", "per_seq": False, "weight": True,
         "ref": True, "dual": True},
        # the smallest update step
        {"name": "head_tiny", "kind": "head", "model": "tiny", "rows": 256, "temperature": 1.0, "hidden": True, "table": True},
        # a short micro-batch: lm_head and its gradient are most of the bytes
        {"name": "head_short", "kind": "head", "model": "1.5B", "rows": 501, "temperature": 1.0, "hidden": True, "table": True},
        # an update micro-batch of odd size
        {"name": "head_update", "kind": "head", "model": "7B", "rows": 4001, "temperature": 1.0, "hidden": True, "table": True},
        # a frozen lm_head: the gradient of the hidden rows alone
        {"name": "head_frozen", "kind": "head", "model": "32B", "rows": 2000, "temperature": 0.8, "hidden": True, "table": False},
        # one small layer: latency only
        {"name": "adamw_tiny", "kind": "adamw", "model": "tiny", "layers": 1, "tied": False, "param": "fp32", "grad": "fp32", "master": False,
         "state": 32, "stochastic": False, "clip": False, "odd": False},
        # weights in bf16 beside a master copy in 32 bits, states in 32 bits, the clip's factor on the way
        {"name": "adamw_master", "kind": "adamw", "model": "1.5B", "layers": 12, "tied": True, "param": "bf16", "grad": "bf16", "master": True,
         "state": 32, "stochastic": False, "clip": True, "odd": False},
        # everything in 32 bits, in one flat buffer in which learned scalars shift the tensors behind them
        {"name": "adamw_odd", "kind": "adamw", "model": "7B", "layers": 1, "tied": False, "param": "fp32", "grad": "fp32", "master": False,
         "state": 32, "stochastic": False, "clip": True, "odd": True},
        # the least memory: weights in bf16 alone and states in 8 bits, rounded stochastically
        {"name": "adamw_8bit", "kind": "adamw", "model": "7B", "layers": 2, "tied": False, "param": "bf16", "grad": "bf16", "master": False,
         "state": 8, "stochastic": True, "clip": True, "odd": False},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 6e12 + w["flops"] / 1.4e15


def _draw(rng):
    kind = rng.choice(["loss", "head", "adamw"])
    c = {"kind": kind}
    if kind == "loss":
        c["tokens"] = _log_uniform(rng, 1, 1 << 20)
        c["seqs"] = min(c["tokens"], _log_uniform(rng, 1, 2048))
        c["reduction"] = rng.choice(["token", "sequence", "sum"])
        for flag, share in (("per_seq", 0.5), ("weight", 0.7), ("ref", 0.6), ("dual", 0.4)):
            c[flag] = rng.random() < share
        return c
    c["model"] = rng.choice(list(MODELS))
    if kind == "head":
        c["rows"], c["temperature"] = _log_uniform(rng, 1, 16384), rng.choice([1.0, 1.0, 0.7, 1.3])
        c["hidden"], c["table"] = rng.choice([(True, True), (True, True), (True, False), (False, True)])
        return c
    c["layers"], c["tied"] = _log_uniform(rng, 1, 32), rng.random() < 0.3
    c["param"], c["state"] = rng.choice(["bf16", "fp32"]), rng.choice([32, 8])
    c["grad"] = rng.choice(["bf16", "fp32"])
    c["master"] = c["param"] == "bf16" and rng.random() < 0.5
    c["stochastic"] = (c["state"] == 8 or (c["param"] == "bf16" and not c["master"])) and rng.random() < 0.7
    c["clip"], c["odd"] = rng.random() < 0.6, c["state"] == 32 and rng.random() < 0.3
    return c


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    while True:
        c = _draw(rng)
        if _cost(c) <= most[c["kind"]]:
            return c


class _Tensors:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape, std=1.0, mean=0.0, dtype=F32):
        out = torch.empty(shape, dtype=dtype, device="cuda")
        step = max(1, (1 << 26) // max(1, math.prod(shape[1:])))
        for r in range(0, shape[0], step):
            part = torch.randn((min(step, shape[0] - r),) + shape[1:], generator=self.g, device="cuda")
            out[r:r + step] = part.mul_(std).add_(mean)
        return out

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda")


# ---------------------------------------------------------------- inputs

def _prepare_loss(case, t):
    T, S = case["tokens"], case["seqs"]
    cuts = torch.randperm(max(1, T - 1), generator=t.g, device="cuda")[:S - 1] + 1 if T > 1 else torch.zeros(0, device="cuda")
    cu = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
    cu[1:S] = cuts.sort().values[:S - 1].int()
    cu[S] = T
    old = -t.uniform(T).mul_(-1).add_(1.0).log_().mul_(-1.2).abs_()      # log-probabilities of sampled tokens: an exponential tail
    s = {"old": old, "logprob": (old + t.normal(T, std=0.15)).clamp_(max=-1e-6), "cu": cu, "weight": None, "ref": None}
    s["advantage"] = t.normal(S if case["per_seq"] else T)
    if case["weight"]:
        s["weight"] = torch.where(t.uniform(T) < 0.3, 0.0, t.uniform(T) + 0.5)
    if case["ref"]:
        s["ref"] = (old + t.normal(T, std=0.25)).clamp_(max=-1e-6)
    if case["per_seq"]:
        s["advantage"] = s["advantage"][:, None].contiguous()
    s.update(low=0.2, high=0.28, dual_at=3.0 if case["dual"] else 0.0, kl=0.04 if case["ref"] else 0.0,
             reduction=case["reduction"], scale=1.0 / S if case["reduction"] == "sequence" else 1.0)
    return s


def _prepare_head(case, t):
    Hq, Hkv, d, H, inter, V = MODELS[case["model"]]
    T = case["rows"]
    table = t.normal(V, H, std=H ** -0.5, dtype=BF)
    target = (t.uniform(T).double() * V).long().clamp_(0, V - 1)
    # the target's logit, up to two above the others' log-sum-exp: one minus its probability keeps its digits in 32 bits
    lean = t.uniform(T) * (math.log(V) + 2.0) * case["temperature"]
    hidden = torch.empty(T, H, dtype=BF, device="cuda")
    lse = torch.empty(T, device="cuda")
    scale = 1.0 / case["temperature"]
    W = table.float()
    for r in range(0, T, 2048):
        x = t.normal(min(2048, T - r), H) + lean[r:r + 2048, None] * W[target[r:r + 2048]]
        hidden[r:r + 2048] = x
        lse[r:r + 2048] = torch.logsumexp((hidden[r:r + 2048].float() @ W.T).mul_(scale), 1)
    d_logprob = t.normal(T, std=1.0 / T) * (t.uniform(T) > 0.2)              # masked tokens have none
    return {"hidden": hidden, "table": table, "target": target.int(), "lse": lse, "d_logprob": d_logprob, "scale": scale,
            "want": (case["hidden"], case["table"])}


def _sizes(case):
    Hq, Hkv, d, H, inter, V = MODELS[case["model"]]
    sizes = [V * H] if case["tied"] else []
    for _ in range(case["layers"]):
        if case["odd"]:
            sizes.append(1)                            # a learned branch scale: what follows it loses its alignment
        sizes += [H, Hq * d * H, Hkv * d * H, Hkv * d * H, H * Hq * d, H, 2 * inter * H, H * inter]
    return sizes + [H]


def _views(flat, sizes):
    return list(torch.split(flat, sizes))


def _prepare_adamw(case, t):
    sizes = _sizes(case)
    N = sum(sizes)
    s = {"sizes": sizes, "lr": 1e-4, "step": 100, "seed": 1234 if case["stochastic"] else None, "state": case["state"], "norm": None,
         "limit": 1.0, "master": None}
    weights = t.normal(N, std=0.02)
    s["param"] = weights.to(DTYPES[case["param"]])
    if case["master"]:
        s["master"] = weights
    s["grad"] = t.normal(N, std=1e-3, dtype=DTYPES[case["grad"]])
    m, v = t.normal(N, std=3e-4), t.normal(N, std=1e-3).square_().mul_(0.5).add_(2.5e-7)
    if case["state"] == 8:
        s["m"], s["m_scale"] = _quantise(m, None)
        s["v"], s["v_scale"] = _quantise(v.sqrt_(), None, positive=True)
    else:
        s["m"], s["v"] = m, v
    if case["clip"]:
        s["norm"] = torch.tensor([1e-3 * math.sqrt(N)], device="cuda") * (1.0 + t.uniform(1))
    # what a trainer holds: views of its flat buffers, one per tensor of the model
    s["lists"] = {k: _views(s[k], sizes) for k in ("param", "grad", "m", "v", "master") if s[k] is not None}
    if case["state"] == 8:
        for k in ("m_scale", "v_scale"):
            s["lists"][k] = _views(s[k], [n // BLOCK for n in sizes])
    return s


def prepare(case, seed):
    t = _Tensors(seed)
    s = {"loss": _prepare_loss, "head": _prepare_head, "adamw": _prepare_adamw}[case["kind"]](case, t)
    s["kind"] = case["kind"]
    return s


# ---------------------------------------------------------------- plain forms

def _loss_terms(s, lp, old, ref):
    """Per token: the policy term, the KL term, their derivatives with respect to the log-probability, whether the first was cut."""
    x64 = s["logprob"].double() - s["old"].double()    # what is near a threshold is decided in 64 bits
    over, under = x64 > math.log1p(s["high"]), x64 < math.log1p(-s["low"])
    T, seq = lp.numel(), None
    if s["advantage"].dim() == 2 or s["reduction"] == "sequence":
        seq = torch.searchsorted(s["cu"][1:], torch.arange(T, device=lp.device, dtype=torch.int32), right=True)
    adv = (s["advantage"][:, 0][seq] if s["advantage"].dim() == 2 else s["advantage"]).to(lp.dtype)
    ratio = torch.exp(lp - old)
    cut = torch.where(adv > 0, over, under)
    bound = torch.where(adv > 0, 1.0 + s["high"], 1.0 - s["low"]).to(lp.dtype)
    value = -adv * torch.where(cut & (adv != 0), bound, ratio)
    if s["dual_at"]:
        far = (adv < 0) & (x64 > math.log(s["dual_at"]))
        value, cut = torch.where(far, -adv * s["dual_at"], value), cut | far
    cut = cut & (adv != 0)
    slope = torch.where(cut, 0.0, -adv * ratio)
    kl = kl_slope = None
    if ref is not None:
        e = torch.expm1(ref - lp)
        kl, kl_slope = e - (ref - lp), -e
    return value, slope, cut, kl, kl_slope, ratio, seq


def _plain_loss(s):
    # in 64 bits: e^d - d - 1 has few digits left in 32 where d is small, as it mostly is
    lp, old, ref = s["logprob"].double(), s["old"].double(), s["ref"].double() if s["ref"] is not None else None
    value, slope, cut, kl, kl_slope, ratio, seq = _loss_terms(s, lp, old, ref)
    T, S = lp.numel(), s["cu"].numel() - 1
    w = s["weight"].double() if s["weight"] is not None else torch.ones_like(lp)
    on = w != 0
    n = on.sum()
    if s["reduction"] == "sequence":
        per = torch.zeros(S, dtype=F64, device=lp.device).index_add_(0, seq, on.double())
        f = s["scale"] / per.clamp(min=1.0)[seq]
    else:
        f = s["scale"] / n.clamp(min=1) if s["reduction"] == "token" else s["scale"]
    f = w * f
    policy = torch.where(on, f * value, 0.0).sum()
    d = slope
    kl_sum = torch.zeros_like(policy)
    if kl is not None:
        kl_sum = torch.where(on, f * kl, 0.0).sum()
        d = d + s["kl"] * kl_slope
    x, count = lp - old, n.clamp(min=1).double()
    stats = torch.stack([policy, kl_sum, (cut & on).sum() / count, torch.where(on, torch.expm1(x) - x, 0.0).sum() / count, n.double()])
    return {"loss": (policy + s["kl"] * kl_sum).float().reshape(1), "d_logprob": torch.where(on, f * d, 0.0).float(), "stats": stats.float()}


def _plain_head(s):
    hidden, table, T = s["hidden"].float(), s["table"].float(), s["hidden"].shape[0]
    z = hidden @ table.T
    d = torch.exp(z.mul_(s["scale"]).sub_(s["lse"][:, None])).neg_()
    d[torch.arange(T, device=d.device), s["target"].long()] += 1.0
    d.mul_((s["d_logprob"] * s["scale"])[:, None])
    out = {}
    if s["want"][0]:
        out["d_hidden"] = (d @ table).to(BF)
    if s["want"][1]:
        out["d_lm_head"] = (d.T @ hidden).to(BF)
    return out


def _mix(x):
    """32 bits from 32 bits, in int64."""
    low = 0xFFFFFFFF
    x = x ^ (x >> 16)
    x = (x * 0x5BD1F3C5) & low
    x = x ^ (x >> 15)
    x = (x * 0x2F4A6E9B) & low
    return x ^ (x >> 16)


def _random(n, seed, step):
    """32 bits for each element of a call: of its place among all elements, the seed and the step."""
    at = torch.arange(n, device="cuda")
    key = _mix(torch.tensor((seed ^ (step * 0x9E3779B9)) & 0xFFFFFFFF, device="cuda"))
    return _mix(((at & 0xFFFFFFFF) * 0x632BE5AB + key + (at >> 32) * 0x85157AF5) & 0xFFFFFFFF)


def _quantise(x, random, positive=False):
    """8-bit values and a power of two for each BLOCK of them.  random: 16 bits an element, or None for the nearest."""
    x = x.view(-1, BLOCK)
    a = x.abs().amax(1)
    f, e = torch.frexp(a)                              # a = f 2^e, f in [1/2, 1): the largest value lands in (224, 448]
    k = torch.where(a > 0, e - 9 + (f > 0.875).int(), -127).clamp(min=-127)
    y = torch.ldexp(x, -k[:, None])
    if random is not None:
        ulp = torch.ldexp(torch.ones_like(y), (torch.frexp(y)[1] - 1).clamp(min=-6) - 3)
        y = torch.copysign(torch.floor(y.abs() / ulp + random.view(-1, BLOCK).float() * 2.0 ** -16) * ulp, y)
    q = y.to(FP8)
    if positive:                                       # what is not zero does not become zero: the step divides by it
        q = torch.where((q.float() == 0) & (x > 0), 2.0 ** -9, q.float()).to(FP8)
    return q.view(-1), (k + 127).to(torch.uint8).view(E8M0)


def _plain_adamw(s):
    p = (s["master"] if s["master"] is not None else s["param"]).float()
    g, eight = s["grad"].float(), s["state"] == 8
    if s["norm"] is not None:
        g = g * torch.where(s["norm"] > s["limit"], s["limit"] / s["norm"], 1.0)
    m, v = s["m"].float(), s["v"].float()
    if eight:
        m = (m.view(-1, BLOCK) * s["m_scale"].float()[:, None]).view(-1)
        v = (v.view(-1, BLOCK) * s["v_scale"].float()[:, None]).view(-1).square()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    root = v.sqrt()
    step = s["lr"] / (1 - BETA1 ** s["step"])
    p = (1 - s["lr"] * DECAY) * p - step * m / (root * (1 - BETA2 ** s["step"]) ** -0.5 + ADAM_EPS)
    r = _random(p.numel(), s["seed"], s["step"]) if s["seed"] is not None else None
    if eight:
        q, k = _quantise(m, None if r is None else r & 0xFFFF)
        s["m"].copy_(q), s["m_scale"].copy_(k)
        q, k = _quantise(root, None if r is None else r >> 16, positive=True)
        s["v"].copy_(q), s["v_scale"].copy_(k)
    else:
        s["m"].copy_(m), s["v"].copy_(v)
    if s["master"] is not None:
        s["master"].copy_(p)
    if s["param"].dtype == BF and s["master"] is None and r is not None:
        bits = p.view(torch.int32) + (_mix(r) & 0xFFFF).int()
        p = (bits & -65536).view(F32)
    s["param"].copy_(p)
    return _adamw_out(s)


def _adamw_out(s):
    names = ["param", "m", "v"] + (["master"] if s["master"] is not None else []) + (["m_scale", "v_scale"] if s["state"] == 8 else [])
    return {k: s[k] for k in names}


# ---------------------------------------------------------------- one pass

def _own(s):
    from paper_2609_35140_b200 import binding as tik
    if s["kind"] == "loss":
        loss, d, stats = tik.tik_policy_loss(s["logprob"], s["old"], s["advantage"], weight=s["weight"], ref_logprob=s["ref"],
                                             cu_seqlens=s["cu"], clip_low=s["low"], clip_high=s["high"], clip_dual=s["dual_at"],
                                             kl_coef=s["kl"], reduction=s["reduction"], scale=s["scale"])
        return {"loss": loss, "d_logprob": d, "stats": stats}
    if s["kind"] == "head":
        got = tik.tik_token_logprob_bwd(s["d_logprob"], s["hidden"], s["table"], s["target"], s["lse"], s["scale"],
                                        need_hidden=s["want"][0], need_lm_head=s["want"][1])
        return {k: v for k, v in zip(("d_hidden", "d_lm_head"), got) if v is not None}
    l = s["lists"]
    tik.tik_adamw(l["param"], l["grad"], l["m"], l["v"], s["lr"], s["step"], beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY,
                  master=l.get("master"), exp_avg_scale=l.get("m_scale"), exp_avg_sq_scale=l.get("v_scale"), norm=s["norm"],
                  max_norm=s["limit"], seed=s["seed"])
    return _adamw_out(s)


def run(state):
    if own:
        return _own(state)
    return {"loss": _plain_loss, "head": _plain_head, "adamw": _plain_adamw}[state["kind"]](state)


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_loss(case, s):
    x = s["logprob"].to(F64) - s["old"].to(F64)
    T = x.numel()
    lengths = (s["cu"][1:] - s["cu"][:-1]).long()
    spread = lambda per: torch.repeat_interleave(per, lengths)  # noqa: E731
    A = spread(s["advantage"].flatten().to(F64)) if case["per_seq"] else s["advantage"].to(F64)
    r = x.exp()
    lo, hi = 1.0 - s["low"], 1.0 + s["high"]
    gain = torch.minimum(r * A, r.clamp(lo, hi) * A)
    live = (r * A <= r.clamp(lo, hi) * A)
    if s["dual_at"]:
        floor = torch.where(A < 0, s["dual_at"] * A, -math.inf)
        live &= gain >= floor
        gain = torch.maximum(gain, floor)
    w = torch.ones_like(x) if s["weight"] is None else s["weight"].to(F64)
    keep = w != 0
    if case["reduction"] == "sum":
        f = w * s["scale"]
    elif case["reduction"] == "token":
        f = w * (s["scale"] / max(1, int(keep.sum())))
    else:
        ends = torch.cat([torch.zeros(1, dtype=F64, device=x.device), keep.to(F64).cumsum(0)])
        count = ends[s["cu"][1:].long()] - ends[s["cu"][:-1].long()]
        f = w * s["scale"] / spread(torch.clamp(count, min=1.0))
    d = -torch.where(live, r * A, 0.0) * f
    policy, kl = (-gain * f).sum(), torch.zeros((), dtype=F64, device=x.device)
    if case["ref"]:
        y = s["ref"].to(F64) - s["logprob"].to(F64)
        kl = (f * (torch.expm1(y) - y)).sum()
        d = d - s["kl"] * f * torch.expm1(y)
    n = max(1, int(keep.sum()))
    stats = torch.stack([policy, kl, (~live & keep).sum() / n, torch.where(keep, torch.expm1(x) - x, 0.0).sum() / n, keep.sum().to(F64)])
    return {"loss": (policy + s["kl"] * kl).reshape(1), "d_logprob": d, "stats": stats}


def _exact_head(case, s):
    T, H = s["hidden"].shape
    W, out = s["table"].to(F64), {}
    dh = torch.empty(T, H, dtype=F64, device="cuda")
    dw = torch.zeros_like(W) if case["table"] else None
    for r in range(0, T, 512):
        x, at = s["hidden"][r:r + 512].to(F64), s["target"][r:r + 512].long()
        p = torch.exp(s["scale"] * (x @ W.T) - s["lse"][r:r + 512, None].to(F64))
        one = torch.nn.functional.one_hot(at, W.shape[0]).to(F64)
        g = (one - p) * (s["scale"] * s["d_logprob"][r:r + 512].to(F64))[:, None]
        if case["hidden"]:
            dh[r:r + 512] = g @ W
        if case["table"]:
            dw.addmm_(g.T, x)
    if case["hidden"]:
        out["d_hidden"] = dh
    if case["table"]:
        out["d_lm_head"] = dw
    return out


def _exact_adamw(case, s):
    out = {}
    per = lambda k: torch.repeat_interleave(s[k].to(F32).to(F64), BLOCK)  # noqa: E731
    g = s["grad"].to(F64)
    if case["clip"]:
        g *= min(1.0, s["limit"] / float(s["norm"]))
    m, v = s["m"].to(F32).to(F64), s["v"].to(F32).to(F64)
    if case["state"] == 8:
        m, v = m * per("m_scale"), (v * per("v_scale")) ** 2
    m.mul_(BETA1).add_(g, alpha=1 - BETA1)
    v.mul_(BETA2).addcmul_(g, g, value=1 - BETA2)
    del g
    p = (s["master"] if case["master"] else s["param"]).to(F64) * (1 - s["lr"] * DECAY)
    bc1, bc2 = 1 - BETA1 ** s["step"], 1 - BETA2 ** s["step"]
    p.sub_((m / bc1) / ((v / bc2).sqrt() + ADAM_EPS), alpha=s["lr"])
    out["param"] = p
    if case["master"]:
        out["master"] = p
    if case["state"] == 32:
        return {**out, "m": m, "v": v}
    # a stored value is the moment (of the second one: its root) in units of the block's power of two
    for name, x in (("m", m), ("v", v.sqrt())):
        a = x.view(-1, BLOCK).abs().amax(1).clamp(min=1e-300)
        k = torch.ceil(torch.log2(a / 448.0)).clamp(min=-127.0)
        out[name], out[name + "_scale"] = (x.view(-1, BLOCK) / torch.exp2(k)[:, None]).view(-1), torch.exp2(k)
    return out


def exact(case, seed):
    return {"loss": _exact_loss, "head": _exact_head, "adamw": _exact_adamw}[case["kind"]](case, prepare(case, seed))


def work(case):
    if case["kind"] == "loss":
        T, S = case["tokens"], case["seqs"]
        planes = 3 + (not case["per_seq"]) + case["weight"] + case["ref"]        # two log-probabilities and the gradient besides
        cu = case["per_seq"] or case["reduction"] == "sequence"
        return {"bytes": 4.0 * planes * T + 4.0 * S * (case["per_seq"] + cu) + 24.0, "flops": 40.0 * T}
    if case["kind"] == "head":
        Hq, Hkv, d, H, inter, V = MODELS[case["model"]]
        T, outs = case["rows"], (case["hidden"], case["table"])
        return {"bytes": 2.0 * H * (T * (1 + outs[0]) + V * (1 + outs[1])) + 12.0 * T, "flops": 2.0 * T * V * H * (1 + sum(outs))}
    N = sum(_sizes(case))
    each = (2.0 if case["grad"] == "bf16" else 4.0) + (4.0 if case["state"] == 8 else 16.0) + (4.0 / BLOCK if case["state"] == 8 else 0.0)
    # the master copy is read and written, and then the weights are only written
    each += 10.0 if case["master"] else 4.0 if case["param"] == "bf16" else 8.0
    return {"bytes": N * each, "flops": 20.0 * N}
