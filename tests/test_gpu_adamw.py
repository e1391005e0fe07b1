"""tik_adamw against its definition in 64 bits, one step from a given state.

Tolerances.  fp32 has half a step of u = 2^-24.  m and v are two roundings of products and one of a sum, the clip's factor two
more on g: off by 5 u of the terms' magnitudes.  The step's quotient has a root, a product, a sum and a division of two steps: 12 u of
itself, plus what m's and v's errors move it by; the weight is one rounding of its sum.  A weight in bf16 is off by another half step, 2^-8
(stochastically rounded: a whole one).  An 8-bit value is off by half a step of e4m3, 2^-4 of itself or 2^-10 of its block's scale
(stochastically: twice that)."""
import math

import pytest
import torch

from paper_2609_35140_b200 import binding as tik

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32, FP8, E8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.float8_e8m0fnu
HYPER = dict(beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)


def blocks(x):
    """x in blocks of 32, the last one filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.numel() % 32)).view(-1, 32)


def scale_values(s, n):
    return torch.exp2(s.view(torch.uint8).double() - 127).repeat_interleave(32)[:n]


def moments(t):
    """(m, v) of a tensor's state in 64 bits."""
    if t["ms"] is None:
        return t["m"].double(), t["v"].double()
    n = t["m"].numel()
    return t["m"].double() * scale_values(t["ms"], n), (t["v"].double() * scale_values(t["vs"], n)) ** 2


def make(sizes, param=BF, grad=BF, master=False, eight=False, seed=0, shift=0):
    """A list of tensors, each `shift` elements into its own buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    tensors = []
    for i, n in enumerate(sizes):
        def place(x):
            buf = torch.zeros(n + shift, dtype=x.dtype, device="cuda")
            out = buf[shift:]
            out.copy_(x)
            return out
        rand = lambda s: torch.randn(n, generator=g, device="cuda") * s  # noqa: E731
        w = rand(0.05)
        p = param if not isinstance(param, (list, tuple)) else param[i % len(param)]
        gt = grad if not isinstance(grad, (list, tuple)) else grad[i % len(grad)]
        t = dict(p=place(w.to(p)), g=place((rand(1e-3) * (1 + 9 * (rand(1.0) > 1.5))).to(gt)), w=None, ms=None, vs=None)
        if master and p == BF:
            t["w"] = place(w)
        m, v = rand(4e-4) * torch.exp(rand(2.0)), (rand(1e-3) * torch.exp(rand(2.0))) ** 2
        if eight:
            c = -(-n // 32)
            t["ms"] = torch.randint(105, 112, (c,), generator=g, device="cuda", dtype=torch.uint8).view(E8)
            t["vs"] = torch.randint(106, 112, (c,), generator=g, device="cuda", dtype=torch.uint8).view(E8)
            code = torch.randint(0, 127, (n,), generator=g, device="cuda", dtype=torch.uint8)
            t["m"] = place(code.view(FP8).float().mul(torch.sign(rand(1.0))).to(FP8))
            t["v"] = place(torch.randint(1, 127, (n,), generator=g, device="cuda", dtype=torch.uint8).view(FP8))
        else:
            t["m"], t["v"] = place(m), place(v)
        tensors.append(t)
    return tensors


def copy(tensors):
    return [{k: (None if v is None else v.clone()) for k, v in t.items()} for t in tensors]


def step(tensors, lr=1e-3, n=7, norm=None, max_norm=1.0, seed=None, **kw):
    col = lambda k: [t[k] for t in tensors]  # noqa: E731
    eight = any(t["ms"] is not None for t in tensors)
    tik.tik_adamw(col("p"), col("g"), col("m"), col("v"), lr, n, **{**HYPER, **kw}, master=col("w") if any(t["w"] is not None for t in tensors) else None,
                  exp_avg_scale=col("ms") if eight else None, exp_avg_sq_scale=col("vs") if eight else None, norm=norm, max_norm=max_norm, seed=seed)


def check(before, after, lr=1e-3, n=7, clip=1.0, seed=None, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1):
    for b, a in zip(before, after):
        if b["p"].numel() == 0:
            continue
        g = b["g"].double() * clip
        m0, v0 = moments(b)
        m, v = beta1 * m0 + (1 - beta1) * g, beta2 * v0 + (1 - beta2) * g * g
        e_m, e_v = 5 * U * (beta1 * m0.abs() + (1 - beta1) * g.abs()), 6 * U * v
        root, denominator = v.sqrt(), (v / (1 - beta2 ** n)).sqrt() + eps
        w0 = (b["w"] if b["w"] is not None else b["p"]).double()
        change = lr / (1 - beta1 ** n) * m / denominator
        w = (1 - lr * weight_decay) * w0 - change
        e_w = 3 * U * (w0.abs() + w.abs()) + 16 * U * change.abs() + lr / (1 - beta1 ** n) / denominator * e_m
        near = lambda got, ref, bound: bool(((got.double() - ref).abs() <= bound + 1e-44).all())  # noqa: E731
        if b["w"] is not None:
            assert near(a["w"], w, e_w)
            assert torch.equal(a["p"], a["w"].to(BF))
        elif b["p"].dtype == F32:
            assert near(a["p"], w, e_w)
        else:
            assert near(a["p"], w, e_w + (2.0 ** -8 if seed is None else 2.0 ** -7) * (w.abs() + e_w) * (1 + 2.0 ** -7))
        if b["ms"] is None:
            assert near(a["m"], m, e_m) and near(a["v"], v, e_v)
            continue
        for q, s, x, e, positive in ((a["m"], a["ms"], m, e_m, False), (a["v"], a["vs"], root, 5 * U * root, True)):
            nn = x.numel()
            top, slack = blocks(x.abs()).amax(1), blocks(e).amax(1)
            k = s.view(torch.uint8).double() - 127
            assert bool((top - slack <= 448 * torch.exp2(k)).all())                                    # it fits
            assert bool(((top + slack > 448 * torch.exp2(k - 1)) | (k == -127)).all())                  # and would not in the next smaller one
            unit, rate = scale_values(s, nn), 2.0 ** -4 if seed is None else 2.0 ** -3
            got = q.double() * unit
            bound = torch.maximum(rate * (x.abs() + e), rate * 2.0 ** -6 * unit) + e
            if positive:                                 # the least value stands in for those below it
                bound = torch.maximum(bound, 2.0 ** -9 * unit)
                assert bool((got[x > 0] > 0).all())
            assert bool(((got - x).abs() <= bound).all())


SIZES = [0, 1, 31, 32, 33, 100, 2047, 2048, 8191, 8192, 8193, 100003]
KINDS = [dict(param=BF, grad=BF, master=True), dict(param=F32, grad=F32), dict(param=BF, grad=F32), dict(param=F32, grad=BF, eight=True),
         dict(param=BF, grad=BF, eight=True), dict(param=BF, grad=F32, master=True, eight=True),
         dict(param=[BF, F32], grad=[BF, F32, F32], master=True), dict(param=[F32, BF], grad=[BF, F32, BF], eight=True)]


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("shift", [0, 1, 8])
@pytest.mark.parametrize("seed", [None, 77])
def test_one_step(kind, shift, seed):
    a = make(SIZES, seed=kind, shift=shift, **KINDS[kind])
    b = copy(a)
    step(a, seed=seed)
    check(b, a, seed=seed)
    for x, y in zip(a, b):
        assert torch.equal(x["g"], y["g"])               # gradients stay


@pytest.mark.parametrize("n,lr,hyper", [(1, 1e-3, {}), (1, 1e-2, dict(beta1=0.0, beta2=0.0, weight_decay=0.0)), (100000, 0.0, {}),
                                        (3, 5e-4, dict(beta1=0.95, beta2=0.99, eps=1e-5))])
def test_hyperparameters(n, lr, hyper):
    for kind in (KINDS[1], KINDS[4]):
        a = make([1000, 37], seed=3, **kind)
        b = copy(a)
        step(a, lr=lr, n=n, **hyper)
        check(b, a, lr=lr, n=n, **{**HYPER, **hyper})


def test_first_step_from_zeros():
    for kind in (KINDS[0], KINDS[4], KINDS[5]):
        a = make([500, 64], seed=4, **kind)
        for t in a:
            t["g"][3], t["g"][40:60] = 0.0, 0.0          # a gradient of zero beside zero moments: the weight only decays
            for k in ("m", "v", "ms", "vs"):
                if t[k] is not None:
                    t[k].view(torch.uint8 if t[k].dtype in (FP8, E8) else t[k].dtype).zero_()
        b = copy(a)
        step(a, n=1)
        check(b, a, n=1)


def test_clip_by_a_norm():
    for kind in (KINDS[0], KINDS[4]):
        a = make([3000, 5], seed=5, **kind)
        norm = tik.tik_grad_norm([t["g"] for t in a])
        limit = float(norm) / 3
        b = copy(a)
        step(a, norm=norm, max_norm=limit)
        check(b, a, clip=float(torch.tensor(limit, dtype=F32)) / float(norm))
        a = copy(b)
        step(a, norm=norm, max_norm=3 * limit * 1.01)     # below the limit
        check(b, a)
        c = copy(b)
        tik.tik_grad_clip([t["g"] for t in c], limit)     # what a clip writes back, within its rounding
        step(c)
        for bad in (math.inf, math.nan):
            a = copy(b)
            step(a, norm=torch.tensor([bad], device="cuda"), max_norm=1.0)
            for x, y in zip(a, b):
                for k in x:
                    assert x[k] is None or torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8))


def test_many_tensors_and_one_have_the_same_bits():
    """Stochastic rounding goes by an element's place in the call: a tensor cut into 900 pieces of whole blocks, over several
    launches, comes out as the whole one."""
    for kind in (KINDS[4], KINDS[2], KINDS[5]):
        whole = make([900 * 96], seed=6, **kind)
        parts = copy(whole)[0]
        cut = lambda v, n: [None] * 900 if v is None else list(v.split(n))  # noqa: E731
        cols = {k: cut(parts[k], 3 if k in ("ms", "vs") else 96) for k in parts}
        step([{k: cols[k][i] for k in cols} for i in range(900)], seed=5)
        step(whole, seed=5)
        for k in parts:
            assert parts[k] is None or torch.equal(parts[k].view(torch.uint8), whole[0][k].view(torch.uint8)), k


def test_vectors_and_single_elements_have_the_same_bits():
    for kind in KINDS:
        for seed in (None, 3):
            a, b = make([5003], seed=7, **kind), make([5003], seed=7, shift=1, **kind)
            step(a, seed=seed)
            step(b, seed=seed)
            for k in a[0]:
                assert a[0][k] is None or torch.equal(a[0][k].contiguous().view(torch.uint8), b[0][k].clone().view(torch.uint8)), k


def test_stochastic_rounding_is_unbiased_and_depends_on_seed_and_step():
    n = 1 << 20
    def run(seed, number):
        t = dict(p=torch.full((n,), 1.0, dtype=BF, device="cuda"), g=torch.full((n,), 0.011, device="cuda"), w=None,
                 m=torch.zeros(n, dtype=FP8, device="cuda"), v=torch.zeros(n, dtype=FP8, device="cuda"),
                 ms=torch.zeros(n // 32, dtype=torch.uint8, device="cuda").view(E8), vs=torch.zeros(n // 32, dtype=torch.uint8, device="cuda").view(E8))
        t["g"][::32] = 0.017                             # the block's scale, so that the others lie between two values
        step([t], lr=1e-3, n=number, seed=seed, weight_decay=0.0)
        return t
    t = run(11, 1)
    pick = torch.arange(n, device="cuda") % 32 != 0
    m, v = moments(t)
    g = float(torch.tensor(0.011))
    for got, want in ((m, 0.1 * g), (v.sqrt(), math.sqrt(0.001) * g), (t["p"].double(), 1.0 - 1e-3)):
        got = got[pick]
        values = torch.unique(got)
        assert values.numel() == 2 and float(values[0]) < want < float(values[1])
        # a mean of n draws between two values: 6 standard deviations, and 16 bits of randomness
        gap = float(values[1] - values[0])
        assert abs(float(got.mean()) - want) <= gap * (6 * 0.5 / math.sqrt(got.numel()) + 2.0 ** -16) + 1e-6 * want
    # neighbours, and the three roundings of an element, do not go together
    up = [(x[pick] > x[pick].mean()).double() for x in (m, v, t["p"].double())]
    up = [(x - x.mean()) / x.std() for x in up]
    for i in range(3):
        for j in range(3):
            a, b = (up[i][:-1], up[j][1:]) if i == j else (up[i], up[j])
            assert abs(float((a * b).mean())) <= 6 / math.sqrt(a.numel())
    same, other, later = run(11, 1), run(12, 1), run(11, 2)
    assert torch.equal(same["m"].view(torch.uint8), t["m"].view(torch.uint8))
    share = lambda x: float((x["v"].view(torch.uint8) != t["v"].view(torch.uint8)).double().mean())  # noqa: E731
    assert share(other) > 0.1 and share(later) > 0.1


def test_what_is_not_finite():
    """Without a norm the gradients' infinities and NaN go into their own elements alone."""
    for kind in (KINDS[1], KINDS[4]):
        a = make([200], seed=8, **kind)
        clean, dirty = copy(a), copy(a)
        dirty[0]["g"][70], dirty[0]["g"][71] = math.inf, math.nan
        clean[0]["g"][70:72] = 0.0
        b = copy(dirty)
        step(dirty)
        assert not torch.isfinite(dirty[0]["m"][70:72].float()).any()
        keep = torch.ones(200, dtype=torch.bool, device="cuda")
        keep[64:96] = a[0]["ms"] is None
        keep[70:72] = False
        step(clean)
        for k in ("p", "m", "v"):
            assert torch.equal(dirty[0][k].float()[keep], clean[0][k].float()[keep])
        assert bool(torch.isfinite(dirty[0]["m"].float()[64:70]).all())


def test_lr_and_step_on_the_device_in_a_graph():
    for kind in (KINDS[0], KINDS[4]):
        a = make([4000, 77], seed=9, **kind)
        b = copy(a)
        lr, number = torch.tensor([1e-3], device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(copy(a), lr=lr, n=number, seed=1)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(a, lr=lr, n=number, seed=1)
            number += 1
        for i in range(1, 5):
            lr.fill_(1e-3 / i)
            g.replay()
            step(b, lr=float(lr), n=i, seed=1)
            for x, y in zip(a, b):
                for k in x:
                    assert x[k] is None or torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)), (i, k)


def test_steps_in_a_row_stay_with_64_bits():
    a = make([3001], seed=10, param=F32, grad=F32)
    t = a[0]
    w, m, v = t["p"].double(), t["m"].double(), t["v"].double()
    e_w, e_m, e_v = (torch.zeros_like(w) for _ in range(3))      # the step's errors, and what earlier ones have become
    for n in range(1, 21):
        t["g"].copy_(torch.randn(3001, device="cuda") * 1e-3)
        g = t["g"].double()
        step(a, n=n)
        e_m = 0.9 * e_m + 5 * U * (0.9 * m.abs() + 0.1 * g.abs())
        m, v = 0.9 * m + 0.1 * g, 0.999 * v + 0.001 * g * g
        e_v = 0.999 * e_v + 6 * U * v
        rate = 1e-3 / (1 - 0.9 ** n) / ((v / (1 - 0.999 ** n)).sqrt() + 1e-8)
        change = rate * m
        e_w = e_w + 3 * U * 2 * w.abs() + change.abs() * (19 * U + e_v / v) + rate * e_m
        w = (1 - 1e-4) * w - change
    assert bool(((t["p"].double() - w).abs() <= e_w).all())


def test_refusals_of_the_binding():
    p, g, m, v = (torch.zeros(64, device="cuda") for _ in range(4))
    for bad in (dict(step=0), dict(step=1.5), dict(lr=-1.0), dict(lr=math.nan), dict(beta1=1.0), dict(eps=0.0), dict(weight_decay=-0.1),
                dict(exp_avg=[m[:32]]), dict(exp_avg=[m.double()]), dict(grads=[g, g]), dict(grads=[g.half()]), dict(exp_avg=[p]),
                dict(exp_avg_sq=[m]), dict(grads=[p]), dict(master=[g]), dict(norm=torch.ones(1, device="cuda"), max_norm=0.0),
                dict(exp_avg_scale=[m]), dict(norm=p[:1]), dict(lr=torch.ones(2, device="cuda")), dict(params=[p.cpu()]),
                dict(step=torch.ones(1, device="cuda")), dict(params=[p[::2]], grads=[g[:32]], exp_avg=[m[:32]], exp_avg_sq=[v[:32]])):
        args = dict(dict(params=[p], grads=[g], exp_avg=[m], exp_avg_sq=[v], lr=1e-3, step=1), **bad)
        with pytest.raises((tik.TikError, ValueError, TypeError)):
            tik.tik_adamw(**args)
    tik.tik_adamw([], [], [], [], 1e-3, 1)
    assert not p.any()
