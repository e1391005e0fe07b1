"""tik_policy_loss against its definition in 64 bits.

Tolerances: per token everything is fp32 (half a step 2^-24, called u).  x = logprob - old is rounded once, expf is off by two
steps: r is off by (|x| + 4) u of itself; y = ref - logprob likewise, expm1f and the tangent's remainder by a few u of their value plus what
y's rounding moves them by, |y| u times their slope.  f is three roundings.  Sums are fp64, so the loss is off by the sum of its terms' bounds and one rounding."""
import math

import pytest
import torch

from paper_2609_35140_b200 import binding as tik

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def make(T, S, seed=0, per_seq=False, weight=True, ref=True, spread=0.3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda n: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    uni = lambda n: torch.rand(n, generator=g, device="cuda")  # noqa: E731
    old = -3 * uni(T)
    cuts = torch.sort((uni(S - 1) * (T + 1)).int().clamp(max=T)).values          # sequences of no tokens among them
    cu = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), cuts, torch.full((1,), T, dtype=torch.int32, device="cuda")])
    return dict(logprob=old + spread * rand(T), old_logprob=old, advantage=rand(S)[:, None].contiguous() if per_seq else rand(T),
                weight=torch.where(uni(T) < 0.4, 0.0, 0.5 + uni(T)) if weight else None, ref_logprob=old + 0.4 * rand(T) if ref else None,
                cu_seqlens=cu)


def expected(logprob, old_logprob, advantage, weight=None, ref_logprob=None, cu_seqlens=None, clip_low=0.2, clip_high=0.2,
             clip_dual=0.0, kl_coef=0.0, reduction="token", scale=1.0):
    low, high, dual, kl_coef, scale = (float(torch.tensor(v, dtype=torch.float32)) for v in (clip_low, clip_high, clip_dual, kl_coef, scale))
    T = logprob.numel()
    dev = logprob.device
    t = torch.arange(T, device=dev)
    inside = torch.ones(T, dtype=torch.bool, device=dev)
    seq = torch.zeros(T, dtype=torch.long, device=dev)
    if cu_seqlens is not None:
        S = cu_seqlens.numel() - 1
        inside = (t >= cu_seqlens[0]) & (t < cu_seqlens[-1])
        seq = torch.searchsorted(cu_seqlens[1:].contiguous(), t.int(), right=True).clamp(max=max(S - 1, 0))
    w = (weight.double() if weight is not None else torch.ones(T, dtype=torch.float64, device=dev)) * inside
    on = inside & (w != 0)
    A = (advantage[:, 0][seq] if advantage.dim() == 2 else advantage).double()
    x = logprob.double() - old_logprob.double()
    r = x.exp()
    pos, neg = A > 0, A < 0
    cut_high, cut_low = pos & (x > math.log1p(high)), neg & (x < math.log1p(-low))
    cut_dual = neg & (x > math.log(dual)) if dual else torch.zeros_like(pos)
    cut = cut_high | cut_low | cut_dual
    at = torch.where(cut_high, 1 + high, torch.where(cut_low, 1 - low, torch.where(cut_dual, dual, r)))
    policy, slope = -A * at, torch.where(cut, 0.0, -A * r)
    e_policy, e_slope = policy.abs() * (x.abs() + 6) * U, slope.abs() * (x.abs() + 6) * U
    kl, kl_slope, e_kl, e_kl_slope = (torch.zeros_like(x) for _ in range(4))
    if ref_logprob is not None:
        y = ref_logprob.double() - logprob.double()
        kl, kl_slope = torch.expm1(y) - y, -torch.expm1(y)
        moved = y.abs() * U
        e_kl = kl * 16 * U + moved * torch.expm1(y).abs() * 2 + torch.where(y.abs() > 0.5, 4 * U * (torch.expm1(y).abs() + y.abs()), 0.0)
        e_kl_slope = kl_slope.abs() * 6 * U + moved * y.exp()
    if reduction == "sequence":
        per = torch.zeros(S, dtype=torch.float64, device=dev).index_add_(0, seq[on], torch.ones(int(on.sum()), dtype=torch.float64, device=dev))
        n = per.clamp(min=1)[seq]
    else:
        n = max(1, int(on.sum())) if reduction == "token" else 1
    f = scale * w / n
    zero = torch.zeros((), dtype=torch.float64, device=dev)
    pick = lambda v: torch.where(on, v, zero)  # noqa: E731
    sums = [pick(f * policy).sum(), pick(f * kl).sum()]
    loss = sums[0] + kl_coef * sums[1]
    e_loss = pick(f.abs() * (e_policy + abs(kl_coef) * e_kl + 4 * U * (policy.abs() + abs(kl_coef) * kl))).sum() + 2 * U * loss.abs()
    d = pick(f * (slope + kl_coef * kl_slope))
    e_d = pick(f.abs() * (e_slope + abs(kl_coef) * e_kl_slope + 5 * U * (slope.abs() + abs(kl_coef) * kl_slope.abs()))) + 2 * U * d.abs()
    count = max(1, int(on.sum()))
    k3 = torch.expm1(x) - x
    stats = torch.stack([sums[0], sums[1], pick(cut.double()).sum() / count, pick(k3).sum() / count, on.sum().double()])
    e_k3 = pick(k3 * 16 * U + x.abs() * U * torch.expm1(x).abs() * 2 + torch.where(x.abs() > 0.5, 4 * U * (torch.expm1(x).abs() + x.abs()), 0.0)).sum() / count
    e_stats = torch.stack([pick(f.abs() * (e_policy + 4 * U * policy.abs())).sum(), pick(f.abs() * (e_kl + 4 * U * kl)).sum(), zero, e_k3, zero]) + 2 * U * stats.abs()
    return (loss, e_loss), (d, e_d), (stats, e_stats)


def check(got, want, inputs_T):
    for out, (ref, bound) in zip(got, want):
        out = out.double().reshape(ref.shape)
        assert bool(((out - ref).abs() <= bound + 1e-38).all()), ((out - ref).abs() - bound).max().item()


def both(a, **kw):
    got = tik.tik_policy_loss(**a, **kw)
    check(got, expected(**a, **kw), a["logprob"].numel())
    return got


@pytest.mark.parametrize("T,S", [(1, 1), (2, 3), (31, 1), (32, 5), (33, 40), (257, 7), (512, 3), (513, 513), (1025, 64), (4096, 17), (4097, 2), (8193, 2),
                                 (20000, 700), (32768, 1), (32769, 9), (60013, 64), (70001, 9000), (300007, 1024)])
@pytest.mark.parametrize("reduction", ["sum", "token", "sequence"])
def test_lengths(T, S, reduction):
    for i, (per_seq, weight, ref) in enumerate([(False, False, False), (True, True, True), (False, True, False), (True, False, True)]):
        a = make(T, S, seed=T + S + i, per_seq=per_seq, weight=weight, ref=ref)
        both(a, reduction=reduction, kl_coef=0.05 if ref else 0.0, scale=1.0 / S, clip_high=0.28, clip_dual=3.0 if i & 1 else 0.0)


@pytest.mark.parametrize("T", [700, 50000])
def test_more_sequences_than_a_cluster_counts(T):
    a = make(T, 9001, seed=3)
    both(a, reduction="sequence", kl_coef=0.1)


@pytest.mark.parametrize("T", [300, 40000])
def test_padded_batch_and_masked_tokens(T):
    """Tokens outside the sequences, and masked ones, may hold anything; a sequence of masked tokens counts for nothing."""
    a = make(T, 6, seed=5)
    cu = a["cu_seqlens"].clone()
    cu[0], cu[-1] = 11, T - 37
    cu.clamp_(11, T - 37)
    cu = cu.sort().values
    a["cu_seqlens"] = cu
    a["weight"][int(cu[2]):int(cu[3])] = 0.0
    for reduction in ("sum", "token", "sequence"):
        clean = both(a, reduction=reduction, kl_coef=0.05)
        b = {k: v.clone() for k, v in a.items()}
        t = torch.arange(T, device="cuda")
        dead = (t < 11) | (t >= T - 37) | (b["weight"] == 0)
        for k, v in (("logprob", float("nan")), ("old_logprob", -float("inf")), ("advantage", float("inf")), ("ref_logprob", float("nan"))):
            b[k][dead] = v
        b["weight"][:11], b["weight"][T - 37:] = 5.0, float("nan")
        got = tik.tik_policy_loss(**b, reduction=reduction, kl_coef=0.05)
        for x, y in zip(got, clean):
            assert torch.equal(x, y)
        assert bool((got[1][dead] == 0).all())


@pytest.mark.parametrize("T", [100, 40000])
def test_all_masked(T):
    a = make(T, 4, seed=6)
    a["weight"].zero_()
    for reduction in ("sum", "token", "sequence"):
        loss, d, stats = tik.tik_policy_loss(**a, reduction=reduction, kl_coef=0.05)
        assert float(loss) == 0 and not d.any() and not stats.any()


def test_thresholds_are_decided_in_64_bits():
    """Tokens a step of fp32 on either side of a threshold, far from and near to zero."""
    low, high, dual = 0.2, 0.28, 3.0
    marks = [math.log1p(float(torch.tensor(high))), math.log1p(-float(torch.tensor(low))), math.log(dual)]
    old = torch.tensor([-0.5, -1.75, -7.0, -2.0 ** -12, -40.0], device="cuda")
    lps, olds = [], []
    for m in marks:
        base = (old.double() + m).float()
        for k in (-2, -1, 0, 1, 2):
            v = base.clone()
            for _ in range(abs(k)):
                v = torch.nextafter(v, torch.full_like(v, math.copysign(math.inf, k)))
            lps.append(v)
            olds.append(old)
    lp, old = torch.cat(lps), torch.cat(olds)
    for sign in (1.0, -1.0):
        a = dict(logprob=lp, old_logprob=old, advantage=torch.full_like(lp, sign))
        both(a, clip_low=low, clip_high=high, clip_dual=dual)
    none = tik.tik_policy_loss(lp, old, torch.zeros_like(lp))
    assert not none[1].any() and float(none[2][2]) == 0


def test_infinities_of_counted_tokens_pass_on():
    a = make(64, 1, seed=7, ref=False, weight=False)
    a["logprob"][3], a["advantage"][3] = 200.0, -1.0               # a ratio beyond fp32, not cut
    loss, d, _ = tik.tik_policy_loss(**a)
    assert float(loss) == math.inf and float(d[3]) == math.inf and bool(torch.isfinite(d[:3]).all())
    loss, d, _ = tik.tik_policy_loss(**a, clip_dual=2.0)
    assert math.isfinite(float(loss)) and float(d[3]) == 0


def test_gradient_against_differences():
    a = make(500, 8, seed=9, per_seq=True)
    kw = dict(kl_coef=0.07, reduction="sequence", scale=0.125, clip_dual=3.0)
    _, d, _ = tik.tik_policy_loss(**a, **kw)
    h = 2.0 ** -10
    step = torch.where(torch.rand(500, device="cuda") < 0.5, -h, h)
    up, down = dict(a), dict(a)
    up["logprob"], down["logprob"] = a["logprob"] + step, a["logprob"] - step
    lu, ld = expected(**up, **kw)[0][0], expected(**down, **kw)[0][0]
    along = (d.double() * (up["logprob"].double() - down["logprob"].double())).sum()
    # second-order terms cancel; a token within h of a threshold is off by its slope, |f A r| 2 h at most
    x = (a["logprob"] - a["old_logprob"]).double()
    close = torch.zeros_like(x, dtype=torch.bool)
    for m in (math.log1p(0.2), math.log1p(-0.2), math.log(3.0)):
        close |= (x - m).abs() < 1.01 * h
    f = expected(**a, **{**kw, "kl_coef": 0.0, "clip_low": 0.0, "clip_high": 0.0})[1][0]        # (only to know the signs in use)
    assert f.shape == d.shape
    weight = a["weight"].double() * 0.125
    worst = (weight * 4.0 * x.exp() * 2 * h)[close].sum() + 500 * 4.0 * h ** 3 + 1e-6 * h
    assert abs((lu - ld) - along) <= worst


def test_without_a_gradient_and_in_place():
    a = make(5000, 12, seed=10)
    loss, d, stats = tik.tik_policy_loss(**a, kl_coef=0.05)
    l2, none, s2 = tik.tik_policy_loss(**a, kl_coef=0.05, grad=False)
    assert none is None and torch.equal(loss, l2) and torch.equal(stats, s2)
    for T in (5000, 50000):
        a = make(T, 12, seed=10)
        loss, d, stats = tik.tik_policy_loss(**a, kl_coef=0.05)
        b = {k: v.clone() for k, v in a.items()}
        l3, d3, _ = tik.tik_policy_loss(**b, kl_coef=0.05, d_logprob=b["logprob"])
        assert d3.data_ptr() == b["logprob"].data_ptr() and torch.equal(d3, d) and torch.equal(l3, loss)


@pytest.mark.parametrize("T", [4097, 60013, 1000003])
def test_a_chain_of_calls_on_one_tensor(T):
    """A call reads what the call before it wrote, without a synchronisation in between: its kernels begin under that call's tail."""
    a = make(T, 12, seed=14)
    kw = dict(kl_coef=0.05, reduction="sum", scale=1e-3)          # (x -> 1e-3 w (-A) exp(x - old): |x| < 1 throughout; with 0.5 it grows to infinity)

    def chain(sync):
        b = dict(a, logprob=a["logprob"].clone(), weight=a["weight"].clone())
        losses = []
        for i in range(12):
            losses.append(tik.tik_policy_loss(**b, **kw, d_logprob=b["weight" if i % 3 == 2 else "logprob"])[0])
            if sync:
                torch.cuda.synchronize()
        return torch.stack(losses), b["logprob"], b["weight"]

    want = chain(True)
    assert bool(want[0].isfinite().all())
    for _ in range(3):
        for x, y in zip(chain(False), want):
            assert torch.equal(x, y)


def test_views_at_odd_addresses():
    T = 1000
    flat = {k: (v if k == "cu_seqlens" else torch.cat([v[:1], v])[1:]) for k, v in make(T, 5, seed=11).items()}
    assert flat["logprob"].data_ptr() % 16 == 4
    both(flat, kl_coef=0.02)


def test_no_tokens():
    e = torch.empty(0, device="cuda")
    loss, d, stats = tik.tik_policy_loss(e, e, e)
    assert float(loss) == 0 and d.numel() == 0 and not stats.any()
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    loss, d, stats = tik.tik_policy_loss(e, e, torch.ones(3, 1, device="cuda"), weight=e, cu_seqlens=cu, reduction="sequence")
    assert float(loss) == 0 and not stats.any()


@pytest.mark.parametrize("T", [900, 100000])
def test_captured_replayed_and_the_same_bits(T):
    a = make(T, 50, seed=12, per_seq=True)
    kw = dict(kl_coef=0.05, reduction="sequence")
    first = tik.tik_policy_loss(**a, **kw)
    for _ in range(5):
        for x, y in zip(first, tik.tik_policy_loss(**a, **kw)):
            assert torch.equal(x, y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = tik.tik_policy_loss(**a, **kw)
    b = make(T, 50, seed=13, per_seq=True)
    for k in a:
        a[k].copy_(b[k])
    for _ in range(3):
        g.replay()
    for x, y in zip(got, tik.tik_policy_loss(**b, **kw)):
        assert torch.equal(x, y)
