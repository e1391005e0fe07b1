"""tik_policy_loss where ratios are far from 1, against the definition and within the tolerances of test_gpu_policy_loss.py."""
import math

import pytest
import torch

from paper_2609_35140_b200 import binding as tik
from test_gpu_policy_loss import expected, make

pytestmark = pytest.mark.gpu
SIZES = [40, 3000, 9000]                                  # one CTA, a cluster, a grid


def compare(a, stats=(0, 1, 2, 4), **kw):
    """Everything but the statistics left out, and what they come to: those of a ratio beyond fp32 are infinite."""
    loss, d, s = tik.tik_policy_loss(**a, **kw)
    (l_ref, l_off), (d_ref, d_off), (s_ref, s_off) = expected(**a, **kw)
    assert abs(float(loss) - float(l_ref)) <= float(l_off) + 1e-38
    assert bool(((d.double() - d_ref).abs() <= d_off + 1e-38).all())
    for i in stats:
        assert abs(float(s[i]) - float(s_ref[i])) <= float(s_off[i]) + 1e-38, i
    return loss, d, s


@pytest.mark.parametrize("T", SIZES)
@pytest.mark.parametrize("per_seq", [False, True])
@pytest.mark.parametrize("dual", [0.0, 3.0])
def test_no_advantage_and_a_ratio_beyond_fp32(T, per_seq, dual):
    """Advantages of a group whose rewards agree are exactly 0: its terms are 0 whatever the ratio is."""
    a = make(T, 5, seed=1, per_seq=per_seq, ref=False)
    none = torch.tensor([1, 3], device="cuda") if per_seq else torch.arange(0, T, 3, device="cuda")
    a["advantage"][none] = 0.0
    a["advantage"][none[0]] = -0.0
    t = torch.arange(T, device="cuda")
    zero = (a["advantage"][:, 0][torch.searchsorted(a["cu_seqlens"][1:].contiguous(), t.int(), right=True).clamp(max=4)] if per_seq else a["advantage"]) == 0
    assert bool(zero.any())
    a["logprob"][zero] = a["old_logprob"][zero] + torch.where(t % 2 == 0, 100.0, 88.8)[zero]
    for reduction in ("sum", "token", "sequence"):
        _, d, stats = compare(a, reduction=reduction, clip_dual=dual)
        assert not d[zero].any()
    # what is not finite itself goes on
    at = int((zero & (a["weight"] != 0)).nonzero()[0])
    for bad in (math.inf, math.nan):
        a["logprob"][at] = bad
        loss, d, _ = tik.tik_policy_loss(**a)
        assert math.isnan(float(loss)) and math.isnan(float(d[at]))


@pytest.mark.parametrize("T", [1] + SIZES)
@pytest.mark.parametrize("reduction", ["sum", "token", "sequence"])
def test_ratios_far_below_one_keep_their_digits(T, reduction):
    """Advantages above 0 of tokens that the policy has left, which no threshold cuts: r down to e^-80."""
    a = make(T, 3, seed=2, weight=False, ref=False)
    t = torch.arange(T, device="cuda")
    a["advantage"] = 0.1 + a["advantage"].abs()
    far = torch.linspace(1.0, 80.0, T, device="cuda") if T > 1 else torch.tensor([12.5], device="cuda")
    a["logprob"] = a["old_logprob"] - far
    _, d, _ = compare(a, stats=range(5), reduction=reduction)
    assert bool((d < 0).all())
    # beside others, and as the smaller side of a threshold
    a["advantage"][t % 3 == 1] *= -1.0
    a["logprob"][t % 4 == 2] = a["old_logprob"][t % 4 == 2] + 0.1
    for ref in (None, a["old_logprob"] + 0.3):
        compare(dict(a, ref_logprob=ref), stats=range(5), reduction=reduction, kl_coef=0.0 if ref is None else 0.05)


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_around_the_ends_of_the_series(sign):
    """x within some steps of -1 and 1, where one way of taking r ends and another begins."""
    old = torch.full((64,), -3.0, device="cuda")
    x = (1.0 + torch.arange(-32, 32, device="cuda") * 2.0 ** -21) * sign
    a = dict(logprob=old + x, old_logprob=old, advantage=torch.linspace(-2, 2, 64, device="cuda"))
    compare(a, stats=range(5), clip_low=0.9, clip_high=9.0)


@pytest.mark.parametrize("T", SIZES)
def test_a_kl_term_that_is_only_looked_at(T):
    """kl_coef 0 beside a reference: the loss and its gradient are those without one, however far off the reference is."""
    a = make(T, 4, seed=3)
    none = dict(a, ref_logprob=None)
    for reduction in ("sum", "token", "sequence"):
        near, far = tik.tik_policy_loss(**a, reduction=reduction), dict(a, ref_logprob=a["logprob"] + 95.0)
        want, got = tik.tik_policy_loss(**none, reduction=reduction), tik.tik_policy_loss(**far, reduction=reduction)
        for x in (near, got):
            assert torch.equal(x[0], want[0]) and torch.equal(x[1], want[1])
            assert torch.equal(x[2][[0, 2, 3, 4]], want[2][[0, 2, 3, 4]])
        assert 0 < float(near[2][1]) < math.inf and float(got[2][1]) == math.inf
