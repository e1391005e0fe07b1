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
