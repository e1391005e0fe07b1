"""tik_adamw's clip by a norm: gradients far above the limit, and a step beside the same step after a clip that was written back.

Tolerances, u = 2^-24.  A clipped gradient has the roundings of the factor and of the product: 2 u.  m: one of 1 - beta1, of the product and of the sum
more, 5 u of the terms' magnitudes.  v: the clipped gradient's twice, one of 1 - beta2, two of products, one of the sum: 8 u, taken as 9.  The step's
quotient: half of v's, a root and a reciprocal of two steps each, two products and a sum: 16 u of itself, taken as 18, and what m's error moves it
by; the weight three more of itself."""
import math

import pytest
import torch

from paper_2609_35140_b200 import binding as tik
from test_gpu_adamw import BF, F32, HYPER, KINDS, U, check, copy, make, moments, scale_values, step

pytestmark = pytest.mark.gpu


def zero_state(tensors):
    for t in tensors:
        for k in ("m", "v", "ms", "vs"):
            if t[k] is not None:
                t[k].view(torch.uint8).zero_()


@pytest.mark.parametrize("zeros", [True, False])
@pytest.mark.parametrize("size", [1e3, 1e12, 1e22, 1e30, 1e34])
def test_gradients_far_above_the_limit(size, zeros):
    a = make([3000, 33], seed=15, **KINDS[1])
    if zeros:
        zero_state(a)
    for t in a:
        t["g"].mul_(size / 1e-3)
    norm = tik.tik_grad_norm([t["g"] for t in a])
    assert math.isfinite(float(norm)) and float(norm) > size
    b = copy(a)
    n, lr = (1, 1e-3) if zeros else (7, 1e-3)
    step(a, n=n, norm=norm, max_norm=1.0)
    for x, y in zip(b, a):
        g = x["g"].double() / float(norm)
        m0, v0 = moments(x)
        m, v = 0.9 * m0 + (1 - 0.9) * g, 0.999 * v0 + (1 - 0.999) * g * g
        e_m, e_v = 5 * U * (0.9 * m0.abs() + 0.1 * g.abs()), 9 * U * v
        denominator = (v / (1 - 0.999 ** n)).sqrt() + HYPER["eps"]
        change = lr / (1 - 0.9 ** n) * m / denominator
        w0 = x["p"].double()
        w = (1 - lr * HYPER["weight_decay"]) * w0 - change
        e_w = 3 * U * (w0.abs() + w.abs()) + 18 * U * change.abs() + lr / (1 - 0.9 ** n) / denominator * e_m
        for got, ref, bound in ((y["m"], m, e_m), (y["v"], v, e_v), (y["p"], w, e_w)):
            assert bool(((got.double() - ref).abs() <= bound + 1e-44).all())


@pytest.mark.parametrize("kind", [3, 5])
def test_gradients_far_above_the_limit_with_8_bit_moments(kind):
    for zeros in (True, False):
        a = make([3000, 33], seed=16, **KINDS[kind])
        if zeros:
            zero_state(a)
        for t in a:
            t["g"].mul_(1e25)
        norm = tik.tik_grad_norm([t["g"] for t in a])
        b = copy(a)
        step(a, n=1 if zeros else 7, norm=norm, max_norm=1.0)
        check(b, a, n=1 if zeros else 7, clip=1.0 / float(norm))


@pytest.mark.parametrize("kind", [0, 1, 2, 4, 5])
def test_a_clip_on_the_way_is_one_that_was_written_back(kind):
    """The two gradients differ by the written one's rounding, 2^-8 of it in bf16 and 2^-24 in fp32; m by as much of its part, the root of v by as
    much of itself; an 8-bit value by that and its own rounding, half a step each: 2^-3 of it, or 2^-9 of its block's unit."""
    a = make([3000, 5], seed=17, **KINDS[kind])
    norm = tik.tik_grad_norm([t["g"] for t in a])
    limit = float(norm) / 3
    c = copy(a)
    before = copy(a)
    step(a, norm=norm, max_norm=limit)
    tik.tik_grad_clip([t["g"] for t in c], limit)
    assert bool((c[0]["g"].float() != a[0]["g"].float()).any())
    step(c)
    for x, y, b in zip(a, c, before):
        rate = (2.0 ** -8 if x["g"].dtype == BF else U) + 12 * U
        g = b["g"].double() / 3 * (1 + 4 * U)
        m0, v0 = moments(b)
        d_m, d_root = rate * 0.1 * g.abs() + 10 * U * 0.9 * m0.abs(), rate * (0.999 * v0 + 0.001 * g * g).sqrt()
        (xm, xv), (ym, yv) = moments(x), moments(y)
        if x["ms"] is not None:
            def unit(k):
                return torch.maximum(*(scale_values(t[k], xm.numel()) for t in (x, y)))
            d_m = d_m + torch.maximum(2.0 ** -3 * torch.maximum(xm.abs(), ym.abs()), 2.0 ** -9 * unit("ms"))
            d_root = d_root + torch.maximum(2.0 ** -3 * torch.maximum(xv, yv).sqrt(), 2.0 ** -9 * unit("vs"))
        assert bool(((xm - ym).abs() <= d_m).all())
        assert bool(((xv.sqrt() - yv.sqrt()).abs() <= d_root).all())
        # the step by m's and the root's differences before they are stored
        denominator = ((0.999 * v0 + 0.001 * g * g) / (1 - 0.999 ** 7)).sqrt() + 1e-8
        m = 0.9 * m0.abs() + 0.1 * g.abs()
        far = 1e-3 / (1 - 0.9 ** 7) / denominator * (rate * 0.1 * g.abs() + m * (rate + 24 * U))
        w = (x["w"] if x["w"] is not None else x["p"]).double(), (y["w"] if y["w"] is not None else y["p"]).double()
        stored = 2.0 ** -7 if x["w"] is None and x["p"].dtype == BF else 0.0
        assert bool(((w[0] - w[1]).abs() <= far + (8 * U + stored) * torch.maximum(w[0].abs(), w[1].abs())).all())


def test_a_clip_changes_no_bit_of_fp32_steps():
    """Scaled by the same factor with the same rounding, wherever that is done."""
    a = make([3000, 5], seed=18, param=F32, grad=F32)
    norm = tik.tik_grad_norm([t["g"] for t in a])
    limit = float(norm) / 3
    c = copy(a)
    step(a, norm=norm, max_norm=limit)
    tik.tik_grad_clip([t["g"] for t in c], limit)
    step(c)
    for x, y in zip(a, c):
        for k in ("p", "m", "v"):
            assert torch.equal(x[k], y[k])
