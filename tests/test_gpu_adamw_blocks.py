"""tik_adamw with 8-bit moments where a block's elements lie far apart: codes that round to 0 beside large ones.

Values far below their block's largest are stored as 0 or 2^-9 of the block's unit: a root that is not 0 as 2^-9, whatever is beside it; a first moment
to the nearest as 0, and with a seed as 2^-9 with the probability of its distance from 0, so that its mean over n draws is its value within 6
standard deviations (of at most half the gap over sqrt(n)) and 16 bits of randomness."""
import math

import pytest
import torch

from test_gpu_adamw import BF, E8, F32, FP8, check, copy, moments, step

pytestmark = pytest.mark.gpu


def scene(n, shift=0, param=F32, master=False):
    """One tensor of n elements from zero 8-bit moments, gradients 1, `shift` elements into its buffers."""
    def place(x):
        buf = torch.zeros(n + shift, dtype=x.dtype, device="cuda")
        out = buf[shift:]
        out.copy_(x)
        return out
    zero = torch.zeros(-(-n // 32), dtype=torch.uint8, device="cuda")
    w = torch.linspace(-1, 1, n, device="cuda")
    return dict(p=place(w.to(param)), g=place(torch.ones(n, device="cuda")), w=place(w) if master else None, ms=zero.clone().view(E8), vs=zero.clone().view(E8),
                m=place(torch.zeros(n, device="cuda").to(FP8)), v=place(torch.zeros(n, device="cuda").to(FP8)))


@pytest.mark.parametrize("seed", [None, 5])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("width,at", [(1, 0), (4, 0), (4, 12), (4, 27), (8, 8), (8, 3), (24, 8), (24, 5), (31, 0), (31, 1)])
@pytest.mark.parametrize("others", [1.0, 0.0])
def test_small_neighbours_of_a_large_element(width, at, shift, seed, others):
    n, tiny = 32 * 2048 + 32, 1e-6
    t = scene(n, shift)
    place = torch.arange(n, device="cuda") % 32
    run = (place >= at) & (place < at + width)
    t["g"].fill_(others)
    t["g"][place == (at + width) % 32] = 1.0               # the block's largest
    t["g"][run] = tiny
    b = copy([t])
    step([t], n=1, seed=seed)
    check(b, [t], n=1, seed=seed)
    code = t["v"].view(torch.uint8)
    assert bool((code[run] == 1).all())                    # 1e-6 of the largest: below half of the least value
    assert bool((code[t["g"] == 0] == 0).all())
    m = t["m"].view(torch.uint8)[run]
    if seed is None:
        assert not m.any()
        return
    assert bool((m <= 1).all())
    unit = float(moments(t)[0].max()) / float(t["m"].float().max()) * 2.0 ** -9
    want = 0.1 * tiny
    assert abs(float(m.double().mean()) * unit - want) <= unit * (3 / math.sqrt(m.numel()) + 2.0 ** -16) + 1e-6 * want


@pytest.mark.parametrize("seed", [None, 6])
def test_a_block_whose_largest_root_doubles(seed):
    """Neighbours at the least value, which the block's new unit makes half of it: they stay."""
    n = 32 * 64
    t = scene(n)
    place = torch.arange(n, device="cuda") % 32
    t["v"].view(torch.uint8).fill_(1)
    t["v"].view(torch.uint8)[place == 9] = 126             # 448
    for k in ("ms", "vs"):
        t[k].view(torch.uint8).fill_(110)
    t["m"].view(torch.uint8).fill_(56)
    t["g"].zero_()
    t["g"][place == 9] = 2 * 448 * 2.0 ** -17 / math.sqrt(0.001)
    b = copy([t])
    step([t], n=50, seed=seed)
    check(b, [t], n=50, seed=seed)
    assert bool((t["v"].view(torch.uint8)[place != 9] == 1).all())


@pytest.mark.parametrize("seed", [None, 7])
@pytest.mark.parametrize("tiny", [1e-4, 1e-6, 1e-9])
def test_vectors_and_single_elements_have_the_same_bits(seed, tiny):
    n = 5003
    g = torch.Generator(device="cuda").manual_seed(1)
    grad = torch.where(torch.rand(n, generator=g, device="cuda") < 0.1, 1.0, tiny) * torch.randn(n, generator=g, device="cuda")
    got = []
    for shift in (0, 1):
        t = scene(n, shift, param=BF)
        t["g"].copy_(grad)
        for i in range(1, 4):
            step([t], n=i, seed=seed)
        got.append([t[k].clone().view(torch.uint8) for k in ("p", "m", "v", "ms", "vs")])
    for x, y in zip(*got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("seed", [None, 8])
@pytest.mark.parametrize("param,master", [(F32, False), (BF, True)])
def test_steps_in_a_row(seed, param, master):
    """Gradients that come and go over six decades: every step from the state that the one before it left."""
    t = scene(32 * 100 + 7, param=param, master=master)
    g = torch.Generator(device="cuda").manual_seed(2)
    for n in range(1, 31):
        size = 10.0 ** torch.randint(-6, 1, (t["g"].numel(),), generator=g, device="cuda").float()
        t["g"].copy_(torch.randn(t["g"].numel(), generator=g, device="cuda") * size * (torch.rand(t["g"].numel(), generator=g, device="cuda") < 0.7))
        b = copy([t])
        step([t], n=n, seed=seed)
        check(b, [t], n=n, seed=seed)
