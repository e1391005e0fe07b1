"""GPU parity of the global gradient norm and of clipping by it: the norm against fp64, the clipped gradients bit for bit from
the norm that was returned."""
import numpy as np
import pytest
import torch

import oracle
from gpu_common import count_diff

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def tik():
    from paper_2609_35140_b200 import binding
    binding.load()
    yield binding
    assert binding.device_status() == 0


def _randn(n, seed, std=1.0, dtype=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, generator=g, device="cuda") * std).to(dtype)


def _norm(grads):
    return oracle.grad_norm([g.double().cpu().numpy() for g in grads])


def _close(got, ref):
    """At most 16 additions in a chain of fp32 squares and three more, all of one sign, then fp64; the root halves that;
    one rounding: ten half steps and a half."""
    assert got.dtype == F32 and got.shape == (1,)
    assert abs(float(got.double()) - ref) <= 11 * U32 * ref, (float(got), ref)


def _expected(g, norm, limit):
    n = np.float32(norm.item())
    if not (n > np.float32(limit) and np.isfinite(n)):
        return g.clone()
    return (g.float() * float(np.float32(limit) / n)).to(g.dtype)


LISTS = {
    "one": [(1, BF)], "one_fp32": [(1, F32)], "row": [(3584, BF)], "ragged": [(n, BF) for n in (1, 7, 8, 9, 4097, 0, 16385, 3)],
    "mixed": [(513, F32), (1025, BF), (0, F32), (2, F32), (33000, F32), (33000, BF)], "chunk": [(8 * 2048 + d, BF) for d in (-1, 0, 1)] + [(4 * 2048 + d, F32) for d in (-1, 0, 1)],
    "large": [(5_000_011, BF), (3_000_001, F32), (11, BF)], "many": [(17 + i % 5, BF if i % 3 else F32) for i in range(2100)],
    "sixty_five": [(100 + i, BF) for i in range(65)], "thousand": [(9, F32)] * 1000, "thousand_one": [(9, BF)] * 1001,
}


@pytest.mark.parametrize("name", list(LISTS))
@pytest.mark.parametrize("factor", [0.37, 1.7])
def test_norm_and_clip(tik, name, factor):
    grads = [_randn(n, i, 0.1, t) for i, (n, t) in enumerate(LISTS[name])]
    keep = [g.clone() for g in grads]
    norm = tik.tik_grad_norm(grads)
    ref = _norm(grads)
    _close(norm, ref)
    limit = factor * ref
    out = [torch.full_like(g, 7.0) for g in grads]
    n2 = tik.tik_grad_clip(grads, limit, out=out)
    assert count_diff(n2, norm) == 0
    n3 = tik.tik_grad_clip(tuple(grads), limit)                        # in place
    assert count_diff(n3, norm) == 0
    for g, k, o in zip(grads, keep, out):
        want = _expected(k, norm, limit)
        assert count_diff(g, want) == 0 and count_diff(o, want) == 0
        assert (factor > 1) == (count_diff(g, k) == 0) or g.numel() == 0 or not bool((k != 0).any())
    # the norm of another call (ranks' norms combined): the same factor from there
    again = [k.clone() for k in keep]
    given = norm.clone()
    assert tik.tik_grad_clip(again, limit, norm=given) is given
    for a, g in zip(again, grads):
        assert count_diff(a, g) == 0


@pytest.mark.parametrize("dtype", [BF, F32])
def test_views_of_a_flat_buffer_at_any_element(tik, dtype):
    """Bases and ends at every offset from a 16-byte boundary, results at other offsets than the gradients; the elements
    between the views stay."""
    per = 8 if dtype == BF else 4
    for shift in range(per):
        flat = _randn(40_000, 3, 1.0, dtype)
        cuts = [(shift, 5), (shift + 9, 1), (shift + 16, 16), (100 + shift, 77), (500 + shift, 20_003 + shift), (30_000, 0), (30_001 + shift, 9000)]
        views = [flat[a:a + n] for a, n in cuts]
        keep = flat.clone()
        ref = _norm(views)
        for to in (None, 0, 1, per - 1):
            flat.copy_(keep)
            if to is None:
                norm = tik.tik_grad_clip(views, 0.1 * ref)
                got, base = flat, keep.clone()
            else:
                got = torch.full((40_016,), 7.0, dtype=dtype, device="cuda")
                base = got.clone()
                norm = tik.tik_grad_clip(views, 0.1 * ref, out=[got[a + to:a + to + n] for a, n in cuts])
                assert count_diff(flat, keep) == 0
            _close(norm, ref)
            for a, n in cuts:
                base[a + (to or 0):a + (to or 0) + n] = _expected(keep[a:a + n], norm, 0.1 * ref)
            assert count_diff(got, base) == 0, (shift, to)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("std", [1e-38, 1e-30, 1e-21, 1e-12, 1e12, 1e19, 1e30, 3e37])
def test_magnitudes_whose_squares_leave_fp32(tik, dtype, std):
    grads = [_randn(3000, 1, std, dtype), torch.zeros(5000, dtype=dtype, device="cuda"), _randn(70_001, 2, std, dtype), _randn(3, 3, std, dtype)]
    ref = _norm(grads)
    norm = tik.tik_grad_norm(grads)
    if ref > 3.4e38:
        assert bool(torch.isinf(norm))
    else:
        # a norm among fp32's subnormal numbers is off by half of their step at most
        assert abs(float(norm.double()) - ref) <= 11 * U32 * ref + 2.0 ** -150


def test_a_sum_of_small_and_large(tik):
    """2^26 ones and one 2^14: fp32 running sums would stop at 2^24."""
    grads = [torch.ones(1 << 26, dtype=BF, device="cuda"), torch.full((1,), 2.0 ** 14, device="cuda")]
    assert float(tik.tik_grad_norm(grads)) == float(np.float32(np.sqrt(2.0 ** 26 + 2.0 ** 28)))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_norm_that_is_not_finite_leaves_the_gradients(tik, bad, dtype):
    grads = [_randn(20_000, 1, 1.0, dtype), _randn(9, 2, 1.0, dtype)]
    for where in (0, 17_777):
        g = [x.clone() for x in grads]
        g[0][where] = bad
        keep = [x.clone() for x in g]
        norm = tik.tik_grad_clip(g, 0.5)
        assert bool(torch.isnan(norm)) if bad != bad else bool(torch.isinf(norm)) and float(norm) > 0
        out = [torch.empty_like(x) for x in g]
        tik.tik_grad_clip(g, 0.5, out=out)
        for x, k, o in zip(g, keep, out):
            assert count_diff(x, k) == 0 and count_diff(o, k) == 0
        given = torch.tensor([bad], device="cuda")
        tik.tik_grad_clip(g, 0.5, norm=given)
        assert all(count_diff(x, k) == 0 for x, k in zip(g, keep))


def test_empty_lists_and_zero_gradients(tik):
    assert float(tik.tik_grad_norm([])) == 0.0 and float(tik.tik_grad_clip([], 1.0)) == 0.0
    none = torch.empty(0, dtype=BF, device="cuda")
    assert float(tik.tik_grad_norm([none, none])) == 0.0 and float(tik.tik_grad_clip((none,), 1.0)) == 0.0
    zeros = [torch.zeros(70_000, dtype=BF, device="cuda"), torch.zeros(5, device="cuda")]
    assert float(tik.tik_grad_clip(zeros, 1e-30)) == 0.0 and all(bool((z == 0).all()) for z in zeros)
    # a tensor listed twice counts twice in the norm
    g = _randn(1000, 1)
    _close(tik.tik_grad_norm([g, g]), np.sqrt(2.0) * _norm([g]))


def test_the_border_is_not_clipped(tik):
    g = torch.tensor([3.0, 4.0], device="cuda")
    tik.tik_grad_clip([g], 5.0)
    assert g.tolist() == [3.0, 4.0]
    tik.tik_grad_clip([g], float(np.nextafter(np.float32(5), np.float32(0))))
    assert g.tolist() != [3.0, 4.0]


def test_captured_and_replayed_on_new_gradients(tik):
    for n_tensors in (5, 300):
        grads = [_randn(1000 + 37 * i, i, 1.0, BF if i % 2 else F32) for i in range(n_tensors)]
        out = [torch.empty_like(g) for g in grads]
        norm = torch.empty(1, device="cuda")
        ws = torch.empty(tik.workspace_bytes(tik.OP_GRAD_NORM, n_tensors), dtype=torch.uint8, device="cuda")
        small = torch.zeros(1, device="cuda")

        def step():
            tik.tik_grad_norm(grads, norm=norm, ws=ws)
            tik.tik_grad_clip(grads, 1.0, norm=norm, out=out)
            small.copy_(tik.tik_grad_clip(out, 0.25, ws=ws))

        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for seed in (50, 60):
            for i, t in enumerate(grads):
                t.copy_(_randn(t.numel(), seed + i, 2.0))
            ws.fill_(255)
            g.replay()
            got = [o.clone() for o in out] + [norm.clone(), small.clone()]
            step()
            for a, b in zip(out + [norm, small], got):
                assert count_diff(a, b) == 0


def test_refused_lists(tik):
    g, out = _randn(64, 1), _randn(64, 2)
    for bad in (lambda: tik.tik_grad_norm([g.half()]), lambda: tik.tik_grad_norm([g.cpu()]), lambda: tik.tik_grad_norm([g[::2]]),
                lambda: tik.tik_grad_clip([g, g], 1.0), lambda: tik.tik_grad_clip([g], 0.0), lambda: tik.tik_grad_clip([g], float("inf")),
                lambda: tik.tik_grad_clip([g[:40], out], 1.0, out=[out[:40], g]), lambda: tik.tik_grad_clip([g[:32]], 1.0, out=[g[16:48]]),
                lambda: tik.tik_grad_norm([g], ws=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(tik.TikError):
            bad()
    for bad in (lambda: tik.tik_grad_clip([g], 1.0, out=[out[:32]]), lambda: tik.tik_grad_clip([g], 1.0, out=[out.float()]),
                lambda: tik.tik_grad_clip([g], 1.0, out=[]), lambda: tik.tik_grad_norm([g], norm=torch.empty(2, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: tik.tik_grad_norm(g), lambda: tik.tik_grad_norm([3.0]), lambda: tik.tik_grad_clip([g], 1.0, out=out)):
        with pytest.raises(TypeError):
            bad()
