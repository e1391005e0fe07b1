"""Policy loss, log-probability gradient and AdamW step on tensors whose offsets pass 31 and 32 bits."""
import math

import pytest
import torch

from paper_2609_35140_b200 import binding as tik
from test_gpu_adamw import E8, F32, FP8, HYPER
from test_gpu_logprob_bwd import U16, U32, expected, near

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
STEP = 1 << 26


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    assert tik.device_status() == 0


def _fill(shape, seed, std=1.0, dtype=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for r in range(0, flat.numel(), STEP):
        n = min(STEP, flat.numel() - r)
        flat[r:r + n] = torch.randn(n, generator=g, device="cuda").mul_(std)
    return out


def _codes(n, low, high, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(n, dtype=torch.uint8, device="cuda")
    for r in range(0, n, STEP):
        out[r:r + STEP] = torch.randint(low, high, (min(STEP, n - r),), generator=g, device="cuda", dtype=torch.uint8)
    return out.view(dtype)


def _same(a, b):
    a, b = a.view(torch.uint8), b.view(torch.uint8)
    return all(torch.equal(a[r:r + (STEP << 3)], b[r:r + (STEP << 3)]) for r in range(0, a.numel(), STEP << 3))


@pytest.mark.parametrize("seed", [None, 3])
def test_adamw_8_bit_whole_and_in_parts(seed):
    """More than 2^32 elements: the whole tensor and three views of it, none of 2^31, come out alike, places of random numbers included."""
    n = (1 << 32) + 12_345
    cuts = [0, (1 << 31) - 32 * 1001, (1 << 32) - 64, n]
    grad = _fill((n,), 1, 1e-3)
    whole = dict(p=_fill((n,), 2, 0.02), m=_codes(n, 0, 127, 3, FP8), v=_codes(n, 1, 127, 4, FP8), ms=_codes(-(-n // 32), 105, 112, 5, E8),
                 vs=_codes(-(-n // 32), 106, 112, 6, E8))
    parts = {k: t.clone() for k, t in whole.items()}

    def step(x, cut):
        of = lambda t, per=1: [t[-(-a // per):-(-b // per)] for a, b in zip(cut, cut[1:])]  # noqa: E731
        tik.tik_adamw(of(x["p"]), of(grad), of(x["m"]), of(x["v"]), 1e-3, 7, **HYPER, exp_avg_scale=of(x["ms"], 32), exp_avg_sq_scale=of(x["vs"], 32), seed=seed)

    before = {k: t[-(n % 32) - 64:].clone() for k, t in whole.items() if k in "pmv"}
    step(whole, [0, n])
    step(parts, cuts)
    for k in whole:
        assert _same(whole[k], parts[k]), k
    for k, t in before.items():
        assert not torch.equal(whole[k][-t.numel():].view(torch.uint8), t.view(torch.uint8)), k


@pytest.mark.parametrize("shift", [0, 1])
def test_adamw_fp32_whole_and_in_parts(shift):
    """More than 2^31 elements, by vectors and by single elements."""
    n = (1 << 31) + 12_345
    bufs = dict(p=_fill((n + shift,), 1, 0.02, F32), m=_fill((n + shift,), 2, 1e-3, F32), v=_fill((n + shift,), 3, 1e-3, F32).square_())
    whole = {k: t[shift:] for k, t in bufs.items()}
    grad = _fill((n + shift,), 4, 1e-3, F32)[shift:]
    parts = {k: t.clone() for k, t in whole.items()}
    cut = (1 << 30) + 5                                    # (the second part begins at another address modulo 16)
    first, last = ({k: t[s].double() for k, t in whole.items()} for s in (slice(0, 50), slice(n - 50, n)))
    tik.tik_adamw([whole["p"]], [grad], [whole["m"]], [whole["v"]], 1e-3, 7, **HYPER)
    of = lambda t: [t[:cut], t[cut:]]  # noqa: E731
    tik.tik_adamw(of(parts["p"]), of(grad), of(parts["m"]), of(parts["v"]), 1e-3, 7, **HYPER)
    for k in whole:
        assert _same(whole[k], parts[k]), k
    for b, s in ((first, slice(0, 50)), (last, slice(n - 50, n))):
        m = 0.9 * b["m"] + 0.1 * grad[s].double()
        assert bool(((whole["m"][s].double() - m).abs() <= 5 * U32 * (0.9 * b["m"].abs() + 0.1 * grad[s].double().abs())).all())


def test_log_probability_gradient_of_many_rows():
    """d_hidden of more than 2^31 elements."""
    T, H, V = 300_007, 8_192, 300
    x, W = _fill((T, H), 1), _fill((V, H), 2, H ** -0.5)
    g = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    d = torch.randn(T, generator=g, device="cuda") * (torch.rand(T, generator=g, device="cuda") > 0.2)
    d[:3], d[T - 3:] = 1.0, -1.0
    lse = torch.empty(T, device="cuda")
    for r in range(0, T, 8192):
        lse[r:r + 8192] = torch.logsumexp(x[r:r + 8192].float() @ W.float().T, 1)
    dh, _ = tik.tik_token_logprob_bwd(d, x, W, ids, lse, need_lm_head=False)
    rows = torch.cat([torch.arange(40, device="cuda"), torch.arange(262_100, 262_180, device="cuda"), torch.arange(T - 40, T, device="cuda")])
    near(dh[rows], expected(d[rows], x[rows], W, ids[rows], lse[rows], 1.0)[0])
    masked = (d == 0).nonzero()[:, 0]
    assert not dh[masked[:100]].any() and not dh[masked[-100:]].any()


@pytest.mark.parametrize("T", [40, 300])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_log_probability_gradient_of_many_words(T, dtype):
    """d_lm_head of more than 2^31 elements, written and, in fp32, added to."""
    V, H = 300_007, 8_192
    W, x = _fill((V, H), 1, H ** -0.5), _fill((T, H), 2)
    at = torch.cat([torch.arange(64, device="cuda"), torch.arange(262_100, 262_180, device="cuda"), torch.arange(V - 64, V, device="cuda")])
    g = torch.Generator(device="cuda").manual_seed(3)
    pick = torch.randint(0, at.numel(), (T,), generator=g, device="cuda")
    pick[0], pick[1] = at.numel() - 1, 0
    d = torch.randn(T, generator=g, device="cuda") * (torch.rand(T, generator=g, device="cuda") > 0.2)
    d[:2] = 1.0
    ids = at[pick].int()
    lse = torch.logsumexp(torch.cat([x.float() @ W[r:r + 32_768].float().T for r in range(0, V, 32_768)], 1), 1)
    d_w = torch.empty(V, H, dtype=dtype, device="cuda")
    tik.tik_token_logprob_bwd(d, x, W, ids, lse, need_hidden=False, d_lm_head=d_w)
    want = expected(d, x, W[at], pick.int(), lse, 1.0)[1]
    near(d_w[at], want, out_u=U16 if dtype == BF else U32)
    if dtype == F32:
        one = d_w[at].clone()
        tik.tik_token_logprob_bwd(d, x, W, ids, lse, need_hidden=False, d_lm_head=d_w, accumulate=True)
        assert torch.equal(d_w[at], 2 * one)


def test_policy_loss_of_as_many_tokens_as_it_takes():
    T = (1 << 31) - 1
    same, weight = torch.zeros(T, device="cuda"), torch.ones(T, device="cuda")      # (the log-probabilities' tensors are one)
    weight[7] = weight[T - 3] = 0.0
    cu = torch.tensor([0, 5, T - 9, T], dtype=torch.int32, device="cuda")
    adv = torch.tensor([[-1.0], [2.0], [-4.0]], device="cuda")
    loss, d, stats = tik.tik_policy_loss(same, same, adv, weight=weight, cu_seqlens=cu, reduction="sequence", scale=0.5)
    # f_t = 0.5 / n: a rounding of it and one of the product
    for s, n in ((slice(0, 5), 5), (slice(5, T - 9), T - 15), (slice(T - 9, T), 8)):
        A = float(adv[0 if n == 5 else 2 if n == 8 else 1])
        assert bool(((d[s][:4096].double() * 2 * n / -A - (weight[s][:4096] != 0).double()).abs() <= 2.0 ** -22).all())
        assert bool(((d[s][-4096:].double() * 2 * n / -A - (weight[s][-4096:] != 0).double()).abs() <= 2.0 ** -22).all())
    assert int((d == 0).sum()) == 2
    assert abs(float(loss) - 1.5) <= 2.0 ** -22 and float(stats[4]) == float(torch.tensor(float(T - 2)))
    loss, d, stats = tik.tik_policy_loss(same, same, adv, weight=weight, cu_seqlens=cu, d_logprob=d)
    want = -(-1.0 * 5 + 2.0 * (T - 15) - 4.0 * 8) / (T - 2)
    assert abs(float(loss) - want) <= 2.0 ** -22 * abs(want) and math.isfinite(float(stats[3]))
    assert abs(float(d[T - 1]) * (T - 2) - 4.0) <= 2.0 ** -20 and float(d[7]) == 0 and float(d[T - 3]) == 0
