"""tik_token_logprob_bwd against its definition in 64 bits.

Tolerances, from the roundings that the operator makes.  Relative half steps: bf16 2^-8, fp32 2^-24.
 * A logit is a chain of H / 16 tensor-core additions in fp32, each off by at most 2^-23 of the terms' magnitudes; the exponent's
   arithmetic and ex2 add a few 2^-23 of |z| + |lse| + 1.  So p is off by E p, with E their sum.
 * d_z = c (hit - p) is off by c p E + 2^-23 |c| before and 2^-8 of itself through its rounding to bf16.
 * A gradient is a chain of K / 16 additions of d_z's products (K: tokens or vocabulary, and 64 parts at most), plus its own rounding.
Every element is held to that bound.  Independent roundings add up like a random walk: the 2-norm of the errors is held to 2^-8 of
the norm of sqrt(sum of squared terms) and of the result, which a single lost column of a sum would exceed, and the norm of what p's
errors come to, which a row's terms share (with a vocabulary of one, p = 1, they are all there is)."""
import pytest
import torch

from paper_2609_35140_b200 import binding as tik

pytestmark = pytest.mark.gpu
U16, U32 = 2.0 ** -8, 2.0 ** -24


def make(T, H, V, seed=0, f=1.0, masked=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    W = (rand(V, H) * H ** -0.5).bfloat16()
    ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    lean = torch.rand(T, 1, generator=g, device="cuda") * 6.0
    x = (rand(T, H) + lean * W.float()[ids.long()]).bfloat16()
    d = rand(T) * (torch.rand(T, generator=g, device="cuda") >= masked)
    lse = torch.empty(T, device="cuda")
    for r in range(0, T, 1024):
        lse[r:r + 1024] = torch.logsumexp(f * (x[r:r + 1024].double() @ W.double().T), 1)
    return d, x, W, ids, lse, f


def expected(d, x, W, ids, lse, f):
    """(d_hidden, its elements' bound, its terms' norm, the norm of what p's errors come to), the same of d_lm_head; 64 bits, rows in blocks."""
    T, H = x.shape
    V = W.shape[0]
    Wd, Wa = W.double(), W.double().abs()
    dh, bh, qh, ph = (torch.empty(T, H, dtype=torch.float64, device="cuda") for _ in range(4))
    dw, bw, qw, pw = (torch.zeros(V, H, dtype=torch.float64, device="cuda") for _ in range(4))
    block = max(1, min(T, (1 << 27) // V))
    for r in range(0, T, block):
        s = slice(r, min(T, r + block))
        xd = x[s].double()
        z = f * (xd @ Wd.T)
        ok = (ids[s] >= 0) & (ids[s] < V) & (d[s] != 0)
        p = torch.exp(z - lse[s, None].double())
        E = (H / 16 + 1) * 2 * U32 * f * (xd.abs() @ Wa.T) + 8 * U32 * (z.abs() + lse[s, None].double().abs() + 1)
        c = (f * d[s].double())[:, None]
        hit = torch.arange(V, device="cuda")[None] == ids[s, None]
        dz = torch.where(ok[:, None], c * (hit.double() - p), 0.0)
        e32 = torch.where(ok[:, None], (1 + U16) * c.abs() * (p * torch.expm1(E) + 2 * U32), 0.0)
        e = U16 * dz.abs() + e32
        dh[s] = dz @ Wd
        bh[s] = e @ Wa + (V / 16 + 66) * 2 * U32 * ((dz.abs() + e) @ Wa)
        qh[s] = (dz.square() @ Wd.square())
        ph[s] = e32 @ Wa
        dw += dz.T @ xd
        bw += e.T @ xd.abs() + (T / 16 + 2) * 2 * U32 * ((dz.abs() + e).T @ xd.abs())
        qw += dz.square().T @ xd.square()
        pw += e32.T @ xd.abs()
    return (dh, bh, qh.sum().sqrt(), ph.norm()), (dw, bw, qw.sum().sqrt(), pw.norm())


def near(got, want, out_u=U16):
    ref, bound, terms, shared = want
    off = (got.double() - ref).abs()
    assert torch.isfinite(got).all()
    assert bool((off <= bound + out_u * (ref.abs() + bound) + 1e-37).all()), (off - bound).max().item()
    assert off.norm() <= U16 * (terms + ref.norm()) + shared + 1e-30, (off.norm() / (terms + ref.norm())).item()


SIZES = [(1, 64, 1), (1, 64, 7), (1, 256, 5003), (2, 192, 64), (63, 64, 255), (64, 320, 256), (127, 128, 257), (128, 64, 1000),
         (129, 1088, 300), (255, 256, 2048), (257, 512, 513), (700, 192, 5003), (1000, 448, 1001)]


@pytest.mark.parametrize("T,H,V", SIZES)
def test_both_gradients(T, H, V):
    args = make(T, H, V, seed=T + H + V)
    dh, dw = tik.tik_token_logprob_bwd(*args)
    assert dh.dtype == dw.dtype == torch.bfloat16 and dh.shape == (T, H) and dw.shape == (V, H)
    a, b = expected(*args)
    near(dh, a)
    near(dw, b)
    assert tik.device_status() == 0


@pytest.mark.parametrize("T,H,V", [(4800, 1024, 1000), (2600, 1792, 777), (300, 64, 40001)])
def test_whole_and_split_tiles(T, H, V):
    """76 tiles on 74 pairs, 77, and a few tiles with a long sum."""
    args = make(T, H, V, seed=5)
    dh, dw = tik.tik_token_logprob_bwd(*args)
    a, b = expected(*args)
    near(dh, a)
    near(dw, b)


@pytest.mark.parametrize("T,H,V", [(16500, 64, 70001), (16500, 512, 66000), (20011, 128, 53761)])
def test_vocabulary_in_chunks(T, H, V):
    """More d_z than 2 GiB: chunks, whole tiles that grow in fp32 beside split ones; last chunks shorter than the others."""
    args = make(T, H, V, seed=6)
    dh, dw = tik.tik_token_logprob_bwd(*args)
    a, b = expected(*args)
    near(dh, a)
    near(dw, b)


@pytest.mark.parametrize("f", [0.5, 1.0, 1.7])
def test_temperature(f):
    args = make(200, 128, 900, seed=9, f=f)
    dh, dw = tik.tik_token_logprob_bwd(*args)
    a, b = expected(*args)
    near(dh, a)
    near(dw, b)


@pytest.mark.parametrize("T,H,V,masked", [(257, 64, 300, 0.0), (900, 192, 1111, 0.9), (1500, 256, 700, 0.5), (4700, 1024, 513, 0.03), (513, 64, 90, 0.999)])
def test_tokens_that_take_no_part(T, H, V, masked):
    """More than one row tile: the others' rows are gathered, by a number that stays on the device."""
    args = make(T, H, V, seed=21, masked=masked)
    dh, dw = tik.tik_token_logprob_bwd(*args)
    a, b = expected(*args)
    near(dh, a)
    near(dw, b)
    assert bool((dh[args[0] == 0] == 0).all())


@pytest.mark.parametrize("T", [200, 600])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_token_takes_part(T, dtype):
    d, x, W, ids, lse, f = make(T, 192, 500, seed=22)
    dw = torch.full((500, 192), 5.0, dtype=dtype, device="cuda")
    dh, _ = tik.tik_token_logprob_bwd(torch.zeros_like(d), x, W, ids, torch.full_like(lse, float("nan")), f, d_lm_head=dw)
    assert not dh.any() and not dw.any()
    keep = torch.full((500, 192), 5.0, device="cuda")
    tik.tik_token_logprob_bwd(torch.zeros_like(d), x, W, ids, lse, f, need_hidden=False, d_lm_head=keep, accumulate=True)
    assert bool((keep == 5.0).all())


@pytest.mark.parametrize("T,V", [(150, 40), (700, 3), (3000, 1000)])
def test_targets_that_many_tokens_share(T, V):
    """More targets among a warp's rows than its list holds."""
    d, x, W, ids, lse, f = make(T, 128, V, seed=23)
    ids[::2] = V - 1
    lse = torch.logsumexp(x.double() @ W.double().T, 1).float()
    dh, dw = tik.tik_token_logprob_bwd(d, x, W, ids, lse, f)
    a, b = expected(d, x, W, ids, lse, f)
    near(dh, a)
    near(dw, b)


def test_the_targets_rounding_is_made_good():
    """Where the target's term is all there is (its probability near 0, the others' spread), the gradients are as near as their own rounding."""
    T, H, V = 40, 256, 4096
    d, x, W, ids, lse, f = make(T, H, V, seed=24, masked=0.0)
    dh, dw = tik.tik_token_logprob_bwd(d, x, W, ids, lse, f)
    for got, want in zip((dh, dw), expected(d, x, W, ids, lse, f)):
        off = (got.double() - want[0]).norm() / want[0].norm()
        assert off <= 2.0 ** -9 * 1.05                   # a rounding to bf16 is off by 2^-8 / sqrt(3) of the norm at most, by 2^-9 nearly always


def test_one_output_alone_has_the_same_bits():
    args = make(333, 256, 1111, seed=1)
    dh, dw = tik.tik_token_logprob_bwd(*args)
    a, none = tik.tik_token_logprob_bwd(*args, need_lm_head=False)
    assert none is None and torch.equal(a, dh)
    none, b = tik.tik_token_logprob_bwd(*args, need_hidden=False)
    assert none is None and torch.equal(b, dw)
    mine = torch.full_like(dh, 7.0), torch.full_like(dw, 7.0)
    got = tik.tik_token_logprob_bwd(*args, d_hidden=mine[0], d_lm_head=mine[1])
    assert got[0].data_ptr() == mine[0].data_ptr() and got[1].data_ptr() == mine[1].data_ptr()
    assert torch.equal(mine[0], dh) and torch.equal(mine[1], dw)


@pytest.mark.parametrize("T,H,V", [(100, 64, 300), (513, 320, 1025)])
def test_fp32_table_and_accumulation(T, H, V):
    first, second = make(T, H, V, seed=2), make(T, H, V, seed=3)
    second = (second[0], second[1], first[2], second[3], torch.logsumexp(second[1].double() @ first[2].double().T, 1).float(), 1.0)
    d_w = torch.full((V, H), 9.0, device="cuda")
    tik.tik_token_logprob_bwd(*first, need_hidden=False, d_lm_head=d_w)
    a = expected(*first)[1]
    near(d_w, a, out_u=U32)
    one = d_w.clone()
    tik.tik_token_logprob_bwd(*second, need_hidden=False, d_lm_head=d_w, accumulate=True)
    alone = torch.empty_like(d_w)
    tik.tik_token_logprob_bwd(*second, need_hidden=False, d_lm_head=alone)
    assert torch.equal(d_w, one + alone)                 # one fp32 addition an element


@pytest.mark.parametrize("T", [256, 300])
def test_masked_tokens_and_bad_targets(T):
    d, x, W, ids, lse, f = make(T, 128, 500, seed=4)
    clean = tik.tik_token_logprob_bwd(d, x, W, ids, lse, f)
    assert tik.device_status() == 0
    lse2 = torch.where(d == 0, float("nan"), lse)        # what masked tokens hold goes nowhere
    lse2[(d == 0).nonzero()[0]] = -float("inf")
    got = tik.tik_token_logprob_bwd(d, x, W, ids, lse2, f)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    assert bool((got[0][d == 0] == 0).all())
    bad = ids.clone()
    bad[d == 0] = -100                                   # nobody looks at a masked token's target
    bad[5], bad[77], bad[T - 1] = -1, 500, 2 ** 31 - 1
    d2 = d.clone()
    d2[5] = d2[77] = d2[T - 1] = 1.0
    got = tik.tik_token_logprob_bwd(d2, x, W, bad, lse, f)
    assert tik.device_status() == tik.DEV_BAD_TARGET and tik.device_status() == 0
    want = torch.where((bad < 0) | (bad >= 500), 0.0, d2)
    ref = tik.tik_token_logprob_bwd(want, x, W, ids, lse, f)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    zero = tik.tik_token_logprob_bwd(torch.zeros_like(d), x, W, ids, lse, f)
    assert not zero[0].any() and not zero[1].any()


@pytest.mark.parametrize("T", [1, 31, 33, 95, 161, 225, 289, 353, 600, 1100])
def test_what_an_earlier_call_left(T):
    """Scratch and accumulators full of NaN: token tiles of every width, what lies behind their last columns is not used."""
    d, x, W, ids, lse, f = make(1024, 128, 19000, seed=31)
    old = tik.tik_token_logprob_bwd(torch.full_like(d, float("nan")), torch.full_like(x, float("nan")), W, ids, lse, f)
    assert bool(old[0].isnan().all()) and bool(old[1].isnan().any())
    args = make(T, 128, 700, seed=T)
    ws = torch.full((tik.workspace_bytes(tik.OP_TOKEN_LOGPROB_BWD, T, H=128, V=700),), 255, dtype=torch.uint8, device="cuda")
    dh, dw = tik.tik_token_logprob_bwd(*args, ws=ws)
    a, b = expected(*args)
    near(dh, a)
    near(dw, b)


def test_no_rows():
    W = torch.randn(40, 64, device="cuda").bfloat16()
    e = torch.empty(0, device="cuda")
    dh, dw = tik.tik_token_logprob_bwd(e, torch.empty(0, 64, device="cuda", dtype=torch.bfloat16), W, e.int(), e)
    assert dh.shape == (0, 64) and dw.shape == (40, 64) and not dw.any()
    keep = torch.full((40, 64), 3.0, device="cuda")
    tik.tik_token_logprob_bwd(e, torch.empty(0, 64, device="cuda", dtype=torch.bfloat16), W, e.int(), e, need_hidden=False,
                              d_lm_head=keep, accumulate=True)
    assert bool((keep == 3.0).all())


def test_differences_of_the_forward():
    """The gradient along its own signs against the forward operator on both sides (its logits are exact to ~2^-22 sqrt(H))."""
    T, H, V = 64, 128, 700
    d, x, W, ids, lse, f = make(T, H, V, seed=11, masked=0.0)
    dh, _ = tik.tik_token_logprob_bwd(d, x, W, ids, lse, f)
    step = 2.0 ** -5 * torch.sign(dh.float())
    up, down = (x.float() + step).bfloat16(), (x.float() - step).bfloat16()
    lp = [tik.tik_token_logprob(v, W, ids, f).double() for v in (up, down)]
    want = (d.double() * (lp[0] - lp[1])).sum()
    along = (dh.double() * (up.double() - down.double())).sum()
    # third derivatives of a log-probability along u: at most (range of u . w)^3, u . w ~ step; the rest is rounding
    reach = ((up.double() - down.double()) / 2 @ W.double().T).abs().amax(1)
    bound = (d.double().abs() * reach ** 3).sum() / 3 + 2 * U16 * (dh.double() * (up.double() - down.double())).norm() * 3 + 1e-4 * d.double().abs().sum()
    assert abs(want - along) <= bound
    assert abs(want) > 3 * bound                         # the direction says something


def test_captured_and_on_another_stream():
    d, x, W, ids, lse, f = make(260, 192, 999, seed=8)
    want = tik.tik_token_logprob_bwd(d, x, W, ids, lse, f)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = tik.tik_token_logprob_bwd(d, x, W, ids, lse, f)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = tik.tik_token_logprob_bwd(d, x, W, ids, lse, f)
    other = make(260, 192, 999, seed=18)
    for a, b in zip((d, x, W, ids, lse), other):
        a.copy_(b)
    for _ in range(3):
        g.replay()
    again = tik.tik_token_logprob_bwd(*other)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def test_the_same_bits_on_every_call():
    args = make(2600, 1792, 3001, seed=12)
    first = tik.tik_token_logprob_bwd(*args)
    for _ in range(4):
        again = tik.tik_token_logprob_bwd(*args)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
