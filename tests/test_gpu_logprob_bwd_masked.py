"""Masked tokens of tik_token_logprob_bwd may hold anything, their hidden rows included, in calls of one row tile as in longer ones."""
import math

import pytest
import torch

from paper_2609_35140_b200 import binding as tik
from test_gpu_logprob_bwd import expected, make, near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,H,V", [(2, 64, 40), (5, 320, 1000), (64, 1088, 300), (200, 192, 5003), (255, 8192, 257), (256, 256, 2048), (257, 192, 500), (700, 320, 999)])
@pytest.mark.parametrize("need", ["both", "table", "hidden"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_masked_tokens_are_not_looked_at(T, H, V, need, dtype):
    d, x, W, ids, lse, f = make(T, H, V, seed=T, masked=0.4)
    d[0], d[T - 1] = 0.0, 1.0
    bad = (T - 2) // 2 if T > 4 else 0                     # one with a gradient and a target outside the vocabulary
    d[bad] = 0.0
    kw = dict(need_hidden=need != "table", need_lm_head=need != "hidden")

    def table():
        return torch.full((V, H), 7.0, dtype=dtype, device="cuda") if need != "hidden" else None

    clean = tik.tik_token_logprob_bwd(d, x, W, ids, lse, f, **kw, d_lm_head=table())
    a, b = expected(d, x, W, ids, lse, f)
    if need != "table":
        near(clean[0], a)
    if need != "hidden":
        near(clean[1], b)
    dead = d == 0
    for value in (math.nan, math.inf, -math.inf):
        y, l2, t2, d2 = x.clone(), lse.clone(), ids.clone(), d.clone()
        y[dead], l2[dead], t2[dead] = value, value, -7
        y[dead, ::3] = 0.0
        if bad:
            d2[bad] = 1.5
        got = tik.tik_token_logprob_bwd(d2, y, W, t2, l2, f, **kw, d_lm_head=table())
        for p, q in zip(got, clean):
            assert (p is None) == (q is None) and (p is None or torch.equal(p, q))
        assert tik.device_status() == (tik.DEV_BAD_TARGET if bad else 0)


@pytest.mark.parametrize("T", [100, 256])
def test_accumulated_and_replayed(T):
    """A graph's second replay finds what the first one left in d_hidden and scratch."""
    d, x, W, ids, lse, f = make(T, 192, 999, seed=41)
    x[d == 0] = math.nan
    d_w, d_x = torch.zeros(999, 192, device="cuda"), torch.full((T, 192), math.nan, device="cuda", dtype=torch.bfloat16)
    one, _ = tik.tik_token_logprob_bwd(d, x, W, ids, lse, f, d_lm_head=(alone := torch.empty_like(d_w)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tik.tik_token_logprob_bwd(d, x, W, ids, lse, f, d_hidden=d_x, d_lm_head=d_w, accumulate=True)
    for i in (1, 2):
        g.replay()
        assert torch.equal(d_x, one)
        assert torch.equal(d_w, i * alone)                 # (doubling is exact)
    assert bool(d_w.isfinite().all())


def test_vocabulary_in_chunks_of_a_short_call():
    """More than 2 GiB of d_z for one row tile: d_lm_head's second chunk still reads the copied rows."""
    T, H, V = 250, 64, 4_200_000
    g = torch.Generator(device="cuda").manual_seed(42)
    W = (torch.randn(V, H, generator=g, device="cuda") * H ** -0.5).bfloat16()
    at = torch.cat([torch.arange(64, device="cuda"), torch.arange(V - 64, V, device="cuda")])
    ids = at[torch.randint(0, 128, (T,), generator=g, device="cuda")].int()
    x = torch.randn(T, H, generator=g, device="cuda").bfloat16()
    d = torch.randn(T, generator=g, device="cuda") * (torch.rand(T, generator=g, device="cuda") > 0.3)
    lse = torch.logsumexp(x.float() @ W.float().T, 1)
    dead = d == 0
    y = torch.where(dead[:, None], math.nan, x)
    clean = tik.tik_token_logprob_bwd(d, x, W, ids, lse)
    got = tik.tik_token_logprob_bwd(d, y, W, ids, lse)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    short = torch.where(ids < 64, ids, ids - (V - 128))    # the same words' rows alone
    near(got[1][at], expected(d, x, W[at], short, lse, 1.0)[1])


@pytest.mark.parametrize("T,H,V", [(256, 65_536, 40), (256, 18_944, 64), (255, 19_200, 65), (250, 40_000, 1), (1, 65_600, 40), (256, 256, 1)])
@pytest.mark.parametrize("hidden", [False, True])
def test_wide_rows_stay_inside_the_workspace(T, H, V, hidden):
    """The rows' copy is wider than the parts of so small a vocabulary's sums; what lies behind the workspace stays."""
    args = make(T, H, V, seed=43, masked=0.3)
    args[0][0] = 1.0
    need = tik.workspace_bytes(tik.OP_TOKEN_LOGPROB_BWD, T, H=H, V=V)
    buf = torch.full((need + (64 << 20),), 171, dtype=torch.uint8, device="cuda")
    dh, dw = tik.tik_token_logprob_bwd(*args, need_hidden=hidden, ws=buf[:need])
    assert bool((buf[need:] == 171).all())
    a, b = expected(*args)
    near(dw, b)
    if hidden:
        near(dh, a)
