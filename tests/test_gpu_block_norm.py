"""GPU parity of the step between two blocks and its gradient against the fp64 oracle, and the bits that it shares with
tik_rmsnorm and between batched and row-by-row use."""
import numpy as np
import pytest
import torch

import oracle
from gpu_common import count_diff

pytestmark = pytest.mark.gpu
U32, UBF = 2.0 ** -24, 2.0 ** -8                     # half a step, relative


@pytest.fixture(scope="module")
def tik():
    from paper_2609_35140_b200 import binding
    binding.load()
    yield binding
    assert binding.device_status() == 0


def _randn(shape, seed, std=1.0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(torch.bfloat16)


def _np(t):
    return None if t is None else t.double().cpu().numpy()


FORMS = [dict(post=True, gate="channel", nxt=True, a=1.0), dict(post=True, gate="token", nxt=True, a=0.22),
         dict(post=False, gate="token", nxt=True, a=-0.5), dict(post=False, gate="channel", nxt=False, a=1.0),
         dict(post=True, gate=None, nxt=True, a=1.0), dict(post=True, gate=None, nxt=False, a=0.0), dict(post=False, gate=None, nxt=True, a=1.0)]
SIZES = [(1, 8), (3, 64), (37, 256), (5, 1000), (2, 1032), (64, 1536), (7, 2056), (19, 3584), (6, 4096), (4, 4104), (9, 5120), (3, 8192)]


def _inputs(T, H, post, gate, nxt, a, seed=0):
    t = {"x": _randn((T, H), seed + 1, 2.0), "residual": _randn((T, H), seed + 2, 4.0), "post": None, "gate": None, "weight": None}
    if post:
        t["post"] = _randn((H,), seed + 3, 0.2, 1.0)
    if gate:
        t["gate"] = _randn((H,) if gate == "channel" else (T, 1), seed + 4, 0.4, 0.3)
    if nxt:
        t["weight"] = _randn((H,), seed + 5, 0.2, 1.0)
    return t


def _forward(tik, t, a, rows=slice(None), **out):
    gate = t["gate"]
    if gate is not None and gate.dim() == 2:
        gate = gate[rows].contiguous()
    return tik.tik_block_norm(t["x"][rows].contiguous(), t["residual"][rows].contiguous(), t["weight"], 1e-6, post_weight=t["post"],
                              gate=gate, branch_scale=a, **out)


@pytest.mark.parametrize("T,H", SIZES + [(512, 264), (513, 264), (2100, 72), (2, 256), (5, 512), (701, 256), (703, 512), (515, 520), (2051, 8), (600, 1032), (530, 3584), (521, 5120)])
@pytest.mark.parametrize("form", FORMS)
def test_forward(tik, T, H, form):
    a = form["a"]
    t = _inputs(T, H, **form)
    buf_s, buf_y = (torch.full((T + 2, H), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    y, s = _forward(tik, t, a, s=buf_s[1:T + 1], **({"y": buf_y[1:T + 1]} if form["nxt"] else {}))
    for buf in (buf_s, buf_y):
        assert bool((buf[0] == 7.0).all()) and bool((buf[T + 1] == 7.0).all())
    a32 = float(np.float32(a))
    ref, u = oracle.block_norm(_np(t["x"]), _np(t["residual"]), float(np.float32(1e-6)), _np(t["post"]), _np(t["gate"]), a32)
    # the branch: at most 64 additions per thread and 8 more of the sum of squares, halved by the root, root, three to five
    # products: under 48 half steps of fp32; the sum: one more of the whole; then one rounding to bf16
    e = 48 * U32 * np.abs(u) + U32 * np.abs(ref)
    assert np.all(np.abs(_np(s) - ref) <= UBF * (np.abs(ref) + e) + e)
    if not form["nxt"]:
        assert y is None
    else:
        want = oracle.rmsnorm(s.float().cpu().numpy(), t["weight"].float().cpu().numpy(), float(np.float32(1e-6)))
        assert np.all(np.abs(_np(y) - want) <= (UBF + 48 * U32) * np.abs(want))
        assert count_diff(y, tik.tik_rmsnorm(s, t["weight"], 1e-6)) == 0           # the norm of the stored sum
    if not form["post"] and not form["gate"] and a == 1.0:
        res = t["residual"].clone()
        assert count_diff(tik.tik_rmsnorm(t["x"], t["weight"], 1e-6, residual=res), y) == 0 and count_diff(res, s) == 0
    # a row alone, and in place
    r = slice(T // 2, T // 2 + 1)
    y1, s1 = _forward(tik, t, a, r)
    assert count_diff(s1, s[r]) == 0 and (y is None or count_diff(y1, y[r]) == 0)
    t2 = {k: None if v is None else v.clone() for k, v in t.items()}
    y2, s2 = tik.tik_block_norm(t2["x"], t2["residual"], t2["weight"], 1e-6, post_weight=t2["post"], gate=t2["gate"], branch_scale=a,
                                s=t2["residual"], y=t2["x"] if form["nxt"] else None)
    assert count_diff(t2["residual"], s) == 0 and (y is None or count_diff(t2["x"], y) == 0)


NAMES = ("d_x", "d_residual", "d_weight", "d_post_weight", "d_gate")


def _check_backward(tik, t, s, dy, ds, a, T, H, **more):
    got = tik.tik_block_norm_bwd(dy, ds, t["x"], s, t["weight"], 1e-6, post_weight=t["post"], gate=t["gate"], branch_scale=a, **more)
    ref, mag = oracle.block_norm_bwd(_np(dy), _np(ds), _np(t["x"]), _np(s), _np(t["weight"]), float(np.float32(1e-6)), _np(t["post"]),
                                     _np(t["gate"]), float(np.float32(a)))
    assert [n for n, g in zip(NAMES, got) if g is not None] == [n for n in NAMES if n in ref]
    for name, g in zip(NAMES, got):
        if g is None:
            continue
        # Every value is a sum of products of row sums (16 to 64 additions per thread, at most 20 across a CTA, each off
        # by half a step of the sum of magnitudes), roots and at most twelve single roundings: under 128 half steps of fp32 of
        # the sum of magnitudes; d_x passes through two such sums.  Sums over tokens add one per token, and at most 300
        # more where CTAs' sums are added up.  bf16 outputs are rounded once more.
        steps = 128 if name == "d_residual" else 256
        if name in ("d_weight", "d_post_weight") or (name == "d_gate" and g.dim() == 1):
            steps += T + 300
        e = steps * U32 * mag[name]
        half = UBF if g.dtype == torch.bfloat16 else U32
        err = np.abs(_np(g) - ref[name])
        assert np.all(err <= half * (np.abs(ref[name]) + e) + e), (name, float(err.max()))
        assert g.dtype == (torch.bfloat16 if name in ("d_x", "d_residual") else torch.float32)
    return got


@pytest.mark.parametrize("T,H", SIZES + [(300, 256), (297, 72), (1500, 264), (613, 3584), (911, 5120)])
@pytest.mark.parametrize("form", FORMS)
def test_backward(tik, T, H, form):
    a = form["a"]
    t = _inputs(T, H, **form, seed=20)
    s, dy, ds = _randn((T, H), 31, 4.0), _randn((T, H), 32) if form["nxt"] else None, _randn((T, H), 33)
    got = _check_backward(tik, t, s, dy, ds, a, T, H)
    again = tik.tik_block_norm_bwd(dy, ds, t["x"], s, t["weight"], 1e-6, post_weight=t["post"], gate=t["gate"], branch_scale=a)
    for g, h in zip(got, again):
        assert g is None or count_diff(g, h) == 0
    if form["nxt"]:
        _check_backward(tik, t, s, dy, None, a, T, H)                              # nothing reaches the stream from further on
    # rows do not depend on the batch
    r = slice(T // 2, T // 2 + 1)
    gate = t["gate"][r].contiguous() if form["gate"] == "token" else t["gate"]
    one = tik.tik_block_norm_bwd(None if dy is None else dy[r].contiguous(), ds[r].contiguous(), t["x"][r].contiguous(), s[r].contiguous(),
                                 t["weight"], 1e-6, post_weight=t["post"], gate=gate, branch_scale=a)
    assert count_diff(one[0], got[0][r]) == 0 and count_diff(one[1], got[1][r]) == 0
    if form["gate"] == "token":
        assert count_diff(one[4], got[4][r]) == 0


@pytest.mark.parametrize("T,H", [(1, 8), (300, 256), (41, 3584), (12, 8192)])
@pytest.mark.parametrize("with_ds", [False, True])
def test_backward_of_the_plain_norm(tik, T, H, with_ds):
    t = {"x": None, "post": None, "gate": None, "weight": _randn((H,), 5, 0.2, 1.0)}
    _check_backward(tik, t, _randn((T, H), 1), _randn((T, H), 2), _randn((T, H), 3) if with_ds else None, 1.0, T, H)


def test_backward_of_no_tokens(tik):
    H = 136
    none = torch.empty(0, H, dtype=torch.bfloat16, device="cuda")
    w, p, g = (_randn((H,), i, 0.2, 1.0) for i in (1, 2, 3))
    dx, dr, dw, dp, dg = tik.tik_block_norm_bwd(none, none, none, none, w, 1e-6, post_weight=p, gate=g)
    assert dx.shape == dr.shape == (0, H) and all(bool((v == 0).all()) and v.shape == (H,) for v in (dw, dp, dg))
    dx, dr, dw, dp, dg = tik.tik_block_norm_bwd(none, none, none, none, w, 1e-6, gate=torch.empty(0, 1, dtype=torch.bfloat16, device="cuda"))
    assert dp is None and dg.shape == (0, 1) and bool((dw == 0).all())
    y, s = tik.tik_block_norm(none, none, w, 1e-6, post_weight=p)
    assert y.shape == s.shape == (0, H)


def test_gradient_against_differences(tik):
    """The loss sum(s o ds) + sum(y o dy) of the forward kernel, moved along random directions.  Its outputs are bf16, so a
    step has to be large against their rounding: along x and the weights by 2^-3, where the second-order part cancels
    between the two signs.  What is left: rounding errors of 2 T H outputs, independent and uniform within half a step
    (their sum has the standard deviation below; 6 of those), and a third-order part, under 2 % of the sum of magnitudes."""
    T, H, a, h = 24, 256, 0.7, 2.0 ** -3
    form = dict(post=True, gate="channel", nxt=True)
    t = _inputs(T, H, a=a, seed=50, **form)
    dy, ds = _randn((T, H), 61), _randn((T, H), 62)

    def loss(t):
        y, s = _forward(tik, t, a)
        noise = (dy.double() * y.double()).square().sum() + (ds.double() * s.double()).square().sum()
        return float((dy.double() * y.double()).sum() + (ds.double() * s.double()).sum()), float(noise)

    _, s = _forward(tik, t, a)
    got = dict(zip(NAMES, tik.tik_block_norm_bwd(dy, ds, t["x"], s, t["weight"], 1e-6, post_weight=t["post"], gate=t["gate"], branch_scale=a)))
    for name, key in (("d_x", "x"), ("d_residual", "residual"), ("d_weight", "weight"), ("d_post_weight", "post"), ("d_gate", "gate")):
        base = t[key]
        # along the gradient's signs, where the change is largest; steps of a power of two around values on a coarse grid are exact
        direction = torch.sign(got[name]).double().view(base.shape)
        coarse = (base.double() * 32).round() / 32
        at = dict(t, **{key: coarse.to(torch.bfloat16)})
        _, s0 = _forward(tik, at, a)
        g = dict(zip(NAMES, tik.tik_block_norm_bwd(dy, ds, at["x"], s0, at["weight"], 1e-6, post_weight=at["post"], gate=at["gate"], branch_scale=a)))
        up, down = (coarse + sign * h * direction for sign in (1, -1))
        moved = [u.to(torch.bfloat16) for u in (up, down)]
        (lu, nu), (ld, nd) = (loss(dict(t, **{key: m})) for m in moved)
        want = float((g[name].double().view(base.shape) * (moved[0].double() - moved[1].double())).sum())
        noise = 6 * UBF / np.sqrt(3.0) * np.sqrt(nu + nd)
        assert want > 0 and abs((lu - ld) - want) <= noise + 0.02 * want, (name, lu - ld, want, noise)


def test_captured_and_replayed(tik):
    T, H, a = 200, 1536, 0.5
    t = _inputs(T, H, True, "token", True, a)
    dy, ds = _randn((T, H), 1), _randn((T, H), 2)
    ws = torch.empty(tik.workspace_bytes(tik.OP_BLOCK_NORM_BWD, T, H=H), dtype=torch.uint8, device="cuda")

    def step():
        y, s = _forward(tik, t, a)
        return (y, s) + tik.tik_block_norm_bwd(dy, ds, t["x"], s, t["weight"], 1e-6, post_weight=t["post"], gate=t["gate"], branch_scale=a, ws=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    gate = t["gate"]
    x, res = t["x"], t["residual"]
    with torch.cuda.graph(g):
        y, s = tik.tik_block_norm(x, res, t["weight"], 1e-6, post_weight=t["post"], gate=gate, branch_scale=a)
        out = (y, s) + tik.tik_block_norm_bwd(dy, ds, x, s, t["weight"], 1e-6, post_weight=t["post"], gate=gate, branch_scale=a, ws=ws)
    for seed in (7, 8):
        x.copy_(_randn((T, H), seed))
        dy.copy_(_randn((T, H), seed + 10))
        ws.fill_(255)
        g.replay()
        for got, want in zip(out, step()):
            assert count_diff(got, want) == 0


@pytest.mark.parametrize("T,H", [(300, 256), (150, 3584), (5, 8192)])
def test_gradients_over_their_inputs(tik, T, H):
    """Through the C interface: d_residual over d_s or d_y, d_x over x, s or d_y."""
    a = 0.7
    t = _inputs(T, H, True, "channel", True, a, seed=70)
    s, dy, ds = _randn((T, H), 71, 4.0), _randn((T, H), 72), _randn((T, H), 73)
    want = tik.tik_block_norm_bwd(dy, ds, t["x"], s, t["weight"], 1e-6, post_weight=t["post"], gate=t["gate"], branch_scale=a)
    ws = torch.empty(tik.workspace_bytes(tik.OP_BLOCK_NORM_BWD, T, H=H), dtype=torch.uint8, device="cuda")
    f32 = [torch.empty(H, device="cuda") for _ in range(3)]
    for over_x, over_r in (("x", "ds"), ("s", "dy"), ("dy", "ds"), ("ds", "x")):
        v = {"x": t["x"].clone(), "s": s.clone(), "dy": dy.clone(), "ds": ds.clone()}
        ptr = lambda k: v[k].data_ptr()
        rc = tik.load().tik_block_norm_bwd(tik.context(), ptr("dy"), ptr("ds"), ptr("x"), ptr("s"), t["post"].data_ptr(), t["gate"].data_ptr(), 1, a,
                                           t["weight"].data_ptr(), 1e-6, ptr(over_x), ptr(over_r), *[f.data_ptr() for f in f32], T, H,
                                           ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        for got, ref in zip([v[over_x], v[over_r]] + f32, want):
            assert count_diff(got, ref) == 0, (over_x, over_r)


def test_refused_tensors(tik):
    x, r, w, s = _randn((4, 64), 1), _randn((4, 64), 2), _randn((64,), 3), _randn((4, 64), 4)
    for bad in (lambda: tik.tik_block_norm(x.float(), r, w, 1e-6), lambda: tik.tik_block_norm(x, r.t().contiguous().t(), w, 1e-6),
                lambda: tik.tik_block_norm(x, r.cpu(), w, 1e-6), lambda: tik.tik_block_norm(x, r, w, -1.0),
                lambda: tik.tik_block_norm(x, r, w, 1e-6, branch_scale=float("nan")), lambda: tik.tik_block_norm(x[:, :60].contiguous(), r[:, :60].contiguous(), w[:60].contiguous(), 1e-6),
                lambda: tik.tik_block_norm_bwd(x, r, x, s, w, 1e-6, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(tik.TikError):
            bad()
    for bad in (lambda: tik.tik_block_norm(x, r[:3], w, 1e-6), lambda: tik.tik_block_norm(x, r, w[:32], 1e-6),
                lambda: tik.tik_block_norm(x, r, w, 1e-6, gate=w[:4]), lambda: tik.tik_block_norm(x, r, w, 1e-6, gate=x),
                lambda: tik.tik_block_norm(x, r, None, 1e-6, y=s), lambda: tik.tik_block_norm_bwd(None, r, x, s, w, 1e-6),
                lambda: tik.tik_block_norm_bwd(None, None, x, s, None, 1e-6), lambda: tik.tik_block_norm_bwd(x, r, None, s, w, 1e-6, post_weight=w),
                lambda: tik.tik_block_norm_bwd(x[:3], r, x, s, w, 1e-6)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("std_x,std_s,eps,zero_rows", [(1.0, 1e-14, 0.0, False), (1e-14, 1.0, 0.0, False), (1.0, 1.0, 1e-28, True), (1e-12, 1e-12, 1e-30, True)])
def test_backward_of_tiny_rows(tik, std_x, std_s, eps, zero_rows):
    """Rows so small that the cube of their norm's factor is beyond fp32, and rows of zeros beside them."""
    T, H = 9, 264
    t = _inputs(T, H, True, "channel", True, 1.0)
    x, s, dy, ds = _randn((T, H), 21, std_x), _randn((T, H), 22, std_s), _randn((T, H), 23), _randn((T, H), 24)
    if zero_rows:
        for z in (x, s):
            z[2] = 0
            z[7] = 0
    got = tik.tik_block_norm_bwd(dy, ds, x, s, t["weight"], eps, post_weight=t["post"], gate=t["gate"])
    ref, mag = oracle.block_norm_bwd(_np(dy), _np(ds), _np(x), _np(s), _np(t["weight"]), float(np.float32(eps)), _np(t["post"]), _np(t["gate"]), 1.0)
    for name, g in zip(NAMES, got):
        # steps as in _check_backward
        steps = 256 + (T + 300 if g.dtype == torch.float32 else 0)
        e = steps * U32 * mag[name]
        half = UBF if g.dtype == torch.bfloat16 else U32
        assert np.all(np.isfinite(ref[name]) == np.isfinite(_np(g)))
        assert np.all(np.abs(_np(g) - ref[name]) <= half * (np.abs(ref[name]) + e) + e), name


@pytest.mark.parametrize("T,H", [(3, 8), (64, 264), (300, 3584)])
def test_results_have_memory_of_their_own(tik, T, H):
    """Small calls make their results in one allocation: the parts are aligned, apart from each other, and usable one by one."""
    t = _inputs(T, H, True, "channel", True, 1.0)
    y, s = _forward(tik, t, 1.0)
    got = tik.tik_block_norm_bwd(y, s, t["x"], s, t["weight"], 1e-6, post_weight=t["post"], gate=t["gate"])
    for group in ((y, s), got):
        spans = sorted((r.data_ptr(), r.data_ptr() + r.numel() * r.element_size()) for r in group)
        assert all(a % 16 == 0 for a, _ in spans) and all(e <= b for (_, e), (b, _) in zip(spans, spans[1:]))
        assert all(r.is_contiguous() for r in group)
    keep = [r.clone() for r in got]
    for i in range(5):
        got[i].add_(1)
        for j in range(i + 1, 5):
            assert count_diff(got[j], keep[j]) == 0
    d_w = got[2]
    want = d_w.clone()
    del got, y, s
    torch.empty(1 << 20, dtype=torch.uint8, device="cuda").fill_(255)
    assert count_diff(d_w, want) == 0
    ds = tik.tik_block_norm_bwd(None, t["x"], None, t["residual"], None, 1e-6)[1]              # one result alone
    assert count_diff(ds, t["x"]) == 0
    empty = tik.tik_block_norm(t["x"][:0], t["residual"][:0], t["weight"], 1e-6)
    assert [tuple(r.shape) for r in empty] == [(0, H), (0, H)]


@pytest.mark.parametrize("T,H", [(9001, 264), (4500, 1032), (3001, 1536), (2401, 2560), (2100, 3584), (1700, 4096), (1501, 5120), (901, 6144), (701, 8192)])
@pytest.mark.parametrize("form", [FORMS[0], FORMS[1], FORMS[6]])
def test_backward_of_many_rows(tik, T, H, form):
    """Rows enough for every slot of the ring to be used again, by other groups than before."""
    t = _inputs(T, H, **form, seed=50)
    s, dy, ds = _randn((T, H), 51, 4.0), _randn((T, H), 52), _randn((T, H), 53)
    _check_backward(tik, t, s, dy, ds, form["a"], T, H)


@pytest.mark.parametrize("H", [72, 264, 3584, 4104])
@pytest.mark.parametrize("std_x,std_s,eps,zeros", [(1.0, 1e-20, 0.0, ""), (1e-20, 1.0, 0.0, ""), (1e-20, 1e-15, 0.0, ""), (1e-15, 1e-20, 0.0, ""),
                                                   (1.0, 1e-21, 0.0, ""), (1e-21, 1.0, 0.0, ""), (1.0, 1e-20, 1e-40, "s"), (1e-20, 1.0, 1e-40, "x")])
@pytest.mark.parametrize("plain", [False, True])
def test_backward_of_rows_whose_mean_square_is_subnormal(tik, std_x, std_s, eps, zeros, H, plain):
    """The forward's factor of such rows is finite, and so are the gradients.  What their mean squares lose: every addition is off by
    2^-150 at most, half a step of fp32's subnormal numbers, so the mean (H additions of squares and under 40 of parts, over
    H; one rounding more) by (2 + 40 / H) 2^-150.  The root halves that relative error, and a gradient's terms hold the root three
    times at most: 1.8 times the mean's relative error of the sum of magnitudes, with a fifth to spare for second order."""
    T = 9
    t = _inputs(T, H, True, "channel", True, 1.0)
    x, s, dy, ds = _randn((T, H), 21, std_x), _randn((T, H), 22, std_s), _randn((T, H), 23), _randn((T, H), 24)
    for z in zeros:
        {"x": x, "s": s}[z][2:5:2] = 0
    eps32 = float(np.float32(eps))
    lost = lambda v: (2 + 40 / H) * 2.0 ** -150 / ((_np(v) ** 2).mean(axis=1).min() + eps32)
    post, gate = (None, None) if plain else (t["post"], t["gate"])
    if plain:
        x = None
    got = tik.tik_block_norm_bwd(dy, ds, x, s, t["weight"], eps, post_weight=post, gate=gate)
    ref, mag = oracle.block_norm_bwd(_np(dy), _np(ds), _np(x), _np(s), _np(t["weight"]), eps32, _np(post), _np(gate), 1.0)
    for name, g in zip(NAMES, got):
        if g is None:
            continue
        # steps as in _check_backward
        steps = 256 + (T + 300 if g.dtype == torch.float32 else 0)
        more = 1.8 * lost(s) + (1.8 * lost(x) if name not in ("d_residual", "d_weight") else 0.0)
        e = (steps * U32 + more) * mag[name]
        half = UBF if g.dtype == torch.bfloat16 else U32
        assert np.all(np.isfinite(ref[name])) and bool(torch.isfinite(g).all()), name
        assert np.all(np.abs(_np(g) - ref[name]) <= half * (np.abs(ref[name]) + e) + e), name


@pytest.mark.parametrize("T,H", [(40, 256), (40, 3584), (3, 5120)])
@pytest.mark.parametrize("gate", ["channel", "token"])
def test_without_a_post_norm_d_x_does_not_depend_on_x(tik, T, H, gate):
    """d_x = branch_scale * gate * G then: infinities and NaN in x reach the gate's gradient alone."""
    t = _inputs(T, H, False, gate, True, 1.0)
    s, dy, ds = _randn((T, H), 2, 4.0), _randn((T, H), 3), _randn((T, H), 4)
    bad = t["x"].clone()
    bad[0, 5], bad[T - 1, H - 1], bad[T // 2] = float("inf"), float("nan"), -float("inf")
    want, got = (tik.tik_block_norm_bwd(dy, ds, x, s, t["weight"], 1e-6, gate=t["gate"], branch_scale=0.5) for x in (t["x"], bad))
    for i in range(3):
        assert count_diff(got[i], want[i]) == 0, NAMES[i]
    clean = torch.ones(got[4].numel(), dtype=torch.bool, device="cuda")
    if gate == "token":
        clean[[0, T - 1, T // 2]] = False
    else:
        clean[:] = False
    assert count_diff(got[4].flatten()[clean], want[4].flatten()[clean]) == 0 and not bool(torch.isfinite(got[4].flatten()[~clean]).any())


@pytest.mark.parametrize("T,H", [(20011, 256), (30000, 72), (9473, 8)])
@pytest.mark.parametrize("form", [FORMS[0], FORMS[1], FORMS[6], None])
def test_backward_of_many_narrow_rows(tik, T, H, form):
    """Groups of one warp: 20 groups share a ring of 64 slots per CTA, which 9472 rows fill for the first time.  (None: the plain norm.)"""
    t = _inputs(T, H, **(form or FORMS[6]), seed=50)
    if form is None:
        t["x"] = None
    s, dy, ds = _randn((T, H), 51, 4.0), _randn((T, H), 52), _randn((T, H), 53)
    got = _check_backward(tik, t, s, dy, ds, form["a"] if form else 1.0, T, H)
    again = tik.tik_block_norm_bwd(dy, ds, t["x"], s, t["weight"], 1e-6, post_weight=t["post"], gate=t["gate"], branch_scale=form["a"] if form else 1.0)
    for g, h in zip(got, again):
        assert g is None or count_diff(g, h) == 0
