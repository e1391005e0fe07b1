"""The operators of a policy update in the order in which a trainer runs them -- embedding, norm, projections, attention, the step
between two blocks, and back, down to clipped gradients -- against torch's autograd in fp64, eagerly, out of a CUDA graph and
on two streams at once."""
import threading

import numpy as np
import pytest
import torch

from gpu_common import count_diff

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
EPS, EMB_SCALE, BRANCH = 1e-6, 4.0, 0.5
V, HQ, HKV, D = 300, 4, 2, 64
H = HQ * D


@pytest.fixture(scope="module")
def tik():
    from paper_2609_35140_b200 import binding
    binding.load()
    yield binding
    assert binding.device_status() == 0


def _randn(shape, g, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(BF)


def _problem(lens, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = sum(lens)
    p = {"table": _randn((V, H), g, 0.25), "w1": _randn((H,), g, 0.2, 1.0), "w2": _randn((H,), g, 0.2, 1.0), "post": _randn((H,), g, 0.2, 1.0),
         "gate": _randn((T, 1), g, 0.3, 0.7), "wq": _randn((H, H), g, 0.06), "wk": _randn((HKV * D, H), g, 0.06),
         "wv": _randn((HKV * D, H), g, 0.06), "wo": _randn((H, H), g, 0.06)}
    data = {"ids": torch.randint(0, V, (T,), generator=g, device="cuda").to(torch.int32), "dy": _randn((T, H), g), "ds": _randn((T, H), g),
            "cu": torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda"), "max": max(lens)}
    return p, data


def _step(tik, p, b, limit):
    """Gradients of sum(y dy) + sum(s ds) with respect to every parameter outside the projections, clipped, and their norm."""
    T, scale = b["ids"].shape[0], 1.0 / D ** 0.5
    h = tik.tik_embedding(b["ids"], p["table"], EMB_SCALE)
    y0 = tik.tik_rmsnorm(h, p["w1"], EPS)
    q, k, v = (tik.tik_linear(y0, p[n]).view(T, -1, D) for n in ("wq", "wk", "wv"))
    lse = torch.empty(T, HQ, device="cuda")
    o = tik.tik_attn_train_fwd(q, k, v, b["cu"], b["max"], scale, lse=lse)
    x = tik.tik_linear(o.view(T, H), p["wo"])
    y, s = tik.tik_block_norm(x, h, p["w2"], EPS, post_weight=p["post"], gate=p["gate"], branch_scale=BRANCH)
    d_x, d_h, d_w2, d_post, d_gate = tik.tik_block_norm_bwd(b["dy"], b["ds"], x, s, p["w2"], EPS, post_weight=p["post"], gate=p["gate"],
                                                            branch_scale=BRANCH)
    back = lambda d, w: tik.tik_linear(d.view(T, -1), p[w].t().contiguous())
    dq, dk, dv = tik.tik_attn_train_bwd(q, k, v, o, back(d_x, "wo").view(T, HQ, D), lse, b["cu"], b["max"], scale)
    d_y0 = back(dq, "wq") + back(dk, "wk") + back(dv, "wv")
    _, d_h, d_w1, _, _ = tik.tik_block_norm_bwd(d_y0, d_h, None, h, p["w1"], EPS)
    grads = [tik.tik_embedding_bwd(d_h, b["ids"], V, EMB_SCALE), d_w1, d_w2, d_post, d_gate]
    norm = tik.tik_grad_clip(grads, limit)
    return {"y": y, "s": s, "norm": norm, "table": grads[0], "w1": grads[1], "w2": grads[2], "post": grads[3], "gate": grads[4]}


def _reference(p, b, lens):
    P = {k: v.double().requires_grad_(True) for k, v in p.items()}
    rms = lambda a, w: a * torch.rsqrt(a.square().mean(-1, keepdim=True) + EPS) * w
    h = P["table"][b["ids"].long()] * EMB_SCALE
    y0 = rms(h, P["w1"])
    o, at = [], 0
    for n in lens:
        z = y0[at:at + n]
        q = (z @ P["wq"].t()).view(n, HQ, D).transpose(0, 1)
        k, v = ((z @ P[w].t()).view(n, HKV, D).transpose(0, 1).repeat_interleave(HQ // HKV, 0) for w in ("wk", "wv"))
        score = q @ k.transpose(1, 2) / D ** 0.5
        score = score.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -torch.inf)
        o.append((score.softmax(-1) @ v).transpose(0, 1).reshape(n, H))
        at += n
    x = torch.cat(o) @ P["wo"].t()
    s = h + BRANCH * P["gate"] * rms(x, P["post"])
    y = rms(s, P["w2"])
    ((y * b["dy"].double()).sum() + (s * b["ds"].double()).sum()).backward()
    got = {k: P[k].grad for k in ("table", "w1", "w2", "post", "gate")}
    got["norm"] = torch.stack([g.square().sum() for g in got.values()]).sum().sqrt().reshape(1)
    got.update(y=y.detach(), s=s.detach())
    return got


# The longest way from a parameter to a gradient passes twelve roundings to bf16 of at most 2^-8 of the value each (embedding, norm,
# projection, weights of the softmax, attention output, projection, stream, norm, and as many of theirs on the way back are
# summed over many rows, where they average out): their sum bounds the relative error of a whole tensor.
TOL = 12 * 2.0 ** -8


@pytest.mark.parametrize("lens,clip", [([1], False), ([130, 1, 77], True), ([513, 300], True), ([2000, 1500, 700], False)])
def test_gradients_of_a_step(tik, lens, clip):
    p, b = _problem(lens, sum(lens))
    ref = _reference(p, b, lens)
    limit = float(ref["norm"]) * (0.1 if clip else 10.0)
    got = _step(tik, p, b, limit)
    for k, want in ref.items():
        if clip and k in ("table", "w1", "w2", "post", "gate"):
            want = want * 0.1
        err = float((got[k].double() - want).norm() / want.norm())
        assert err <= TOL, (k, err)
    if clip:
        total = torch.stack([got[k].double().square().sum() for k in ("table", "w1", "w2", "post", "gate")]).sum().sqrt()
        assert abs(float(total) / limit - 1) <= 2.0 ** -8


def test_a_step_out_of_a_graph(tik):
    lens = [400, 333]
    p, b = _problem(lens, 5)
    _step(tik, p, b, 1.0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = _step(tik, p, b, 1.0)
    for seed in (6, 7):
        p2, b2 = _problem(lens, seed)
        for k in p:
            p[k].copy_(p2[k])
        for k in ("ids", "dy", "ds"):
            b[k].copy_(b2[k])
        g.replay()
        for k, want in _step(tik, p2, b2, 1.0).items():
            assert count_diff(out[k], want) == 0, k


def test_steps_of_threads_on_streams_of_their_own(tik):
    problems = [_problem([200 + 50 * i, 90], 20 + i) for i in range(3)]
    want = [_step(tik, p, b, 1.0) for p, b in problems]
    torch.cuda.synchronize()
    got = [None] * len(problems)

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(10):
                got[i] = _step(tik, *problems[i], 1.0)
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(problems))]
    [t.start() for t in threads]
    [t.join() for t in threads]
    for a, w in zip(got, want):
        for k in w:
            assert count_diff(a[k], w[k]) == 0, k


def test_calls_through_buffers_that_are_written_again(tik):
    """Chains without a synchronisation, each call's inputs written by the one before it: whatever runs under its predecessor's tail
    sees what a synchronised chain sees."""
    g = torch.Generator(device="cuda").manual_seed(9)
    W, K = 20_000, 1024
    tables = [_randn((W, K), g) for _ in range(2)]
    sizes = [200, 3000, 6000, 20_000, 257, 66_000, 4608]
    ids = [torch.randint(0, W, (n,), generator=g, device="cuda").to(torch.int32) for n in sizes]
    w = _randn((K,), g, 0.1, 1.0)

    def chain(sync):
        a, b = (t.clone() for t in tables)
        seen = []
        for i, n in enumerate(sizes * 2):
            step = (lambda: torch.cuda.synchronize()) if sync else (lambda: None)
            idx = ids[i % len(sizes)]
            if i % 3 == 1:
                idx = torch.roll(idx, i)                       # written just before the call that reads it
            y = tik.tik_embedding(idx, a, 0.5); step()
            y, s = tik.tik_block_norm(y, y, w, EPS, post_weight=w); step()
            dx, dr, dw, dp, _ = tik.tik_block_norm_bwd(y, s, y, s, w, EPS, post_weight=w); step()
            tik.tik_embedding_bwd(dx, idx, W, 1.0, d_table=b, accumulate=i % 4 == 3); step()
            seen.append(tik.tik_grad_clip([b, dw, dp], 100.0 + i)); step()
            tik.tik_embedding_bwd(dr, idx, W, 1.0, d_table=b, accumulate=True); step()
            a, b = b, a                                        # the next lookup reads what was just added up
        torch.cuda.synchronize()
        return seen + [a, b]

    for x, y in zip(chain(False), chain(True)):
        assert count_diff(x, y) == 0


def test_launch_counts(tik):
    """Kernels per call: the ones that the header states."""
    def launches(f):
        n = tik.kernel_launches()
        f()
        return tik.kernel_launches() - n
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, V, (5000,), generator=g, device="cuda").to(torch.int32)
    table, dy = _randn((V, H), g), _randn((5000, H), g)
    assert launches(lambda: tik.tik_embedding(ids, table)) == 1
    assert launches(lambda: tik.tik_embedding_bwd(dy, ids, V)) == 3
    many, long_ids = _randn((65_537, H), g), torch.randint(0, V, (65_537,), generator=g, device="cuda").to(torch.int32)
    assert launches(lambda: tik.tik_embedding_bwd(many, long_ids, V)) == 5            # one digit of nine bits
    assert launches(lambda: tik.tik_embedding_bwd(dy[:200].contiguous(), ids[:200].contiguous(), V)) == 1
    w = _randn((H,), g)
    assert launches(lambda: tik.tik_block_norm(dy, dy, w, EPS, post_weight=w, gate=w)) == 1
    assert launches(lambda: tik.tik_block_norm_bwd(dy, dy, dy, dy, w, EPS)) == 2
    assert launches(lambda: tik.tik_grad_norm([table, dy])) == 2 and launches(lambda: tik.tik_grad_clip([table, dy], 1e9)) == 2
    assert launches(lambda: tik.tik_grad_clip([table, dy], 1e9, norm=torch.ones(1, device="cuda"))) == 1
