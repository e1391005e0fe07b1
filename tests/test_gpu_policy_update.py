"""A policy update's ends in the order in which a trainer runs them -- norm, log-probabilities, loss, and back through lm_head and the norm
to the gradient norm and the optimiser -- against torch in fp64 and the oracles, eagerly, out of a graph and on threads' own streams."""
import threading

import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-6
LOSS = dict(clip_low=0.2, clip_high=0.28, clip_dual=3.0, kl_coef=0.05, reduction="sequence")
ADAM = dict(beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def tik():
    from paper_2609_35140_b200 import binding
    binding.load()
    yield binding
    assert binding.device_status() == 0


def _problem(lens, H, V, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    T, S = sum(lens), len(lens)
    master = [rand(V, H) * H ** -0.5, 1 + 0.2 * rand(H)]
    b = {"x": rand(T, H).to(BF), "ids": torch.randint(0, V, (T,), generator=g, device="cuda").to(torch.int32),
         "adv": rand(S, 1), "cu": torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda"),
         "weight": (torch.rand(T, generator=g, device="cuda") > 0.3).float()}
    b["old"] = -8 + 0.3 * rand(T)
    b["ref"] = b["old"] + 0.2 * rand(T)
    state = {"master": master, "param": [m.to(BF) for m in master], "m": [torch.zeros_like(m) for m in master],
             "v": [torch.zeros_like(m) for m in master], "step": torch.ones(1, dtype=torch.int32, device="cuda")}
    return b, state


def _update(tik, b, st, limit, lr=1e-3):
    W, w = st["param"]
    T, H = b["x"].shape
    y = tik.tik_rmsnorm(b["x"], w, EPS)
    lse = torch.empty(T, device="cuda")
    lp = tik.tik_token_logprob(y, W, b["ids"], 1.0, lse=lse)
    loss, d_lp, stats = tik.tik_policy_loss(lp, b["old"], b["adv"], weight=b["weight"], ref_logprob=b["ref"], cu_seqlens=b["cu"],
                                            scale=1.0 / b["adv"].shape[0], **LOSS)
    d_y, d_W = tik.tik_token_logprob_bwd(d_lp, y, W, b["ids"], lse, 1.0)
    _, d_x, d_w, _, _ = tik.tik_block_norm_bwd(d_y, None, None, b["x"], w, EPS)
    norm = tik.tik_grad_norm([d_W, d_w])
    tik.tik_adamw(st["param"], [d_W, d_w], st["m"], st["v"], lr, st["step"], master=st["master"], norm=norm, max_norm=limit, **ADAM)
    st["step"] += 1
    return {"loss": loss, "stats": stats, "lp": lp, "d_lp": d_lp, "d_x": d_x, "d_W": d_W, "d_w": d_w, "norm": norm}


def _reference(b, W, w, d_lp):
    """The loss, and the gradients that d_lp comes to: a token whose ratio is within a rounding of a threshold is cut or not by the
    log-probability's last bits, so what the loss's gradient is at these log-probabilities is asked of the oracle."""
    x, W, w = (t.double().requires_grad_(True) for t in (b["x"], W, w))
    y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
    lp = torch.log_softmax(y @ W.T, 1).gather(1, b["ids"].long()[:, None])[:, 0]
    lens = (b["cu"][1:] - b["cu"][:-1]).long()
    A = b["adv"][:, 0].double().repeat_interleave(lens)
    r = torch.exp(lp - b["old"].double())
    gain = torch.minimum(r * A, r.clamp(0.8, 1.28) * A)
    gain = torch.where(A < 0, torch.maximum(gain, 3.0 * A), gain)
    k = b["ref"].double() - lp
    token = (-gain + 0.05 * (torch.exp(k) - k - 1)) * b["weight"].double()
    seq = torch.arange(len(lens), device="cuda").repeat_interleave(lens)
    n = torch.zeros(len(lens), dtype=torch.float64, device="cuda").index_add_(0, seq, b["weight"].double()).clamp(min=1)
    loss = (token / n[seq]).sum() / len(lens)
    (lp * d_lp.double()).sum().backward()
    return {"loss": loss.detach().reshape(1), "lp": lp.detach(), "d_x": x.grad, "d_W": W.grad, "d_w": w.grad}


# From the inputs to a gradient: roundings to bf16 of y, d_z, d_y or d_W, d_x (2^-8 of the value each at most); a rounding of y moves the
# logits by 2^-8 / sqrt(3) of their spread over sqrt(H) terms, and with them the probabilities and ratios that gradients go with.
TOL = 6 * 2.0 ** -8


@pytest.mark.parametrize("lens,H,V", [([1], 64, 50), ([100, 3, 60], 128, 1000), ([300, 1, 250, 77], 320, 3001)])
def test_an_update_against_autograd(tik, lens, H, V):
    b, st = _problem(lens, H, V, sum(lens))
    b["weight"][0] = 1.0
    lp = torch.log_softmax((lambda y: y @ st["param"][0].double().T)(tik.tik_rmsnorm(b["x"], st["param"][1], EPS).double()), 1)
    g = torch.Generator(device="cuda").manual_seed(1)
    b["old"] = (lp.gather(1, b["ids"].long()[:, None])[:, 0] + 0.15 * torch.randn(sum(lens), generator=g, device="cuda")).float()
    b["ref"] = b["old"] - 0.1
    weights = [t.clone() for t in st["param"]]
    before = {k: [t.clone() for t in v] for k, v in st.items() if k != "step"}
    limit = 1e9
    got = _update(tik, b, st, limit)
    ref = _reference(b, *weights, got["d_lp"])
    for k, want in ref.items():
        err = float((got[k].double() - want).norm() / want.norm())
        assert err <= TOL, (k, err)
    loss, d, stats = oracle.policy_loss(got["lp"].cpu().numpy(), b["old"].cpu().numpy(), b["adv"].cpu().numpy(), b["weight"].cpu().numpy(),
                                        b["ref"].cpu().numpy(), b["cu"].cpu().numpy(), scale=1.0 / len(lens), **LOSS)
    assert np.abs(got["d_lp"].cpu().numpy() - d).max() <= 2.0 ** -20 * np.abs(d).max()
    assert abs(float(got["loss"]) - loss) <= 2.0 ** -20 * (abs(stats[0]) + abs(stats[1]) + np.abs(b["adv"].cpu().numpy()).max())
    for i, name in enumerate(("d_W", "d_w")):
        w, m, v = oracle.adamw(before["master"][i].cpu().numpy(), got[name].float().cpu().numpy(), before["m"][i].cpu().numpy(),
                               before["v"][i].cpu().numpy(), 1e-3, 1, **ADAM)
        assert np.abs(st["master"][i].cpu().numpy() - w).max() <= 2.0 ** -22 * (np.abs(w).max() + 1e-3)
        assert torch.equal(st["param"][i], st["master"][i].to(BF))


def test_updates_out_of_a_graph(tik):
    b, st = _problem([120, 200], 128, 777, 3)
    b2, st2 = _problem([120, 200], 128, 777, 3)
    _update(tik, *_problem([120, 200], 128, 777, 4), 1.0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = _update(tik, b, st, 0.01)
    for i in range(4):
        b3, _ = _problem([120, 200], 128, 777, 50 + i)
        for k in b:
            b[k].copy_(b3[k])
            b2[k].copy_(b3[k])
        g.replay()
        want = _update(tik, b2, st2, 0.01)
        for k in want:
            assert torch.equal(out[k], want[k]), (i, k)
        for k in ("master", "param", "m", "v"):
            for x, y in zip(st[k], st2[k]):
                assert torch.equal(x, y), (i, k)


def test_updates_of_threads_on_streams_of_their_own(tik):
    shapes = [([150, 90], 128, 700), ([300], 64, 2001), ([40, 5, 260], 192, 333)]
    def run(i):
        b, st = _problem(*shapes[i], 20 + i)
        for _ in range(5):
            out = _update(tik, b, st, 0.05)
        return out, st
    want = [run(i) for i in range(3)]
    torch.cuda.synchronize()
    got = [None] * 3

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            got[i] = run(i)
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(3)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    for (o, st), (w, sw) in zip(got, want):
        for k in w:
            assert torch.equal(o[k], w[k]), k
        for k in ("master", "param", "m", "v"):
            for x, y in zip(st[k], sw[k]):
                assert torch.equal(x, y), k


def test_chains_without_a_synchronisation(tik):
    """Calls of changing sizes through buffers that are written again, on one stream: whatever runs under its predecessor's tail sees what a
    synchronised chain sees."""
    def chain(sync):
        step = torch.cuda.synchronize if sync else (lambda: None)
        g = torch.Generator(device="cuda").manual_seed(5)
        H, V = 192, 1500
        W = (torch.randn(V, H, generator=g, device="cuda") * H ** -0.5).to(BF)
        big = torch.randn(3000, H, generator=g, device="cuda").to(BF)
        ids = torch.randint(0, V, (3000,), generator=g, device="cuda").to(torch.int32)
        acc, m, v = torch.zeros(V, H, device="cuda"), torch.zeros(V, H, device="cuda"), torch.zeros(V, H, device="cuda")
        ws = torch.empty(tik.workspace_bytes(tik.OP_TOKEN_LOGPROB_BWD, 3000, H=H, V=V), dtype=torch.uint8, device="cuda")
        lws = torch.empty(tik.workspace_bytes(tik.OP_POLICY_LOSS, 3000, max_ctx=1), dtype=torch.uint8, device="cuda")
        seen = []
        for i, n in enumerate([3000, 100, 700, 1, 256, 2999, 257, 64] * 2):
            x = big[:n].contiguous(); lse = torch.empty(n, device="cuda")
            lp = tik.tik_token_logprob(x, W, ids[:n], lse=lse); step()
            loss, d, _ = tik.tik_policy_loss(lp, lp - 0.1, torch.ones_like(lp), ws=lws); step()
            dx, _ = tik.tik_token_logprob_bwd(d, x, W, ids[:n], lse, d_lm_head=acc, accumulate=i % 3 > 0, ws=ws); step()
            tik.tik_adamw([W], [acc], [m], [v], 1e-3, i + 1, seed=i); step()
            seen += [loss.clone(), dx]
        torch.cuda.synchronize()
        return seen + [W, m, v, acc]
    for x, y in zip(chain(False), chain(True)):
        assert torch.equal(x, y)


def test_launch_counts(tik):
    """Kernels per call: the ones that the header states."""
    def launches(f):
        n = tik.kernel_launches()
        f()
        return tik.kernel_launches() - n
    z = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    assert launches(lambda: tik.tik_policy_loss(z(4096), z(4096), z(4096))) == 1
    assert launches(lambda: tik.tik_policy_loss(z(4097), z(4097), z(4097))) == 2
    x, W = torch.zeros(300, 64, device="cuda", dtype=BF), torch.zeros(500, 64, device="cuda", dtype=BF)
    back = lambda n, **kw: tik.tik_token_logprob_bwd(z(n), x[:n], W, z(n).int(), z(n), **kw)  # noqa: E731
    assert launches(lambda: back(256)) == 3 and launches(lambda: back(257)) == 5
    assert launches(lambda: back(256, need_hidden=False)) == 2 and launches(lambda: back(256, need_lm_head=False)) == 3
    many = [z(8) for _ in range(401 * 4)]
    assert launches(lambda: tik.tik_adamw(many[:401], many[401:802], many[802:1203], many[1203:], 1e-3, 1)) == 2
    assert launches(lambda: tik.tik_adamw(many[:400], many[401:801], many[802:1202], many[1203:1603], 1e-3, 1)) == 1
