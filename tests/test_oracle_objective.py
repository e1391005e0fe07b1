"""Pins for the oracles of the policy loss, the log-probability gradient and the AdamW step: torch's autograd and optimiser in fp64, and
closed forms."""
import math

import numpy as np
import pytest
import torch

import oracle


def _loss_inputs(T=40, S=5, seed=1):
    rng = np.random.default_rng(seed)
    cu = np.concatenate([[0], np.sort(rng.integers(0, T + 1, S - 1)), [T]])
    old = -3 * rng.random(T)
    return dict(logprob=old + 0.5 * rng.standard_normal(T), old_logprob=old, ref_logprob=old + 0.3 * rng.standard_normal(T),
                weight=np.where(rng.random(T) < 0.3, 0.0, 0.5 + rng.random(T)), cu_seqlens=cu), rng


@pytest.mark.parametrize("reduction", ["sum", "token", "sequence"])
@pytest.mark.parametrize("per_seq,dual,kl", [(False, 0.0, 0.0), (True, 3.0, 0.1), (False, 1.5, 0.05)])
def test_policy_loss_against_autograd(reduction, per_seq, dual, kl):
    a, rng = _loss_inputs()
    T, S = 40, 5
    adv = rng.standard_normal((S, 1)) if per_seq else rng.standard_normal(T)
    loss, d, stats = oracle.policy_loss(advantage=adv, clip_high=0.28, clip_dual=dual, kl_coef=kl, reduction=reduction, scale=0.5, **a)
    lp = torch.tensor(a["logprob"], requires_grad=True)
    seq = np.repeat(np.arange(S), np.diff(a["cu_seqlens"]))
    A = torch.tensor(adv[seq, 0] if per_seq else adv)
    r = torch.exp(lp - torch.tensor(a["old_logprob"]))
    gain = torch.minimum(r * A, r.clamp(0.8, 1.28) * A)
    if dual:
        gain = torch.where(A < 0, torch.maximum(gain, dual * A), gain)
    y = torch.tensor(a["ref_logprob"]) - lp
    token = -gain + kl * (torch.exp(y) - y - 1)
    on = torch.tensor(a["weight"] != 0)
    w = torch.tensor(a["weight"])
    if reduction == "sequence":
        n = torch.tensor([max(1, int(on[torch.tensor(seq == s)].sum())) for s in range(S)])[torch.tensor(seq)]
    else:
        n = int(on.sum()) if reduction == "token" else 1
    want = (0.5 * w * token / n).sum()
    want.backward()
    assert abs(loss - want.item()) < 1e-12
    assert np.abs(d - lp.grad.numpy()).max() < 1e-12
    assert stats[4] == int(on.sum())


def test_policy_loss_closed_forms():
    lp, adv = np.array([-1.0, -2.0, -0.5]), np.array([1.0, -2.0, 0.5])
    loss, d, stats = oracle.policy_loss(lp, lp, adv)                       # on-policy: ratios of one
    assert abs(loss + adv.mean()) < 1e-15 and np.allclose(d, -adv / 3) and stats[2] == 0 and stats[3] == 0
    loss, d, stats = oracle.policy_loss(lp + np.log(2.0), lp, adv)         # doubled probabilities: good ones are cut at 1.2
    assert abs(loss - (-1.2 + 4.0 - 0.6) / 3) < 1e-12 and d[0] == d[2] == 0 and abs(d[1] - 4.0 / 3) < 1e-12 and abs(stats[2] - 2 / 3) < 1e-15
    assert abs(stats[3] - (1 - np.log(2.0))) < 1e-12


def test_logprob_gradient_against_autograd_and_sums():
    rng = np.random.default_rng(2)
    T, H, V, f = 6, 5, 9, 1.4
    x, W, g, ids = rng.standard_normal((T, H)), rng.standard_normal((V, H)), rng.standard_normal(T), rng.integers(0, V, T)
    g[2], ids[4] = 0.0, -1
    X, L = torch.tensor(x, requires_grad=True), torch.tensor(W, requires_grad=True)
    z = f * X @ L.T
    lse = torch.logsumexp(z, 1)
    lp = (torch.log_softmax(z, 1) * torch.nn.functional.one_hot(torch.tensor(np.maximum(ids, 0)), V)).sum(1)
    (lp * torch.tensor(np.where(ids < 0, 0.0, g))).sum().backward()
    dx, dW, dz = oracle.token_logprob_bwd(g, x, W, ids, lse.detach().numpy(), f)
    assert np.abs(dx - X.grad.numpy()).max() < 1e-12 and np.abs(dW - L.grad.numpy()).max() < 1e-12
    assert np.abs(dz.sum(axis=1)).max() < 1e-12                            # a log-probability does not change when all logits move together


@pytest.mark.parametrize("decay", [0.0, 0.1])
def test_adamw_against_the_optimiser_in_fp64(decay):
    rng = np.random.default_rng(3)
    p = torch.nn.Parameter(torch.tensor(rng.standard_normal(20)))
    opt = torch.optim.AdamW([p], lr=3e-3, betas=(0.9, 0.99), eps=1e-6, weight_decay=decay)
    w, m, v = p.detach().numpy().copy(), np.zeros(20), np.zeros(20)
    for step in range(1, 6):
        g = rng.standard_normal(20)
        p.grad = torch.tensor(g)
        opt.step()
        w, m, v = oracle.adamw(w, g, m, v, 3e-3, step, 0.9, 0.99, 1e-6, decay)
        assert np.abs(w - p.detach().numpy()).max() < 1e-13


def test_adamw_first_step_is_the_sign():
    w, _, _ = oracle.adamw(np.zeros(3), np.array([2.0, -0.5, 0.0]), np.zeros(3), np.zeros(3), 0.1, 1)
    assert np.abs(w - [-0.1, 0.1, 0.0]).max() < 1e-8


def test_e4m3_against_torch_and_scales():
    values = oracle.e4m3_values()
    theirs = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(values, theirs, equal_nan=True) and np.nanmax(values) == 448.0
    for top, k in ((448.0, 0), (448.0001, 1), (224.0, -1), (1.75, -8), (1.7501, -7), (1.0, -8), (0.0, -127), (2.0 ** -200, -127)):
        assert oracle.block_scale([0.0, -top]) == k, top
        assert k == -127 or 224.0 * 2.0 ** k < top <= 448.0 * 2.0 ** k
    assert math.isnan(values[127]) and math.isnan(values[255])
