"""Pins for the oracles of the embedding gradient, the step between two blocks and its gradient, and the gradient norm:
torch's autograd in fp64, finite differences and closed forms."""
import numpy as np
import pytest
import torch

import oracle


def _t(a):
    return torch.from_numpy(np.asarray(a, dtype=np.float64)).requires_grad_(True)


def _rms(v, w, eps):
    return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + eps) * w


@pytest.mark.parametrize("post,gate,nxt,a", [(True, "channel", True, 0.7), (True, "token", True, -0.3), (False, "token", True, 1.0),
                                             (False, "channel", False, 0.5), (True, None, False, 1.0), (False, None, True, 1.0)])
def test_block_norm_and_its_gradient_against_autograd(post, gate, nxt, a):
    rng = np.random.default_rng(3)
    T, H, eps = 7, 24, 1e-3
    x, res, dy, ds = (rng.standard_normal((T, H)) for _ in range(4))
    w, wp = (1 + 0.3 * rng.standard_normal(H) for _ in range(2))
    g = {"channel": rng.standard_normal(H), "token": rng.standard_normal((T, 1)), None: None}[gate]
    X, R, W, P = _t(x), _t(res), _t(w), _t(wp)
    Gt = _t(g) if g is not None else None
    n = _rms(X, P, eps) if post else X
    S = R + a * (Gt * n if Gt is not None else n)
    loss = (S * torch.from_numpy(ds)).sum()
    if nxt:
        loss = loss + (_rms(S, W, eps) * torch.from_numpy(dy)).sum()
    loss.backward()
    s, u = oracle.block_norm(x, res, eps, wp if post else None, g, a)
    assert np.abs(s - S.detach().numpy()).max() < 1e-13 and np.abs(res + u - s).max() < 1e-13
    got, mag = oracle.block_norm_bwd(dy if nxt else None, ds, x, s, w if nxt else None, eps, wp if post else None, g, a)
    want = {"d_x": X.grad, "d_residual": R.grad}
    if nxt:
        want["d_weight"] = W.grad
    if post:
        want["d_post_weight"] = P.grad
    if g is not None:
        want["d_gate"] = Gt.grad
    assert sorted(got) == sorted(want) == sorted(mag)
    for k, v in want.items():
        assert np.abs(got[k] - v.numpy()).max() < 1e-12, k
        assert got[k].shape == mag[k].shape and np.all(mag[k] >= np.abs(got[k]) - 1e-12), k


def test_block_norm_gradient_against_differences():
    rng = np.random.default_rng(4)
    T, H, eps, h = 3, 8, 1e-2, 1e-6
    x, res, dy, ds = (rng.standard_normal((T, H)) for _ in range(4))
    w, wp, g = (1 + 0.3 * rng.standard_normal(H) for _ in range(3))

    def loss(x, res, w, wp, g):
        s, _ = oracle.block_norm(x, res, eps, wp, g, 0.6)
        return float((ds * s).sum() + (dy * s / np.sqrt((s * s).mean(1, keepdims=True) + eps) * w).sum())

    s, _ = oracle.block_norm(x, res, eps, wp, g, 0.6)
    got, _ = oracle.block_norm_bwd(dy, ds, x, s, w, eps, wp, g, 0.6)
    args = [x, res, w, wp, g]
    for i, name in enumerate(("d_x", "d_residual", "d_weight", "d_post_weight", "d_gate")):
        flat = args[i].reshape(-1)
        for j in range(flat.size):
            keep = flat[j]
            flat[j] = keep + h
            up = loss(*args)
            flat[j] = keep - h
            down = loss(*args)
            flat[j] = keep
            assert abs((up - down) / (2 * h) - got[name].reshape(-1)[j]) < 1e-7, (name, j)


def test_plain_norm_gradient_is_orthogonal_to_its_row():
    """A norm does not see its row's length: without eps the gradient has no part along the row."""
    rng = np.random.default_rng(5)
    s, dy = rng.standard_normal((5, 16)), rng.standard_normal((5, 16))
    got, _ = oracle.block_norm_bwd(dy, None, None, s, np.ones(16), 0.0)
    assert sorted(got) == ["d_residual", "d_weight"] and np.abs((got["d_residual"] * s).sum(1)).max() < 1e-13
    ones, _ = oracle.block_norm_bwd(dy, None, None, np.full((5, 16), 2.0), np.ones(16), 0.0)
    assert np.abs(ones["d_residual"] - (dy - dy.mean(1, keepdims=True)) / 2).max() < 1e-14      # closed form
    assert np.abs(ones["d_weight"] - dy.sum(0)).max() < 1e-14


def test_embedding_gradient_against_autograd_and_a_count():
    rng = np.random.default_rng(6)
    ids = np.array([3, 0, 3, 9, 3, -1, 10, 9])
    d_y = rng.standard_normal((8, 4))
    got, mag, n = oracle.embedding_bwd(d_y, ids, 10, 0.5)
    table = torch.zeros(10, 4, dtype=torch.float64, requires_grad=True)
    ok = (ids >= 0) & (ids < 10)
    (0.5 * table[torch.from_numpy(ids[ok])] * torch.from_numpy(d_y[ok])).sum().backward()
    assert np.abs(got - table.grad.numpy()).max() < 1e-14
    assert n.tolist() == [1, 0, 0, 3, 0, 0, 0, 0, 0, 2] and np.all(mag >= np.abs(got) - 1e-15)
    counts, _, _ = oracle.embedding_bwd(np.ones((8, 4)), ids, 10, 2.0)
    assert np.array_equal(counts[:, 0], 2.0 * n)


def test_gradient_norm_closed_forms():
    assert oracle.grad_norm([np.array([3.0]), np.array([[4.0]])]) == 5.0
    assert oracle.grad_norm([]) == 0.0 and oracle.grad_norm([np.zeros(0), np.zeros(3)]) == 0.0
    assert abs(oracle.grad_norm([np.full((10, 10), 2.0)]) - 20.0) < 1e-14
    assert abs(oracle.grad_norm([np.full(4, 1e30, dtype=np.float32)]) / 2e30 - 1) < 1e-7       # squares beyond fp32
    assert np.isinf(oracle.grad_norm([np.array([np.inf])])) and np.isnan(oracle.grad_norm([np.array([np.nan, np.inf])]))
