"""Tensors of more than 2^31 elements: offsets that pass 32 bits, in the last rows and elements above all."""
import numpy as np
import pytest
import torch

import oracle
from gpu_common import count_diff

pytestmark = pytest.mark.gpu
BF, U32, UBF = torch.bfloat16, 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def tik():
    from paper_2609_35140_b200 import binding
    binding.load()
    yield binding
    assert binding.device_status() == 0
    torch.cuda.empty_cache()


def _fill(rows, cols, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(rows, cols, dtype=BF, device="cuda")
    for r in range(0, rows, 1 << 14):
        n = min(1 << 14, rows - r)
        out[r:r + n] = torch.randn(n, cols, generator=g, device="cuda").mul_(std)
    return out


def test_lookup_and_gradient_behind_2_31_elements(tik):
    V, H = 140_003, 16_384                                    # 2.29e9 elements
    table = _fill(V, H, 1)
    T = 300
    ids = torch.from_numpy(np.random.default_rng(1).integers(V - 40, V, T)).to(torch.int32).cuda()
    ids[:3] = torch.tensor([0, V - 1, V - 1], dtype=torch.int32)
    y = tik.tik_embedding(ids, table)
    assert count_diff(y, table[ids.long()]) == 0
    before = table[V - 41:].clone()
    tik.tik_embedding_bwd(y, ids, V, 0.5, d_table=table, accumulate=True)
    ref, mag, n = oracle.embedding_bwd(y.float().cpu().numpy(), (ids.cpu().numpy() - (V - 41)), 41, 0.5)
    e = (n[:, None] + 2) * U32 * (mag + before.double().abs().cpu().numpy())
    want = ref + before.double().cpu().numpy()
    assert np.all(np.abs(table[V - 41:].double().cpu().numpy() - want) <= UBF * (np.abs(want) + e) + e)
    tik.tik_embedding_bwd(y, ids, V, 0.5, d_table=table)      # the whole table: zeros up to its end
    got = table[V - 41:].double().cpu().numpy()
    assert np.all(np.abs(got - ref) <= UBF * (np.abs(ref) + e) + e)
    rest = table[1:V - 41]
    assert all(bool((rest[r:r + 20_000] == 0).all()) for r in range(0, rest.shape[0], 20_000))


def test_many_tokens(tik):
    T, V, H = 300_007, 5_003, 8_192                           # 2.46e9 elements of gradients, the sort's list in global memory
    dy = _fill(T, H, 2)
    ids = torch.from_numpy(np.random.default_rng(2).integers(0, V - 3, T)).to(torch.int32).cuda()
    rare = torch.tensor([5, T // 2, T - 2, T - 1], device="cuda")
    ids[rare] = torch.tensor([V - 3, V - 2, V - 2, V - 1], dtype=torch.int32, device="cuda")
    got = tik.tik_embedding_bwd(dy, ids, V, 1.0, d_table=torch.empty(V, H, device="cuda"))
    assert count_diff(got[V - 3], dy[5].float()) == 0 and count_diff(got[V - 1], dy[T - 1].float()) == 0
    assert count_diff(got[V - 2], dy[T // 2].float() + dy[T - 2].float()) == 0
    for v in (0, V // 2):
        rows = dy[(ids == v).nonzero().flatten()].double()
        assert bool(((got[v].double() - rows.sum(0)).abs() <= (rows.shape[0] + 2) * U32 * rows.abs().sum(0)).all())
    y = tik.tik_embedding(ids, got.to(BF), 2.0, y=dy)
    at = torch.tensor([0, T - 3, T - 1], device="cuda")
    assert count_diff(y[at], (got.to(BF)[ids[at].long()].float() * 2).to(BF)) == 0


def test_block_norm_of_many_rows(tik):
    T, H = 270_001, 8_192                                     # 2.21e9 elements
    x, res = _fill(T, H, 3, 2.0), _fill(T, H, 4, 4.0)
    w, p = (torch.ones(H, device="cuda", dtype=BF) for _ in range(2))
    gate = torch.full((T, 1), 0.5, dtype=BF, device="cuda")
    y, s = tik.tik_block_norm(x, res, w, 1e-6, post_weight=p, gate=gate)
    tail = slice(T - 5, T)
    y1, s1 = tik.tik_block_norm(x[tail].contiguous(), res[tail].contiguous(), w, 1e-6, post_weight=p, gate=gate[tail].contiguous())
    assert count_diff(y[tail], y1) == 0 and count_diff(s[tail], s1) == 0
    del res
    dx, dr, dw, dp, dg = tik.tik_block_norm_bwd(y, s, x, s, w, 1e-6, post_weight=p, gate=gate)
    one = tik.tik_block_norm_bwd(y1, s1, x[tail].contiguous(), s1, w, 1e-6, post_weight=p, gate=gate[tail].contiguous())
    assert count_diff(dx[tail], one[0]) == 0 and count_diff(dr[tail], one[1]) == 0 and count_diff(dg[tail], one[4]) == 0
    # the weight's gradient, summed here in parts: 2 T additions of fp32 against fp64
    ref = torch.zeros(H, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(ref)
    for r in range(0, T, 1 << 14):
        a, v = y[r:r + (1 << 14)].double(), s[r:r + (1 << 14)].double()
        t = a * v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6)
        ref += t.sum(0)
        mag += t.abs().sum(0)
    assert bool(((dw.double() - ref).abs() <= (T / 148 + 600) * U32 * mag).all())        # a CTA's rows, and what is added up of them


def test_gradients_of_2_31_elements(tik):
    n = (1 << 31) + 12_345
    flat = torch.zeros(n + 3, dtype=BF, device="cuda")
    for dst in (flat[:n], flat[3:]):                          # 16-byte aligned, and 6 bytes off
        flat.zero_()
        at = torch.tensor([0, 1, 1 << 30, (1 << 31) - 1, 1 << 31, n - 2, n - 1], device="cuda")
        dst[at] = 3.0
        norm = tik.tik_grad_clip([dst], 0.5)
        assert float(norm) == float(np.float32(np.sqrt(9.0 * 7)))
        want = (torch.tensor(3.0) * float(np.float32(0.5) / np.float32(norm.item()))).to(BF)
        assert bool((dst[at].cpu() == want).all()) and int((dst != 0).sum()) == 7
