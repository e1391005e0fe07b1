"""GPU parity of the embedding lookup and its gradient: exact where one rounding decides, against the fp64 oracle within the
roundings of the sums elsewhere; bits that do not depend on the call, the batch or the scratch."""
import numpy as np
import pytest
import torch

import oracle
from gpu_common import count_diff

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24                                     # half a step of fp32, relative
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}


@pytest.fixture(scope="module")
def tik():
    from paper_2609_35140_b200 import binding
    binding.load()
    yield binding
    assert binding.device_status() == 0


def _randn(shape, seed, std=1.0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _i32(v):
    return torch.as_tensor(np.ascontiguousarray(v), dtype=torch.int32).cuda()


@pytest.mark.parametrize("T,V,H", [(1, 1, 8), (1, 2048, 3584), (5, 7, 72), (257, 2048, 256), (1000, 300, 1544), (64, 1000, 8192),
                                   (3, 11, 20000)])
@pytest.mark.parametrize("scale", [1.0, 0.3, -7.5, 0.0])
def test_lookup(tik, T, V, H, scale):
    rng = np.random.default_rng(T + V)
    ids, table = _i32(rng.integers(0, V, T)), _randn((V, H), 1)
    buf = torch.full((T + 2, H), 7.0, dtype=torch.bfloat16, device="cuda")
    y = tik.tik_embedding(ids, table, scale, y=buf[1:T + 1])
    assert count_diff(y, (table[ids.long()].float() * np.float32(scale)).to(torch.bfloat16)) == 0
    assert bool((buf[0] == 7.0).all()) and bool((buf[T + 1] == 7.0).all())
    assert count_diff(tik.tik_embedding(ids, table, scale), y) == 0


def test_ids_out_of_range_give_zeros_and_a_flag(tik):
    V, H = 40, 64
    ids, table = _i32([0, -1, 39, 40, 2 ** 31 - 1, -2 ** 31, 5]), _randn((V, H), 2)
    y = tik.tik_embedding(ids, table, 2.0)
    assert tik.device_status() == tik.DEV_BAD_TOKEN
    good = [0, 2, 6]
    assert count_diff(y[good], (table[ids[good].long()].float() * 2).to(torch.bfloat16)) == 0
    assert bool((y[[1, 3, 4, 5]] == 0).all())
    d = tik.tik_embedding_bwd(_randn((7, H), 3), ids, V)
    assert tik.device_status() == tik.DEV_BAD_TOKEN
    assert bool((d.float().abs().sum(1) > 0).nonzero().flatten().cpu().eq(torch.tensor([0, 5, 39])).all())
    assert tik.tik_embedding(_i32([]), table).shape == (0, H)


def _check_bwd(tik, d_y, ids, V, scale, dtype, accumulate, seed):
    T, H = d_y.shape
    old = _randn((V + 2, H), seed, 2.0, dtype)
    buf = old.clone()
    got = tik.tik_embedding_bwd(d_y, ids, V, scale, d_table=buf[1:V + 1], accumulate=accumulate)
    assert got.data_ptr() == buf[1].data_ptr() and count_diff(buf[:1], old[:1]) == 0 and count_diff(buf[V + 1:], old[V + 1:]) == 0
    scale = float(np.float32(scale))
    ref, mag, n = oracle.embedding_bwd(d_y.float().cpu().numpy(), ids.cpu().numpy(), V, scale)
    if accumulate:
        before = old[1:V + 1].double().cpu().numpy()
        touched = n > 0
        assert np.array_equal(got.double().cpu().numpy()[~touched], before[~touched])         # bit for bit what it was
        ref, mag = np.where(touched[:, None], ref + before, before), mag + np.abs(before)
    # n - 1 additions, the scale and the addition to the old value, each off by half a step of fp32 of a value no larger
    # than the sum of magnitudes; then one rounding to the table's type
    fp32 = (n[:, None] + 2) * U32 * mag
    err = np.abs(got.double().cpu().numpy() - ref)
    assert np.all(err <= HALF[dtype] * (np.abs(ref) + fp32) + fp32), float((err - HALF[dtype] * np.abs(ref)).max())
    return got


def _ids(kind, T, V, rng):
    if kind == "zipf":
        return (np.floor(np.exp(rng.random(T) * np.log(V + 1))).astype(np.int64) - 1) * 7 % V
    if kind == "uniform":
        return rng.integers(0, V, T)
    if kind == "one":
        return np.full(T, V // 2)
    if kind == "distinct":
        return rng.permutation(max(V, T))[:T] % V
    if kind == "few":
        return rng.integers(0, 3, T) * (V // 3)
    return np.sort(rng.integers(0, V, T))[::-1]                                                # "falling"


@pytest.mark.parametrize("T,V,H,kind", [
    (1, 1, 8, "one"), (1, 5000, 72, "uniform"), (2, 3, 3584, "one"), (31, 40, 64, "falling"), (33, 1000, 1536, "distinct"),
    (64, 64, 200, "one"), (65, 64, 200, "one"), (127, 2, 264, "uniform"), (128, 9, 64, "few"), (129, 151936, 8, "zipf"), (256, 2048, 256, "zipf"),
    (700, 33, 520, "few"), (1000, 151936, 16, "uniform"), (1023, 100, 72, "one"), (1025, 4097, 136, "zipf"), (3000, 2048, 256, "zipf"),
    (4097, 300, 64, "falling"), (9001, 152064, 24, "zipf"), (20011, 17, 40, "zipf"), (16384, 70000, 8, "distinct"), (33000, 5000, 8, "one"),
    (255, 40, 264, "few"), (256, 700, 3584, "one"), (256, 3, 64, "uniform"), (257, 3, 64, "uniform"), (200, 5, 75776, "uniform"), (90, 4, 20000, "one"),
    (4096, 500, 16, "zipf"), (4608, 151936, 16, "zipf"), (4609, 151936, 16, "zipf"), (8193, 2000, 16, "uniform"), (65536, 152064, 8, "zipf"), (65537, 152064, 8, "zipf"), (70001, 300, 8, "one"), (100003, 600000, 8, "uniform"),
    (131072, 3, 16, "falling")])
@pytest.mark.parametrize("dtype,accumulate", [(torch.bfloat16, False), (torch.float32, False), (torch.bfloat16, True), (torch.float32, True)])
def test_gradient(tik, T, V, H, kind, dtype, accumulate):
    ids = _i32(_ids(kind, T, V, np.random.default_rng(T)))
    d_y = _randn((T, H), T + 1)
    a = _check_bwd(tik, d_y, ids, V, -1.7, dtype, accumulate, 5)
    if not accumulate:
        assert count_diff(tik.tik_embedding_bwd(d_y, ids, V, -1.7, d_table=torch.empty_like(a)), a) == 0
        if dtype == torch.bfloat16:
            assert count_diff(tik.tik_embedding_bwd(d_y, ids, V, -1.7), a) == 0


def test_gradient_of_no_tokens(tik):
    d_y, ids = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), _i32([])
    full = torch.full((9, 64), 3.0, device="cuda")
    tik.tik_embedding_bwd(d_y, ids, 9, d_table=full, accumulate=True)
    assert bool((full == 3.0).all())
    tik.tik_embedding_bwd(d_y, ids, 9, d_table=full)
    assert bool((full == 0.0).all())
    # ids that are all out of range: zeros, or nothing touched
    ids, d_y = _i32([-1, 9]), _randn((2, 64), 1)
    assert bool((tik.tik_embedding_bwd(d_y, ids, 9) == 0).all())
    full.fill_(3.0)
    tik.tik_embedding_bwd(d_y, ids, 9, d_table=full, accumulate=True)
    assert bool((full == 3.0).all()) and tik.device_status() == tik.DEV_BAD_TOKEN


@pytest.mark.parametrize("n", [1, 5, 64, 65, 200, 3000])
def test_a_rows_bits_depend_on_its_own_tokens_only(tik, n):
    """The same n gradients of one id, alone and scattered in order among thousands of tokens of other ids."""
    H, V, T = 328, 5000, 4 * n + 2000
    rng = np.random.default_rng(n)
    d_y = _randn((T, H), 11)
    at = np.sort(rng.permutation(T)[:n])
    ids = rng.integers(0, V - 1, T)
    ids[ids >= 1234] += 1                                                                      # every id but 1234
    ids[at] = 1234
    alone = torch.empty(V, H, device="cuda")
    among = torch.empty(V, H, device="cuda")
    tik.tik_embedding_bwd(d_y[torch.from_numpy(at).cuda()].contiguous(), _i32(np.full(n, 1234)), V, 0.9, d_table=alone)
    tik.tik_embedding_bwd(d_y, _i32(ids), V, 0.9, d_table=among)
    assert count_diff(alone[1234], among[1234]) == 0 and bool((alone[1234] != 0).any())


def test_gradient_against_differences(tik):
    """y = scale * table[ids] is linear: the loss moves by exactly the gradient times the step."""
    V, H, T = 12, 16, 50
    ids, d_y = _i32(np.random.default_rng(1).integers(0, V, T)), _randn((T, H), 4)
    table = (_randn((V, H), 5) * 0).to(torch.bfloat16)
    got = tik.tik_embedding_bwd(d_y, ids, V, 2.0, d_table=torch.empty(V, H, device="cuda"))
    for v in range(V):
        for h in (0, 7, 15):
            step = table.clone()
            step[v, h] = 1.0                                                                   # y has entries 0 and 2: exact
            diff = (tik.tik_embedding(ids, step, 2.0).double() * d_y.double()).sum()
            n = int((ids == v).sum())
            assert abs(float(diff - got[v, h].double())) <= (n + 2) * U32 * 2 * float(d_y[ids == v, h].double().abs().sum()) + 1e-30


def test_captured_and_replayed_on_new_ids(tik):
    T, V, H = 1500, 3000, 256
    rng = np.random.default_rng(2)
    ids, table, d_y = _i32(_ids("zipf", T, V, rng)), _randn((V, H), 1), _randn((T, H), 2)
    y, grad = torch.empty_like(d_y), torch.zeros(V, H, device="cuda")
    ws = torch.empty(tik.workspace_bytes(tik.OP_EMBEDDING_BWD, T, H=H, V=V), dtype=torch.uint8, device="cuda")

    def step():
        tik.tik_embedding(ids, table, 1.5, y=y)
        tik.tik_embedding_bwd(d_y, ids, V, 1.5, d_table=grad, ws=ws)
        tik.tik_embedding_bwd(y, ids, V, 0.5, d_table=grad, accumulate=True, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for seed in (3, 4):
        ids.copy_(_i32(_ids("zipf" if seed == 3 else "few", T, V, rng)))
        d_y.copy_(_randn((T, H), seed))
        ws.fill_(255)                                                                          # nothing is kept there
        g.replay()
        got = (y.clone(), grad.clone())
        step()
        assert count_diff(y, got[0]) == 0 and count_diff(grad, got[1]) == 0


def test_refused_tensors(tik):
    ids, table, d_y = _i32([1, 2]), _randn((4, 64), 1), _randn((2, 64), 2)
    for bad in (lambda: tik.tik_embedding(ids.long(), table), lambda: tik.tik_embedding(ids.cpu(), table), lambda: tik.tik_embedding(ids, table.float()),
                lambda: tik.tik_embedding(ids, table[:, :32]), lambda: tik.tik_embedding(ids, table[:, :60].contiguous()),
                lambda: tik.tik_embedding_bwd(d_y.float(), ids, 4), lambda: tik.tik_embedding_bwd(d_y, ids, 4, d_table=table.half()),
                lambda: tik.tik_embedding_bwd(d_y, ids, 4, ws=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(tik.TikError):
            bad()
    for bad in (lambda: tik.tik_embedding(ids.view(2, 1), table), lambda: tik.tik_embedding(ids, table, y=d_y[:1]),
                lambda: tik.tik_embedding_bwd(d_y, ids[:1], 4), lambda: tik.tik_embedding_bwd(d_y, ids, 5, d_table=table),
                lambda: tik.tik_embedding_bwd(d_y, ids, 0), lambda: tik.tik_embedding_bwd(d_y, ids, 4, accumulate=True)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("n", [1, 33, 200, 5000, 66000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_a_rows_bits_among_more_tokens_than_one_cluster_sorts(tik, n, accumulate):
    """As above, for lists that many CTAs sort, against the call on the row's own gradients by whichever path takes those."""
    H, V, T = 72, 3000, 70_001
    rng = np.random.default_rng(n)
    d_y, old = _randn((T, H), 12), _randn((V, H), 13, 2.0, torch.float32)
    at = np.sort(rng.permutation(T)[:n])
    ids = rng.integers(0, V - 1, T)
    ids[ids >= 1234] += 1
    ids[at] = 1234
    alone, among = old.clone(), old.clone()
    tik.tik_embedding_bwd(d_y[torch.from_numpy(at).cuda()].contiguous(), _i32(np.full(n, 1234)), V, 0.9, d_table=alone, accumulate=accumulate)
    tik.tik_embedding_bwd(d_y, _i32(ids), V, 0.9, d_table=among, accumulate=accumulate)
    assert count_diff(alone[1234], among[1234]) == 0 and count_diff(alone[1234], old[1234]) > 0


@pytest.mark.parametrize("dtype,accumulate", [(torch.bfloat16, False), (torch.float32, True)])
def test_more_long_runs_than_a_cta_sets_aside(tik, dtype, accumulate):
    """Seven runs of 36 tokens in 782 slices of columns: about 37 items of several pieces for each of 148 CTAs, which set 32 aside for all
    of their warps and add up the others warp by warp.  The same bits as by columns in parts, where none is left over."""
    V, H, step = 8, 200_000, 8000
    ids = _i32(np.random.default_rng(6).permutation(np.concatenate([np.repeat(np.arange(7), 36), np.full(4, 7)])))
    d_y, old = _randn((256, H), 1), _randn((V, H), 2, 2.0, dtype)
    got = tik.tik_embedding_bwd(d_y, ids, V, -1.7, d_table=old.clone(), accumulate=accumulate)
    for c in range(0, H, step):
        part = tik.tik_embedding_bwd(d_y[:, c:c + step].contiguous(), ids, V, -1.7, d_table=old[:, c:c + step].contiguous(), accumulate=accumulate)
        assert count_diff(got[:, c:c + step].contiguous(), part) == 0, c
    _check_bwd(tik, d_y[:, :step].contiguous(), ids, V, -1.7, dtype, accumulate, 5)
