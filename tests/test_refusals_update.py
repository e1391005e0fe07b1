"""What the embedding, block-norm and gradient-norm entry points refuse, asked of the C interface through a stand-in context:
every refusal comes before anything is queued, so none of this needs a GPU (and with one it is left out: were a check
lost, the call would reach it with made-up addresses)."""
import ctypes
import random

import pytest
import torch

from paper_2609_35140_b200 import binding as tik

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
A, B, C, D, E = (1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20)     # 16-byte aligned addresses that nothing reads
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ctx():
    lib = tik.load()
    lib.tik_selftest_context.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]
    c = ctypes.c_void_p()
    assert lib.tik_selftest_context(ctypes.byref(c), 148) == OK
    yield c
    lib.tik_destroy(c)


def _call(name, order, base, **changed):
    args = dict(base, **changed)
    return getattr(tik.load(), name)(*[args[k] for k in order])


EMBED = dict(ids=A, table=B, y=C, scale=1.0, T=5, V=10, H=64, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(T=-1), INVALID), (dict(V=0), INVALID), (dict(H=0), INVALID), (dict(scale=INF), INVALID), (dict(scale=NAN), INVALID),
    (dict(H=60), UNSUPPORTED), (dict(ids=None), INVALID), (dict(table=None), INVALID), (dict(y=None), INVALID),
    (dict(table=B + 8), UNSUPPORTED), (dict(y=C + 2), UNSUPPORTED), (dict(T=1 << 31), UNSUPPORTED), (dict(T=0, ids=None, y=None), OK)])
def test_embedding(ctx, changed, code):
    assert _call("tik_embedding", ["ctx", *EMBED], EMBED, ctx=ctx, **changed) == code


EMBED_BWD = dict(d_y=A, ids=B, d_table=C, type=0, accumulate=0, scale=1.0, T=5, V=10, H=64, ws=D, ws_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(T=-1), INVALID), (dict(V=0), INVALID), (dict(H=-8), INVALID), (dict(scale=NAN), INVALID), (dict(type=2), INVALID),
    (dict(H=4), UNSUPPORTED), (dict(H=(1 << 23) + 8, ws_bytes=1 << 62), UNSUPPORTED), (dict(d_y=None), INVALID), (dict(ids=None), INVALID), (dict(d_table=None), INVALID),
    (dict(T=0, d_table=None), INVALID), (dict(d_y=A + 4), UNSUPPORTED), (dict(d_table=C + 8), UNSUPPORTED), (dict(ws=D + 4), UNSUPPORTED),
    (dict(T=1 << 30, ws_bytes=1 << 62), UNSUPPORTED), (dict(V=1 << 30), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws_bytes=39), WORKSPACE),
    (dict(T=0, accumulate=1, d_y=None, ids=None), OK)])
def test_embedding_bwd(ctx, changed, code):
    assert _call("tik_embedding_bwd", ["ctx", *EMBED_BWD], EMBED_BWD, ctx=ctx, **changed) == code


NORM = dict(x=A, residual=B, post=None, gate=None, kind=0, a=1.0, weight=D, s=B, y=C, eps=1e-6, T=5, H=64, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(T=-1), INVALID), (dict(H=0), INVALID), (dict(H=12), UNSUPPORTED), (dict(H=8200), UNSUPPORTED), (dict(eps=-1.0), INVALID),
    (dict(eps=NAN), INVALID), (dict(a=INF), INVALID), (dict(kind=3, gate=E), INVALID), (dict(kind=1), INVALID), (dict(gate=E), INVALID),
    (dict(x=None), INVALID), (dict(residual=None), INVALID), (dict(s=None), INVALID), (dict(y=None), INVALID), (dict(weight=None), INVALID),
    (dict(x=A + 2), UNSUPPORTED), (dict(post=E + 8), UNSUPPORTED), (dict(gate=E + 8, kind=1), UNSUPPORTED), (dict(y=C + 8), UNSUPPORTED),
    (dict(T=1 << 31), UNSUPPORTED), (dict(T=0, x=None, residual=None, s=None, y=None), OK)])
def test_block_norm(ctx, changed, code):
    assert _call("tik_block_norm", ["ctx", *NORM], NORM, ctx=ctx, **changed) == code


NORM_BWD = dict(d_y=A, d_s=B, x=C, s=D, post=None, gate=None, kind=0, a=1.0, weight=E, eps=1e-6, d_x=A, d_residual=B, d_weight=C,
                d_post=None, d_gate=None, T=5, H=64, ws=D, ws_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(T=-1), INVALID), (dict(H=20), UNSUPPORTED), (dict(eps=INF), INVALID), (dict(a=NAN), INVALID), (dict(d_y=None), INVALID),
    (dict(weight=None), INVALID), (dict(d_weight=None), INVALID), (dict(weight=None, d_weight=None), INVALID), (dict(post=E), INVALID),
    (dict(d_post=E), INVALID), (dict(gate=E, kind=1), INVALID), (dict(d_gate=E), INVALID), (dict(x=None), INVALID), (dict(d_x=None), INVALID),
    (dict(x=None, d_x=None, post=E, d_post=E), INVALID), (dict(x=None, d_x=None, gate=E, kind=2, d_gate=E), INVALID), (dict(s=None), INVALID),
    (dict(d_residual=None), INVALID), (dict(d_y=None, weight=None, d_weight=None, d_s=None), INVALID), (dict(s=D + 2), UNSUPPORTED),
    (dict(ws=D + 8), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws_bytes=5 * 2 * 64 * 4 - 1), WORKSPACE)])
def test_block_norm_bwd(ctx, changed, code):
    assert _call("tik_block_norm_bwd", ["ctx", *NORM_BWD], NORM_BWD, ctx=ctx, **changed) == code


def _list(kind, values):
    return (kind * len(values))(*values)


def _norm(ctx, ptrs, numel, types, n=None, norm=A, ws=B, ws_bytes=1 << 20):
    return tik.load().tik_grad_norm(ctx, _list(ctypes.c_void_p, ptrs), _list(ctypes.c_int64, numel), _list(ctypes.c_int, types),
                                    len(ptrs) if n is None else n, norm, ws, ws_bytes, None)


def _clip(ctx, ptrs, numel, types, out=None, max_norm=1.0, norm=A, given=0, ws=B, ws_bytes=1 << 20, n=None):
    return tik.load().tik_grad_clip(ctx, _list(ctypes.c_void_p, ptrs), None if out is None else _list(ctypes.c_void_p, out),
                                    _list(ctypes.c_int64, numel), _list(ctypes.c_int, types), len(ptrs) if n is None else n, max_norm,
                                    norm, given, ws, ws_bytes, None)


def test_gradient_lists(ctx):
    for f in (_norm, _clip):
        assert f(ctx, [C], [4], [0], n=-1) == INVALID
        assert f(ctx, [C, D], [4, -1], [0, 0]) == INVALID
        assert f(ctx, [C], [4], [2]) == INVALID
        assert f(ctx, [None], [4], [0]) == INVALID
        assert f(ctx, [C], [4], [0], norm=None) == INVALID
        assert f(ctx, [C + 1], [4], [0]) == UNSUPPORTED
        assert f(ctx, [C + 2], [4], [1]) == UNSUPPORTED
        assert f(ctx, [C], [1 << 40], [0]) == UNSUPPORTED
        assert f(ctx, [C, D], [(1 << 40) - 8, 8], [0, 0]) == UNSUPPORTED
        assert f(ctx, [C], [4], [0], ws=B + 8) == UNSUPPORTED
        assert f(ctx, [C], [4], [0], ws=None) == WORKSPACE
        assert f(ctx, [C], [4], [0], ws_bytes=8) == WORKSPACE
    for bad in (0.0, -1.0, INF, NAN):
        assert _clip(ctx, [C], [4], [0], max_norm=bad) == INVALID
    assert _clip(ctx, [C], [4], [0], out=[None]) == INVALID
    assert _clip(ctx, [C], [4], [1], out=[D + 2]) == UNSUPPORTED


def test_written_tensors_may_not_overlap(ctx):
    """An element that two tensors share would be scaled once or twice, as the kernel's blocks happen to run."""
    def refused(*a, **k):
        # n passes every other check: without the overlap the call would go on to a launch
        return _clip(ctx, *a, **k) == INVALID and b"overlap" in tik.load().tik_last_error(ctx)
    assert refused([C, C], [4, 4], [0, 0])                                    # the same tensor twice (tied weights listed twice)
    assert refused([C, C + 6], [4, 4], [0, 0])                                # one element
    assert refused([C + 8, D, C], [4, 4, 2 * 4], [0, 0, 0])                   # unsorted
    assert refused([C, D], [4, 4], [0, 0], out=[E, E])                        # two results in one place
    assert refused([C, D], [4, 4], [0, 0], out=[D, E])                        # a result over another input
    assert refused([C], [4], [0], out=[C + 2])                                # a shifted copy of itself
    assert refused([C, D], [4, 4], [1, 0], out=[C, C + 14])                   # fp32: 16 bytes


def test_overlap_rule_against_all_pairs(ctx):
    """Random lists: refused exactly where a written range meets another written one or an input that is not written."""
    rng = random.Random(3)
    for _ in range(3000):
        n = rng.randint(1, 6)
        ins, numel = [16 * rng.randint(1, 60) for _ in range(n)], [rng.choice([0, 4, 8, 16, 40]) for _ in range(n)]
        outs = None if rng.random() < 0.4 else [i if rng.random() < 0.3 else 16 * rng.randint(1, 60) for i in ins]
        to = outs or ins
        W = [(to[k], to[k] + 2 * numel[k]) for k in range(n) if numel[k]]
        R = [(ins[k], ins[k] + 2 * numel[k]) for k in range(n) if numel[k] and ins[k] != to[k]]
        meet = lambda a, b: a[0] < b[1] and b[0] < a[1]
        overlap = any(meet(W[i], W[j]) for i in range(len(W)) for j in range(i)) or any(meet(a, b) for a in W for b in R)
        # without scratch a list that passes is refused for that
        assert _clip(ctx, ins, numel, [0] * n, out=outs, ws=None, ws_bytes=0) == (INVALID if overlap else WORKSPACE)


def test_scratch_sizes():
    assert tik.workspace_bytes(tik.OP_BLOCK_NORM_BWD, 5, H=64) == 5 * 2 * 64 * 4
    assert tik.workspace_bytes(tik.OP_EMBEDDING_BWD, 5, H=64, V=10) >= 40
    assert tik.workspace_bytes(tik.OP_GRAD_NORM, 1) > 8
    for H in (8200, 1 << 20, 1 << 29, (1 << 31) - 8):        # (sizes that the gradient refuses)
        assert tik.workspace_bytes(tik.OP_BLOCK_NORM_BWD, 5, H=H) == 0
    for op in (tik.OP_BLOCK_NORM_BWD, tik.OP_EMBEDDING_BWD, tik.OP_GRAD_NORM):
        assert tik.workspace_bytes(op, 0, H=64, V=10) == 0


@pytest.mark.parametrize("changed", [dict(kind=1), dict(kind=1, d_gate=E), dict(kind=1, gate=E), dict(kind=1, gate=E, post=E, d_post=E)])
@pytest.mark.parametrize("T", [0, 5])
def test_block_norm_bwd_wants_a_channel_gate_and_its_gradient_for_any_number_of_rows(ctx, changed, T):
    """d_gate [H] is written (zeros) where there are no rows, too."""
    assert _call("tik_block_norm_bwd", ["ctx", *NORM_BWD], NORM_BWD, ctx=ctx, T=T, ws=None, **changed) == INVALID


def test_block_norm_bwd_of_no_rows_needs_no_token_gate(ctx):
    """Its [0] elements have no address.  (Without weights nothing is to be written: no launch.)"""
    none = dict(d_y=None, d_s=None, x=None, s=None, weight=None, d_x=None, d_residual=None, d_weight=None)
    assert _call("tik_block_norm_bwd", ["ctx", *NORM_BWD], NORM_BWD, ctx=ctx, T=0, ws=None, kind=2, **none) == OK


def test_the_norm_of_a_clip_is_no_gradient(ctx):
    """The norm is written beside the gradients' reads where it is computed, and read beside their writes where it is given."""
    def refused(*a, **k):
        # (without scratch a list that passes is refused for that, or goes on to a launch where the norm is given)
        return _clip(ctx, *a, **k) == INVALID and b"overlap" in tik.load().tik_last_error(ctx)
    none = dict(ws=None, ws_bytes=0)
    for given in (0, 1):
        assert refused([C, D], [4, 4], [1, 1], norm=C + 12, given=given, **none)                  # an element of a tensor clipped in place
        assert refused([C], [4], [0], norm=C + 4, given=given, **none)                            # bf16: two of them
        assert refused([C, D], [4, 4], [1, 1], out=[C, E], norm=E, given=given, **none)           # an element of a result
    assert refused([C], [4], [1], out=[D], norm=C, **none)                                        # computed, over an input
    assert _clip(ctx, [C], [4], [1], norm=C + 16, **none) == WORKSPACE                            # next to it
    assert _clip(ctx, [C], [4], [0], norm=C - 4, **none) == WORKSPACE
    assert _clip(ctx, [C, D], [0, 4], [1, 1], norm=C, **none) == WORKSPACE                        # a tensor of no elements
    assert _clip(ctx, [], [], [], given=1, **none) == OK
