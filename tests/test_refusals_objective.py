"""What the policy loss, the log-probability gradient and the AdamW step refuse, asked of the C interface through a stand-in
context: every refusal comes before anything is queued, so none of this needs a GPU (and with one it is left out: were a check
lost, the call would reach it with made-up addresses)."""
import ctypes

import pytest
import torch

from paper_2609_35140_b200 import binding as tik

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
A, B, C, D, E, F, G, H_ = ((i + 1) << 20 for i in range(8))       # 16-byte aligned addresses that nothing reads
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ctx():
    lib = tik.load()
    lib.tik_selftest_context.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]
    c = ctypes.c_void_p()
    assert lib.tik_selftest_context(ctypes.byref(c), 148) == OK
    yield c
    lib.tik_destroy(c)


LOGPROB = dict(d=A, x=B, w=C, ids=D, lse=E, dx=F, dw=G, type=0, accumulate=0, T=5, H=64, V=10, f=1.0, ws=H_, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(T=-1), INVALID), (dict(H=0), INVALID), (dict(V=0), INVALID), (dict(f=0.0), INVALID), (dict(f=-1.0), INVALID), (dict(f=INF), INVALID),
    (dict(f=NAN), INVALID), (dict(type=2), INVALID), (dict(accumulate=1), INVALID), (dict(accumulate=1, dw=None, type=1), INVALID),
    (dict(dx=None, dw=None), INVALID), (dict(H=96), UNSUPPORTED), (dict(V=(1 << 30) + 1), UNSUPPORTED), (dict(d=None), INVALID), (dict(x=None), INVALID),
    (dict(w=None), INVALID), (dict(ids=None), INVALID), (dict(lse=None), INVALID), (dict(x=B + 8), UNSUPPORTED), (dict(w=C + 2), UNSUPPORTED),
    (dict(dx=F + 4), UNSUPPORTED), (dict(dw=G + 8), UNSUPPORTED), (dict(ws=H_ + 8), UNSUPPORTED), (dict(T=(1 << 31) - 256), UNSUPPORTED),
    (dict(dx=B), INVALID), (dict(dx=C + 16), INVALID), (dict(dw=B + 512), INVALID), (dict(dw=F), INVALID), (dict(dw=E), INVALID),
    (dict(dx=F, dw=F + 624, type=1), INVALID), (dict(ws=None), WORKSPACE), (dict(ws_bytes=100), WORKSPACE), (dict(T=0, dx=None, dw=None), OK),
    (dict(T=0, dw=None, d=None, x=None, ids=None, lse=None), OK), (dict(T=0, type=1, accumulate=1, d=None, x=None, ws=None), OK)])
def test_logprob_bwd(ctx, changed, code):
    args = dict(LOGPROB, **changed)
    assert tik.load().tik_token_logprob_bwd(ctx, *args.values()) == code


LOSS = dict(lp=A, old=B, adv=C, per=0, weight=None, ref=None, cu=D, S=2, T=5, low=0.2, high=0.2, dual=0.0, kl=0.0, reduction=1, scale=1.0, loss=E, d=F,
            stats=G, ws=H_, ws_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(T=-1), INVALID), (dict(S=-1), INVALID), (dict(low=-0.1), INVALID), (dict(low=1.0), INVALID), (dict(low=NAN), INVALID), (dict(high=-0.1), INVALID),
    (dict(high=INF), INVALID), (dict(dual=1.0), INVALID), (dict(dual=0.5), INVALID), (dict(dual=INF), INVALID), (dict(kl=NAN), INVALID),
    (dict(scale=INF), INVALID), (dict(reduction=3), INVALID), (dict(reduction=-1), INVALID), (dict(loss=None), INVALID), (dict(lp=None), INVALID),
    (dict(old=None), INVALID), (dict(adv=None), INVALID), (dict(reduction=2, cu=None), INVALID), (dict(reduction=2, S=0), INVALID),
    (dict(per=1, cu=None), INVALID), (dict(kl=0.1), INVALID), (dict(T=1 << 31), UNSUPPORTED), (dict(lp=A + 2), UNSUPPORTED), (dict(cu=D + 1), UNSUPPORTED),
    (dict(d=F + 2), UNSUPPORTED), (dict(ws=H_ + 4), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws_bytes=64), WORKSPACE)])
def test_policy_loss(ctx, changed, code):
    args = dict(LOSS, **changed)
    assert tik.load().tik_policy_loss(ctx, *args.values()) == code


def _step(ctx, n=2, numel=(64, 33), p=(A, B), g=(C, D), m=(E, F), v=(G, H_), master=None, ms=None, vs=None, pt=(1, 1), gt=(1, 1), state=1, lr=1e-3,
          beta1=0.9, beta2=0.999, eps=1e-8, decay=0.1, step=1, lr_device=None, step_device=None, norm=None, max_norm=1.0):
    def array(values, kind=ctypes.c_void_p):
        return None if values is None else (kind * len(values))(*values)
    return tik.load().tik_adamw(ctx, array(p), array(pt, ctypes.c_int), array(g), array(gt, ctypes.c_int), array(master), array(m), array(v), array(ms),
                                array(vs), state, array(numel, ctypes.c_int64), n, lr, beta1, beta2, eps, decay, step, lr_device, step_device, norm, max_norm,
                                0, 0, None)


EIGHT = dict(state=2, ms=(9 << 20, 10 << 20), vs=(11 << 20, 12 << 20))


@pytest.mark.parametrize("changed,code", [
    (dict(n=-1), INVALID), (dict(state=0), INVALID), (dict(state=3), INVALID), (dict(lr=-1.0), INVALID), (dict(lr=NAN), INVALID), (dict(lr=1e39), INVALID),
    (dict(beta1=1.0), INVALID), (dict(beta1=-0.1), INVALID), (dict(beta2=1.0), INVALID), (dict(beta2=NAN), INVALID), (dict(eps=0.0), INVALID),
    (dict(eps=1e-60), INVALID), (dict(eps=INF), INVALID), (dict(decay=-1.0), INVALID), (dict(decay=INF), INVALID), (dict(step=0), INVALID),
    (dict(norm=9 << 20, max_norm=0.0), INVALID), (dict(norm=9 << 20, max_norm=INF), INVALID), (dict(p=None), INVALID), (dict(g=None), INVALID),
    (dict(m=None), INVALID), (dict(v=None), INVALID), (dict(numel=None), INVALID), (dict(state=2), INVALID), (dict(numel=(64, -1)), INVALID),
    (dict(pt=(1, 2)), INVALID), (dict(gt=(5, 1)), INVALID), (dict(p=(A, None)), INVALID), (dict(m=(None, F)), INVALID),
    (dict(master=(9 << 20, 10 << 20)), INVALID), (dict(master=(None, None), pt=(0, 1)), INVALID), (dict(numel=(64, 1 << 40)), UNSUPPORTED),
    (dict(p=(A + 2, B)), UNSUPPORTED), (dict(g=(C, D + 1), gt=(1, 0)), UNSUPPORTED), (dict(m=(E, F + 3)), UNSUPPORTED),
    (dict(lr_device=9 << 20 | 2), UNSUPPORTED), (dict(norm=9 << 20 | 1), UNSUPPORTED),
    (dict(EIGHT, ms=(9 << 20, None)), INVALID),
    # ranges that meet
    (dict(p=(A, A)), INVALID), (dict(p=(A, A + 252)), INVALID), (dict(g=(A, D)), INVALID), (dict(g=(C, B + 128)), INVALID), (dict(m=(G, F)), INVALID),
    (dict(norm=A + 4), INVALID), (dict(step_device=H_ + 128), INVALID), (dict(EIGHT, ms=(9 << 20, (9 << 20) + 1)), INVALID),
    (dict(EIGHT, vs=(E + 63, 12 << 20)), INVALID)])
def test_adamw(ctx, changed, code):
    assert _step(ctx, **changed) == code


@pytest.mark.parametrize("changed", [
    dict(n=0, p=None, g=None, m=None, v=None, numel=None, pt=None, gt=None), dict(numel=(0, 0), p=(None, None), g=(None, None), m=(None, None), v=(None, None)),
    dict(n=0, state=2)])
def test_adamw_of_nothing(ctx, changed):
    assert _step(ctx, **changed) == OK


def test_scratch():
    assert tik.workspace_bytes(tik.OP_TOKEN_LOGPROB_BWD, 0, H=64, V=10) == 0
    # d_z [256][64] bf16, one tile's part, a number per row
    assert tik.workspace_bytes(tik.OP_TOKEN_LOGPROB_BWD, 5, H=64, V=10) == 64 * 512 + 256 * 256 * 4 + 256
    # a chunk's d_z stays within 2 GiB
    for T, V in ((7000, 152064), (16384, 152064), (100000, 152064), (1 << 22, 151936)):
        whole = tik.workspace_bytes(tik.OP_TOKEN_LOGPROB_BWD, T, H=256, V=V)
        assert whole <= (2 << 30) + T * 256 * 6 + 16 * T + (1 << 27)
    assert tik.workspace_bytes(tik.OP_POLICY_LOSS, 100, max_ctx=7) == 16 + 592 * 5 * 8 + 592 * 4
    assert tik.workspace_bytes(tik.OP_POLICY_LOSS, 100, max_ctx=1001) == 16 + 592 * 5 * 8 + 4016
