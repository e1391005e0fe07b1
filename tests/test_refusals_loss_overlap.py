"""Which tensors of a policy loss may share memory, asked of the C interface through a stand-in context.  Every call lacks its workspace, which is
asked for last: one that is not refused for an overlap is refused for that, and nothing is ever queued."""
import ctypes
import itertools

import pytest

from paper_2609_35140_b200 import binding as tik

OK, INVALID, WORKSPACE = 0, -1, -3
T, S = 40, 3
NAMES = ("lp", "old", "adv", "weight", "ref", "cu", "loss", "d", "stats")
AT = {name: (i + 1) << 20 for i, name in enumerate(NAMES)}        # addresses that nothing reads


@pytest.fixture(scope="module")
def ctx():
    lib = tik.load()
    lib.tik_selftest_context.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]
    c = ctypes.c_void_p()
    assert lib.tik_selftest_context(ctypes.byref(c), 148) == OK
    yield c
    lib.tik_destroy(c)


def ask(ctx, per=0, tokens=T, **at):
    a = dict(AT, **at)
    return tik.load().tik_policy_loss(ctx, a["lp"], a["old"], a["adv"], per, a["weight"], a["ref"], a["cu"], S, tokens, 0.2, 0.2, 0.0, 0.1, 1, 1.0, a["loss"],
                                      a["d"], a["stats"], None, 0, None)


@pytest.mark.parametrize("per", [0, 1])
@pytest.mark.parametrize("out", ["loss", "d", "stats"])
@pytest.mark.parametrize("other", NAMES)
def test_overlap_rule_against_all_places(ctx, out, other, per):
    if out == other:
        return
    sizes = dict(lp=T, old=T, adv=S if per else T, weight=T, ref=T, cu=S + 1, loss=1, d=T, stats=5)
    for shift in range(-2 * T, 2 * T + 1):
        place = AT[other] + 4 * shift
        refused = shift < sizes[other] and -shift < sizes[out]
        if out == "d" and shift == 0 and (other in ("lp", "old", "weight", "ref") or (other == "adv" and not per)):
            refused = False                                # the gradient in place of an input
        assert ask(ctx, per, **{out: place}) == (INVALID if refused else WORKSPACE), shift


def test_in_place_beside_a_shifted_view(ctx):
    assert ask(ctx, d=AT["lp"], old=AT["lp"]) == WORKSPACE         # two inputs may be one
    assert ask(ctx, d=AT["lp"], old=AT["lp"] + 4) == INVALID
    for a, b in itertools.combinations(("lp", "old", "adv", "weight", "ref"), 2):
        assert ask(ctx, **{b: AT[a] + 8}) == WORKSPACE             # inputs may overlap as they like


def test_absent_tensors_and_no_tokens(ctx):
    assert ask(ctx, d=None, stats=None) == WORKSPACE
    assert ask(ctx, tokens=0, d=AT["lp"] + 4) == WORKSPACE
    assert ask(ctx, tokens=0, loss=AT["lp"], stats=AT["old"]) == WORKSPACE
    assert ask(ctx, tokens=0, loss=AT["stats"] + 16) == INVALID
