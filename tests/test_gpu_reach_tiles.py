"""The long-context calls where tests/test_gpu_reach.py's small grids do not lead: enough rows for
the 128-row tiles (and more of them than workgroups, so that they come from the queue), strided
groups, peaked scores and infinite or NaN slots behind the last row in the shared and weighed calls.
Bounds as derived there."""
import numpy as np
import pytest
import torch

from tests.parity import wm  # noqa: F401
from tests.test_gpu_reach import U, _close, _close_out, _ew, _make, _oracle, _setup, _ws

pytestmark = pytest.mark.gpu


def _bury(c, paper, gs=1, gq=0):
    """The slots that no row reads (behind each sequence's last row) hold NaN and infinities."""
    for b, c0 in enumerate(c["ctx"]):
        hi = c0 + gq + gs * (c["T"] - 1) + (0 if paper else 1)
        c["Kc"][:, b, :, hi:] = float("nan")
        c["Vc"][:, b, :, hi:] = float("inf")


def _many(T, ctx, d, seed=30, **kw):
    """384 heads: up to 512 tiles of 128 rows of at most 128 tokens, twice as many of up to 256."""
    return _make(seed, L=8, B=4, T=T, Hq=12, Hkv=4, d=d, k=3, S=max(ctx) + T + 9, ctx=ctx,
                 chan_map=[2, 0, 2, 1, 1, 0, 2, 0], **kw)


@pytest.mark.parametrize("T,ctx,window,sinks", [
    (65, (0, 40, 300, 901), 50, 4),      # a gap between the first slots and the windows
    (128, (0, 7, 700, 64), 130, 65),     # ... of more first slots than a block of 64 holds
    (130, (0, 500, 33, 260), 64, 0),     # from the queue, no first slots
    (255, (3, 0, 611, 64), 100, 33)])
@pytest.mark.parametrize("d", [64, 96])
@pytest.mark.parametrize("paper", [True, False])
def test_window_tiles(wm, d, T, ctx, window, sinks, paper):
    c = _many(T, ctx, d)
    print("window tiles", d, T, ctx, window, sinks, paper, flush=True)
    r = _oracle(c, paper, window=window, sinks=sinks)
    _bury(c, paper)
    dims, params, t, cl, O = _setup(wm, c, paper)
    for _ in range(2):  # the queue starts anew at every call
        wm.channel_attend_window(dims, params, t["Q"], c["map"], cl, window, sinks, t["Kc"],
                                 t["Vc"], O, ws=_ws(wm, wm.workspace_size(dims, wm.OP_WINDOW_ATTEND)))
        torch.cuda.synchronize()
        _close_out(c, r, O, "O")


@pytest.mark.parametrize("T,ctx,P", [(65, (0, 40, 3, 90), 64), (128, (0, 7, 70, 64), 333),
                                     (130, (50, 0, 33, 26), 1), (255, (3, 0, 11, 64), 129)])
@pytest.mark.parametrize("d", [64, 96])
@pytest.mark.parametrize("paper", [True, False])
def test_shared_tiles(wm, d, T, ctx, P, paper):
    c = _many(T, ctx, d, seed=31, P=P)
    print("shared tiles", d, T, ctx, P, paper, flush=True)
    r = _oracle(c, paper)
    c["Kp"][:, :, P:] = c["Vp"][:, :, P:] = float("nan")
    _bury(c, paper)
    dims, params, t, cl, O = _setup(wm, c, paper)
    wm.channel_attend_shared(dims, params, t["Q"], c["map"], cl, P, t["Kp"], t["Vp"], t["Kc"],
                             t["Vc"], O, ws=_ws(wm, wm.shared_workspace(dims, P)))
    torch.cuda.synchronize()
    _close_out(c, r, O, "O")


def _weigh(wm, c, paper, gs=1, gq=0):
    r = _oracle(c, paper, gs, gq)
    _bury(c, paper, gs, gq)
    dims, params, t, cl, O = _setup(wm, c, paper, gs, gq)
    weight = torch.zeros((c["k"], c["B"], c["Hkv"], c["S"]), device="cuda")
    wm.channel_attend_weigh(dims, params, t["Q"], c["map"], cl, t["Kc"], t["Vc"], O, weight,
                            ws=_ws(wm, wm.workspace_size(dims, wm.OP_WEIGH_ATTEND)))
    torch.cuda.synchronize()
    _close_out(c, r, O, "O")
    rows = max(c["map"].count(x) for x in c["map"]) * (c["Hq"] // c["Hkv"]) * c["T"]
    n = rows + max(c["ctx"]) + gs * c["T"]  # a slot's rows, and a row's slots in its normaliser
    _close(weight, r["weight"], (2 * _ew(c, r) + (n + 5) * U) * r["weight"], "weight")


@pytest.mark.parametrize("T,ctx", [(65, (0, 40, 300, 201)), (128, (0, 7, 70, 64)),
                                   (255, (3, 0, 111, 64))])
@pytest.mark.parametrize("d", [64, 96])
@pytest.mark.parametrize("paper", [True, False])
def test_weigh_tiles(wm, d, T, ctx, paper):
    print("weigh tiles", d, T, ctx, paper, flush=True)
    _weigh(wm, _many(T, ctx, d, seed=32), paper)


GROUPS = [(4, 1, 40), (8, 7, 3), (3, 0, 70), (5, 2, 1)]
KINDS = [("bf16", 64), ("bf16", 96), ("bf16", 32), ("f32", 64), ("f32", 32)]


@pytest.mark.parametrize("gs,gq,T", GROUPS)
@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("paper", [True, False])
def test_weigh_of_a_strided_group(wm, dtype, d, gs, gq, T, paper):
    print("weigh group", dtype, d, gs, gq, T, paper, flush=True)
    _weigh(wm, _make(33, T=T, d=d, S=60 + gs * T + 3, dtype=dtype, ctx=(60, 5)), paper, gs, gq)


@pytest.mark.parametrize("gs,gq,T", GROUPS)
@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("paper", [True, False])
def test_shared_of_a_strided_group(wm, dtype, d, gs, gq, T, paper):
    c = _make(34, T=T, d=d, S=60 + gs * T + 3, dtype=dtype, ctx=(60, 5), P=90)
    print("shared group", dtype, d, gs, gq, T, paper, flush=True)
    r = _oracle(c, paper, gs, gq)
    _bury(c, paper, gs, gq)
    dims, params, t, cl, O = _setup(wm, c, paper, gs, gq)
    wm.channel_attend_shared(dims, params, t["Q"], c["map"], cl, 90, t["Kp"], t["Vp"], t["Kc"],
                             t["Vc"], O)
    torch.cuda.synchronize()
    _close_out(c, r, O, "O")


@pytest.mark.parametrize("T", [1, 4, 100])
@pytest.mark.parametrize("dtype,d", KINDS)
def test_peaked_scores(wm, dtype, d, T):
    """One slot may outweigh every other by many powers of two, in the prefix or behind it."""
    c = _make(35, T=T, d=d, S=200 + T, dtype=dtype, ctx=(200, 17), P=333, peak=12.0)
    print("peaked", dtype, d, T, flush=True)
    r = _oracle(c, True)
    dims, params, t, cl, O = _setup(wm, c, True)
    wm.channel_attend_shared(dims, params, t["Q"], c["map"], cl, 333, t["Kp"], t["Vp"], t["Kc"],
                             t["Vc"], O)
    torch.cuda.synchronize()
    _close_out(c, r, O, "O")
    _weigh(wm, _make(36, T=T, d=d, S=200 + T, dtype=dtype, ctx=(200, 17), peak=12.0), True)


@pytest.mark.parametrize("T", [1, 3, 40])
@pytest.mark.parametrize("d", [64, 96])
def test_shared_scores_far_below_zero(wm, d, T):
    """Every score of the prefix, or every own one, so low that exp of it alone is zero in fp32."""
    for low in ("Kp", "Kc"):
        c = _make(37, T=T, d=d, S=90 + T, ctx=(90, 64), P=130)
        c["Q"] = c["Q"].abs() + 0.5
        c[low] = -16 * c[low].abs() - 2
        print("low", low, d, T, flush=True)
        for paper in (False, True):
            r = _oracle(c, paper)
            dims, params, t, cl, O = _setup(wm, c, paper)
            wm.channel_attend_shared(dims, params, t["Q"], c["map"], cl, 130, t["Kp"], t["Vp"],
                                     t["Kc"], t["Vc"], O)
            torch.cuda.synchronize()
            _close_out(c, r, O, "O")


@pytest.mark.parametrize("dtype,d,T,ctx,P", [
    ("bf16", 64, 5, 40, 1400), ("bf16", 96, 8, 0, 1500), ("bf16", 64, 16, 33, 2200),
    ("f32", 64, 5, 40, 700), ("f32", 32, 16, 0, 830), ("bf16", 32, 8, 30, 550)])
@pytest.mark.parametrize("paper", [True, False])
def test_batch_of_short_questions(wm, dtype, d, T, ctx, P, paper):
    """So many heads over so long a prefix that the batch's rows of 5 to 16 tokens meet it
    together."""
    B = 16
    c = _make(39, L=12, B=B, T=T, Hq=12, Hkv=6, d=d, k=4, S=ctx + T + 2, dtype=dtype, P=P,
              ctx=[ctx * b // (B - 1) for b in range(B)])
    print("questions", dtype, d, T, ctx, P, paper, flush=True)
    assert 12 * B * 12 * P * (32 - T) >= (80e6 if dtype == "bf16" and d != 32 else 30e6)
    r = _oracle(c, paper)
    c["Kp"][:, :, P:] = c["Vp"][:, :, P:] = float("nan")
    _bury(c, paper)
    dims, params, t, cl, O = _setup(wm, c, paper)
    wm.channel_attend_shared(dims, params, t["Q"], c["map"], cl, P, t["Kp"], t["Vp"], t["Kc"],
                             t["Vc"], O, ws=_ws(wm, wm.shared_workspace(dims, P)))
    torch.cuda.synchronize()
    _close_out(c, r, O, "O")


def test_prefix_alone(wm):
    """Sequences with nothing of their own: in the paper's mask a first token reads the prefix
    and the dummy only."""
    for T, dtype, d in ((1, "bf16", 64), (1, "bf16", 96), (1, "f32", 32), (6, "bf16", 64)):
        c = _make(38, T=T, d=d, S=T, dtype=dtype, ctx=(0, 0), P=65)
        r = _oracle(c, True)
        _bury(c, True)
        dims, params, t, _, O = _setup(wm, c, True)
        wm.channel_attend_shared(dims, params, t["Q"], c["map"], None, 65, t["Kp"], t["Vp"],
                                 t["Kc"], t["Vc"], O)
        torch.cuda.synchronize()
        _close_out(c, r, O, "O of %d tokens" % T)
        if T == 1:
            assert np.isfinite(O.float().cpu().numpy()).all()
