"""GPU parity of attention over parts of a long context with the float64 oracle
(oracle/reach.py): the window with its first slots and its gradients, the shared prefix, and the
weights slots receive.

Tolerances, per element. A score sums d products of size at most sigma = max sum |q k| / sqrt(d),
each addition off by half a step of fp32 (2^-24), so a weight is off by at most
ew = 2^-24 ((d + 12) sigma + 16) of itself (the scaling, the argument of the exponential and the
exponential itself in the 12 and the 16), its normaliser by as much, and a sum of n terms adds
n 2^-24 of their size S. fp32 results: (2 ew + (n + 4) 2^-24) S. bf16 results of few tokens
(T <= 4, weights with 24 bits) are rounded once more, 2^-8 |O|; of longer calls the weights are
bf16 too, each off by at most 2^-8, the normaliser with them: 2^-8 (2 |O| + S). Gradients: the
scores of dP and D add 2 (d + 12) 2^-24 to the terms' size, which the oracle sums in absolute
values."""
import numpy as np
import pytest
import torch

from oracle import reach
from tests.parity import wm  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _make(seed, L=3, B=2, T=1, Hq=2, Hkv=1, d=64, k=2, S=64, dtype="bf16", ctx=(0, 0), P=0,
          chan_map=None, peak=1.0):
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=g).to(dt)

    c = dict(L=L, B=B, T=T, Hq=Hq, Hkv=Hkv, d=d, k=k, S=S, dtype=dtype, ctx=list(ctx), P=P,
             map=chan_map or [l % k for l in range(L)])
    c.update(Q=(normal(L, B, Hq, T, d).float() * peak).to(dt), Kc=normal(k, B, Hkv, S, d),
             Vc=normal(k, B, Hkv, S, d), Kd=normal(k, Hkv, d), Vd=normal(k, Hkv, d))
    if P:
        c.update(Kp=normal(k, Hkv, P + 3, d), Vp=normal(k, Hkv, P + 3, d))
    return c


def _setup(wm, c, paper, gs=1, gq=0, ctx_max=None):
    dims = wm.make_dims(c["B"], c["T"], c["L"], c["k"], 64, c["Hq"], c["Hkv"], c["d"],
                        S_cap=c["S"], ctx_max=max(c["ctx"]) if ctx_max is None else ctx_max,
                        dtype=wm.BF16 if c["dtype"] == "bf16" else wm.F32, groups=gs, group=gq,
                        mask_mode=wm.MASK_PAPER if paper else wm.MASK_INCLUSIVE)
    t = {n: c[n].cuda() for n in ("Q", "Kc", "Vc", "Kd", "Vd", "Kp", "Vp") if n in c}
    none = torch.zeros(8, device="cuda", dtype=c["Q"].dtype)
    params = wm.ParamSet({n: t.get(n, none) for n in wm.PARAM_NAMES})
    ctx = torch.tensor(c["ctx"], dtype=torch.int32, device="cuda")
    O = torch.full((c["L"], c["B"], c["T"], c["Hq"] * c["d"]), float("nan"), device="cuda",
                   dtype=c["Q"].dtype)
    return dims, params, t, ctx, O


def _oracle(c, paper, gs=1, gq=0, window=None, sinks=0, **kw):
    if c["P"]:
        kw.update(Kp=c["Kp"][:, :, :c["P"]], Vp=c["Vp"][:, :, :c["P"]])
    return reach.attend(c["Q"], c["map"], c["ctx"], c["Kc"], c["Vc"], c["Kd"], c["Vd"], paper,
                        window, sinks, gs, gq, **kw)


def _ew(c, r):
    return U * ((c["d"] + 12) * r["sigma"] + 16)


def _close(got, want, tol, name):
    got = got.detach().cpu().double().numpy()
    assert np.isfinite(got).all(), name
    over = np.abs(got - want) - tol
    assert over.max() <= 0, "%s: off by %.3g past its bound of %.3g" % (
        name, over.max(), np.broadcast_to(tol, over.shape).reshape(-1)[over.argmax()])


def _close_out(c, r, O, name):
    n = max(c["ctx"]) + c["P"] + c["T"] + 1
    tol = (2 * _ew(c, r) + (n + 4) * U) * r["S"]
    if c["dtype"] == "bf16":
        a = np.abs(r["O"])
        tol = tol + (2.0 ** -8 * a if c["T"] <= 4 else 2.0 ** -8 * (2 * a + r["S"]))
    _close(O, r["O"], tol, name)


def _ws(wm, nbytes):
    """A workspace that held something else before."""
    return torch.full((max(nbytes, 256),), 0xFF, dtype=torch.uint8, device="cuda")


SHAPES = [("bf16", 64, 4, 2), ("bf16", 96, 6, 3), ("bf16", 32, 2, 1), ("f32", 64, 2, 2),
          ("f32", 32, 4, 2)]
# (T, ctx of two sequences, window, sinks)
WINDOWS = [(1, (0, 0), 1, 0), (1, (1, 700), 64, 4), (1, (90, 333), 500, 65), (2, (5, 300), 7, 1),
           (4, (63, 257), 33, 0), (1, (4000, 2011), 1000, 16), (3, (40, 41), 1000, 1000),
           (5, (0, 30), 1, 2), (33, (0, 100), 16, 0), (65, (200, 3), 64, 5), (130, (0, 0), 40, 1),
           (300, (77, 500), 129, 70), (200, (900, 0), 2000, 3), (257, (0, 64), 63, 64)]


@pytest.mark.parametrize("T,ctx,window,sinks", WINDOWS)
@pytest.mark.parametrize("dtype,d,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("paper", [True, False])
def test_window(wm, dtype, d, Hq, Hkv, T, ctx, window, sinks, paper):
    c = _make(1, T=T, Hq=Hq, Hkv=Hkv, d=d, S=max(ctx) + T + 5, dtype=dtype, ctx=ctx,
              chan_map=[1, 0, 1])
    print("window", dtype, d, T, ctx, window, sinks, paper, flush=True)
    r = _oracle(c, paper, window=window, sinks=sinks)
    # slots that no row of the call reads hold NaN: before the window, past the last row
    lim = np.array(ctx)[:, None] + (0 if paper else 1)
    slot = np.arange(c["S"])[None]
    dead = (slot >= lim + T - 1) | ((slot < lim - window) & (slot >= sinks))
    for n in ("Kc", "Vc"):
        c[n] = c[n].masked_fill(torch.from_numpy(dead)[None, :, None, :, None], float("nan"))
    dims, params, t, cl, O = _setup(wm, c, paper)
    wm.channel_attend_window(dims, params, t["Q"], c["map"], cl, window, sinks, t["Kc"], t["Vc"],
                             O, ws=_ws(wm, wm.workspace_size(dims, wm.OP_WINDOW_ATTEND)))
    torch.cuda.synchronize()
    _close_out(c, r, O, "O")


@pytest.mark.parametrize("gs,gq,T", [(4, 1, 40), (8, 7, 3), (3, 0, 70)])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 96), ("f32", 32)])
def test_window_of_a_strided_group(wm, dtype, d, gs, gq, T):
    c = _make(2, T=T, d=d, S=20 + gs * T, dtype=dtype, ctx=(20, 3))
    r = _oracle(c, True, gs, gq, window=50, sinks=2)
    dims, params, t, cl, O = _setup(wm, c, True, gs, gq)
    wm.channel_attend_window(dims, params, t["Q"], c["map"], cl, 50, 2, t["Kc"], t["Vc"], O)
    torch.cuda.synchronize()
    _close_out(c, r, O, "O")


@pytest.mark.parametrize("T", [1, 4, 100])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 96), ("f32", 64)])
def test_window_peaked_scores(wm, dtype, d, T):
    """One slot may outweigh every other by many powers of two, wherever it sits."""
    c = _make(3, T=T, d=d, S=400 + T, dtype=dtype, ctx=(400, 317), peak=12.0)
    r = _oracle(c, True, window=150, sinks=9)
    dims, params, t, cl, O = _setup(wm, c, True)
    wm.channel_attend_window(dims, params, t["Q"], c["map"], cl, 150, 9, t["Kc"], t["Vc"], O)
    torch.cuda.synchronize()
    _close_out(c, r, O, "O")


def test_whole_window_is_channel_attend(wm):
    """A window past the cache's end reads what wm_channel_attend reads."""
    c = _make(4, T=70, S=200, ctx=(100, 31))
    r = _oracle(c, True)
    dims, params, t, cl, O = _setup(wm, c, True)
    for window in (200, 2 ** 31 - 1):
        wm.channel_attend_window(dims, params, t["Q"], c["map"], cl, window, 0, t["Kc"], t["Vc"],
                                 O)
        torch.cuda.synchronize()
        _close_out(c, r, O, "O")


GRADS = [(1, (0, 5), 3, 0), (1, (100, 0), 1000, 4), (3, (7, 40), 20, 30), (40, (0, 0), 16, 2),
         (130, (0, 70), 64, 0), (300, (0, 0), 100, 5), (70, (130, 43), 4000, 0),
         (33, (500, 200), 65, 70)]


@pytest.mark.parametrize("T,ctx,window,sinks", GRADS)
@pytest.mark.parametrize("d,Hq,Hkv", [(64, 4, 2), (96, 6, 3), (64, 2, 2)])
@pytest.mark.parametrize("paper", [True, False])
def test_window_backward(wm, d, Hq, Hkv, T, ctx, window, sinks, paper):
    c = _make(5, L=5, k=3, T=T, Hq=Hq, Hkv=Hkv, d=d, S=max(ctx) + T + 7, ctx=ctx,
              chan_map=[2, 0, 2, 2, 0])
    print("window backward", d, T, ctx, window, sinks, paper, flush=True)
    g = torch.Generator().manual_seed(6)
    dO = torch.randn((5, 2, T, Hq * d), generator=g).bfloat16()
    O = torch.from_numpy(_oracle(c, paper, window=window, sinks=sinks)["O"]).bfloat16()
    r = _oracle(c, paper, window=window, sinks=sinks, dO=dO, O_given=O)
    dims, params, t, cl, _ = _setup(wm, c, paper)
    shapes = dict(dQ=t["Q"].shape, dKc=t["Kc"].shape, dVc=t["Vc"].shape, dKd=t["Kd"].shape,
                  dVd=t["Vd"].shape)
    out = {n: torch.full(s, float("nan"), device="cuda") for n, s in shapes.items()}
    args = (dims, params, t["Q"], c["map"], cl, window, sinks, t["Kc"], t["Vc"], O.cuda(),
            dO.cuda(), *out.values())
    ws = _ws(wm, wm.workspace_size(dims, wm.OP_WINDOW_BACKWARD))
    wm.channel_attend_window_backward(*args, ws=ws)
    torch.cuda.synchronize()
    first = {n: x.clone() for n, x in out.items()}
    n = 3 * (Hq // Hkv) * 2 * T + max(ctx) + T  # terms of the longest sum
    rel = 2 * _ew(c, r) + (n + 2 * (d + 12) + 8) * U
    for name, x in out.items():
        if name not in ("dKc", "dVc"):
            _close(x, r[name], rel * r[name + "_abs"], name)
            continue
        for b, c0 in enumerate(ctx):  # slots below ctx + T are written, the others left
            _close(x[:, b, :, :c0 + T], r[name][:, b, :, :c0 + T],
                   rel * r[name + "_abs"][:, b, :, :c0 + T], "%s of sequence %d" % (name, b))
            assert torch.isnan(x[:, b, :, c0 + T:]).all()
        assert not x[1, 0, :, :ctx[0] + T].any()  # channel 1 has no consumer
    wm.channel_attend_window_backward(*args, ws=ws)
    torch.cuda.synchronize()
    for name, x in out.items():  # fixed order of every sum
        assert torch.equal(x.nan_to_num(7.0), first[name].nan_to_num(7.0)), name


def test_window_backward_of_a_strided_group(wm):
    c = _make(7, T=40, d=64, S=150, ctx=(20, 3))
    dO = torch.randn((3, 2, 40, 128), generator=torch.Generator().manual_seed(8)).bfloat16()
    O = torch.from_numpy(_oracle(c, True, 3, 2, window=50, sinks=2)["O"]).bfloat16()
    r = _oracle(c, True, 3, 2, window=50, sinks=2, dO=dO, O_given=O)
    dims, params, t, cl, _ = _setup(wm, c, True, 3, 2)
    out = [torch.full(t[n].shape, float("nan"), device="cuda")
           for n in ("Q", "Kc", "Vc", "Kd", "Vd")]
    wm.channel_attend_window_backward(dims, params, t["Q"], c["map"], cl, 50, 2, t["Kc"], t["Vc"],
                                      O.cuda(), dO.cuda(), *out)
    torch.cuda.synchronize()
    rel = 2 * _ew(c, r) + (300 + 2 * 76 + 8) * U
    for name, x in zip(("dQ", "dKc", "dVc", "dKd", "dVd"), out):
        if x.dim() == 5 and name != "dQ":
            for b, c0 in enumerate(c["ctx"]):
                hi = c0 + 2 + 3 * 39 + 1
                _close(x[:, b, :, :hi], r[name][:, b, :, :hi], rel * r[name + "_abs"][:, b, :, :hi],
                       name)
                assert torch.isnan(x[:, b, :, hi:]).all()
        else:
            _close(x, r[name], rel * r[name + "_abs"], name)


# (T, ctx of three sequences, prefix)
PREFIXES = [(1, (0, 1, 2), 1), (1, (0, 30, 300), 64), (1, (5, 0, 77), 1111), (2, (0, 3, 90), 63),
            (4, (10, 200, 0), 130), (5, (0, 1, 2), 33), (37, (0, 50, 7), 65), (130, (40, 0, 3), 200),
            (1, (9, 8, 7), 0), (20, (9, 8, 7), 0)]


@pytest.mark.parametrize("T,ctx,P", PREFIXES)
@pytest.mark.parametrize("dtype,d,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("paper", [True, False])
def test_shared_prefix(wm, dtype, d, Hq, Hkv, T, ctx, P, paper):
    c = _make(9, B=3, T=T, Hq=Hq, Hkv=Hkv, d=d, S=max(ctx) + T + 5, dtype=dtype, ctx=ctx, P=P,
              chan_map=[1, 0, 1])
    print("shared", dtype, d, T, ctx, P, paper, flush=True)
    r = _oracle(c, paper)
    if P:  # past the prefix, and past the last row: anything
        c["Kp"][:, :, P:] = c["Vp"][:, :, P:] = float("nan")
    for b, c0 in enumerate(ctx):
        hi = c0 + T - (1 if paper else 0)
        c["Kc"][:, b, :, hi:] = c["Vc"][:, b, :, hi:] = float("nan")
    dims, params, t, cl, O = _setup(wm, c, paper)
    wm.channel_attend_shared(dims, params, t["Q"], c["map"], cl, P, t.get("Kp"), t.get("Vp"),
                             t["Kc"], t["Vc"], O, ws=_ws(wm, wm.shared_workspace(dims, P)))
    torch.cuda.synchronize()
    _close_out(c, r, O, "O")


@pytest.mark.parametrize("T,Hq,Hkv,d", [(1, 6, 3, 96), (3, 4, 2, 64)])
def test_shared_prefix_of_many_rows(wm, T, Hq, Hkv, d):
    """More rows per prefix slice than one tile holds: 40 sequences x 2 consumers x 2 heads."""
    ctx = [(7 * b) % 60 for b in range(40)]
    c = _make(10, L=4, B=40, T=T, Hq=Hq, Hkv=Hkv, d=d, S=70, ctx=ctx, P=777)
    r = _oracle(c, True)
    dims, params, t, cl, O = _setup(wm, c, True)
    wm.channel_attend_shared(dims, params, t["Q"], c["map"], cl, 777, t["Kp"], t["Vp"], t["Kc"],
                             t["Vc"], O)
    torch.cuda.synchronize()
    _close_out(c, r, O, "O")


WEIGHS = [(1, (0, 1)), (1, (64, 333)), (1, (2500, 3001)), (3, (40, 700)), (4, (0, 5)), (5, (0, 20)),
          (64, (0, 0)), (130, (33, 500)), (300, (0, 1))]


@pytest.mark.parametrize("T,ctx", WEIGHS)
@pytest.mark.parametrize("dtype,d,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("paper", [True, False])
def test_weigh(wm, dtype, d, Hq, Hkv, T, ctx, paper):
    c = _make(11, L=5, k=3, T=T, Hq=Hq, Hkv=Hkv, d=d, S=max(ctx) + T + 5, dtype=dtype, ctx=ctx,
              chan_map=[2, 0, 2, 2, 0])
    print("weigh", dtype, d, T, ctx, paper, flush=True)
    r = _oracle(c, paper)
    dims, params, t, cl, O = _setup(wm, c, paper)
    before = torch.rand((3, 2, Hkv, c["S"]), generator=torch.Generator().manual_seed(12))
    for b, c0 in enumerate(ctx):
        before[:, b, :, c0 + T:] = float("nan")  # slots no row reads are left as they are
    weight = before.cuda()
    wm.channel_attend_weigh(dims, params, t["Q"], c["map"], cl, t["Kc"], t["Vc"], O, weight,
                            ws=_ws(wm, wm.workspace_size(dims, wm.OP_WEIGH_ATTEND)))
    torch.cuda.synchronize()
    _close_out(c, r, O, "O")
    n = 3 * (Hq // Hkv) * T + max(ctx) + T  # a slot's rows, and a row's slots in its normaliser
    w0 = before.double().numpy()
    for b, c0 in enumerate(ctx):
        hi = c0 + T
        want = w0[:, b, :, :hi] + r["weight"][:, b, :, :hi]
        _close(weight[:, b, :, :hi], want, (2 * _ew(c, r) + (n + 4) * U) *
               r["weight"][:, b, :, :hi] + U * np.abs(want), "weight of sequence %d" % b)
        assert torch.isnan(weight[:, b, :, hi:]).all()
    assert torch.equal(weight[1, 0, :, :ctx[0] + T].cpu(), before[1, 0, :, :ctx[0] + T])
