"""The long-context calls as programs use them: a prefix shared by sequences that go on with the
library's own projections, decoding that weighs its slots, evicts and goes on, captured graphs
replayed between eager work, two streams at once, caches past 2^31 elements, context lengths past
their bound.

fp32 throughout where results are compared with float64: a chain's caches are read back, so each
call is held to its own bound (the module test_gpu_reach derives it)."""
import numpy as np
import pytest
import torch

from oracle import reach
from tests import synth
from tests.parity import _bias, _dev, wm  # noqa: F401
from tests.test_gpu_reach import U, _close, _close_out, _ew, _make, _oracle, _setup

pytestmark = pytest.mark.gpu
THETA = 1e6


def _model(wm, B, S, T, ctx_max, dtype="f32"):
    """A small model's dims, parameters and map; d = 64, 4 layers, 2 channels, 4 / 2 heads."""
    w = synth.small("reach_use", B=B, T_new=T, L=4, k=2, D=64, Hq=4, Hkv=2, d=64, ctx=S - T,
                    dtype=dtype)
    P = wm.ParamSet(_dev(synth.make_params(w, _bias(w))))

    def dims(T, S, ctx_max, B=B):
        return wm.make_dims(B, T, 4, 2, 64, 4, 2, 64, S_cap=S, ctx_max=ctx_max,
                            dtype=wm.F32 if dtype == "f32" else wm.BF16, rope_theta=THETA)
    return P, dims, [0, 1, 0, 1]


def _case(params, cmap, Q, Kc, Vc, ctx, **more):
    """What tests.test_gpu_reach's checks read, of tensors that a chain made."""
    L, B, Hq, T, d = Q.shape
    c = dict(L=L, B=B, T=T, Hq=Hq, Hkv=Kc.shape[2], d=d, k=2, S=Kc.shape[3], dtype="f32",
             ctx=list(ctx), P=0, map=cmap, Q=Q.cpu(), Kc=Kc.cpu(), Vc=Vc.cpu(),
             Kd=params.tensors["Kd"].cpu(), Vd=params.tensors["Vd"].cpu())
    c.update(more)
    return c


def test_sequences_that_share_a_prefix(wm):
    """A prompt's cache laid out once; three sequences pool their own tokens at positions from 0
    and attend both. The same as attention over the whole: the same tokens pooled behind copies of
    the prompt, positions from the prompt's end, which the shared call sees only through RoPE's
    relative positions (and a dummy turned to match). Keys and queries of either run are off by
    their fp32 rounding and by the angle's (2^-21), of their size: scores by 6 2^-21 sigma more
    than a call's own bound."""
    n, own, T = 77, 40, 5
    P, dims, cmap = _model(wm, 3, 128, T, 100)
    g = torch.Generator().manual_seed(1)
    prompt = torch.randn((1, n, 4, 64), generator=g).cuda()
    H0 = torch.randn((3, own, 4, 64), generator=g).cuda()
    H1 = torch.randn((3, T, 4, 64), generator=g).cuda()
    f32 = dict(device="cuda", dtype=torch.float32)
    K1, V1 = (torch.zeros((2, 1, 2, n, 64), **f32) for _ in range(2))
    wm.pool(dims(n, n, 0, B=1), P, prompt, None, K1, V1)
    Kp, Vp = (torch.empty((2, 2, n + 3, 64), **f32) for _ in range(2))
    Kd = torch.empty_like(P.tensors["Kd"])
    wm.prefix_share(dims(0, n, n, B=1), K1, V1, 0, n, Kp, Vp, Kd=P.tensors["Kd"], Kd_out=Kd)
    Ps = wm.ParamSet({**P.tensors, "Kd": Kd})

    def run(start):
        """Own tokens behind `start` slots: queries of the new ones, caches, context lengths."""
        S = start + own + T
        Kc, Vc = (torch.zeros((2, 3, 2, S, 64), **f32) for _ in range(2))
        if start:
            Kc[..., :start, :], Vc[..., :start, :] = K1, V1
        c0 = torch.full((3,), start, dtype=torch.int32, device="cuda")
        c1 = c0 + own
        wm.pool(dims(own, S, start), P, H0, c0, Kc, Vc)
        d1 = dims(T, S, start + own)
        wm.pool(d1, P, H1, c1, Kc, Vc)
        Q = torch.empty((4, 3, 4, T, 64), **f32)
        wm.q_project(d1, P, H1, c1, Q)
        return d1, Q, Kc, Vc, c1

    d1, Q, Kc, Vc, c1 = run(0)
    O = torch.empty((4, 3, T, 256), **f32)
    wm.channel_attend_shared(d1, Ps, Q, cmap, c1, n, Kp, Vp, Kc, Vc, O)
    d2, Q2, K2, V2, c2 = run(n)
    O2 = torch.empty_like(O)
    wm.channel_attend(d2, P, Q2, cmap, c2, K2, V2, O2)
    torch.cuda.synchronize()
    c = _case(Ps, cmap, Q, Kc, Vc, [own] * 3, P=n, Kp=Kp.cpu(), Vp=Vp.cpu())
    r = _oracle(c, True)
    _close_out(c, r, O, "shared")
    tol = 2 * (2 * _ew(c, r) + (n + own + T) * U) + 2 * 6 * 2.0 ** -21 * r["sigma"]
    _close(O2, O.cpu().double().numpy(), tol * r["S"], "whole and shared")


def test_decode_weigh_evict_and_go_on(wm):
    """Tokens decoded one by one with their weights added up; the caches cut to 24 slots; more
    tokens appended by wm_pool at the new positions, read whole and through a window."""
    B, S, keep = 2, 64, 24
    P, dims, cmap = _model(wm, B, S, 1, S - 1)
    g = torch.Generator().manual_seed(2)
    f32 = dict(device="cuda", dtype=torch.float32)
    Kc, Vc = (torch.full((2, B, 2, S, 64), float("nan"), **f32) for _ in range(2))
    H = torch.randn((B, 40, 4, 64), generator=g).cuda()
    c0 = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    Kc[:, 1, :, :5], Vc[:, 1, :, :5] = torch.randn((2, 2, 2, 5, 64), generator=g).cuda()
    wm.pool(dims(40, S, 5), P, H, c0, Kc, Vc)
    weight = torch.zeros((2, B, 2, S), **f32)
    ctx, want = [40, 45], np.zeros((2, B, 2, S))
    Q, O = torch.empty((4, B, 4, 1, 64), **f32), torch.empty((4, B, 1, 256), **f32)

    def token(Kc, Vc, weight, ctx, S):
        h = torch.randn((B, 1, 4, 64), generator=g).cuda()
        d = dims(1, S, max(ctx))
        at = torch.tensor(ctx, dtype=torch.int32, device="cuda")
        wm.q_project(d, P, h, at, Q)
        wm.channel_attend_weigh(d, P, Q, cmap, at, Kc, Vc, O, weight)
        torch.cuda.synchronize()
        c = _case(P, cmap, Q, Kc, Vc, ctx)
        r = _oracle(c, True)
        _close_out(c, r, O, "weighed token")
        win = torch.empty_like(O)
        wm.channel_attend_window(d, P, Q, cmap, at, 7, 2, Kc, Vc, win)
        _close_out(c, _oracle(c, True, window=7, sinks=2), win, "window over the same cache")
        wm.pool(d, P, h, at, Kc, Vc)
        return r["weight"], _ew(c, r)

    off = 0.0
    for _ in range(6):
        w, ew = token(Kc, Vc, weight, ctx, S)
        want, off = want + w, max(off, 2 * ew)
        ctx = [n + 1 for n in ctx]
    torch.cuda.synchronize()
    _close(weight, want, (off + (max(ctx) + 4 + 6) * U) * want, "accumulated weight")
    So = 40
    Ko, Vo = (torch.full((2, B, 2, So, 64), float("nan"), **f32) for _ in range(2))
    wo, co = torch.empty((2, B, 2, So), **f32), torch.empty(B, dtype=torch.int32, device="cuda")
    kept = torch.empty((2, B, 2, keep), dtype=torch.int32, device="cuda")
    wm.cache_evict(dims(0, S, max(ctx)), torch.tensor(ctx, dtype=torch.int32, device="cuda"),
                   keep, 2, 8, weight, Kc, Vc, co, wo, Ko, Vo, kept=kept)
    torch.cuda.synchronize()
    assert co.tolist() == [keep, keep]
    wh = weight.cpu().double().numpy()
    for ch in range(2):
        for b in range(B):
            for h in range(2):
                slots = reach.evict_slots(wh[ch, b, h], ctx[b], keep, 2, 8)
                assert kept[ch, b, h].tolist() == slots
                x = Kc[ch, b, h, slots].cpu().double().numpy()
                _close(Ko[ch, b, h, :keep], reach.turn(x, np.arange(keep) - np.array(slots), THETA),
                       2.0 ** -20 * (np.abs(x) + np.abs(np.roll(x, 32, 1))) + 1e-30, "moved keys")
    ctx = [keep, keep]
    for _ in range(3):  # the weights go on adding up in the new cache
        token(Ko, Vo, wo, ctx, So)
        ctx = [n + 1 for n in ctx]


def _calls(wm, seed=20, B=2):
    """name -> (call, outputs): one call of every kind on buffers of its own."""
    got = {}
    for T in (1, 70):
        c = _make(seed + T, B=B, T=T, Hq=4, Hkv=2, d=64, S=300 + T, ctx=[300, 120][:B], P=100)
        dims, P, t, cl, O = _setup(wm, c, True)

        def window(dims=dims, P=P, t=t, cl=cl, O=O, c=c,
                   ws=wm.workspace(dims, wm.OP_WINDOW_ATTEND)):
            wm.channel_attend_window(dims, P, t["Q"], c["map"], cl, 64, 4, t["Kc"], t["Vc"], O, ws=ws)
        got["window%d" % T] = (window, [O])
        O2 = torch.empty_like(O)

        def shared(dims=dims, P=P, t=t, cl=cl, O=O2, c=c,
                   ws=torch.empty(wm.shared_workspace(dims, 100), dtype=torch.uint8, device="cuda")):
            wm.channel_attend_shared(dims, P, t["Q"], c["map"], cl, 100, t["Kp"], t["Vp"], t["Kc"],
                                     t["Vc"], O, ws=ws)
        got["shared%d" % T] = (shared, [O2])
        O3, w = torch.empty_like(O), torch.empty((2, B, 2, c["S"]), device="cuda")

        def weigh(dims=dims, P=P, t=t, cl=cl, O=O3, w=w, c=c,
                  ws=wm.workspace(dims, wm.OP_WEIGH_ATTEND)):
            w.zero_()
            wm.channel_attend_weigh(dims, P, t["Q"], c["map"], cl, t["Kc"], t["Vc"], O, w, ws=ws)
        got["weigh%d" % T] = (weigh, [O3, w])
        O4 = torch.randn(O.shape, device="cuda").to(O.dtype)
        out = [torch.zeros(t[n].shape, device="cuda") for n in ("Q", "Kc", "Vc", "Kd", "Vd")]

        def grad(dims=dims, P=P, t=t, cl=cl, O=O4, c=c, out=out,
                 ws=wm.workspace(dims, wm.OP_WINDOW_BACKWARD)):
            wm.channel_attend_window_backward(dims, P, t["Q"], c["map"], cl, 64, 40, t["Kc"],
                                              t["Vc"], O, O, *out, ws=ws)
        got["grad%d" % T] = (grad, out)
        if T == 1:
            Ko, Vo = (torch.zeros((2, B, 2, 100, 64), device="cuda", dtype=O.dtype)
                      for _ in range(2))
            wt = torch.rand((2, B, 2, c["S"]), device="cuda")
            wo, co = torch.empty((2, B, 2, 100), device="cuda"), torch.empty_like(cl)

            def evict(dims=dims, t=t, cl=cl, wt=wt, wo=wo, co=co, Ko=Ko, Vo=Vo,
                      ws=wm.workspace(dims, wm.OP_CACHE_EVICT)):
                wm.cache_evict(dims, cl, 90, 3, 20, wt, t["Kc"], t["Vc"], co, wo, Ko, Vo, ws=ws)
            got["evict"] = (evict, [Ko, Vo, wo, co])
            Kq, Vq = (torch.zeros((2, 2, 64, 64), device="cuda", dtype=O.dtype) for _ in range(2))

            def share(dims=dims, t=t, Kp=Kq, Vp=Vq):
                wm.prefix_share(dims, t["Kc"], t["Vc"], B - 1, 60, Kp, Vp)
            got["share"] = (share, [Kq, Vq])
    return got


def test_captured_and_replayed(wm):
    """Every call captured into a graph of its own; replays between eager work on other inputs and
    synchronisations give the eager result bit for bit."""
    calls = _calls(wm)
    side = torch.cuda.Stream()
    for name, (call, outs) in calls.items():
        print("capture", name, flush=True)
        call()
        torch.cuda.synchronize()
        want = [x.clone() for x in outs]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            call()
        side.synchronize()
        with torch.cuda.graph(g):
            call()
        for i in range(4):
            for x in outs:
                x.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), (name, i)
            torch.randn(1 << 16, device="cuda").sum().item()  # the program's own work
            call()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), (name, i)


def test_two_streams(wm):
    """Calls on two streams, each with its own buffers, interleaved without waiting."""
    a, b = _calls(wm, 20), _calls(wm, 40)
    want = []
    for calls in (a, b):
        for call, _ in calls.values():
            call()
        torch.cuda.synchronize()
        want.append({n: [x.clone() for x in outs] for n, (_, outs) in calls.items()})
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for name in a:
            for calls, s in zip((a, b), streams):
                with torch.cuda.stream(s):
                    calls[name][0]()
    torch.cuda.synchronize()
    for calls, w in zip((a, b), want):
        for n, (_, outs) in calls.items():
            assert all(torch.equal(x, y) for x, y in zip(outs, w[n])), n


def test_context_past_its_bound_acts_as_the_bound(wm):
    """A ctx_len entry past ctx_max (or negative) reads and writes inside the buffers; the other
    sequences keep their results."""
    for T in (1, 40):
        c = _make(50, B=3, T=T, Hq=2, Hkv=2, d=64, S=200 + T, ctx=(100, 100, 60), P=50)
        dims, P, t, cl, O = _setup(wm, c, True, ctx_max=100)
        wild = torch.tensor([2 ** 31 - 1, -5, 60], dtype=torch.int32, device="cuda")
        tame = torch.tensor([100, 0, 60], dtype=torch.int32, device="cuda")
        res = []
        for cl in (tame, wild):
            w = torch.zeros((2, 3, 2, c["S"]), device="cuda")
            outs = [torch.empty_like(O) for _ in range(3)]
            wm.channel_attend_window(dims, P, t["Q"], c["map"], cl, 30, 4, t["Kc"], t["Vc"], outs[0])
            wm.channel_attend_shared(dims, P, t["Q"], c["map"], cl, 50, t["Kp"], t["Vp"], t["Kc"],
                                     t["Vc"], outs[1])
            wm.channel_attend_weigh(dims, P, t["Q"], c["map"], cl, t["Kc"], t["Vc"], outs[2], w)
            Ko, Vo = (torch.zeros((2, 3, 2, 64, 64), device="cuda", dtype=O.dtype) for _ in range(2))
            wo, co = torch.empty((2, 3, 2, 64), device="cuda"), torch.empty_like(cl)
            wm.cache_evict(dims, cl, 64, 1, 9, w, t["Kc"], t["Vc"], co, wo, Ko, Vo)
            torch.cuda.synchronize()
            res.append([*outs, w, Ko, Vo, wo, co])
        assert all(torch.equal(x, y) for x, y in zip(*res))


def test_caches_past_32_bits(wm):
    """2.7 billion elements a cache: the last sequence's slices lie past every 32-bit offset."""
    k, B, Hkv, d, S, n = 1, 40, 8, 64, 131072, 131000
    g = torch.Generator(device="cuda").manual_seed(3)
    Kc, Vc = (torch.zeros((k, B, Hkv, S, d), device="cuda", dtype=torch.bfloat16)
              for _ in range(2))
    for x in (Kc, Vc):
        x[:, -1].normal_(generator=g)
    weight = torch.zeros((k, B, Hkv, S), device="cuda")
    weight[:, -1].uniform_(generator=g)
    dims = wm.make_dims(B, 1, 1, k, 64, Hkv, Hkv, d, S_cap=S, ctx_max=n, dtype=wm.BF16,
                        rope_theta=THETA)
    ctx = torch.tensor([1] * (B - 1) + [n], dtype=torch.int32, device="cuda")
    Q = torch.randn((1, B, Hkv, 1, d), generator=torch.Generator().manual_seed(4)).bfloat16()
    Kd = torch.randn((1, Hkv, d), generator=torch.Generator().manual_seed(5)).bfloat16()
    P = wm.ParamSet({m: Kd.cuda() for m in wm.PARAM_NAMES})
    O = torch.empty((1, B, 1, Hkv * d), device="cuda", dtype=torch.bfloat16)
    wm.channel_attend_window(dims, P, Q.cuda(), [0], ctx, 500, 3, Kc, Vc, O)
    torch.cuda.synchronize()
    # the slots that the last sequence reads, as a cache of its own
    slots = [0, 1, 2, *range(n - 500, n)]
    c = dict(L=1, B=1, T=1, Hq=Hkv, Hkv=Hkv, d=d, k=1, S=503, dtype="bf16", ctx=[503], P=0, map=[0],
             Q=Q[:, -1:], Kc=Kc[:, -1:, :, slots].cpu(), Vc=Vc[:, -1:, :, slots].cpu(), Kd=Kd, Vd=Kd)
    _close_out(c, _oracle(c, True), O[:, -1:], "last sequence")
    keep = 256
    Ko, Vo = (torch.zeros((k, B, Hkv, keep, d), device="cuda", dtype=torch.bfloat16)
              for _ in range(2))
    wo, co = torch.empty((k, B, Hkv, keep), device="cuda"), torch.empty_like(ctx)
    kept = torch.empty((k, B, Hkv, keep), device="cuda", dtype=torch.int32)
    wm.cache_evict(dims, ctx, keep, 2, 100, weight, Kc, Vc, co, wo, Ko, Vo, kept=kept)
    torch.cuda.synchronize()
    for h in (0, Hkv - 1):
        want = reach.evict_slots(weight[0, -1, h].cpu().double().numpy(), n, keep, 2, 100)
        assert kept[0, -1, h].tolist() == want
        assert torch.equal(Vo[0, -1, h], Vc[0, -1, h, want])
        assert torch.equal(wo[0, -1, h], weight[0, -1, h, want])
