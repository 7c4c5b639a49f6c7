"""Host-side checks of the long-context calls (no GPU needed): every refusal comes back with its
code before anything is launched, and nothing is asked of empty calls."""
import ctypes

import pytest
import torch

from tests.test_boundary import wm  # noqa: F401


def _dims(wm, **kw):
    base = dict(B=2, T_new=3, L=4, k=2, D=64, Hq=4, Hkv=2, d=64, S_cap=32, ctx_max=8,
                dtype=wm.BF16)
    base.update(kw)
    return wm.make_dims(**base)


# Addresses that are never read: every call below is refused, or has nothing to do.
def _at(n):
    return ctypes.c_void_p((1 << 40) + n * (1 << 30))


def _attend(wm, call, dims, before=(), after=(), cmap=(0, 1, 0, 1), params=True, **ptr):
    p = {n: _at(i) for i, n in enumerate(("Q", "ctx", "Kc", "Vc", "O", "ws"))}
    p.update(ptr)
    P = wm.Params(*[(1 << 41)] * 12) if params else None
    m = (ctypes.c_int32 * len(cmap))(*cmap) if cmap else None
    return getattr(wm.lib(), call)(
        ctypes.byref(dims), ctypes.byref(P) if P else None, p["Q"], m, p["ctx"], *before, p["Kc"],
        p["Vc"], p["O"], *after, p["ws"], ptr.get("ws_bytes", 1 << 30), None)


CALLS = {"wm_channel_attend_window": ((16, 4), ()),
         "wm_channel_attend_window_backward": ((16, 4), tuple(range(10, 16))),
         "wm_channel_attend_shared": ((16, 16, 8, 9), ()),
         "wm_channel_attend_weigh": ((), (10,))}


def _call(wm, name, dims, before=None, after=None, **kw):
    b, a = CALLS[name]
    b = list(b if before is None else before)
    if name == "wm_channel_attend_shared":
        b[2:] = [_at(x) if isinstance(x, int) else x for x in b[2:]]
    a = [_at(x) if isinstance(x, int) else x for x in (a if after is None else after)]
    return _attend(wm, name, dims, b, a, **kw)


@pytest.mark.parametrize("name", CALLS)
def test_attention_refusals(wm, name):
    ok = _dims(wm)
    for kw in (dict(Q=None), dict(Kc=None), dict(Vc=None), dict(O=None), dict(params=False),
               dict(cmap=None), dict(Q=ctypes.c_void_p((1 << 40) + 2))):
        assert _call(wm, name, ok, **kw) == wm.ERR_ARG, kw
    assert _call(wm, name, ok, cmap=(0, 1, 2, 0)) == wm.ERR_MAP
    for kw, code in ((dict(d=48), "ERR_SHAPE"), (dict(dtype=5), "ERR_DTYPE"),
                     (dict(ctx_max=30), "ERR_CAPACITY"), (dict(mask_mode=3), "ERR_DTYPE"),
                     (dict(Hq=3), "ERR_SHAPE"), (dict(T_new=-1), "ERR_ARG")):
        assert _call(wm, name, _dims(wm, **kw)) == getattr(wm, code), kw
    assert _call(wm, name, _dims(wm, B=0)) == wm.OK
    assert _call(wm, name, _dims(wm, T_new=0)) == wm.OK


@pytest.mark.parametrize("name,op", [("wm_channel_attend_window", "OP_WINDOW_ATTEND"),
                                     ("wm_channel_attend_window_backward", "OP_WINDOW_BACKWARD"),
                                     ("wm_channel_attend_shared", None),
                                     ("wm_channel_attend_weigh", "OP_WEIGH_ATTEND")])
def test_workspace_refusals(wm, name, op):
    d = _dims(wm, T_new=1)
    need = wm.workspace_size(d, getattr(wm, op)) if op else wm.shared_workspace(d, 16)
    if need == 0:
        return
    assert _call(wm, name, d, ws=None) == wm.ERR_WORKSPACE
    assert _call(wm, name, d, ws=ctypes.c_void_p((1 << 40) + 16)) == wm.ERR_WORKSPACE
    assert _call(wm, name, d, ws_bytes=need - 1) == wm.ERR_WORKSPACE


def test_window_refusals(wm):
    for name in ("wm_channel_attend_window", "wm_channel_attend_window_backward"):
        for w, s in ((0, 0), (-1, 0), (1, -1), (-2 ** 31, 0)):
            assert _call(wm, name, _dims(wm), before=(w, s)) == wm.ERR_ARG
    name = "wm_channel_attend_window_backward"
    assert _call(wm, name, _dims(wm, dtype=wm.F32)) == wm.ERR_DTYPE
    assert _call(wm, name, _dims(wm, d=32)) == wm.ERR_SHAPE
    for i in range(6):
        outs = [None if i == j else 10 + j for j in range(6)]
        assert _call(wm, name, _dims(wm), after=outs) == wm.ERR_ARG


def test_shared_refusals(wm):
    name = "wm_channel_attend_shared"
    assert _call(wm, name, _dims(wm), before=(-1, 16, 8, 9)) == wm.ERR_ARG
    assert _call(wm, name, _dims(wm), before=(17, 16, 8, 9)) == wm.ERR_CAPACITY
    assert _call(wm, name, _dims(wm), before=(4, 16, None, 9)) == wm.ERR_ARG
    assert _call(wm, name, _dims(wm), before=(4, 16, 8, None)) == wm.ERR_ARG
    assert _call(wm, name, _dims(wm), before=(4, 1 << 25, 8, 9)) == wm.ERR_SHAPE
    assert wm.shared_workspace(_dims(wm), -1) == 0
    assert wm.shared_workspace(_dims(wm, d=48), 4) == 0


def test_weigh_refusals(wm):
    assert _call(wm, "wm_channel_attend_weigh", _dims(wm), after=(None,)) == wm.ERR_ARG


def _share(wm, dims, seq=0, n=4, cap=16, ptrs=(0, 1, 2, 3), kd=(None, None)):
    return wm.lib().wm_prefix_share(ctypes.byref(dims), *[None if p is None else _at(p)
                                                          for p in ptrs[:2]], seq, n, cap,
                                    *[None if p is None else _at(p) for p in (*ptrs[2:], *kd)],
                                    None)


def test_prefix_share_refusals(wm):
    d = _dims(wm)
    for kw, code in ((dict(seq=-1), "ERR_ARG"), (dict(seq=2), "ERR_ARG"), (dict(n=0), "ERR_ARG"),
                     (dict(n=33, cap=64), "ERR_CAPACITY"), (dict(n=17), "ERR_CAPACITY"),
                     (dict(cap=1 << 25), "ERR_SHAPE"), (dict(ptrs=(0, 1, 0, 3)), "ERR_ARG"),
                     (dict(ptrs=(0, 1, 2, 2)), "ERR_ARG"), (dict(ptrs=(0, 1, 2, 1)), "ERR_ARG"),
                     (dict(kd=(4, None)), "ERR_ARG"), (dict(kd=(None, 4)), "ERR_ARG"),
                     (dict(kd=(4, 4)), "ERR_ARG"), (dict(kd=(4, 1)), "ERR_ARG"),
                     (dict(kd=(2, 5)), "ERR_ARG")):
        assert _share(wm, d, **kw) == getattr(wm, code), kw
    for i in range(4):
        assert _share(wm, d, ptrs=[None if i == j else j for j in range(4)]) == wm.ERR_ARG
    assert _share(wm, _dims(wm, B=0)) == wm.ERR_ARG  # there is no sequence to take


def _evict(wm, dims, keep=4, first=1, recent=2, S_out=8, ws_bytes=1 << 20, **ptr):
    names = ("ctx", "weight", "Kc", "Vc", "ctx_out", "weight_out", "Ko", "Vo", "kept", "ws")
    p = {n: _at(i) for i, n in enumerate(names)}
    p.update(ptr)
    return wm.lib().wm_cache_evict(ctypes.byref(dims), p["ctx"], keep, first, recent, p["weight"],
                                   p["Kc"], p["Vc"], S_out, p["ctx_out"], p["weight_out"],
                                   p["Ko"], p["Vo"], p["kept"], p["ws"], ws_bytes, None)


def test_evict_refusals(wm):
    d = _dims(wm)
    for kw in (dict(keep=0), dict(first=-1), dict(recent=-1), dict(first=3), dict(recent=4),
               dict(first=2 ** 31 - 1, recent=2 ** 31 - 1)):
        assert _evict(wm, d, **kw) == wm.ERR_ARG, kw
    assert _evict(wm, d, S_out=3) == wm.ERR_CAPACITY
    assert _evict(wm, d, S_out=1 << 25) == wm.ERR_SHAPE
    assert _evict(wm, _dims(wm, ctx_max=30)) == wm.ERR_CAPACITY
    for n in ("weight", "Kc", "Vc", "ctx_out", "weight_out", "Ko", "Vo"):
        assert _evict(wm, d, **{n: None}) == wm.ERR_ARG, n
    assert _evict(wm, d, ctx_out=ctypes.c_void_p((1 << 40) + 2)) == wm.ERR_ARG
    assert _evict(wm, d, kept=ctypes.c_void_p((1 << 40) + 2)) == wm.ERR_ARG
    assert _evict(wm, d, ws=None) == wm.ERR_WORKSPACE
    assert _evict(wm, d, ws_bytes=8) == wm.ERR_WORKSPACE
    # outputs apart from the inputs and from each other
    for out, other in (("Ko", "Kc"), ("Vo", "Vc"), ("weight_out", "weight"), ("ctx_out", "ctx"),
                       ("Ko", "Vo"), ("kept", "ctx_out"), ("ws", "weight")):
        at = dict(zip(("ctx", "weight", "Kc", "Vc", "ctx_out", "weight_out", "Ko", "Vo", "kept"),
                      range(9)))[other]
        assert _evict(wm, d, **{out: _at(at)}) == wm.ERR_ARG, (out, other)
    assert _evict(wm, _dims(wm, B=0)) == wm.OK


def test_binding_checks_shapes_and_types(wm):
    d = _dims(wm, T_new=1)
    bf = dict(dtype=torch.bfloat16)
    Q, O = torch.zeros((4, 2, 4, 1, 64), **bf), torch.zeros((4, 2, 1, 256), **bf)
    K = torch.zeros((2, 2, 2, 32, 64), **bf)
    ctx = torch.zeros(2, dtype=torch.int32)
    for bad in (dict(Q=Q[:3].contiguous()), dict(Q=Q.float()), dict(ctx=ctx.long()),
                dict(K=K[..., :16, :].contiguous()), dict(O=O.float())):
        a = dict(Q=Q, ctx=ctx, K=K, O=O) | bad
        with pytest.raises(ValueError):
            wm.channel_attend_window(d, None, a["Q"], [0, 1, 0, 1], a["ctx"], 8, 0, a["K"], K,
                                     a["O"])
    with pytest.raises(ValueError):
        wm.channel_attend_weigh(d, None, Q, [0, 1, 0, 1], ctx, K, K, O, torch.zeros(2, 2, 2, 31))
    with pytest.raises(ValueError):
        wm.cache_evict(d, ctx, 4, 0, 0, torch.zeros(2, 2, 2, 32), K, K, ctx.clone(),
                       torch.zeros(2, 2, 2, 8), torch.zeros((2, 2, 2, 8, 64), **bf),
                       torch.zeros((2, 2, 2, 9, 64), **bf))
