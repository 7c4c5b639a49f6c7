"""GPU parity of the moves of cache rows with the float64 oracle (oracle/reach.py): eviction by
accumulated weight and the layout of a shared prefix. Which slots are kept is exact; a moved key
is off by its rounding (2^-8 of itself in bf16, 2^-24 in fp32) and by the fp32 rotation: angle,
sine and cosine off by at most 2^-21, two products and a sum of |x1| + |x2|; values, weights
and keys that stay where they are are bit for bit."""
import numpy as np
import pytest
import torch

from oracle import reach
from tests.parity import wm  # noqa: F401

pytestmark = pytest.mark.gpu
THETA = 1e6


def _caches(seed, k, B, Hkv, S, d, dtype, holes=True):
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    Kc, Vc = (torch.randn((k, B, Hkv, S, d), generator=g).to(dt) for _ in range(2))
    w = torch.rand((k, B, Hkv, S), generator=g).round(decimals=2)  # ties
    if holes:
        w[torch.rand(w.shape, generator=g) < 0.3] = 0.0
        w[torch.rand(w.shape, generator=g) < 0.05] = float("nan")
        w[torch.rand(w.shape, generator=g) < 0.05] = -0.0
        w[torch.rand(w.shape, generator=g) < 0.02] = float("inf")
    return Kc, Vc, w


def _key_tol(x, dtype):
    h = x.shape[-1] // 2
    size = np.abs(x[:, :h]) + np.abs(x[:, h:])
    return 2.0 ** -21 * np.concatenate([size, size], 1), 2.0 ** (-8 if dtype == "bf16" else -24)


def _check_keys(got, x, by, dtype, name):
    want = reach.turn(x, by, THETA)
    tol, half = _key_tol(x, dtype)
    over = np.abs(got - want) - (tol + half * (np.abs(want) + tol))
    assert over.max(initial=-1.0) <= 0, "%s: past its bound by %.3g" % (name, over.max())


# (ctx of two sequences, keep, first, recent)
EVICTS = [((0, 1), 1, 0, 0), ((10, 9), 4, 1, 2), ((100, 64), 64, 0, 64), ((300, 17), 65, 4, 0),
          ((1500, 1023), 700, 4, 256), ((1025, 3333), 1024, 0, 1), ((200, 200), 199, 199, 0),
          ((77, 50), 500, 10, 30), ((2048, 2049), 2047, 0, 0), ((90, 40), 30, 0, 0)]


@pytest.mark.parametrize("ctx,keep,first,recent", EVICTS)
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 96), ("bf16", 32), ("f32", 64),
                                     ("f32", 32)])
@pytest.mark.parametrize("spare", [0, 13])
def test_evict(wm, dtype, d, ctx, keep, first, recent, spare):
    k, B, Hkv, S, So = 2, 2, 3, max(ctx) + 9, keep + spare
    print("evict", dtype, d, ctx, keep, first, recent, flush=True)
    Kc, Vc, w = _caches(1, k, B, Hkv, S, d, dtype)
    dims = wm.make_dims(B, 0, k, k, 64, Hkv, Hkv, d, S_cap=S, ctx_max=max(ctx), rope_theta=THETA,
                        dtype=wm.BF16 if dtype == "bf16" else wm.F32)
    nan = float("nan")
    Ko = torch.full((k, B, Hkv, So, d), nan, dtype=Kc.dtype, device="cuda")
    Vo = torch.full_like(Ko, nan)
    wo = torch.full((k, B, Hkv, So), nan, device="cuda")
    co = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    kept = torch.full((k, B, Hkv, keep), -7, dtype=torch.int32, device="cuda")
    ws = torch.full((max(256, wm.workspace_size(dims, wm.OP_CACHE_EVICT)),), 0xFF,
                    dtype=torch.uint8, device="cuda")
    cl = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    args = (dims, cl, keep, first, recent, w.cuda(), Kc.cuda(), Vc.cuda(), co, wo, Ko, Vo)
    wm.cache_evict(*args, kept=kept, ws=ws)
    torch.cuda.synchronize()
    assert co.tolist() == [min(n, keep) for n in ctx]
    for c in range(k):
        for b, n in enumerate(ctx):
            m = min(n, keep)
            for h in range(Hkv):
                name = "channel %d sequence %d head %d" % (c, b, h)
                slots = reach.evict_slots(w[c, b, h].double().numpy(), n, keep, first, recent)
                assert kept[c, b, h].tolist() == slots + [-1] * (keep - m), name
                by = np.arange(m) - np.array(slots, dtype=np.int64)
                _check_keys(Ko[c, b, h, :m].cpu().double().numpy(),
                            Kc[c, b, h, slots].double().numpy(), by, dtype, name)
                still = torch.from_numpy(by == 0)
                assert torch.equal(Ko[c, b, h, :m].cpu()[still], Kc[c, b, h, slots][still])
                assert torch.equal(Vo[c, b, h, :m].cpu(), Vc[c, b, h, slots])
                assert np.array_equal(wo[c, b, h, :m].cpu().numpy(), w[c, b, h, slots].numpy(),
                                      equal_nan=True)
                assert not wo[c, b, h, m:].any()
                assert torch.isnan(Ko[c, b, h, m:]).all() and torch.isnan(Vo[c, b, h, m:]).all()
    again = [torch.full_like(x, nan) for x in (Ko, Vo)]
    wm.cache_evict(*args[:-2], *again, ws=ws)  # without the kept slots' list
    torch.cuda.synchronize()
    for x, y in zip(again, (Ko, Vo)):
        assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))


def test_evict_far_positions(wm):
    """Angles of moves over 100 thousand positions; equal weights everywhere: the lowest stay."""
    n, keep, d = 120_001, 300, 32
    Kc, Vc, _ = _caches(2, 1, 1, 1, n, d, "f32")
    w = torch.ones((1, 1, 1, n))
    w[..., 100_000:] = 2.0
    dims = wm.make_dims(1, 0, 1, 1, 64, 1, 1, d, S_cap=n, ctx_max=n, rope_theta=THETA,
                        dtype=wm.F32)
    Ko, Vo = (torch.empty((1, 1, 1, keep, d), device="cuda") for _ in range(2))
    wo, co = torch.empty((1, 1, 1, keep), device="cuda"), torch.empty(1, dtype=torch.int32,
                                                                      device="cuda")
    wm.cache_evict(dims, torch.tensor([n], dtype=torch.int32, device="cuda"), keep, 5, 10,
                   w.cuda(), Kc.cuda(), Vc.cuda(), co, wo, Ko, Vo)
    torch.cuda.synchronize()
    slots = [*range(5), *range(100_000, 100_285), *range(n - 10, n)]
    _check_keys(Ko[0, 0, 0].cpu().double().numpy(), Kc[0, 0, 0, slots].double().numpy(),
                np.arange(keep) - np.array(slots), "f32", "far keys")
    assert torch.equal(Vo[0, 0, 0].cpu(), Vc[0, 0, 0, slots])


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 96), ("bf16", 32), ("f32", 64),
                                     ("f32", 32)])
@pytest.mark.parametrize("P,P_cap,seq", [(1, 1, 0), (65, 100, 1), (700, 700, 2)])
def test_prefix_share(wm, dtype, d, P, P_cap, seq):
    k, B, Hkv, S = 2, 3, 2, P + 11
    Kc, Vc, _ = _caches(3, k, B, Hkv, S, d, dtype, holes=False)
    dims = wm.make_dims(B, 0, k, k, 64, Hkv, Hkv, d, S_cap=S, ctx_max=P, rope_theta=THETA,
                        dtype=wm.BF16 if dtype == "bf16" else wm.F32)
    Kp = torch.full((k, Hkv, P_cap, d), float("nan"), dtype=Kc.dtype, device="cuda")
    Vp = torch.full_like(Kp, float("nan"))
    Kd = torch.randn((k, Hkv, d), generator=torch.Generator().manual_seed(4)).to(Kc.dtype)
    Kd_out = torch.full_like(Kd, float("nan"), device="cuda")
    wm.prefix_share(dims, Kc.cuda(), Vc.cuda(), seq, P, Kp, Vp, Kd=Kd.cuda(), Kd_out=Kd_out)
    torch.cuda.synchronize()
    _check_keys(Kd_out.cpu().double().numpy().reshape(-1, d), Kd.double().numpy().reshape(-1, d),
                np.full(k * Hkv, -P), dtype, "dummy")
    for c in range(k):
        for h in range(Hkv):
            _check_keys(Kp[c, h, :P].cpu().double().numpy(), Kc[c, seq, h, :P].double().numpy(),
                        np.full(P, -P), dtype, "prefix")
    assert torch.equal(Vp[:, :, :P].cpu(), Vc[:, seq, :, :P])
    assert torch.isnan(Kp[:, :, P:]).all() and torch.isnan(Vp[:, :, P:]).all()
