"""Pins of the window, shared-prefix and eviction oracle (oracle/reach.py): against the
framework's own attention oracle where both say the same, brute force and differences."""
import numpy as np
import pytest

from oracle import reach


def _case(seed, L=2, B=2, Hq=2, Hkv=1, T=5, d=4, k=2, S=12):
    r = np.random.default_rng(seed)
    return dict(Q=r.normal(size=(L, B, Hq, T, d)), chan_map=[l % k for l in range(L)],
                ctx=[3, 6][:B], Kc=r.normal(size=(k, B, Hkv, S, d)),
                Vc=r.normal(size=(k, B, Hkv, S, d)), Kd=r.normal(size=(k, Hkv, d)),
                Vd=r.normal(size=(k, Hkv, d)))


@pytest.mark.parametrize("paper", [True, False])
def test_whole_window_is_channel_attention(oracle_lib, paper):
    o = oracle_lib
    c = _case(1)
    dims = o.Dims(B=2, T_new=5, L=2, k=2, D=32, Hq=2, Hkv=1, d=4, S_cap=12,
                  mask_mode=o.MASK_PAPER if paper else o.MASK_INCLUSIVE)
    P = {n: np.zeros(1) for n in o.PARAM_NAMES}
    P.update(Kd=c["Kd"], Vd=c["Vd"])
    want = o.channel_attend(dims, P, c["Q"], c["chan_map"], np.array(c["ctx"], np.int32), c["Kc"],
                            c["Vc"])
    np.testing.assert_allclose(reach.attend(**c, mask_paper=paper)["O"], want, atol=1e-12)


@pytest.mark.parametrize("paper", [True, False])
@pytest.mark.parametrize("window,sinks,gs,gq", [(1, 0, 1, 0), (3, 2, 1, 0), (2, 1, 2, 1),
                                                (100, 0, 1, 0), (4, 100, 1, 0)])
def test_window_by_brute_force(paper, window, sinks, gs, gq):
    c = _case(2, S=20)
    got = reach.attend(**c, mask_paper=paper, window=window, sinks=sinks, gs=gs, gq=gq)
    for l in range(2):
        for b in range(2):
            for h in range(2):
                for i in range(5):
                    t = c["ctx"][b] + gq + gs * i
                    slots = range(t) if paper else range(t + 1)
                    mine = [s for n, s in enumerate(reversed(slots)) if n < window or s < sinks]
                    ch = c["chan_map"][l]
                    ks = [c["Kc"][ch, b, 0, s] for s in mine]
                    vs = [c["Vc"][ch, b, 0, s] for s in mine]
                    if paper:
                        ks.append(c["Kd"][ch, 0])
                        vs.append(c["Vd"][ch, 0])
                    e = [np.exp(c["Q"][l, b, h, i] @ x / 2.0) for x in ks]
                    want = sum(a * v for a, v in zip(e, vs)) / sum(e)
                    np.testing.assert_allclose(got["O"][l, b, i, 4 * h:4 * h + 4], want,
                                               atol=1e-12)


def test_shared_prefix_is_a_longer_cache():
    """A prefix is the same as its slots in front of every sequence's own."""
    c = _case(3)
    r = np.random.default_rng(4)
    Kp, Vp = r.normal(size=(2, 1, 7, 4)), r.normal(size=(2, 1, 7, 4))
    got = reach.attend(**c, Kp=Kp, Vp=Vp)
    front = {n: np.concatenate([np.repeat(p[:, None], 2, 1), c[n]], 3)
             for n, p in (("Kc", Kp), ("Vc", Vp))}
    want = reach.attend(**{**c, **front, "ctx": [x + 7 for x in c["ctx"]]})
    np.testing.assert_allclose(got["O"], want["O"], atol=1e-12)
    np.testing.assert_allclose(got["weight"], want["weight"][..., 7:], atol=1e-12)


def test_weights_of_a_row_sum_to_one():
    c = _case(5)
    w = reach.attend(**c, mask_paper=False, window=4, sinks=1)["weight"]
    # channel 0 has one consumer: per sequence, query heads x tokens rows
    np.testing.assert_allclose(w[0].sum((1, 2)), 2 * 5, atol=1e-12)


@pytest.mark.parametrize("paper", [True, False])
def test_window_gradients_by_differences(paper):
    c = _case(6)
    how = dict(mask_paper=paper, window=3, sinks=2)
    dO = np.random.default_rng(7).normal(size=(2, 2, 5, 8))
    g = reach.attend(**c, **how, dO=dO)
    r = np.random.default_rng(8)
    for n in ("Q", "Kc", "Vc", "Kd", "Vd"):
        v = r.normal(size=c[n].shape)
        f = [(reach.attend(**{**c, n: c[n] + e * v}, **how)["O"] * dO).sum() for e in (1e-5, -1e-5)]
        np.testing.assert_allclose((g["d" + n] * v).sum(), (f[0] - f[1]) / 2e-5, rtol=1e-6,
                                   atol=1e-8)


def test_evicted_slots_and_turned_keys(oracle_lib):
    w = np.array([9., 1., 5., 5., np.nan, 7., 5., 0., 3.])
    assert reach.evict_slots(w, 9, 9, 0, 0) == list(range(9))
    assert reach.evict_slots(w, 9, 5, 1, 2) == [0, 2, 5, 7, 8]
    assert reach.evict_slots(w, 9, 8, 0, 0) == [0, 1, 2, 3, 5, 6, 7, 8]
    assert reach.evict_slots(w, 9, 2, 1, 1) == [0, 8]
    x = np.random.default_rng(9).normal(size=(3, 32))
    at = [np.stack([oracle_lib.rope(v, p, 1e4) for v, p in zip(x, ps)])
          for ps in ((40, 41, 50), (10, 11, 19))]
    np.testing.assert_allclose(reach.turn(at[0], [-30, -30, -31], 1e4), at[1], atol=1e-12)
