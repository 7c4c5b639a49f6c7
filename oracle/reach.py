"""Plain float64 numpy statement of attention over parts of a long context: a window of the
cache with a few first slots, a prefix shared by the batch, the weight each slot receives, and
the eviction of the lightest slots. Test infrastructure only, like the rest of the package.

Arrays as in oracle/__init__.py; rows sit at position ctx[b] + gq + gs i. `mask_paper`: slots
below the position and the dummy; else slots up to the position and no dummy.
"""
from __future__ import annotations

import numpy as np


def _np(a):
    if hasattr(a, "detach"):
        a = a.detach().to("cpu").double().numpy()
    return np.asarray(a, dtype=np.float64)


def _reads(pos, S, mask_paper, window, sinks):
    """[T, S] truth values: may the row at position pos[i] read slot s."""
    lim = pos[:, None] + (0 if mask_paper else 1)
    s = np.arange(S)[None, :]
    return (s < lim) & ((s >= lim - window) | (s < sinks))


def attend(Q, chan_map, ctx, Kc, Vc, Kd, Vd, mask_paper=True, window=None, sinks=0, gs=1, gq=0,
           Kp=None, Vp=None, dO=None, O_given=None):
    """A dict: O [L, B, T, Hq d]; S [L, B, T, Hq d], the sum of P |v| (the size of the terms O is
    summed from); sigma, the largest sum |q_e k_e| / sqrt(d); weight [k, B, Hkv, S] and, with dO
    (and O_given, default O), dQ, dKc, dVc, dKd, dVd, each with its sum of absolute terms under
    the name + "_abs"."""
    Q, Kc, Vc, Kd, Vd = (_np(a) for a in (Q, Kc, Vc, Kd, Vd))
    L, B, Hq, T, d = Q.shape
    k, _, Hkv, S, _ = Kc.shape
    G, scale = Hq // Hkv, 1 / np.sqrt(d)
    P = 0 if Kp is None else Kp.shape[2]
    if P:
        Kp, Vp = _np(Kp), _np(Vp)
    window = S if window is None else window
    out = {"O": np.zeros((L, B, T, Hq * d)), "S": np.zeros((L, B, T, Hq * d)), "sigma": 0.0,
           "weight": np.zeros((k, B, Hkv, S))}
    if dO is not None:
        dO = _np(dO).reshape(L, B, T, Hq, d)
        for n, shape in (("dQ", Q.shape), ("dKc", Kc.shape), ("dVc", Vc.shape),
                         ("dKd", Kd.shape), ("dVd", Vd.shape)):
            out[n], out[n + "_abs"] = np.zeros(shape), np.zeros(shape)
    for l in range(L):
        c = chan_map[l]
        for b in range(B):
            pos = int(ctx[b]) + gq + gs * np.arange(T)
            see = np.ones((T, P + S + 1), dtype=bool)
            see[:, P:P + S] = _reads(pos, S, mask_paper, window, sinks)
            see[:, -1] = mask_paper
            for h in range(Hq):
                kv = h // G
                K, V = np.empty((P + S + 1, d)), np.empty((P + S + 1, d))
                if P:
                    K[:P], V[:P] = Kp[c, kv], Vp[c, kv]
                # slots no row reads hold anything: they take no part
                used = see[:, P:P + S].any(0)[:, None]
                K[P:P + S] = np.where(used, Kc[c, b, kv], 0)
                V[P:P + S] = np.where(used, Vc[c, b, kv], 0)
                K[-1], V[-1] = Kd[c, kv], Vd[c, kv]
                q = Q[l, b, h]
                z = np.where(see, q @ K.T * scale, -np.inf)
                size = np.where(see, np.abs(q) @ np.abs(K).T * scale, 0)
                out["sigma"] = max(out["sigma"], size.max())
                w = np.exp(z - z.max(1, keepdims=True))
                w /= w.sum(1, keepdims=True)
                cols = slice(h * d, (h + 1) * d)
                out["O"][l, b, :, cols] = w @ V
                out["S"][l, b, :, cols] = w @ np.abs(V)
                out["weight"][c, b, kv] += w[:, P:P + S].sum(0)
                if dO is None:
                    continue
                g = dO[l, b, :, h]
                o = out["O"][l, b, :, cols] if O_given is None else \
                    _np(O_given)[l, b, :, cols]
                ds = w * (g @ V.T - (g * o).sum(1, keepdims=True)) * scale
                big = w * (np.abs(g) @ np.abs(V).T +
                           (np.abs(g) * np.abs(o)).sum(1, keepdims=True)) * scale
                for tag, x, aq, ak, ag in (("", ds, q, K, g),
                                           ("_abs", big, np.abs(q), np.abs(K), np.abs(g))):
                    out["dQ" + tag][l, b, h] = x @ ak
                    dk, dv = x.T @ aq, w.T @ ag
                    out["dKc" + tag][c, b, kv] += dk[P:P + S]
                    out["dVc" + tag][c, b, kv] += dv[P:P + S]
                    out["dKd" + tag][c, kv] += dk[-1]
                    out["dVd" + tag][c, kv] += dv[-1]
    return out


def turn(x, by, theta):
    """Keys x [n, d] turned by `by` [n] positions (rotate-half)."""
    d = x.shape[-1]
    a = np.asarray(by, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(d // 2) / d)
    x1, x2 = x[:, :d // 2], x[:, d // 2:]
    return np.concatenate([x1 * np.cos(a) - x2 * np.sin(a), x2 * np.cos(a) + x1 * np.sin(a)], 1)


def evict_slots(weight, n, keep, first, recent):
    """The kept slots of one slice of n slots, ascending."""
    if n <= keep:
        return list(range(n))
    w = np.where(np.isnan(weight), -np.inf, weight)
    nan = np.isnan(weight)
    middle = sorted(range(first, n - recent), key=lambda s: (nan[s], -w[s], s))
    return sorted([*range(first), *middle[:keep - first - recent], *range(n - recent, n)])
