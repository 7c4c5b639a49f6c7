"""Timed cases of the operators that keep a long context cheap: attention over a window of
the cache, over a prefix that a batch shares, and the eviction of what attention passes by.

Kinds:
  window   wm.channel_attend_window: each row reads the `window` slots up to its position and
           the first `sinks` slots (T = 1..4: decode; larger: a prompt or a chunk of one)
  grad     wm.channel_attend_window_backward: the gradients of a full-sequence window call
  shared   wm.channel_attend_shared: every sequence reads one prefix and its own cache
  share    wm.prefix_share: lays a prefix out for it, from the cache of the call that made it
  weigh    wm.channel_attend_weigh: attention that adds up the weight each slot receives
  evict    wm.cache_evict: the heaviest slots move to a smaller cache, keys turned to their
           new positions
The shapes are the repository's models: 16 layers of 6 / 3 heads of 96, 12 layers of 12 heads
of 64, 24 layers of 16 heads of 64. Queries and keys have unit RMS (both are normalised),
values likewise; a slot's accumulated weight is log-normal, and zero for some.
"""
import math

import torch

own = False

PAPER = dict(L=16, D=512, Hq=6, Hkv=3, d=96)
MID = dict(L=12, D=768, Hq=12, Hkv=12, d=64)
WIDE = dict(L=24, D=1024, Hq=16, Hkv=16, d=64)
MODELS = {"paper": PAPER, "mid": MID, "wide": WIDE}
CHANNELS = {"paper": (4, 8, 16), "mid": (6, 12), "wide": (6, 12)}
THETA = 1e6


def _case(kind, model, k, B, T, name=None, **more):
    c = dict(kind=kind, k=k, B=B, T=T, ctx=0, ragged=False, dtype="bf16", inclusive=False,
             window=0, sinks=0, prefix=0, keep=0, first=0, recent=0)
    c.update(MODELS[model])
    c.update(more)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # One user's chat over a bounded window: latency counts.
        _case("window", "paper", 8, 1, 1, "window_decode_b1", ctx=4001, window=1024, sinks=4),
        # A batch of long conversations, each reading the last 2048 of up to 8191 slots.
        _case("window", "wide", 12, 16, 1, "window_decode_b16", ctx=8191, ragged=True,
              window=2048, sinks=16),
        # A long prompt in one call.
        _case("window", "mid", 6, 1, 4001, "window_t4001_l12", window=1024, sinks=4),
        # Training rows of the 16-layer model under a window.
        _case("grad", "paper", 8, 2, 2048, "window_grad_t2048", window=512, sinks=4),
        # A ragged chunk after a cached context, standard causal, no sinks.
        _case("grad", "mid", 6, 3, 333, "window_grad_t333", ctx=200, ragged=True, window=129,
              inclusive=True),
        # Many users of one system prompt, one token each.
        _case("shared", "wide", 12, 64, 1, "shared_decode_b64", ctx=300, ragged=True,
              prefix=4096),
        # Their questions, read in one call, in single precision.
        _case("shared", "mid", 6, 5, 37, "shared_t37_f32", ctx=50, ragged=True, prefix=777,
              dtype="f32"),
        # That prompt, laid out once.
        _case("share", "wide", 12, 1, 0, "share_p4001", ctx=4050, prefix=4001),
        # Decoding while the weights are added up.
        _case("weigh", "wide", 12, 8, 1, "weigh_decode_b8", ctx=4001, ragged=True),
        # A prompt's weights, every row of it.
        _case("weigh", "paper", 8, 2, 1023, "weigh_t1023"),
        # A batch's caches cut to a quarter.
        _case("evict", "wide", 12, 8, 0, "evict_b8_8k", ctx=8191, ragged=True, keep=2048,
              first=4, recent=256),
        # One small cache in single precision.
        _case("evict", "mid", 6, 1, 0, "evict_b1_f32", ctx=900, keep=511, first=1, recent=64,
              dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["window", "window", "chunk", "grad", "shared", "shared", "share",
                       "weigh", "weigh", "evict", "evict"])
    model = rng.choice(["paper", "mid", "wide"])
    k = rng.choice(CHANNELS[model])
    more = dict(inclusive=rng.random() < 0.3)
    if model != "paper" and rng.random() < 0.2:
        more["dtype"] = "f32"
    f32 = "dtype" in more
    win = dict(window=_log(rng, 16, 2048), sinks=rng.choice([0, 1, 4, 16, 65]))
    if kind == "window":
        ctx = _log(rng, 100, 8191)
        B = _log(rng, 1, max(1, min(32, (4 if f32 else 16) * 4096 // ctx)))
        return _case("window", model, k, B, rng.choice([1, 1, 2, 3, 4]), ctx=ctx,
                     ragged=B > 1, **win, **more)
    if kind == "chunk":
        T = _log(rng, 5, 700 if f32 else 2048)
        return _case("window", model, k, _log(rng, 1, max(1, min(16, 2048 // T))), T,
                     ctx=rng.choice([0, _log(rng, 50, 1000)]), ragged=True, **win, **more)
    if kind == "grad":
        more.pop("dtype", None)
        T = _log(rng, 1, 900)
        return _case("grad", model, k, _log(rng, 1, max(1, min(8, 900 // T))), T,
                     ctx=rng.choice([0, _log(rng, 20, 500)]), ragged=True, **win, **more)
    if kind == "shared":
        T = rng.choice([1, 1, 1, 2, 4, _log(rng, 5, 200)])
        B = _log(rng, 1, max(1, min(64, (64 if f32 else 256) // T)))
        return _case("shared", model, k, B, T, ctx=_log(rng, 1, 300), ragged=True,
                     prefix=_log(rng, 50, 4096), **more)
    if kind == "share":
        more.pop("inclusive")
        P = _log(rng, 50, 4096)
        return _case("share", model, k, _log(rng, 1, 4), 0, ctx=P + rng.randint(0, 99), prefix=P,
                     **more)
    if kind == "weigh":
        if rng.random() < 0.5:
            ctx = _log(rng, 100, 4096)
            B = _log(rng, 1, max(1, min(16, 4 * 4096 // ctx)))
            return _case("weigh", model, k, B, rng.choice([1, 1, 2, 4]), ctx=ctx, ragged=True,
                         **more)
        T = _log(rng, 5, 500 if f32 else 1023)
        return _case("weigh", model, k, _log(rng, 1, max(1, min(8, 1024 // T))), T,
                     ctx=rng.choice([0, _log(rng, 20, 500)]), ragged=True, **more)
    more.pop("inclusive")
    ctx = _log(rng, 64, 8191)
    B = _log(rng, 1, max(1, min(16, (6 if f32 else 12) * 4096 // ctx)))
    keep = _log(rng, 16, ctx)
    first = min(keep, rng.choice([0, 1, 4]))
    return _case("evict", model, k, B, 0, ctx=ctx, ragged=True, keep=keep, first=first,
                 recent=rng.randint(0, keep - first), **more)


# ------------------------------------------------------------------ inputs

def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _inputs(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    L, k, Hq, Hkv, d, B, T = (c[n] for n in ("L", "k", "Hq", "Hkv", "d", "B", "T"))
    dt = _dtype(c)

    def normal(*shape):
        return torch.empty(shape, device="cuda", dtype=dt).normal_(generator=gen)

    s = {"c": c, "map": [l % k for l in range(L)], "S": (c["ctx"] + T + 63) // 64 * 64}
    lo = c["ctx"] // 2 if c["ragged"] else c["ctx"]
    s["ctx"] = torch.randint(lo, c["ctx"] + 1, (B,), generator=gen, device="cuda",
                             dtype=torch.int32)
    s["Kc"], s["Vc"] = normal(k, B, Hkv, s["S"], d), normal(k, B, Hkv, s["S"], d)
    if T:
        s["Q"] = normal(L, B, Hq, T, d)
        s["Kd"], s["Vd"] = normal(k, Hkv, d), normal(k, Hkv, d)
        s["O"] = torch.empty((L, B, T, Hq * d), device="cuda", dtype=dt)
    f32 = dict(device="cuda", dtype=torch.float32)
    if c["kind"] == "shared":
        s["Kp"], s["Vp"] = (normal(k, Hkv, (c["prefix"] + 63) // 64 * 64, d) for _ in range(2))
    if c["kind"] == "share":
        s["Kp"], s["Vp"] = (torch.zeros((k, Hkv, c["prefix"], d), device="cuda", dtype=dt)
                            for _ in range(2))
    if c["kind"] in ("weigh", "evict"):
        w = torch.empty((k, B, Hkv, s["S"]), **f32).normal_(generator=gen).mul_(1.5).exp_()
        if c["kind"] == "weigh":  # what a few tokens have added before
            w.mul_(1e-3)
        s["weight"] = w.masked_fill_(torch.rand(w.shape, generator=gen, **f32) < 0.1, 0.0)
    if c["kind"] == "evict":
        So = s["So"] = (c["keep"] + 63) // 64 * 64
        s["Ko"] = torch.zeros((k, B, Hkv, So, d), device="cuda", dtype=dt)
        s["Vo"] = torch.zeros_like(s["Ko"])
        s["weight_out"] = torch.empty((k, B, Hkv, So), **f32)
        s["ctx_out"] = torch.empty_like(s["ctx"])
        s["kept"] = torch.empty((k, B, Hkv, c["keep"]), device="cuda", dtype=torch.int32)
    if c["kind"] == "grad":
        s["dO"] = normal(L, B, T, Hq * d)
        s["dQ"] = torch.zeros((L, B, Hq, T, d), **f32)
        s["dKc"], s["dVc"] = (torch.zeros((k, B, Hkv, s["S"], d), **f32) for _ in range(2))
        s["dKd"], s["dVd"] = (torch.zeros((k, Hkv, d), **f32) for _ in range(2))
    return s


def _attention_output(s):
    """The forward's output that a training step holds for its backward."""
    s["O"].copy_(_attend(s, *_window_slots(s))[0])


def prepare(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    if c["kind"] == "grad":
        _attention_output(s)
    if own:
        import paper_2608_18486_amd as wm
        s["wm"] = wm
        s["dims"] = dims = wm.make_dims(
            c["B"], c["T"], c["L"], c["k"], c["D"], c["Hq"], c["Hkv"], c["d"], S_cap=s["S"],
            ctx_max=c["ctx"], dtype=wm.dtype_code(_dtype(c)), rope_theta=THETA,
            mask_mode=wm.MASK_INCLUSIVE if c["inclusive"] else wm.MASK_PAPER)
        s["params"] = None
        if c["T"]:
            none = torch.zeros(8, device="cuda", dtype=_dtype(c))
            s["params"] = wm.ParamSet({n: s.get(n, none) for n in wm.PARAM_NAMES})
        if c["kind"] == "shared":
            s["ws"] = torch.empty(max(256, wm.shared_workspace(dims, c["prefix"])),
                                  dtype=torch.uint8, device="cuda")
        elif c["kind"] != "share":
            s["ws"] = wm.workspace(dims, {"window": wm.OP_WINDOW_ATTEND,
                                          "grad": wm.OP_WINDOW_BACKWARD,
                                          "weigh": wm.OP_WEIGH_ATTEND,
                                          "evict": wm.OP_CACHE_EVICT}[c["kind"]])
    return s


# ------------------------------------------------------------- the plain forms

def _rows(s):
    """(slots the row may see end here, exclusive) [B, T, 1] and the slot indices [S]."""
    c = s["c"]
    at = s["ctx"].long()[:, None] + torch.arange(c["T"], device="cuda")
    return (at + (1 if c["inclusive"] else 0))[..., None], torch.arange(s["S"], device="cuda")


def _causal_slots(s):
    lim, slot = _rows(s)
    return (slot < lim,)


def _window_slots(s):
    lim, slot = _rows(s)
    c = s["c"]
    return ((slot < lim) & ((slot >= lim - c["window"]) | (slot < c["sinks"])),)


def _by_layer(s, cache):
    """[k, ...] to the layers' own channels, in 32 bits."""
    return cache[s["map"]].float()


def _scores(s, q, K):
    """q [..., n, d] against K [..., S, d], scaled."""
    return torch.matmul(q, K.transpose(-1, -2).contiguous()) * s["c"]["d"] ** -0.5


def _attend(s, see):
    """Output [L, B, T, Hq d], weights [L, B, Hkv, G T, S], the dummy's [..., 1]; 32 bits."""
    c = s["c"]
    L, Hq, Hkv, d, B, T = (c[n] for n in ("L", "Hq", "Hkv", "d", "B", "T"))
    G = Hq // Hkv
    q = s["Q"].float().reshape(L, B, Hkv, G * T, d)
    K, V = _by_layer(s, s["Kc"]), _by_layer(s, s["Vc"])
    see = see[:, None, None].expand(B, 1, G, T, s["S"]).reshape(B, 1, G * T, s["S"])
    x = _scores(s, q, K).masked_fill_(~see, -math.inf)
    kd, vd = (_by_layer(s, s[n])[:, None, :, None] for n in ("Kd", "Vd"))
    xd = (q * kd).sum(-1, keepdim=True) * d ** -0.5
    if c["inclusive"]:
        xd = torch.full_like(xd, -math.inf)
    m = torch.maximum(x.amax(-1, keepdim=True), xd)
    p, pd = x.sub_(m).exp_(), (xd - m).exp()
    total = p.sum(-1, keepdim=True) + pd
    p, pd = p.div_(total), pd / total
    o = torch.matmul(p, V) + pd * vd
    return _token_major(c, o), p, pd


def _token_major(c, o):
    L, Hq, d, B, T = (c[n] for n in ("L", "Hq", "d", "B", "T"))
    return o.reshape(L, B, Hq, T, d).transpose(2, 3).reshape(L, B, T, Hq * d)


def _to_channels(s, x):
    """The sum over each channel's layers of x [L, ...]."""
    hot = torch.zeros((s["c"]["k"], s["c"]["L"]), device="cuda")
    hot[s["map"], list(range(s["c"]["L"]))] = 1.0
    return torch.matmul(hot, x.reshape(s["c"]["L"], -1)).reshape(-1, *x.shape[1:])


def _plain_grad(s):
    c = s["c"]
    L, Hq, Hkv, d, B, T = (c[n] for n in ("L", "Hq", "Hkv", "d", "B", "T"))
    G = Hq // Hkv
    _, p, pd = _attend(s, *_window_slots(s))
    q = s["Q"].float().reshape(L, B, Hkv, G * T, d)

    def head_major(x):
        return x.float().reshape(L, B, T, Hq, d).transpose(2, 3).reshape(L, B, Hkv, G * T, d)

    dO, O = head_major(s["dO"]), head_major(s["O"])
    delta = (dO * O).sum(-1, keepdim=True)
    K, V = _by_layer(s, s["Kc"]), _by_layer(s, s["Vc"])
    kd, vd = (_by_layer(s, s[n])[:, None, :, None] for n in ("Kd", "Vd"))
    dS = torch.matmul(dO, V.transpose(-1, -2).contiguous()).sub_(delta).mul_(p)
    dSd = ((dO * vd).sum(-1, keepdim=True) - delta) * pd
    scale = d ** -0.5
    dQ = (torch.matmul(dS, K) + dSd * kd) * scale
    dK = torch.matmul(dS.transpose(-1, -2).contiguous(), q) * scale
    dV = torch.matmul(p.transpose(-1, -2).contiguous(), dO)
    s["dKc"].copy_(_to_channels(s, dK))
    s["dVc"].copy_(_to_channels(s, dV))
    s["dKd"].copy_(_to_channels(s, (dSd * q).sum((1, 3))) * scale)
    s["dVd"].copy_(_to_channels(s, (pd * dO).sum((1, 3))))
    s["dQ"].copy_(dQ.reshape(L, B, Hq, T, d))


def _plain_shared(s):
    c = s["c"]
    L, Hq, Hkv, d, B, T, P = (c[n] for n in ("L", "Hq", "Hkv", "d", "B", "T", "prefix"))
    G = Hq // Hkv
    q = s["Q"].float().reshape(L, B, Hkv, G * T, d)
    # the prefix once for the whole batch: its rows side by side
    qp = q.transpose(1, 2).reshape(L, Hkv, B * G * T, d)
    Kp, Vp = _by_layer(s, s["Kp"][:, :, :P]), _by_layer(s, s["Vp"][:, :, :P])
    xp = _scores(s, qp, Kp).reshape(L, Hkv, B, G * T, P).transpose(1, 2)
    (see,) = _causal_slots(s)
    see = see[:, None, None].expand(B, 1, G, T, s["S"]).reshape(B, 1, G * T, s["S"])
    x = _scores(s, q, _by_layer(s, s["Kc"])).masked_fill(~see, -math.inf)
    kd, vd = (_by_layer(s, s[n])[:, None, :, None] for n in ("Kd", "Vd"))
    xd = (q * kd).sum(-1, keepdim=True) * d ** -0.5
    if c["inclusive"]:
        xd = torch.full_like(xd, -math.inf)
    m = torch.maximum(torch.maximum(x.amax(-1, keepdim=True), xp.amax(-1, keepdim=True)), xd)
    x, xp, xd = (x - m).exp(), (xp - m).exp(), (xd - m).exp()
    total = x.sum(-1, keepdim=True) + xp.sum(-1, keepdim=True) + xd
    op = torch.matmul(xp.transpose(1, 2).reshape(L, Hkv, B * G * T, P), Vp)
    op = op.reshape(L, Hkv, B, G * T, d).transpose(1, 2)
    o = (torch.matmul(x, _by_layer(s, s["Vc"])) + op + xd * vd) / total
    s["O"].copy_(_token_major(c, o))


def _turned(x, by):
    """Keys x [..., d] turned by `by` [...] positions; the angles in 64 bits."""
    d = x.shape[-1]
    f = THETA ** (-2.0 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d)
    a = by.double()[..., None] * f
    cs, sn = a.cos().to(x.dtype), a.sin().to(x.dtype)
    x1, x2 = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([x1 * cs - x2 * sn, x2 * cs + x1 * sn], -1)


def _plain_evict(s):
    c = s["c"]
    keep, So, S = c["keep"], s["So"], s["S"]
    slot = torch.arange(S, device="cuda")
    ctx = s["ctx"].long()[:, None, None]  # [B, 1, 1] against [k, B, Hkv, S]
    n = ctx.clamp(max=keep)
    w = s["weight"]
    rank = torch.where((slot < c["first"]) | (slot >= ctx - c["recent"]) | (ctx <= keep),
                       math.inf, w)
    rank = torch.where(slot < ctx, rank, -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    j = torch.arange(keep, device="cuda")
    order = torch.where(j < n, order, S).sort(-1).values  # kept slots in ascending order
    took = (j < n).expand(order.shape)
    src = order.clamp(max=S - 1)
    rows = src[..., None].expand(*src.shape, c["d"])
    K = _turned(torch.gather(s["Kc"], 3, rows).float(), j - src)
    V = torch.gather(s["Vc"], 3, rows)
    s["Ko"][..., :keep, :] = torch.where(took[..., None], K.to(_dtype(c)), s["Ko"][..., :keep, :])
    s["Vo"][..., :keep, :] = torch.where(took[..., None], V, s["Vo"][..., :keep, :])
    s["weight_out"].zero_()
    s["weight_out"][..., :keep] = torch.where(took, torch.gather(w, 3, src), 0.0)
    s["ctx_out"].copy_(n.reshape(-1))
    s["kept"].copy_(torch.where(took, order, -1))


def _plain_share(s):
    c = s["c"]
    P, seq = c["prefix"], c["B"] - 1
    by = torch.full((P,), -P, device="cuda")
    s["Kp"].copy_(_turned(s["Kc"][:, seq, :, :P].float(), by))
    s["Vp"].copy_(s["Vc"][:, seq, :, :P])


def _plain(s):
    kind = s["c"]["kind"]
    if kind == "window":
        s["O"].copy_(_attend(s, *_window_slots(s))[0])
    elif kind == "grad":
        _plain_grad(s)
    elif kind == "shared":
        _plain_shared(s)
    elif kind == "share":
        _plain_share(s)
    elif kind == "weigh":
        c = s["c"]
        o, p, _ = _attend(s, *_causal_slots(s))
        s["O"].copy_(o)
        s["weight"] += _to_channels(s, p.sum(-2)).reshape(s["weight"].shape)
    else:
        _plain_evict(s)


# ------------------------------------------------------------ the framework's calls

def _own(s):
    wm, c, dims = s["wm"], s["c"], s["dims"]
    kind = c["kind"]
    if kind == "window":
        wm.channel_attend_window(dims, s["params"], s["Q"], s["map"], s["ctx"], c["window"],
                                 c["sinks"], s["Kc"], s["Vc"], s["O"], ws=s["ws"])
    elif kind == "grad":
        wm.channel_attend_window_backward(
            dims, s["params"], s["Q"], s["map"], s["ctx"], c["window"], c["sinks"], s["Kc"],
            s["Vc"], s["O"], s["dO"], s["dQ"], s["dKc"], s["dVc"], s["dKd"], s["dVd"],
            ws=s["ws"])
    elif kind == "shared":
        wm.channel_attend_shared(dims, s["params"], s["Q"], s["map"], s["ctx"], c["prefix"],
                                 s["Kp"], s["Vp"], s["Kc"], s["Vc"], s["O"], ws=s["ws"])
    elif kind == "share":
        wm.prefix_share(dims, s["Kc"], s["Vc"], c["B"] - 1, c["prefix"], s["Kp"], s["Vp"])
    elif kind == "weigh":
        wm.channel_attend_weigh(dims, s["params"], s["Q"], s["map"], s["ctx"], s["Kc"],
                                s["Vc"], s["O"], s["weight"], ws=s["ws"])
    else:
        wm.cache_evict(dims, s["ctx"], c["keep"], c["first"], c["recent"], s["weight"],
                       s["Kc"], s["Vc"], s["ctx_out"], s["weight_out"], s["Ko"], s["Vo"],
                       kept=s["kept"], ws=s["ws"])


OUTPUTS = {"window": ("O",), "grad": ("dQ", "dKc", "dVc", "dKd", "dVd"), "shared": ("O",),
           "share": ("Kp", "Vp"), "weigh": ("O", "weight"),
           "evict": ("Ko", "Vo", "weight_out", "ctx_out", "kept")}


def run(s):
    if own:
        _own(s)
    else:
        _plain(s)
    return {n: s[n] for n in OUTPUTS[s["c"]["kind"]]}


# -------------------------------------------------------------------- work

def work(case):
    c = case
    L, k, Hq, Hkv, d, B, T = (c[n] for n in ("L", "k", "Hq", "Hkv", "d", "B", "T"))
    es = 4 if c["dtype"] == "f32" else 2
    ctx = 0.75 * c["ctx"] if c["ragged"] else float(c["ctx"])
    row = Hkv * d * es  # one slot of one channel, keys or values
    if c["kind"] == "share":
        return {"bytes": 4.0 * k * c["prefix"] * row, "flops": 3.0 * k * c["prefix"] * Hkv * d}
    if c["kind"] == "evict":
        n = min(ctx, c["keep"])
        bytes_ = k * B * (4 * n * row + Hkv * 4 * (ctx + 2 * n))
        return {"bytes": float(bytes_), "flops": 3.0 * k * B * n * Hkv * d}
    # slots read: per row (flops), and in all (bytes)
    incl = 1 if c["inclusive"] else 0
    if c["kind"] in ("window", "grad"):
        span = c["window"] + c["sinks"]
        seen = sum(min(ctx + i + incl, span) for i in range(T))
        held = min(ctx + T - 1 + incl, span + T - 1)
    else:
        seen = sum(ctx + i + incl for i in range(T))
        held = ctx + T - 1 + incl
    rows = 2.0 * L * B * T * Hq * d * es  # queries and outputs
    attend = 4.0 * d * Hq * L * B * seen
    cache = 2.0 * k * B * held * row
    if c["kind"] == "grad":  # scores, dP, dV, dS K, dS Q; the written slots of both gradients
        written = 2.0 * k * B * Hkv * d * 4 * (ctx + T)
        return {"bytes": 1.5 * rows + rows / es * 2 + cache + written, "flops": 2.5 * attend}
    if c["kind"] == "shared":
        return {"bytes": rows + cache + 2.0 * k * c["prefix"] * row,
                "flops": attend + 4.0 * d * Hq * L * B * T * c["prefix"]}
    if c["kind"] == "weigh":
        return {"bytes": rows + cache + 8.0 * k * B * Hkv * held,
                "flops": attend + 2.0 * Hq * L * B * seen}
    return {"bytes": rows + cache, "flops": attend}


# ------------------------------------------------- the same from the definitions, 64 bits

def _exact_layer(c, s, l, reads):
    """Layer l over its channel: rows' weights over [prefix | cache] slots, the dummy's weight,
    and the values, all in 64 bits; reads(t, j): may the row at position t read cache slot j."""
    ch, G = l % c["k"], c["Hq"] // c["Hkv"]
    T, P, B = c["T"], c["prefix"], c["B"]
    K, V = s["Kc"][ch].double(), s["Vc"][ch].double()  # [B, Hkv, S, d]
    pos = s["ctx"].long()[:, None, None] + torch.arange(T, device="cuda")[:, None]
    may = reads(pos, torch.arange(s["S"], device="cuda"))  # [B, T, S]
    if P:
        K = torch.cat([s["Kp"][ch, :, :P].double().expand(B, -1, -1, -1), K], 2)
        V = torch.cat([s["Vp"][ch, :, :P].double().expand(B, -1, -1, -1), V], 2)
        may = torch.cat([torch.ones_like(may[..., :1]).expand(B, T, P), may], 2)
    K, V = K.repeat_interleave(G, 1), V.repeat_interleave(G, 1)  # [B, Hq, P + S, d]
    q = s["Q"][l].double()  # [B, Hq, T, d]
    kd = s["Kd"][ch].double().repeat_interleave(G, 0)[:, None]
    vd = s["Vd"][ch].double().repeat_interleave(G, 0)[:, None]
    z = torch.matmul(q, K.transpose(2, 3).contiguous()) / math.sqrt(c["d"])
    z = torch.where(may[:, None], z, -math.inf)
    zd = (q * kd).sum(3, keepdim=True) / math.sqrt(c["d"])
    if c["inclusive"]:
        zd = torch.full_like(zd, -math.inf)
    w = torch.softmax(torch.cat([z, zd], 3), 3)
    return q, K, V, kd, vd, w[..., :-1], w[..., -1:]


def _exact_attention(c, s, reads):
    L, k, Hq, Hkv, d, B, T = (c[n] for n in ("L", "k", "Hq", "Hkv", "d", "B", "T"))
    G, f64 = Hq // Hkv, dict(device="cuda", dtype=torch.float64)
    O = torch.empty((L, B, T, Hq * d), **f64)
    weight = s["weight"].double() if c["kind"] == "weigh" else None
    g = {}
    if c["kind"] == "grad":
        g = {"dQ": torch.empty((L, B, Hq, T, d), **f64),
             "dKc": torch.zeros((k, B, Hkv, s["S"], d), **f64),
             "dVc": torch.zeros((k, B, Hkv, s["S"], d), **f64),
             "dKd": torch.zeros((k, Hkv, d), **f64), "dVd": torch.zeros((k, Hkv, d), **f64)}
    for l in range(L):
        ch = l % k
        q, K, V, kd, vd, w, wd = _exact_layer(c, s, l, reads)
        if weight is not None:
            weight[ch] += w.reshape(B, Hkv, G * T, -1).sum(2)
        if not g:
            O[l] = (torch.matmul(w, V) + wd * vd).transpose(1, 2).reshape(B, T, Hq * d)
            continue
        dO, o = (s[n][l].double().reshape(B, T, Hq, d).transpose(1, 2) for n in ("dO", "O"))
        delta = (dO * o).sum(3, keepdim=True)
        ds = w * (torch.matmul(dO, V.transpose(2, 3).contiguous()) - delta) / math.sqrt(d)
        dsd = wd * ((dO * vd).sum(3, keepdim=True) - delta) / math.sqrt(d)
        g["dQ"][l] = torch.matmul(ds, K) + dsd * kd

        def heads(x):
            return x.reshape(B, Hkv, G, *x.shape[2:]).sum(2)

        g["dKc"][ch] += heads(torch.matmul(ds.transpose(2, 3).contiguous(), q))
        g["dVc"][ch] += heads(torch.matmul(w.transpose(2, 3).contiguous(), dO))
        g["dKd"][ch] += heads((dsd * q).sum(2, keepdim=True)).sum((0, 2))
        g["dVd"][ch] += heads((wd * dO).sum(2, keepdim=True)).sum((0, 2))
    if g:
        return g
    return {"O": O} if weight is None else {"O": O, "weight": weight}


def _exact_turn(x, delta):
    """x [n, d] by delta [n] positions, as complex numbers."""
    h = x.shape[-1] // 2
    freq = torch.exp(-math.log(THETA) / h * torch.arange(h, device="cuda", dtype=torch.float64))
    z = torch.complex(x[:, :h].double(), x[:, h:].double())
    z = z * torch.polar(torch.ones_like(z.real), delta.double()[:, None] * freq)
    return torch.cat([z.real, z.imag], 1)


def _exact_evict(c, s):
    k, Hkv, d, B, keep, So = (*(c[n] for n in ("k", "Hkv", "d", "B", "keep")), s["So"])
    f64 = dict(device="cuda", dtype=torch.float64)
    Ko, Vo = torch.zeros((k, B, Hkv, So, d), **f64), torch.zeros((k, B, Hkv, So, d), **f64)
    W = torch.zeros((k, B, Hkv, So), **f64)
    kept = torch.full((k, B, Hkv, keep), -1, device="cuda", dtype=torch.int32)
    lens = s["ctx"].tolist()
    for b, n in enumerate(lens):
        to = torch.arange(min(n, keep), device="cuda")
        for ch in range(k):
            for h in range(Hkv):
                src = to
                if n > keep:
                    lo, hi = c["first"], max(c["first"], n - c["recent"])
                    more = keep - lo - (n - hi)
                    by = torch.argsort(-s["weight"][ch, b, h, lo:hi].double(), stable=True)
                    src = torch.cat([to[:lo], lo + by[:more].sort().values,
                                     torch.arange(hi, n, device="cuda")])
                m = len(src)
                Ko[ch, b, h, :m] = _exact_turn(s["Kc"][ch, b, h, src], to - src)
                Vo[ch, b, h, :m] = s["Vc"][ch, b, h, src].double()
                W[ch, b, h, :m] = s["weight"][ch, b, h, src].double()
                kept[ch, b, h, :m] = src.to(torch.int32)
    ctx = torch.tensor([min(n, keep) for n in lens], device="cuda", dtype=torch.int32)
    return {"Ko": Ko, "Vo": Vo, "weight_out": W, "ctx_out": ctx, "kept": kept}


def exact(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    incl = 1 if c["inclusive"] else 0
    if c["kind"] == "share":
        P = c["prefix"]
        by = torch.full((P,), -P, device="cuda")
        Kp = torch.stack([torch.stack([_exact_turn(s["Kc"][j, -1, h, :P], by)
                                       for h in range(c["Hkv"])]) for j in range(c["k"])])
        return {"Kp": Kp, "Vp": s["Vc"][:, -1, :, :P].double()}
    if c["kind"] == "evict":
        return _exact_evict(c, s)
    if c["kind"] in ("window", "grad"):
        def reads(t, j):
            return (j < t + incl) & ((j >= t + incl - c["window"]) | (j < c["sinks"]))
        if c["kind"] == "grad":
            _attention_output(s)
    else:
        def reads(t, j):
            return j < t + incl
    return _exact_attention(c, s, reads)
