"""The operators of an agent's memory, as cases that can be timed: attention with a decay for each head, and group norm.

Kinds of case:

  step           one token of each agent of a prediction batch, whose states lie in slots (``decay_attention_step``)
  segments       packed sequences of unequal length, an update's segments or whole prompts (``decay_attention``)
  segments_grad  the gradient of that (``decay_attention_grad``)
  norm           group norm with an activation, channels last (``group_norm``)
  norm_grad      its gradient (``group_norm_grad``)

``own`` False computes them in their plain form, in 32 bits; True calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

T_MAX = 5
EPS = 1e-5


def _step(name, agents, slots, heads, key, value, dtype):
    return {"name": name, "kind": "step", "agents": agents, "slots": slots, "heads": heads, "key": key, "value": value,
            "dtype": dtype}


def _segments(name, kind, segments, tokens, heads, key, value, dtype, states, starts):
    """tokens: of all segments together; states: whether segments begin in a given state and hand one on (or its gradient
    back); starts: share of the tokens at which an episode begins."""
    return {"name": name, "kind": kind, "segments": segments, "tokens": tokens, "heads": heads, "key": key, "value": value,
            "dtype": dtype, "states": states, "starts": starts}


def _norm(name, kind, samples, positions, channels, groups, act, dtype):
    return {"name": name, "kind": kind, "samples": samples, "positions": positions, "channels": channels, "groups": groups,
            "act": act, "dtype": dtype}


def listed():
    return [
        # one agent that plays alone: the latency of a call
        _step("step 1 agent f32", 1, 64, 4, 16, 32, "f32"),
        # a full prediction batch of a wide memory
        _step("step 512 agents bf16", 512, 1024, 16, 64, 64, "bf16"),
        # an update of 512 agents, five steps or fewer each, with the memory of a 256-unit net
        _segments("segments 512x5 f32", "segments", 512, 2301, 4, 16, 32, "f32", True, 0.02),
        # one long prompt
        _segments("prompt 16384 bf16", "segments", 1, 16384, 8, 128, 128, "bf16", False, 0.0),
        # whole episodes of uneven length, head sizes that are no power of two
        _segments("episodes 24 f32", "segments", 24, 6001, 6, 48, 80, "f32", True, 0.001),
        # the gradient of the update above
        _segments("segments 512x5 grad f32", "segments_grad", 512, 2301, 4, 16, 32, "f32", True, 0.02),
        # training on packed episodes
        _segments("episodes 16 grad bf16", "segments_grad", 16, 8190, 8, 64, 64, "bf16", False, 0.001),
        # training on one long sequence
        _segments("sequence 4096 grad f32", "segments_grad", 1, 4096, 4, 128, 128, "f32", True, 0.0),
        # what the memory of the 256-unit net reads out in an update
        _norm("norm 2560 tokens f32", "norm", 2560, 1, 128, 4, "relu", "f32"),
        # maps of 32x32
        _norm("norm 64 maps bf16", "norm", 64, 1024, 512, 32, "silu", "bf16"),
        # a wide memory's read-out in training
        _norm("norm grad 8192 tokens bf16", "norm_grad", 8192, 1, 1024, 16, "silu", "bf16"),
        # maps of 9x9, an odd number of frames, no activation
        _norm("norm grad 37 maps f32", "norm_grad", 37, 81, 96, 8, "none", "f32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))


def draw(rng):
    kind = rng.choice(["step", "step", "segments", "segments", "segments", "segments_grad", "segments_grad", "segments_grad",
                       "norm", "norm", "norm_grad", "norm_grad"])
    dtype = rng.choice(["f32", "bf16"])
    if kind in ("norm", "norm_grad"):
        groups, wide = _log(rng, 1, 32), _log(rng, 2, 128)
        channels = groups * wide
        samples = _log(rng, 1, 8192)
        positions = 1 if rng.random() < 0.5 else _log(rng, 2, 1024)
        positions = max(1, min(positions, (1 << 24) // (samples * channels)))
        # the rectifier's gradient jumps where its argument crosses zero
        act = rng.choice(["none", "relu", "silu"] if kind == "norm" else ["none", "silu"])
        c = _norm("", kind, samples, positions, channels, groups, act, dtype)
    else:
        heads = _log(rng, 1, 16)
        key, value = (rng.choice([16, 32, 64, 128, rng.randint(8, 128)]) for _ in range(2))
        if kind == "step":
            agents = _log(rng, 1, 512)
            c = _step("", agents, agents + _log(rng, 1, 512), heads, key, value, dtype)
        else:
            tokens = min(_log(rng, 8, 8192), int(math.sqrt(5e8 / heads)))
            segments = min(_log(rng, 1, 512), max(1, (1 << 24) // (heads * key * value)))
            if segments > tokens:
                tokens = segments * T_MAX * 9 // 10
            c = _segments("", kind, segments, tokens, heads, key, value, dtype, rng.random() < 0.5,
                          rng.choice([0.0, 0.0, 0.002, 0.05]))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs --

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _lengths(case, seed):
    """Lengths of the segments, some of them short; a seed's own cuts."""
    n, tokens = case["segments"], case["tokens"]
    r = np.random.default_rng(seed)
    if n == 1:
        return np.array([tokens])
    if tokens <= n * T_MAX:
        left = np.full(n, T_MAX)                       # t_max steps each, but for those whose episode ended
        while left.sum() > tokens:
            at = r.integers(0, n, size=left.sum() - tokens)
            np.subtract.at(left, at, 1)
            np.maximum(left, 0, out=left)
        return left
    cuts = np.sort(r.integers(0, tokens + 1, size=n - 1))
    return np.diff(np.concatenate([[0], cuts, [tokens]]))


def _decay(heads):
    """From a quarter lost per step to half a percent."""
    return [1.0 - 2.0 ** -(2.0 + 5.5 * h / max(1, heads - 1)) for h in range(heads)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DTYPE[case["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    s = {"case": case}
    if case["kind"] in ("norm", "norm_grad"):
        n, p, c, g = (case[k] for k in ("samples", "positions", "channels", "groups"))
        s["x"] = (torch.randn(n, p, c, generator=gen, device="cuda") * 1.5 + torch.randn(c, generator=gen, device="cuda")).to(dt)
        s["gamma"] = 1 + 0.2 * normal(c, dtype=torch.float32)
        s["beta"] = 0.2 * normal(c, dtype=torch.float32)
        s["y"] = torch.empty_like(s["x"])
        s["stats"] = torch.empty(n, g, 2, device="cuda")
        if case["kind"] == "norm_grad":
            s["dy"] = normal(n, p, c)
            x = s["x"].double().view(n, p, g, c // g)
            mean, var = x.mean((1, 3)), x.var((1, 3), unbiased=False)
            s["stats"].copy_(torch.stack([mean, 1 / torch.sqrt(var + EPS)], -1))      # as the forward pass leaves them
            s["dgamma"], s["dbeta"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        torch.cuda.synchronize()
        return s
    h, dk, dv = case["heads"], case["key"], case["value"]
    s["decay"], s["scale"] = _decay(h), dk ** -0.5
    if case["kind"] == "step":
        b = case["agents"]
        s["q"], s["k"], s["v"] = normal(b, h, dk), normal(b, h, dk), normal(b, h, dv)
        s["states"] = normal(case["slots"], h, dv, dk, dtype=torch.float32)
        s["slots"] = torch.randperm(case["slots"], generator=gen, device="cuda")[:b].to(torch.int32)
        s["starts"] = (torch.rand(b, generator=gen, device="cuda") < 0.02).to(torch.uint8)
        s["out"] = torch.empty(b, h, dv, dtype=dt, device="cuda")
    else:
        n, t = case["segments"], case["tokens"]
        s["q"], s["k"], s["v"] = normal(t, h, dk), normal(t, h, dk), normal(t, h, dv)
        s["seg_start"] = torch.from_numpy(np.concatenate([[0], np.cumsum(_lengths(case, seed))]).astype(np.int32)).cuda()
        s["starts"] = (torch.rand(t, generator=gen, device="cuda") < case["starts"]).to(torch.uint8) if case["starts"] else None
        s["state_in"] = normal(n, h, dv, dk, dtype=torch.float32) if case["states"] else None
        if case["kind"] == "segments":
            s["out"] = torch.empty(t, h, dv, dtype=dt, device="cuda")
            s["state_out"] = torch.empty(n, h, dv, dk, device="cuda") if case["states"] else None
        else:
            s["dout"] = normal(t, h, dv)
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[k]) for k in ("q", "k", "v"))
            s["dstate_out"] = normal(n, h, dv, dk, dtype=torch.float32) if case["states"] else None
            s["dstate_in"] = torch.empty(n, h, dv, dk, device="cuda") if case["states"] else None
    torch.cuda.synchronize()
    return s


# -------------------------------------------------------------- plain forms --

def _powers(s, count):
    """decay[h] ** i for i < count, [heads, count]; in 64 bits, because the exponents are long."""
    d = torch.tensor(s["decay"], dtype=torch.float32, device="cuda").double()
    return torch.pow(d[:, None], torch.arange(count, device="cuda").double()).float()


def _runs(s):
    """Of every token: its segment, its position there, the number of its episode, and whether its segment's first state still
    counts.  An episode begins with a segment and at a start."""
    t, start = s["q"].shape[0], s["seg_start"].long()
    at = torch.arange(t, device="cuda")
    seg = torch.searchsorted(start[1:].contiguous(), at, right=True)
    first = start[seg]
    begun = s["starts"].long().cumsum(0) if s["starts"] is not None else torch.zeros_like(at)
    before = torch.where(first > 0, begun[(first - 1).clamp(min=0)], torch.zeros_like(begun))      # starts in earlier segments
    return seg, at - first, seg * (t + 1) + begun, begun == before


def _weights(s):
    """[heads, t, t]: decay ** (i - j) where token i sees token j, else 0."""
    t = s["q"].shape[0]
    _, _, run, _ = _runs(s)
    at = torch.arange(t, device="cuda")
    ago = at[:, None] - at[None, :]
    sees = (ago >= 0) & (run[:, None] == run[None, :])
    return _powers(s, t)[:, ago.clamp(min=0)] * sees


def _by_head(x):
    return x.float().transpose(0, 1).contiguous()                        # [heads, t, d]


def _tokens_of(x, dtype):
    return x.transpose(0, 1).to(dtype).contiguous()                      # [t, heads, d]


def _plain_segments(s):
    q, k, v, dt = _by_head(s["q"]), _by_head(s["k"]), _by_head(s["v"]), s["out"].dtype
    t, n = s["q"].shape[0], s["seg_start"].numel() - 1
    w = _weights(s)
    o = torch.matmul(torch.matmul(q, k.transpose(1, 2).contiguous()) * w, v)
    if s["state_in"] is None:
        return {"out": _tokens_of(o * s["scale"], dt)}
    seg, pos, run, fresh = _runs(s)
    p = _powers(s, t + 1)
    # the state that a segment began with: o_i += decay^(i+1) state q_i
    seen = torch.matmul(s["state_in"][seg], s["q"].float()[..., None])[..., 0].transpose(0, 1)      # [heads, t, dv]
    o = o + seen * (p[:, pos + 1] * fresh)[..., None]
    # the state that it hands on: what its last token sees
    last = (s["seg_start"][1:].long() - 1).clamp(min=0)
    length = s["seg_start"].diff().long()
    some = (length > 0)
    kw = w[:, last] * some[None, :, None]                                 # [heads, n, t]
    state = torch.zeros_like(s["state_in"]).transpose(0, 1).contiguous()      # [heads, n, dv, dk]
    tok = torch.arange(t, device="cuda")
    each = kw[:, seg, tok]                                                # decay ** (last - j) of token j, [heads, t]
    state.index_add_(1, seg, (v * each[..., None])[..., :, None] * k[..., None, :])
    kept = torch.where(some, fresh[last], torch.ones_like(some))
    state = state.transpose(0, 1) + s["state_in"] * (p[:, length].transpose(0, 1) * kept[:, None])[..., None, None]
    return {"out": _tokens_of(o * s["scale"], dt), "state_out": state.contiguous()}


def _plain_segments_grad(s):
    q, k, v, do, dt = _by_head(s["q"]), _by_head(s["k"]), _by_head(s["v"]), _by_head(s["dout"]) * s["scale"], s["dq"].dtype
    t = s["q"].shape[0]
    w = _weights(s)
    ds = torch.matmul(do, v.transpose(1, 2).contiguous()) * w             # gradient of the weighted scores
    sc = torch.matmul(q, k.transpose(1, 2).contiguous()) * w
    dq, dk, dv = torch.matmul(ds, k), torch.matmul(ds.transpose(1, 2).contiguous(), q), torch.matmul(sc.transpose(1, 2).contiguous(), do)
    if s["state_in"] is None:
        return {"dq": _tokens_of(dq, dt), "dk": _tokens_of(dk, dt), "dv": _tokens_of(dv, dt)}
    seg, pos, run, fresh = _runs(s)
    p = _powers(s, t + 1)
    begun = (p[:, pos + 1] * fresh)[..., None]                            # weight of the state that the segment began with
    dq = dq + torch.matmul(do.transpose(0, 1)[..., None, :], s["state_in"][seg])[..., 0, :].transpose(0, 1) * begun
    length, n = s["seg_start"].diff().long(), s["seg_start"].numel() - 1
    some = length > 0
    dstate = torch.zeros_like(s["state_in"]).transpose(0, 1).contiguous()
    dstate.index_add_(1, seg, (do * begun)[..., :, None] * q[..., None, :])
    last = (s["seg_start"][1:].long() - 1).clamp(min=0)
    kept = torch.where(some, fresh[last], torch.ones_like(some))
    handed = s["dstate_out"] * (p[:, length].transpose(0, 1) * kept[:, None])[..., None, None]
    # the state handed on: token j's share of it is decay ** (last - j) if its episode lasts that long
    each = (p[:, last[seg] - torch.arange(t, device="cuda")] * (run == run[last[seg]])).transpose(0, 1)[..., None]      # [t, heads, 1]
    g = s["dstate_out"][seg]                                              # [t, heads, dv, dk]
    dv = dv + (torch.matmul(g, s["k"].float()[..., None])[..., 0] * each).transpose(0, 1)
    dk = dk + (torch.matmul(s["v"].float()[..., None, :], g)[..., 0, :] * each).transpose(0, 1)
    return {"dq": _tokens_of(dq, dt), "dk": _tokens_of(dk, dt), "dv": _tokens_of(dv, dt),
            "dstate_in": (dstate.transpose(0, 1) + handed).contiguous()}


def _plain_step(s):
    d = torch.tensor(s["decay"], dtype=torch.float32, device="cuda")[None, :, None, None]
    at = s["slots"].long()
    state = s["states"][at] * (s["starts"] == 0)[:, None, None, None]
    state = state * d + s["v"].float()[..., :, None] * s["k"].float()[..., None, :]
    s["states"][at] = state
    o = (state * s["q"].float()[..., None, :]).sum(-1) * s["scale"]
    return {"out": o.to(s["out"].dtype), "states": s["states"]}


def _plain_norm(s):
    c = s["case"]
    n, p, ch, g = s["x"].shape[0], s["x"].shape[1], s["x"].shape[2], c["groups"]
    x = s["x"].float().view(n, p, g, ch // g)
    mean = x.mean((1, 3), keepdim=True)
    off = x - mean
    rstd = 1 / torch.sqrt((off * off).mean((1, 3), keepdim=True) + EPS)
    z = (off * rstd).view(n, p, ch) * s["gamma"] + s["beta"]
    y = torch.where(z > 0, z, torch.zeros_like(z)) if c["act"] == "relu" else z / (1 + torch.exp(-z)) if c["act"] == "silu" else z
    return {"y": y.to(s["x"].dtype), "stats": torch.stack([mean, rstd], -1).view(n, g, 2)}


def _plain_norm_grad(s):
    c = s["case"]
    n, p, ch, g = s["x"].shape[0], s["x"].shape[1], s["x"].shape[2], c["groups"]
    mean, rstd = s["stats"][..., 0].view(n, 1, g, 1), s["stats"][..., 1].view(n, 1, g, 1)
    xh = (s["x"].float().view(n, p, g, ch // g) - mean) * rstd
    dz = s["dy"].float()
    if c["act"] == "silu":
        z = xh.view(n, p, ch) * s["gamma"] + s["beta"]
        sig = 1 / (1 + torch.exp(-z))
        dz = dz * sig * (1 + z * (1 - sig))
    dgamma, dbeta = (dz * xh.view(n, p, ch)).sum((0, 1)), dz.sum((0, 1))
    d = (dz * s["gamma"]).view(n, p, g, ch // g)
    dx = rstd * (d - d.mean((1, 3), keepdim=True) - xh * (d * xh).mean((1, 3), keepdim=True))
    return {"dx": dx.view(n, p, ch).to(s["x"].dtype), "dgamma": dgamma, "dbeta": dbeta}


# --------------------------------------------------------------- the passes --

def _own(s):
    import paper_1611_06256_amd as g
    kind, c = s["case"]["kind"], s["case"]
    if kind == "step":
        g.decay_attention_step(s["q"], s["k"], s["v"], s["decay"], s["states"], s["out"], slots=s["slots"], starts=s["starts"],
                               scale=s["scale"])
        return {"out": s["out"], "states": s["states"]}
    if kind == "segments":
        g.decay_attention(s["q"], s["k"], s["v"], s["decay"], s["out"], seg_start=s["seg_start"], starts=s["starts"],
                          state_in=s["state_in"], state_out=s["state_out"], scale=s["scale"])
        return {k: s[k] for k in ("out", "state_out") if s[k] is not None}
    if kind == "segments_grad":
        g.decay_attention_grad(s["q"], s["k"], s["v"], s["decay"], s["dout"], s["dq"], s["dk"], s["dv"], seg_start=s["seg_start"],
                               starts=s["starts"], state_in=s["state_in"], dstate_out=s["dstate_out"], dstate_in=s["dstate_in"],
                               scale=s["scale"])
        return {k: s[k] for k in ("dq", "dk", "dv", "dstate_in") if s[k] is not None}
    if kind == "norm":
        g.group_norm(s["x"], s["gamma"], s["beta"], c["groups"], s["y"], stats=s["stats"], act=c["act"], eps=EPS)
        return {"y": s["y"], "stats": s["stats"]}
    g.group_norm_grad(s["x"], s["dy"], s["gamma"], s["beta"], s["stats"], c["groups"], s["y"], s["dgamma"], s["dbeta"], act=c["act"])
    return {"dx": s["y"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


_PLAIN = {"step": _plain_step, "segments": _plain_segments, "segments_grad": _plain_segments_grad, "norm": _plain_norm,
          "norm_grad": _plain_norm_grad}


def run(s):
    return _own(s) if own else _PLAIN[s["case"]["kind"]](s)


# ------------------------------------------------------- what a pass takes --

def work(case):
    kind, size = case["kind"], 4 if case["dtype"] == "f32" else 2
    if kind in ("norm", "norm_grad"):
        elements = case["samples"] * case["positions"] * case["channels"]
        small = 8 * case["samples"] * case["groups"] + 8 * case["channels"]
        if kind == "norm":
            return {"bytes": 2 * elements * size + small, "flops": 10 * elements}
        return {"bytes": 3 * elements * size + small + 8 * case["channels"], "flops": 20 * elements}
    h, dk, dv = case["heads"], case["key"], case["value"]
    if kind == "step":
        b = case["agents"]
        return {"bytes": b * h * (8 * dk * dv + 2 * size * (dk + dv)) + 5 * b, "flops": 4 * b * h * dk * dv}
    t, n = case["tokens"], case["segments"]
    flags = 4 * (n + 1) + (t if case["starts"] else 0)
    state = 4 * n * h * dk * dv
    # the state takes a token up and is read out once for each output
    if kind == "segments":
        return {"bytes": t * h * 2 * (dk + dv) * size + flags + (2 * state if case["states"] else 0), "flops": 4 * t * h * dk * dv}
    return {"bytes": t * h * (4 * dk + 3 * dv) * size + flags + (3 * state if case["states"] else 0), "flops": 10 * t * h * dk * dv}


# ------------------------------------------------------------------- exact --

def _walk(s, backwards=False):
    """Of the t-th token of every segment, from the first on or from the last back: which one it is, and which segments have one."""
    start = s["seg_start"].long()
    length = start.diff()
    for t in range(int(length.max())):
        there = t < length
        yield torch.where(there, (start[1:] - 1 - t) if backwards else start[:-1] + t, torch.zeros_like(length)), there


def _scatter(to, at, there, x):
    to[at[there]] = x[there]


def _exact_segments(s, grad):
    """Token by token, by the recurrence, in 64 bits."""
    q, k, v = (s[x].double() for x in "qkv")
    n, (t, h, dk), dv = s["seg_start"].numel() - 1, q.shape, v.shape[2]
    d = torch.tensor(s["decay"], dtype=torch.float32, device="cuda").double()[None, :, None, None]
    new = s["starts"].bool() if s["starts"] is not None else torch.zeros(t, dtype=torch.bool, device="cuda")
    state = s["state_in"].double() if s["state_in"] is not None else torch.zeros(n, h, dv, dk, dtype=torch.float64, device="cuda")
    by = s["dout"].double() if grad else None
    got = torch.zeros(t, h, dk if grad else dv, dtype=torch.float64, device="cuda")
    for at, there in _walk(s):
        kept = torch.where(new[at][:, None, None, None], torch.zeros_like(state), state)
        kept = kept * d + v[at][..., None] * k[at][..., None, :]
        state = torch.where(there[:, None, None, None], kept, state)
        o = (state * by[at][..., None]).sum(-2) if grad else (state * q[at][..., None, :]).sum(-1)
        _scatter(got, at, there, o * s["scale"])
    if not grad:
        return {"out": got, **({"state_out": state} if s["state_out"] is not None else {})}
    # back: g is the gradient of the state behind a token
    g = s["dstate_out"].double() if s["dstate_out"] is not None else torch.zeros_like(state)
    dk_, dv_ = torch.zeros_like(k), torch.zeros_like(v)
    for at, there in _walk(s, True):
        here = g + s["scale"] * by[at][..., None] * q[at][..., None, :]
        _scatter(dk_, at, there, (here * v[at][..., None]).sum(-2))
        _scatter(dv_, at, there, (here * k[at][..., None, :]).sum(-1))
        here = torch.where(new[at][:, None, None, None], torch.zeros_like(g), here * d)
        g = torch.where(there[:, None, None, None], here, g)
    return {"dq": got, "dk": dk_, "dv": dv_, **({"dstate_in": g} if s["dstate_in"] is not None else {})}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "segments":
        return _exact_segments(s, False)
    if kind == "segments_grad":
        return _exact_segments(s, True)
    if kind == "step":
        q, k, v, states = (s[x].double() for x in ("q", "k", "v", "states"))
        d = torch.tensor(s["decay"], dtype=torch.float32, device="cuda").double()
        out = torch.zeros(q.shape[0], q.shape[1], v.shape[2], dtype=torch.float64, device="cuda")
        for i, (at, new) in enumerate(zip(s["slots"].tolist(), s["starts"].tolist())):
            states[at] = (0 if new else d[:, None, None] * states[at]) + v[i][:, :, None] * k[i][:, None, :]
            out[i] = s["scale"] * (states[at] * q[i][:, None, :]).sum(-1)
        return {"out": out, "states": states}
    n, p, c = s["x"].shape
    g = case["groups"]
    x = s["x"].double().view(n, p, g, c // g).permute(0, 2, 1, 3).reshape(n, g, -1)            # a row for each group
    gamma, beta = (s[w].double().view(1, g, 1, c // g).expand(1, g, p, c // g).reshape(1, g, -1) for w in ("gamma", "beta"))

    def back(y):
        return y.view(n, g, p, c // g).permute(0, 2, 1, 3).reshape(n, p, c)

    if kind == "norm":
        var, mean = torch.var_mean(x, 2, unbiased=False)
        rstd = (var + EPS) ** -0.5
    else:
        mean, rstd = s["stats"][..., 0].double(), s["stats"][..., 1].double()
    xh = (x - mean[..., None]) * rstd[..., None]
    z = xh * gamma + beta
    if kind == "norm":
        y = {"none": z, "relu": z.clamp(min=0), "silu": z * torch.sigmoid(z)}[case["act"]]
        return {"y": back(y), "stats": torch.stack([mean, rstd], -1)}
    dz = s["dy"].double().view(n, p, g, c // g).permute(0, 2, 1, 3).reshape(n, g, -1)
    if case["act"] == "silu":
        dz = dz * torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    e = dz * gamma
    dx = (e - e.mean(2, keepdim=True) - xh * (e * xh).mean(2, keepdim=True)) * rstd[..., None]
    return {"dx": back(dx), "dgamma": back(dz * xh).sum((0, 1)), "dbeta": back(dz).sum((0, 1))}
