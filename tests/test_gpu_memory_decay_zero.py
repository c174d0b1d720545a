"""Decays of which nothing, or nothing that is a number, is left within a tile, with tokens that are not finite: they reach what they
are part of and nothing else, the same token by token and chunked.  With a decay of zero a token is part of its own output and, the last
one of a segment, of the state behind it; with any other decay of all that comes behind, however small its share.

Bounds of what stays finite as for fp32 sums: (2 * tokens + dims + 24) * 2^-24 of the sum of magnitudes, with bfloat16 tensors 2^-8 of
the result and 2^-16 of the sum more."""
import pytest
import torch

import paper_1611_06256_amd as g

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
DECAY = [0.0, 0.05, 1e-30]


def walk(s, f):
    """out, state behind, dq, dk, dv and the gradient of the first state, token by token in 64 bits, what is decayed by zero being zero."""
    q, k, v, do, x, g_ = (f(s[n].double()) for n in ("q", "k", "v", "dout", "state_in", "dstate_out"))
    d = torch.tensor(DECAY, dtype=F32).double()[:, None, None]

    def faded(x):
        return torch.where(d == 0, torch.zeros_like(x), x * d)

    out, dq, dk, dv = torch.empty_like(v), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    for t in range(q.shape[0]):
        x = faded(torch.zeros_like(x) if s["starts"][t] else x) + v[t][:, :, None] * k[t][:, None, :]
        out[t], dq[t] = (x * q[t][:, None, :]).sum(-1), (x * do[t][:, :, None]).sum(-2)
    for t in reversed(range(q.shape[0])):
        here = g_ + do[t][:, :, None] * q[t][:, None, :]
        dk[t], dv[t] = (here * v[t][:, :, None]).sum(-2), (here * k[t][:, None, :]).sum(-1)
        g_ = torch.zeros_like(here) if s["starts"][t] else faded(here)
    return {"out": out, "state": x, "dq": dq, "dk": dk, "dv": dv, "dstate": g_}


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("at", ["first", "last"])
@pytest.mark.parametrize("starts", [False, True], ids=["", "starts"])
@pytest.mark.parametrize("n", [11, 65, 90, 600])
def test_numbers_that_are_not_finite_at_small_decays(n, starts, at, dtype):
    print(f"decay zero {n} {starts} {at} {dtype}", flush=True)
    h, dk, dv = len(DECAY), 16, 16
    gen = torch.Generator().manual_seed(n)
    s = {name: torch.randn(n, h, w, generator=gen).to(dtype) for name, w in (("q", dk), ("k", dk), ("v", dv), ("dout", dv))}
    for name in ("state_in", "dstate_out"):
        s[name] = torch.randn(1, h, dv, dk, generator=gen)[0]
    s["starts"] = torch.zeros(n, dtype=torch.uint8)
    if starts:
        s["starts"][[n // 3, n // 2]] = 1
    first = 1 if at == "first" else n - 5
    for i, (name, bad) in enumerate((("k", float("inf")), ("v", float("nan")), ("q", float("-inf")), ("dout", float("inf")))):
        s[name][first + i, :, 3 + i] = bad
    want, size = walk(s, lambda t: t), walk(s, torch.abs)
    d = {k: v.cuda() for k, v in s.items()}
    got = {k: torch.full(want[k].shape, 7.0, dtype=dtype, device="cuda") for k in ("out", "dq", "dk", "dv")}
    got.update({k: torch.full((1, h, dv, dk), 7.0, device="cuda") for k in ("state", "dstate")})
    kw = dict(starts=d["starts"], state_in=d["state_in"][None].contiguous())
    g.decay_attention(d["q"], d["k"], d["v"], DECAY, got["out"], state_out=got["state"], **kw)
    g.decay_attention_grad(d["q"], d["k"], d["v"], DECAY, d["dout"], got["dq"], got["dk"], got["dv"], dstate_out=d["dstate_out"][None].contiguous(),
                           dstate_in=got["dstate"], **kw)
    torch.cuda.synchronize()
    for what, a in got.items():
        a, b, m = a.double().cpu().view(want[what].shape), want[what], size[what]
        there = torch.isfinite(b)
        assert torch.equal(torch.isfinite(a), there), f"{what}: {int((torch.isfinite(a) != there).sum())} of {a.numel()} finite or not where they should not be"
        tol = (2 * n + dk + dv + 24) * 2.0 ** -24 * m + 1e-30
        if dtype == BF16 and "state" not in what:
            tol = tol + 2.0 ** -8 * b.abs() + 2.0 ** -16 * m
        assert bool(((a - b).abs() <= tol)[there].all()), f"{what}: {float((a - b).abs()[there].max()):.3g} off"
