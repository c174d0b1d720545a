"""The memory operators where a call is large enough for the variants that small ones do not take: states past the caches, spans' states
four numbers at a time, and a second direction's that lie behind an odd number of the first one's.

M is a result's sum of products with every factor's magnitude in its place; bounds are those of fp32 sums, (2 * tokens + dims + 24) *
2^-24 * M, and with bfloat16 tensors 2^-8 of the result and 2^-16 * M more."""
import ctypes as C

import pytest
import torch

import paper_1611_06256_amd as g
from paper_1611_06256_amd import binding

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def near(got, want, size, factors, what, dtype=F32):
    tol = factors * 2.0 ** -24 * size
    if dtype == BF16:
        tol = tol + 2.0 ** -8 * want.abs() + 2.0 ** -16 * size
    over = ((got.double() - want).abs() - tol).max()
    assert torch.isfinite(got).all() and float(over) <= 1e-30, f"{what}: {float(over):.3g} more than allowed"


def exact(s, decay, scale, f):
    """out, the state behind, dq, dk, dv and the gradient of the first state, of [segments, tokens, heads, .] segments of equal length
    in 64 bits by the recurrence; f is what goes over each input first."""
    q, k, v, do, x, gx = (f(s[n].double()) for n in ("q", "k", "v", "dout", "state_in", "dstate_out"))
    d, new = torch.tensor(decay, dtype=F32).double().cuda()[None, :, None, None], s["starts"].bool()[..., None, None, None]
    out, dq, dk, dv = torch.empty_like(v), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    for t in range(q.shape[1]):
        x = torch.where(new[:, t], torch.zeros_like(x), x) * d + v[:, t, :, :, None] * k[:, t, :, None, :]
        out[:, t] = scale * (x * q[:, t, :, None, :]).sum(-1)
        dq[:, t] = scale * (x * do[:, t, :, :, None]).sum(-2)
    for t in reversed(range(q.shape[1])):
        here = gx + scale * do[:, t, :, :, None] * q[:, t, :, None, :]
        dk[:, t] = (here * v[:, t, :, :, None]).sum(-2)
        dv[:, t] = (here * k[:, t, :, None, :]).sum(-1)
        gx = torch.where(new[:, t], torch.zeros_like(here), here * d)
    return {"out": out, "state": x, "dq": dq, "dk": dk, "dv": dv, "dstate": gx}


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("segments,tokens,heads,dk,dv", [(11, 500, 3, 128, 128), (43, 500, 3, 64, 64), (58, 600, 3, 64, 48)])
def test_many_large_states_between_spans(segments, tokens, heads, dk, dv, dtype):
    print(f"large {segments} {tokens} {heads} {dk} {dv} {dtype}", flush=True)
    decay, scale, n = [0.99, 0.9, 0.999], dk ** -0.5, segments * tokens
    host = (C.c_float * heads)(*decay)
    d = binding._DecayDesc(heads, dk, dv, int(dtype == BF16), C.cast(host, C.POINTER(C.c_float)), scale)
    scratch = g.load_library().ga3c_decay_attention_workspace(C.byref(d), segments, n, 1)
    places = scratch // (8 * (dk * dv + 1))
    # the second direction's states begin behind a number of floats that is no multiple of four, were a number kept behind each state;
    # segments have several spans
    assert places % heads == 0 and places % 4 and n // (places // heads) < tokens
    assert 2 * segments * heads * dk * dv >= 1 << 20
    gen = torch.Generator(device="cuda").manual_seed(7)
    s = {name: torch.randn(segments, tokens, heads, w, generator=gen, device="cuda").to(dtype)
         for name, w in (("q", dk), ("k", dk), ("v", dv), ("dout", dv))}
    for name in ("state_in", "dstate_out"):
        s[name] = torch.randn(segments, heads, dv, dk, generator=gen, device="cuda")
    s["starts"] = (torch.rand(segments, tokens, generator=gen, device="cuda") < 0.002).to(torch.uint8)
    flat = {k: v.flatten(0, 1) if v.dim() == 4 and not k.startswith(("state", "dstate")) else v for k, v in s.items()}
    got = {k: torch.full((n, heads, w), float("nan"), dtype=dtype, device="cuda") for k, w in (("out", dv), ("dq", dk), ("dk", dk), ("dv", dv))}
    got.update({k: torch.full_like(s["state_in"], float("nan")) for k in ("state", "dstate")})
    kw = dict(segments=segments, starts=s["starts"].flatten(), state_in=s["state_in"], scale=scale)
    g.decay_attention(flat["q"], flat["k"], flat["v"], decay, got["out"], state_out=got["state"], **kw)
    g.decay_attention_grad(flat["q"], flat["k"], flat["v"], decay, flat["dout"], got["dq"], got["dk"], got["dv"], dstate_out=s["dstate_out"],
                           dstate_in=got["dstate"], **kw)
    torch.cuda.synchronize()
    want, size = (exact(s, decay, scale, f) for f in (lambda t: t, torch.abs))
    for what in got:
        near(got[what].view(want[what].shape), want[what], size[what], 2 * tokens + dk + dv + 24, what, F32 if "state" in what else dtype)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,slots,heads,dk,dv", [(300, 330, 16, 64, 64), (150, 151, 8, 128, 128), (1100, 1100, 8, 20, 100)])
def test_steps_of_states_past_the_caches(n, slots, heads, dk, dv, dtype):
    """A slot twice and three times, padded entries, starts."""
    print(f"steps {n} {slots} {heads} {dk} {dv} {dtype}", flush=True)
    assert n * heads * dk * dv * 4 >= 64 << 20
    gen = torch.Generator(device="cuda").manual_seed(n)
    decay, scale = [0.5 + 0.5 * i / (heads - 1) for i in range(heads)], dk ** -0.5
    states = torch.randn(slots, heads, dv, dk, generator=gen, device="cuda")
    q, k, v = (torch.randn(n, heads, w, generator=gen, device="cuda").to(dtype) for w in (dk, dk, dv))
    where = torch.randperm(slots, generator=gen, device="cuda")[:n].to(torch.int32)
    where[7], where[n // 2], where[n - 1] = -1, where[3], where[3]
    where[20], where[n - 2] = slots, where[11]
    starts = (torch.rand(n, generator=gen, device="cuda") < 0.1).to(torch.uint8)
    starts[n // 2] = 0
    kept, size = states.double(), states.double().abs()
    out = torch.full((n, heads, dv), float("nan"), dtype=dtype, device="cuda")
    g.decay_attention_step(q, k, v, decay, states, out, slots=where, starts=starts, scale=scale)
    torch.cuda.synchronize()
    d = torch.tensor(decay, dtype=F32).double().cuda()[:, None, None]
    want, mag = (torch.empty(n, heads, dv, dtype=torch.float64, device="cuda") for _ in range(2))
    for i, (at, new) in enumerate(zip(where.tolist(), starts.tolist())):
        for x, to, f in ((kept, want, lambda t: t), (size, mag, torch.abs)):
            a, b, c = (f(t[i].double()) for t in (q, k, v))
            st = (x[at] * d if 0 <= at < slots and not new else 0) + c[:, :, None] * b[:, None, :]
            to[i] = scale * (st * a[:, None, :]).sum(-1)
            if 0 <= at < slots:
                x[at] = st
    near(out, want, mag, 2 * 3 + dk + 24, "out", dtype)
    near(states, kept, size, 2 * 3 + 24, "states")
