"""How many bits the memory operators keep with bfloat16 tensors: as many as fp32 arithmetic on them, up to the result's own rounding.

M is the result's sum of products with every factor's magnitude in its place.  Sums, states and decays are fp32: (2 * tokens + dims + 24)
roundings of 2^-24 on the way of a term, of M at most.  On the way into a product, a weighted score or the state that is read out is two
bfloat16 terms, which leave 2^-8 of 2^-8 of it: 2^-16 M.  The result is rounded once: 2^-8 of it.
"""
import numpy as np
import pytest
import torch

import memory_reference as ref
import paper_1611_06256_amd as g

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
CASES = [
    # lens, heads, key, value, states, starts, decay
    ([700], 2, 64, 64, True, None, [0.998, 0.9]),                     # spans
    ([300, 64, 65, 1], 3, 128, 128, True, 0.01, [0.99, 0.75, 1.0]),
    ([90, 200], 2, 48, 128, False, None, [0.97, 0.999]),
    ([130, 129], 2, 128, 40, True, 0.02, [0.97, 0.999]),
    ([5, 3, 0, 5, 5], 2, 16, 32, True, 0.2, [0.75, 0.99]),            # token by token
]


def inputs(case, seed=11):
    lens, h, dk, dv, states, starts, decay = case
    gen, n = torch.Generator().manual_seed(seed), sum(lens)
    s = {name: torch.randn(n, h, d, generator=gen).to(BF16) for name, d in (("q", dk), ("k", dk), ("v", dv), ("dout", dv))}
    s["starts"] = (torch.rand(n, generator=gen) < starts).to(torch.uint8) if starts else None
    for name in ("state_in", "dstate_out"):
        s[name] = torch.randn(len(lens), h, dv, dk, generator=gen) if states else None
    return s


def results(case, s, handed):
    """out, dq, dk, dv; handed: the states and their gradient are asked for, too, and come behind them."""
    lens, h, dk, dv, _, _, decay = case
    d = {k: None if v is None else v.cuda() for k, v in s.items()}
    table = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    got = [torch.full(s[x].shape, float("nan"), dtype=BF16, device="cuda") for x in ("v", "q", "k", "v")]
    states = [torch.full((len(lens), h, dv, dk), float("nan"), device="cuda") if handed else None for _ in range(2)]
    kw = dict(seg_start=table, starts=d["starts"], state_in=d["state_in"], scale=dk ** -0.5)
    g.decay_attention(d["q"], d["k"], d["v"], decay, got[0], state_out=states[0], **kw)
    g.decay_attention_grad(d["q"], d["k"], d["v"], decay, d["dout"], *got[1:], dstate_out=d["dstate_out"], dstate_in=states[1], **kw)
    torch.cuda.synchronize()
    return got + ([x for x in states] if handed else [])


@pytest.mark.parametrize("case", range(len(CASES)))
def test_results_are_those_of_fp32_arithmetic(case):
    print(f"rounding case {case}", flush=True)
    case = CASES[case]
    lens, h, dk, dv, _, _, decay = case
    s = inputs(case)
    got = results(case, s, False)
    exact, size = [], []
    for to, f in ((exact, lambda t: t.double()), (size, lambda t: t.double().abs())):
        w = {k: f(v) if v is not None and k != "starts" else v for k, v in s.items()}
        to.append(ref.attention(w["q"], w["k"], w["v"], decay, lens, w["starts"], w["state_in"], dk ** -0.5)[0])
        to += ref.attention_grad(w["q"], w["k"], w["v"], decay, lens, w["dout"], w["starts"], w["state_in"], w["dstate_out"], dk ** -0.5)[:3]
    factors = 2 * max(lens) + dk + dv + 24
    for what, a, x, m in zip(("out", "dq", "dk", "dv"), got, exact, size):
        over = (a.double().cpu() - x).abs() - (2.0 ** -8 * x.abs() + (2.0 ** -16 + factors * 2.0 ** -24) * m)
        assert not (over > 0).any() and torch.isfinite(a).all(), f"{what}: {int((over > 0).sum())} of {over.numel()}, {float(over.max()):.3g} more than allowed"


@pytest.mark.parametrize("case", range(len(CASES)))
def test_asking_for_states_changes_no_result(case):
    print(f"states case {case}", flush=True)
    case = CASES[case]
    s = inputs(case)
    for what, a, b in zip(("out", "dq", "dk", "dv"), results(case, s, False), results(case, s, True)):
        assert torch.equal(a, b), what
