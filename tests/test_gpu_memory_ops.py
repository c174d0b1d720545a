"""The memory operators on the GPU against their plain forms in 64 bits.

Tolerances.  A result is a sum of products; M is the same sum with every factor's magnitude in its place.  A term passes at most one
rounding per token that its state is carried over, one per element of the sum that it is read out with, and a handful in its factors
(decays are powers: an exponent's rounding is worth up to as many again as the token is far), so fp32 results are within
(2 * tokens + dims + 24) * 2^-24 * M.  With bfloat16 tensors the result's own rounding adds 2^-8 of it, and up to three factors of a
term (weighted score, carried state, key with its decay) may be rounded to bfloat16: 3 * 2^-8 * M.  States are fp32 with either.
"""
import numpy as np
import pytest
import torch

import memory_reference as ref
import paper_1611_06256_amd as g

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
STEP = 2.0 ** -24


def near(got, want, size, factors, what, dtype=F32):
    """factors: roundings of fp32 on the way of a term."""
    tol = factors * STEP * size
    if dtype == BF16:
        tol = tol + 2.0 ** -8 * want.abs() + 3 * 2.0 ** -8 * size
    off = (got.detach().double().cpu() - want).abs()
    assert torch.isfinite(got).all(), what
    over = (off - tol).max().item() if off.numel() else -1.0
    assert over <= 1e-30, f"{what}: {off.max().item():.3g} off, {over:.3g} more than allowed"


def make(lens, h, dk, dv, dtype, states, starts, fused, seed=3):
    gen = torch.Generator().manual_seed(seed)
    n = sum(lens)

    def normal(*shape, dt=dtype):
        return torch.randn(*shape, generator=gen).to(dt)

    if fused:                 # slices of one matrix, odd distances between the heads
        m = normal(n, h * (2 * dk + dv) + 3).cuda()
        q, k = (m[:, i * h * dk:(i + 1) * h * dk].unflatten(1, (h, dk)) for i in range(2))
        v = m[:, 2 * h * dk:2 * h * dk + h * dv].unflatten(1, (h, dv))
    else:
        q, k, v = normal(n, h, dk).cuda(), normal(n, h, dk).cuda(), normal(n, h, dv).cuda()
    s = {"q": q, "k": k, "v": v, "dout": normal(n, h, dv).cuda(),
         "starts": (torch.rand(n, generator=gen) < starts).to(torch.uint8).cuda() if starts is not None else None}
    for name in ("state_in", "dstate_out"):
        s[name] = normal(len(lens), h, dv, dk, dt=F32).cuda() if states else None
    s["seg_start"] = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()
    return s


def wide(t):
    return None if t is None else t.detach().double().cpu()


CASES = [
    # lens, heads, key, value, states, starts, decay, fused
    ([1], 1, 1, 1, False, None, [0.5], False),
    ([1], 3, 16, 32, True, None, [0.25, 0.9, 1.0], False),
    ([5, 5, 3, 0, 1, 5, 2, 5], 4, 16, 32, True, 0.2, [0.75, 0.9, 0.99, 1.0], True),
    ([0, 0, 7, 0], 2, 3, 5, True, 0.3, [0.0, 1.0], False),
    ([63, 64, 65], 2, 17, 33, False, None, [0.97, 0.5], False),
    ([130], 2, 64, 64, True, 1.0, [0.9, 0.99], False),              # every token begins an episode
    ([31, 100, 1, 200], 3, 48, 80, True, 0.02, [0.9, 0.99, 0.999], True),
    ([257], 2, 128, 128, True, None, [0.995, 0.9], False),
    ([300, 20], 1, 128, 16, False, 0.01, [1.0], False),
    ([90, 33], 2, 8, 127, True, 0.05, [0.0, 0.98], False),
    ([700], 1, 32, 64, True, 0.002, [0.998], False),
    ([1100, 3, 900], 2, 64, 48, True, 0.001, [0.99, 0.9995], False),
    ([1] * 60 + [300] + [2] * 40, 2, 32, 16, True, 0.01, [0.97, 0.5], False),      # short ones and a long one
    ([1, 2, 3, 70, 4, 0], 3, 100, 20, False, None, [0.9, 0.8, 1.0], True),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_and_its_gradient(case, dtype):
    print(f"attention case {case} {dtype}", flush=True)
    check_attention(CASES[case], dtype)


def check_attention(case, dtype):
    lens, h, dk, dv, states, starts, decay, fused = case
    s = make(lens, h, dk, dv, dtype, states, starts, fused)
    n, segs, scale = sum(lens), len(lens), dk ** -0.5
    out = torch.full((n, h, dv), float("nan"), dtype=dtype, device="cuda")
    state_out = torch.full((segs, h, dv, dk), float("nan"), device="cuda")
    g.decay_attention(s["q"], s["k"], s["v"], decay, out, seg_start=s["seg_start"], starts=s["starts"], state_in=s["state_in"],
                      state_out=state_out, scale=scale)
    only = torch.full_like(out, float("nan"))                 # without the states behind the segments
    g.decay_attention(s["q"], s["k"], s["v"], decay, only, seg_start=s["seg_start"], starts=s["starts"], state_in=s["state_in"], scale=scale)
    dq, dk_, dv_ = (torch.full(s[x].shape, float("nan"), dtype=dtype, device="cuda") for x in "qkv")
    dstate = torch.full_like(state_out, float("nan"))
    g.decay_attention_grad(s["q"], s["k"], s["v"], decay, s["dout"], dq, dk_, dv_, seg_start=s["seg_start"], starts=s["starts"],
                           state_in=s["state_in"], dstate_out=s["dstate_out"], dstate_in=dstate, scale=scale)
    torch.cuda.synchronize()

    w = {k: wide(v) for k, v in s.items()}
    size = {k: v.abs() if v is not None and k not in ("starts", "seg_start") else v for k, v in w.items()}
    factors = 2 * max(lens) + dk + dv + 24
    want = ref.attention(w["q"], w["k"], w["v"], decay, lens, w["starts"], w["state_in"], scale)
    mags = ref.attention(size["q"], size["k"], size["v"], decay, lens, w["starts"], size["state_in"], scale)
    near(out, want[0], mags[0], factors, "out", dtype)
    near(only, want[0], mags[0], factors, "out alone", dtype)
    near(state_out, want[1], mags[1], factors, "state_out")
    want = ref.attention_grad(w["q"], w["k"], w["v"], decay, lens, w["dout"], w["starts"], w["state_in"], w["dstate_out"], scale)
    mags = ref.attention_grad(size["q"], size["k"], size["v"], decay, lens, size["dout"], w["starts"], size["state_in"], size["dstate_out"], scale)
    for got, a, m, what in zip((dq, dk_, dv_), want, mags, ("dq", "dk", "dv")):
        near(got, a, m, factors, what, dtype)
    near(dstate, want[3], mags[3], factors, "dstate_in")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(62, 30), (30, 126), (114, 61), (126, 90)])
def test_rows_of_whole_words_and_odd_ones(dk, dv, dtype):
    """Sizes that are no multiple of 16 bytes, on tiles that are full, end early, and are cut by starts."""
    print(f"attention {dk} {dv} {dtype}", flush=True)
    check_attention(([64, 300, 33, 129], 2, dk, dv, True, 0.01, [0.5, 0.99], False), dtype)


def test_gradient_against_differences():
    lens, h, dk, dv, decay, scale = [37, 5, 90], 2, 24, 40, [0.9, 0.99], 0.2
    s = make(lens, h, dk, dv, F32, True, 0.03, False, seed=5)
    dq, dk_, dv_, ds = (torch.empty_like(s[x]) for x in ("q", "k", "v", "state_in"))
    g.decay_attention_grad(s["q"], s["k"], s["v"], decay, s["dout"], dq, dk_, dv_, seg_start=s["seg_start"], starts=s["starts"],
                           state_in=s["state_in"], dstate_out=s["dstate_out"], dstate_in=ds, scale=scale)
    torch.cuda.synchronize()
    w = {k: wide(v) for k, v in s.items()}

    def loss(x):
        o, st = ref.attention(x["q"], x["k"], x["v"], decay, lens, w["starts"], x["state_in"], scale)
        return float((o * w["dout"]).sum() + (st * w["dstate_out"]).sum())

    gen = torch.Generator().manual_seed(6)
    for name, grad in (("q", dq), ("k", dk_), ("v", dv_), ("state_in", ds)):
        way = torch.randn(w[name].shape, generator=gen, dtype=torch.float64)
        ends = [loss({**w, name: w[name] + e * way}) for e in (1e-4, -1e-4)]       # quadratic at most in each: no error of the step
        got = wide(grad)
        assert abs((ends[0] - ends[1]) / 2e-4 - float((got * way).sum())) <= 400 * STEP * float((got * way).abs().sum()) + 1e-7, name


def test_equal_segments_need_no_table():
    lens, h, dk, dv, decay = [6] * 7, 2, 16, 16, [0.9, 0.8]
    s = make(lens, h, dk, dv, F32, True, 0.1, False)
    got = [[torch.empty(42, h, dv, device="cuda"), torch.empty(7, h, dv, dk, device="cuda")] for _ in range(2)]
    for (o, st), kw in zip(got, (dict(seg_start=s["seg_start"]), dict(segments=7))):
        g.decay_attention(s["q"], s["k"], s["v"], decay, o, starts=s["starts"], state_in=s["state_in"], state_out=st, **kw)
    torch.cuda.synchronize()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_a_start_hides_whatever_came_before():
    # infinities and NaN in the state and in tokens of an earlier episode do not reach a later one
    h, dk, dv, decay = 2, 32, 32, [0.9, 0.0]
    for lens in ([40], [200]):
        cut = lens[0] // 2
        s = make(lens, h, dk, dv, F32, True, None, False)
        starts = torch.zeros(lens[0], dtype=torch.uint8, device="cuda")
        starts[cut] = 1
        clean = [torch.empty(lens[0], h, dv, device="cuda"), torch.empty(1, h, dv, dk, device="cuda")]
        g.decay_attention(s["q"], s["k"], s["v"], decay, clean[0], starts=starts, state_in=s["state_in"], state_out=clean[1])
        s["state_in"][0, 0, 3, 4] = float("inf")
        s["state_in"][0, 1, 0, 0] = float("nan")
        got = [torch.empty_like(x) for x in clean]
        g.decay_attention(s["q"], s["k"], s["v"], decay, got[0], starts=starts, state_in=s["state_in"], state_out=got[1])
        torch.cuda.synchronize()
        assert torch.equal(got[0][cut:], clean[0][cut:]) and torch.equal(got[1], clean[1])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens", [[20], [90], [600]], ids=["20", "90", "600"])
def test_numbers_that_are_not_finite_stay_where_they_belong(lens, dtype):
    # a token that is not finite reaches neither the tokens before it nor, past a start, those behind it; nor other segments
    lens = lens + [17]
    h, dk, dv, decay, n = 2, 32, 48, [0.9, 0.99], lens[0]
    bad, cut = n // 3, n // 2
    s = make(lens, h, dk, dv, dtype, True, None, False)
    s["starts"] = torch.zeros(sum(lens), dtype=torch.uint8, device="cuda")
    s["starts"][cut] = 1
    w = {k: wide(v) for k, v in s.items()}
    size = {k: v.abs() if k not in ("starts", "seg_start") else v for k, v in w.items()}
    s["v"][bad, 0, 5] = float("inf")
    s["k"][bad + 1, 1, 7] = float("nan")
    s["q"][bad + 2, 0, 3] = float("nan")
    s["dout"][bad + 3, 1, 2] = float("-inf")
    out, state = torch.empty(sum(lens), h, dv, dtype=dtype, device="cuda"), torch.empty(2, h, dv, dk, device="cuda")
    kw = dict(seg_start=s["seg_start"], starts=s["starts"], state_in=s["state_in"])
    g.decay_attention(s["q"], s["k"], s["v"], decay, out, state_out=state, **kw)
    grads = [torch.empty_like(s[x]) for x in "qkv"] + [torch.empty_like(state)]
    g.decay_attention_grad(s["q"], s["k"], s["v"], decay, s["dout"], *grads[:3], dstate_out=s["dstate_out"], dstate_in=grads[3], **kw)
    torch.cuda.synchronize()
    factors = 2 * n + dk + dv + 24
    want = ref.attention(w["q"], w["k"], w["v"], decay, lens, w["starts"], w["state_in"])
    mags = ref.attention(size["q"], size["k"], size["v"], decay, lens, w["starts"], size["state_in"])
    for part in (slice(0, bad), slice(cut, None)):
        near(out[part], want[0][part], mags[0][part], factors, f"out {part}", dtype)
    near(state, want[1], mags[1], factors, "state_out")
    assert not torch.isfinite(out[bad]).all()
    want = ref.attention_grad(w["q"], w["k"], w["v"], decay, lens, w["dout"], w["starts"], w["state_in"], w["dstate_out"])
    mags = ref.attention_grad(size["q"], size["k"], size["v"], decay, lens, size["dout"], w["starts"], size["state_in"], size["dstate_out"])
    for got, a, m, what in zip(grads, want, mags, ("dq", "dk", "dv")):
        near(got[cut:], a[cut:], m[cut:], factors, what, dtype)
        if what == "dq":
            near(got[:bad], a[:bad], m[:bad], factors, what, dtype)
    near(grads[3][1], want[3][1], mags[3][1], factors, "dstate_in")


def test_a_bad_table_stays_within_the_arrays():
    # what lies behind the arrays is the test's own
    h, dk, dv, n = 2, 16, 16, 50
    s = make([n], h, dk, dv, F32, True, None, False)
    room = torch.full((n + 64, h, dv), 7.0, device="cuda")
    for table in ([0, 30, 20, 50], [-5, 10, 900, 50], [60, 70, 80, 90], [10, 5, 0, -1]):
        t = torch.tensor(table, dtype=torch.int32, device="cuda")
        st = torch.zeros(3, h, dv, dk, device="cuda")
        g.decay_attention(s["q"], s["k"], s["v"], [0.9, 0.5], room[:n], seg_start=t, state_out=st)
        torch.cuda.synchronize()
        assert bool((room[n:] == 7.0).all()), table


# ------------------------------------------------------------------- single tokens --

@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens", [[4, 1, 0, 9], [300, 700, 0, 65]], ids=["short", "long"])
def test_rows_outside_the_segments_are_left_as_they_were(lens, dtype):
    front, rear, h, dk, dv, decay = 7, 140, 3, 32, 48, [0.5, 0.95, 0.99]
    s = make([front] + lens + [rear], h, dk, dv, dtype, False, 0.02, False)
    n, end = front + sum(lens) + rear, front + sum(lens)
    inside = torch.tensor([front], dtype=torch.int32, device="cuda") + torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()
    for k in ("q", "k", "v", "dout"):         # what lies there is nobody's
        s[k][:front] = float("nan")
        s[k][end:] = float("inf")
    e = lambda d: torch.full((n, h, d), 7.0, dtype=dtype, device="cuda")  # noqa: E731
    got = [e(dv), e(dk), e(dk), e(dv)]
    g.decay_attention(s["q"], s["k"], s["v"], decay, got[0], seg_start=inside, starts=s["starts"])
    g.decay_attention_grad(s["q"], s["k"], s["v"], decay, s["dout"], *got[1:], seg_start=inside, starts=s["starts"])
    part = {k: s[k][front:end].contiguous() for k in ("q", "k", "v", "dout", "starts")}
    want = [t[front:end].clone() for t in (e(dv), e(dk), e(dk), e(dv))]
    g.decay_attention(part["q"], part["k"], part["v"], decay, want[0], seg_start=inside - front, starts=part["starts"])
    g.decay_attention_grad(part["q"], part["k"], part["v"], decay, part["dout"], *want[1:], seg_start=inside - front, starts=part["starts"])
    torch.cuda.synchronize()
    args = [wide(part[x]) for x in ("q", "k", "v", "dout")]
    factors = 2 * max(lens) + max(dk, dv) + 24
    exact, size = [], []
    for x, to in ((args, exact), ([t.abs() for t in args], size)):
        to.append(ref.attention(*x[:3], decay, lens, wide(part["starts"]))[0])
        to += ref.attention_grad(*x[:3], decay, lens, x[3], wide(part["starts"]))[:3]
    for what, a, b, x, m in zip(("out", "dq", "dk", "dv"), got, want, exact, size):
        assert bool((a[:front] == 7).all()) and bool((a[end:] == 7).all()), what
        near(a[front:end], x, m, factors, what, dtype)
        near(b, x, m, factors, what, dtype)


def test_two_calls_at_once_on_two_streams():
    lens, h, dk, dv, decay = [3000, 900, 5000], 4, 64, 64, [0.9, 0.97, 0.99, 0.999]
    sets = [make(lens, h, dk, dv, F32, True, 0.001, False, seed=i) for i in range(2)]
    n = sum(lens)

    def run(s, stream=None):
        e = lambda d: torch.empty(n, h, d, device="cuda")  # noqa: E731
        out = [e(dv), e(dk), e(dk), e(dv), torch.empty_like(s["state_in"]), torch.empty_like(s["state_in"])]
        torch.cuda.synchronize()
        seg = dict(seg_start=s["seg_start"], starts=s["starts"], state_in=s["state_in"], stream=stream)

        def go():
            g.decay_attention(s["q"], s["k"], s["v"], decay, out[0], state_out=out[4], **seg)
            g.decay_attention_grad(s["q"], s["k"], s["v"], decay, s["dout"], *out[1:4], dstate_out=s["dstate_out"], dstate_in=out[5], **seg)
        return go, out
    alone = [run(s) for s in sets]
    for go, _ in alone:
        go()
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    both = [run(s, stream) for s, stream in zip(sets, streams)]
    for _ in range(4):
        for go, _ in both:
            go()
    torch.cuda.synchronize()
    for (_, a), (_, b) in zip(alone, both):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_single_token_of_a_wide_matrix():
    """One token's distance to the next is nobody's business."""
    h, dk, dv = 2, 8, 8
    m = torch.randn(1, h * (2 * dk + dv), generator=torch.Generator().manual_seed(5)).cuda()
    q, k, v = (t.unflatten(1, (h, 8)).as_strided((1, h, 8), (1 << 30, 8, 1)) for t in (m[:, :16], m[:, 16:32], m[:, 32:]))
    out, state = torch.empty(1, h, dv, device="cuda"), torch.empty(1, h, dv, dk, device="cuda")
    g.decay_attention(q, k, v, [0.5, 0.9], out, state_out=state)
    torch.cuda.synchronize()
    want = wide(v)[0][:, :, None] * wide(k)[0][:, None, :]
    assert float((wide(state)[0] - want).abs().max()) <= 1e-6 * float(want.abs().max())
    assert float((wide(out)[0] - (want @ wide(q)[0][:, :, None])[..., 0]).abs().max()) <= 1e-5 * float(want.abs().max())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,slots,h,dk,dv", [(1, 1, 1, 1, 1), (1, 5, 4, 16, 32), (7, 20, 2, 17, 33), (33, 64, 3, 64, 64), (64, 64, 2, 128, 128),
                                             (300, 400, 2, 48, 80)])
def test_steps(n, slots, h, dk, dv, dtype):
    print(f"step {n} {slots} {h} {dk} {dv} {dtype}", flush=True)
    gen = torch.Generator().manual_seed(n)
    decay, scale = [0.5 + 0.5 * i / max(1, h - 1) for i in range(h)], dk ** -0.5
    states = torch.randn(slots, h, dv, dk, generator=gen)
    kept, dev = states.double(), states.cuda()
    size = kept.abs()
    for step in range(3):
        q, k, v = (torch.randn(n, h, d, generator=gen).to(dtype) for d in (dk, dk, dv))
        where = torch.randperm(slots, generator=gen)[:n].to(torch.int32)
        starts = (torch.rand(n, generator=gen) < 0.2).to(torch.uint8) if step else None
        out = torch.full((n, h, dv), float("nan"), dtype=dtype, device="cuda")
        g.decay_attention_step(q.cuda(), k.cuda(), v.cuda(), decay, dev, out, slots=where.cuda(), starts=None if starts is None else starts.cuda(),
                               scale=scale)
        torch.cuda.synchronize()
        at = where.long()
        want, st = ref.attention(q.double(), k.double(), v.double(), decay, [1] * n, starts, kept[at], scale)
        mag, sz = ref.attention(q.double().abs(), k.double().abs(), v.double().abs(), decay, [1] * n, starts, size[at], scale)
        kept[at], size[at] = st, sz
        near(out, want, mag, 2 * 3 + dk + 24, "out", dtype)
        near(dev, kept, size, 2 * 3 + 24, "states")             # those of no token too: as they were


def test_steps_with_one_slot_several_times_padded_entries_and_no_slots():
    gen = torch.Generator().manual_seed(9)
    h, dk, dv, slots, n, decay = 2, 16, 32, 6, 11, [0.9, 0.6]
    where = [2, -1, 0, 2, 6, 2, 0, 5, 1000000, 2, -7]
    states = torch.randn(slots, h, dv, dk, generator=gen)
    q, k, v = (torch.randn(n, h, d, generator=gen) for d in (dk, dk, dv))
    starts = torch.tensor([0, 0, 0, 0, 1, 1, 0, 0, 0, 0, 0], dtype=torch.uint8)
    dev, out = states.cuda(), torch.empty(n, h, dv, device="cuda")
    g.decay_attention_step(q.cuda(), k.cuda(), v.cuda(), decay, dev, out, slots=torch.tensor(where, dtype=torch.int32).cuda(), starts=starts.cuda())
    torch.cuda.synchronize()
    kept, size = states.double(), states.double().abs()
    for i, at in enumerate(where):
        there = 0 <= at < slots
        zero = torch.zeros(1, h, dv, dk, dtype=torch.float64)
        args = [x[i:i + 1].double() for x in (q, k, v)]
        o, st = ref.attention(*args, decay, [1], starts[i:i + 1], kept[at:at + 1] if there else zero)
        m, sz = ref.attention(*[x.abs() for x in args], decay, [1], starts[i:i + 1], size[at:at + 1] if there else zero)
        near(out[i:i + 1], o, m, 2 * 4 + dk + 24, f"entry {i}")
        if there:
            kept[at], size[at] = st[0], sz[0]
    near(dev, kept, size, 2 * 4 + 24, "states")
    # without slots token i has state i; the states behind the last token stay as they are
    dev2, out2 = states.cuda(), torch.empty(4, h, dv, device="cuda")
    dev3, out3 = states.cuda(), torch.empty(4, h, dv, device="cuda")
    args = [x[:4].cuda() for x in (q, k, v)]
    g.decay_attention_step(*args, decay, dev2, out2)
    g.decay_attention_step(*args, decay, dev3, out3, slots=torch.arange(4, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(out2, out3) and torch.equal(dev2, dev3) and torch.equal(dev2[4:].cpu(), states[4:])


def test_steps_are_the_segments_of_an_update():
    # an agent's tokens one by one, and all at once: the same memory
    gen = torch.Generator().manual_seed(12)
    n, t, h, dk, dv, decay = 5, 9, 4, 16, 32, [0.7, 0.9, 0.97, 0.99]
    q, k, v = (torch.randn(n, t, h, d, generator=gen).cuda() for d in (dk, dk, dv))
    starts = (torch.rand(n, t, generator=gen) < 0.2).to(torch.uint8).cuda()
    first = torch.randn(n, h, dv, dk, generator=gen).cuda()
    states, outs = first.clone(), []
    for i in range(t):
        o = torch.empty(n, h, dv, device="cuda")
        g.decay_attention_step(q[:, i], k[:, i], v[:, i], decay, states, o, starts=starts[:, i].contiguous(), scale=0.25)
        outs.append(o)
    out, last = torch.empty(n * t, h, dv, device="cuda"), torch.empty_like(first)
    g.decay_attention(*[x.flatten(0, 1) for x in (q, k, v)], decay, out, segments=n, starts=starts.flatten(), state_in=first, state_out=last, scale=0.25)
    torch.cuda.synchronize()
    a, b = torch.stack(outs, 1).flatten(0, 1), out
    assert float((a - b).abs().max()) <= 2 * (2 * t + dk + 24) * STEP * float(dk * t * 9)       # each within its bound of the exact one
    assert float((states - last).abs().max()) <= 2 * (2 * t + 24) * STEP * float(t * 16)


# ---------------------------------------------------------------------- group norm --

def norm_near(got, want, tol, what, dtype):
    if dtype == BF16:
        tol = tol + 2.0 ** -8 * want.abs()
    off = (got.double().cpu() - want).abs()
    assert torch.isfinite(got).all(), what
    assert bool((off <= tol).all()), f"{what}: {float(off.max()):.3g} off, {float((off - tol).max()):.3g} more than allowed"


NORMS = [
    # samples, positions, channels, groups
    (1, 1, 1, 1), (1, 1, 6, 3), (3, 1, 128, 4), (257, 1, 128, 4), (5, 1, 1024, 16), (40, 1, 96, 1), (2, 81, 96, 8), (3, 400, 32, 32),
    (2, 17, 33, 11), (1, 1024, 64, 2), (2, 5000, 16, 4), (1, 3, 4099, 1), (7, 4, 8, 8), (130, 1, 250, 5), (2, 36, 512, 32), (1, 1, 8192, 2),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", NORMS, ids=[f"{'x'.join(map(str, s))}" for s in NORMS])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_group_norm_and_its_gradient(shape, act, dtype):
    n, p, c, groups = shape
    print(f"norm {shape} {act} {dtype}", flush=True)
    gen = torch.Generator().manual_seed(n * p + c)
    x = (2 * torch.randn(n, p, c, generator=gen) + torch.randn(c, generator=gen)).to(dtype)
    gamma, beta = 1 + 0.3 * torch.randn(c, generator=gen), 0.3 * torch.randn(c, generator=gen)
    eps = 1e-3
    # a row holds the channels and 5 elements of somebody else's
    room = torch.full((n, p, c + 5), 3.0, dtype=dtype, device="cuda")
    xr = room.clone()
    xr[..., :c] = x.cuda()
    y, stats = room.clone(), torch.empty(n, groups, 2, device="cuda")
    g.group_norm(xr[..., :c], gamma.cuda(), beta.cuda(), groups, y[..., :c], stats=stats, act=act, eps=eps)
    torch.cuda.synchronize()
    xd = x.double()
    mean, rstd, xh = ref.norm_parts(xd, groups, eps)
    z = xh * gamma.double() + beta.double()
    # a mean is a sum of m numbers by 64 threads or more; an element's distance from it has the rounding of both
    m = p * (c // groups)
    k = (m / 64 + 16) * STEP
    each = (c // groups,)
    spread = xd.abs().view(n, p, groups, -1).mean((1, 3))[:, None, :, None].expand(n, p, groups, *each).reshape(n, p, c)
    r = rstd[:, None, :, None].expand(n, p, groups, *each).reshape(n, p, c)
    xh_tol = k * (spread + xd.abs()) * r + 2 * k * xh.abs() * (1 + (spread * r) ** 2 * k)
    tol = 1.2 * (xh_tol * gamma.double().abs() + 8 * STEP * (z.abs() + beta.double().abs()))
    norm_near(y[..., :c], ref.activation(z, act), tol, "y", dtype)
    assert bool((y[..., c:] == 3.0).all())
    norm_near(stats[..., 0], mean, k * xd.abs().view(n, p, groups, -1).mean((1, 3)), "mean", F32)
    norm_near(stats[..., 1], rstd, 2 * k * rstd * (1 + k * (xd.abs().view(n, p, groups, -1).mean((1, 3)) * rstd) ** 2), "rstd", F32)

    dy = torch.randn(n, p, c, generator=gen)
    dy[z.abs() < 1e-3 * (1 + z.abs())] = 0          # the rectifier's gradient jumps at zero
    dy = dy.to(dtype)
    dyr, dx = room.clone(), room.clone()
    dyr[..., :c] = dy.cuda()
    dgamma, dbeta = torch.full((c,), float("nan"), device="cuda"), torch.full((c,), float("nan"), device="cuda")
    g.group_norm_grad(xr[..., :c], dyr[..., :c], gamma.cuda(), beta.cuda(), stats, groups, dx[..., :c], dgamma, dbeta, act=act)
    torch.cuda.synchronize()
    leaves = [t.double().clone().requires_grad_() for t in (xd, gamma, beta)]
    want = torch.autograd.grad((ref.group_norm(*leaves, groups, act, eps) * dy.double()).sum(), leaves)
    zl = z.clone().requires_grad_()
    dz = torch.autograd.grad((ref.activation(zl, act) * dy.double()).sum(), zl)[0]
    d = dz * gamma.double()
    # the slope of an activation changes by at most half of what its argument does
    d_tol = 4 * STEP * d.abs() + 0.5 * (tol if act == "silu" else 0 * tol) * (dy.double() * gamma.double()).abs()

    def of_group(t):
        return t.view(n, p, groups, -1).mean((1, 3))[:, None, :, None].expand(n, p, groups, *each).reshape(n, p, c)

    a_tol = of_group(d_tol) + k * of_group(d.abs())
    b_tol = of_group(d_tol * xh.abs() + d.abs() * xh_tol) + k * of_group((d * xh).abs())
    b = of_group(d * xh).abs()
    dx_tol = 1.2 * (r * (d_tol + a_tol + xh.abs() * b_tol + xh_tol * b) + 4 * k * r * (d.abs() + of_group(d).abs() + xh.abs() * b))
    norm_near(dx[..., :c], want[0], dx_tol, "dx", dtype)
    assert bool((dx[..., c:] == 3.0).all())
    kk = (n * p / 64 + 16) * STEP
    dz_tol = d_tol / gamma.double().abs()
    norm_near(dgamma, want[1], 1.2 * (dz_tol * xh.abs() + dz.abs() * xh_tol + kk * (dz * xh).abs()).sum((0, 1)), "dgamma", F32)
    norm_near(dbeta, want[2], 1.2 * (dz_tol + kk * dz.abs()).sum((0, 1)), "dbeta", F32)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 300001, 8, 2), (2, 70001, 24, 3), (3, 9000, 65, 5)], ids=["300001", "70001", "9000"])
def test_group_norm_of_samples_of_many_chunks(shape, dtype):
    test_group_norm_and_its_gradient(shape, "silu", dtype)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("shape", [(3, 1, 64, 4), (3, 20, 64, 4), (3, 5000, 64, 4), (2, 1, 4099, 1)], ids=["rows", "tiles", "chunks", "wide"])
def test_group_norm_keeps_nan_to_its_group(shape, act):
    n, p, c, groups = shape
    x = torch.randn(n, p, c, generator=torch.Generator().manual_seed(1))
    x[1, p // 2, 0] = float("nan")
    y, w = torch.empty(n, p, c, device="cuda"), torch.ones(c, device="cuda")
    g.group_norm(x.cuda(), w, 0 * w, groups, y, act=act)
    torch.cuda.synchronize()
    want = torch.zeros(n, p, c, dtype=torch.bool)
    want[1, :, :c // groups] = True
    assert torch.equal(torch.isnan(y).cpu(), want)


def test_group_norm_of_no_samples_and_of_a_constant():
    z = torch.empty(0, 5, 32, device="cuda")
    w, b = torch.ones(32, device="cuda"), torch.zeros(32, device="cuda")
    g.group_norm(z, w, b, 4, torch.empty_like(z))
    dg, db = torch.full((32,), 9.0, device="cuda"), torch.full((32,), 9.0, device="cuda")
    g.group_norm_grad(z, z, w, b, torch.empty(0, 4, 2, device="cuda"), 4, torch.empty_like(z), dg, db)
    x = torch.full((2, 6, 32), 5.0, device="cuda")
    y, st = torch.empty_like(x), torch.empty(2, 4, 2, device="cuda")
    g.group_norm(x, w, b + 0.5, 4, y, stats=st, eps=1e-5)
    torch.cuda.synchronize()
    assert bool((dg == 0).all()) and bool((db == 0).all())
    assert bool((y == 0.5).all()) and bool((st[..., 0] == 5).all()) and torch.allclose(st[..., 1], torch.full_like(st[..., 1], 1e-5 ** -0.5))


def test_another_offset_does_not_cost_the_variance():
    # numbers far from zero: the squares are taken around the mean
    gen = torch.Generator().manual_seed(2)
    for shape, groups in (((6, 1, 128), 4), ((2, 2000, 16), 4)):
        x = (3000 + torch.randn(*shape, generator=gen))
        st = torch.empty(shape[0], groups, 2, device="cuda")
        w = torch.ones(shape[2], device="cuda")
        y = torch.empty(shape, device="cuda")
        g.group_norm(x.cuda(), w, 0 * w, groups, y, stats=st)
        torch.cuda.synchronize()
        mean, rstd, _ = ref.norm_parts(x.double(), groups, 1e-5)
        # the mean is off by a few roundings of 3000 (2^-12 each); a variance around it by the square of that
        assert float((st[..., 0].double().cpu() - mean).abs().max()) <= 16 * 2.0 ** -13
        assert float((st[..., 1].double().cpu() / rstd - 1).abs().max()) <= 1e-4


# ----------------------------------------------------------- streams, graphs, together --

def test_another_stream_and_a_captured_chain():
    """Attention, norm, and both gradients as one chain: on a stream of its own, and replayed from a graph."""
    lens, h, dk, dv, decay = [5, 3, 0, 5, 200], 4, 16, 32, [0.75, 0.9, 0.97, 0.99]
    s = make(lens, h, dk, dv, F32, True, 0.1, True)
    n, c = sum(lens), h * dv
    gen = torch.Generator().manual_seed(4)
    gamma, beta, dy = torch.randn(c, generator=gen).cuda(), torch.randn(c, generator=gen).cuda(), torch.randn(n, c, generator=gen).cuda()

    def buffers():
        e = lambda *shape: torch.full(shape, float("nan"), device="cuda")  # noqa: E731
        return {"o": e(n, h, dv), "state": e(len(lens), h, dv, dk), "y": e(n, c), "stats": e(n, h, 2), "do": e(n, h, dv), "dgamma": e(c),
                "dbeta": e(c), "dq": e(n, h, dk), "dk": e(n, h, dk), "dv": e(n, h, dv), "dstate": e(len(lens), h, dv, dk)}

    def chain(b, stream=None):
        seg = dict(seg_start=s["seg_start"], starts=s["starts"], state_in=s["state_in"], scale=0.25, stream=stream)
        g.decay_attention(s["q"], s["k"], s["v"], decay, b["o"], state_out=b["state"], **seg)
        g.group_norm(b["o"].flatten(1), gamma, beta, h, b["y"], stats=b["stats"], act="silu", stream=stream)
        g.group_norm_grad(b["o"].flatten(1), dy, gamma, beta, b["stats"], h, b["do"].flatten(1), b["dgamma"], b["dbeta"], act="silu", stream=stream)
        g.decay_attention_grad(s["q"], s["k"], s["v"], decay, b["do"], b["dq"], b["dk"], b["dv"], dstate_in=b["dstate"], **seg)

    want = buffers()
    chain(want)
    torch.cuda.synchronize()
    # the chain as one function of its inputs
    w = {k: wide(v) for k, v in s.items()}
    leaves = [x.clone().requires_grad_() for x in (w["q"], w["k"], w["v"], w["state_in"], wide(gamma), wide(beta))]
    o, st = ref.attention(*leaves[:3], decay, lens, w["starts"], leaves[3], 0.25)
    y = ref.group_norm(o.view(n, 1, c), leaves[4], leaves[5], h, "silu", 1e-5).view(n, c)
    grads = torch.autograd.grad((y * wide(dy)).sum(), leaves)
    for name, a in [("y", y), ("state", st)] + list(zip(("dq", "dk", "dv", "dstate", "dgamma", "dbeta"), grads)):
        a = a.detach()
        # a group whose spread is small divides the roundings of attention by it
        assert float((wide(want[name]) - a).norm() / a.norm()) <= 2e-5, name
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = buffers()
    torch.cuda.synchronize()
    chain(got, side)
    side.synchronize()
    for k in want:
        assert torch.equal(got[k], want[k]), k
    graphs, outs = [], []
    for _ in range(2):                  # two graphs of the same calls, replayed in turn
        b = buffers()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            chain(b)
        graphs.append(graph)
        outs.append(b)
    for replay in range(3):
        for b in outs:
            for t in b.values():
                t.fill_(float("nan"))
        chain(got)                      # the program's own work between the replays
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for b in outs + [got]:
            for k in want:
                assert torch.equal(b[k], want[k]), (replay, k)
