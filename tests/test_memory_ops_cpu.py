"""The memory operators without a GPU: what they refuse before they touch the device, and the tests' own reference."""
import ctypes as C

import pytest
import torch

import memory_reference as ref
import paper_1611_06256_amd as g
from paper_1611_06256_amd import binding

A = 1 << 20                                    # an address that nobody reads


def desc(heads=2, key=16, value=32, dtype=0, decay=(0.5, 0.9), scale=1.0):
    d = (C.c_float * max(1, len(decay)))(*decay)
    return binding._DecayDesc(heads, key, value, dtype, C.cast(d, C.POINTER(C.c_float)), scale)


def views(n, dims, heads=2, place=A):
    return [binding._Heads(place + (i << 24), heads * d, d) for i, d in enumerate(dims)]


def forward(lib, d, v, n_segments=2, n_tokens=8, table=None, state_in=None, state_out=None, ws=None, nbytes=1 << 30):
    return lib.ga3c_decay_attention(C.byref(d), *[C.byref(x) if x else None for x in v], table, None, n_segments, n_tokens, state_in,
                                    state_out, ws, nbytes, None)


def test_attention_refuses_bad_descriptions():
    lib = g.load_library()
    v = views(8, [16, 16, 32, 32])
    cases = [(dict(heads=0), b"n_heads"), (dict(heads=129, decay=[0.5] * 129), b"n_heads"), (dict(key=0), b"key_dim"),
             (dict(key=129), b"key_dim"), (dict(value=0), b"value_dim"), (dict(value=129), b"value_dim"), (dict(dtype=2), b"dtype"),
             (dict(decay=(0.5, 1.5)), b"decay of head 1"), (dict(decay=(-0.1, 0.5)), b"decay of head 0"),
             (dict(decay=(0.5, float("nan"))), b"decay of head 1"), (dict(scale=float("inf")), b"scale"),
             (dict(scale=float("nan")), b"scale")]
    for kw, text in cases:
        assert forward(lib, desc(**kw), v) == -1 and text in lib.ga3c_last_error(), kw
        step = lib.ga3c_decay_attention_step(C.byref(desc(**kw)), *[C.byref(x) for x in v], None, None, 4, A, 8, None)
        assert step == -1 and text in lib.ga3c_last_error(), kw
        assert lib.ga3c_decay_attention_workspace(C.byref(desc(**kw)), 2, 8, 1) == 0
    assert lib.ga3c_decay_attention(None, *[C.byref(x) for x in v], None, None, 2, 8, None, None, None, 0, None) == -1
    no_decay = binding._DecayDesc(2, 16, 32, 0, None, 1.0)
    assert forward(lib, no_decay, v) == -1 and b"null" in lib.ga3c_last_error()


def test_attention_refuses_bad_tensors():
    lib = g.load_library()
    d, H = desc(), binding._Heads
    good = views(8, [16, 16, 32, 32])
    for i in range(4):
        v = list(good)
        v[i] = None
        assert forward(lib, d, v) == -1 and b"null tensor" in lib.ga3c_last_error()
        v[i] = H(None, 64, 32)
        assert forward(lib, d, v) == -1 and b"null tensor" in lib.ga3c_last_error()
        v[i] = H(A + (i << 24) + 2, 64, 32)
        assert forward(lib, d, v) == -1 and b"aligned" in lib.ga3c_last_error()
    for i in range(3):
        v = list(good)
        v[i] = H(A + (i << 24), -64, 32)
        assert forward(lib, d, v) == -1 and b"negative stride" in lib.ga3c_last_error()
        v = list(good)
        v[3] = H(good[i].data, 64, 32)
        assert forward(lib, d, v) == -1 and b"one of the inputs" in lib.ga3c_last_error()
    for token, head in ((0, 32), (64, 0), (63, 32), (31, 512), (64, 31)):
        v = list(good)
        v[3] = H(A + (3 << 24), token, head)
        assert forward(lib, d, v) == -1 and b"overlap" in lib.ga3c_last_error(), (token, head)
    assert forward(lib, d, good, n_segments=3) == -1 and b"equal segments" in lib.ga3c_last_error()
    assert forward(lib, d, good, n_segments=0) == -1 and b"without a segment" in lib.ga3c_last_error()
    assert forward(lib, d, good, n_segments=-1) == -1 and forward(lib, d, good, n_tokens=-8) == -1
    assert forward(lib, d, good, state_in=A, state_out=A) == -1 and b"state_out" in lib.ga3c_last_error()
    assert forward(lib, d, good, state_in=A, state_out=A + 4096) == -1
    assert forward(lib, d, good, n_segments=0, n_tokens=0) == 0          # nothing to do


def test_attention_grad_and_step_refuse():
    lib = g.load_library()
    d = desc()

    def grad(v, state_in=None, dstate_out=None, dstate_in=None):
        return lib.ga3c_decay_attention_grad(C.byref(d), *[C.byref(x) if x else None for x in v], None, None, 2, 8, state_in,
                                             dstate_out, dstate_in, None, 1 << 30, None)

    good = views(8, [16, 16, 32, 32, 16, 16, 32])
    for i in range(7):
        v = list(good)
        v[i] = None
        assert grad(v) == -1 and b"null tensor" in lib.ga3c_last_error()
    v = list(good)
    v[5] = binding._Heads(good[4].data, 32, 16)
    assert grad(v) == -1 and b"two outputs" in lib.ga3c_last_error()
    v[5] = binding._Heads(good[1].data, 32, 16)
    assert grad(v) == -1 and b"one of the inputs" in lib.ga3c_last_error()
    assert grad(good, state_in=A, dstate_in=A) == -1 and grad(good, dstate_out=A, dstate_in=A) == -1

    def step(n, slots, states, n_slots):
        return lib.ga3c_decay_attention_step(C.byref(d), *[C.byref(x) for x in good[:4]], slots, None, n, states, n_slots, None)

    assert step(-1, None, A, 8) == -1 and step(4, None, A, -1) == -1
    assert step(9, None, A, 8) == -1 and b"9 tokens for 8 states" in lib.ga3c_last_error()
    assert step(4, A, None, 8) == -1 and b"null states" in lib.ga3c_last_error()
    assert step(0, None, None, 0) == 0


def test_group_norm_refuses():
    lib = g.load_library()

    def norm(channels=64, groups=4, dtype=0, act=0, eps=1e-5, x=A, xs=64, gamma=A, beta=A, y=2 * A, ys=64, samples=3, positions=2):
        d = binding._NormDesc(channels, groups, dtype, act, eps)
        return lib.ga3c_group_norm(C.byref(d), x, xs, gamma, beta, y, ys, None, samples, positions, None, 1 << 30, None)

    for kw, text in [(dict(channels=0), b"equal groups"), (dict(groups=0), b"equal groups"), (dict(groups=5), b"equal groups"),
                     (dict(dtype=7), b"dtype"), (dict(act=3), b"activation"), (dict(eps=-1.0), b"eps"), (dict(eps=float("nan")), b"eps"),
                     (dict(x=None), b"null"), (dict(y=None), b"null"), (dict(gamma=None), b"null"), (dict(beta=None), b"null"),
                     (dict(xs=63), b"closer"), (dict(ys=0), b"closer"), (dict(y=A), b"is the input"), (dict(x=A + 2), b"aligned"),
                     (dict(samples=-1), b"negative"), (dict(positions=-1), b"negative"), (dict(positions=0), b"without a position")]:
        assert norm(**kw) == -1 and text in lib.ga3c_last_error(), kw
    assert norm(samples=0) == 0

    d = binding._NormDesc(64, 4, 0, 2, 0.0)

    def grad(x=A, dy=2 * A, stats=A, dx=3 * A, dgamma=A, dbeta=A, xs=64):
        return lib.ga3c_group_norm_grad(C.byref(d), x, xs, dy, 64, A, A, stats, dx, 64, dgamma, dbeta, 3, 2, None, 1 << 30, None)

    for kw in (dict(x=None), dict(dy=None), dict(stats=None), dict(dx=None), dict(dgamma=None), dict(dbeta=None), dict(xs=10),
               dict(dx=A), dict(dx=2 * A)):
        assert grad(**kw) == -1, kw


def test_calls_that_are_too_large_are_refused():
    lib = g.load_library()
    d, v = desc(), views(8, [16, 16, 32, 32])
    assert forward(lib, d, v, n_segments=(1 << 22) + 1, n_tokens=1 << 24, table=A) == -1 and b"2^22 segments" in lib.ga3c_last_error()
    assert forward(lib, d, v, n_segments=1, n_tokens=(1 << 28) + 1) == -1 and b"2^28 tokens" in lib.ga3c_last_error()
    n = (1 << 22) + 1
    assert lib.ga3c_decay_attention_step(C.byref(d), *[C.byref(x) for x in v], None, None, n, A, n, None) == -1
    assert b"2^22 tokens" in lib.ga3c_last_error()
    # one position (rows), a few, and groups wider than a block
    for channels, groups, samples, positions in ((1024, 256, 1 << 24, 1), (64, 4, 1 << 24, 4), (1 << 20, 128, 1 << 24, 1)):
        nd = binding._NormDesc(channels, groups, 1, 0, 1e-5)
        rc = lib.ga3c_group_norm(C.byref(nd), A, channels, A, A, A + (1 << 30), channels, None, samples, positions, A, 1 << 60, None)
        assert rc == -1 and b"too many samples" in lib.ga3c_last_error(), channels


def test_scratch_is_a_state_per_span_whatever_the_segments():
    lib = g.load_library()
    d = desc(heads=2, key=64, value=128)
    for tokens in (1, 127, 128, 5000, 1 << 20):
        for segments in (1, 3, 700, 60000, 300000):
            for grad in (0, 1):
                most = (1 + grad) * (tokens // 128) * 2 * (64 * 128 + 1) * 4
                assert lib.ga3c_decay_attention_workspace(C.byref(d), segments, tokens, grad) <= most, (tokens, segments)


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(4, 2, 16)
    with pytest.raises(g.Ga3cError, match="GPU tensor"):
        g.decay_attention(x, x, x, [0.5, 0.5], torch.empty_like(x))
    with pytest.raises(g.Ga3cError, match="GPU tensor"):
        g.decay_attention_step(x, x, x, [0.5, 0.5], torch.zeros(4, 2, 16, 16), torch.empty_like(x))
    with pytest.raises(g.Ga3cError, match="GPU tensor"):
        g.group_norm(x, torch.ones(16), torch.zeros(16), 4, torch.empty_like(x))


def test_reference_against_the_sum_over_tokens_and_differences():
    # the recurrence is the sum over earlier tokens of the same episode, and its gradient that of differences
    gen = torch.Generator().manual_seed(1)
    lens, h, dk, dv, decay, scale = [4, 0, 7], 2, 3, 5, [0.7, 1.0], 0.4
    n = sum(lens)
    q, k, v = (torch.randn(n, h, d, generator=gen, dtype=torch.float64) for d in (dk, dk, dv))
    s0 = torch.randn(3, h, dv, dk, generator=gen, dtype=torch.float64)
    starts = torch.zeros(n, dtype=torch.uint8)
    starts[[2, 8]] = 1
    out, states = ref.attention(q, k, v, decay, lens, starts, s0, scale)
    d32 = torch.tensor(decay).double()
    for i, (a, b) in enumerate(ref.segments(lens)):
        for t in range(a, b):
            first = max([j for j in range(a, t + 1) if starts[j]], default=None)
            want = sum(d32[:, None] ** (t - j) * (q[t] * k[j]).sum(-1, keepdim=True) * v[j] for j in range(first if first is not None else a, t + 1))
            if first is None:
                want = want + d32[:, None] ** (t - a + 1) * (s0[i] * q[t][:, None, :]).sum(-1)
            assert torch.allclose(out[t], scale * want, atol=1e-12)
    assert torch.equal(states[1], s0[1])
    dout, ds = torch.randn_like(out), torch.randn_like(states)
    grads = ref.attention_grad(q, k, v, decay, lens, dout, starts, s0, ds, scale)

    def loss(*x):
        o, s = ref.attention(x[0], x[1], x[2], decay, lens, starts, x[3], scale)
        return float((o * dout).sum() + (s * ds).sum())

    for i, gr in enumerate(grads):
        x = [q, k, v, s0]
        way = torch.randn_like(x[i])
        ends = [loss(*[y + e * way if j == i else y for j, y in enumerate(x)]) for e in (1e-5, -1e-5)]
        assert abs((ends[0] - ends[1]) / 2e-5 - float((gr * way).sum())) < 1e-6


def test_networks_with_a_memory_are_checked():
    lib = g.load_library()
    ctx = C.c_void_p()
    net = g.SMALL_NET(6).c()

    def create(n=net, **kw):
        m = binding._MemoryDesc(4, 16, 32, (C.c_float * 16)(0.5, 0.6, 0.7, 1.0))
        for k, v in kw.items():
            setattr(m, k, v)
        return lib.ga3c_create_memory(C.byref(n) if n else None, C.byref(m), 1, 1, C.byref(ctx))

    for kw, text in [(dict(heads=0), b"heads"), (dict(heads=17), b"heads"), (dict(key_dim=0), b"key_dim"), (dict(value_dim=129), b"key_dim"),
                     (dict(heads=3), b"fc_units = 256"), (dict(decay=(C.c_float * 16)(0.5, 0.5, 2.0, 0.5)), b"decay of head 2"),
                     (dict(decay=(C.c_float * 16)(float("nan"))), b"decay of head 0"), (dict(n=None), b"null")]:
        assert create(**kw) == -1 and text in lib.ga3c_last_error() and not ctx.value, kw
    net.math = 1
    assert create() == -1 and b"math" in lib.ga3c_last_error()
    assert lib.ga3c_predict_memory(None, A, 1, None, None, A, 1, None, None, None, None, None, None) == -1
    assert lib.ga3c_predict_memory(None, A, 1, None, None, None, 1, None, None, None, None, None, None) == -1
    assert lib.ga3c_predict_memory(None, A, 2, None, None, A, 1, None, None, None, None, None, None) == -1
    hp = g.HParams().c()
    assert lib.ga3c_train_step_memory(None, A, A, A, A, None, None, None, 1, 5, C.byref(hp), None, None) == -1
    with pytest.raises(g.Ga3cError, match="decay"):
        g.MemoryDesc(heads=3).c()
    assert C.sizeof(binding._MemoryDesc) == 76 and C.sizeof(binding._DecayDesc) == 32 and C.sizeof(binding._NormDesc) == 20
