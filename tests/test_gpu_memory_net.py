"""A network with a memory between the fc layer and the heads, on the GPU, against the same network in 64 bits: predictions step by
step, updates on segments, and the two together.

Bounds are those of the network without a memory: 1e-4 of the largest on outputs, 1e-3 of each parameter tensor's largest on its
gradient (sums of fp32 products through the same layers; the memory's own are within 1e-5)."""
import dataclasses

import numpy as np
import pytest
import torch

import ga3c_synth as synth
import memory_reference as ref
import paper_1611_06256_amd as g

pytestmark = pytest.mark.gpu

SMALL = (dataclasses.replace(g.SMALL_NET(6)), g.MemoryDesc())
# 51 units: nothing is a multiple of four
ODD = (g.NetDesc(in_c=2, in_h=20, in_w=24, conv=((8, 4, 2),), fc_units=51, n_actions=3), g.MemoryDesc(heads=3, key_dim=5, value_dim=7, decay=(0.5, 0.9, 1.0)))
LARGE = (dataclasses.replace(g.LARGE_NET(5)), g.MemoryDesc(heads=4, key_dim=32, value_dim=64))


def net_of(desc, memory, pred, train, seed=5):
    net = g.Ga3c(desc, pred, train, memory)
    theta = synth.perturbed_theta(seed, net.offsets(), net.n_params)
    off = net.offsets()
    rng = np.random.default_rng(seed)
    for name, mean in (("memory.gamma", 1.0), ("memory.beta", 0.1)):
        at, shape = off[name]
        theta[at:at + shape[0]] = (mean + 0.2 * rng.standard_normal(shape[0])).astype(np.float32)
    net.params_set(torch.from_numpy(theta).cuda())
    return net, theta


def reference(net, theta, frames, lens, starts, states):
    """logits, values and the states behind the segments, of frames [n, C, H, W] in 64 bits; theta: a tensor."""
    d, m = net.desc, net.memory
    p = {k: theta[at:at + int(np.prod(shape))].view(shape) for k, (at, shape) in net.offsets().items()}
    x = frames.double() / 255
    for i, (_, _, stride) in enumerate(d.conv):
        x = torch.relu(torch.nn.functional.conv2d(x, p[f"conv{i + 1}.W"], p[f"conv{i + 1}.b"], stride=stride))
    x = torch.relu(x.flatten(1) @ p["fc.W"].T + p["fc.b"])
    n, hk = x.shape[0], m.heads * m.key_dim
    q, k, v = x[:, :hk].view(n, m.heads, -1), x[:, hk:2 * hk].view(n, m.heads, -1), x[:, 2 * hk:].view(n, m.heads, -1)
    o, behind = ref.attention(q, k, v, m.decay, lens, starts, states, m.key_dim ** -0.5)
    out = ref.group_norm(o.reshape(n, 1, -1), p["memory.gamma"], p["memory.beta"], m.heads, "relu", 1e-5).view(n, -1)
    y = torch.cat([x[:, :2 * hk], x[:, 2 * hk:] + out], 1)
    return y @ p["policy.W"].T + p["policy.b"], (y @ p["value.W"].T + p["value.b"])[:, 0], behind


def rel(got, want):
    want = want.detach().double()
    return float((got.detach().double().cpu() - want).abs().max() / want.abs().max().clamp(min=1e-12))


def random_frames(seed, n, desc):
    return torch.from_numpy(np.random.default_rng(seed).integers(0, 256, (n, desc.in_c, desc.in_h, desc.in_w), dtype=np.uint8))


@pytest.mark.parametrize("generic", [False, True], ids=["own", "generic"])
@pytest.mark.parametrize("which", [SMALL, ODD, LARGE], ids=["small", "odd", "large"])
def test_predictions_carry_the_memory_on(which, generic):
    desc, memory = which
    agents = 9
    net, theta = net_of(desc, memory, 64, 0)
    net.use_generic_kernels(generic)
    th = torch.from_numpy(theta).double()
    gen = torch.Generator().manual_seed(3)
    states = 0.1 * torch.rand(agents, memory.heads, memory.value_dim, memory.key_dim, generator=gen)
    kept, dev = states.double(), states.cuda()
    for step, (B, named) in enumerate([(9, False), (4, True), (9, True), (1, True), (7, True)]):
        print(f"memory predict {desc.fc_units} generic={generic} step {step}", flush=True)
        frames = random_frames(10 + step, B, desc)
        who = torch.randperm(agents, generator=gen)[:B].to(torch.int32) if named else torch.arange(B, dtype=torch.int32)
        starts = (torch.rand(B, generator=gen) < 0.3).to(torch.uint8) if step else None
        out = {"logits": torch.full((B, desc.n_actions), float("nan"), device="cuda"), "values": torch.full((B,), float("nan"), device="cuda"),
               "probs": torch.full((B, desc.n_actions), float("nan"), device="cuda"), "actions": torch.full((B,), -1, dtype=torch.int32, device="cuda")}
        u = torch.rand(B, generator=gen)
        net.predict_memory(frames.cuda(), dev, agents=who.cuda() if named else None, starts=None if starts is None else starts.cuda(), uniforms=u.cuda(), **out)
        torch.cuda.synchronize()
        logits, values, behind = reference(net, th, frames, [1] * B, starts, kept[who.long()])
        kept[who.long()] = behind
        assert rel(out["logits"], logits) <= 1e-4 and rel(out["values"], values) <= 1e-4
        assert rel(out["probs"], torch.softmax(logits, 1)) <= 1e-4 and rel(dev, kept) <= 1e-4
        cdf = out["probs"].cpu().cumsum(1)
        drawn = [next((j for j in range(desc.n_actions) if cdf[i, j] > u[i]), desc.n_actions - 1) for i in range(B)]
        near_edge = [(cdf[i] - u[i]).abs().min() < 1e-5 for i in range(B)]
        assert all(a == b or e for a, b, e in zip(out["actions"].tolist(), drawn, near_edge))
    net.close()


HP = g.HParams(beta=0.01, clip_norm=0.0)


def loss(logits, values, actions, returns, hp):
    p = torch.softmax(logits, 1)
    adv = returns - values
    policy = -(torch.log(p.gather(1, actions.long()[:, None])[:, 0]) * adv.detach()).sum()
    entropy = -(p * torch.log(p)).sum()
    return policy - hp.beta * entropy + hp.value_coef * (adv ** 2).sum()


def returns_of(rewards, dones, bootstrap, lens, gamma):
    out = torch.zeros_like(rewards, dtype=torch.float64)
    for i, (a, b) in enumerate(ref.segments(lens)):
        r = float(bootstrap[i])
        for t in range(b - 1, a - 1, -1):
            r = float(rewards[t]) + float(np.float32(gamma)) * (0.0 if dones[t] else r)
            out[t] = r
    return out


@pytest.mark.parametrize("generic", [False, True], ids=["own", "generic"])
@pytest.mark.parametrize("which,lens", [(SMALL, [5] * 8), (SMALL, [5, 2, 0, 5, 1, 4, 60]), (ODD, [3, 1, 6]), (LARGE, [5, 5, 3, 5])],
                         ids=["small8x5", "small_ragged", "odd", "large"])
def test_updates_against_automatic_differentiation(which, lens, generic):
    desc, memory = which
    n, N = sum(lens), len(lens)
    print(f"memory update {desc.fc_units} {lens} generic={generic}", flush=True)
    net, theta = net_of(desc, memory, 1, n + 7)
    net.use_generic_kernels(generic)
    gen = torch.Generator().manual_seed(n)
    frames = random_frames(20, n, desc)
    actions = torch.randint(0, desc.n_actions, (n,), generator=gen, dtype=torch.int32)
    rewards, bootstrap = torch.randn(n, generator=gen), torch.randn(N, generator=gen)
    dones = (torch.rand(n, generator=gen) < 0.2).to(torch.uint8)
    states = 0.3 * torch.rand(N, memory.heads, memory.value_dim, memory.key_dim, generator=gen)
    equal = len(set(lens)) == 1
    lead = (N, lens[0]) if equal else (n,)
    table = None if equal else torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()
    stats = torch.zeros(8, device="cuda")
    given = states.cuda()
    net.train_step_memory(frames.view(*lead, *frames.shape[1:]).cuda(), actions.view(lead).cuda(), rewards.view(lead).cuda(), dones.view(lead).cuda(),
                          bootstrap.cuda(), HP, seg_start=table, states=given, stats=stats)
    torch.cuda.synchronize()
    starts = torch.zeros(n, dtype=torch.uint8)
    for a, b in ref.segments(lens):
        starts[a + 1:b] = dones[a:b - 1] if b - a > 1 else starts[a + 1:b]
    th = torch.from_numpy(theta).double().requires_grad_()
    logits, values, _ = reference(net, th, frames, lens, starts, states.double())
    total = loss(logits, values, actions, returns_of(rewards, dones, bootstrap, lens, HP.gamma), HP)
    (want,) = torch.autograd.grad(total, th)
    got_logits = net.train_debug_get(1, torch.empty(n, desc.n_actions, device="cuda"))
    got_values = net.train_debug_get(2, torch.empty(n, device="cuda"))
    grad, theta2 = net.params_get(2), net.params_get(0)
    torch.cuda.synchronize()
    assert rel(got_logits, logits) <= 1e-4 and rel(got_values, values) <= 1e-4
    for name, (at, shape) in net.offsets().items():
        part = slice(at, at + int(np.prod(shape)))
        assert rel(grad[part], want[part]) <= 1e-3, name
    assert abs(float(stats[3]) / float(want.norm()) - 1) <= 1e-3
    # Eq. 3 from zero: g = (1 - decay) d^2
    gsq = (1 - HP.rms_decay) * want ** 2
    step = -HP.lr * want / torch.sqrt(gsq + HP.rms_eps)
    assert rel(theta2.cpu().double() - torch.from_numpy(theta).double(), step) <= 2e-3
    assert torch.equal(given.cpu(), states)
    net.close()


def test_agents_play_and_learn():
    # predictions of several steps, then the update on what they saw: the update's own forward pass tells what the agents were told
    desc, memory = SMALL
    N, T = 12, 5
    net, theta = net_of(desc, memory, N, N * T)
    states, gen = net.memory_states(N), torch.Generator().manual_seed(8)
    frames = random_frames(30, N * T, desc).view(N, T, desc.in_c, desc.in_h, desc.in_w).cuda()
    dones = (torch.rand(N, T, generator=gen) < 0.15).to(torch.uint8)
    dones[:, -1] = 0
    fresh = torch.ones(N, dtype=torch.uint8, device="cuda")            # every episode begins
    states.fill_(float("nan"))                                         # what was there before does not count
    before, told, actions = torch.zeros_like(states), [], torch.zeros(N, T, dtype=torch.int32, device="cuda")
    for t in range(T):
        values, drawn = torch.empty(N, device="cuda"), torch.empty(N, dtype=torch.int32, device="cuda")
        net.predict_memory(frames[:, t].contiguous(), states, starts=fresh, uniforms=torch.rand(N, generator=gen).cuda(), values=values, actions=drawn)
        told.append(values)
        actions[:, t] = drawn
        fresh = dones[:, t].contiguous().cuda()
    rewards = torch.randn(N, T, generator=gen).cuda()
    net.train_step_memory(frames, actions, rewards, dones.cuda(), told[-1], HP, states=before)
    seen = net.train_debug_get(2, torch.empty(N * T, device="cuda"))
    torch.cuda.synchronize()
    assert rel(seen.view(N, T), torch.stack(told, 1).cpu()) <= 2e-4
    moved = net.params_get(0).cpu() - torch.from_numpy(theta)
    for name in ("memory.gamma", "memory.beta", "fc.W", "conv1.W"):
        at, shape = net.offsets()[name]
        assert float(moved[at:at + int(np.prod(shape))].abs().max()) > 0, name
    prof = None
    net.profile_enable(True)
    net.train_step_memory(frames, actions, rewards, dones.cuda(), told[-1], HP, states=before)
    prof = net.profile_read()
    assert {"memory_features", "memory_fwd", "memory_norm", "memory_bwd"} <= set(prof)
    net.close()


def test_a_network_with_a_memory_refuses_the_calls_without_one_and_the_other_way_round():
    desc, memory = SMALL
    net = g.Ga3c(desc, 8, 40, memory)
    plain = g.Ga3c(desc, 8, 40)
    net.params_init(3)
    at, shape = net.offsets()["memory.gamma"]
    got = net.params_get(0)
    torch.cuda.synchronize()
    assert bool((got[at:at + 128] == 1).all()) and bool((got[at + 128:at + 256] == 0).all()) and shape == (128,)
    assert net.n_params == plain.n_params + 256
    f8 = torch.zeros(8, 4, 84, 84, dtype=torch.uint8, device="cuda")
    seg = (f8.view(4, 2, 4, 84, 84), torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda"),
           torch.zeros(4, 2, dtype=torch.uint8, device="cuda"))
    flat = [x.flatten(0, 1) for x in seg]
    table = torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    with pytest.raises(g.Ga3cError, match="has a memory"):
        net.predict(f8)
    with pytest.raises(g.Ga3cError, match="has a memory"):
        net.train_step(*seg, None, HP)
    with pytest.raises(g.Ga3cError, match="has a memory"):
        net.train_step_ragged(*flat, table, None, HP)
    with pytest.raises(g.Ga3cError, match="memory"):
        g.Scheduler(net, HP, predict_cap=8, train_min=5, train_cap=40)
    states = net.memory_states(8)
    with pytest.raises(g.Ga3cError, match="no memory"):
        plain.predict_memory(f8, states)
    with pytest.raises(g.Ga3cError, match="no memory"):
        plain.train_step_memory(*seg, None, HP)
    with pytest.raises(g.Ga3cError, match="expected states"):
        net.predict_memory(f8, torch.zeros(8, 4, 16, 32, device="cuda"))
    with pytest.raises(g.Ga3cError, match="8 frames for 4 states"):
        net.predict_memory(f8, net.memory_states(4))
    with pytest.raises(g.Ga3cError, match="outside"):
        net.predict_memory(torch.zeros(9, 4, 84, 84, dtype=torch.uint8, device="cuda"), net.memory_states(9))
    with pytest.raises(g.Ga3cError, match="above capacity"):
        net.train_step_memory(torch.zeros(41, 1, 4, 84, 84, dtype=torch.uint8, device="cuda"), *[torch.zeros(41, 1, dtype=t, device="cuda") for t in
                              (torch.int32, torch.float32, torch.uint8)], None, HP)
    net.predict_memory(f8[:0], states)                  # nothing to do
    net.train_step_memory(*[x[:0] for x in seg], None, HP)
    torch.cuda.synchronize()
    net.close(), plain.close()
