"""Plain 64-bit forms of the memory operators, for the tests: straight from the definitions, token by token."""
import torch


def segments(lens):
    at, out = 0, []
    for n in lens:
        out.append((at, at + n))
        at += n
    return out


def attention(q, k, v, decay, lens, starts=None, state_in=None, scale=1.0):
    """out [tokens, heads, value_dim] and the states behind the segments [segments, heads, value_dim, key_dim]."""
    h, dk, dv = q.shape[1], q.shape[2], v.shape[2]
    d = torch.as_tensor(decay, dtype=torch.float32).double()[:, None, None]
    out, states = [], []
    for i, (a, b) in enumerate(segments(lens)):
        s = state_in[i] if state_in is not None else torch.zeros(h, dv, dk, dtype=torch.float64)
        for t in range(a, b):
            if starts is not None and starts[t]:
                s = torch.zeros_like(s)
            s = d * s + v[t][:, :, None] * k[t][:, None, :]
            out.append(scale * (s * q[t][:, None, :]).sum(-1))
        states.append(s)
    empty = torch.zeros(0, h, dv, dtype=torch.float64)
    return torch.stack(out) if out else empty, torch.stack(states)


def attention_grad(q, k, v, decay, lens, dout, starts=None, state_in=None, dstate_out=None, scale=1.0):
    """dq, dk, dv, dstate_in, by automatic differentiation of the above."""
    h, dk, dv = q.shape[1], q.shape[2], v.shape[2]
    if state_in is None:
        state_in = torch.zeros(len(lens), h, dv, dk, dtype=torch.float64)
    args = [x.clone().requires_grad_() for x in (q, k, v, state_in)]
    out, states = attention(args[0], args[1], args[2], decay, lens, starts, args[3], scale)
    total = (out * dout).sum()
    if dstate_out is not None:
        total = total + (states * dstate_out).sum()
    got = torch.autograd.grad(total, args, allow_unused=True)
    return [torch.zeros_like(x) if g is None else g for x, g in zip(args, got)]


def activation(z, act):
    return {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, torch.zeros_like(z)), "silu": lambda: z / (1 + torch.exp(-z))}[act]()


def norm_parts(x, groups, eps):
    """Mean and 1 / standard deviation [samples, groups] and the normalised x, of x [samples, positions, channels]."""
    n, p, c = x.shape
    y = x.view(n, p, groups, c // groups)
    mean = y.mean((1, 3))
    rstd = 1 / torch.sqrt(((y - mean[:, None, :, None]) ** 2).mean((1, 3)) + eps)
    return mean, rstd, ((y - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(n, p, c)


def group_norm(x, gamma, beta, groups, act, eps):
    return activation(norm_parts(x, groups, eps)[2] * gamma + beta, act)
