"""Definitions of the gated block's operators in 64 bits on the CPU, written as they are read; gradients by reverse-mode
differentiation (seq_oracle.gradients).  Used by the tests alone; shares nothing with the kernels."""
import torch


def steps_of(lengths, T, B):
    return [T] * B if lengths is None else [min(max(int(v), 0), T) for v in lengths]


def recurrence(x, i, r, decay, sharpness=8.0, init=None, lengths=None):
    """-> y [T,B,D], state [B,D].  1 - a^2 as (1 - a)(1 + a), with 1 - a = -expm1(l)."""
    T, B, D = x.shape
    n = torch.tensor(steps_of(lengths, T, B))[:, None]
    rate = sharpness * torch.nn.functional.softplus(decay, threshold=1e9)
    h = init if init is not None else torch.zeros(B, D, dtype=x.dtype)
    ys = []
    for t in range(T):
        l = -rate / (1 + torch.exp(-r[t]))
        taken = -torch.expm1(l)
        new = (1 - taken) * h + torch.sqrt(taken * (2 - taken)) * x[t] / (1 + torch.exp(-i[t]))
        h = torch.where(t < n, new, h)
        ys.append(torch.where(t < n, new, torch.zeros_like(new)))
    return torch.stack(ys) if T else torch.zeros_like(x), h


def norm(x, groups, weight=None, bias=None, silu=True, eps=1e-5, per_step=False, lengths=None):
    T, B, D = x.shape
    n, columns = steps_of(lengths, T, B), []
    for b in range(B):
        rows = x[:n[b], b].reshape(n[b], groups, D // groups)
        if n[b]:
            over = (2,) if per_step else (0, 2)
            rows = rows - rows.mean(over, keepdim=True)
            rows = rows / torch.sqrt((rows * rows).mean(over, keepdim=True) + eps)
        v = rows.reshape(n[b], D)
        v = v * weight if weight is not None else v
        v = v + bias if bias is not None else v
        v = v / (1 + torch.exp(-v)) if silu else v
        columns.append(torch.cat((v, torch.zeros_like(x[n[b]:, b]))))
    return (torch.stack(columns, 1),)


def units(x, gate, up, act="silu", lengths=None):
    T, B, D = x.shape
    n, columns = steps_of(lengths, T, B), []
    for b in range(B):
        rows = x[:n[b], b]
        g, u = rows @ gate.t(), rows @ up.t()
        f = g / (1 + torch.exp(-g)) if act == "silu" else 0.5 * g * (1 + torch.erf(g * 0.5 ** 0.5))
        columns.append(torch.cat((f * u, torch.zeros(T - n[b], len(gate), dtype=x.dtype))))
    return (torch.stack(columns, 1),)
