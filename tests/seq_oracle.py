"""Definitions of the sequence operators in 64 bits on the CPU, step by step; gradients by reverse-mode
differentiation of those definitions.  Used by the tests alone; shares nothing with the kernels."""
import torch


def conv(x, weight, bias=None, init=None, lengths=None, silu=True):
    """-> y [T,B,D], state [W-1,B,D]."""
    T, B, D = x.shape
    W = weight.shape[1]
    rows = list(init.unbind(0)) if init is not None else [torch.zeros(B, D, dtype=x.dtype) for _ in range(W - 1)]
    rows += list(x.unbind(0))
    n = [T] * B if lengths is None else [min(max(int(v), 0), T) for v in lengths]
    live = torch.tensor(n)
    ys = []
    for t in range(T):
        v = torch.zeros(B, D, dtype=x.dtype) if bias is None else bias.expand(B, D)
        for k in range(W):
            v = v + weight[:, k] * rows[t + k]
        if silu:
            v = v / (1 + torch.exp(-v))
        ys.append(torch.where((t < live)[:, None], v, torch.zeros_like(v)))
    y = torch.stack(ys) if T else torch.zeros_like(x)
    state = [torch.stack([rows[n[b] + j][b] for b in range(B)]) for j in range(W - 1)]
    return y, torch.stack(state) if state else torch.zeros(0, B, D, dtype=x.dtype)


def scan(x, dt, A, Bv, Cv, D=None, z=None, dt_bias=None, softplus=True, init=None, lengths=None):
    """Bv, Cv [T,B,G,N] -> y [T,B,D], state [B,D,N]."""
    T, nb, nd = x.shape
    N, G = A.shape[1], Bv.shape[2]
    group = torch.arange(nd) // (nd // G)
    live = torch.tensor([T] * nb if lengths is None else [min(max(int(v), 0), T) for v in lengths])
    h = init if init is not None else torch.zeros(nb, nd, N, dtype=x.dtype)
    ys = []
    for t in range(T):
        on = (t < live)[:, None]
        raw = dt[t] + (dt_bias if dt_bias is not None else 0.0)
        delta = torch.nn.functional.softplus(raw, threshold=1e9) if softplus else raw
        new = torch.exp(delta[..., None] * A) * h + (delta * x[t])[..., None] * Bv[t][:, group]
        h = torch.where(on[..., None], new, h)
        y = (h * Cv[t][:, group]).sum(-1)
        if D is not None:
            y = y + D * x[t]
        if z is not None:
            y = y * z[t] / (1 + torch.exp(-z[t]))
        ys.append(torch.where(on, y, torch.zeros_like(y)))
    return torch.stack(ys) if T else torch.zeros_like(x), h


def gradients(f, inputs, outputs_grads):
    """d sum_i <grad_i, f(inputs)_i> / d inputs, for a dict of tensors (None: absent)."""
    leaves = {k: v.detach().clone().requires_grad_(True) for k, v in inputs.items() if v is not None}
    total = sum((g * o).sum() for o, g in zip(f(**leaves), outputs_grads) if g is not None)
    got = torch.autograd.grad(total, list(leaves.values()), allow_unused=True)
    return {k: (g if g is not None else torch.zeros_like(v)) for (k, v), g in zip(leaves.items(), got)}


E4M3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()   # value of every code


def adamw(p, g, m, v, step, lr, betas, eps, decay):
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    update = (m / (1 - betas[0] ** step)) / ((v / (1 - betas[1] ** step)).sqrt() + eps)
    return p - lr * decay * p - lr * update, m, v
