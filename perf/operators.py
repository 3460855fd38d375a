"""Sequence operators and the optimiser step, as cases that can be timed and compared with their plain forms.

Three operators, in the library's layout (time-major [T][B][D], channels fastest):

  conv    short causal convolution along time, one filter of W taps per channel, with SiLU
  scan    selective scan: N leaky states per channel whose decay and input gain follow the data
  adamw   one AdamW step over all tensors of a model, moments in 32 bits or in 8

A case says what is done (`do`), the sizes, the type of the streamed tensors (`type`; parameters, states and
the gradients of parameters are always float32) and which optional parts take part:

  conv        a prompt: outputs and the last W - 1 inputs, which a streaming user keeps
  conv_train  the same, and the gradients of everything it read
  conv_step   one token of every sequence, the kept inputs moved on in place
  scan        a prompt: outputs and the last state
  scan_train  the same, and the gradients of everything it read
  scan_step   one token of every sequence, the state moved on in place
  adamw       one optimiser step

`ragged` draws a length for every sequence, from 0 to T; `init` starts from given states; `groups` is the number
of channel groups that have input and output vectors (B and C) of their own.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}
BLOCK = 128                    # elements of an 8-bit state that share a scale
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
MOST = 1 << 28                 # states over time (T * B * D * N) of the largest listed case


def _conv(name, do, T, B, D, W=4, type="bf16", ragged=False, init=False):
    case = dict(do=do, T=T, B=B, D=D, W=W, type=type, ragged=ragged, init=init)
    return dict(name=name, **case) if name else case


def _scan(name, do, T, B, D, N=16, groups=1, type="bf16", gate=True, ragged=False, init=False):
    case = dict(do=do, T=T, B=B, D=D, N=N, groups=groups, type=type, gate=gate, ragged=ragged, init=init)
    return dict(name=name, **case) if name else case


def _adamw(name, sizes, repeat, bits, type="fp32"):
    case = dict(do="adamw", sizes=sizes, repeat=repeat, bits=bits, type=type)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # a batch of prompts before decoding starts
        _conv("conv_prompt", "conv", 1024, 8, 2048),
        # training at the shape of the benchmark's wide layers, with sequences of different lengths
        _conv("conv_train", "conv_train", 256, 128, 1024, ragged=True),
        # one token of 64 streams: latency
        _conv("conv_step", "conv_step", 1, 64, 2048),
        # the same batch of prompts as above
        _scan("scan_prompt", "scan", 1024, 8, 2048),
        # a single long prompt: few channels in flight, many steps
        _scan("scan_long", "scan", 8192, 1, 1024),
        # a training step at the same size: the largest case
        _scan("scan_train", "scan_train", 1024, 8, 2048),
        # sizes that are multiples of nothing, fp32, no gate, two groups, starting from given states
        _scan("scan_ragged", "scan_train", 101, 51, 130, N=11, groups=2, type="fp32", gate=False, ragged=True, init=True),
        # one token of 64 streams: the state passes through once
        _scan("scan_step", "scan_step", 1, 64, 2048),
        # one token of one stream on a narrow layer: pure latency
        _scan("scan_token", "scan_step", 1, 1, 128, type="fp32"),
        # the headline network's six tensors: latency
        _adamw("adamw_small", "700-128-128-20", 1, 32),
        # many middling tensors, bfloat16 gradients, moments in 8 bits
        _adamw("adamw8_many", "700-512-512-20", 12, 8, type="bf16"),
        # the deepest benchmark network eight times over
        _adamw("adamw_deep", "700-2048-2048-2048-20", 8, 32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, unit):
    """A size: as often a round one as any other."""
    n = _log(rng, lo, hi)
    return max(unit, n // unit * unit) if rng.random() < 0.5 else n


def draw(rng):
    do = rng.choices(("conv", "conv_train", "conv_step", "scan", "scan_train", "scan_step", "adamw"), (2, 2, 1, 3, 4, 2, 3))[0]
    type = rng.choices(("bf16", "fp32"), (2, 1))[0]
    if do == "adamw":
        sizes = [rng.choice((700, 64, _log(rng, 40, 1000)))] + [_size(rng, 16, 2048, 64) for _ in range(rng.randrange(1, 4))] + [rng.randrange(2, 40)]
        each = sum(a * b + b for a, b in zip(sizes, sizes[1:]))
        return _adamw(None, "-".join(map(str, sizes)), _log(rng, 1, max(1, min(24, 70_000_000 // each))), rng.choice((8, 32)), type=type)
    one = do.endswith("step")
    T, B, D = 1 if one else _size(rng, 4, 8192, 16), _log(rng, 1, 256 if one else 128), _size(rng, 16, 4096, 64)
    N = rng.choice((16, 16, 16, 8, 32, 64, rng.randrange(1, 33))) if do.startswith("scan") else 16
    while T * B * D * N > MOST:
        if B > 1:
            B //= 2
        else:
            T //= 2
    ragged, init = not one and rng.random() < 0.3, not one and rng.random() < 0.3
    if do.startswith("conv"):
        return _conv(None, do, T, B, D, W=rng.choice((4, 4, 3, 2)), type=type, ragged=ragged, init=init)
    groups = rng.choice([1, 1] + [g for g in (2, 4) if D % g == 0])
    return _scan(None, do, T, B, D, N=N, groups=groups, type=type, gate=rng.random() < 0.7, ragged=ragged, init=init)


# ---------------------------------------------------------------------------------------------------- inputs

def _shapes(case):
    sizes = [int(n) for n in case["sizes"].split("-")]
    return [s for a, b in zip(sizes, sizes[1:]) for s in ((a, b), (b,))] * case["repeat"]


def _offsets(shapes):
    """Where each tensor starts in the flat buffers: at a multiple of BLOCK."""
    at = [0]
    for s in shapes:
        at.append(at[-1] + -(-math.prod(s) // BLOCK) * BLOCK)
    return at


def _prepare_adamw(case, rand):
    shapes = _shapes(case)
    at = _offsets(shapes)
    s = {"shapes": shapes, "at": at, "bits": case["bits"], "step": 10, "seed": 1234}
    # values that a model has some steps into its training: weights and gradients of each tensor on a scale of its own
    weights, grads = rand(at[-1]), rand(at[-1]) * torch.exp(rand(at[-1]))
    s["flat"], s["grad"] = torch.zeros_like(weights), torch.zeros_like(weights, dtype=TYPES[case["type"]])
    s["params"] = [s["flat"][i:i + math.prod(n)].view(n) for i, n in zip(at, shapes)]
    s["grads"] = [s["grad"][i:i + math.prod(n)].view(n) for i, n in zip(at, shapes)]
    for p, g, i, n in zip(s["params"], s["grads"], at, shapes):
        p.copy_(weights[i:i + p.numel()].view(n) / math.sqrt(n[0]))
        g.copy_(grads[i:i + p.numel()].view(n) * (0.01 / math.sqrt(n[-1])))
    if case["bits"] == 32:
        s["m"] = 0.6 * s["grad"].float()
        s["v"] = 0.01 * s["grad"].float().square()
    else:
        zero = torch.zeros(at[-1], device="cuda")
        s["m"], s["v"] = zero.to(torch.float8_e4m3fn), zero.to(torch.float8_e4m3fn)
        s["m_scale"], s["v_scale"] = torch.ones(at[-1] // BLOCK, device="cuda"), torch.ones(at[-1] // BLOCK, device="cuda")
        # (moments as a step from zero leaves them, on the grid of the 8-bit type)
        m, v = 0.6 * s["grad"].float(), 0.1 * s["grad"].float().abs()
        for codes, scale, x in ((s["m"], s["m_scale"], m), (s["v"], s["v_scale"], v)):
            scale.copy_(_scale_of(x.view(-1, BLOCK).abs().amax(1)))
            codes.copy_((x.view(-1, BLOCK) / scale[:, None]).view(-1).to(torch.float8_e4m3fn))
    if own:
        from paper_2402_18994_amd import AdamW
        s["opt"] = AdamW(s["params"], lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY, state_bits=case["bits"], seed=s["seed"])
        s["opt"].load_state_dict({k: s[k] for k in ("step", "m", "v", "m_scale", "v_scale") if k in s})
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1009 + 17)

    def rand(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if case["do"] == "adamw":
        return _prepare_adamw(case, rand) | {"do": "adamw"}
    T, B, D, t = case["T"], case["B"], case["D"], TYPES[case["type"]]
    s = {"do": case["do"], "init": None, "lengths": None}
    if case["ragged"]:
        s["lengths"] = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    step = case["do"].endswith("step")
    lead = (B,) if step else (T, B)
    if case["do"].startswith("conv"):
        W = case["W"]
        s["x"] = rand(*lead, D).to(t)
        s["weight"], s["bias"] = rand(D, W) / math.sqrt(W), 0.1 * rand(D)
        if step:
            s["state"] = rand(W - 1, B, D).to(t)
        elif case["init"]:
            s["init"] = rand(W - 1, B, D).to(t)
        if case["do"] == "conv_train":
            s["dy"], s["d_state"] = rand(T, B, D).to(t), None
        return s
    N, G = case["N"], case["groups"]
    s["x"], s["dt"] = rand(*lead, D).to(t), (0.5 * rand(*lead, D)).to(t)
    s["B"], s["C"] = rand(*lead, G, N).to(t), rand(*lead, G, N).to(t)
    s["z"] = rand(*lead, D).to(t) if case["gate"] else None
    # decays over the usual range: state n of a channel forgets about n + 1 times as fast as its first one, and step
    # sizes from 0.001 to 0.1 behind the softplus
    s["A"] = -torch.exp(torch.log(torch.arange(1, N + 1, device="cuda").float()) + 0.2 * rand(D, N))
    step_size = torch.exp(torch.rand(D, generator=gen, device="cuda") * math.log(100.0) + math.log(0.001))
    s["dt_bias"] = step_size + torch.log(-torch.expm1(-step_size))
    s["D"] = 1 + 0.1 * rand(D)
    if step:
        s["state"] = rand(B, D, N)
    elif case["init"]:
        s["init"] = rand(B, D, N)
    if case["do"] == "scan_train":
        s["dy"], s["d_state"] = rand(T, B, D).to(t), (rand(B, D, N) if case["init"] else None)
    return s


# ------------------------------------------------------------------------------------------- convolution, plain

def _silu(x):
    return x * torch.sigmoid(x)


def _silu_slope(x):
    s = torch.sigmoid(x)
    return s * (1 + x * (1 - s))


def _valid(s, T, B):
    """[T, B, 1]: whether a step is within its sequence."""
    if s["lengths"] is None:
        return None
    return (torch.arange(T, device="cuda")[:, None] < s["lengths"][None, :])[..., None]


def _kept(s, T, B, K):
    """[K, B]: the rows of the extended input (K rows of `init`, then T rows) that the state keeps."""
    n = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device="cuda")
    return torch.arange(K, device="cuda")[:, None] + n[None, :]


def _conv_forward(s):
    x, w = s["x"], s["weight"]
    (T, B, D), W = x.shape, w.shape[1]
    before = s["init"] if s["init"] is not None else torch.zeros((W - 1, B, D), device="cuda", dtype=x.dtype)
    long = torch.cat((before, x)).float()
    pre = s["bias"] + sum(long[k:k + T] * w[:, k] for k in range(W))
    y, valid = _silu(pre), _valid(s, T, B)
    if valid is not None:
        y = torch.where(valid, y, torch.zeros_like(y))
    state = torch.gather(torch.cat((before, x)), 0, _kept(s, T, B, W - 1)[..., None].expand(W - 1, B, D))
    return y.to(x.dtype), state, long, pre


def _conv_backward(s, long, pre):
    x, w = s["x"], s["weight"]
    (T, B, D), W = x.shape, w.shape[1]
    d = s["dy"].float() * _silu_slope(pre)
    valid = _valid(s, T, B)
    if valid is not None:
        d = torch.where(valid, d, torch.zeros_like(d))
    d_long = torch.zeros_like(long)
    for k in range(W):
        d_long[k:k + T] += d * w[:, k]
    dw = torch.stack([(d * long[k:k + T]).sum((0, 1)) for k in range(W)], 1)
    out = {"dx": d_long[W - 1:].to(x.dtype), "dweight": dw, "dbias": d.sum((0, 1))}
    if s["init"] is not None:
        out["dinit"] = d_long[:W - 1].to(x.dtype)
    return out


def _conv_step(s):
    x, w, state = s["x"], s["weight"], s["state"]
    long = torch.cat((state, x[None]))
    y = _silu(s["bias"] + (long.float() * w.t()[:, None]).sum(0))
    state.copy_(long[1:])
    return {"y": y.to(x.dtype), "state": state}


# ---------------------------------------------------------------------------------------------------- scan, plain

def _softplus(x):
    return torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))


def _prefix(a, b):
    """h_t = a_t h_(t-1) + b_t along the first axis by doubling: log2(T) passes over all steps at once."""
    n = 1
    while n < len(a):
        b = torch.cat((b[:n], torch.addcmul(b[n:], a[n:], b[:-n])))
        a = torch.cat((a[:n], a[n:] * a[:-n]))
        n *= 2
    return b


def _spread(v, D):
    """[.., G, N] -> [.., D, N] in float32."""
    return v.float().repeat_interleave(D // v.shape[-2], -2)


def _scan_forward(s):
    x = s["x"].float()
    T, B, D = x.shape
    delta = _softplus(s["dt"].float() + s["dt_bias"])
    valid = _valid(s, T, B)
    if valid is not None:
        zero = torch.zeros_like(x)
        x, delta = torch.where(valid, x, zero), torch.where(valid, delta, zero)
    a = torch.exp(delta[..., None] * s["A"])
    b = (delta * x)[..., None] * _spread(s["B"], D)
    if s["init"] is not None:
        b[0] += a[0] * s["init"]
    h = _prefix(a, b)
    y0 = (h * _spread(s["C"], D)).sum(-1) + s["D"] * x
    y = y0 * _silu(s["z"].float()) if s["z"] is not None else y0
    if valid is not None:
        y = torch.where(valid, y, zero)
    return y.to(s["x"].dtype), h[-1].clone(), (x, delta, a, h, y0, valid)


def _scan_backward(s, x, delta, a, h, y0, valid):
    T, B, D = x.shape
    G, N = s["B"].shape[-2:]
    t, dy = s["x"].dtype, s["dy"].float()
    out = {}
    if valid is not None:
        dy = torch.where(valid, dy, torch.zeros_like(dy))
    if s["z"] is not None:
        z = s["z"].float()
        out["dz"] = (dy * y0 * _silu_slope(z)).to(t)
        dy = dy * _silu(z)
    g = dy[..., None] * _spread(s["C"], D)
    if s["d_state"] is not None:
        g[-1] += s["d_state"]
    after = torch.cat((a[1:], torch.ones_like(a[:1])))
    g = _prefix(after.flip(0), g.flip(0)).flip(0)
    Bd = _spread(s["B"], D)
    gB = (g * Bd).sum(-1)
    dx = gB * delta + dy * s["D"]
    first = s["init"] if s["init"] is not None else torch.zeros_like(h[0])
    ga = g * a
    u = ga * torch.cat((first[None], h[:-1]))
    out["dA"] = (u * delta[..., None]).sum((0, 1))
    d_delta = (u * s["A"]).sum(-1) + gB * x
    raw = s["dt"].float() + s["dt_bias"]
    ddt = d_delta * torch.sigmoid(raw)
    if valid is not None:
        zero = torch.zeros_like(dx)
        dx, ddt = torch.where(valid, dx, zero), torch.where(valid, ddt, zero)
    out["dx"], out["ddt"] = dx.to(t), ddt.to(t)
    out["ddt_bias"], out["dD"] = ddt.sum((0, 1)), (dy * x).sum((0, 1))
    out["dB"] = (g * (delta * x)[..., None]).view(T, B, G, D // G, N).sum(3).to(t)
    out["dC"] = (h * dy[..., None]).view(T, B, G, D // G, N).sum(3).to(t)
    if s["init"] is not None:
        out["dinit"] = ga[0]
    return out


def _scan_step(s):
    x, D = s["x"].float(), s["x"].shape[-1]
    delta = _softplus(s["dt"].float() + s["dt_bias"])
    h = torch.exp(delta[..., None] * s["A"]) * s["state"] + (delta * x)[..., None] * _spread(s["B"], D)
    s["state"].copy_(h)
    y = (h * _spread(s["C"], D)).sum(-1) + s["D"] * x
    if s["z"] is not None:
        y = y * _silu(s["z"].float())
    return {"y": y.to(s["x"].dtype), "state": s["state"]}


# --------------------------------------------------------------------------------------------------- AdamW, plain

def _scale_of(top):
    """The least power of two that brings `top` to at most 448, the largest value of the 8-bit type (from 2^-60 up)."""
    bits = top.view(torch.int32)
    e = ((bits + 0x1FFFFF) >> 23) - 127 - 8
    return torch.exp2(torch.clamp(e, min=-60).double()).float()


def _mix(x):
    """32 bits of a counter, stirred (in int64, of which the low 32 bits count)."""
    x = ((x ^ (x >> 16)) * 0xB504F335) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xDDB3D743) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _salt(seed, step):
    return _mix((seed * 0x9E3779B1 + step * 0x85EBCA77) & 0xFFFFFFFF)


def _grid(y):
    """Of magnitudes y <= 448: the exponent of the 8-bit type's binade and y in its steps there."""
    e = torch.clamp((y.view(torch.int32) >> 23) - 127, min=-6)
    return e, y * torch.exp2((3 - e).float())


def _codes(e, steps, sign):
    return ((e + 6) * 8 + steps.int() + sign * 128).to(torch.uint8).view(torch.float8_e4m3fn)


def _pack_m(m, rand):
    """First moments -> 8-bit codes and block scales: up or down with the probability that keeps the mean."""
    blocks = m.view(-1, BLOCK)
    scale = _scale_of(blocks.abs().amax(1))
    y = (blocks * (1 / scale)[:, None]).view(-1)
    e, a = _grid(y.abs())
    low = torch.floor(a)
    up = ((rand & 0xFFFF).float() + 0.5) * (1 / 65536) < a - low
    return _codes(e, low + up, (y < 0).int()), scale


def _pack_v(v, rand):
    """Second moments, kept as their roots; the mean that is kept is that of the moment itself, and one above zero
    never becomes zero."""
    blocks = v.view(-1, BLOCK)
    scale = _scale_of(torch.sqrt(blocks.amax(1)))
    inverse = (1 / scale)[:, None]
    w = (blocks * inverse * inverse).view(-1)
    e, a = _grid(torch.sqrt(w))
    low = torch.floor(a)
    step = torch.exp2((e - 3).float())
    lo, hi = low * step, (low + 1) * step
    up = ((rand >> 16).float() + 0.5) * (1 / 65536) * (hi * hi - lo * lo) < w - lo * lo
    up = up | ((w > 0) & (e == -6) & (low == 0))
    return _codes(e, low + up, 0), scale


def _adamw_step(s):
    """All tensors at once: they lie in one buffer each here, with zeros in the gaps, which a step leaves as they are."""
    s["step"] += 1
    k1, k2 = LR / (1 - BETA1 ** s["step"]), 1 / math.sqrt(1 - BETA2 ** s["step"])
    p, g, m, v = s["flat"], s["grad"].float(), s["m"], s["v"]
    if s["bits"] == 8:
        m = (m.float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (v.float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1).square()
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    p.copy_(p * (1 - LR * DECAY) - m * k1 / (torch.sqrt(v) * k2 + EPS))
    if s["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        where = torch.arange(len(p), device="cuda")
        rand = _mix(((where & 0xFFFFFFFF) * 0x9E3779B1 + (where >> 32) * 0xC2B2AE3D + _salt(s["seed"], s["step"])) & 0xFFFFFFFF)
        s["m"], s["m_scale"] = _pack_m(m, rand)
        s["v"], s["v_scale"] = _pack_v(v, rand)
    return {k: s[k] for k in ("flat", "m", "v", "m_scale", "v_scale") if k in s}


# -------------------------------------------------------------------------------------------- the library's calls

def _run_own(s):
    import paper_2402_18994_amd as snn
    do = s["do"]
    if do == "adamw":
        s["opt"].step(s["grads"])
        return {"flat": s["flat"]} | {k: v for k, v in s["opt"].state_dict().items() if k != "step"}
    if do == "conv_step":
        return {"y": snn.causal_conv_step(s["x"], s["state"], s["weight"], s["bias"]), "state": s["state"]}
    if do == "scan_step":
        y = snn.selective_scan_step(s["x"], s["dt"], s["state"], s["A"], s["B"], s["C"], s["D"], s["z"], s["dt_bias"])
        return {"y": y, "state": s["state"]}
    if do.startswith("conv"):
        y, state = snn.causal_conv(s["x"], s["weight"], s["bias"], init=s["init"], lengths=s["lengths"])
        out = {"y": y, "state": state}
        if do == "conv_train":
            g = snn.causal_conv_backward(s["dy"], s["x"], s["weight"], s["bias"], init=s["init"], lengths=s["lengths"])
            out |= {k: v for k, v in g._asdict().items() if v is not None}
        return out
    train = do == "scan_train"
    y, state, saved = snn.selective_scan(s["x"], s["dt"], s["A"], s["B"], s["C"], s["D"], s["z"], s["dt_bias"],
                                         init=s["init"], lengths=s["lengths"], save=train)
    out = {"y": y, "state": state}
    if train:
        g = snn.selective_scan_backward(s["dy"], saved, s["x"], s["dt"], s["A"], s["B"], s["C"], s["D"], s["z"], s["dt_bias"],
                                        init=s["init"], lengths=s["lengths"], d_state=s["d_state"])
        out |= {k: v for k, v in g._asdict().items() if v is not None}
    return out


def run(s):
    if own:
        return _run_own(s)
    do = s["do"]
    if do == "adamw":
        return _adamw_step(s)
    if do == "conv_step":
        return _conv_step(s)
    if do == "scan_step":
        return _scan_step(s)
    if do.startswith("conv"):
        y, state, long, pre = _conv_forward(s)
        return {"y": y, "state": state} | (_conv_backward(s, long, pre) if do == "conv_train" else {})
    y, state, kept = _scan_forward(s)
    return {"y": y, "state": state} | (_scan_backward(s, *kept) if do == "scan_train" else {})


def work(case):
    if case["do"] == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * (8 + SIZE[case["type"]] + state), "flops": n * 14}
    T, B, D, z = case["T"], case["B"], case["D"], SIZE[case["type"]]
    e, train = T * B * D, case["do"].endswith("train")
    if case["do"].startswith("conv"):
        W = case["W"]
        streams = 4 if train else 2                       # x, y, and dy, dx
        state = (W - 1) * B * D * z * (2 if case["do"] == "conv_step" or case["init"] else 1)
        return {"bytes": e * streams * z + state + 4 * D * (W + 1) * (2 if train else 1), "flops": e * (2 * W + 5) * (3 if train else 1)}
    N, G = case["N"], case["groups"]
    gate = int(case["gate"])
    streams = 3 + gate + (3 + gate if train else 0)       # x, dt, y, z, and dy, dx, ddt, dz
    rows = T * B * G * N * 2 * z * (2 if train else 1)
    state = B * D * N * 4 * (2 if case["do"] == "scan_step" or case["init"] else 1)
    return {"bytes": e * streams * z + rows + state + D * (N + 2) * 4 * (2 if train else 1), "flops": e * (N * (20 if train else 7) + 12)}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _exact_conv(s):
    x, w, bias = s["x"].double(), s["weight"].double(), s["bias"].double()
    if s["do"] == "conv_step":
        x, past = x[None], s["state"].double()
    else:
        past = s["init"].double() if s["init"] is not None else x.new_zeros((w.shape[1] - 1,) + x.shape[1:])
    T, W = len(x), w.shape[1]
    lengths = [T] * x.shape[1] if s["lengths"] is None else s["lengths"].tolist()
    window = past.unbind(0) + x.unbind(0)
    train = s["do"] == "conv_train"
    y, dx = torch.zeros_like(x), torch.zeros_like(torch.stack(window))
    dw, db = torch.zeros_like(w), torch.zeros_like(bias)
    live = torch.tensor(lengths, device="cuda")
    for t in range(T):
        on = (t < live)[:, None]
        taps = torch.stack(window[t:t + W], -1)
        v = (taps * w).sum(-1) + bias
        gate = 1 / (1 + torch.exp(-v))
        y[t] = torch.where(on, v * gate, 0.0)
        if train:
            d = torch.where(on, s["dy"][t].double() * (gate + v * gate * (1 - gate)), 0.0)
            dx[t:t + W] += torch.movedim(d[..., None] * w, -1, 0)
            dw += (d[..., None] * torch.where(on[..., None], taps, 0.0)).sum(0)
            db += d.sum(0)
    state = torch.stack([torch.stack([window[n + j][b] for b, n in enumerate(lengths)]) for j in range(W - 1)])
    out = {"y": y[0] if s["do"] == "conv_step" else y, "state": state}
    if train:
        out |= {"dx": dx[W - 1:], "dweight": dw, "dbias": db}
        if s["init"] is not None:
            out["dinit"] = dx[:W - 1]
    return out


def _exact_scan(s):
    step = s["do"] == "scan_step"
    lead = (lambda v: v.double()[None]) if step else (lambda v: v.double())
    x, A, skip = lead(s["x"]), s["A"].double(), s["D"].double()
    Bv, Cv, z = lead(s["B"]), lead(s["C"]), lead(s["z"]) if s["z"] is not None else None
    raw = lead(s["dt"]) + s["dt_bias"].double()
    delta = torch.logaddexp(raw, torch.zeros_like(raw))
    T, nB, nD = x.shape
    G, N = Bv.shape[2:]
    group = torch.arange(nD, device="cuda") // (nD // G)
    h = s["state"].double() if step else s["init"].double() if s["init"] is not None else x.new_zeros((nB, nD, N))
    live = torch.full((nB,), T, device="cuda") if s["lengths"] is None else s["lengths"]
    train = s["do"] == "scan_train"
    y, inner, past = torch.zeros_like(x), torch.zeros_like(x), []
    for t in range(T):
        on = (t < live)[:, None]
        past.append(h if train else None)
        new = torch.exp(delta[t][..., None] * A) * h + (delta[t] * x[t])[..., None] * Bv[t][:, group]
        h = torch.where(on[..., None], new, h)
        inner[t] = (h * Cv[t][:, group]).sum(-1) + skip * x[t]
        y[t] = torch.where(on, inner[t] * (z[t] / (1 + torch.exp(-z[t])) if z is not None else 1.0), 0.0)
    out = {"y": y[0] if step else y, "state": h}
    if not train:
        return out
    q = s["d_state"].double() if s["d_state"] is not None else torch.zeros_like(h)
    d = {"dx": torch.zeros_like(x), "ddt": torch.zeros_like(x), "dA": torch.zeros_like(A), "dB": torch.zeros_like(Bv),
         "dC": torch.zeros_like(Cv), "dD": torch.zeros_like(skip), "ddt_bias": torch.zeros_like(skip)}
    if z is not None:
        d["dz"] = torch.zeros_like(x)
    after = h
    for t in reversed(range(T)):
        on = (t < live)[:, None]
        dy = torch.where(on, s["dy"][t].double(), 0.0)
        if z is not None:
            gate = 1 / (1 + torch.exp(-z[t]))
            d["dz"][t] = dy * inner[t] * (gate + z[t] * gate * (1 - gate))
            dy = dy * z[t] * gate
        b, c = Bv[t][:, group], Cv[t][:, group]
        g = q + dy[..., None] * c
        d["dC"][t].index_add_(1, group, after * dy[..., None])
        decay = torch.exp(delta[t][..., None] * A)
        live_g = torch.where(on[..., None], g, 0.0)
        d["dB"][t].index_add_(1, group, live_g * (delta[t] * x[t])[..., None])
        along_b = (live_g * b).sum(-1)
        pull = live_g * past[t] * decay
        d["dx"][t] = dy * skip + along_b * delta[t]
        d["ddt"][t] = ((pull * A).sum(-1) + along_b * x[t]) / (1 + torch.exp(-raw[t]))
        d["dA"] += (pull * delta[t][..., None]).sum(0)
        d["dD"] += (dy * x[t]).sum(0)
        d["ddt_bias"] += d["ddt"][t].sum(0)
        q = torch.where(on[..., None], g * decay, q)
        after = past[t]
    if s["init"] is not None:
        d["dinit"] = q
    return out | d


def _exact_adamw(s):
    """Parameters and 32-bit moments; what is rounded to 8 bits has no value in 64."""
    t = s["step"] + 1
    m, v, g = s["m"].double(), s["v"].double(), s["grad"].double()
    if s["bits"] == 8:
        m = m * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (v * s["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    update = (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + EPS)
    p = s["flat"].double()
    p = p - LR * DECAY * p - LR * update
    if s["bits"] == 8:
        return {"flat": p, "m": None, "v": None, "m_scale": None, "v_scale": None}
    return {"flat": p, "m": m, "v": v}


def exact(case, seed):
    s = prepare(case, seed)
    if case["do"] == "adamw":
        return _exact_adamw(s)
    return _exact_conv(s) if case["do"].startswith("conv") else _exact_scan(s)
