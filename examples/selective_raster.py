"""A sequence classifier over spike rasters from the sequence operators: trained on whole rasters, served step by step.

    raster -> product -> short convolution -> selective scan -> product, mean over time -> class

The raster is that of a named configuration of workloads.py; each class is given channel rates of its own, so that there is
something to learn.  Training runs the convolution and the scan with their gradients and one AdamW step for all
tensors (moments in 32 or in 8 bits); serving feeds the same rasters one step at a time through the token forms, which
carry the convolution's last inputs and the scan's state, and has to come to the same classes.

    python examples/selective_raster.py [--config shd_ff128] [--width 256] [--states 16] [--steps 60] [--state-bits 8]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import workloads                                                                    # noqa: E402
import paper_2402_18994_amd as snn                                                  # noqa: E402

TAPS = 4


def parameters(channels, width, states, classes, seed):
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen)
    step = torch.exp(torch.rand(width, generator=gen) * 4.6 - 6.9)                  # 0.001 to 0.1
    p = {"W_in": rand(channels, 2 * width) / channels ** 0.5 * 3, "filter": rand(width, TAPS) / TAPS ** 0.5, "filter_bias": torch.zeros(width),
         "W_step": rand(width, width + 2 * states) / width ** 0.5, "dt_bias": step + torch.log(-torch.expm1(-step)),
         "A": -torch.arange(1, states + 1).float().expand(width, states).contiguous(), "skip": torch.ones(width), "W_out": rand(width, classes) / width ** 0.5}
    return {k: v.cuda() for k, v in p.items()}


class Classifier:
    def __init__(self, p, states, type=torch.bfloat16):
        self.p, self.N, self.type = p, states, type

    def _split(self, u):
        width = self.p["skip"].numel()
        q = u @ self.p["W_step"].to(self.type)
        return q[..., :width], q[..., width:width + self.N], q[..., width + self.N:]

    def forward(self, raster):
        """-> class scores [B, C] and what backward needs."""
        p, width = self.p, self.p["skip"].numel()
        s = raster.to(self.type)
        xz = s @ p["W_in"].to(self.type)
        x, z = xz[..., :width], xz[..., width:]
        u, _ = snn.causal_conv(x, p["filter"], p["filter_bias"])
        dt, B, C = self._split(u)
        out = snn.selective_scan(u, dt, p["A"], B, C, p["skip"], z, p["dt_bias"], save=True)
        return out.y.float().mean(0) @ p["W_out"], (s, x, z, u, dt, B, C, out)

    def backward(self, d_scores, kept):
        p = self.p
        s, x, z, u, dt, B, C, out = kept
        T, nb, width = u.shape
        mean = out.y.float().mean(0)
        dy = ((d_scores @ p["W_out"].t()) / T).to(self.type).expand(T, nb, width)
        g = snn.selective_scan_backward(dy, out.saved, u, dt, p["A"], B, C, p["skip"], z, p["dt_bias"])
        dq = torch.cat((g.ddt, g.dB, g.dC), -1)
        du = g.dx + dq @ p["W_step"].to(self.type).t().contiguous()
        c = snn.causal_conv_backward(du, x, p["filter"], p["filter_bias"])
        dxz = torch.cat((c.dx, g.dz), -1)
        rows = lambda v: v.reshape(T * nb, -1)
        return {"W_in": (rows(s).t() @ rows(dxz)).float(), "filter": c.dweight, "filter_bias": c.dbias, "W_step": (rows(u).t() @ rows(dq)).float(),
                "dt_bias": g.ddt_bias, "A": g.dA, "skip": g.dD, "W_out": mean.t() @ d_scores}

    def stream(self, raster):
        """The same scores, one step of every sequence at a time."""
        p, width = self.p, self.p["skip"].numel()
        T, nb = raster.shape[:2]
        window = torch.zeros(TAPS - 1, nb, width, device="cuda", dtype=self.type)
        state = torch.zeros(nb, width, self.N, device="cuda")
        total = torch.zeros(nb, width, device="cuda")
        for t in range(T):
            xz = raster[t].to(self.type) @ p["W_in"].to(self.type)
            u = snn.causal_conv_step(xz[:, :width], window, p["filter"], p["filter_bias"])
            dt, B, C = self._split(u)
            total += snn.selective_scan_step(u, dt, state, p["A"], B, C, p["skip"], xz[:, width:], p["dt_bias"])
        return (total / T) @ p["W_out"]


def rasters(wl, classes, seed):
    """Rasters of the configuration's size: channel rates are drawn once per class, spikes independently."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rates = 0.005 + 0.035 * torch.rand(classes, wl.sizes[0], generator=torch.Generator().manual_seed(3)).cuda()
    labels = torch.randint(0, classes, (wl.B,), generator=gen, device="cuda")
    return (torch.rand(wl.T, wl.B, wl.sizes[0], generator=gen, device="cuda") < rates[labels]), labels


def train(config="shd_ff128", width=256, states=16, steps=60, lr=3e-3, state_bits=8, seed=0, say=print):
    wl = workloads.CONFIGS[config]
    classes = wl.sizes[-1]
    p = parameters(wl.sizes[0], width, states, classes, seed)
    model, names = Classifier(p, states), sorted(p)
    decay = [0.01 if k.startswith("W_") else 0.0 for k in names]
    opt = snn.AdamW([p[k] for k in names], lr=lr, weight_decay=decay, state_bits=state_bits, seed=seed)
    losses = []
    for i in range(steps):
        x, labels = rasters(wl, classes, seed + 100 + i)
        scores, kept = model.forward(x)
        losses.append(torch.nn.functional.cross_entropy(scores, labels))
        d = torch.softmax(scores, 1)
        d[torch.arange(len(labels), device="cuda"), labels] -= 1
        grads = model.backward(d / len(labels), kept)
        opt.step([grads[k].contiguous() for k in names])
        if i % 20 == 19:
            say("step %d: loss %.4f" % (i + 1, losses[-1].item()))
    x, labels = rasters(wl, classes, seed + 99)
    whole, _ = model.forward(x)
    tokens = model.stream(x)
    return {"first": losses[0].item(), "last": losses[-1].item(), "right": (whole.argmax(1) == labels).float().mean().item(),
            "apart": ((whole - tokens).norm() / whole.norm()).item(), "same": (whole.argmax(1) == tokens.argmax(1)).float().mean().item()}


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    a.add_argument("--config", default="shd_ff128", choices=sorted(workloads.CONFIGS))
    a.add_argument("--width", type=int, default=256)
    a.add_argument("--states", type=int, default=16)
    a.add_argument("--steps", type=int, default=60)
    a.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    o = a.parse_args()
    r = train(o.config, o.width, o.states, o.steps, state_bits=o.state_bits)
    print("loss %.4f -> %.4f; %.1f %% of new rasters right; streamed scores %.2g apart, %.1f %% of the classes the same"
          % (r["first"], r["last"], 100 * r["right"], r["apart"], 100 * r["same"]))
