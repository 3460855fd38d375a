"""The gated block's operators at the ends of what they accept, on the GPU: magnitudes, counts, and the tails of an activation.

Each tolerance is derived where it stands; 2^-24 is half a step of fp32."""
import math

import pytest
import torch

from tests import block_oracle as oracle
from tests.seq_oracle import gradients
from tests.test_seq_ops import TYPES, close, half_step, on_gpu, rand, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", (8, 900))
def test_group_norm_of_values_whose_squares_overflow(T):
    """fp32 values around 3e19 with a spread of a thousandth of that, whose squares around the mean are fp32 numbers and whose own
    are not: in one workgroup, and in chunks.  A mean goes through less than 40 roundings (additions of a thread's rows, over lanes, wavefronts and chunks), each
    2^-24 of itself, 1000 2^-24 of the spread; what else there is is 2^-24 of an output."""
    from paper_2402_18994_amd import group_norm
    gen = torch.Generator().manual_seed(T)
    x = rounded(3e19 + 3e16 * rand(gen, T, 3, 64))
    n = torch.tensor([T, T // 2 + 1, 0], dtype=torch.int32)
    (want,) = oracle.norm(x, 2, silu=False, lengths=n)
    y = group_norm(on_gpu(x), 2, silu=False, lengths=on_gpu(n, torch.int32)).y.double().cpu()
    assert torch.isfinite(y).all() and (y - want).abs().max().item() < 40 * 1000 * 2.0 ** -24


@pytest.mark.parametrize("type", tuple(TYPES))
@pytest.mark.parametrize("T", (8, 900))
@pytest.mark.parametrize("value", (-2.0 ** 100, 3000.0))
def test_group_norm_of_equal_values(value, T, type):
    """Their deviations are zero, and the outputs the activation of the bias: in one workgroup, and in chunks."""
    from paper_2402_18994_amd import group_norm
    gen = torch.Generator().manual_seed(T)
    bias, t = rounded(rand(gen, 64)), TYPES[type]
    x = on_gpu(torch.full((T, 3, 64), value), t)
    y = group_norm(x, 2, bias=on_gpu(bias)).y
    close("y", y, (bias / (1 + torch.exp(-bias))).expand(T, 3, 64), 1, half_step(t))


@pytest.mark.parametrize("type", tuple(TYPES))
@pytest.mark.parametrize("T", (4, 900))
@pytest.mark.parametrize("value", (-2.0 ** 100, 3000.0, 2.0 ** 120))
def test_group_norm_gradients_of_equal_values(value, T, type):
    """Deviations of zero: dweight is zero, dbias = sum q with q = dy silu'(bias), dx = rstd (p - mean(p)) with p = q w, rstd = eps^(-1/2)."""
    from paper_2402_18994_amd import group_norm, group_norm_backward
    gen = torch.Generator().manual_seed(T)
    w, bias, t = rounded(1 + 0.2 * rand(gen, 64)), rounded(rand(gen, 64)), TYPES[type]
    dy, x = rounded(rand(gen, T, 3, 64), t), on_gpu(torch.full((T, 3, 64), value), t)
    saved = group_norm(x, 2, on_gpu(w), on_gpu(bias), save=True).saved
    g = group_norm_backward(on_gpu(dy, t), saved, x, 2, on_gpu(w), on_gpu(bias))
    s = 1 / (1 + torch.exp(-bias))
    q = dy * s * (1 + bias * (1 - s))
    p = (q * w).view(T, 3, 2, 32)
    dx = ((p - p.mean((0, 3), keepdim=True)) / math.sqrt(1e-5)).view(T, 3, 64)
    assert (g.dweight == 0).all()
    close("dbias", g.dbias, q.sum((0, 1)), 3 * T, 2.0 ** -24)
    close("dx", g.dx, dx, 32 * T, half_step(t))


@pytest.mark.parametrize("T,C", ((4, 1), (2, 8)))
def test_group_norm_of_many_sequences_and_groups(T, C):
    """2^24 of them, more workgroups of 256 than a launch's first dimension counts threads: one channel a group, and eight (whose reverse pass
    runs in chunks).  Sequences stand alone, so the last ones are those of a call of their own; sums of whole numbers are exact."""
    from paper_2402_18994_amd import group_norm, group_norm_backward
    B, G = 1 << 16, 256
    gen = torch.Generator("cuda").manual_seed(T)
    x = torch.randn(T, B, G * C, device="cuda", generator=gen).to(torch.bfloat16)
    dy = torch.randint(-1, 2, (T, B, G * C), device="cuda", generator=gen, dtype=torch.int8).to(torch.bfloat16)
    bias = torch.zeros(G * C, device="cuda")
    o = group_norm(x, G, None, bias, silu=False, save=True)
    g = group_norm_backward(dy, o.saved, x, G, None, bias, silu=False)
    for at in (slice(0, 3), slice(B // 2 - 1, B // 2 + 2), slice(B - 3, B)):
        few = group_norm(x[:, at], G, None, bias, silu=False, save=True)
        assert torch.equal(o.y[:, at], few.y)
        assert torch.equal(g.dx[:, at], group_norm_backward(dy[:, at], few.saved, x[:, at], G, None, bias, silu=False).dx)
    assert torch.equal(g.dbias.double(), dy.sum((0, 1), dtype=torch.float64))


@pytest.mark.parametrize("rows", (1, 300))
def test_gelu_far_from_zero(rows):
    """GELU and its slope where they are small, every value by itself: units of one input, x = 1 and up = 1, give act(gate), and with dy = 1 dup is act(gate)
    and dgate is act'(gate) in each of `rows` equal rows.

    Off by: z = g / sqrt(2) is rounded twice, 2^-23 of itself, which moves erfc(z), whose logarithm's slope is -(2 z + 1 / z) at most, by (g^2 + 1)
    2^-23 of itself; ten halves of a last place for erfc itself and the products.  In the slope exp(-g^2 / 2) has its argument rounded four times, 2 g^2
    2^-24, and where g < -3 the terms, which differ in sign, are at most 1.3 times their sum.  Sums of equal rows: sqrt(rows) 2^-24 more, rows 2^-24 at most."""
    from paper_2402_18994_amd import gated_units, gated_units_backward
    for low, high in ((-9.0, -3.0), (0.25, 9.0)):
        g = rounded(torch.linspace(low, high, 193, dtype=torch.float64))
        x, gate, up = torch.ones(rows, 1, 1, device="cuda"), on_gpu(g)[:, None], torch.ones(193, 1, device="cuda")
        o = gated_units(x, gate, up, act="gelu", save=True)
        d = gated_units_backward(torch.ones_like(o.y), o.saved, x, gate, up, act="gelu")
        act = 0.5 * g * torch.erfc(-g * 0.5 ** 0.5)
        slope = 0.5 * torch.erfc(-g * 0.5 ** 0.5) + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
        off = (g * g + 1) * 2.0 ** -23 + 10 * 2.0 ** -24
        sums = rows * 2.0 ** -24 if rows > 1 else 0.0
        for name, got, want, tol in (("y", o.y[0, 0], act, off), ("last y", o.y[-1, 0], act, off), ("dup", d.dup[:, 0] / rows, act, off + sums),
                                     ("dgate", d.dgate[:, 0] / rows, slope, 1.3 * (off + g * g * 2.0 ** -23 + 4 * 2.0 ** -24) + sums)):
            worst = ((got.double().cpu() - want).abs() / want.abs() / tol).max().item()
            assert worst <= 1, (name, low, worst)


@pytest.mark.parametrize("T,C,per_step", ((4, 32, False), (900, 32, False), (6, 32, True), (6, 1024, True), (6, 4096, True)))
@pytest.mark.parametrize("type", tuple(TYPES))
def test_group_norm_of_the_least_spread(T, C, per_step, type):
    """Values of +-2^-65 and no eps: the variance, 2^-130, is below the least normal number, and the outputs are +-1 all the same."""
    from paper_2402_18994_amd import group_norm, group_norm_backward
    gen = torch.Generator().manual_seed(C)
    t = TYPES[type]
    sign = 1.0 - 2.0 * (torch.arange(2 * C) % 2).double().expand(T, 3, 2 * C)
    x, dy = sign * 2.0 ** -65, rounded(rand(gen, T, 3, 2 * C), t)
    kw = dict(silu=False, eps=0.0, per_step=per_step)
    o = group_norm(on_gpu(x, t), 2, save=True, **kw)
    assert torch.equal(o.y.double().cpu(), sign)
    g = group_norm_backward(on_gpu(dy, t), o.saved, on_gpu(x, t), 2, **kw)
    want = gradients(lambda **k: oracle.norm(k["x"], 2, **kw), {"x": x}, (dy,))
    close("dx", g.dx, want["x"], C * (1 if per_step else T), half_step(t))


def test_units_gradients_of_no_steps():
    """Matrices of 2^32 elements, more than a launch's first dimension counts threads, get gradients of zero."""
    from paper_2402_18994_amd import gated_units, gated_units_backward
    F = D = 1 << 16
    x, gate, up = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((0, 1, D), (F, D), (F, D)))
    o = gated_units(x, gate, up, save=True)
    g = gated_units_backward(o.y, o.saved, x, gate, up)
    for v in (g.dgate, g.dup):
        assert not v.view(torch.int64).any()


@pytest.mark.parametrize("T", (1, 20, 200))
def test_recurrence_of_the_largest_sharpness(T):
    """3e38 is a finite number: channels with a decay of -inf keep their state for good, those with any other forget at once, y = sigmoid(i) x."""
    from paper_2402_18994_amd import gated_recurrence, gated_recurrence_backward, gated_recurrence_step
    B, D = 2, 70
    gen = torch.Generator().manual_seed(T)
    x, i, r, init = (rounded(rand(gen, *s)) for s in ((T, B, D), (T, B, D), (T, B, D), (B, D)))
    decay = torch.where(torch.arange(D) % 2 == 0, float("-inf"), 0.0).float().cuda()
    args = [on_gpu(v) for v in (x, i, r)]
    want = torch.where(torch.arange(D) % 2 == 0, init, x / (1 + torch.exp(-i)))
    o = gated_recurrence(*args, decay, sharpness=3e38, init=on_gpu(init), save=True)
    close("y", o.y, want, 1, 2.0 ** -24)
    g = gated_recurrence_backward(torch.ones_like(args[0]), o.saved, *args, decay, sharpness=3e38, init=on_gpu(init))
    assert all(torch.isfinite(v).all() for v in g)
    assert torch.equal(g.dinit.cpu(), torch.where(torch.arange(D) % 2 == 0, float(T), 0.0).expand(B, D))
    state = on_gpu(init)
    close("step", gated_recurrence_step(*(v[0] for v in args), state, decay, sharpness=3e38), want[0], 1, 2.0 ** -24)


@pytest.mark.parametrize("T,C,per_step", ((8, 64, False), (900, 64, False), (8, 64, True), (8, 1024, True)))
def test_group_norm_of_a_variance_beyond_fp32(T, C, per_step):
    """Values of +-1e20, whose squares are no fp32 numbers, give the outputs of a deviation of zero, as the header says, and finite gradients."""
    from paper_2402_18994_amd import group_norm, group_norm_backward
    gen = torch.Generator().manual_seed(C)
    bias = rounded(rand(gen, 2 * C))
    x = on_gpu((1e20 - 2e20 * (torch.arange(2 * C) % 2)).expand(T, 3, 2 * C).contiguous())
    o = group_norm(x, 2, bias=on_gpu(bias), per_step=per_step, save=True)
    close("y", o.y, (bias / (1 + torch.exp(-bias))).expand(T, 3, 2 * C), 1, 2.0 ** -24)
    g = group_norm_backward(torch.ones_like(x), o.saved, x, 2, bias=on_gpu(bias), per_step=per_step)
    assert torch.isfinite(g.dx).all() and torch.isfinite(g.dbias).all()


@pytest.mark.parametrize("T,C,per_step", ((7, 40, False), (300, 30, False), (7, 24, True), (5, 100, True), (5, 650, True), (5, 1000, True), (5, 5000, True)))
@pytest.mark.parametrize("type", tuple(TYPES))
def test_group_norm_of_equal_values_whatever_their_number(T, C, per_step, type):
    """Numbers of values that are no powers of two: the mean of equal ones, whose sum is exact, is their value all the same, and the outputs are the activation of the
    bias.  (Rows of more than 512 channels are a wavefront's, which holds them or loads them again; 40 sequences of 300 steps go through wide workgroups.)"""
    from paper_2402_18994_amd import group_norm, group_norm_backward
    gen = torch.Generator().manual_seed(C)
    B, t = 40 if T == 300 else 3, TYPES[type]
    bias = rounded(rand(gen, 2 * C))
    x = on_gpu(torch.tensor([3000.0, -11.0]).repeat_interleave(C).expand(T, B, 2 * C).contiguous(), t)
    o = group_norm(x, 2, bias=on_gpu(bias), per_step=per_step, save=True)
    close("y", o.y, (bias / (1 + torch.exp(-bias))).expand(T, B, 2 * C), 1, half_step(t))
    g = group_norm_backward(torch.ones_like(x), o.saved, x, 2, on_gpu(torch.ones(2 * C)), on_gpu(bias), per_step=per_step)
    assert (g.dweight == 0).all()
