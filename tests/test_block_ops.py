"""The operators of a gated block with their gradients on the GPU against their definitions in 64 bits (block_oracle.py), at the sizes and masks where they can go wrong.

Tolerances are those of test_seq_ops.py: half a step of the type that a value is rounded to, and TERM sqrt(n + 16) 2^-24 of the
tensor's scale for the fp32 chain before it, n the number of terms that come together in a value."""
import math

import pytest
import torch

from tests import block_oracle as oracle
from tests.seq_oracle import gradients
from tests.test_seq_ops import TYPES, close, half_step, lengths_of, on_gpu, rand, rounded

pytestmark = pytest.mark.gpu


def dead(v, n, with_=float("nan")):
    """A copy with `with_` in the steps that do not exist."""
    v = v.clone()
    if n is not None:
        for b in range(v.shape[1]):
            v[int(n[b]):, b] = with_
    return v


def same(a, b):
    return all((p is None and q is None) or torch.equal(p, q) for p, q in zip(a, b))


# ------------------------------------------------------------------------------------------------ recurrence

REC = [  # T, B, D, type, init, lengths
    (1, 1, 1, "fp32", False, "none"),
    (1, 3, 8, "bf16", True, "none"),
    (2, 2, 64, "fp32", True, "some"),
    (7, 5, 65, "bf16", True, "some"),
    (8, 1, 66, "bf16", False, "none"),
    (9, 3, 130, "fp32", True, "some"),
    (63, 2, 128, "bf16", False, "some"),
    (64, 2, 129, "fp32", True, "none"),
    (65, 4, 40, "bf16", True, "some"),
    (128, 3, 20, "fp32", False, "some"),
    (129, 1, 256, "bf16", True, "none"),
    (300, 90, 192, "bf16", True, "some"),            # workgroups for the whole chip: one segment
    (300, 86, 191, "fp32", True, "some"),
    (1100, 2, 72, "fp32", True, "some"),             # cut along time
    (2050, 1, 33, "bf16", True, "none"),
    (40, 3, 16, "bf16", True, "zero"),
    (0, 2, 8, "fp32", True, "none"),
]


def rec_case(T, B, D, type, init, lengths):
    gen = torch.Generator().manual_seed(T * 137 + D)
    t = TYPES[type]
    x, i, r = (rounded(rand(gen, T, B, D), t) for _ in range(3))
    decay = rounded(rand(gen, D) - 3)
    return gen, t, x, i, r, decay, rounded(rand(gen, B, D)) if init else None, lengths_of(lengths, T, B, gen)


@pytest.mark.parametrize("case", REC, ids=lambda c: "-".join(map(str, c)))
def test_recurrence_and_its_gradients(case):
    from paper_2402_18994_amd import gated_recurrence, gated_recurrence_backward
    T, B, D, _, _, _ = case
    gen, t, x, i, r, decay, init, n = rec_case(*case)
    print(f"\n[case] recurrence {case}", flush=True)
    gx, gi, gr = (on_gpu(dead(v, n), t) for v in (x, i, r))
    gd, g0, gn = on_gpu(decay), on_gpu(init), on_gpu(n, torch.int32)
    y, state, saved = gated_recurrence(gx, gi, gr, gd, init=g0, lengths=gn, save=True)
    wy, ws = oracle.recurrence(x, i, r, decay, init=init, lengths=n)
    h = half_step(t)
    close("y", y, wy, T, h)
    close("state", state, ws, T, 2.0 ** -24)
    bare = gated_recurrence(gx, gi, gr, gd, init=g0, lengths=gn)
    assert bare.saved is None and torch.equal(bare.y, y) and torch.equal(bare.state, state)
    dy, ds = rounded(rand(gen, T, B, D), t), rounded(rand(gen, B, D))
    args = (on_gpu(dead(dy, n), t), saved, gx, gi, gr, gd)
    g = gated_recurrence_backward(*args, init=g0, lengths=gn, d_state=on_gpu(ds))
    want = gradients(lambda **k: oracle.recurrence(k["x"], k["i"], k["r"], k["decay"], init=k.get("init"), lengths=n),
                     {"x": x, "i": i, "r": r, "decay": decay, "init": init}, (dy, ds))
    for name, got in (("x", g.dx), ("i", g.di), ("r", g.dr)):
        close("d" + name, got, want[name], T, h)
    close("ddecay", g.ddecay, want["decay"], T * B, 2.0 ** -24)
    assert (g.dinit is None) == (init is None)
    if init is not None:
        close("dinit", g.dinit, want["init"], T, 2.0 ** -24)
    assert same(g, gated_recurrence_backward(*args, init=g0, lengths=gn, d_state=on_gpu(ds)))


@pytest.mark.parametrize("B,D,type", [(1, 1, "fp32"), (3, 8, "bf16"), (5, 130, "bf16"), (2, 67, "fp32")])
def test_recurrence_steps_are_the_recurrence(B, D, type):
    from paper_2402_18994_amd import gated_recurrence, gated_recurrence_step
    T = 21
    _, t, x, i, r, decay, _, _ = rec_case(T, B, D, type, False, "none")
    gx, gi, gr, gd = on_gpu(x, t), on_gpu(i, t), on_gpu(r, t), on_gpu(decay)
    whole = gated_recurrence(gx, gi, gr, gd)
    begun = gated_recurrence(gx[:10], gi[:10], gr[:10], gd)
    state, ys = begun.state, [begun.y]
    for k in range(10, T):
        ys.append(gated_recurrence_step(gx[k], gi[k], gr[k], state, gd)[None])
    wy, ws = oracle.recurrence(x, i, r, decay)
    close("y", torch.cat(ys), wy, T, half_step(t))
    close("state", state, ws, T, 2.0 ** -24)
    close("whole", whole.state, ws, T, 2.0 ** -24)


@pytest.mark.parametrize("type", ("fp32", "bf16"))
@pytest.mark.parametrize("how", ("batch first", "parts of rows", "odd start"))
def test_recurrence_strides(type, how):
    """Batch-major memory, parts of wider rows, rows that start at an odd channel: the same values."""
    from paper_2402_18994_amd import gated_recurrence, gated_recurrence_backward
    T, B, D = 70, 3, 68
    gen, t, x, i, r, decay, init, n = rec_case(T, B, D, type, True, "some")

    def place(v):
        if how == "batch first":
            return v.transpose(0, 1).contiguous().transpose(0, 1)
        wide = torch.full((T, B, 2 * D + 3), float("nan"), dtype=v.dtype, device=v.device)
        at = 2 if how == "parts of rows" else 1
        wide[..., at:at + D] = v
        return wide[..., at:at + D]

    dy = on_gpu(rounded(rand(gen, T, B, D), t), t)
    plain = [on_gpu(v, t) for v in (x, i, r)]
    kw = dict(init=on_gpu(init), lengths=on_gpu(n, torch.int32))
    a = gated_recurrence(*plain, on_gpu(decay), save=True, **kw)
    b = gated_recurrence(*map(place, plain), on_gpu(decay), save=True, **kw)
    close("y", b.y, a.y.double().cpu(), T, 2 * half_step(t))
    ga = gated_recurrence_backward(dy, a.saved, *plain, on_gpu(decay), **kw)
    gb = gated_recurrence_backward(place(dy), b.saved, *map(place, plain), on_gpu(decay), **kw)
    for k in ("dx", "di", "dr", "ddecay", "dinit"):
        close(k, getattr(gb, k), getattr(ga, k).double().cpu(), T, 2 * half_step(t))
    still = gated_recurrence_backward(dy[:1].expand(T, B, D), a.saved, *plain, on_gpu(decay), **kw)      # one row for every step
    again = gated_recurrence_backward(dy[:1].expand(T, B, D).contiguous(), a.saved, *plain, on_gpu(decay), **kw)
    assert same(still, again)


def test_recurrence_ends_of_the_gates():
    """Gates that are wholly open or shut, a decay of -inf and one of +inf: the limits, and no NaN in any gradient."""
    from paper_2402_18994_amd import gated_recurrence, gated_recurrence_backward
    T, B = 20, 1
    ends = (float("-inf"), -200.0, -90.0, -30.0, 0.0, 30.0, 200.0, float("inf"))
    r, decay = (v.reshape(-1) for v in torch.meshgrid(torch.tensor(ends), torch.tensor((float("-inf"), -100.0, -20.0, 0.0, 50.0, float("inf"))), indexing="ij"))
    D = len(r)
    gen = torch.Generator().manual_seed(5)
    x = rounded(rand(gen, T, B, D))
    i = torch.tensor(ends).repeat(D)[:D].double().expand(T, B, D).contiguous()
    args = (on_gpu(x), on_gpu(i), on_gpu(r.double().expand(T, B, D).contiguous()), on_gpu(decay.double()))
    y, state, saved = gated_recurrence(*args, init=on_gpu(torch.ones(B, D)), save=True)
    # a gate below the least normal fp32 number, 2^-126, is shut, which counts where it meets an infinite rate alone
    rho = torch.sigmoid(r.double())
    rho[rho < 2.0 ** -126] = 0
    a = torch.exp(-8 * torch.where(rho > 0, torch.nn.functional.softplus(decay.double()) * rho, torch.zeros_like(rho)))
    h, s = torch.ones(B, D, dtype=torch.float64), torch.sqrt((1 - a) * (1 + a))
    for t in range(T):
        h = a * h + s * torch.sigmoid(i[t]) * x[t]
    # (1 - a rounds to a multiple of 2^-53 in 64 bits: gates that are shut all but a little are off by the root of that)
    assert torch.isfinite(y).all() and (state.double().cpu() - h).abs().max().item() < 2.0 ** -18
    g = gated_recurrence_backward(torch.ones_like(args[0]), saved, *args, init=on_gpu(torch.ones(B, D)))
    for v in g:
        assert torch.isfinite(v).all()
    open_ = (decay == float("-inf"))[None]
    assert torch.equal(state.cpu()[open_], torch.ones_like(state.cpu()[open_]))              # kept for good
    assert torch.equal(g.dinit.cpu()[open_], torch.full_like(g.dinit.cpu()[open_], float(T)))


def test_recurrence_infinities_stay_where_they_are():
    """An infinity or a NaN of one channel of one sequence reaches no other."""
    from paper_2402_18994_amd import gated_recurrence, gated_recurrence_backward
    T, B, D = 150, 3, 70
    gen, t, x, i, r, decay, _, _ = rec_case(T, B, D, "fp32", False, "none")
    clean = [on_gpu(v) for v in (x, i, r)]
    bad = [v.clone() for v in clean]
    bad[0][17, 1, 3], bad[1][40, 2, 5], bad[2][60, 0, 69] = float("inf"), float("nan"), float("nan")
    hit = torch.zeros(B, D, dtype=torch.bool)
    hit[1, 3] = hit[2, 5] = hit[0, 69] = True
    dy = on_gpu(rounded(rand(gen, T, B, D)))
    a, b = (gated_recurrence(*v, on_gpu(decay), save=True) for v in (clean, bad))
    ga, gb = (gated_recurrence_backward(dy, o.saved, *v, on_gpu(decay)) for o, v in ((a, clean), (b, bad)))
    for p, q in ((a.y, b.y), (ga.dx, gb.dx), (ga.di, gb.di), (ga.dr, gb.dr)):
        assert torch.equal(p[:, ~hit], q[:, ~hit])
    assert torch.equal(a.y[:17], b.y[:17]) and not torch.isfinite(b.y[17:, 1, 3]).any() and torch.isnan(b.y[60:, 0, 69]).all()
    assert torch.equal(ga.ddecay[6:69], gb.ddecay[6:69]) and torch.isnan(gb.ddecay[69])


# ------------------------------------------------------------------------------------------------ group norm

NORM = [  # T, B, D, groups, type, silu, per_step, lengths, weight, bias
    (1, 1, 1, 1, "fp32", False, False, "none", True, True),
    (1, 3, 8, 2, "bf16", True, True, "none", True, True),
    (2, 2, 6, 3, "fp32", True, False, "some", True, False),
    (7, 5, 65, 5, "bf16", True, False, "some", False, True),
    (9, 4, 130, 5, "fp32", False, True, "some", True, True),
    (33, 3, 64, 1, "bf16", False, False, "some", True, True),
    (40, 3, 96, 4, "fp32", True, False, "zero", True, True),
    (64, 2, 1040, 2, "bf16", True, True, "some", True, True),            # more threads a row than a wavefront
    (50, 2, 1001, 1, "fp32", True, True, "none", True, True),
    (30, 2, 3001, 1, "bf16", True, True, "some", True, True),            # rows of more than one block of columns
    (30, 2, 3001, 1, "fp32", False, False, "some", True, True),
    (5, 1, 16384, 1, "bf16", True, False, "none", True, True),
    (3, 1, 16383, 1, "fp32", True, False, "none", True, True),
    (600, 2, 64, 2, "fp32", True, False, "some", True, True),            # several chunks a sequence
    (2000, 1, 72, 1, "bf16", True, False, "none", True, True),
    (300, 66, 128, 2, "bf16", True, False, "some", True, True),          # one chunk of a wide workgroup
    (700, 40, 32, 8, "bf16", True, True, "some", True, True),            # a workgroup takes several chunks
    (0, 2, 8, 2, "fp32", True, False, "none", True, True),
]


def norm_case(T, B, D, groups, type, silu, per_step, lengths, weight, bias):
    gen = torch.Generator().manual_seed(T * 139 + D)
    t = TYPES[type]
    x = rounded(rand(gen, T, B, D) * torch.exp(0.5 * rand(gen, D)) + rand(gen, D), t)
    w, b = (rounded(1 + 0.2 * rand(gen, D)) if weight else None), (rounded(0.2 * rand(gen, D)) if bias else None)
    return gen, t, x, w, b, lengths_of(lengths, T, B, gen)


@pytest.mark.parametrize("case", NORM, ids=lambda c: "-".join(map(str, c)))
def test_group_norm_and_its_gradients(case):
    from paper_2402_18994_amd import group_norm, group_norm_backward
    T, B, D, groups, _, silu, per_step, _, _, _ = case
    gen, t, x, w, b, n = norm_case(*case)
    print(f"\n[case] group norm {case}", flush=True)
    gx, gw, gb, gn = on_gpu(dead(x, n), t), on_gpu(w), on_gpu(b), on_gpu(n, torch.int32)
    kw = dict(silu=silu, per_step=per_step)
    y, saved = group_norm(gx, groups, gw, gb, lengths=gn, save=True, **kw)
    many = D // groups * (1 if per_step else max(T, 1))
    h = half_step(t)
    (wy,) = oracle.norm(x, groups, w, b, lengths=n, **kw)
    close("y", y, wy, many, h)
    bare = group_norm(gx, groups, gw, gb, lengths=gn, **kw)
    assert bare.saved is None and torch.equal(bare.y, y)
    dy = rounded(rand(gen, T, B, D), t)
    args = (on_gpu(dead(dy, n), t), saved, gx, groups, gw, gb)
    g = group_norm_backward(*args, lengths=gn, **kw)
    want = gradients(lambda **k: oracle.norm(k["x"], groups, k.get("w"), k.get("b"), lengths=n, **kw), {"x": x, "w": w, "b": b}, (dy,))
    if many > 1:
        close("dx", g.dx, want["x"], many, h)
    else:                                                # (one value: its deviation is zero, and so is its gradient)
        assert (g.dx == 0).all()
    assert (g.dweight is None) == (w is None) and (g.dbias is None) == (b is None)
    if w is not None:
        close("dweight", g.dweight, want["w"], T * B, 2.0 ** -24)
    if b is not None:
        close("dbias", g.dbias, want["b"], T * B, 2.0 ** -24)
    assert same(g, group_norm_backward(*args, lengths=gn, **kw))


@pytest.mark.parametrize("B,D,groups,type", [(1, 8, 1, "fp32"), (64, 2048, 16, "bf16"), (5, 130, 5, "bf16"), (3, 66, 66, "fp32"), (2, 3001, 1, "fp32")])
def test_group_norm_steps_are_the_steps(B, D, groups, type):
    from paper_2402_18994_amd import group_norm, group_norm_step
    _, t, x, w, b, _ = norm_case(4, B, D, groups, type, True, True, "none", True, True)
    gx, gw, gb = on_gpu(x, t), on_gpu(w), on_gpu(b)
    whole = group_norm(gx, groups, gw, gb, per_step=True).y
    (want,) = oracle.norm(x, groups, w, b, per_step=True)
    for k in range(4):
        y = group_norm_step(gx[k], groups, gw, gb)
        close("step", y, want[k], D // groups, half_step(t))
        close("step of the whole", y, whole[k].double().cpu(), D // groups, 2 * half_step(t))


@pytest.mark.parametrize("per_step", (False, True))
@pytest.mark.parametrize("type", ("fp32", "bf16"))
@pytest.mark.parametrize("how", ("batch first", "parts of rows", "odd start"))
def test_group_norm_strides(type, how, per_step):
    from paper_2402_18994_amd import group_norm, group_norm_backward
    T, B, D, groups = 70, 3, 64, 4
    gen, t, x, w, b, n = norm_case(T, B, D, groups, type, True, per_step, "some", True, True)

    def place(v):
        if how == "batch first":
            return v.transpose(0, 1).contiguous().transpose(0, 1)
        wide = torch.full((T, B, 2 * D + 3), float("nan"), dtype=v.dtype, device=v.device)
        at = 2 if how == "parts of rows" else 1
        wide[..., at:at + D] = v
        return wide[..., at:at + D]

    gx, gdy, gw, gb = on_gpu(x, t), on_gpu(rounded(rand(gen, T, B, D), t), t), on_gpu(w), on_gpu(b)
    kw = dict(per_step=per_step, lengths=on_gpu(n, torch.int32))
    a = group_norm(gx, groups, gw, gb, save=True, **kw)
    c = group_norm(place(gx), groups, gw, gb, save=True, **kw)
    close("y", c.y, a.y.double().cpu(), T, 2 * half_step(t))
    ga = group_norm_backward(gdy, a.saved, gx, groups, gw, gb, **kw)
    gc = group_norm_backward(place(gdy), c.saved, place(gx), groups, gw, gb, **kw)
    for k in ("dx", "dweight", "dbias"):
        close(k, getattr(gc, k), getattr(ga, k).double().cpu(), T, 2 * half_step(t))
    one = group_norm_backward(gdy[:1].expand(T, B, D), a.saved, gx, groups, gw, gb, **kw)
    assert same(one, group_norm_backward(gdy[:1].expand(T, B, D).contiguous(), a.saved, gx, groups, gw, gb, **kw))


def test_group_norm_far_from_zero():
    """Values whose mean is 4096 times their spread: the squares are taken around the mean.  x is exact; the mean is off by a
    rounding or two of 2^-24, 2^-11 of the spread, and that is what the outputs may be off by."""
    from paper_2402_18994_amd import group_norm
    gen = torch.Generator().manual_seed(3)
    for T, per_step in ((900, False), (40, True)):
        x = rounded(4096 + rand(gen, T, 2, 64))
        (want,) = oracle.norm(x, 2, silu=False, per_step=per_step)
        y = group_norm(on_gpu(x), 2, silu=False, per_step=per_step).y.double().cpu()
        assert (y - want).abs().max().item() < 3 * 2.0 ** -11


def test_group_norm_infinities_stay_in_their_group():
    from paper_2402_18994_amd import group_norm, group_norm_backward
    T, B, D, groups = 40, 3, 24, 3
    gen, t, x, w, b, _ = norm_case(T, B, D, groups, "fp32", True, False, "none", True, True)
    dy = on_gpu(rounded(rand(gen, T, B, D)))
    for per_step in (False, True):
        clean, bad = on_gpu(x), on_gpu(x)
        bad[7, 1, 9] = float("nan")
        hit = torch.zeros(T, B, D, dtype=torch.bool)
        hit[7 if per_step else slice(None), 1, 8:16] = True
        a, c = (group_norm(v, groups, on_gpu(w), on_gpu(b), per_step=per_step, save=True) for v in (clean, bad))
        ga, gc = (group_norm_backward(dy, o.saved, v, groups, on_gpu(w), on_gpu(b), per_step=per_step) for o, v in ((a, clean), (c, bad)))
        for p, q in ((a.y, c.y), (ga.dx, gc.dx)):
            assert torch.equal(p[~hit], q[~hit]) and torch.isnan(q[hit]).all()
        assert torch.equal(ga.dweight[16:], gc.dweight[16:]) and torch.isnan(gc.dweight[8:16]).all()
