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
    (5, 2, 16383, 1, "bf16", True, True, "some", True, True),            # as many channels as there may be, each alignment
    (5, 2, 16382, 1, "fp32", True, True, "some", True, True),
    (5, 2, 16384, 1, "fp32", True, True, "some", True, True),
    (5, 2, 16384, 1, "bf16", True, True, "some", True, True),
    (5, 2, 16382, 1, "bf16", False, False, "some", True, True),
    (600, 2, 64, 2, "fp32", True, False, "some", True, True),            # several chunks a sequence
    (2000, 1, 72, 1, "bf16", True, False, "none", True, True),
    (300, 66, 128, 2, "bf16", True, False, "some", True, True),          # one chunk of a wide workgroup
    (700, 40, 32, 8, "bf16", True, True, "some", True, True),            # a workgroup takes several chunks
    (0, 2, 8, 2, "fp32", True, False, "none", True, True),
    (30, 3, 4000, 2, "bf16", True, True, "some", True, True),            # rows that a wavefront takes, each count of vectors and alignment
    (21, 3, 8192, 1, "bf16", False, True, "some", False, True),
    (21, 3, 2050, 1, "bf16", True, True, "some", True, False),
    (40, 2, 1030, 1, "bf16", True, True, "zero", True, True),
    (21, 3, 4095, 1, "bf16", True, True, "some", True, True),
    (33, 3, 516, 2, "fp32", True, True, "some", True, True),
    (21, 3, 4096, 1, "fp32", False, True, "some", True, True),
    (21, 3, 4094, 1, "fp32", True, True, "some", True, True),
    (1, 5, 2047, 1, "fp32", True, True, "none", True, True),
    (900, 9, 1040, 8, "fp32", True, True, "some", True, True),           # dw and db of several chunks of rows
    (600, 9, 1044, 4, "bf16", True, True, "some", True, True),
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


def test_group_norm_of_more_rows_than_a_launch_is_wide():
    """Rows stand alone, so the last ones of many are those of a call of their own; sums of whole numbers are exact."""
    from paper_2402_18994_amd import group_norm, group_norm_backward
    T, B, D = 70000, 64, 65                               # 4.48 million rows: more than 2^20 workgroups of four
    x = torch.randn(T, B, D, device="cuda", generator=torch.Generator("cuda").manual_seed(5)).to(torch.bfloat16)
    dy = torch.randint(-1, 2, (T, B, D), device="cuda", generator=torch.Generator("cuda").manual_seed(6), dtype=torch.int8).to(torch.bfloat16)
    bias = torch.zeros(D, device="cuda")
    kw = dict(silu=False, per_step=True)
    o = group_norm(x, 1, None, bias, save=True, **kw)
    g = group_norm_backward(dy, o.saved, x, 1, None, bias, **kw)
    for part in (slice(0, 3), slice(35000, 35003), slice(T - 3, T)):
        few = group_norm(x[part], 1, None, bias, save=True, **kw)
        assert torch.equal(o.y[part], few.y)
        assert torch.equal(g.dx[part], group_norm_backward(dy[part], few.saved, x[part], 1, None, bias, **kw).dx)
    assert torch.equal(g.dbias.double(), dy.sum((0, 1), dtype=torch.float64))


@pytest.mark.parametrize("D", (64, 1040, 4096, 8448))
@pytest.mark.parametrize("type", tuple(TYPES))
def test_group_norm_parameters_anywhere(D, type):
    """Weights and biases need no more than the alignment of a float32, however wide x is read."""
    from paper_2402_18994_amd import group_norm, group_norm_backward
    gen = torch.Generator().manual_seed(D)
    x, dy = (on_gpu(rand(gen, 70, 3, D), TYPES[type]) for _ in range(2))
    wide = on_gpu(rand(gen, 2, D + 1))
    w, b = wide[0, 1:], wide[1, :D]
    assert w.data_ptr() % 16 == 4
    for per_step in (False, True):
        a, c = (group_norm(x, 1, *p, per_step=per_step, save=True) for p in ((w, b), (w.clone(), b.clone())))
        assert same(a, c)
        assert same(*(group_norm_backward(dy, a.saved, x, 1, *p, per_step=per_step) for p in ((w, b), (w.clone(), b.clone()))))


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


# ------------------------------------------------------------------------------------------------ gated units

UNITS = [  # T, B, D, F, type, act, lengths
    (1, 1, 1, 1, "fp32", "silu", "none"),
    (1, 3, 8, 5, "bf16", "gelu", "none"),
    (2, 2, 64, 64, "bf16", "silu", "some"),
    (3, 3, 64, 33, "fp32", "silu", "some"),
    (7, 5, 65, 130, "bf16", "silu", "some"),
    (9, 4, 130, 67, "fp32", "gelu", "some"),
    (31, 1, 256, 96, "bf16", "gelu", "none"),
    (32, 2, 64, 200, "fp32", "silu", "none"),
    (65, 2, 128, 128, "bf16", "silu", "some"),
    (40, 3, 96, 40, "bf16", "silu", "zero"),
    (129, 3, 72, 260, "fp32", "silu", "some"),
    (300, 8, 192, 136, "bf16", "gelu", "some"),          # sums over many rows: parts of the contraction
    (700, 4, 40, 70, "fp32", "gelu", "some"),
    (513, 6, 704, 2056, "bf16", "silu", "some"),         # wide tiles with edges
    (0, 2, 8, 4, "fp32", "silu", "none"),
]


def units_case(T, B, D, F, type, act, lengths):
    gen = torch.Generator().manual_seed(T * 149 + D)
    t = TYPES[type]
    x = rounded(rand(gen, T, B, D), t)
    gate, up = (rounded(rand(gen, F, D) / math.sqrt(D), t) for _ in range(2))
    return gen, t, x, gate, up, lengths_of(lengths, T, B, gen)


@pytest.mark.parametrize("case", UNITS, ids=lambda c: "-".join(map(str, c)))
def test_units_and_their_gradients(case):
    """In the reverse pass dG and dU enter the products rounded to the streamed type: half a step more, of every term.  (fp32 values
    enter as three pieces of bfloat16; the products left out are below 2^-24 of a term, one of TERM.)"""
    from paper_2402_18994_amd import gated_units, gated_units_backward
    T, B, D, F, _, act, _ = case
    gen, t, x, gate, up, n = units_case(*case)
    print(f"\n[case] units {case}", flush=True)
    gx, gg, gu, gn = on_gpu(dead(x, n), t), on_gpu(gate, t), on_gpu(up, t), on_gpu(n, torch.int32)
    y, saved = gated_units(gx, gg, gu, act=act, lengths=gn, save=True)
    h = half_step(t)
    (wy,) = oracle.units(x, gate, up, act, n)
    close("y", y, wy, D, h)
    bare = gated_units(gx, gg, gu, act=act, lengths=gn)
    assert bare.saved is None and torch.equal(bare.y, y)
    dy = rounded(rand(gen, T, B, F), t)
    args = (on_gpu(dead(dy, n), t), saved, gx, gg, gu)
    g = gated_units_backward(*args, act=act, lengths=gn)
    want = gradients(lambda **k: oracle.units(k["x"], k["gate"], k["up"], act, n), {"x": x, "gate": gate, "up": up}, (dy,))
    for name, got, terms in (("x", g.dx, 2 * F), ("gate", g.dgate, T * B), ("up", g.dup, T * B)):
        # a sum of `terms` products, each off by up to h: at random, sqrt(terms) h of a term's size, which is what the sum's
        # own size is; a single value may be four times that off
        assert got.shape == want[name].shape
        off = (got.double().cpu() - want[name]).abs()
        if off.numel():
            wide = want[name].abs().max().item() * 4 * h
            assert torch.isfinite(got).all() and off.max().item() <= wide + 8 * 32 * math.sqrt(terms + 16) * 2.0 ** -24 * want[name].abs().max().item()
            assert torch.linalg.norm(got.double().cpu() - want[name]).item() <= (2 * h + 32 * math.sqrt(terms + 16) * 2.0 ** -24) * torch.linalg.norm(want[name]).item() + 1e-30, name
    if n is not None:
        for b in range(B):
            assert (g.dx[int(n[b]):, b] == 0).all() and (y[int(n[b]):, b] == 0).all()
    assert same(g, gated_units_backward(*args, act=act, lengths=gn))


@pytest.mark.parametrize("B,D,F,type", [(1, 64, 48, "bf16"), (64, 256, 96, "bf16"), (17, 192, 130, "bf16"), (3, 130, 70, "fp32"), (33, 64, 64, "fp32"),
                                        (5, 65, 40, "bf16"), (200, 128, 72, "bf16"), (1, 1, 1, "fp32"),
                                        (128, 192, 33, "bf16"), (129, 192, 33, "bf16"), (250, 132, 20, "fp32"), (100, 131, 50, "bf16"), (257, 64, 16, "fp32")])
def test_units_steps_are_the_units(B, D, F, type):
    from paper_2402_18994_amd import gated_units, gated_units_step
    for act in ("silu", "gelu"):
        _, t, x, gate, up, _ = units_case(3, B, D, F, type, act, "none")
        gx, gg, gu = on_gpu(x, t), on_gpu(gate, t), on_gpu(up, t)
        whole = gated_units(gx, gg, gu, act=act).y
        (want,) = oracle.units(x, gate, up, act)
        for k in range(3):
            y = gated_units_step(gx[k], gg, gu, act=act)
            close("step", y, want[k], D, half_step(t))
            close("step of the whole", y, whole[k].double().cpu(), D, 2 * half_step(t))


@pytest.mark.parametrize("type", ("fp32", "bf16"))
@pytest.mark.parametrize("how", ("batch first", "parts of rows", "odd start", "wide apart"))
@pytest.mark.parametrize("rows", (17, 110))
def test_units_strides(type, how, rows):
    from paper_2402_18994_amd import gated_units, gated_units_backward
    T, B, D, F = rows, 3, 64, 72
    gen, t, x, gate, up, n = units_case(T, B, D, F, type, "silu", "some")

    def place(v):
        if how == "batch first":
            return v.transpose(0, 1).contiguous().transpose(0, 1)
        E = v.shape[-1]
        wide = torch.full((T, B, 2 * E + (0 if how == "wide apart" else 3)), float("nan"), dtype=v.dtype, device=v.device)
        at = {"parts of rows": 2, "odd start": 1, "wide apart": 8}[how]
        wide[..., at:at + E] = v
        return wide[..., at:at + E]

    gx, gdy, gg, gu = on_gpu(x, t), on_gpu(rounded(rand(gen, T, B, F), t), t), on_gpu(gate, t), on_gpu(up, t)
    kw = dict(lengths=on_gpu(n, torch.int32))
    a = gated_units(gx, gg, gu, save=True, **kw)
    c = gated_units(place(gx), gg, gu, save=True, **kw)
    # (sums of few rows run in another order where rows do not lie in 16-byte pieces)
    close("y", c.y, a.y.double().cpu(), D, 2 * half_step(t))
    ga, gc = gated_units_backward(gdy, a.saved, gx, gg, gu, **kw), gated_units_backward(place(gdy), c.saved, place(gx), gg, gu, **kw)
    for k in ("dx", "dgate", "dup"):
        close(k, getattr(gc, k), getattr(ga, k).double().cpu(), T * B + 2 * F, 2 * half_step(t))
    again = gated_units_backward(place(gdy), a.saved, place(gx), gg, gu, **kw)
    assert same(ga, again)
    one = gated_units_backward(gdy[:1].expand(T, B, F), a.saved, gx, gg, gu, **kw)
    assert same(one, gated_units_backward(gdy[:1].expand(T, B, F).contiguous(), a.saved, gx, gg, gu, **kw))
    # matrices that start at an odd element
    odd = torch.zeros(2 * F * D + 1, dtype=t, device="cuda")
    og, ou = odd[1:1 + F * D].view(F, D), odd[1 + F * D:].view(F, D)
    og.copy_(gg)
    ou.copy_(gu)
    close("odd matrices", gated_units(gx, og, ou, **kw).y, a.y.double().cpu(), D, 2 * half_step(t))


@pytest.mark.parametrize("T", (40, 300))
def test_units_of_large_and_small_values(T):
    """fp32 over its range, for few rows (fp32 products) and for more (pieces): the largest values round up to infinity in bfloat16,
    the lower pieces of the smallest ones still count."""
    from paper_2402_18994_amd import gated_units
    gen = torch.Generator().manual_seed(11)
    x = rounded(rand(gen, T, 1, 64))
    x[0, 0, 0] = 3.4028234663852886e38
    x[1] *= 2.0 ** 100
    x[2] *= 2.0 ** -90
    gate, up = rounded(rand(gen, 32, 64)), rounded(rand(gen, 32, 64))
    gate[:, 0] = up[:, 0] = 2.0 ** -126
    y = gated_units(on_gpu(x), on_gpu(gate), on_gpu(2.0 ** -20 * up), act="silu")
    # a piece is a bfloat16 number, a multiple of 2^-133: what an operand has below that (here 2^-20 up[:, 0] = 2^-146) does not enter
    enters = lambda v: torch.round(v * 2.0 ** 133) * 2.0 ** -133 if T > 256 else v
    (want,) = oracle.units(x, gate, enters(2.0 ** -20 * up))
    for k in (0, 3):
        close("row", y.y[k], want[k], 64, 2.0 ** -24)
    assert torch.isfinite(y.y[0]).all()
    large = gated_units(on_gpu(x), on_gpu(gate), on_gpu(up * 2.0 ** 100)).y[2]
    close("small", large, oracle.units(x, gate, up * 2.0 ** 100)[0][2], 64, 2.0 ** -24)


def test_units_infinities_stay_in_their_row():
    from paper_2402_18994_amd import gated_units
    for type in ("fp32", "bf16"):
        _, t, x, gate, up, _ = units_case(50, 2, 64, 40, type, "silu", "none")
        bad = on_gpu(x, t)
        bad[7, 1, 3], bad[9, 0, 5] = float("inf"), float("nan")
        a, c = gated_units(on_gpu(x, t), on_gpu(gate, t), on_gpu(up, t)).y, gated_units(bad, on_gpu(gate, t), on_gpu(up, t)).y
        keep = torch.ones(50, 2, dtype=torch.bool)
        keep[7, 1] = keep[9, 0] = False
        assert torch.equal(a[keep], c[keep]) and not torch.isfinite(c[7, 1]).any() and torch.isnan(c[9, 0]).all()


# ------------------------------------------------------------------------------------------------ together

def block_parameters(gen, D, F):
    p = {"weight": 1 + 0.1 * rand(gen, D), "bias": 0.1 * rand(gen, D), "W_i": rand(gen, D, D) / math.sqrt(D), "W_r": rand(gen, D, D) / math.sqrt(D),
         "decay": rand(gen, D) - 3, "gate": rand(gen, F, D) / math.sqrt(D), "up": rand(gen, F, D) / math.sqrt(D)}
    return {k: rounded(v) for k, v in p.items()}


def block_forward(p, x, groups, lengths):
    """norm -> gates -> recurrence -> units; -> y and what the reverse pass needs."""
    import paper_2402_18994_amd as snn
    n = snn.group_norm(x, groups, p["weight"], p["bias"], per_step=True, lengths=lengths, save=True)
    i, r = n.y @ p["W_i"], n.y @ p["W_r"]
    h = snn.gated_recurrence(n.y, i, r, p["decay"], lengths=lengths, save=True)
    u = snn.gated_units(h.y, p["gate"], p["up"], lengths=lengths, save=True)
    return u.y, (n, i, r, h, u)


def block_backward(p, x, groups, lengths, kept, dy):
    import paper_2402_18994_amd as snn
    n, i, r, h, u = kept
    gu = snn.gated_units_backward(dy, u.saved, h.y, p["gate"], p["up"], lengths=lengths)
    gh = snn.gated_recurrence_backward(gu.dx, h.saved, n.y, i, r, p["decay"], lengths=lengths)
    dn = gh.dx + gh.di @ p["W_i"].t() + gh.dr @ p["W_r"].t()
    gn = snn.group_norm_backward(dn, n.saved, x, groups, p["weight"], p["bias"], per_step=True, lengths=lengths)
    rows = n.y.flatten(0, 1).t()
    return {"x": gn.dx, "weight": gn.dweight, "bias": gn.dbias, "W_i": rows @ gh.di.flatten(0, 1), "W_r": rows @ gh.dr.flatten(0, 1),
            "decay": gh.ddecay, "gate": gu.dgate, "up": gu.dup}


@pytest.mark.parametrize("lengths", ("none", "some"))
def test_a_block_of_all_three(lengths):
    """Values and gradients through the whole block, and the same block served step by step."""
    import paper_2402_18994_amd as snn
    T, B, D, F, groups = 90, 5, 64, 96, 4
    gen = torch.Generator().manual_seed(21)
    p, x, dy, n = block_parameters(gen, D, F), rounded(rand(gen, T, B, D)), rounded(rand(gen, T, B, F)), lengths_of(lengths, T, B, gen)
    gp, gx, gn = {k: on_gpu(v) for k, v in p.items()}, on_gpu(x), on_gpu(n, torch.int32)
    y, kept = block_forward(gp, gx, groups, gn)
    got = block_backward(gp, gx, groups, gn, kept, on_gpu(dy))

    def whole(x, weight, bias, W_i, W_r, decay, gate, up):
        (v,) = oracle.norm(x, groups, weight, bias, per_step=True, lengths=n)
        h, _ = oracle.recurrence(v, v @ W_i, v @ W_r, decay, lengths=n)
        return oracle.units(h, gate, up, "silu", n)

    close("y", y, whole(x, **p)[0], T + D, 2.0 ** -24)
    want = gradients(whole, {"x": x, **p}, (dy,))
    for k, v in got.items():
        close(k, v, want[k], T * B, 2.0 ** -24)
    if n is None:
        state = torch.zeros(B, D, device="cuda")
        for t in range(T):
            v = snn.group_norm_step(gx[t], groups, gp["weight"], gp["bias"])
            h = snn.gated_recurrence_step(v, v @ gp["W_i"], v @ gp["W_r"], state, gp["decay"])
            close(f"step {t}", snn.gated_units_step(h, gp["gate"], gp["up"]), y[t].double().cpu(), T + D, 2.0 ** -24)


@pytest.mark.parametrize("per_step", (True, False))
def test_a_captured_training_step_repeats(per_step):
    """Forward and reverse pass of all three in one graph, replayed on new inputs with eager work between: the eager results."""
    import paper_2402_18994_amd as snn
    T, B, D, F, groups = 260, 3, 128, 192, 4
    gen = torch.Generator().manual_seed(22)
    t = torch.bfloat16
    fresh = lambda *s: on_gpu(rand(gen, *s), t)
    w, b, decay = on_gpu(1 + 0.1 * rand(gen, D)), on_gpu(0.1 * rand(gen, D)), on_gpu(rand(gen, D) - 3)
    gate, up = fresh(F, D) / 11, fresh(F, D) / 11
    x, i, r, dy, dh = fresh(T, B, D), fresh(T, B, D), fresh(T, B, D), fresh(T, B, F), fresh(T, B, D)
    n = torch.tensor([T, 5, 100], dtype=torch.int32, device="cuda")

    def step():
        a = snn.group_norm(x, groups, w, b, per_step=per_step, lengths=n, save=True)
        h = snn.gated_recurrence(a.y, i, r, decay, lengths=n, save=True)
        u = snn.gated_units(h.y, gate, up, lengths=n, save=True)
        gu = snn.gated_units_backward(dy, u.saved, h.y, gate, up, lengths=n)
        gh = snn.gated_recurrence_backward(gu.dx, h.saved, a.y, i, r, decay, lengths=n)
        ga = snn.group_norm_backward(gh.dx, a.saved, x, groups, w, b, per_step=per_step, lengths=n)
        return [u.y, h.state, *gu, *gh[:4], *ga]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager = step()                                       # (on another stream than the current one)
    torch.cuda.current_stream().wait_stream(side)
    assert same(eager, step())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        for v in (x, i, r, dy):
            v.copy_(fresh(*v.shape))
        n[1] = 5 + 60 * k
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        assert same(out, want), k


def test_shapes_and_types_that_do_not_fit_are_refused():
    import paper_2402_18994_amd as snn
    x, d = torch.zeros(4, 2, 8, device="cuda"), torch.zeros(8, device="cuda")
    w = torch.zeros(6, 8, device="cuda")
    bad = [lambda: snn.gated_recurrence(x, x[:3], x, d), lambda: snn.gated_recurrence(x, x, x.bfloat16(), d), lambda: snn.gated_recurrence(x, x, x, d[:7]),
           lambda: snn.gated_recurrence(x, x, x, None), lambda: snn.gated_recurrence(x, x, x, d, sharpness=0.0), lambda: snn.gated_recurrence(x, x, x, d, sharpness=1e39),
           lambda: snn.gated_recurrence(x, x, x, d, sharpness=float("nan")), lambda: snn.group_norm(x, 2.0), lambda: snn.group_norm(x, 2, eps=1e40), lambda: snn.gated_units(x, None, w),
           lambda: snn.gated_recurrence(x[0], x[0], x[0], d),
           lambda: snn.gated_recurrence(x, x, x, d, init=torch.zeros(2, 7, device="cuda")), lambda: snn.gated_recurrence(x, x, x, d.cpu()),
           lambda: snn.gated_recurrence_backward(x, None, x, x, x, d), lambda: snn.gated_recurrence_step(x[0], x[0], x[0], None, d),
           lambda: snn.gated_recurrence_step(x[0], x[0], x[0], torch.zeros(2, 8, device="cuda").bfloat16(), d),
           lambda: snn.gated_recurrence_backward(x, torch.zeros(3, device="cuda"), x, x, x, d),
           lambda: snn.group_norm(x, 3), lambda: snn.group_norm(x, 0), lambda: snn.group_norm(x, 2, d[:4]), lambda: snn.group_norm(x, 2, eps=-1.0),
           lambda: snn.group_norm(x.transpose(1, 2), 2), lambda: snn.group_norm(x, 2, lengths=torch.zeros(2, device="cuda")),
           lambda: snn.group_norm_backward(x, None, x, 2), lambda: snn.group_norm_step(x, 2),
           lambda: snn.gated_units(x, w, w[:5]), lambda: snn.gated_units(x, w, w.bfloat16()), lambda: snn.gated_units(x, w[:, :7], w), lambda: snn.gated_units(x, w, None),
           lambda: snn.gated_units(x, w, w, act="relu"), lambda: snn.gated_units(x, w.t().contiguous().t(), w), lambda: snn.gated_units_step(x, w, w),
           lambda: snn.gated_units_backward(x, torch.zeros(3, device="cuda"), x, w, w), lambda: snn.gated_units_backward(x, None, x, w, w)]
    for k, f in enumerate(bad):
        with pytest.raises(snn.SnnError):
            f()
            print("call", k, "was taken")


# ------------------------------------------------------------------------------------------------ differences

def check_differences(f, inputs, grads, dys, seed):
    """<gradient, v> against (L(x + e v) - L(x - e v)) / 2e with L = sum of <dy, output>, in fp32 on the GPU, sums in 64 bits; v standard normal.

    e = 2^-9.  Rounding: outputs are off by a few 2^-24 of themselves, at random, which e divides: 2^-22 2^8 |dy y| = 2^-14 |dy y|.  Truncation: e^2 / 6 of
    the third derivative along v, which is some ten times the first for functions of a few steps of order one: 2^-16 |gradient|.  Both
    are below 2^-11 of their norms with room for the factors that were not counted."""
    gen = torch.Generator().manual_seed(seed)
    e = 2.0 ** -9
    for name, g in grads.items():
        v = torch.randn(inputs[name].shape, generator=gen).cuda()
        total, size = [], 0.0
        for sign in (1, -1):
            # (both ends as fp32 holds them: the difference is theirs)
            outs = f(**(inputs | {name: inputs[name] + sign * e * v}))
            total.append(sum((dy.double() * o.double()).sum() for dy, o in zip(dys, outs)).item())
            size = sum(((dy.double() * o.double()) ** 2).sum() for dy, o in zip(dys, outs)).sqrt().item()
        step = ((inputs[name] + e * v).double() - (inputs[name] - e * v).double()) / (2 * e)
        want = (g.double() * step).sum().item()
        got = (total[0] - total[1]) / (2 * e)
        assert abs(got - want) <= 2.0 ** -11 * (torch.linalg.norm(g.double()).item() + size) * 2, (name, got, want)


@pytest.mark.parametrize("T", (5, 40))
def test_gradients_are_the_differences(T):
    import paper_2402_18994_amd as snn
    B, D, F, groups = 2, 24, 20, 3
    gen = torch.Generator().manual_seed(T)
    r = lambda *s: torch.randn(*s, generator=gen).cuda()
    n = torch.tensor([T, T - 2], dtype=torch.int32, device="cuda")
    i = {"x": r(T, B, D), "i": r(T, B, D), "r": r(T, B, D), "decay": r(D) - 2, "init": r(B, D)}
    dys = (r(T, B, D), r(B, D))
    o = snn.gated_recurrence(**i, lengths=n, save=True)
    g = snn.gated_recurrence_backward(dys[0], o.saved, **i, lengths=n, d_state=dys[1])
    check_differences(lambda **k: snn.gated_recurrence(**k, lengths=n)[:2], i, dict(zip(("x", "i", "r", "decay", "init"), g)), dys, 1)
    for per_step in (False, True):
        i = {"x": r(T, B, D), "weight": 1 + 0.1 * r(D), "bias": 0.1 * r(D)}
        kw = dict(groups=groups, per_step=per_step, lengths=n)
        o = snn.group_norm(**i, save=True, **kw)
        g = snn.group_norm_backward(dys[0], o.saved, **i, **kw)
        check_differences(lambda **k: snn.group_norm(**k, **kw)[:1], i, dict(zip(("x", "weight", "bias"), g)), dys[:1], 2)
    for act in ("silu", "gelu"):
        i = {"x": r(T, B, D), "gate": r(F, D) / 5, "up": r(F, D) / 5}
        dy = r(T, B, F)
        o = snn.gated_units(**i, act=act, lengths=n, save=True)
        g = snn.gated_units_backward(dy, o.saved, **i, act=act, lengths=n)
        check_differences(lambda **k: snn.gated_units(**k, act=act, lengths=n)[:1], i, dict(zip(("x", "gate", "up"), g)), (dy,), 3)


# ------------------------------------------------------------------------------------------------ far apart

def test_sequences_that_lie_more_than_2_31_elements_apart():
    """Offsets are 64 bits wide: the sequences of a batch lie 2^31 + 64 elements apart."""
    import paper_2402_18994_amd as snn
    T, B, D, F = 70, 2, 64, 40
    far = (1 << 31) + 64
    store = torch.empty(far + T * D * 8, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator().manual_seed(9)
    fresh = lambda *s: torch.randn(*s, generator=gen).bfloat16().cuda()
    at = [0]

    def apart(v):
        w = store.as_strided(v.shape, (v.shape[-1], far, 1), at[0])
        at[0] += T * v.shape[-1]
        w.copy_(v)
        return w

    x, i, r, dy = (fresh(T, B, D) for _ in range(4))
    dyf = fresh(T, B, F)
    fx, fi, fr, fdy, fdyf = map(apart, (x, i, r, dy, dyf))
    decay, gate, up = torch.randn(D, generator=gen).cuda() - 3, fresh(F, D) / 8, fresh(F, D) / 8
    a, b = snn.gated_recurrence(x, i, r, decay, save=True), snn.gated_recurrence(fx, fi, fr, decay, save=True)
    assert same(a, b)
    assert same(snn.gated_recurrence_backward(dy, a.saved, x, i, r, decay), snn.gated_recurrence_backward(fdy, a.saved, fx, fi, fr, decay))
    for per_step in (False, True):
        a, b = (snn.group_norm(v, 4, per_step=per_step, save=True) for v in (x, fx))
        assert same(a, b)
        assert same(snn.group_norm_backward(dy, a.saved, x, 4, per_step=per_step), snn.group_norm_backward(fdy, a.saved, fx, 4, per_step=per_step))
    a, b = (snn.gated_units(v, gate, up, save=True) for v in (x, fx))
    close("y", b.y, a.y.double().cpu(), D, 2 * half_step(torch.bfloat16))
    assert same(snn.gated_units_backward(dyf, a.saved, x, gate, up), snn.gated_units_backward(fdyf, a.saved, fx, gate, up))
    for v in (x, fx):
        steps = snn.group_norm_step(v[3], 4), snn.gated_units_step(v[3], gate, up), snn.gated_recurrence_step(v[3], v[4], v[5], torch.zeros(B, D, device="cuda"), decay)
        if v is x:
            want = steps
    close("step of units", steps[1], want[1].double().cpu(), D, 2 * half_step(torch.bfloat16))
    assert torch.equal(steps[0], want[0]) and torch.equal(steps[2], want[2])
