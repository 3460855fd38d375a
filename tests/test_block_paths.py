"""Every kernel that calls of the gated block's operators choose between, each by a case that takes it.

What a call takes is decided by the rules of csrc/block_rules.hpp, which the host compiler builds into a program here: `test_every_path_has_a_case` asks it
about all cases, those of test_block_ops.py among them, and names the paths that none takes.  The cases themselves are checked as there."""
import itertools
import subprocess

import pytest
import torch

from tests import test_block_ops as block
from tests.helpers import host_program
from tests.test_seq_ops import TYPES, on_gpu, rand

VECTORS = {"fp32": (4, 2, 1), "bf16": (8, 2, 1)}     # channels that are read at a time


def norm_cases():
    """T, B, D, groups, type, silu, per_step, lengths, weight, bias; C channels a group, so that vectors of `vec` fit and no wider ones."""
    for type in TYPES:
        for vec in VECTORS[type]:
            case = lambda T, B, C, groups, silu, per_step: (T, B, C * groups, groups, type, silu, per_step, "some", True, True)
            C = {8: 64, 4: 64, 2: 66, 1: 65}[vec]
            rows = {8: 256, 4: 128, 2: 64, 1: 32}[vec]               # that 256 threads hold
            yield case(rows // 3, 3, C, 2, True, False)              # a sequence's group at once
            yield case(rows + rows // 3, 33, C, 2, False, False)     # in a wider workgroup
            yield case(4 * rows + 5, 3, C, 2, True, False)           # in chunks
            yield case(2 * rows + 7, 9, C, 20, True, False)          # in chunks of more rows a thread than are in flight
            for silu in (True, False):
                yield case(11, 3, min(C, 64 * vec - 1), 2, silu, True)      # each step, a workgroup with several
            yield case(220, 5, {8: 8, 4: 4, 2: 6, 1: 3}[vec], {8: 1024, 4: 1024, 2: 500, 1: 500}[vec], True, True)   # which takes several lots of them
            for vectors in (3, 9, 20, 65):                           # and rows of so many vectors a lane
                yield case(7, 3, min((vectors * 64 - 5) * vec, 16384 - 8 + vec), 1, vectors % 2 == 0, True)
    yield (1030, 8, 2048, 32, "bf16", True, False, "some", True, True)
    yield (257, 51, 130, 5, "fp32", False, False, "some", True, True)


REC = [  # T, B, D, type, init, lengths
    (300, 90, 191, "bf16", True, "some"),            # one channel a lane, workgroups for the whole chip
    (300, 45, 192, "bf16", True, "some"),            # for the forward pass, not for the reverse one
    (300, 45, 190, "fp32", True, "some"),
    (50, 90, 130, "bf16", True, "some"),             # too few steps for wide workgroups
    (50, 90, 129, "bf16", False, "some"),
    (50, 90, 131, "fp32", True, "some"),
    (1100, 2, 73, "bf16", True, "some"),
]

UNITS = [  # T, B, D, F, type, act, lengths
    (101, 3, 2048, 70, "bf16", "silu", "some"),      # the forward contraction in parts: operands as they lie,
    (101, 3, 2050, 70, "bf16", "gelu", "some"),      # laid out first,
    (90, 3, 400, 70, "fp32", "silu", "some"),        # in pieces,
    (90, 3, 401, 330, "fp32", "gelu", "some"),       # in pieces of which none is whole
    (400, 4, 72, 3600, "fp32", "silu", "some"),      # wide tiles, forward
    (400, 4, 72, 3599, "bf16", "gelu", "some"),
    (700, 3, 72, 1100, "fp32", "gelu", "some"),      # small tiles, more than compute units
    (700, 3, 72, 1101, "bf16", "silu", "some"),
    (500, 3, 2050, 2056, "bf16", "silu", "some"),    # wide tiles, reverse, parts of one product,
    (500, 3, 2050, 2056, "fp32", "silu", "some"),
    (700, 3, 2800, 1050, "bf16", "gelu", "some"),    # none
    (700, 3, 2800, 1050, "fp32", "gelu", "some"),
    (600, 3, 1100, 1030, "fp32", "silu", "some"),    # small tiles, more than compute units, reverse
    (1200, 3, 500, 500, "bf16", "silu", "some"),
    (5, 3, 33, 17, "fp32", "silu", "some"), (5, 3, 33, 17, "bf16", "silu", "some"), (5, 5, 33, 17, "fp32", "silu", "some"), (5, 5, 33, 17, "bf16", "silu", "some"),
    (5, 3, 40, 17, "fp32", "silu", "some"), (5, 3, 40, 17, "bf16", "silu", "some"), (5, 5, 40, 17, "fp32", "silu", "some"), (5, 5, 40, 17, "bf16", "silu", "some"),
    (50, 2, 40, 17, "fp32", "silu", "some"), (50, 2, 33, 17, "fp32", "silu", "some"),
]

PROGRAM = r'''
#include "block_rules.hpp"
#include <cstdio>
using namespace snn;
static void *const at = (void *)4096;
int main() {                     // per line: operator T B D (groups or F) type per_step
  char what;
  int T, B, D, n, type, per_step;
  while (scanf(" %c %d %d %d %d %d %d", &what, &T, &B, &D, &n, &type, &per_step) == 7) {
    const snn_rows x{at, (int64_t)B * D, D};
    if (what == 'n') {
      snn_norm_args a{};
      a.T = T; a.B = B; a.D = D; a.groups = n; a.type = type; a.per_step = per_step; a.x = a.y = x;
      const snn_norm_grads g{x, x, nullptr, nullptr};
      for (int back = 0; back < 2; ++back) {
        const int vec = norm_vector(a, back ? &g : nullptr);
        const NormCut c = norm_cut(a, vec, back);
        printf("%d %d %d %d %d %d ", vec, c.nt, (int)c.chunks, c.long_row, c.loops, c.R);
      }
    } else if (what == 'r') {
      snn_recurrence_args a{};
      a.T = T; a.B = B; a.D = D; a.type = type; a.x = a.i = a.r = a.y = x;
      snn_recurrence_grads g{};
      g.dy = g.dx = g.di = g.dr = x;
      for (int back = 0; back < 2; ++back) {
        const int vec = two_channels(a, back ? &g : nullptr) ? 2 : 1;
        const RecCut c = recurrence_cut(a, vec, back);
        printf("%d %d %d ", vec, c.waves, c.nseg);
      }
    } else {
      snn_units_args a{};
      a.T = T; a.B = B; a.D = D; a.F = n; a.type = type; a.x = x; a.gate = a.up = at;
      const Product f = units_product(a);
      const UnitsPlan p = units_plan(a);
      const auto workgroups = [](const Product &p) { return (int64_t)p.mt * p.nt * p.splits; };
      int64_t row;
      printf("%d %d %d %d %d %d %d ", few_rows(a), few_in_pieces(a), few_blocks(T * B), x_direct(a, row), f.tile.wide, f.splits, gemm_stages(workgroups(f), f.tile.wide));
      printf("%d %d %d %d ", p.dx.tile.wide, p.dx.splits, p.dw.splits, gemm_stages(workgroups(p.dx) + workgroups(p.dw), p.dx.tile.wide));
    }
    printf("\n");
  }
}
'''


def answers(lines):
    out = subprocess.run([host_program(PROGRAM)], input="\n".join(" ".join(map(str, l)) for l in lines), check=True, capture_output=True, text=True).stdout
    return [list(map(int, l.split())) for l in out.splitlines()]


def norm_paths(case, a):
    _, _, _, _, type, silu, per_step, *_ = case
    for back, (vec, threads, chunks, row, lots, rows) in ((False, a[:6]), (True, a[6:])):
        if not per_step:
            yield back, type, vec, ("chunks" if rows <= 4 else "long chunks") if chunks else f"at once, {threads}"
        elif row:
            yield back, type, vec, "rows, again" if row < 0 else f"rows of {row}"
        else:
            yield back, type, vec, "steps" + (f", silu {silu}" if back else "")
            if lots > 1:
                yield back, type, vec, "lots of steps"


def wanted_norm_paths():
    for type in TYPES:
        for vec in VECTORS[type]:
            whole = {"at once, 256", "at once, 512"}
            forward = whole | {"chunks", "long chunks", "steps", "lots of steps", "rows of 4", "rows of 16", "rows, again"} | ({f"rows of {64 // vec}"} if vec <= 2 else set())
            back = (whole if vec <= 2 else set()) | {"chunks", "long chunks", "steps, silu True", "steps, silu False", "lots of steps", "rows of 4", "rows, again"}
            yield from ((False, type, vec, p) for p in forward)
            yield from ((True, type, vec, p) for p in back)


def rec_paths(case, a):
    for back, (vec, waves, segments) in ((False, a[:3]), (True, a[3:])):
        yield back, case[3], vec, waves, segments > 1


def wanted_rec_paths():
    for type, vec in (("fp32", 1), ("bf16", 2), ("bf16", 1)):
        for back in (False, True):
            yield from ((back, type, vec, waves, cut) for waves, cut in ((8 if back else 16, False), (4, False), (4, True)))


def units_paths(case, a):
    few, pieces, blocks, direct, wide, parts, stages, wide_back, parts_dx, parts_dw, stages_back = a
    type = case[4]
    if few:
        yield type, "few rows", pieces, blocks
    else:
        yield type, "forward", wide, stages, parts > 1
        yield type, "forward", "as it lies" if direct else "laid out", parts > 1
    yield type, "reverse", wide_back, stages_back
    yield type, "parts of dx" if parts_dx > 1 else "dx at once", wide_back
    yield type, "parts of dw" if parts_dw > 1 else "dw at once", wide_back


def wanted_units_paths():
    for type in TYPES:
        yield from ((type, "few rows", pieces, blocks) for pieces, blocks in itertools.product((0, 1), (1, 2, 4)))
        yield from ((type, "forward", *p) for p in ((1, 2, False), (0, 4, False), (0, 2, False), (0, 4, True)))
        yield from ((type, "forward", how, parts) for how in (("laid out", "as it lies") if type == "bf16" else ("laid out",)) for parts in (False, True))
        yield from ((type, "reverse", *p) for p in ((1, 2), (0, 4), (0, 2)))
        yield from ((type, what, wide) for what in ("parts of dx", "dx at once", "dw at once") for wide in (0, 1))
        yield type, "parts of dw", 0


@pytest.mark.parametrize("op", ("n", "r", "u"))
def test_every_path_has_a_case(op):
    kind = lambda t: list(TYPES).index(t)
    if op == "n":
        cases, paths, wanted = block.NORM + list(norm_cases()), norm_paths, wanted_norm_paths
        lines = [("n", *c[:4], kind(c[4]), int(c[6])) for c in cases]
    elif op == "r":
        cases, paths, wanted = block.REC + REC, rec_paths, wanted_rec_paths
        lines = [("r", *c[:3], 1, kind(c[3]), 0) for c in cases]
    else:
        cases, paths, wanted = block.UNITS + UNITS, units_paths, wanted_units_paths
        lines = [("u", *c[:4], kind(c[4]), 0) for c in cases]
    taken = {p for c, a in zip(cases, answers(lines)) for p in paths(c, a)}
    assert not set(wanted()) - taken, sorted(map(str, set(wanted()) - taken))


@pytest.mark.gpu
@pytest.mark.parametrize("case", norm_cases(), ids=lambda c: "-".join(map(str, c)))
def test_group_norm_of_every_path(case):
    block.test_group_norm_and_its_gradients(case)


@pytest.mark.gpu
@pytest.mark.parametrize("case", REC, ids=lambda c: "-".join(map(str, c)))
def test_recurrence_of_every_path(case):
    block.test_recurrence_and_its_gradients(case)


@pytest.mark.gpu
@pytest.mark.parametrize("case", UNITS, ids=lambda c: "-".join(map(str, c)))
def test_units_of_every_path(case):
    block.test_units_and_their_gradients(case)


@pytest.mark.gpu
@pytest.mark.parametrize("per_step", (False, True))
@pytest.mark.parametrize("T,B", ((40, 3), (900, 3), (130, 40)))
@pytest.mark.parametrize("bad", (float("nan"), float("inf")))
def test_group_norm_keeps_what_is_no_number_in_its_group(T, B, per_step, bad):
    """In one workgroup, in chunks, in a wide workgroup: outputs and gradients of other groups are those of clean values, bit for bit, the group's own are NaN."""
    from paper_2402_18994_amd import group_norm, group_norm_backward
    groups, D = 3, 72
    gen = torch.Generator().manual_seed(T)
    x, dy, w, b = (on_gpu(rand(gen, *s)) for s in ((T, B, D), (T, B, D), (D,), (D,)))
    spoilt, hit = x.clone(), torch.zeros(T, B, D, dtype=torch.bool)
    spoilt[T - 7, 1, 30] = bad
    hit[T - 7 if per_step else slice(None), 1, 24:48] = True
    kw = dict(per_step=per_step)
    a, c = (group_norm(v, groups, w, b, save=True, **kw) for v in (x, spoilt))
    ga, gc = (group_norm_backward(dy, o.saved, v, groups, w, b, **kw) for o, v in ((a, x), (c, spoilt)))
    for p, q in ((a.y, c.y), (ga.dx, gc.dx)):
        assert torch.equal(p[~hit], q[~hit]) and torch.isnan(q[hit]).all()
    other = [*range(24), *range(48, 72)]
    for p, q in ((ga.dweight, gc.dweight), (ga.dbias, gc.dbias)):
        assert torch.equal(p[other], q[other]) and torch.isnan(q[24:48]).all()
