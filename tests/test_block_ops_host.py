"""Host-side checks of the gated block's operators that need no GPU: the header's layout, and what the entry points refuse before
they touch a device."""
import ctypes as C
import os

import pytest

from paper_2402_18994_amd import binding, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, ARG, SHAPE, WORKSPACE = 1, 2, 3, 4
P = 1 << 20                     # an address that nothing reads: every call here is refused before
OPS = ("recurrence", "norm", "units")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.library_path()):
        from paper_2402_18994_amd import build
        build.build()
    return ops._lib()


def test_the_binding_has_the_headers_layout(tmp_path):
    structs = {"snn_recurrence_args": ops._RecArgs, "snn_recurrence_grads": ops._RecGrads, "snn_norm_args": ops._NormArgs,
               "snn_norm_grads": ops._NormGrads, "snn_units_args": ops._UnitsArgs, "snn_units_grads": ops._UnitsGrads}
    lines = []
    for n, s in structs.items():
        lines.append(f'printf("{n} %zu\\n", sizeof({n}));')
        lines += [f'printf("{n}.{f} %zu\\n", offsetof({n}, {f}));' for f, _ in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "snn_ops.h"\nint main(void) {' + "\n".join(lines) + "return 0;}\n")
    assert os.system(f"gcc -std=c99 -Wall -Werror -I{ROOT}/include -o {tmp_path}/layout {src}") == 0
    said = dict(l.split() for l in os.popen(f"{tmp_path}/layout").read().splitlines())
    for n, s in structs.items():
        assert int(said[n]) == C.sizeof(s), n
        for f, _ in s._fields_:
            assert int(said[f"{n}.{f}"]) == getattr(s, f).offset, (n, f)


def rows(n, at=P):
    return ops._Rows(at, 2 * n, n)


def none():
    return ops._Rows(None, 0, 0)


def args(op, **kw):
    if op == "recurrence":
        a = ops._RecArgs(4, 2, 8, 0, 8.0, rows(8), rows(8), rows(8), rows(8), P, None, None, P)
    elif op == "norm":
        a = ops._NormArgs(4, 2, 8, 2, 0, 1, 0, 1e-5, rows(8), rows(8), P, P, None)
    else:
        a = ops._UnitsArgs(4, 2, 8, 12, 0, 0, rows(8), rows(12), P, P, None)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def grads(op, **kw):
    if op == "recurrence":
        g = ops._RecGrads(rows(8), None, rows(8), rows(8), rows(8), P, None)
    elif op == "norm":
        g = ops._NormGrads(rows(8), rows(8), P, P)
    else:
        g = ops._UnitsGrads(rows(12), rows(8), P, P)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


COMMON = [(dict(T=-1), ARG), (dict(B=0), ARG), (dict(D=0), ARG), (dict(type=2), ARG), (dict(x=none()), NULL), (dict(y=none()), NULL),
          (dict(x=rows(8, P + 2)), ARG), (dict(lengths=P + 1), ARG), (dict(D=1 << 23), ARG)]
OWN = {
    "recurrence": [(dict(sharpness=0.0), ARG), (dict(sharpness=-1.0), ARG), (dict(sharpness=float("nan")), ARG), (dict(sharpness=float("inf")), ARG),
                   (dict(i=none()), NULL), (dict(r=none()), NULL), (dict(decay=None), NULL), (dict(decay=P + 2), ARG), (dict(init=P + 2), ARG),
                   (dict(B=1 << 22), ARG), (dict(x=ops._Rows(P, -16, 8)), ARG), (dict(r=ops._Rows(P, 1 << 26, 8)), ARG), (dict(state=P + 2), ARG)],
    "norm": [(dict(groups=0), ARG), (dict(groups=3), ARG), (dict(groups=-2), ARG), (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG),
             (dict(D=1 << 15, groups=1), ARG), (dict(T=1 << 30, B=4), ARG), (dict(T=1 << 29, B=2), ARG), (dict(weight=P + 2), ARG), (dict(bias=P + 1), ARG)],
    "units": [(dict(F=0), ARG), (dict(F=-4), ARG), (dict(act=2), ARG), (dict(act=-1), ARG), (dict(F=(1 << 18) + 1), ARG), (dict(T=1 << 28), ARG),
              (dict(gate=None), NULL), (dict(up=None), NULL), (dict(gate=P + 2), ARG), (dict(up=P + 2), ARG)],
}


def forward(lib, op, a, saved=None, ws=None, size=0):
    return getattr(lib, f"snn_{op}_forward")(C.byref(a) if a is not None else None, saved, ws, size, None)


def needed(lib, op, a, backward):
    n = C.c_size_t(0)
    assert getattr(lib, f"snn_{op}_workspace_bytes")(C.byref(a), backward, C.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("op,change,status", [(op, *c) for op in OPS for c in COMMON + OWN[op]])
def test_refusals(lib, op, change, status):
    assert forward(lib, op, args(op, **change), None, P, 1 << 40) == status
    assert lib.snn_last_error(None)


@pytest.mark.parametrize("op", OPS)
def test_refusals_of_workspaces_and_gradients(lib, op):
    n = C.c_size_t(0)
    call = lambda name: getattr(lib, f"snn_{op}_{name}")
    assert forward(lib, op, None) == NULL
    assert call("workspace_bytes")(C.byref(args(op)), 0, None) == NULL and call("workspace_bytes")(None, 0, C.byref(n)) == NULL
    assert call("saved_bytes")(C.byref(args(op)), None) == NULL and call("saved_bytes")(C.byref(args(op, B=0)), C.byref(n)) == ARG
    assert call("workspace_bytes")(C.byref(args(op, D=-1)), 1, C.byref(n)) == ARG
    assert forward(lib, op, args(op), P + 4, P, 1 << 40) == ARG                            # saved is not aligned
    long = args(op, T=100000, B=1)
    need = needed(lib, op, long, 0)
    assert need > 0
    for ws, size in ((None, need), (P, need - 1), (P + 8, need)):
        assert forward(lib, op, long, None, ws, size) == WORKSPACE
    back = lambda a, g, saved=P, ws=P, size=1 << 40: call("backward")(C.byref(a) if a is not None else None, C.byref(g) if g is not None else None, saved, ws, size, None)
    g = grads(op)
    assert back(None, g) == NULL and back(args(op), None) == NULL and back(args(op), g, saved=None) == NULL
    assert back(args(op), grads(op, dy=none())) == NULL and back(args(op), grads(op, dx=none())) == NULL
    assert back(args(op), g, saved=P + 4) == ARG and back(args(op), grads(op, dy=rows(8, P + 2))) == ARG
    assert back(args(op), g, ws=None) == WORKSPACE and back(args(op), g, ws=P + 4) == WORKSPACE
    assert back(args(op), g, size=needed(lib, op, args(op), 1) - 1) == WORKSPACE
    if op == "recurrence":
        assert back(args(op), grads(op, ddecay=None)) == NULL and back(args(op), grads(op, di=ops._Rows(P, -8, 8))) == ARG
    if op == "units":
        assert back(args(op), grads(op, dgate=None)) == NULL and back(args(op), grads(op, dup=P + 1)) == ARG
    if op == "norm":
        assert back(args(op), grads(op, dweight=P + 1)) == ARG


def test_refusals_of_a_recurrence_step(lib):
    step = lambda **kw: lib.snn_recurrence_step(C.byref(args("recurrence", **({"T": 1} | kw))), None)
    assert lib.snn_recurrence_step(None, None) == NULL
    assert step(T=2) == ARG and step(init=P) == ARG and step(lengths=P) == ARG and step(state=None) == NULL


def test_sizes_of_what_is_saved(lib):
    n = C.c_size_t(0)
    for op, kw, size in (("recurrence", dict(T=17), 3 * 2 * 8 * 4), ("norm", {}, 2 * 2 * 8), ("norm", dict(per_step=1), 4 * 2 * 2 * 8),
                         ("units", dict(F=33), 32 * 64 * 8)):
        assert getattr(lib, f"snn_{op}_saved_bytes")(C.byref(args(op, **kw)), C.byref(n)) == 0 and n.value == size, op


def test_tensors_that_do_not_fit_are_refused_before_a_device_is_looked_for():
    """On a machine without a GPU every tensor is on the wrong device, and that is what is said."""
    import torch
    import paper_2402_18994_amd as snn
    x = torch.zeros(4, 2, 8)
    for f in (lambda: snn.gated_recurrence(x, x, x, torch.zeros(8)), lambda: snn.group_norm(x, 2), lambda: snn.gated_units(x, torch.zeros(3, 8), torch.zeros(3, 8))):
        with pytest.raises(binding.SnnError, match="HIP device"):
            f()
    with pytest.raises(binding.SnnError, match="float32 or bfloat16"):
        snn.group_norm(x.half(), 2)
