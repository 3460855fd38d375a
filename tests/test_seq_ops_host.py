"""Host-side checks of the sequence operators and AdamW that need no GPU: the header, the exported symbols, what the
entry points refuse before they touch a device, and that nothing else runs in their place."""
import ctypes as C
import os
import re

import pytest

from paper_2402_18994_amd import binding, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, ARG, SHAPE, WORKSPACE, HIP = 1, 2, 3, 4, 6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.library_path()):
        from paper_2402_18994_amd import build
        build.build()
    return ops._lib()


def test_every_declared_entry_point_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "snn_ops.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(snn_[a-z_]+)\s*\(", text)))
    assert {"snn_conv_forward", "snn_scan_backward", "snn_scan_step", "snn_adamw_step"} <= set(names)
    for n in names:
        assert hasattr(lib, n), n


def test_header_is_plain_c_and_the_binding_has_its_layout(tmp_path):
    structs = {"snn_rows": ops._Rows, "snn_conv_args": ops._ConvArgs, "snn_conv_grads": ops._ConvGrads, "snn_scan_args": ops._ScanArgs,
               "snn_scan_grads": ops._ScanGrads, "snn_adamw_tensor": ops._AdamTensor, "snn_adamw_args": ops._AdamArgs}
    lines = []
    for n, s in structs.items():
        lines.append(f'printf("{n} %zu\\n", sizeof({n}));')
        lines += [f'printf("{n}.{f} %zu\\n", offsetof({n}, {f}));' for f, _ in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "snn_ops.h"\nint main(void) {' + "\n".join(lines) + "return 0;}\n")
    assert os.system(f"gcc -std=c99 -Wall -Werror -I{ROOT}/include -o {tmp_path}/layout {src}") == 0
    said = dict(l.split() for l in os.popen(f"{tmp_path}/layout").read().splitlines())
    for n, s in structs.items():
        assert int(said[n]) == C.sizeof(s), n
        for f, _ in s._fields_:
            assert int(said[f"{n}.{f}"]) == getattr(s, f).offset, (n, f)


P = 1 << 20                     # an address that nothing reads: every call here is refused before


def conv(**kw):
    a = ops._ConvArgs(4, 2, 8, 4, 0, 1, ops._Rows(P, 16, 8), ops._Rows(P, 16, 8), P, P, None, None, P)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def scan(**kw):
    r = lambda n: ops._Rows(P, 2 * n, n)
    a = ops._ScanArgs(4, 2, 8, 16, 1, 0, 1, r(8), r(8), r(8), r(16), r(16), r(8), P, P, P, None, None, P)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def none():
    return ops._Rows(None, 0, 0)


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), ARG), (dict(B=0), ARG), (dict(D=0), ARG), (dict(W=0), ARG), (dict(W=9), ARG), (dict(type=2), ARG),
    (dict(B=1 << 20, D=1 << 12), ARG), (dict(weight=None), NULL), (dict(x=none()), NULL), (dict(y=none()), NULL),
    (dict(x=ops._Rows(P + 2, 16, 8)), ARG), (dict(bias=P + 1), ARG), (dict(init=P + 2), ARG), (dict(lengths=P + 1), ARG)])
def test_convolution_refusals(lib, change, status):
    assert lib.snn_conv_forward(C.byref(conv(**change)), None) == status
    assert lib.snn_last_error(None)


def test_convolution_refusals_of_gradients_and_steps(lib):
    n = C.c_size_t(0)
    assert lib.snn_conv_forward(None, None) == NULL and lib.snn_conv_step(None, None) == NULL
    assert lib.snn_conv_workspace_bytes(C.byref(conv()), None) == NULL
    assert lib.snn_conv_workspace_bytes(C.byref(conv(W=9)), C.byref(n)) == ARG
    assert lib.snn_conv_workspace_bytes(C.byref(conv()), C.byref(n)) == 0 and n.value >= 5 * 8 * 4
    g = ops._ConvGrads(ops._Rows(P, 16, 8), ops._Rows(P, 16, 8), None, P, P, None)
    call = lambda a, g, ws, size: lib.snn_conv_backward(C.byref(a), C.byref(g), ws, size, None)
    assert lib.snn_conv_backward(C.byref(conv()), None, P, 1 << 20, None) == NULL
    assert call(conv(), ops._ConvGrads(ops._Rows(P, 16, 8), ops._Rows(P, 16, 8), None, None, P, None), P, 1 << 20) == NULL
    assert call(conv(), ops._ConvGrads(none(), ops._Rows(P, 16, 8), None, P, P, None), P, 1 << 20) == NULL
    assert call(conv(), g, None, 1 << 20) == WORKSPACE
    assert call(conv(), g, P + 4, 1 << 20) == WORKSPACE
    assert call(conv(), g, P, n.value - 1) == WORKSPACE
    assert call(conv(), ops._ConvGrads(ops._Rows(P + 1, 16, 8), ops._Rows(P, 16, 8), None, P, P, None), P, 1 << 20) == ARG
    for bad, status in ((dict(T=2), ARG), (dict(T=1, init=P), ARG), (dict(T=1, lengths=P), ARG), (dict(T=1, state=None), NULL)):
        assert lib.snn_conv_step(C.byref(conv(**bad)), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), ARG), (dict(B=0), ARG), (dict(D=-8), ARG), (dict(N=0), ARG), (dict(N=65), ARG), (dict(groups=0), ARG), (dict(groups=3), ARG),
    (dict(type=7), ARG), (dict(B=1 << 20, D=64), ARG), (dict(T=1 << 30, B=8), ARG), (dict(B=1 << 18, D=64, groups=64), ARG), (dict(A=None), NULL), (dict(x=none()), NULL),
    (dict(dt=none()), NULL), (dict(bv=none()), NULL), (dict(cv=none()), NULL), (dict(y=none()), NULL), (dict(z=ops._Rows(P + 2, 8, 8)), ARG), (dict(skip=P + 2), ARG)])
def test_scan_refusals(lib, change, status):
    assert lib.snn_scan_forward(C.byref(scan(**change)), None, None, 0, None) == status
    assert lib.snn_last_error(None)


def test_scan_refusals_of_workspaces_gradients_and_steps(lib):
    n = C.c_size_t(0)
    long = scan(T=1024)
    assert lib.snn_scan_workspace_bytes(C.byref(long), 0, None) == NULL
    assert lib.snn_scan_workspace_bytes(C.byref(long), 0, C.byref(n)) == 0 and n.value > 0      # cut in chunks of time
    assert lib.snn_scan_forward(C.byref(long), None, None, 0, None) == WORKSPACE
    assert lib.snn_scan_forward(C.byref(long), None, P, n.value - 1, None) == WORKSPACE
    assert lib.snn_scan_forward(C.byref(long), P + 4, P, n.value, None) == ARG
    assert lib.snn_scan_saved_bytes(C.byref(scan(T=17)), C.byref(n)) == 0 and n.value == 2 * 2 * 8 * 16 * 4
    r = ops._Rows(P, 16, 8)
    full = dict(dy=r, d_state=None, dx=r, ddt=r, dz=r, dbv=r, dcv=r, dA=P, dskip=P, ddt_bias=P, dinit=None)
    call = lambda saved=P, ws=P, size=1 << 30, **kw: lib.snn_scan_backward(C.byref(scan()), C.byref(ops._ScanGrads(**(full | kw))), saved, ws, size, None)
    assert lib.snn_scan_backward(C.byref(scan()), None, P, P, 1 << 30, None) == NULL
    assert call(saved=None) == NULL
    for name in ("dy", "dx", "ddt", "dz", "dbv", "dcv"):
        assert call(**{name: none()}) == NULL, name
        assert call(**{name: ops._Rows(P + 1, 16, 8)}) == ARG, name
    assert call(dA=None) == NULL
    assert call(saved=P + 8) == ARG and call(dskip=P + 1) == ARG
    assert call(ws=None) == WORKSPACE and call(size=16) == WORKSPACE
    for bad, status in ((dict(T=2), ARG), (dict(T=1, init=P), ARG), (dict(T=1, lengths=P), ARG), (dict(T=1, state=None), NULL)):
        assert lib.snn_scan_step(C.byref(scan(**bad)), None) == status


def test_adamw_refusals(lib):
    def call(count=1, null=False, tensor=None, **kw):
        a = ops._AdamArgs(32, 0, P, P, None, None, 1, 0, 1e-3, 0.9, 0.999, 1e-8, 1.0)
        for k, v in kw.items():
            setattr(a, k, v)
        t = (ops._AdamTensor * 1)(ops._AdamTensor(**(dict(param=P, grad=P, copy=None, n=8, at=0, weight_decay=0.0) | (tensor or {}))))
        return lib.snn_adamw_step(C.byref(a), None if null else t, count, None)

    assert lib.snn_adamw_step(None, None, 0, None) == NULL
    assert call(null=True) == NULL and call(count=-1) == ARG
    for kw in (dict(bits=16), dict(grad_type=2), dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=float("nan")), dict(eps=-1.0),
               dict(lr=float("inf")), dict(grad_scale=float("nan")), dict(m=P + 4)):
        assert call(**kw) == ARG, kw
    assert call(m=None) == NULL and call(bits=8) == NULL
    for t, status in ((dict(n=-1), ARG), (dict(at=64), ARG), (dict(at=-128), ARG), (dict(param=None), NULL), (dict(grad=None), NULL),
                      (dict(param=P + 2), ARG), (dict(copy=P + 1), ARG), (dict(n=1 << 36), ARG), (dict(weight_decay=float("inf")), ARG)):
        assert call(tensor=t) == status, t
    assert call(count=0) == 0 and call(tensor=dict(n=0)) == 0       # nothing to do
    assert lib.snn_adamw_network_elements(None, None) == NULL and lib.snn_adamw_network_step(None, None, 0.0) == NULL


def test_python_entry_points_refuse_before_a_launch(lib):
    import torch
    x = torch.zeros(4, 2, 8)
    w = torch.zeros(8, 4)
    with pytest.raises(binding.SnnError):                            # tensors of the host: there is no other path
        ops.causal_conv(x, w)
    with pytest.raises(binding.SnnError):
        ops.causal_conv(x.to(torch.float16), w)
    with pytest.raises(binding.SnnError):
        ops.selective_scan(x, x, torch.zeros(8, 16), torch.zeros(4, 2, 16), torch.zeros(4, 2, 16))
    with pytest.raises(binding.SnnError):
        ops.AdamW([w])
    with pytest.raises(binding.SnnError):
        ops.AdamW([])


def test_adamw_refuses_tensors_that_share_memory(lib):
    """All tensors are updated at once: the same one twice, or two that overlap, would be a race."""
    def call(*tensors):
        a = ops._AdamArgs(8, 0, P, P, P, P, 1, 0, 1e-3, 0.9, 0.999, 1e-8, 1.0)
        t = (ops._AdamTensor * len(tensors))(*(ops._AdamTensor(**(dict(grad=P, copy=None, weight_decay=0.0) | x)) for x in tensors))
        return lib.snn_adamw_step(C.byref(a), t, len(tensors), None), lib.snn_last_error(None)

    far = [dict(param=P + 4096 * i, n=200, at=256 * i) for i in range(600)]      # (more than are looked at without memory of their own)
    for order in (lambda v: v, lambda v: v[::-1], lambda v: v[1::2] + v[::2]):
        for extra in (dict(param=P, n=200), dict(param=P + 4096 * 7 + 796, n=1), dict(param=P - 4, n=2), dict(param=P - 4096, n=4096), dict(param=1 << 30, copy=P + 398, n=1),
                      dict(param=1 << 30, copy=1 << 30, n=4)):
            for some in (far[:9], far):
                status, text = call(*order(some + [dict(at=1 << 20) | extra]))
                assert status == ARG and b"share memory" in text, extra
        for at in (0, 128, 256 * 8, 256 * 8 + 128):
            status, text = call(*order(far[:9] + [dict(param=1 << 30, n=129, at=at)]))
            assert status == ARG and b"share a block" in text, at
    status, text = call(dict(param=P, copy=1 << 30, n=64, at=0), dict(param=P + 4096, copy=(1 << 30) + 126, n=64, at=128))
    assert status == ARG and b"share memory" in text
    assert call(dict(param=P, n=0, at=0), dict(param=P, n=0, at=0))[0] == 0      # nothing in them


def test_pieces_that_touch_do_not_overlap(tmp_path):
    """The host's comparison by itself, on pieces that may not be launched here: neighbours that touch, any order."""
    text = open(os.path.join(ROOT, "paper_2402_18994_amd", "csrc", "adamw.hip")).read()
    body = text[text.index("struct Piece {"):text.index("// Workgroups of one launch update all tensors at once")]
    src = tmp_path / "pieces.cpp"
    src.write_text("#include <algorithm>\n#include <cstdint>\n#include <cstddef>\n" + body + """
int main() {
  Piece touch[] = {{512, 768}, {0, 256}, {256, 512}, {768, 769}};
  Piece one[] = {{5, 9}};
  Piece share[] = {{512, 768}, {0, 257}, {256, 512}};
  Piece inside[] = {{0, 1000}, {10, 20}};
  return overlap(touch, 4) || overlap(one, 1) || overlap(one, 0) || !overlap(share, 3) || !overlap(inside, 2);
}
""")
    assert os.system(f"g++ -std=c++17 -Wall -Werror -o {tmp_path}/pieces {src}") == 0
    assert os.system(f"{tmp_path}/pieces") == 0
