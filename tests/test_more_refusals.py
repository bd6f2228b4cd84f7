"""What the heads' gated layers, table lookups and orthogonalised updates refuse at the C entries and in Python, before any GPU work."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch
from torch.autograd import forward_ad

from paper_2011_12490_amd import derf, heads

INVALID = derf.DERF_ERR_INVALID_ARG
P = 4096  # an aligned address that no refused call may look at


def lib():
    return derf.lib()


def refused(rc, text):
    assert rc == INVALID
    assert text in lib().derf_last_error(), lib().derf_last_error()


# ---- gated layers ---------------------------------------------------------------------

@pytest.mark.parametrize("R,K,I,O,act,prec", [
    (-1, 4, 8, 8, 0, 0), (1 << 31, 4, 8, 8, 0, 0), (8, 0, 8, 8, 0, 0), (8, 257, 8, 8, 0, 0), (8, 4, 0, 8, 0, 0),
    (8, 4, 8, 65537, 0, 0), (8, 4, 8, 8, 0, 3), (8, 4, 16384, 16384, 0, 0), (8, 4, 32768, 16384, 0, 1)])
def test_gated_sizes(R, K, I, O, act, prec):
    L = lib()
    assert L.derf_heads_gated_workspace(R, K, I, O, prec) == -1
    assert L.derf_heads_gated(P, 1 << 18, P, P, P, R, K, I, O, act, prec, P, 1 << 18, P, 1 << 18, None) == INVALID
    assert L.derf_heads_gated_backward(P, 1 << 18, P, 1 << 18, P, 1 << 18, P, P, R, K, I, O, act, prec, P, 1 << 18, P, P,
                                       P, 1 << 60, None) == INVALID


def test_gated_arrays():
    L = lib()

    def forward(x=P, xs=16, w=P, b=P, off=P, act=0, y=P, ys=24, pre=P, ps=48):
        return L.derf_heads_gated(x, xs, w, b, off, 8, 4, 16, 24, act, 1, y, ys, pre, ps, None)

    def backward(dy=P, ds=24, pre=P, ps=48, x=P, xs=16, w=P, off=P, act=0, dx=P, dxs=16, dw=P, db=P, ws=P, n=1 << 40):
        return L.derf_heads_gated_backward(dy, ds, pre, ps, x, xs, w, off, 8, 4, 16, 24, act, 1, dx, dxs, dw, db, ws, n,
                                           None)

    refused(forward(x=None), b"null x")
    refused(forward(xs=15), b"stride")
    refused(forward(xs=1 << 21), b"2^21")
    refused(forward(w=None), b"null w")
    refused(forward(b=P + 2), b"bias is not aligned")
    refused(forward(off=None), b"null offsets")
    refused(forward(act=4), b"activation")
    refused(forward(act=-1), b"activation")
    refused(forward(ys=23), b"stride")
    refused(forward(ps=47), b"stride")
    refused(forward(pre=P + 1), b"pre is not aligned")
    refused(backward(dy=None), b"null dy")
    refused(backward(pre=None), b"null pre")
    refused(backward(ps=47), b"stride")
    refused(backward(x=None), b"null x")
    refused(backward(w=None), b"null w")
    refused(backward(act=4), b"activation")
    refused(backward(dxs=15), b"stride")
    refused(backward(dw=P + 1), b"out_w is not aligned")
    refused(backward(db=P + 2), b"out_bias is not aligned")
    need = L.derf_heads_gated_workspace(8, 4, 16, 24, 1)
    assert need > 0
    refused(backward(n=need - 1), b"workspace")
    refused(backward(ws=P + 8, n=need), b"workspace")
    refused(backward(ws=None, n=need), b"workspace")
    # nothing to do
    assert L.derf_heads_gated(None, 16, None, None, None, 0, 4, 16, 24, 0, 1, None, 24, None, 48, None) == derf.DERF_OK


def test_gated_refuses_host_tensors():
    x, w, off = torch.zeros((4, 8)), torch.zeros((3, 2, 5, 8)), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: heads.gated(x, w, None, off), lambda: heads.gated_backward(x, x, x, w, off)):
        with pytest.raises(ValueError):
            call()


# ---- lookups --------------------------------------------------------------------------

@pytest.mark.parametrize("T,V,D,scale,prec", [(-1, 4, 8, 1.0, 0), (1 << 31, 4, 8, 1.0, 0), (4, 0, 8, 1.0, 0), (4, 1 << 31, 8, 1.0, 0),
                                              (4, 4, 0, 1.0, 0), (4, 4, 65537, 1.0, 1)])
def test_lookup_sizes(T, V, D, scale, prec):
    L = lib()
    assert L.derf_lookup_workspace(T, V, D) == -1
    assert L.derf_lookup(P, 1 << 17, P, T, V, D, scale, prec, P, 1 << 17, None) == INVALID
    assert L.derf_lookup_backward(P, 1 << 17, P, T, V, D, scale, prec, P, P, 1 << 60, None) == INVALID


def test_lookup_arrays():
    L = lib()

    def forward(table=P, ts=8, ids=P, scale=1.0, prec=0, out=P, os=8):
        return L.derf_lookup(table, ts, ids, 4, 5, 8, scale, prec, out, os, None)

    def backward(dout=P, ds=8, ids=P, scale=1.0, prec=0, out=P, ws=P, n=1 << 40):
        return L.derf_lookup_backward(dout, ds, ids, 4, 5, 8, scale, prec, out, ws, n, None)

    refused(forward(table=None), b"null table")
    refused(forward(ts=7), b"stride")
    refused(forward(ids=P + 2), b"ids is not aligned")
    refused(forward(ids=None), b"null ids")
    refused(forward(scale=float("nan")), b"scale")
    refused(forward(prec=2), b"precision")
    refused(forward(out=None), b"null out")
    refused(forward(os=7), b"stride")
    refused(backward(dout=None), b"null dout")
    refused(backward(ds=-8), b"stride")
    refused(backward(ids=None), b"null ids")
    refused(backward(scale=float("inf")), b"scale")
    refused(backward(out=P + 2), b"out is not aligned")
    need = L.derf_lookup_workspace(4000, 5, 8)
    assert need > 0
    for ws, n in ((P, need - 1), (None, need), (P + 8, need)):
        refused(L.derf_lookup_backward(P, 8, P, 4000, 5, 8, 1.0, 0, P, ws, n, None), b"workspace")
    assert L.derf_lookup(None, 8, None, 0, 5, 8, 1.0, 0, None, 8, None) == derf.DERF_OK


def test_lookup_refuses_host_tensors():
    x, ids = torch.zeros((4, 8)), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: heads.lookup(x, ids), lambda: heads.lookup_backward(x, ids, 5)):
        with pytest.raises(ValueError):
            call()


# ---- orthogonalised updates -------------------------------------------------------------

@pytest.mark.parametrize("K,O,I,n,prec", [(-1, 8, 8, 5, 0), (32769, 8, 8, 5, 0), (4, 0, 8, 5, 0), (4, 8, 16385, 5, 0), (4, 8, 8, 5, 2)])
def test_orthogonalise_sizes(K, O, I, n, prec):
    L = lib()
    assert L.derf_orthogonalise_workspace(K, O, I, prec) == -1
    assert L.derf_orthogonalise(P, K, O, I, n, prec, P, P, 1 << 60, None) == INVALID


def test_orthogonalise_arrays():
    L = lib()

    def call(x=P, n=5, out=P, ws=P, size=1 << 50):
        return L.derf_orthogonalise(x, 3, 400, 500, n, 0, out, ws, size, None)

    refused(call(x=None), b"null x")
    refused(call(x=P + 2), b"x is not aligned")
    refused(call(n=0), b"iterations")
    refused(call(n=21), b"iterations")
    refused(call(out=None), b"null out")
    need = L.derf_orthogonalise_workspace(3, 400, 500, 0)
    refused(call(size=need - 1), b"workspace")
    refused(call(ws=P + 8), b"workspace")
    assert L.derf_orthogonalise(None, 0, 40, 50, 5, 0, None, None, 1 << 30, None) == derf.DERF_OK


def _matrices(**kw):
    t = dict(param=P, grad=P, m=P, copy=None, num_matrices=2, fan_out=8, fan_in=9, param_precision=0, grad_precision=0)
    t.update(kw)
    return derf.derf_muon_tensor(**t)


@pytest.mark.parametrize("kw,text", [
    (dict(num_matrices=-1), b"matrices"), (dict(num_matrices=32769), b"matrices"), (dict(fan_out=0), b"matrices"),
    (dict(fan_in=16385), b"matrices"), (dict(param=None), b"null array"), (dict(grad=None), b"null array"), (dict(m=None), b"null array"),
    (dict(param_precision=2), b"precision"), (dict(grad_precision=-1), b"precision"), (dict(m=P + 2), b"aligned"),
    (dict(copy=P + 1), b"aligned"), (dict(grad=P + 2), b"aligned")])
def test_muon_tensors(kw, text):
    h = ctypes.c_void_p(1)
    t = _matrices(**kw)
    refused(lib().derf_muon_create(ctypes.byref(h), ctypes.byref(t), 1), text)
    assert not h.value


@pytest.mark.parametrize("first,second", [
    (dict(), dict()), (dict(), dict(param=P + 64)), (dict(m=1 << 20), dict(param=1 << 21, grad=(1 << 20) + 572, m=1 << 22)),
    (dict(param=1 << 20, m=1 << 21, copy=(1 << 20) + 286), None), (dict(param=1 << 20, m=(1 << 20) + 575), None),
    (dict(param=1 << 20, m=1 << 21), dict(param=1 << 22, m=1 << 23, copy=1 << 20))])
def test_muon_arrays_that_share_memory(first, second):
    """Arrays of 2 matrices of 8 x 9: 576 bytes in float, 288 in bf16."""
    h = ctypes.c_void_p(1)
    tensors = [_matrices(**t) for t in (first, second) if t is not None]
    table = (derf.derf_muon_tensor * len(tensors))(*tensors)
    if first.get("m") == (1 << 20) + 575:
        refused(lib().derf_muon_create(ctypes.byref(h), table, len(tensors)), b"aligned")
    else:
        refused(lib().derf_muon_create(ctypes.byref(h), table, len(tensors)), b"shares memory")
    assert not h.value


def test_muon_calls():
    L = lib()
    h = ctypes.c_void_p(1)
    refused(L.derf_muon_create(None, None, 0), b"null out")
    refused(L.derf_muon_create(ctypes.byref(h), None, 1), b"num_tensors")
    refused(L.derf_muon_create(ctypes.byref(h), None, -1), b"num_tensors")
    refused(L.derf_muon_step(None, 0.1, 0.9, 1, 0.0, 5, None, None), b"null optimizer")
    L.derf_muon_destroy(None)
    # an optimizer of no matrices needs no GPU: its scalars are still checked
    empty = _matrices(num_matrices=0, param=None, grad=None, m=None)
    assert L.derf_muon_create(ctypes.byref(h), ctypes.byref(empty), 1) == derf.DERF_OK
    good = dict(lr=0.02, momentum=0.9, nesterov=1, weight_decay=0.0, iterations=5)
    for kw in (dict(lr=-1.0), dict(lr=float("nan")), dict(momentum=1.0), dict(momentum=-0.1), dict(weight_decay=float("inf")),
               dict(iterations=0), dict(iterations=21)):
        assert L.derf_muon_step(h, *dict(good, **kw).values(), None, None) == INVALID, kw
    refused(L.derf_muon_step(h, *good.values(), P + 2, None), b"grad_scale")
    assert L.derf_muon_step(h, *good.values(), None, None) == derf.DERF_OK
    L.derf_muon_destroy(h)


def test_muon_tensor_has_the_headers_layout(tmp_path):
    """A C program prints the struct's size and offsets; the binding's mirror has the same."""
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no gcc")
    mirror = derf.derf_muon_tensor
    names = [f[0] for f in mirror._fields_]
    prints = "".join('printf(" %%zu", offsetof(derf_muon_tensor, %s));\n' % n for n in names)
    source = tmp_path / "layout.c"
    source.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "derf.h"\n'
                      'int main(void) {\nprintf("%zu", sizeof(derf_muon_tensor));\n' + prints + "return 0;\n}\n")
    program = str(tmp_path / "layout")
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run([cc, "-I", include, str(source), "-o", program], check=True)
    got = [int(v) for v in subprocess.run([program], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(mirror)] + [getattr(mirror, n).offset for n in names]


def test_muon_refuses_host_tensors():
    x = torch.zeros((4, 8))
    for call in (lambda: heads.orthogonalise(x), lambda: heads.Muon([x], [x])):
        with pytest.raises(ValueError):
            call()


def test_forward_mode_tangents():
    x = torch.zeros((4, 8))
    heads._no_tangent(x, "x")
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        heads._no_tangent(x, "x")
        heads._no_tangent(forward_ad.unpack_dual(dual).primal, "x")
        for t in (dual, dual[1:], dual * 2):
            with pytest.raises(ValueError, match="y has a forward-mode tangent"):
                heads._no_tangent(t, "y")
