"""What the training operators refuse, before any GPU work: sizes, strides,
alignment and null arrays at the C entries, tensors that do not fit in Python."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2011_12490_amd import derf, heads

INVALID = derf.DERF_ERR_INVALID_ARG
P = 4096  # an aligned address that no refused call may look at


def lib():
    return derf.lib()


def refused(rc, text):
    assert rc == INVALID
    assert text in lib().derf_last_error()


@pytest.mark.parametrize("T,k,K", [(-1, 1, 4), (4, 0, 4), (4, 17, 4), (1 << 30, 2, 4), (4, 2, 0), (4, 2, 257)])
def test_route_sizes(T, k, K):
    assert lib().derf_route_workspace(T, k, K) == -1
    assert lib().derf_route(P, T, k, K, P, P, P, P, 1 << 40, None) == INVALID


def test_route_arrays():
    L = lib()
    need = L.derf_route_workspace(1 << 20, 2, 16)
    assert need > 0
    refused(L.derf_route(P, 1 << 20, 2, 16, P, P, P, P, need - 1, None), b"workspace")
    refused(L.derf_route(P, 1 << 20, 2, 16, P, P, P, None, need, None), b"workspace")
    refused(L.derf_route(P, 1 << 20, 2, 16, P, P, P, P + 8, need, None), b"workspace")
    refused(L.derf_route(None, 8, 2, 16, P, P, P, P, 1 << 20, None), b"null heads")
    refused(L.derf_route(P, 8, 2, 16, None, P, P, P, 1 << 20, None), b"null out_offsets")
    refused(L.derf_route(P, 8, 2, 16, P, P + 2, P, P, 1 << 20, None), b"out_pair is not aligned")


@pytest.mark.parametrize("T,k,D,prec,stride,text", [
    (-1, 2, 8, 0, 8, b"num_tokens"), (4, 0, 8, 0, 8, b"top_k"), (1 << 31, 1, 8, 0, 8, b"2^31"),
    (4, 2, 0, 0, 8, b"dim"), (4, 2, 65537, 0, 65537, b"dim"), (4, 2, 8, 2, 8, b"precision"),
    (4, 2, 8, 0, 7, b"stride"), (4, 2, 8, 1, -8, b"stride")])
def test_rows_sizes(T, k, D, prec, stride, text):
    L = lib()
    refused(L.derf_dispatch(P, stride, P, T, k, D, prec, P, max(stride, D), None), text)
    refused(L.derf_combine(P, stride, P, P, T, k, D, prec, P, max(stride, D), None), text)
    refused(L.derf_combine_backward(P, stride, P, max(stride, D), P, P, T, k, D, prec, P,
                                    max(stride, D), P, None), text)


def test_rows_arrays():
    L = lib()
    refused(L.derf_dispatch(None, 8, P, 4, 2, 8, 0, P, 8, None), b"null x")
    refused(L.derf_dispatch(P + 2, 8, P, 4, 2, 8, 0, P, 8, None), b"not aligned")
    refused(L.derf_dispatch(P + 1, 8, P, 4, 2, 8, 1, P, 8, None), b"not aligned")
    refused(L.derf_dispatch(P, 8, None, 4, 2, 8, 0, P, 8, None), b"null row")
    refused(L.derf_combine(P, 8, None, P, 4, 2, 8, 0, None, 8, None), b"null out")
    refused(L.derf_combine(P, 8, P + 2, P, 4, 2, 8, 0, P, 8, None), b"weights is not aligned")
    refused(L.derf_combine_backward(P, 8, None, 8, P, P, 4, 2, 8, 0, P, 8, P, None), b"null rows")
    refused(L.derf_combine_backward(P, 8, P, 8, P, P, 4, 2, 8, 0, None, 8, P, None), b"null out_rows")
    # nothing to do
    assert L.derf_dispatch(None, 8, None, 0, 2, 8, 0, None, 8, None) == derf.DERF_OK
    assert L.derf_combine(None, 8, None, None, 0, 2, 8, 0, None, 8, None) == derf.DERF_OK


@pytest.mark.parametrize("R,K,I,O,prec", [(-1, 4, 8, 8, 0), (1 << 31, 4, 8, 8, 0), (8, 0, 8, 8, 0), (8, 257, 8, 8, 0),
                                          (8, 4, 0, 8, 0), (8, 4, 8, 65537, 0), (8, 4, 8, 8, 3)])
def test_linear_sizes(R, K, I, O, prec):
    L = lib()
    assert L.derf_heads_linear_workspace(R, K, I, O, 1, prec) == -1
    assert L.derf_heads_linear(P, 1 << 17, P, P, P, R, K, I, O, 0, prec, P, 1 << 17, None) == INVALID
    assert L.derf_heads_linear_backward(P, 1 << 17, P, 1 << 17, P, None, 0, P, R, K, I, O, prec, P, 1 << 17, P, P,
                                        P, 1 << 40, None) == INVALID


def test_linear_arrays():
    L = lib()

    def forward(x=P, xs=16, w=P, b=P, off=P, y=P, ys=24):
        return L.derf_heads_linear(x, xs, w, b, off, 8, 4, 16, 24, 1, 1, y, ys, None)

    def backward(dy=P, ds=24, x=P, xs=16, w=P, y=P, ys=24, off=P, dx=P, dxs=16, dw=P, db=P, ws=P, n=1 << 40):
        return L.derf_heads_linear_backward(dy, ds, x, xs, w, y, ys, off, 8, 4, 16, 24, 1, dx, dxs, dw, db, ws, n, None)

    refused(forward(x=None), b"null x")
    refused(forward(xs=15), b"stride")
    refused(forward(w=None), b"null w")
    refused(forward(b=P + 2), b"bias is not aligned")
    refused(forward(off=None), b"null offsets")
    refused(forward(ys=23), b"stride")
    refused(forward(y=P + 1), b"y is not aligned")
    refused(backward(dy=None), b"null dy")
    refused(backward(ds=23), b"stride")
    refused(backward(x=None), b"null x")
    refused(backward(w=None), b"null w")
    refused(backward(ys=3), b"stride")
    refused(backward(off=None), b"null offsets")
    refused(backward(dxs=15), b"stride")
    refused(backward(dw=P + 2), b"out_w is not aligned")
    refused(backward(db=P + 1), b"out_bias is not aligned")
    if L.derf_heads_linear_workspace(8, 4, 16, 24, 1, 1) > 0:
        refused(backward(n=0), b"workspace")


def _tensor(**kw):
    t = dict(param=P, grad=P, m=P, v=P, m_scale=P, v_scale=P, copy=None, n=10, param_precision=0, grad_precision=0)
    t.update(kw)
    return derf.derf_adamw_tensor(**t)


@pytest.mark.parametrize("kw,bits,text", [
    (dict(n=-1), 32, b"values"), (dict(n=1 << 40), 32, b"values"), (dict(param=None), 32, b"null array"),
    (dict(grad=None), 32, b"null array"), (dict(v=None), 8, b"null array"), (dict(m_scale=None), 8, b"null scales"),
    (dict(param_precision=2), 32, b"precision"), (dict(m=P + 2), 32, b"aligned"), (dict(copy=P + 1), 8, b"aligned"),
    (dict(v_scale=P + 2), 8, b"aligned"), (dict(), 16, b"state_bits")])
def test_adamw_tensors(kw, bits, text):
    h = ctypes.c_void_p(1)
    t = _tensor(**kw)
    refused(lib().derf_adamw_create(ctypes.byref(h), ctypes.byref(t), 1, bits), text)
    assert not h.value


def test_adamw_calls():
    L = lib()
    h = ctypes.c_void_p(1)
    refused(L.derf_adamw_create(None, None, 0, 32), b"null out")
    refused(L.derf_adamw_create(ctypes.byref(h), None, 1, 32), b"num_tensors")
    refused(L.derf_adamw_create(ctypes.byref(h), None, -1, 32), b"num_tensors")
    refused(L.derf_adamw_step(None, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1, None, None), b"null optimizer")
    L.derf_adamw_destroy(None)
    # an optimizer of no values needs no GPU: its scalars are still checked
    empty = _tensor(n=0, param=None, grad=None, m=None, v=None)
    assert L.derf_adamw_create(ctypes.byref(h), ctypes.byref(empty), 1, 32) == derf.DERF_OK
    good = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, step=1)
    for kw in (dict(lr=-1.0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=float("inf")),
               dict(weight_decay=-1e-3), dict(step=0)):
        a = dict(good, **kw)
        assert L.derf_adamw_step(h, *a.values(), None, None) == INVALID, kw
    refused(L.derf_adamw_step(h, *good.values(), P + 2, None), b"grad_scale")
    assert L.derf_adamw_step(h, *good.values(), None, None) == derf.DERF_OK
    L.derf_adamw_destroy(h)


def test_python_refuses_host_tensors():
    ids = torch.zeros((4, 2), dtype=torch.int32)
    x = torch.zeros((4, 8))
    r = heads.Routing(torch.zeros(4, dtype=torch.int32), torch.zeros(8, dtype=torch.int32), ids, 3)
    w, off = torch.zeros((3, 5, 8)), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: heads.route(ids, 3), lambda: heads.dispatch(x, r), lambda: heads.combine(x, r),
                 lambda: heads.combine_backward(x, x, r), lambda: heads.linear(x, w, None, off),
                 lambda: heads.linear_backward(x, x, w, off), lambda: heads.AdamW([x], [x])):
        with pytest.raises(ValueError):
            call()


def test_adamw_tensor_has_the_headers_layout(tmp_path):
    """A C program prints the struct's size and offsets; the binding's mirror has the same."""
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no gcc")
    mirror = derf.derf_adamw_tensor
    names = [f[0] for f in mirror._fields_]
    prints = "".join('printf(" %%zu", offsetof(derf_adamw_tensor, %s));\n' % n for n in names)
    source = tmp_path / "layout.c"
    source.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "derf.h"\n'
                      'int main(void) {\nprintf("%zu", sizeof(derf_adamw_tensor));\n' + prints + "return 0;\n}\n")
    program = str(tmp_path / "layout")
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run([cc, "-I", include, str(source), "-o", program], check=True)
    got = [int(v) for v in subprocess.run([program], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(mirror)] + [getattr(mirror, n).offset for n in names]
