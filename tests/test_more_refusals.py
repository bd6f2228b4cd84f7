"""What the heads' gated layers and table lookups refuse at the C entries and in Python, before any GPU work."""
import pytest
import torch

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
    need = L.derf_lookup_workspace(4, 5, 8)
    assert need > 0
    refused(backward(n=need - 1), b"workspace")
    refused(backward(ws=None), b"workspace")
    assert L.derf_lookup(None, 8, None, 0, 5, 8, 1.0, 0, None, 8, None) == derf.DERF_OK


def test_lookup_refuses_host_tensors():
    x, ids = torch.zeros((4, 8)), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: heads.lookup(x, ids), lambda: heads.lookup_backward(x, ids, 5)):
        with pytest.raises(ValueError):
            call()
