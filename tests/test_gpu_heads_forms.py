"""The heads' layers in each form that the library has a kernel for, and with each
choice of outputs, against plain float64 (tolerances: test_gpu_heads.py).
test_linear_forms.py checks that these and that module's cases reach every kernel."""
import numpy as np
import pytest
import torch

from paper_2011_12490_amd import heads
from test_gpu_heads import BF16, FP32, assert_near, layer, rand

pytestmark = pytest.mark.gpu

# Rows that stream past weights in LDS: every depth in steps of 128 bytes, one and two
# widths of a workgroup's, results in whole 128-byte lines and others
STREAM_ROWS = ([20000, 0, 12900, 37], 63)
STREAM_FORWARD = [(I, O) for I in (20, 40, 70, 100, 150, 250, 319) for O in (50, 64, 100, 128)]
STREAM_BACKWARD = [(I, O) for I in (50, 64, 200, 256) for O in (20, 40, 100)]

# Large tiles, more of them than compute units, on ragged heads, with rows without a head and a part
# of a tile's columns: the layer of the first, the rows' gradient of the second (whose weights'
# gradient is split into stretches, so that both are not one launch)
LARGE = [([13000, 0, 9700, 1, 1200], 130, 520, 1032), ([13000, 0, 9700, 1, 1200], 130, 1032, 520)]

# For each choice of outputs: narrow, odd, wide, deep and few rows
OUTPUT_CASES = [([300, 0, 41], 9, 63, 128), ([300, 0, 41], 9, 40, 24), ([2000, 700], 0, 319, 256), ([700, 900], 5, 520, 1032),
                ([3, 0, 60, 1], 2, 40, 1500), ([3000, 1], 7, 256, 3)]
# (dx, dW, db) wanted
OUTPUTS = [(True, False, False), (False, True, False), (False, False, True), (True, True, False), (True, False, True),
           (False, True, True)]


def check_forward(counts, tail, I, O, relu, dtype):
    x, w, b, offsets, _ = layer(counts, tail, I, O, 0, 0, dtype, I * O)
    y = heads.linear(x, w, b, offsets, relu)
    ends = offsets.tolist()
    for h in range(len(counts)):
        s = slice(ends[h], ends[h + 1])
        xd, wd, bd = x[s].double(), w[h].double(), b[h].double()
        want = xd @ wd.T + bd
        assert_near(y[s], want.clamp_min(0) if relu else want, xd.abs() @ wd.abs().T + bd.abs(), I + 1)
    assert not bool(y[ends[-1]:].any())


def gradients(dy, x, w, offsets, y, outputs):
    """heads.linear_backward with the given ones of dx, dW, db at the C entry, the rest
    None, and without the inputs that only those need."""
    (R, I), (K, O) = x.shape, w.shape[:2]
    new = lambda wanted, *shape, dtype=FP32: torch.full(shape, 7.0, dtype=dtype, device="cuda") if wanted else None  # noqa: E731
    dx, dw, db = new(outputs[0], R, I, dtype=x.dtype), new(outputs[1], K, O, I), new(outputs[2], K, O)
    prec = heads._PRECISION[x.dtype]
    need = heads._workspace_bytes("derf_heads_linear_workspace", R, K, I, O, int(y is not None), prec)
    ws = torch.empty((max(need, 16),), dtype=torch.uint8, device="cuda")
    heads._call("derf_heads_linear_backward", x.device, dy.data_ptr(), O, x.data_ptr() if outputs[1] else None, I,
                w.data_ptr() if outputs[0] else None, heads._ptr(y), O, offsets.data_ptr(), R, K, I, O, prec, heads._ptr(dx), I,
                heads._ptr(dw), heads._ptr(db), ws.data_ptr(), need)
    return dx, dw, db


def check_backward(counts, tail, I, O, relu, dtype, outputs=((True, True, True),)):
    x, w, _, offsets, g = layer(counts, tail, I, O, 0, 0, dtype, I + 3 * O)
    R, ends = x.shape[0], offsets.tolist()
    dy = rand(g, R, O).to(dtype)
    y = rand(g, R, O).clamp_min(0).to(dtype) if relu else None
    if tail:
        dy[R - tail:] = float("nan")
    for wanted in outputs:
        dx, dw, db = gradients(dy, x, w, offsets, y, wanted)
        for h in range(len(counts)):
            s = slice(ends[h], ends[h + 1])
            dz = dy[s].double()
            if relu:
                dz = torch.where(y[s] > 0, dz, 0.0)
            xd, wd = x[s].double(), w[h].double()
            if dx is not None:
                assert_near(dx[s], dz @ wd, dz.abs() @ wd.abs(), O)
            if dw is not None:
                assert_near(dw[h], dz.T @ xd, dz.abs().T @ xd.abs(), counts[h])
            if db is not None:
                assert_near(db[h], dz.sum(0), dz.abs().sum(0), counts[h])
        if dx is not None:
            assert not bool(dx[ends[-1]:].any())


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("I,O", STREAM_FORWARD)
def test_streaming_layers(I, O, dtype):
    check_forward(*STREAM_ROWS, I, O, O % 3 == 1, dtype)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("I,O", STREAM_BACKWARD)
def test_streaming_gradients(I, O, relu, dtype):
    check_backward(*STREAM_ROWS, I, O, relu, dtype, [(True, True, True), (True, False, False)])


@pytest.mark.parametrize("counts,tail,I,O", LARGE)
def test_large_tiles(counts, tail, I, O):
    check_forward(counts, tail, I, O, True, BF16)
    for relu in (False, True):
        check_backward(counts, tail, I, O, relu, BF16)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("counts,tail,I,O", OUTPUT_CASES)
def test_each_choice_of_outputs(counts, tail, I, O, relu, dtype):
    check_backward(counts, tail, I, O, relu, dtype, OUTPUTS)


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_no_rows_leave_zeros_in_each_choice_of_outputs(dtype):
    for I, O in ((63, 128), (319, 256)):
        x, w, _, offsets, _ = layer([0, 0], 0, I, O, 0, 0, dtype, 1)
        for wanted in OUTPUTS:
            _, dw, db = gradients(x.new_empty((0, O)), x, w, offsets, None, wanted)
            assert all(out is None or not bool(out.any()) for out in (dw, db))
