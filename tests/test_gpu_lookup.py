"""Table lookups and their gradient on the GPU against plain implementations.

A looked-up row is exact: one product in float32, rounded once to the table's type, as
torch does it.  A gradient's row of n samples is within (n + 1) 2^-24 of the samples'
magnitudes summed, whatever the order, and the scale costs one more rounding; (2 n + 8)
2^-24 is allowed.  Rows without a sample are zero.
"""
import numpy as np
import pytest
import torch

from paper_2011_12490_amd import heads
from test_gpu_heads import BF16, FP32, gen, rand, strided

pytestmark = pytest.mark.gpu

CASES = [  # samples, rows, dim, pad, shift, how ids are drawn
    (0, 5, 8, 0, 0, "even"), (1, 1, 1, 0, 0, "even"), (1, 1000, 3, 0, 0, "even"), (5, 2, 7, 0, 0, "even"), (31, 3, 9, 2, 1, "even"),
    (64, 500, 48, 0, 0, "masked"), (33, 1, 64, 0, 0, "even"), (100, 70, 5, 0, 0, "none"), (1000, 65, 33, 1, 1, "masked"),
    (8192, 300, 16, 0, 0, "skewed"), (8192, 1 << 20, 4, 0, 0, "even"), (8193, 255, 12, 0, 0, "masked"), (8200, 256, 31, 0, 0, "even"),
    (9000, 1023, 2, 0, 0, "skewed"), (9000, 1024, 130, 2, 0, "even"), (30000, 100000, 64, 0, 0, "masked"), (40000, 3, 96, 0, 0, "skewed"),
    (50000, 1, 8, 0, 0, "even"), (70000, 70000, 1, 0, 0, "masked"), (100000, 5000, 48, 0, 0, "skewed"), (20000, 600, 1000, 0, 0, "skewed"),
    (12000, 2000, 2050, 0, 0, "masked"), (200000, 17, 20, 0, 0, "one"), (65536, 40, 256, 0, 0, "sorted"), (256, 9, 734, 0, 0, "skewed"), (257, 9, 734, 0, 0, "skewed"),
    (200, 100000, 64, 0, 0, "masked"), (1500, 20000, 360, 0, 0, "masked"), (300000, 2, 130, 0, 0, "masked"), (5000, 4, 33, 1, 1, "one"),
    (70000, 3000, 8, 0, 0, "sorted"), (600000, 700, 3, 0, 0, "skewed"), (9000, (1 << 21) + 5, 3, 0, 0, "even"),
    (280001, 5000, 512, 0, 0, "masked"), (512, 9, 33, 0, 0, "masked"), (513, 1024, 850, 1, 0, "skewed"), (1024, 70000, 8, 0, 0, "masked"),
    (1024, 1, 3, 0, 0, "even"), (400, 3000, 1, 0, 0, "one"), (1024, 40000, 70, 0, 0, "one"), (900000, 2, 4, 0, 0, "skewed")]


def ids_of(g, T, V, how):
    u = torch.rand(T, generator=g, device="cuda").double()
    ids = (V * (u ** 4 if how == "skewed" else u)).long().clamp_max(V - 1)
    if how == "masked":
        odd = torch.rand(T, generator=g, device="cuda")
        ids = torch.where(odd < 0.1, -1, torch.where(odd < 0.15, V, torch.where(odd < 0.2, 2 ** 31 - 1, torch.where(odd < 0.22, -2 ** 31, ids))))
    if how == "none":
        ids = torch.full_like(ids, -7)
    if how == "one":
        ids = torch.full_like(ids, V - 1)
    if how == "sorted":
        ids = ids.sort().values
    return ids.int()


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("T,V,D,pad,shift,how", CASES)
def test_lookup(T, V, D, pad, shift, how, dtype):
    g = gen(T + V)
    ids = ids_of(g, T, V, how)
    table = strided(rand(g, V, D).to(dtype), pad, shift)
    out = heads.lookup(table, ids, 1.7, strided(torch.full((T, D), 7.0, dtype=dtype, device="cuda"), pad, shift))
    has = ((ids >= 0) & (ids < V))[:, None]
    want = torch.where(has, table[ids.long().clamp(0, V - 1)].float() * 1.7, 0.0).to(dtype)
    assert torch.equal(out, want)
    if pad and T > 1:
        assert bool(out.as_strided((T - 1, pad), (D + pad, 1), out.storage_offset() + D).isnan().all())
    assert torch.equal(heads.lookup(table, ids), torch.where(has, table[ids.long().clamp(0, V - 1)], torch.zeros((), dtype=dtype, device="cuda")))


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("T,V,D,pad,shift,how", CASES)
def test_lookup_gradient(T, V, D, pad, shift, how, dtype):
    g = gen(T + 3 * V)
    ids = ids_of(g, T, V, how)
    dout = strided(rand(g, T, D).to(dtype), pad, shift)
    has = (ids >= 0) & (ids < V)
    dout[~has] = float("nan")  # not looked at
    got = heads.lookup_backward(dout, ids, V, 0.3, out=torch.full((V, D), 7.0, device="cuda"))
    at, rows = ids[has].long(), dout[has].double()
    new = lambda: torch.zeros(V, D, dtype=torch.float64, device="cuda")  # noqa: E731
    want, size = new().index_add_(0, at, rows) * float(np.float32(0.3)), new().index_add_(0, at, rows.abs()) * 0.3
    n = torch.bincount(at, minlength=V)[:, None]
    assert bool(((got.double() - want).abs() <= (2 * n + 8) * 2.0 ** -24 * size + 2.0 ** -130).all())
    assert torch.equal(heads.lookup_backward(dout, ids, V, 0.3), got)


def test_long_tables_pass_32_bits():
    """Rows that start beyond 2^32 bytes and 2^31 elements, and a gradient as large."""
    V, D = (1 << 23) + 3, 300
    ids = torch.tensor([0, V - 1, V - 1, 1 << 23, 7, -1], dtype=torch.int32, device="cuda")
    table = torch.zeros(V, D, dtype=BF16, device="cuda")
    for i in (0, V - 1, 1 << 23, 7):
        table[i] = i % 97 + 1
    rows = heads.lookup(table, ids)
    assert torch.equal(rows[:5], table[ids[:5].long()]) and not bool(rows[5].any())
    del table
    grad = heads.lookup_backward(rows, ids, V, out=torch.full((V, D), 3.0, device="cuda"))
    assert bool((grad[V - 1] == 2 * rows[1].float()).all()) and bool((grad[1 << 23] == rows[3].float()).all())
    assert int((grad != 0).any(1).sum()) == 4


def test_against_differences():
    """The gradient is that of the looked-up rows: linear, so a difference of any size is exact but for roundings."""
    g = gen(5)
    ids = ids_of(g, 300, 20, "masked")
    table, dout, way = rand(g, 20, 13), rand(g, 300, 13), rand(g, 20, 13)
    there, back = (heads.lookup(table + s * way, ids, 2.5).double() for s in (0.5, -0.5))
    slope = ((there - back) * dout.double()).sum()
    got = (heads.lookup_backward(dout, ids, 20, 2.5).double() * way.double()).sum()
    # 3,900 terms, each off by a few roundings of values of magnitude 10
    assert abs(float(got - slope)) < 3900 * 10 * 8 * 2.0 ** -24


def test_not_finite_values_stay_in_their_rows():
    ids = torch.arange(4, dtype=torch.int32, device="cuda").repeat(50)
    dout = torch.ones(200, 40, device="cuda")
    dout[5, 3], dout[10, 0] = float("nan"), float("inf")
    got = heads.lookup_backward(dout, ids, 4)
    assert bool(got[1, 3].isnan()) and bool(got[2, 0] == float("inf"))
    got[1, 3] = got[2, 0] = 50
    assert bool((got == 50).all())


@pytest.mark.parametrize("T", [3000, 40000])
def test_on_a_stream_and_from_a_graph(T):
    g = gen(8)
    V, D = 700, 40
    table, dout, ids = rand(g, V, D), rand(g, T, D), ids_of(g, T, V, "skewed")
    others = [(rand(g, V, D), rand(g, T, D), ids_of(g, T, V, how)) for how in ("masked", "one", "even")]

    def run():
        return heads.lookup(table, ids, 3.0), heads.lookup_backward(dout, ids, V, 3.0)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        there = run()
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(there, run()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for new in others:
        for old, x in zip((table, dout, ids), new):
            old.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(captured, run()))


def test_python_refusals():
    table, ids = torch.zeros(5, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    dout = torch.zeros(4, 8, device="cuda")
    for call in (lambda: heads.lookup(table, ids.long()), lambda: heads.lookup(table, ids[:, None]), lambda: heads.lookup(table[:0], ids),
                 lambda: heads.lookup(table.double(), ids), lambda: heads.lookup(table, ids, float("nan")),
                 lambda: heads.lookup(table, ids, out=table), lambda: heads.lookup(table.requires_grad_(), ids),
                 lambda: heads.lookup_backward(dout, ids[:3], 5), lambda: heads.lookup_backward(dout, ids, 0),
                 lambda: heads.lookup_backward(dout, ids, 5, out=dout)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("D", [1, 3, 48, 77, 1030])
def test_few_samples(D, dtype):
    """Up to 256 samples, on both sides of the choice between one launch and the sort: one row for
    all, runs, more columns than a workgroup's, tables of more rows than groups."""
    g = gen(D)
    for T in (15, 16, 17, 95, 96, 97, 255, 256):
        for V in (1, 2, 9, 130, 6000):
            for how in ("masked", "one", "sorted"):
                ids = ids_of(g, T, V, how)
                dout = rand(g, T, D).to(dtype)
                has = (ids >= 0) & (ids < V)
                dout[~has] = float("nan")
                got = heads.lookup_backward(dout, ids, V, 0.3, out=torch.full((V, D), 7.0, device="cuda"))
                at, rows = ids[has].long(), dout[has].double()
                want, size = (torch.zeros(V, D, dtype=torch.float64, device="cuda").index_add_(0, at, x) for x in (rows, rows.abs()))
                n = torch.bincount(at, minlength=V)[:, None]
                bound = (2 * n + 8) * 2.0 ** -24 * 0.3 * size + 2.0 ** -130
                assert bool(((got.double() - float(np.float32(0.3)) * want).abs() <= bound).all()), (T, V, how)
