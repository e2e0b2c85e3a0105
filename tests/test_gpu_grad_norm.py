"""The gradient norm and its clip factor against sums in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2609_34334_b200 import binding as hb
from train_ref import DT

pytestmark = pytest.mark.gpu
TOL = 2.0 ** -24 * 1.001   # one rounding to binary32; the binary64 sum is off by far less


@pytest.fixture(scope="module")
def comm():
    c = hb.Comm(2, 0)
    c.set_scratch(torch.full((hb.grad_norm_scratch_bytes(),), 255, dtype=torch.uint8, device="cuda"))   # NaN, were it read before it is written
    yield c
    c.destroy()


def norm(comm, xs, dtype, max_norm=1.0, **more):
    out = torch.full((4,), 7.0, device="cuda")
    comm.grad_norm(hb.Tensors(xs, dtype), out[1:3], max_norm=max_norm, **more)
    a = out.cpu().tolist()
    assert a[0] == a[3] == 7.0
    return a[1], a[2]


def check(got, xs, max_norm):
    want = math.sqrt(sum(float((x.double() ** 2).sum()) for x in xs))
    factor = min(1.0, max_norm / (want + 1e-6))
    assert abs(got[0] - want) <= TOL * want + 1e-45 and abs(got[1] - factor) <= TOL * factor, (got, want, factor)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("off", [0, 1, 3])
@pytest.mark.parametrize("counts", [[1], [0, 5, 0], [7, 8, 9, 15, 16, 17], [8192], [8193, 1, 100_001], [3_000_007], list(range(1, 65)), list(range(66)), [37] * 2500])
def test_formula(comm, dtype, off, counts):
    g = torch.Generator(device="cuda").manual_seed(len(counts))
    buf = torch.randn(sum(counts) + off + 8, generator=g, device="cuda").to(DT[dtype])
    xs, at = [], off
    for n in counts:
        xs.append(buf[at:at + n])
        at += n
    for max_norm in (1.0, 1e9, math.inf):
        check(norm(comm, xs, dtype, max_norm), xs, max_norm)
    assert norm(comm, xs, dtype) == norm(comm, xs, dtype)


# A tile is 16 KiB of one vector: 32 of them are summed in one launch, 33 in two; the empty vectors between fill no place of the tables of 64 and 1024.
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tiles", [1, 31, 32, 33])
def test_one_launch_and_two(comm, dtype, tiles):
    n = 16384 // torch.finfo(DT[dtype]).bits * 8
    x = torch.randn(tiles * n, generator=torch.Generator(device="cuda").manual_seed(tiles), device="cuda").to(DT[dtype])
    empty = x[:0]
    for xs in ([x], [x[i * n:(i + 1) * n] for i in range(tiles)], [v for i in range(tiles) for v in (empty, empty, empty, x[i * n:(i + 1) * n])] + [empty] * 1100):
        first = norm(comm, xs, dtype, 5.0)
        check(first, xs, 5.0)
        assert norm(comm, xs, dtype, 5.0) == first


@pytest.mark.parametrize("k", [64, 65, 1024, 1025, 2049])
def test_full_tables_with_empty_vectors(comm, k):
    x = torch.randn(k, 5, generator=torch.Generator(device="cuda").manual_seed(k), device="cuda")
    xs = [v for row in x for v in (row, row[:0])]
    check(norm(comm, xs, "fp32"), xs, 1.0)


def test_few_tiles_captured(comm):
    x = torch.randn(9, 4097, device="cuda")
    t, out = hb.Tensors(list(x), "fp32"), torch.zeros(2, device="cuda")
    comm.grad_norm(t, out, max_norm=3.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        comm.grad_norm(t, out, max_norm=3.0, stream=torch.cuda.current_stream())
    for k in range(3):
        x.mul_(1.5)
        graph.replay()
        check(out.cpu().tolist(), [x.cpu()], 3.0)


def test_no_vectors(comm):
    assert norm(comm, [], "fp32") == (0.0, 1.0)
    assert norm(comm, [torch.zeros(5, device="cuda")], "fp32") == (0.0, 1.0)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("at", [0, 4999, 70_000])
def test_not_finite(comm, bad, at):
    for dtype in ("fp32", "bf16"):
        x = torch.ones(70_001, dtype=DT[dtype], device="cuda")
        x[at] = bad
        n, f = norm(comm, [x], dtype)
        assert not math.isfinite(n) and math.isnan(f)


def test_squares_outside_binary32(comm):
    for x in (1e-30, 1e25):
        check(norm(comm, [torch.full((1000,), x, device="cuda")], "fp32"), [torch.full((1000,), x)], 1.0)


def test_captured_and_on_another_stream(comm):
    x = torch.randn(100_000, device="cuda")
    t, out, side = hb.Tensors([x[:70_000], x[70_000:]], "fp32"), torch.zeros(2, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        comm.grad_norm(t, out, max_norm=3.0, stream=side)
    for k in range(3):
        x.mul_(1.5)
        graph.replay()
        check(out.cpu().tolist(), [x.cpu()], 3.0)


def test_more_elements_than_32_bits_count(comm):
    n = (1 << 32) + 11
    x = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    x[0], x[1 << 31], x[n - 1] = 3.0, 4.0, 12.0
    assert norm(comm, [x], "bf16", 26.0) == (13.0, 1.0)


@pytest.mark.parametrize("max_norm", [1.0, 1e-6, 1e-7])
def test_no_vectors(comm, max_norm):
    """A norm of 0, and the factor that the formula gives for it."""
    check(norm(comm, [], "fp32", max_norm), [], max_norm)
