"""The router, its counts and its balance loss against the definitions in 64 bits, forward and backward."""
import math

import pytest
import torch

from paper_2609_34334_b200 import binding as hb
from train_ref import DT, HALF, U, losses, route, route_backward

pytestmark = pytest.mark.gpu
BAL, Z = 0.02, 0.003


def make(R, tokens, E, dtype, seed=0, pad=0.1, closed=0.1, ties=False, ld=None, off=0):
    g = torch.Generator().manual_seed(seed)
    ld = E if ld is None else ld
    out = []
    for t in tokens:
        x = torch.randn(t, E, generator=g) * 2
        if ties:
            x = x.round() * torch.where(torch.rand(t, E, generator=g) < 0.5, -1.0, 1.0)   # +0 and -0 among them
        x[torch.rand(t, E, generator=g) < closed] = -math.inf
        x[torch.rand(t, generator=g) < pad] = -math.inf
        flat = torch.full((off + max(t, 1) * ld,), math.nan, dtype=DT[dtype], device="cuda")
        v = flat[off:].view(max(t, 1), ld)[:t, :E]
        v.copy_(x.to(DT[dtype]))
        out.append(v)
    return out


class Call:
    def __init__(self, R, tokens, E, K, dtype, normalize, per_rank, x, ld=None):
        self.comm = hb.Comm(R, 0)
        n = hb.route_scratch_bytes(R, max(tokens), E)
        self.comm.set_scratch(torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda"))
        self.R, self.tokens, self.E, self.K, self.dtype, self.normalize, self.per_rank, self.x, self.ld = R, tokens, E, K, dtype, normalize, per_rank, x, ld
        self.groups = R if per_rank else 1
        self.indices = [torch.full((t + 1, K), -77, dtype=torch.int32, device="cuda") for t in tokens]
        self.weights = [torch.full((t + 1, K), -77.0, device="cuda") for t in tokens]
        self.counts = torch.full((R, E + 1), -77, dtype=torch.int32, device="cuda")
        self.loss = torch.full((self.groups * 2 + 1,), -77.0, device="cuda")
        self.saved = torch.full((self.groups * (E + 1) + 1,), -77.0, device="cuda")

    def forward(self, **more):
        self.comm.route(self.x, self.tokens, self.E, self.K, self.dtype, self.indices, self.weights, list(self.counts), self.loss, self.saved, balance_coef=BAL, z_coef=Z,
                        normalize=self.normalize, per_rank=self.per_rank, ld=self.ld, **more)
        return self

    def check(self):
        parts = []
        for r in range(self.R):
            x = self.x[r].cpu().double()
            i, w, p, lse, open_, rel = route(x, self.K, self.normalize)
            t = self.tokens[r]
            gi, gw = self.indices[r].cpu(), self.weights[r].cpu().double()
            assert torch.equal(gi[:t], i.to(torch.int32)) and (gi[t] == -77).all() and (gw[t] == -77).all()
            tol = (4 if self.normalize else 2) * rel.max(1, keepdim=True).values if t else 0.0
            assert ((gw[:t] - w).abs() <= tol * w + 1e-44).all()
            c = torch.bincount(i[i >= 0], minlength=self.E)
            assert torch.equal(self.counts[r, :self.E].cpu().long(), c) and int(self.counts[r, self.E]) == int(open_.sum())
            parts.append((p, lse, i, open_))
        for g in range(self.groups):
            here = parts[g:g + 1] if self.per_rank else parts
            loss, saved = losses(here, self.E, self.K, BAL, Z)
            got, sv = self.loss[2 * g:2 * g + 2].cpu().double(), self.saved[g * (self.E + 1):(g + 1) * (self.E + 1)].cpu().double()
            # sums of positive numbers: p's own error (below 200 u here), at most as many adds in a lane as the CTA has rows
            adds = max(64, sum(self.tokens) // 592 + 64) + 20
            assert ((got - loss).abs() <= (200 + adds) * U * loss.abs() + 1e-44).all(), (got, loss)
            assert ((sv - saved).abs() <= 2 * U * saved.abs()).all()
        assert self.loss[-1] == -77 and self.saved[-1] == -77
        return self


SHAPES = [(1, [1], 1, 1), (3, [300, 1, 77], 2, 2), (2, [70, 9], 9, 9), (8, [5] * 8, 32, 31), (2, [3, 5], 4, 2), (3, [17, 0, 40], 8, 8), (2, [100, 33], 16, 16), (4, [64, 1, 63, 65], 61, 3), (2, [257, 300], 64, 6), (2, [50, 20], 96, 4), (8, [40] * 8, 128, 8),
          (2, [100, 77], 256, 8), (1, [130], 257, 5), (2, [33, 30], 512, 32), (1, [19], 1000, 7), (2, [9, 8], 1024, 1), (64, [3] * 64, 60, 2), (2, [5000, 4000], 32, 2),
          (1, [4200], 8, 8), (1, [4200], 16, 3), (1, [4200], 61, 3), (2, [4000, 201], 64, 6), (1, [4200], 100, 8), (1, [4200], 30, 14), (1, [4200], 14, 8), (1, [4200], 128, 16), (1, [4200], 5, 1),
          (8, [100] * 8, 32, 4), (8, [60] * 8, 64, 2), (1, [5000], 128, 2), (1, [5000], 256, 2)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("R,tokens,E,K", SHAPES)
def test_forward(R, tokens, E, K, dtype):
    for normalize, per_rank in ((True, False), (False, True)):
        c = Call(R, tokens, E, K, dtype, normalize, per_rank, make(R, tokens, E, dtype, seed=E))
        c.forward().check()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("E", [6, 16, 61, 128, 256, 512])
def test_ties_go_to_the_lowest_expert(E, dtype):
    c = Call(2, [60, 50], E, min(E, 6), dtype, True, False, make(2, [60, 50], E, dtype, ties=True, closed=0.02))
    c.forward().check()
    same = [torch.zeros(9, E, dtype=DT[dtype], device="cuda")] * 2
    c = Call(2, [9, 9], E, min(E, 6), dtype, False, False, same).forward().check()
    assert (c.indices[0][:9].cpu() == torch.arange(min(E, 6))).all()


@pytest.mark.parametrize("E,ld,off", [(64, 72, 0), (64, 65, 0), (64, 64, 1), (61, 100, 3), (256, 1024, 8), (8, 9, 2)])
def test_strides_and_offsets(E, ld, off):
    for dtype in ("fp32", "bf16"):
        c = Call(2, [30, 41], E, 2, dtype, True, False, make(2, [30, 41], E, dtype, ld=ld, off=off), ld=ld)
        c.forward().check()


def test_nothing_open_anywhere():
    x = [torch.full((20, 16), -math.inf, device="cuda") for _ in range(2)]
    for per_rank in (False, True):
        c = Call(2, [20, 20], 16, 2, "fp32", True, per_rank, x).forward().check()
        assert not c.loss[:-1].any() and not c.saved[:-1].any()
    c = Call(2, [0, 0], 16, 2, "fp32", True, False, [None, None])
    c.indices = c.weights = [None, None]
    c.comm.route(c.x, c.tokens, 16, 2, "fp32", c.indices, c.weights, list(c.counts), c.loss, c.saved)
    assert not c.counts.any() and not c.loss[:-1].any() and not c.saved[:-1].any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("E", [8, 61, 256])
def test_the_lowest_number_is_a_logit(E, dtype):
    """Rows and entries masked with the type's lowest number, not with -infinity."""
    low = torch.finfo(DT[dtype]).min
    x = torch.randn(6, E, device="cuda").to(DT[dtype])
    x[0] = low
    x[1, 1:] = low
    x[2, ::2] = low
    c = Call(1, [6], E, 3, dtype, False, False, [x])
    c.comm.route(c.x, c.tokens, E, 3, dtype, c.indices, c.weights, list(c.counts), c.loss, c.saved, balance_coef=BAL, z_coef=0.0, normalize=False)
    i, w, p, _, _, rel = route(x.cpu().double(), 3, False)
    assert torch.equal(c.indices[0][:6].cpu().long(), i) and int(c.counts[0, E]) == 6
    # the bound of each weight's own distance from the row's largest; below the least normal number it is 0
    assert ((c.weights[0][:6].cpu().double() - w).abs() <= 2 * torch.gather(rel, 1, i) * w + 2.0 ** -126).all()
    assert float(c.loss[1]) == 0.0 and math.isfinite(float(c.loss[0]))
    out = [torch.zeros(7, E, dtype=DT[dtype], device="cuda")]
    backward(c, [torch.ones(7, 3, device="cuda")], None, out)
    assert out[0].isfinite().all()


def test_small_grids_captured_and_repeated():
    """The form that ends inside one cluster: captured, replayed on new logits, and the same bits as an eager call; one communicator for several shapes."""
    comm = hb.Comm(8, 0)
    n = max(hb.route_scratch_bytes(8, 64, E) for E in (8, 64, 256, 1024))
    scratch = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    comm.set_scratch(scratch)
    side = torch.cuda.Stream()
    for E, K, T in ((8, 2, 5), (64, 6, 16), (256, 8, 1), (1024, 32, 3), (64, 6, 64), (64, 6, 0)):
        calls = []
        for _ in range(2):
            c = Call(8, [T] * 8, E, K, "bf16", True, False, None)
            c.comm = comm
            c.x = make(8, [max(T, 1)] * 8, E, "bf16")
            calls.append(c)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls[0].forward(stream=side)
        for _ in range(3):
            for a, b in zip(calls[0].x, calls[1].x):
                a.add_(torch.randn_like(a))
                b.copy_(a)
            graph.replay()
            calls[1].forward()
            torch.cuda.synchronize()
            for name in ("counts", "loss", "saved"):
                assert torch.equal(getattr(calls[0], name), getattr(calls[1], name)), (E, name)
            for name in ("indices", "weights"):
                assert all(torch.equal(a, b) for a, b in zip(getattr(calls[0], name), getattr(calls[1], name))), (E, name)
    comm.destroy()


@pytest.mark.parametrize("E", [8, 61, 256])
def test_nan_is_not_chosen_and_shows(E):
    x = make(1, [40], E, "fp32", pad=0, closed=0)
    x[0][7, 3] = math.nan
    x[0][9, :] = math.nan
    c = Call(1, [40], E, 3, "fp32", True, False, x).forward()
    i, w = c.indices[0].cpu(), c.weights[0].cpu()
    assert 3 not in i[7].tolist() and (i[7] >= 0).all() and w[7].isnan().all()
    assert (i[9] == -1).all() and (w[9] == 0).all()
    assert c.loss[:2].isnan().all() or c.loss[0].isnan()
    assert int(c.counts[0, E]) == 39
    keep = [k for k in range(40) if k not in (7, 9)]
    assert w[keep].isfinite().all()
    x = make(1, [4], E, "fp32", pad=0, closed=0)
    x[0][1, 2] = math.inf
    c = Call(1, [4], E, 3, "fp32", True, False, x).forward()
    assert c.indices[0][1, 0] == 2 and c.weights[0][1].isnan().all() and c.loss[0].isnan()


def test_far_apart_and_large_logits():
    for scale in (1e3, 3e37):
        x = [t * scale for t in make(1, [50], 64, "fp32", pad=0, closed=0)]
        c = Call(1, [50], 64, 4, "fp32", False, False, x).forward()
        i, w, p, *_ = route(x[0].cpu().double(), 4, False)
        assert torch.equal(c.indices[0][:50].cpu().long(), i) and c.weights[0][:50].isfinite().all()
        assert ((c.weights[0][:50].cpu().double() - w).abs() < 1e-3).all()   # a gap of 90 and more leaves nothing: the rest is below 1e-38 or the gap's rounding


def test_the_same_call_gives_the_same_bits_also_captured():
    x = make(4, [3000, 2900, 3100, 2000], 128, "bf16")
    c = Call(4, [3000, 2900, 3100, 2000], 128, 8, "bf16", True, False, x).forward().check()
    first = [t.clone() for t in (*c.indices, *c.weights, c.counts, c.loss, c.saved)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.forward(stream=side)
    for _ in range(3):
        for t in (c.counts, c.loss, c.saved):
            t.fill_(-77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (*c.indices, *c.weights, c.counts, c.loss, c.saved)))


# ------------------------------------------------------------------------------------------------ backward


def backward(c, dweights, dloss, dlogits, **more):
    c.comm.route_backward(c.x, c.tokens, c.E, c.K, c.dtype, c.indices if dweights is not None else None, c.saved, dweights, dloss, dlogits, normalize=c.normalize,
                          per_rank=c.per_rank, ld=c.ld, **more)


def check_backward(c, dweights, dloss, got, x=None):
    saved = c.saved[:-1].view(c.groups, c.E + 1).cpu().double()
    for r in range(c.R):
        t = c.tokens[r]
        g = r if c.per_rank else 0
        dw = None if dweights is None else dweights[r][:t].cpu().double()
        want, tol = route_backward((c.x if x is None else x)[r][:t].cpu().double(), c.indices[r][:t].cpu(), saved[g], dw, 1.0 if dloss is None else float(dloss[g]), c.normalize)
        have = got[r][:t].cpu().double()
        rounding = HALF[c.dtype] * want.abs() * 1.01 + (1e-40 if c.dtype == "bf16" else 0.0)
        assert ((have - want).abs() <= tol + rounding).all(), (r, (have - want).abs().max())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("R,tokens,E,K", SHAPES)
def test_backward(R, tokens, E, K, dtype):
    for normalize, per_rank in ((True, False), (False, True)):
        c = Call(R, tokens, E, K, dtype, normalize, per_rank, make(R, tokens, E, dtype, seed=E)).forward()
        g = torch.Generator(device="cuda").manual_seed(1)
        dw = [torch.randn(t + 1, K, generator=g, device="cuda") * 1e-2 for t in tokens]
        dloss = torch.randn(c.groups, generator=g, device="cuda")
        out = [torch.full((t + 1, E), 5.0, dtype=DT[dtype], device="cuda") for t in tokens]
        for a, b in ((dw, dloss), (None, dloss), (dw, None)):
            backward(c, a, b, out)
            check_backward(c, a, b, out)
        assert all((o[-1] == 5).all() for o in out)


@pytest.mark.parametrize("normalize", [True, False])
def test_gradients_beside_no_choice_are_not_read(normalize):
    """Rows of padding and rows with fewer open experts than choices: what lies in dweights beside -1 may be anything."""
    E, K, T = 16, 4, 30
    x = make(1, [T], E, "fp32", pad=0.3, closed=0.8)
    c = Call(1, [T], E, K, "fp32", normalize, False, x).forward()
    dw = torch.randn(T, K, device="cuda")
    none = c.indices[0][:T] < 0
    assert none.any() and not none.all()
    bad = torch.where(none, math.nan, dw)
    out = [torch.zeros(T, E, device="cuda")]
    backward(c, [bad], None, out)
    check_backward(c, [torch.where(none, 0.0, dw)], None, out)
    closed = (x[0] == -math.inf).all(1)
    assert closed.any() and not out[0][closed].any()


@pytest.mark.parametrize("E,ld,dld,off", [(64, 72, 80, 0), (64, 65, 64, 0), (61, 100, 61, 3), (256, 256, 264, 0), (8, 9, 11, 2)])
def test_backward_strides(E, ld, dld, off):
    for dtype in ("fp32", "bf16"):
        c = Call(2, [30, 41], E, 2, dtype, True, False, make(2, [30, 41], E, dtype, ld=ld, off=off), ld=ld).forward()
        dw = [torch.randn(t, 2, device="cuda") for t in c.tokens]
        wide = [torch.full((t, dld), 5.0, dtype=DT[dtype], device="cuda") for t in c.tokens]
        backward(c, dw, None, wide, dld=dld)
        check_backward(c, dw, None, [o[:, :E] for o in wide])
        assert all((o[:, E:] == 5).all() for o in wide)


@pytest.mark.parametrize("E", [16, 61, 256])
def test_backward_in_place(E):
    for dtype in ("fp32", "bf16"):
        c = Call(2, [200, 100], E, 4, dtype, False, False, make(2, [200, 100], E, dtype)).forward()
        dw = [torch.randn(t, 4, device="cuda") for t in c.tokens]
        before = [x.clone() for x in c.x]
        backward(c, dw, None, c.x)
        check_backward(c, dw, None, c.x, before)


def test_backward_with_indices_of_the_callers_own():
    """Any indices may come: beyond the experts they are ignored, twice in a row they count twice."""
    E, K = 64, 4
    c = Call(1, [3], E, K, "fp32", False, False, make(1, [3], E, "fp32", pad=0, closed=0)).forward()
    c.indices[0][:3] = torch.tensor([[5, 5, 9, 9], [-1, 64, 1 << 30, 7], [-5, -1, -1, -1]], dtype=torch.int32, device="cuda")
    for c.normalize in (False, True):
        dw, out = [torch.randn(3, K, device="cuda")], [torch.zeros(3, E, device="cuda")]
        backward(c, dw, None, out)
        check_backward(c, dw, None, out)


@pytest.mark.parametrize("normalize", [True, False])
def test_gradient_against_differences(normalize):
    """Central differences of the 64-bit loss, f held fixed; the selection does not change within the step."""
    E, K, T = 12, 3, 6
    x = make(1, [T], E, "fp32", pad=0, closed=0.1)
    c = Call(1, [T], E, K, "fp32", normalize, False, x).forward()
    dw = [torch.randn(T, K, device="cuda")]
    out = [torch.zeros(T, E, device="cuda")]
    backward(c, dw, None, out)
    base = x[0].cpu().double()
    i0, _, _, _, open0, _ = route(base, K, normalize)
    counts = torch.bincount(i0[i0 >= 0], minlength=E).double()

    def value(y):
        i, w, p, lse, _, _ = route(y, K, normalize)
        assert torch.equal(i, i0)
        return float(BAL * E * (counts / (K * T) * p.sum(0) / T).sum() + Z * (lse ** 2).sum() / T + (w * dw[0].cpu().double()).sum())
    h = 1e-5
    for t in range(T):
        for e in range(E):
            if base[t, e] == -math.inf:
                assert out[0][t, e] == 0
                continue
            up, down = base.clone(), base.clone()
            up[t, e] += h
            down[t, e] -= h
            # the third derivative of these sums of softmax terms is below 10 of their size: h^2 of it, and 1e-16 / h of rounding; binary32 of the kernel
            assert abs((value(up) - value(down)) / (2 * h) - float(out[0][t, e])) < 1e-5 * (1 + float(dw[0].abs().max()))


def test_rows_far_apart():
    """Offsets beyond 32 bits between the rows."""
    ld, T, E = 1 << 20, 4200, 64
    flat = torch.zeros(T * ld, dtype=torch.bfloat16, device="cuda")
    x = flat.view(T, ld)[:, :E]
    x.copy_(torch.randn(T, E, generator=torch.Generator().manual_seed(2)).bfloat16())
    c = Call(1, [T], E, 4, "bf16", True, False, [x], ld=ld).forward().check()
    dw = [torch.randn(T, 4, device="cuda")]
    before = [x.clone()]
    backward(c, dw, None, [x], dld=ld)
    check_backward(c, dw, None, [x], before)


# ------------------------------------------------------------------------------------------------ what a row's neighbours must not change


def distinct_rows(T, E, seed=0):
    """Rows without equal logits."""
    x = torch.randn(T, E, generator=torch.Generator().manual_seed(seed)).cuda()
    assert all(r.unique().numel() == E for r in x[:50])
    return x


@pytest.mark.parametrize("E,K", [(32, 4), (61, 4), (64, 8), (128, 8)])
def test_weights_do_not_depend_on_neighbours_or_the_grid(E, K):
    """The normalised weights of a row have the same bits beside rows with equal logits, in another place, and in a call of few rows, which lays a row over
    other lanes: the chosen are added in the order of their ranks."""
    T = 5000   # beyond the lines to one cluster and to many rows: several rows share a warp
    x = distinct_rows(T, E)
    want = Call(1, [T], E, K, "fp32", True, False, [x]).forward()
    w, i = want.weights[0][:T], want.indices[0][:T]
    tied = x.clone()
    tied[1::2] = 1.0
    got = Call(1, [T], E, K, "fp32", True, False, [tied]).forward()
    assert torch.equal(got.weights[0][:T:2], w[::2]) and torch.equal(got.indices[0][:T:2], i[::2])
    order = torch.randperm(T, generator=torch.Generator().manual_seed(1)).cuda()
    got = Call(1, [T], E, K, "fp32", True, False, [x[order].contiguous()]).forward()
    assert torch.equal(got.weights[0][:T], w[order]) and torch.equal(got.indices[0][:T], i[order])
    for at in (0, 16, 2000):
        got = Call(1, [16], E, K, "fp32", True, False, [x[at:at + 16]]).forward()
        assert torch.equal(got.weights[0][:16], w[at:at + 16]) and torch.equal(got.indices[0][:16], i[at:at + 16])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("E,K", [(32, 4), (64, 8), (61, 6), (128, 12), (256, 8), (512, 32), (1024, 32)])
def test_rows_of_many_equal_logits(E, K, dtype):
    """All alike; alike but for a few above, below or closed; two or three values; next to rows without equal ones; in one cluster and in many CTAs."""
    for T in (24, 4500 if E <= 256 else 600):
        g = torch.Generator().manual_seed(E + T)
        x = torch.randn(T, E, generator=g)
        x[0::6] = 0.0
        x[1::6] = torch.randint(0, 2, (len(x[1::6]), E), generator=g).float() * 0.5
        x[2::6] = torch.randint(-1, 2, (len(x[2::6]), E), generator=g).float()
        few = torch.rand(len(x[3::6]), E, generator=g)
        x[3::6] = torch.where(few < 0.02, few * 50, torch.where(few > 0.98, -1.0, -0.0))
        x[4::6] = torch.where(torch.rand(len(x[4::6]), E, generator=g) < 0.7, -math.inf, 2.0)
        c = Call(1, [T], E, K, dtype, True, False, [x.cuda().to(DT[dtype])])
        c.forward().check()


def per_call_us(c, reps=5):
    for _ in range(2):
        c.forward()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(reps):
        c.forward()
    e1.record()
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) * 1e3 / reps


@pytest.mark.parametrize("E,K,times", [(64, 4, 6), (256, 8, 6), (1024, 32, 8)])
def test_equal_logits_are_not_far_slower(E, K, times):
    """A router that starts from zeros, rows of padding that are not masked: such a row's choice takes topk searches of what a lane holds (E / 32 logits or
    so) and a maximum over the lanes, where another row's takes two maxima: a small multiple, not a number that grows with the square of the experts."""
    T = 32_000
    x = torch.randn(T, E, device="cuda")
    usual = per_call_us(Call(1, [T], E, K, "fp32", True, False, [x]))
    alike = per_call_us(Call(1, [T], E, K, "fp32", True, False, [torch.zeros_like(x)]))
    print("%d experts, topk %d: %.1f us, all alike %.1f us" % (E, K, usual, alike))
    assert alike < times * usual


@pytest.mark.parametrize("T", [4, 5000])
@pytest.mark.parametrize("E", [8, 61, 256])
@pytest.mark.parametrize("row", ["one", "all", "rest closed"])
def test_a_nan_reaches_both_losses(row, E, T):
    """One row of a call alone: a NaN among numbers, nothing but NaN, NaN with the rest closed (the last two choose nothing and count nowhere)."""
    x = torch.randn(T, E, device="cuda")
    if row == "rest closed":
        x[1] = -math.inf
    x[1, 3 if row != "all" else slice(None)] = math.nan
    c = Call(1, [T], E, 3, "fp32", True, False, [x]).forward()
    assert c.loss[0].isnan() and c.loss[1].isnan()
    assert int(c.counts[0, E]) == (T if row == "one" else T - 1)
    assert c.saved[:E + 1].isfinite().all()
    out = [torch.zeros(T, E, device="cuda")]
    backward(c, [torch.ones(T, 3, device="cuda")], None, out)
    assert out[0][1].isnan().all() and out[0][0].isfinite().all() and out[0][2:].isfinite().all()
    c = Call(1, [1], E, 3, "fp32", True, False, [x[1:2]]).forward()   # and as the only row
    assert c.loss[0].isnan() and c.loss[1].isnan() and c.saved[:E + 1].isfinite().all()
    c.comm.route(c.x, c.tokens, E, 3, "fp32", c.indices, c.weights, list(c.counts), c.loss, c.saved, balance_coef=BAL, z_coef=0.0)
    assert c.loss[0].isnan() and float(c.loss[1]) == 0.0
