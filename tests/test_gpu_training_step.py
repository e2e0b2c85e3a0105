"""The operators of a training step together with the collectives that they stand between, as a program runs them."""
import pytest
import torch

from paper_2609_34334_b200 import binding as hb

pytestmark = pytest.mark.gpu


def communicator(R, n, dtype="fp32", tokens=0, experts=1):
    c = hb.Comm(R, 0)
    nbytes = max(hb.scratch_bytes_direct(R, n, dtype), hb.grad_norm_scratch_bytes(), hb.route_scratch_bytes(R, tokens, experts) if tokens else 0)
    c.keep = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
    c.set_scratch(c.keep, nbytes)
    return c


class Shards:
    def __init__(self, R, q, state, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.R, self.q, self.state = R, q, state
        start = torch.randn(R * q, generator=g, device="cuda")
        self.grads = [torch.randn(R * q, generator=g, device="cuda") for _ in range(R)]
        self.params = [start.clone() for _ in range(R)]
        self.own = [self.params[r][r * q:(r + 1) * q] for r in range(R)]
        self.sums = [torch.zeros(q, device="cuda") for _ in range(R)]
        dt = torch.float32 if state == "fp32" else torch.float8_e4m3fn
        self.m, self.v = ([torch.zeros(q, dtype=dt, device="cuda") for _ in range(R)] for _ in range(2))
        self.ms, self.vs = ([torch.zeros(-(-q // 256), device="cuda") for _ in range(R)] for _ in range(2))
        self.norm = torch.zeros(2, device="cuda")

    def table(self):
        return hb.AdamTensors(self.own, self.sums, self.m, self.v, "fp32", "fp32", state=self.state, exp_avg_scale=self.ms, exp_avg_sq_scale=self.vs, weight_decay=0.1)

    def all(self):
        return [t.view(torch.uint8) for t in (*self.params, *self.m, *self.v, *self.ms, *self.vs)]


@pytest.mark.parametrize("state", ["fp32", "8bit"])
@pytest.mark.parametrize("R,q", [(2, 4096), (5, 1003), (8, 20_000)])
def test_sharded_step_equals_its_parts(R, q, state):
    """Binary32 gradients: the reduce-scatter rounds where the sharded kernel adds, so the bits are the same, step after step."""
    comm = communicator(R, R * q)
    a, b = Shards(R, q, state), Shards(R, q, state)
    table, sums = b.table(), hb.Tensors(b.sums, "fp32")
    for k in range(3):
        comm.sharded_adamw(a.grads, a.params, a.m, a.v, R * q, "fp32", "fp32", 1e-2, k + 1, state=state, exp_avg_scale=a.ms, exp_avg_sq_scale=a.vs, weight_decay=0.1,
                           grad_scale=1.0 / R, seed=k)
        comm.reduce_scatter(b.grads, b.sums, q, "fp32")
        comm.grad_norm(sums, b.norm, max_norm=1e9)
        comm.adamw(table, 1e-2, k + 1, grad_scale=1.0 / R, factor=b.norm[1:], seed=k)
        comm.allgather(b.own, b.params, q, "fp32")
        assert all(torch.equal(x, y) for x, y in zip(a.all(), b.all())), k
    assert float(b.norm[1]) == 1.0
    comm.destroy()


@pytest.mark.parametrize("path", [hb.PATH_CE, hb.PATH_SM])
def test_clipped_step_skips_what_is_not_finite(path):
    R, q = 4, 3000
    comm = communicator(R, R * q)
    comm.set_path(path)
    s = Shards(R, q, "fp32")
    table, sums = s.table(), hb.Tensors(s.sums, "fp32")

    def run():
        comm.reduce_scatter(s.grads, s.sums, q, "fp32")
        comm.grad_norm(sums, s.norm, max_norm=0.5)
        comm.adamw(table, 1e-2, 1, factor=s.norm[1:])
        comm.allgather(s.own, s.params, q, "fp32")
    before = [t.clone() for t in s.all()]
    good = s.grads[2][17].clone()
    s.grads[2][17] = float("inf")
    run()
    assert all(torch.equal(x, y) for x, y in zip(before, s.all()))
    s.grads[2][17] = good
    run()
    total = sum(g.double() for g in s.grads)
    n = float(total.norm())
    assert abs(float(s.norm[0]) / n - 1) < 1e-6 and abs(float(s.norm[1]) / (0.5 / n) - 1) < 1e-5
    m = torch.cat(s.m).double()
    want = 0.1 * total * (0.5 / n)   # first step from zero: (1 - beta1) * clipped gradient; 4 adds and 6 roundings of binary32
    assert ((m - want).abs() <= 12 * 2.0 ** -24 * 0.1 * (0.5 / n) * sum(g.double().abs() for g in s.grads)).all()
    comm.destroy()


def test_two_captured_steps_share_a_communicator():
    """Two graphs that use the same scratch, replayed in turn on one stream, against eager calls."""
    R, q, T, E, K = 4, 2500, 300, 48, 3
    comm = communicator(R, R * q, tokens=T, experts=E)
    a, b = Shards(R, q, "fp32"), Shards(R, q, "fp32")
    x = [torch.randn(T, E, device="cuda") for _ in range(R)]
    out = [dict(indices=[torch.zeros(T, K, dtype=torch.int32, device="cuda") for _ in range(R)], weights=[torch.zeros(T, K, device="cuda") for _ in range(R)],
                counts=torch.zeros(R, E + 1, dtype=torch.int32, device="cuda"), loss=torch.zeros(2, device="cuda"), saved=torch.zeros(E + 1, device="cuda"),
                dlogits=[torch.zeros(T, E, device="cuda") for _ in range(R)]) for _ in range(2)]
    tables, sums = [s.table() for s in (a, b)], [hb.Tensors(s.sums, "fp32") for s in (a, b)]
    side = torch.cuda.Stream()

    def optimizer(k, stream):
        s = (a, b)[k]
        comm.grad_norm(sums[k], s.norm, max_norm=0.5, stream=stream)
        comm.adamw(tables[k], 1e-2, 1, factor=s.norm[1:], stream=stream)

    def layer(k, stream):
        o = out[k]
        comm.route(x, [T] * R, E, K, "fp32", o["indices"], o["weights"], list(o["counts"]), o["loss"], o["saved"], z_coef=1e-3, stream=stream)
        comm.route_backward(x, [T] * R, E, K, "fp32", o["indices"], o["saved"], o["weights"], None, o["dlogits"], stream=stream)
    for s in (a, b):
        for k, t in enumerate(s.sums):
            t.copy_(s.grads[0][k * q:(k + 1) * q])
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph, fn in zip(graphs, (optimizer, layer)):
        with torch.cuda.graph(graph, stream=side):
            fn(0, side)
    for _ in range(3):
        for k in range(R):
            x[k].mul_(1.1)
        for graph in graphs:
            graph.replay()
        optimizer(1, None)
        layer(1, None)
        torch.cuda.synchronize()
        assert all(torch.equal(p, r) for p, r in zip(a.all(), b.all()))
        for name in ("counts", "loss", "saved"):
            assert torch.equal(out[0][name], out[1][name]), name
        for name in ("indices", "weights", "dlogits"):
            assert all(torch.equal(p, r) for p, r in zip(out[0][name], out[1][name])), name
    comm.destroy()


@pytest.mark.parametrize("E,K", [(8, 1), (64, 2)])
def test_routed_tokens_through_the_exchange(E, K):
    """Router, exchange with its counts, a stand-in for the experts, exchange back, weights, and the gradient of it all in torch's autograd."""
    R, T, width = 4, [200, 150, 0, 333], 64
    comm = communicator(R, 16, tokens=max(T), experts=E)
    x = [torch.randn(t, E, device="cuda") for t in T]
    rows = [torch.randn(t, width, device="cuda") for t in T]
    indices = [torch.zeros(t, K, dtype=torch.int32, device="cuda") for t in T]
    weights = [torch.zeros(t, K, device="cuda") for t in T]
    counts, loss, saved = torch.zeros(R, E + 1, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(E + 1, device="cuda")
    comm.route(x, T, E, K, "fp32", indices, weights, list(counts), loss, saved, balance_coef=0.01, z_coef=1e-3)
    c = counts[:, :E].view(R, R, E // R).sum(2).cpu().tolist()
    order = [torch.argsort(i.view(-1), stable=True) for i in indices]
    send = [rows[r].repeat_interleave(K, 0)[order[r]].contiguous() for r in range(R)]
    sendcounts = [c[u][v] * width for u in range(R) for v in range(R)]
    sdispls = [sum(c[u][:v]) * width for u in range(R) for v in range(R)]
    rdispls = [sum(c[a][v] for a in range(u)) * width for v in range(R) for u in range(R)]
    recv = [torch.zeros(max(1, sum(c[u][v] for u in range(R))) * width, device="cuda") for v in range(R)]
    room = lambda ts: [t if t.numel() else torch.zeros(1, device="cuda") for t in ts]  # noqa: E731
    comm.alltoallv(room(send), sendcounts, sdispls, recv, rdispls, "fp32")
    done = [t * 2.0 for t in recv]
    back = [torch.zeros_like(t) for t in send]
    flip = lambda a: [a[v * R + u] for u in range(R) for v in range(R)]  # noqa: E731
    comm.alltoallv(done, flip(sendcounts), rdispls, room(back), sdispls, "fp32")
    dy = [torch.randn(t, width, device="cuda") for t in T]
    dweights, dlogits = [], [torch.zeros_like(t) for t in x]
    for r in range(R):
        y = torch.empty_like(back[r])
        y[order[r]] = back[r]
        assert torch.equal(y, (rows[r] * 2.0).repeat_interleave(K, 0))
        dweights.append((y.view(T[r], K, width) * dy[r][:, None]).sum(2).contiguous())
    comm.route_backward(x, T, E, K, "fp32", indices, saved, dweights, None, dlogits)
    # the same in 64 bits by autograd
    leaves = [t.double().requires_grad_() for t in x]
    n = sum(T)
    f = sum(torch.bincount(i.view(-1).long(), minlength=E) for i in indices).double() / (K * n)
    p = torch.softmax(torch.cat(leaves), 1)
    total = 0.01 * E * (f * p.sum(0) / n).sum() + 1e-3 * (torch.logsumexp(torch.cat(leaves), 1) ** 2).sum() / n
    for r in range(R):
        w = torch.gather(torch.softmax(leaves[r], 1), 1, indices[r].long())
        w = w / w.sum(1, keepdim=True)
        total = total + (w[:, :, None] * (rows[r].double() * 2.0)[:, None] * dy[r].double()[:, None]).sum()
    total.backward()
    for r in range(R):
        if T[r]:
            g = leaves[r].grad
            # dweights: a sum of 64 products in binary32; then products of numbers off by less than 100 u, twice
            size = 1e-6 + (dweights[r].abs().max() + 2 * width * 2.0 ** -24 * 64 * 16)
            assert ((dlogits[r].double() - g).abs() <= 300 * 2.0 ** -24 * size).all()
    comm.destroy()


def test_operators_beside_handshake_mode():
    """In handshake mode collectives go through the proxy, the operators into the caller's stream; the order on the stream holds."""
    R, q = 2, 4096
    comm = communicator(R, R * q)
    comm.set_path(hb.PATH_SM)
    comm.set_param("handshake", 1)
    a, b = Shards(R, q, "fp32"), Shards(R, q, "fp32")
    table, plain = b.table(), communicator(R, R * q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for k in range(5):
        plain.sharded_adamw(a.grads, a.params, a.m, a.v, R * q, "fp32", "fp32", 1e-2, k + 1, weight_decay=0.1)
        comm.reduce_scatter(b.grads, b.sums, q, "fp32", side)
        comm.adamw(table, 1e-2, k + 1, stream=side)
        comm.allgather(b.own, b.params, q, "fp32", side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.all()[:3 * R], b.all()[:3 * R]))
    assert comm.async_error() == hb.OK
    comm.destroy()
    plain.destroy()


def test_the_current_device_and_stream_stay():
    comm = communicator(2, 1000)
    s = Shards(2, 500, "fp32")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        comm.adamw(s.table(), 1e-2, 1)
        assert torch.cuda.current_stream() == side and torch.cuda.current_device() == 0
    torch.cuda.synchronize()
    comm.destroy()


@pytest.mark.parametrize("R,limit", [(4, 0.5), (8, 3.0), (3, 1e3)])
def test_the_clipped_step_of_a_mean(R, limit):
    """Gradients that are a mean over the ranks (grad_scale 1 / R): the norm is that of the sums as they lie in memory, so clipping the mean to `limit` takes a max_norm of
    limit * R."""
    q = 3000
    comm = communicator(R, R * q)
    s = Shards(R, q, "fp32", seed=R)
    table, sums = s.table(), hb.Tensors(s.sums, "fp32")
    comm.reduce_scatter(s.grads, s.sums, q, "fp32")
    comm.grad_norm(sums, s.norm, max_norm=limit * R)
    comm.adamw(table, 1e-2, 1, grad_scale=1.0 / R, factor=s.norm[1:])
    torch.cuda.synchronize()
    mean = sum(g.double() for g in s.grads) / R
    n = float(mean.norm())
    clipped = mean * min(1.0, limit / n)
    # (1 - beta1) * clipped: up to 8 adds of the sum, the factor's own rounding and 6 more of binary32; 1e-6 / (R n) of the factor's guard
    tol = (16 * 2.0 ** -24 + 1e-6 / (R * n)) * 0.1 * min(1.0, limit / n) * sum(g.double().abs() for g in s.grads) / R
    assert ((torch.cat(s.m).double() - 0.1 * clipped).abs() <= tol).all()
    assert (n > limit) == (limit < 1e3)
    comm.destroy()


def test_the_sweep_clips_the_mean(monkeypatch, capsys):
    """The step command's clipped form: what it clips to, after the mean's scale, is a norm of 1."""
    from types import SimpleNamespace

    from paper_2609_34334_b200 import sweep

    clips, scales = [], []
    norm, adamw = hb.Comm.grad_norm, hb.Comm.adamw

    def seen_norm(self, grads, out, max_norm=float("inf"), stream=None):
        clips.append(max_norm)
        return norm(self, grads, out, max_norm=max_norm, stream=stream)

    def seen_adamw(self, tensors, lr, step, **more):
        scales.append(more["grad_scale"])
        return adamw(self, tensors, lr, step, **more)

    monkeypatch.setattr(hb.Comm, "grad_norm", seen_norm)
    monkeypatch.setattr(hb.Comm, "adamw", seen_adamw)
    sweep.step(SimpleNamespace(buckets=1))
    assert len(clips) == len(scales) > 0
    assert all(abs(c * s - 1.0) < 1e-12 for c, s in zip(clips, scales)), (clips[0], scales[0])
    assert '"delivered_bit_exact": true' in capsys.readouterr().out
