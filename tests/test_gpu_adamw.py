"""AdamW over many tensors and on sharded ranks against the formulas in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2609_34334_b200 import binding as hb
from paper_2609_34334_b200 import diag as hd
from train_ref import BLOCK, DT, HALF, adamw, check_codes, decode, words

pytestmark = pytest.mark.gpu
B1, B2, EPS = 0.9, 0.95, 1e-8
KINDS = [("fp32", False), ("bf16", False), ("bf16", True)]
FORMS = [(p, w, g, s) for p, w in KINDS for g in ("fp32", "bf16") for s in ("fp32", "8bit")]


@pytest.fixture(scope="module")
def comm():
    c = hb.Comm(4, 0)
    yield c
    c.destroy()


class Set:
    """Tensors packed into one buffer for each array, `gap` elements between them and in front (their distance from an aligned place), filled with
    a pattern that must survive."""

    def __init__(self, counts, param, master, grad, state, gap=0, seed=0, first=False):
        g = torch.Generator().manual_seed(seed)
        self.counts, self.param, self.master, self.grad, self.state, self.seed = counts, param, master, grad, state, seed
        self.offsets, at = [], gap
        for n in counts:
            self.offsets.append(at)
            at += n + gap if gap else (n + 63) // 64 * 64
        self.total = at + 64
        z = lambda s: torch.randn(self.total, generator=g) * s  # noqa: E731
        self.cpu = {"p": z(0.02).to(DT[param]), "g": z(1e-2).to(DT[grad])}
        if master:
            self.cpu["w"] = self.cpu["p"].float() + z(1e-5)
        m, v = (torch.zeros(self.total), torch.zeros(self.total)) if first else (z(2e-3), z(1e-2) ** 2 + 1e-9)
        if state == "fp32":
            self.cpu["m"], self.cpu["v"] = m, v
        else:
            per = [(n + BLOCK - 1) // BLOCK for n in counts]
            self.sat = [sum(per[:k]) + 3 * k for k in range(len(per))]      # three floats between the tensors' scales
            self.per = per
            for k in "mv":
                self.cpu[k] = (z(60.0).clamp(-448, 448) * (0 if first else 1)).to(torch.float8_e4m3fn)
                self.cpu[k + "s"] = torch.rand(sum(per) + 3 * len(per) + 3, generator=g) * 1e-4 + 1e-6
            self.cpu["v"] = self.cpu["v"].float().abs().to(torch.float8_e4m3fn)
        self.dev = {k: t.cuda() for k, t in self.cpu.items()}

    def views(self, k, src=None):
        src = self.dev if src is None else src
        if k not in src:
            return None
        if k.endswith("s"):
            return [src[k][a:a + n] for a, n in zip(self.sat, self.per)]
        return [src[k][o:o + n] for o, n in zip(self.offsets, self.counts)]

    def table(self, decay=0.0):
        v = self.views
        return hb.AdamTensors(v("p"), v("g"), v("m"), v("v"), self.param, self.grad, state=self.state, master=v("w"), exp_avg_scale=v("ms"), exp_avg_sq_scale=v("vs"), weight_decay=decay)

    def now(self):
        return {k: t.cpu() for k, t in self.dev.items()}

    def check(self, got, lr, step, decay, scale, seed):
        """got: now(); every tensor against the formula from the values in self.cpu, everything between them as it was."""
        untouched = {k: torch.ones(t.numel(), dtype=torch.bool) for k, t in self.cpu.items()}
        old = {k: self.views(k, self.cpu) for k in self.cpu}
        new = {k: self.views(k, got) for k in self.cpu}
        inside = {k: self.views(k, untouched) for k in self.cpu}
        for k, n in enumerate(self.counts):
            for name in self.cpu:
                if name != "g" and n:
                    inside[name][k].fill_(False)
            if n == 0:
                continue
            p = old["w" if self.master else "p"][k].double()
            if self.state == "fp32":
                m, v = old["m"][k].double(), old["v"][k].double()
            else:
                m, v = decode(old["m"][k], old["ms"][k]), decode(old["v"][k], old["vs"][k]) ** 2
            d = decay[k] if isinstance(decay, list) else decay
            wp, wm, wv, ep, em, ev = adamw(p, old["g"][k].double(), m, v, lr, step, B1, B2, EPS, d, scale)
            if self.master:
                assert ((new["w"][k].double() - wp).abs() <= ep).all(), k
            rounding = HALF[self.param] * wp.abs() * 1.01 if self.param == "bf16" else 0.0
            assert ((new["p"][k].double() - wp).abs() <= ep + rounding).all(), k
            if self.master:
                assert torch.equal(new["p"][k], new["w"][k].to(DT[self.param])), k
            if self.state == "fp32":
                assert ((new["m"][k].double() - wm).abs() <= em).all() and ((new["v"][k].double() - wv).abs() <= ev).all(), k
            else:
                w = words(seed, k, n)
                check_codes(new["m"][k], new["ms"][k], wm, em, w, False)
                root = wv.sqrt()
                check_codes(new["v"][k], new["vs"][k], root, root * 6 * 2.0 ** -24 + 1e-30, w, True)
        for name in self.cpu:
            keep = untouched[name]
            a, b = (x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x for x in (got[name], self.cpu[name]))
            assert torch.equal(a[keep], b[keep]), name


COUNTS = [1, 255, 0, 256, 257, 4096, 31, 513, 8, 2048 + 7, 100_003]


@pytest.mark.parametrize("param,master,grad,state", FORMS)
@pytest.mark.parametrize("gap", [0, 1, 3])
def test_formula(comm, param, master, grad, state, gap):
    s = Set(COUNTS, param, master, grad, state, gap, seed=gap)
    decay = [0.1 if k % 2 else 0.0 for k in range(len(COUNTS))]
    factor = torch.tensor([0.5], device="cuda")
    comm.adamw(s.table(decay), 1e-3, 7, beta1=B1, beta2=B2, eps=EPS, grad_scale=0.25, factor=factor, seed=99)
    s.check(s.now(), 1e-3, 7, decay, 0.125, 99)


def test_root_equals_the_correctly_rounded_one_for_every_number():
    counts = torch.zeros(2, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    assert hd.selftest_root(counts) == hb.OK
    torch.cuda.synchronize()
    assert counts.tolist() == [0, 192 * 2 ** 23 + 1]


def bits_of_a_step(p, g, m, v, ms, vs, scale, seed, tensor):
    """The states of a step in numpy's binary32, operation by operation as the header has them: (m, v) or (codes, scales of m, of the root)."""
    f = np.float32
    x = g * f(scale)
    if ms is not None:
        m, v = (c * s for c, s in ((m, ms), (v, vs)))
        v = v * v
    m = m * f(B1) + x * f(1 - B1)
    v = v * f(B2) + (x * x) * f(1 - B2)
    if ms is None:
        return m, v
    w = words(seed, tensor, len(g)).numpy()
    out = []
    for y, rnd, root in ((m, w & 0xFFFF, False), (np.sqrt(v), w >> 16, True)):
        full = np.zeros(-(-len(y) // BLOCK) * BLOCK, f)
        full[:len(y)] = y
        top = np.abs(full.reshape(-1, BLOCK)).max(1)
        some = top > f(1e-35)
        with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
            inv = np.where(some, (f(1) / top) * f(448), f(0)).astype(f)
        u = y * np.repeat(inv, BLOCK)[:len(y)]
        small = np.abs(u) < f(2.0 ** -6)
        shift = np.where(small, f(2.0 ** -6), f(0))
        b = (np.abs(u) + shift).astype(f).view(np.uint32) + (rnd.astype(np.uint32) << np.uint32(4)) & np.uint32(0xFFF00000)
        q = b.view(f) - shift
        if root:
            q = np.where((u > 0) & (q == 0), f(2.0 ** -9), q)
        out += [np.copysign(q, u), np.where(some, top * f(1 / 448), f(0)).astype(f)]
    return out


@pytest.mark.parametrize("state", ["fp32", "8bit"])
@pytest.mark.parametrize("gap", [0, 3])
@pytest.mark.parametrize("zeros", [0.0, 0.5])
def test_states_bit_for_bit(comm, state, gap, zeros):
    s = Set([257, 65_536, 5000], "bf16", False, "bf16", state, gap, seed=11)
    if zeros:   # numbers in the codes' lowest range, roots outside the fast one
        for k in "gmv":
            hit = torch.rand(s.total, generator=torch.Generator().manual_seed(3)) < zeros
            s.cpu[k] = torch.where(hit, torch.zeros_like(s.cpu[k].float()), s.cpu[k].float() * torch.logspace(-8, 0, s.total)).to(s.cpu[k].dtype)
            s.dev[k].copy_(s.cpu[k])
    comm.adamw(s.table(), 1e-3, 3, beta1=B1, beta2=B2, grad_scale=0.3, seed=77)
    got = s.now()
    for k, n in enumerate(s.counts):
        a = lambda name, src: s.views(name, src)[k].float().numpy()  # noqa: E731
        rep = lambda name: np.repeat(a(name, s.cpu), BLOCK)[:n] if state == "8bit" else None  # noqa: E731
        want = bits_of_a_step(None, a("g", s.cpu), a("m", s.cpu), a("v", s.cpu), rep("ms"), rep("vs"), 0.3, 77, k)
        names = ("m", "v") if state == "fp32" else ("m", "ms", "v", "vs")
        for name, w in zip(names, want):
            have = a(name, got)
            assert np.array_equal(have, w), (name, k, np.flatnonzero(have != w)[:5], have[have != w][:5], w[have != w][:5])


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_first_step_from_zero(comm, state):
    s = Set([300, 70_000], "bf16", True, "bf16", state, first=True)
    if state == "8bit":
        for k in ("ms", "vs"):
            s.cpu[k].zero_()
            s.dev[k].zero_()
    comm.adamw(s.table(0.1), 1e-3, 1, beta1=B1, beta2=B2, eps=EPS, seed=1)
    s.check(s.now(), 1e-3, 1, 0.1, 1.0, 1)


@pytest.mark.parametrize("n", [31, 33, 96, 97, 420, 421, 900])
@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_many_tensors(comm, n, state):
    """More than one table, and both of their sizes."""
    rng = np.random.RandomState(n)
    counts = [int(x) for x in rng.randint(0, 700, n)]
    s = Set(counts, "bf16", False, "bf16", state, gap=n % 2, seed=n)
    comm.adamw(s.table(0.01), 1e-3, 3, beta1=B1, beta2=B2, eps=EPS, seed=5)
    s.check(s.now(), 1e-3, 3, 0.01, 1.0, 5)


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_alignment_changes_no_bit(comm, state):
    counts, out = [2048, 5000, 256], []
    for gap in (0, 64, 5):
        s = Set(counts, "fp32", False, "fp32", state, gap)
        ref = Set(counts, "fp32", False, "fp32", state, 0)
        for k in s.dev:
            for a, b in zip(s.views(k), ref.views(k)):
                a.copy_(b)
        comm.adamw(s.table(), 1e-3, 3, beta1=B1, beta2=B2, seed=8)
        out.append({k: torch.cat([x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x for x in s.views(k)]).cpu() for k in s.dev})
    for o in out[1:]:
        for k in o:
            assert torch.equal(o[k], out[0][k]), k


def test_seed_changes_the_rounding_and_nothing_else(comm):
    got = []
    for seed in (1, 1, 2):
        s = Set([10_000], "fp32", False, "fp32", "8bit")
        comm.adamw(s.table(), 1e-3, 3, beta1=B1, beta2=B2, seed=seed)
        got.append(s.now())
    for k in got[0]:
        same = lambda a, b: torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8))  # noqa: E731
        assert same(got[0], got[1]), k
        assert same(got[0], got[2]) == (k not in "mv"), k


def test_an_average_moves_by_less_than_a_code(comm):
    """Stochastic rounding: 400 steps that each move m by a hundredth of a code's step end where the sum of them is."""
    n = 64 * BLOCK
    one = torch.ones(n, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros(n // BLOCK, device="cuda") for _ in range(2))
    m.fill_(200.0)
    ms.fill_(1.0)
    m[::BLOCK] = 448.0    # keeps the blocks' scale
    g = torch.full((n,), 200.0, device="cuda")
    g[1::2] = 232.0
    g[::BLOCK] = 448.0
    t = hb.AdamTensors([one], [g], [m], [v], "fp32", "fp32", state="8bit", exp_avg_scale=[ms], exp_avg_sq_scale=[vs])
    for k in range(400):
        comm.adamw(t, 0.0, 1, beta1=0.995, beta2=0.5, seed=k)
    x = (m.float() * ms.repeat_interleave(BLOCK)).cpu().double()
    want = 232 - 32 * 0.995 ** 400
    # each of 400 roundings adds at most (16/2)^2 of variance and decays with 0.995^2: below 64 / (1 - 0.995^2) = 6400 for one element, and 8160 elements of one kind
    assert abs(x[1::2].mean() - want) < 5 * 80 / math.sqrt(8000)
    assert torch.equal(one.cpu(), torch.ones(n))   # lr 0


def test_a_nan_factor_skips_the_step(comm):
    for state in ("fp32", "8bit"):
        s = Set([777, 256], "bf16", True, "bf16", state)
        comm.adamw(s.table(0.1), 1e-3, 3, factor=torch.tensor([math.nan], device="cuda"))
        got = s.now()
        for k in got:
            assert torch.equal(got[k].view(torch.uint8), s.cpu[k].view(torch.uint8)), k


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_gradients_that_are_not_finite_stay_in_their_element_or_block(comm, bad):
    s = Set([1000], "fp32", False, "fp32", "fp32")
    s.cpu["g"][300] = bad
    s.dev["g"][300] = bad
    comm.adamw(s.table(), 1e-3, 3, beta1=B1, beta2=B2)
    got = s.now()
    for k in "pmv":
        x = s.views(k, got)[0]
        assert not torch.isfinite(x[300]) and torch.isfinite(x[:300]).all() and torch.isfinite(x[301:]).all(), k
    s = Set([1000], "fp32", False, "fp32", "8bit")
    s.dev["g"][300] = bad
    comm.adamw(s.table(), 1e-3, 3, beta1=B1, beta2=B2)
    got = s.now()
    for k in "mv":
        x = decode(s.views(k, got)[0], s.views(k + "s", got)[0])
        assert not torch.isfinite(x[256:512]).any() and torch.isfinite(x[:256]).all() and torch.isfinite(x[512:]).all(), k


def test_extreme_values(comm):
    """Gradients whose squares vanish or are subnormal, zero gradients, blocks too small for a scale."""
    n = 4 * BLOCK
    g = torch.zeros(n)
    g[:BLOCK] = torch.logspace(-38, -18, BLOCK)
    g[BLOCK:2 * BLOCK] = torch.logspace(-5, 15, BLOCK)
    g[2 * BLOCK:3 * BLOCK] = 1e-37
    for state in ("fp32", "8bit"):
        s = Set([n], "fp32", False, "fp32", state, first=True)
        for k in ("ms", "vs"):
            if k in s.cpu:
                s.cpu[k].zero_()
                s.dev[k].zero_()
        s.cpu["g"][:n] = g
        s.dev["g"][:n] = g.cuda()
        comm.adamw(s.table(), 1e-3, 1, beta1=B1, beta2=B2, eps=EPS, seed=3)
        got = s.now()
        if state == "fp32":
            s.check(got, 1e-3, 1, 0.0, 1.0, 3)
        else:
            for k in ("p", "m", "v", "ms", "vs"):
                assert torch.isfinite(got[k].float()).all(), k
            m = decode(s.views("m", got)[0], s.views("ms", got)[0])
            assert (m[2 * BLOCK:] == 0).all() and (m[BLOCK:2 * BLOCK].max() > 0)
            root = s.views("v", got)[0].float()
            assert (root[BLOCK:2 * BLOCK] > 0).all()   # a root above zero stays above zero


def test_rates_on_the_device_in_a_captured_step(comm):
    s, ref = (Set([5000, 77], "bf16", True, "bf16", "8bit", seed=4) for _ in range(2))
    rates = torch.zeros(4, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    t, tr = s.table(0.1), ref.table(0.1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        comm.adamw(t, 0.0, 1, beta1=B1, beta2=B2, rates=rates, stream=side)
    for step in (1, 2, 3):
        rates.copy_(hb.adamw_rates(1e-3 * step, step, B1, B2, seed=step))
        before = ref.now()
        graph.replay()
        comm.adamw(tr, 1e-3 * step, step, beta1=B1, beta2=B2, seed=step)
        torch.cuda.synchronize()
        # the bias terms are rounded on the way through the record: the weights by a few more u of the step, the states not at all
        a, b = s.now(), ref.now()
        for k in ("m", "v", "ms", "vs"):
            assert torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)), (k, step)
        move = (b["w"].double() - before["w"].double()).abs()
        assert ((a["w"].double() - b["w"].double()).abs() <= 8 * 2.0 ** -24 * (move + b["w"].double().abs())).all()
        for k in s.dev:
            s.dev[k].copy_(ref.dev[k])


def test_an_empty_plan_and_shared_gradients(comm):
    comm.adamw(hb.AdamTensors([], [], [], [], "fp32", "fp32"), 1e-3, 1)
    g = torch.randn(300, device="cuda")
    z = lambda: [torch.zeros(300, device="cuda") for _ in range(2)]  # noqa: E731
    p, m, v = z(), z(), z()
    t = hb.AdamTensors(p, [g, g], m, v, "fp32", "fp32")
    comm.adamw(t, 1e-3, 1)
    t.destroy()
    torch.cuda.synchronize()
    assert p[0].any() and all(torch.equal(a[0], a[1]) for a in (p, m, v))


def test_other_streams_and_repeated_calls(comm):
    s, ref = (Set([200_000], "bf16", True, "bf16", "fp32") for _ in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    t, tr = s.table(), ref.table()
    for k in range(20):
        comm.adamw(t, 1e-3, k + 1, beta1=B1, beta2=B2, stream=side)
        comm.adamw(tr, 1e-3, k + 1, beta1=B1, beta2=B2)
    torch.cuda.synchronize()
    a, b = s.now(), ref.now()
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_more_elements_than_32_bits_count(comm):
    n = (1 << 32) + 300
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, v = (torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros((n + BLOCK - 1) // BLOCK, device="cuda") for _ in range(2))
    tail = slice(n - 812, n)
    start = n - 812
    assert start % BLOCK == 0
    x = torch.randn(812, generator=torch.Generator().manual_seed(1)).bfloat16()
    g[tail] = x.cuda()
    g[:256] = x[:256].cuda()
    t = hb.AdamTensors([p], [g], [m], [v], "bf16", "bf16", state="8bit", exp_avg_scale=[ms], exp_avg_sq_scale=[vs])
    comm.adamw(t, 1e-3, 1, beta1=B1, beta2=B2, eps=EPS, seed=6)
    zero = torch.zeros(812, dtype=torch.float64)
    for at, k in ((0, 256), (start, 812)):
        gg = x[:k].double()
        wp, wm, wv, ep, em, ev = adamw(zero[:k], gg, zero[:k], zero[:k], 1e-3, 1, B1, B2, EPS, 0.0, 1.0)
        got = p[at:at + k].cpu().double()
        assert ((got - wp).abs() <= ep + HALF["bf16"] * wp.abs() * 1.01).all()
        w = words(6, 0, k, at)
        b0, b1 = at // BLOCK, at // BLOCK + (k + BLOCK - 1) // BLOCK
        check_codes(m[at:at + k].cpu(), ms[b0:b1].cpu(), wm, em, w, False)
        check_codes(v[at:at + k].cpu(), vs[b0:b1].cpu(), wv.sqrt(), wv.sqrt() * 6 * 2.0 ** -24, w, True)
    assert not p[256:start].any() and not ms[1:start // BLOCK].any()


# ------------------------------------------------------------------------------------------------ sharded


def sharded(R, n, param, master, grad, state, off=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    q = (n + R - 1) // R
    cut = [(min(c * q, n), min((c + 1) * q, n)) for c in range(R)]
    room = lambda k, dt: [torch.zeros(k + 40, dtype=dt, device="cuda")[off:off + k] for _ in range(R)]  # noqa: E731
    s = dict(q=q, cut=cut, g=[(torch.randn(n, generator=g) * 1e-2).to(DT[grad]) for _ in range(R)], p=(torch.randn(n, generator=g) * 0.02).to(DT[param]))
    s["w"] = s["p"].float() if master else None
    d = s["dev"] = {"g": room(n, DT[grad]), "p": room(n, DT[param])}
    for r in range(R):
        d["g"][r].copy_(s["g"][r])
        d["p"][r].copy_(s["p"])
    if master:
        d["w"] = room(q, torch.float32)
        for c, (a, b) in enumerate(cut):
            d["w"][c][:b - a] = s["w"][a:b].cuda()
    if state == "fp32":
        s["m"], s["v"] = torch.randn(n, generator=g) * 2e-3, (torch.randn(n, generator=g) * 1e-2) ** 2 + 1e-9
        d["m"], d["v"] = room(q, torch.float32), room(q, torch.float32)
    else:
        s["m"] = (torch.randn(n, generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
        s["v"] = (torch.rand(n, generator=g) * 448).to(torch.float8_e4m3fn)
        d["m"], d["v"] = room(q, torch.float8_e4m3fn), room(q, torch.float8_e4m3fn)
        nb = (q + BLOCK - 1) // BLOCK
        for k in ("ms", "vs"):
            s[k] = [torch.rand(nb, generator=g) * 1e-4 + 1e-6 for _ in range(R)]
            d[k] = [x.cuda() for x in s[k]]
    for c, (a, b) in enumerate(cut):
        for k in "mv":
            d[k][c][:b - a] = s[k][a:b].cuda()
    return s


@pytest.mark.parametrize("R,n", [(1, 1000), (2, 4096), (3, 1), (5, 7), (4, 100_003), (8, 8 * 2048), (6, 50_009), (16, 3000), (64, 64 * 256), (4, 4 * 1026), (3, 3 * 2054 - 1), (8, 8 * 1300)])
@pytest.mark.parametrize("param,master,grad,state", FORMS)
def test_sharded_formula(R, n, param, master, grad, state):
    comm = hb.Comm(R, 0)
    s = sharded(R, n, param, master, grad, state, off=0 if n in (4104, 6161, 10400) else (R * n) % 3, seed=R)   # the last three: pairs of elements
    d = s["dev"]
    lr, step, scale, seed = 1e-3, 5, 1.0 / R, 31
    comm.sharded_adamw(d["g"], d["p"], d["m"], d["v"], n, param, grad, lr, step, state=state, master=d.get("w"), exp_avg_scale=d.get("ms"), exp_avg_sq_scale=d.get("vs"), beta1=B1,
                       beta2=B2, eps=EPS, weight_decay=0.1, grad_scale=scale, seed=seed)
    got = {k: [x.cpu() for x in xs] for k, xs in d.items()}
    for r in range(1, R):
        assert torch.equal(got["p"][r], got["p"][0])
    for c, (a, b) in enumerate(s["cut"]):
        k = b - a
        if not k:
            continue
        parts = torch.stack([x[a:b].double() for x in s["g"]])
        # R - 1 adds in binary32: off by u times the partial sums, of which none is larger than the sum of the sizes
        extra = (R - 1) * 2.0 ** -24 * parts.abs().sum(0) * scale
        if state == "fp32":
            m, v = s["m"][a:b].double(), s["v"][a:b].double()
        else:
            m, v = decode(s["m"][a:b], s["ms"][c]), decode(s["v"][a:b], s["vs"][c]) ** 2
        p = (s["w"] if master else s["p"])[a:b].double()
        g = parts.sum(0)
        wp, wm, wv, ep, em, ev = adamw(p, g, m, v, lr, step, B1, B2, EPS, 0.1, scale)
        below = wv.sqrt() / math.sqrt(1 - B2 ** step) + EPS
        size = lr / (1 - B1 ** step)
        em = em + (1 - B1) * extra
        dv = (1 - B2) * (2 * (g * scale).abs() * extra + extra * extra)
        ev = ev + dv
        eroot = wv.sqrt() * 6 * 2.0 ** -24 + dv / (2 * wv.sqrt()) * 1.01 + 1e-30
        ep = ep + size * ((1 - B1) * extra / below + wm.abs() * (dv / (2 * wv.sqrt()) * 1.01 / math.sqrt(1 - B2 ** step)) / below ** 2)
        rounding = HALF["bf16"] * wp.abs() * 1.01 if param == "bf16" else 0.0
        assert ((got["p"][0][a:b].double() - wp).abs() <= ep + rounding).all()
        if master:
            assert ((got["w"][c][:k].double() - wp).abs() <= ep).all()
            assert torch.equal(got["w"][c][:k].to(DT[param]), got["p"][0][a:b])
        if state == "fp32":
            assert ((got["m"][c][:k].double() - wm).abs() <= em).all() and ((got["v"][c][:k].double() - wv).abs() <= ev).all()
        else:
            nb = (k + BLOCK - 1) // BLOCK
            w = words(seed, c, k)
            check_codes(got["m"][c][:k], got["ms"][c][:nb], wm, em, w, False)
            check_codes(got["v"][c][:k], got["vs"][c][:nb], wv.sqrt(), eroot, w, True)
            assert torch.equal(got["ms"][c][nb:], s["ms"][c][nb:])
    for r in range(R):
        assert torch.equal(got["g"][r], s["g"][r])
    comm.destroy()


def test_sharded_with_more_elements_than_32_bits_count():
    R, n = 2, (1 << 32) + 600
    q, comm = n // 2, hb.Comm(2, 0)
    bf = lambda k: [torch.zeros(k, dtype=torch.bfloat16, device="cuda") for _ in range(R)]  # noqa: E731
    g, p = bf(n), bf(n)
    m, v = ([torch.zeros(q, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(R)] for _ in range(2))
    ms, vs = ([torch.zeros(-(-q // BLOCK), device="cuda") for _ in range(R)] for _ in range(2))
    start = q // BLOCK * BLOCK                      # of rank 1's last block
    k = q - start
    x = torch.randn(2, k, generator=torch.Generator().manual_seed(1)).bfloat16()
    for r in range(R):
        g[r][n - k:] = x[r].cuda()
    comm.sharded_adamw(g, p, m, v, n, "bf16", "bf16", 1e-3, 1, state="8bit", exp_avg_scale=ms, exp_avg_sq_scale=vs, beta1=B1, beta2=B2, eps=EPS, seed=4)
    zero = torch.zeros(k, dtype=torch.float64)
    s = x.double().sum(0)                           # of two bf16 numbers: one rounding, of at most u of their sizes, in binary32
    extra = 2.0 ** -24 * x.double().abs().sum(0)
    wp, wm, wv, ep, em, ev = adamw(zero, s, zero, zero, 1e-3, 1, B1, B2, EPS, 0.0, 1.0)
    # the first step's quotient is +-1 but for eps: the sum's error moves m and the root alike
    for r in range(R):
        assert ((p[r][n - k:].cpu().double() - wp).abs() <= ep + HALF["bf16"] * wp.abs() * 1.01 + 1e-3 * 2 * extra / (s.abs() + EPS)).all()
        assert not p[r][:n - k].any()
    w = words(4, 1, k, start)
    check_codes(m[1][start:].cpu(), ms[1][-1:].cpu(), wm, em + (1 - B1) * extra, w, False)
    root = wv.sqrt()
    check_codes(v[1][start:].cpu(), vs[1][-1:].cpu(), root, root * 6 * 2.0 ** -24 + math.sqrt(1 - B2) * extra, w, True)
    assert not ms[0].any() and not ms[1][:-1].any()
    comm.destroy()


def test_sharded_factor_and_capture():
    R, n = 4, 10_000
    comm = hb.Comm(R, 0)
    s, ref = (sharded(R, n, "bf16", True, "bf16", "fp32") for _ in range(2))

    def call(d, **more):
        comm.sharded_adamw(d["g"], d["p"], d["m"], d["v"], n, "bf16", "bf16", 1e-3, 2, master=d["w"], beta1=B1, beta2=B2, **more)
    call(s["dev"], factor=torch.tensor([math.nan], device="cuda"))
    for k in ("p", "w", "m", "v"):
        assert all(torch.equal(a, b) for a, b in zip(s["dev"][k], ref["dev"][k])), k
    side, half = torch.cuda.Stream(), torch.tensor([0.5], device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(s["dev"], factor=half, stream=side)
    for _ in range(3):
        graph.replay()
        call(ref["dev"], factor=half)
    torch.cuda.synchronize()
    for k in ("p", "w", "m", "v"):
        assert all(torch.equal(a, b) for a, b in zip(s["dev"][k], ref["dev"][k])), k
    comm.destroy()


@pytest.mark.parametrize("grad", ["fp32", "bf16"])
def test_sharded_adds_in_the_rings_order(grad):
    """Gradients whose binary32 sum depends on the order: beta1 = 0 shows the sum in m."""
    R, n = 5, 5 * 64
    comm = hb.Comm(R, 0)
    s = sharded(R, n, "fp32", False, grad, "fp32")
    d = s["dev"]
    gen = torch.Generator().manual_seed(9)
    for r in range(R):
        d["g"][r].copy_((torch.randn(n, generator=gen) * 10.0 ** (r - 2)).to(DT[grad]))
    comm.sharded_adamw(d["g"], d["p"], d["m"], d["v"], n, "fp32", grad, 1e-3, 1, beta1=0.0, beta2=0.5)
    g = [x.cpu().float().numpy() for x in d["g"]]
    for c, (a, b) in enumerate(s["cut"]):
        acc = g[(c + 1) % R][a:b].copy()
        for j in range(2, R + 1):
            acc = (acc + g[(c + j) % R][a:b]).astype(np.float32)
        assert np.array_equal(acc, d["m"][c].cpu().numpy()[:b - a])
    comm.destroy()


@pytest.mark.parametrize("state", ["fp32", "8bit"])
@pytest.mark.parametrize("n", [32, 127, 128, 129])
def test_numbers_of_tensors_at_the_tables_ends(comm, n, state):
    test_many_tensors(comm, n, state)
