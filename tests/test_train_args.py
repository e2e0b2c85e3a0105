"""Refusals of the operators of a training step: all of them come before anything touches a device."""
import ctypes
import math

import pytest

from paper_2609_34334_b200 import binding as hb
from paper_2609_34334_b200 import diag as hd

K = 1 << 20


def plan(rows, param="fp32", grad="fp32", state="fp32", decay=0.0):
    """rows: dicts of addresses."""
    n = len(rows)
    get = lambda k: [r.get(k, 0) for r in rows]  # noqa: E731
    some = lambda k: get(k) if any(k in r for r in rows) else None  # noqa: E731
    return hb.AdamTensors(get("p"), get("g"), get("m"), get("v"), param, grad, state=state, master=some("w"), exp_avg_scale=some("ms"), exp_avg_sq_scale=some("vs"),
                          weight_decay=decay, counts=[r["n"] for r in rows] if n else [])


def row(k=0, n=1000, **more):
    at = (k + 1) * 100 * K
    return dict(p=at, g=at + K, m=at + 2 * K, v=at + 3 * K, n=n, **more)


def code(fn, *a, **k):
    with pytest.raises(hb.HocclError) as e:
        fn(*a, **k)
    return e.value.code


class HostComm(hb.Comm):
    """A communicator without a device."""

    def __init__(self, R):
        self._h = ctypes.c_void_p()
        self.R, self._keep = R, []
        assert hd.lib().hoccl_comm_init_host_only(ctypes.byref(self._h), R) == hb.OK


def test_plans_that_are_served():
    plan([])
    plan([dict(n=0)])
    plan([row(k, n=1 + k) for k in range(1000)])
    plan([row(w=50 * K), row(1, w=60 * K)], param="bf16")
    plan([row(ms=50 * K, vs=51 * K)], param="bf16", grad="bf16", state="8bit")
    plan([dict(row(), g=1 << 40), dict(row(1), g=1 << 40)])                  # gradients may be shared
    plan([dict(row(n=256), m=3 * K + 1, v=4 * K + 3, ms=50 * K, vs=51 * K)], state="8bit")   # bytes need no alignment


@pytest.mark.parametrize("rows,kw,want", [
    ([dict(row(), p=0)], {}, hb.ERR_INVALID_ARG),
    ([dict(row(), g=0)], {}, hb.ERR_INVALID_ARG),
    ([dict(row(), m=0)], {}, hb.ERR_INVALID_ARG),
    ([dict(row(), p=K + 2)], {}, hb.ERR_INVALID_ARG),
    ([dict(row(), g=K + 1)], dict(grad="bf16"), hb.ERR_INVALID_ARG),
    ([dict(row(), v=8 * K + 2)], {}, hb.ERR_INVALID_ARG),
    ([row(w=50 * K)], {}, hb.ERR_UNSUPPORTED),                                # a master beside binary32 weights
    ([row(w=50 * K), row(1)], dict(param="bf16"), hb.ERR_INVALID_ARG),        # of some tensors only
    ([row()], dict(state="8bit"), hb.ERR_INVALID_ARG),                        # no scales
    ([row(ms=50 * K, vs=51 * K + 2)], dict(state="8bit"), hb.ERR_INVALID_ARG),
    ([row(), row()], {}, hb.ERR_INVALID_ARG),                                 # the same tensor twice
    ([dict(row(), m=100 * K + 3996)], {}, hb.ERR_INVALID_ARG),                # the last element of p
    ([dict(row(), g=100 * K + 3996)], {}, hb.ERR_INVALID_ARG),
    ([row(ms=50 * K, vs=50 * K + 12)], dict(state="8bit"), hb.ERR_INVALID_ARG),
    ([row()], dict(param=7), hb.ERR_UNSUPPORTED),
    ([row()], dict(grad=-1), hb.ERR_UNSUPPORTED),
    ([row()], dict(state=2), hb.ERR_UNSUPPORTED),
    ([row()], dict(decay=math.nan), hb.ERR_INVALID_ARG),
    ([row(n=1 << 60)], {}, hb.ERR_INVALID_ARG),
])
def test_plans_that_are_refused(rows, kw, want):
    assert code(plan, rows, **kw) == want


def test_plan_checks_tensors():
    import torch
    f = lambda n: torch.zeros(n)  # noqa: E731
    with pytest.raises(ValueError):
        hb.AdamTensors([f(8)[::2]], [f(4)], [f(4)], [f(4)], "fp32", "fp32")
    with pytest.raises(ValueError):
        hb.AdamTensors([f(8)], [f(8)], [f(7)], [f(8)], "fp32", "fp32")
    with pytest.raises(ValueError):
        hb.AdamTensors([f(8)], [f(8)], [f(8)], [], "fp32", "fp32")
    with pytest.raises(ValueError):
        hb.AdamTensors([f(257)], [f(257)], [f(257)], [f(257)], "fp32", "fp32", state="8bit", exp_avg_scale=[f(1)], exp_avg_sq_scale=[f(2)])
    hb.AdamTensors([f(257)], [f(257)], [f(257)], [f(257)], "fp32", "fp32")
    with pytest.raises(ValueError):
        hb.Tensors([f(8)[::2]], "fp32")


BAD_NUMBERS = [dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=1e-60), dict(step=0),
               dict(step=-3), dict(grad_scale=math.inf), dict(lr=1e39), dict(grad_scale=-1e39), dict(factor=2), dict(rates=8)]


@pytest.mark.parametrize("bad", BAD_NUMBERS)
def test_steps_that_are_refused(bad):
    c, t = HostComm(2), plan([row()])
    good = dict(lr=1e-3, step=1, stream=0)
    assert code(c.adamw, t, **good) == hb.ERR_CUDA     # no device
    assert code(c.adamw, t, **{**good, **bad}) == hb.ERR_INVALID_ARG
    s = dict(good, state="fp32")
    lists = [[(k * 10 + r + 1) * K for r in range(2)] for k in range(4)]
    assert code(c.sharded_adamw, *lists, 64, "fp32", "fp32", **s) == hb.ERR_CUDA
    assert code(c.sharded_adamw, *lists, 64, "fp32", "fp32", **{**s, **bad}) == hb.ERR_INVALID_ARG
    assert hb._calls.adamw_step(c._h.value, None, 1e-3, 1, 0.9, 0.99, 1e-8, 1.0, None, None, 0, 0) == hb.ERR_INVALID_ARG
    assert hb._calls.adamw_step(None, t._h.value, 1e-3, 1, 0.9, 0.99, 1e-8, 1.0, None, None, 0, 0) == hb.ERR_INVALID_ARG


@pytest.mark.parametrize("change,want", [
    (dict(), hb.ERR_CUDA), (dict(count=0), hb.OK),
    (dict(grads=[K, 0]), hb.ERR_INVALID_ARG), (dict(params=[11 * K, 12 * K + 2]), hb.ERR_INVALID_ARG), (dict(params=[11 * K, 11 * K]), hb.ERR_INVALID_ARG),
    (dict(params=[11 * K, 11 * K + 128]), hb.ERR_INVALID_ARG), (dict(params=[K, 12 * K]), hb.ERR_INVALID_ARG), (dict(exp_avg=[21 * K, 0]), hb.ERR_INVALID_ARG),
    (dict(exp_avg=[21 * K, 21 * K + 120]), hb.ERR_INVALID_ARG), (dict(exp_avg=[21 * K, 0], count=1), hb.ERR_CUDA),   # rank 1's chunk is empty
    (dict(exp_avg=[21 * K, 21 * K + 128]), hb.ERR_CUDA),                                                          # 32 elements each
    (dict(state="8bit"), hb.ERR_INVALID_ARG), (dict(state="8bit", exp_avg_scale=[51 * K, 52 * K], exp_avg_sq_scale=[53 * K, 54 * K]), hb.ERR_CUDA),
    (dict(master=[55 * K, 56 * K]), hb.ERR_UNSUPPORTED), (dict(master=[55 * K, 56 * K], param_dtype="bf16"), hb.ERR_CUDA),
    (dict(master=[55 * K, 0], param_dtype="bf16"), hb.ERR_INVALID_ARG), (dict(param_dtype=9), hb.ERR_UNSUPPORTED), (dict(weight_decay=math.inf), hb.ERR_INVALID_ARG),
    (dict(count=1 << 50), hb.ERR_INVALID_ARG),
])
def test_sharded_arguments(change, want):
    c = HostComm(2)
    a = dict(grads=[K, 2 * K], params=[11 * K, 12 * K], exp_avg=[21 * K, 22 * K], exp_avg_sq=[31 * K, 32 * K], count=64, param_dtype="fp32", grad_dtype="fp32", lr=1e-3, step=1,
             stream=0)
    a.update(change)
    if want == hb.OK:
        c.sharded_adamw(**a)
    else:
        assert code(c.sharded_adamw, **a) == want


def test_norm_arguments():
    c = HostComm(2)
    good = hb.Tensors([K, 2 * K], "fp32", counts=[5, 6])
    assert code(c.grad_norm, good, 64, stream=0) == hb.ERR_SCRATCH
    c.set_scratch(256, hb.grad_norm_scratch_bytes() - 1)
    assert code(c.grad_norm, good, 64, stream=0) == hb.ERR_SCRATCH
    c.set_scratch(256, hb.grad_norm_scratch_bytes())
    assert code(c.grad_norm, good, 64, stream=0) == hb.ERR_CUDA
    assert code(c.grad_norm, hb.Tensors([0, K], "bf16", counts=[0, 7]), 64, stream=0) == hb.ERR_CUDA
    for t, out, more in ((good, 0, {}), (good, 2, {}), (good, 64, dict(max_norm=0.0)), (good, 64, dict(max_norm=math.nan)), (hb.Tensors([0], "fp32", counts=[4]), 64, {}),
                         (hb.Tensors([K + 2], "fp32", counts=[4]), 64, {}), (hb.Tensors([K], "fp32", counts=[1 << 60]), 64, {})):
        assert code(c.grad_norm, t, out, stream=0, **more) == hb.ERR_INVALID_ARG
    assert code(c.grad_norm, hb.Tensors([K], 5, counts=[4]), 64, stream=0) == hb.ERR_UNSUPPORTED


def test_route_arguments():
    c = HostComm(2)
    a = dict(logits=[K, 2 * K], tokens=[4, 3], experts=16, topk=2, dtype="fp32", indices=[3 * K, 4 * K], weights=[5 * K, 6 * K], counts=[7 * K, 8 * K], loss=9 * K, saved=10 * K, stream=0)
    b = dict(logits=[K, 2 * K], tokens=[4, 3], experts=16, topk=2, dtype="fp32", indices=[3 * K, 4 * K], saved=10 * K, dweights=[5 * K, 6 * K], dloss=None, dlogits=[11 * K, 12 * K], stream=0)
    assert code(c.route, **a) == hb.ERR_SCRATCH
    assert code(c.route_backward, **b) == hb.ERR_CUDA
    need = hb.route_scratch_bytes(2, 4, 16)
    assert 0 < need < 1 << 20 and hb.route_scratch_bytes(0, 4, 16) == 0 and hb.route_scratch_bytes(2, 4, 1025) == 0
    c.set_scratch(256 * K, need)
    assert code(c.route, **a) == hb.ERR_CUDA
    inv, uns = hb.ERR_INVALID_ARG, hb.ERR_UNSUPPORTED
    for change, want in ((dict(experts=0), inv), (dict(experts=1025, ld=2000), inv), (dict(topk=0), inv), (dict(topk=17), inv), (dict(experts=64, topk=33), inv), (dict(ld=15), inv),
                         (dict(tokens=[1 << 31, 1]), inv), (dict(tokens=[-1, 1]), inv), (dict(dtype=3), uns), (dict(normalize=2), inv), (dict(per_rank=-1), inv),
                         (dict(logits=[K, 0]), inv), (dict(logits=[K, 2 * K + 2]), inv), (dict(indices=[3 * K, 4 * K + 2]), inv)):
        assert code(c.route, **{**a, **change}) == want, change
        if "indices" not in change:
            assert code(c.route_backward, **{**b, **change}) == want, change
    for change in (dict(weights=[5 * K, 5 * K]), dict(indices=[3 * K, 5 * K]), dict(counts=[7 * K, 0]), dict(counts=[7 * K, 7 * K + 64]), dict(loss=0), dict(saved=9 * K + 4), dict(loss=6),
                   dict(balance_coef=math.nan), dict(z_coef=math.inf), dict(weights=[K + 4, 6 * K])):
        assert code(c.route, **{**a, **change}) == inv, change
    for change in (dict(dlogits=[11 * K, 0]), dict(dlogits=[11 * K, 11 * K + 64]), dict(dlogits=[K, 2 * K], dld=17), dict(dld=15), dict(saved=0), dict(saved=11 * K), dict(dloss=2),
                   dict(indices=None), dict(dweights=[5 * K, 0]), dict(dlogits=[11 * K, 5 * K])):
        assert code(c.route_backward, **{**b, **change}) == inv, change
    for change in (dict(dlogits=[K, 2 * K]), dict(indices=None, dweights=None), dict(dloss=64), dict(dlogits=[K, 2 * K], ld=18, dld=18)):
        assert code(c.route_backward, **{**b, **change}) == hb.ERR_CUDA, change
    c.route_backward(**{**b, "tokens": [0, 0]})                                  # nothing to do
    assert code(c.route, **{**a, "tokens": [0, 0], "logits": [0, 0], "indices": [0, 0], "weights": [0, 0]}) == hb.ERR_CUDA   # the counts are written


def test_rates_record():
    import struct
    r = hb.adamw_rates(0.25, 3, 0.5, 0.0, seed=1 << 31 | 5)
    assert struct.unpack("<fffI", bytes(r.numpy().tobytes())) == (0.25, 0.875, 1.0, 1 << 31 | 5)


def test_tables_check_the_size_of_elements():
    """A tensor of the right length whose elements are smaller than the call takes them for would be read, and written, beyond its end."""
    import torch
    t = {"fp32": torch.float32, "bf16": torch.bfloat16, "8bit": torch.float8_e4m3fn}
    good = dict(param="bf16", grad="bf16", m="fp32", v="fp32", master="fp32", ms="fp32", vs="fp32")

    def table(state="fp32", n=256, **kinds):
        k = {**good, **kinds}
        x = {name: [torch.zeros(n if name not in ("ms", "vs") else -(-n // 256), dtype=t[kind])] for name, kind in k.items()}
        return hb.AdamTensors(x["param"], x["grad"], x["m"], x["v"], "bf16", "bf16", state=state, master=x["master"], exp_avg_scale=x["ms"], exp_avg_sq_scale=x["vs"])

    table()
    table(state="8bit", m="8bit", v="8bit")
    for bad in (dict(param="fp32"), dict(param="8bit"), dict(grad="fp32"), dict(grad="8bit"), dict(m="bf16"), dict(v="bf16"), dict(master="bf16"), dict(m="8bit")):
        with pytest.raises(ValueError):
            table(**bad)
    for bad in (dict(m="fp32", v="8bit"), dict(m="8bit", v="bf16"), dict(m="8bit", v="8bit", ms="bf16"), dict(m="8bit", v="8bit", vs="bf16")):
        with pytest.raises(ValueError):
            table(state="8bit", **bad)
    with pytest.raises(ValueError):
        hb.Tensors([torch.zeros(8, dtype=torch.bfloat16)], "fp32")
    with pytest.raises(ValueError):
        hb.Tensors([torch.zeros(8)], "bf16")
    with pytest.raises(ValueError):
        hb.Tensors([torch.zeros(8)], "fp32", counts=[9])
    with pytest.raises(ValueError):
        hb.Tensors([torch.zeros(8)[::2]], "fp32", counts=[4])
    hb.Tensors([torch.zeros(8)], "fp32", counts=[7])
    hb.Tensors([torch.zeros(8, dtype=torch.int32)], "fp32")   # four bytes are four bytes


def test_route_wants_a_number_of_tokens_for_every_rank():
    c = HostComm(2)
    c.set_scratch(256 * K, hb.route_scratch_bytes(2, 4, 16))
    a = dict(logits=[K, 2 * K], experts=16, topk=2, dtype="fp32", indices=[3 * K, 4 * K], weights=[5 * K, 6 * K], counts=[7 * K, 8 * K], loss=9 * K, saved=10 * K, stream=0)
    b = dict(logits=[K, 2 * K], experts=16, topk=2, dtype="fp32", indices=[3 * K, 4 * K], saved=10 * K, dweights=[5 * K, 6 * K], dloss=None, dlogits=[11 * K, 12 * K], stream=0)
    for tokens in ([4], [], [4, 3, 2]):
        with pytest.raises(ValueError):
            c.route(tokens=tokens, **a)
        with pytest.raises(ValueError):
            c.route_backward(tokens=tokens, **b)
    assert code(c.route, tokens=[4, 3], **a) == hb.ERR_CUDA and code(c.route_backward, tokens=(4, 3), **b) == hb.ERR_CUDA


def test_an_eps_whose_reciprocal_is_not_normal_is_refused():
    """The step divides by numbers from eps on with a reciprocal that gives 0 where the true one is below the least normal number."""
    c, t = HostComm(2), plan([row()])
    for eps, want in ((2.0 ** 126, hb.ERR_CUDA), (1e38, hb.ERR_INVALID_ARG), (3e38, hb.ERR_INVALID_ARG)):
        assert code(c.adamw, t, lr=1e-3, step=1, eps=eps, stream=0) == want


def test_scratch_that_overlaps_a_callers_buffer_is_refused():
    c = HostComm(2)
    need = hb.grad_norm_scratch_bytes()
    c.set_scratch(8 * K, need + 4096)
    inside, behind, across = 8 * K + need - 4, 8 * K + need, 8 * K - 16
    for at, want in ((inside, hb.ERR_INVALID_ARG), (across, hb.ERR_INVALID_ARG), (behind, hb.ERR_CUDA), (8 * K - 32, hb.ERR_CUDA)):
        assert code(c.grad_norm, hb.Tensors([K, at], "fp32", counts=[5, 8]), 64, stream=0) == want, at
    for out, want in ((inside - 4, hb.ERR_INVALID_ARG), (8 * K - 4, hb.ERR_INVALID_ARG), (behind, hb.ERR_CUDA), (8 * K - 8, hb.ERR_CUDA)):
        assert code(c.grad_norm, hb.Tensors([K], "fp32", counts=[5]), out, stream=0) == want, out
    a = dict(logits=[K, 2 * K], tokens=[4, 3], experts=16, topk=2, dtype="fp32", indices=[3 * K, 4 * K], weights=[5 * K, 6 * K], counts=[7 * K, 9 * K], loss=10 * K, saved=11 * K, stream=0)
    assert code(c.route, **a) == hb.ERR_CUDA
    used = 2 * (2 * 16 + 2) * 4   # two ranks with one CTA each
    assert used <= hb.route_scratch_bytes(2, 4, 16) <= need
    for at, want in ((8 * K, hb.ERR_INVALID_ARG), (8 * K + used - 4, hb.ERR_INVALID_ARG), (8 * K - 4, hb.ERR_INVALID_ARG), (8 * K + 4096, hb.ERR_CUDA), (8 * K - 1024, hb.ERR_CUDA)):
        for name in ("logits", "indices", "weights", "counts"):
            assert code(c.route, **{**a, name: [a[name][0], at]}) == want, (name, at)
        for name in ("loss", "saved"):
            assert code(c.route, **{**a, name: at}) == want, (name, at)
