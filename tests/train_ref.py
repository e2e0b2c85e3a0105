"""Plain 64-bit forms of the operators of a training step, on the CPU, with bounds on what binary32 arithmetic may be off (first order in u)."""
import math

import torch

U = 2.0 ** -24            # binary32's rounding, relative
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}   # a rounding to the type: half of finfo.eps
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 256


def mix(h):
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & 0xFFFFFFFF
    return h ^ (h >> 16)


def words(seed, tensor, n, start=0):
    """The 32 random bits of elements start .. start + n - 1."""
    i = torch.arange(start, start + n, dtype=torch.int64)
    key = mix((seed + tensor * 0x9E3779B9) & 0xFFFFFFFF)
    return mix(((i & 0xFFFFFFFF) + (i >> 32) * 0x632BE5AB + key) & 0xFFFFFFFF)


def decode(codes, scales):
    """codes: e4m3 tensor, scales: binary32."""
    return codes.double() * scales.double().repeat_interleave(BLOCK)[:codes.numel()]


def adamw(p, g, m, v, lr, step, beta1, beta2, eps, decay, scale):
    """One tensor in 64 bits: new p, m, v and bounds on their errors in binary32.

    x = scale * g: 2 roundings (scale's own and the product's).  m: the constants and products 2 (3 where m is a code times its scale), x 2, the sum 1: at most
    6 u of the terms' sizes.  v: x^2 5, constant and product 2, sum 1: 8 u (a decoded root squared 3, product 2, sum 1).  The root 4 u and 2^-23 of its own = 6 u;
    times the bias' root 2, eps and sum 2: 10 u.  The quotient 4 u (2 ulp), times the step size 2: 16 u.  p * keep 3 u, the difference 1 u."""
    x = scale * g
    new_m = beta1 * m + (1 - beta1) * x
    em = 6 * U * (beta1 * m.abs() + (1 - beta1) * x.abs()) + 1e-44   # (the least subnormal number is 1.4e-45)
    new_v = beta2 * v + (1 - beta2) * x * x
    ev = 8 * U * new_v + 1e-44
    below = new_v.sqrt() / math.sqrt(1 - beta2 ** step) + eps
    size = lr / (1 - beta1 ** step)
    keep = 1 - lr * decay
    new_p = p * keep - size * new_m / below
    # ev counts twice where v is near the least number, for the root's sake: relative 1/2 of ev / v is in the 10 u for all other v
    slip = torch.where(new_v > 1e-37, 0.0, (ev.sqrt() / math.sqrt(1 - beta2 ** step)) / below)
    ep = 4 * U * p.abs() + size * (em + (16 * U + slip) * new_m.abs()) / below + U * new_p.abs()
    return new_p, new_m, new_v, ep, em, ev


def check_codes(codes, scales, value, err, word, root):
    """codes and scales against `value` (its binary32 form off by at most `err`), random bits `word`: the scale is the block's largest / 448, every code is the e4m3
    number that the rounding picks, unless `err` reaches over the border, where it may be the neighbour."""
    n = value.numel()
    pad = -n % BLOCK
    full, fe = torch.nn.functional.pad(value, (0, pad)).view(-1, BLOCK), torch.nn.functional.pad(err, (0, pad)).view(-1, BLOCK)
    top, off = full.abs().max(1).values, fe.max(1).values
    some = top > 1e-35
    got = scales.double()
    assert got.numel() == top.numel()
    assert ((got - torch.where(some, top / 448, 0.0)).abs() <= off / 448 + 2 * U * got + 1e-44).all()
    top = torch.where(some, top, 1.0)
    u = (full.abs() / top[:, None] * 448).reshape(-1)[:n]
    u = torch.where(some.repeat_interleave(BLOCK)[:n], u, 0.0)
    # u in binary32: the value's error, the largest one's, the quotient's, the product's and the added 2^-6's rounding
    eu = (fe / top[:, None] * 448).reshape(-1)[:n] + u * ((off / top).repeat_interleave(BLOCK)[:n] + 4 * U) + 2.0 ** -6 * 2 * U
    rnd = (word >> 16 if root else word & 0xFFFF).double() / 65536
    step = 2.0 ** (torch.log2(u.clamp(min=2.0 ** -6)).floor() - 3)
    at = u / step + rnd
    want = (at.floor() * step).clamp(max=448.0)
    if root:
        want = torch.where((u > 0) & (want == 0), 2.0 ** -9, want)
    have = codes.double().abs()
    near = (at - at.round()).abs() <= eu / step + 2.0 ** -30
    wrong = have != want
    assert not (wrong & ~near).any(), (have[wrong & ~near][:5], want[wrong & ~near][:5], u[wrong & ~near][:5])
    assert ((have - want).abs()[wrong] <= 2 * step[wrong]).all()   # the neighbour, also across a power of two
    assert near.double().mean() < 0.02 or n < 512                  # the border is met rarely, or this says nothing
    some_sign = have > 0
    assert (torch.sign(codes.double())[some_sign] == torch.sign(value)[some_sign]).all()


def route(x, topk, normalize):
    """One rank's rows in 64 bits: indices, weights, p, log of the sums, which rows count, and the relative error bound of p in binary32."""
    nan = x.isnan()
    clean = torch.where(nan, -math.inf, x)
    order = torch.sort(clean, dim=1, descending=True, stable=True).indices[:, :topk]
    chosen = torch.gather(clean, 1, order) > -math.inf
    top = clean.max(1, keepdim=True).values
    open_ = top > -math.inf
    safe = torch.where(open_, top, 0.0)
    e = torch.exp(x - safe)
    total = torch.where(open_, e.sum(1, keepdim=True), 1.0)
    p = e / total
    lse = torch.where(open_, safe + torch.log(total), 0.0)
    w = torch.where(chosen, torch.gather(p, 1, order), 0.0)
    if normalize:
        w = torch.where(chosen, w / w.sum(1, keepdim=True), 0.0)
    # __expf is off by 2 + 1.173 |d| ulp at d = x - top, the difference's rounding by d / 2 more; the sum by the same under p, where d is at most ln E
    # on average, and by its adds (a lane's 32 and 5 levels at most); the reciprocal and the product by 2
    d = torch.where(torch.isfinite(x), safe - x, 0.0)
    rel = 2 * U * (2 + 1.7 * d + 2 + 1.7 * math.log(x.shape[1]) + 37 + 2)
    return torch.where(chosen, order, -1), w, p, lse, open_[:, 0], rel


def losses(parts, E, topk, balance, z):
    """parts: (p, lse, indices, open) of the ranks of one group -> (losses, saved)."""
    n = float(sum(o.sum() for _, _, _, o in parts))
    c = sum(torch.bincount(i[i >= 0], minlength=E).double() for _, _, i, _ in parts)
    P = sum(p.sum(0) for p, _, _, _ in parts)
    Z = sum((l ** 2).sum() for _, l, _, _ in parts)
    if n == 0:
        return torch.zeros(2, dtype=torch.float64), torch.zeros(E + 1, dtype=torch.float64)
    f = c / (topk * n)
    return torch.stack([balance * E * (f * P).sum() / n, z * Z / n]), torch.cat([balance * E * f / n, torch.tensor([2 * z / n], dtype=torch.float64)])


def route_backward(x, indices, saved, dweights, dloss, normalize):
    """dlogits in 64 bits and a bound on their error in binary32."""
    E = x.shape[1]
    _, _, p, lse, open_, rel = route(x, 1, False)
    c, z = saved[:E] * dloss, saved[E] * dloss
    ok = (indices >= 0) & (indices < E)
    at = torch.where(ok, indices, 0).long()
    wide, wide_abs = torch.zeros_like(p), torch.zeros_like(p)
    shift = (p * c).sum(1, keepdim=True) - z * lse
    size = p * (c.abs() + (p * c.abs()).sum(1, keepdim=True) + (z * lse).abs())
    if dweights is not None:
        w = torch.where(ok, torch.gather(p, 1, at), 0.0)
        dw = torch.where(ok, dweights, 0.0)
        per = 1.0
        if normalize:
            s = w.sum(1, keepdim=True)
            per = torch.where(s > 0, 1 / s, 0.0)
        inner = (w * dw).sum(1, keepdim=True) * per
        inner_abs = (w * dw.abs()).sum(1, keepdim=True) * per
        wide.scatter_add_(1, at, w * per * (dw - (inner if normalize else 0.0)))
        wide_abs.scatter_add_(1, at, w * per * (dw.abs() + inner_abs))
        if not normalize:
            shift = shift + inner
            size = size + p * inner_abs
    d = torch.where(open_[:, None], p * (c - shift) + wide, 0.0)
    # products of up to three numbers off by `rel` (p, a weight's sum, a mean under p) and a few roundings
    return d, (4 * rel.max(1, keepdim=True).values + 16 * U) * (size + wide_abs) + 1e-44
