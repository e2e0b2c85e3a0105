"""The operators of a training step that stand beside the collectives: the AdamW step over many tensors (states in 32 or 8 bits), the
gradient norm with its clip factor, the step on ranks that each keep a shard of the optimizer's state, and the router of an
expert-parallel layer with its balance loss, forward and backward.  `run` computes them in plain torch operations or, where `own` is
true, through the library's public binding.
"""
from __future__ import annotations

import functools
import math
import random

import torch

own = False

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}
BETA1, BETA2, EPS, DECAY = 0.9, 0.95, 1e-8, 0.1
BLOCK = 256          # elements that share a scale in 8-bit states
MAX_NORM = 1.0
BALANCE, ZLOSS = 0.01, 0.001


def listed():
    return [
        # the norm weights and biases of a small model: latency
        dict(name="adamw_vectors", op="adamw", layout="vectors", tensors=48, width=4096, state="fp32", param="fp32", master=False, grad="fp32", odd=False, step=1),
        # one transformer layer of the benchmark's model (hidden 4096, FFN 16384): bf16 weights and gradients, fp32 master weights and states
        dict(name="adamw_layer", op="adamw", layout="layer", hidden=4096, ffn=16384, state="fp32", param="bf16", master=True, grad="bf16", odd=False, step=1000),
        # the same layer with states in 8 bits
        dict(name="adamw8_layer", op="adamw", layout="layer", hidden=4096, ffn=16384, state="8bit", param="bf16", master=True, grad="bf16", odd=False, step=1000),
        # tensors of many lengths, none a multiple of anything, packed into one buffer without alignment
        dict(name="adamw8_ragged", op="adamw", layout="ragged", tensors=96, low=1, high=1_500_000, state="8bit", param="bf16", master=False, grad="bf16", odd=True, step=20),
        # the norm of a layer's gradients, before they are clipped
        dict(name="norm_layer", op="norm", layout="layer", hidden=4096, ffn=16384, grad="bf16", odd=False),
        # the norm of many ragged fp32 gradients
        dict(name="norm_ragged", op="norm", layout="ragged", tensors=96, low=1, high=1_500_000, grad="fp32", odd=True),
        # a sharded optimizer's 25 MiB bucket over 8 ranks
        dict(name="sharded_25m", op="sharded", R=8, count=13_107_200, state="fp32", param="bf16", master=True, grad="bf16", step=1000),
        # a vector whose length is not a multiple of anything, fp32, 6 ranks
        dict(name="sharded_ragged_fp32_r6", op="sharded", R=6, count=500_009, state="8bit", param="fp32", master=False, grad="fp32", step=20),
        # serving: 8 ranks with a few tokens each
        dict(name="route_decode", op="route", R=8, tokens=16, experts=64, topk=6, dtype="bf16", normalize=True, per_rank=False, padded=0.0),
        # expert-parallel training: 4096 tokens a rank, as the exchange of expert-parallel dispatch has them, some of them padding
        dict(name="route_train", op="route", R=8, tokens=4096, experts=256, topk=8, dtype="fp32", normalize=True, per_rank=False, padded=0.05),
        # their gradient
        dict(name="route_backward_train", op="route_backward", R=8, tokens=4096, experts=256, topk=8, dtype="fp32", normalize=True, per_rank=False, padded=0.05),
        # an odd number of experts, few ranks, a loss of its own for every rank, weights as the softmax leaves them
        dict(name="route_backward_odd", op="route_backward", R=3, tokens=1777, experts=61, topk=2, dtype="bf16", normalize=False, per_rank=True, padded=0.1),
    ]


def _log_uniform(rng: random.Random, lo: float, hi: float) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["adamw", "adamw", "adamw", "norm", "norm", "sharded", "sharded", "route", "route", "route_backward", "route_backward"])
    if op in ("route", "route_backward"):
        experts = _log_uniform(rng, 4, 512)
        R = rng.choice([1, 2, 3, 4, 8, 8])
        tokens = _log_uniform(rng, 1, min(16384, 4_000_000 / (R * experts) * 2))
        return dict(op=op, R=R, tokens=tokens, experts=experts, topk=rng.randrange(1, min(8, experts) + 1), dtype=rng.choice(["bf16", "fp32"]),
                    normalize=rng.random() < 0.6, per_rank=rng.random() < 0.3, padded=rng.choice([0.0, 0.03, 0.3]))
    param = rng.choice(["bf16", "bf16", "fp32"])
    case = dict(op=op, state=rng.choice(["fp32", "8bit"]), param=param, master=param == "bf16" and rng.random() < 0.7, grad=rng.choice(["bf16", "fp32"]),
                step=_log_uniform(rng, 1, 100_000))
    if op == "sharded":
        case["R"] = R = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 8, 16])
        case["count"] = _log_uniform(rng, 1000, 100_000_000 / R) | rng.randrange(2)
        return case
    case["odd"] = rng.random() < 0.3
    layout = case["layout"] = rng.choice(["vectors", "layer", "ragged"])
    if layout == "vectors":
        case["tensors"], case["width"] = rng.randrange(1, 800), _log_uniform(rng, 16, 20_000)
    elif layout == "layer":
        case["hidden"] = _log_uniform(rng, 128, 3500)
        case["ffn"] = int(case["hidden"] * rng.uniform(2.5, 4.0))
    else:
        case["tensors"], case["low"], case["high"] = rng.randrange(2, 300), 1, _log_uniform(rng, 1000, 1_000_000)
    if op == "norm":
        for k in ("state", "param", "master", "step"):
            del case[k]
    return case


# ------------------------------------------------------------------------------------------------ what a program has in hand


def _counts(case):
    """Elements of each tensor."""
    if case["layout"] == "vectors":
        return [case["width"]] * case["tensors"]
    if case["layout"] == "layer":   # attention in and out, both FFN matrices, two norms' weights and biases
        h, f = case["hidden"], case["ffn"]
        return [3 * h * h, h * h, h * f, f * h, h, h, h, h]
    rng = random.Random(case["tensors"] * 1_000_003 + case["high"])
    return [_log_uniform(rng, case["low"], case["high"]) | 1 for _ in range(case["tensors"])]


def _offsets(counts, odd):
    """Places of the tensors in one buffer: 64-element boundaries, or one after the other."""
    at, out = int(odd), []
    for n in counts:
        out.append(at)
        at += n if odd else (n + 63) // 64 * 64
    return out, at


def _views(buf, offsets, counts):
    return [buf[o:o + n] for o, n in zip(offsets, counts)]


def _decays(counts):
    """Matrices are decayed, vectors are not."""
    return [DECAY if n > 20_000 else 0.0 for n in counts]


def _lr(case):
    return 2e-5


def _zeros(n, dt):
    return torch.zeros(n, dtype=dt, device="cuda")


def _blocks(counts, offsets, spare):
    """Where the elements of all tensors' blocks lie in the buffer, [blocks, BLOCK]: behind a tensor's end that is the spare place; which tensor each block
    belongs to, and the index of each element in it."""
    n, o = (torch.tensor(x, device="cuda") for x in (counts, offsets))
    per = (n + BLOCK - 1) // BLOCK
    tensor = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), per)
    index = (torch.arange(len(tensor), device="cuda") - (per.cumsum(0) - per)[tensor])[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    return dict(per=per.tolist(), tensor=tensor, index=index, place=torch.where(index < n[tensor][:, None], o[tensor][:, None] + index, spare))


def _prepare_adamw(case, normal):
    counts = _counts(case)
    offsets, total = _offsets(counts, case["odd"])
    s = dict(counts=counts, decays=_decays(counts), step=case["step"], seed=case["step"] * 77 + 5, total=total)
    # one place more than the tensors need: see _blocks
    wide = s["wide"] = {"param": normal(total + 1, 0.02).to(DT[case["param"]]), "grad": normal(total + 1, 1e-3).to(DT[case["grad"]])}
    first = case["step"] == 1   # the states start at zero
    m = _zeros(total + 1, torch.float32) if first else normal(total + 1, 2e-4)
    v = _zeros(total + 1, torch.float32) if first else (normal(total + 1, 1e-3).square() + 1e-8) * 0.5
    if case["master"]:
        wide["master"] = wide["param"].float()
    if case["state"] == "fp32":
        wide["m"], wide["v"] = m, v
    else:
        b = s["blocks"] = _blocks(counts, offsets, total)
        wide["m"], wide["v"] = (_zeros(total + 1, torch.float8_e4m3fn) for _ in range(2))
        s["flat_scales"] = {k: _zeros(len(b["tensor"]), torch.float32) for k in ("m_scale", "v_scale")}
        at = [sum(b["per"][:k]) for k in range(len(counts))]
        s.update({k: _views(f, at, b["per"]) for k, f in s["flat_scales"].items()})
        _scatter8(s, "m", m[b["place"]], 1, False)
        _scatter8(s, "v", v.sqrt()[b["place"]], 1, True)
    for k in wide:
        s[k] = _views(wide[k], offsets, counts)
    s["decay"] = torch.tensor(s["decays"], device="cuda")
    s["factor"] = torch.full((1,), 0.7, device="cuda")
    if own:
        from paper_2609_34334_b200 import binding as hb

        s["comm"] = _comm(8)
        s["table"] = hb.AdamTensors(s["param"], s["grad"], s["m"], s["v"], case["param"], case["grad"], state=case["state"], master=s.get("master"),
                                    exp_avg_scale=s.get("m_scale"), exp_avg_sq_scale=s.get("v_scale"), weight_decay=s["decays"])
    return s


def _prepare_norm(case, normal):
    counts = _counts(case)
    offsets, total = _offsets(counts, case["odd"])
    s = dict(counts=counts, grad=_views(normal(total, 1e-3).to(DT[case["grad"]]), offsets, counts), out=_zeros(2, torch.float32))
    if own:
        from paper_2609_34334_b200 import binding as hb

        s["comm"] = _comm(8, hb.grad_norm_scratch_bytes())
        s["table"] = hb.Tensors(s["grad"], case["grad"])
    return s


def _prepare_sharded(case, normal):
    """Rank r's gradients and weights are row r; its shard of the state (chunk r of q elements) is row r of the state's buffers."""
    R, n = case["R"], case["count"]
    q = (n + R - 1) // R
    pitch, room = (n + 63) // 64 * 64, (q + BLOCK - 1) // BLOCK * BLOCK
    s = dict(q=q, step=case["step"], seed=case["step"] * 77 + 5)
    s["grad"] = normal(R * pitch, 1e-3).to(DT[case["grad"]]).view(R, pitch)[:, :n]
    s["param"] = normal(pitch, 0.02).to(DT[case["param"]]).repeat(R, 1)[:, :n]
    if case["master"]:
        flat = _zeros(R * q, torch.float32)
        flat[:n] = s["param"][0].float()
        s["master"] = _zeros((R, room), torch.float32)
        s["master"][:, :q] = flat.view(R, q)
    inside = torch.zeros(R, room, dtype=torch.bool, device="cuda")
    inside[:, :q] = (torch.arange(R * q, device="cuda") < n).view(R, q)
    first = case["step"] == 1
    m, v = ((normal(R * room, sd).view(R, room) if not first else _zeros((R, room), torch.float32)).masked_fill(~inside, 0.0) for sd in (2e-4, 1e-3))
    v = (v.square() + (0.0 if first else 1e-8)).masked_fill(~inside, 0.0)
    if case["state"] == "fp32":
        s["m"], s["v"] = m, v
    else:
        s["m"], s["v"] = (_zeros((R, room), torch.float8_e4m3fn) for _ in range(2))
        s["m_scale"], s["v_scale"] = (_zeros((R, room // BLOCK), torch.float32) for _ in range(2))
        ranks = torch.arange(R, device="cuda")
        _store8_rows(m, s["m"], s["m_scale"], 1, ranks, False)
        _store8_rows(v.sqrt(), s["v"], s["v_scale"], 1, ranks, True)
    s["inside"] = inside
    if own:
        s["comm"] = _comm(R)
        for k in ("grad", "param", "master", "m", "v", "m_scale", "v_scale"):
            if k in s:
                s[k + "_rows"] = list(s[k])
    return s


def _prepare_route(case, normal):
    R, E, K, dt = case["R"], case["experts"], case["topk"], DT[case["dtype"]]
    # the ranks hold about as many tokens each
    tokens = [max(1, case["tokens"] - 3 * r) if case["tokens"] > 64 else case["tokens"] for r in range(R)]
    at = [sum(tokens[:r]) for r in range(R)]
    N = sum(tokens)
    logits = normal(N * E, 1.0).view(N, E) + normal(E, 0.5)   # some experts are more popular
    u = normal(N, 1.0)
    if case["padded"]:   # rows of padding: no expert is open to them
        logits.masked_fill_((u > -1.41421356 * _erfinv(2 * case["padded"] - 1))[:, None], -math.inf)
    s = dict(tokens=tokens, logits=logits.to(dt))
    s["rank"] = torch.repeat_interleave(torch.arange(R, device="cuda"), torch.tensor(tokens, device="cuda"))
    split = lambda t: [t[a:a + n] for a, n in zip(at, tokens)]  # noqa: E731
    groups = R if case["per_rank"] else 1
    if case["op"] == "route":
        s["indices"], s["weights"] = torch.zeros(N, K, dtype=torch.int32, device="cuda"), _zeros((N, K), torch.float32)
        s["counts"], s["loss"], s["saved"] = torch.zeros(R, E + 1, dtype=torch.int32, device="cuda"), _zeros((groups, 2), torch.float32), _zeros((groups, E + 1), torch.float32)
    else:
        f = _route_plain(case, s)
        s["indices"], s["saved"] = f["indices"], f["saved"]
        s["dweights"], s["dloss"] = normal(N * K, 1e-3).view(N, K), torch.full((groups,), 1.5, device="cuda")
        s["dlogits"] = torch.zeros(N, E, dtype=dt, device="cuda")
    if own:
        from paper_2609_34334_b200 import binding as hb

        s["comm"] = _comm(R, hb.route_scratch_bytes(R, max(tokens), E))
        for k in ("logits", "indices", "weights", "dweights", "dlogits"):
            if k in s:
                s[k + "_of"] = split(s[k])
        if "counts" in s:
            s["counts_of"] = list(s["counts"])
    return s


@functools.lru_cache(None)
def _comm(R, scratch=0):
    """A communicator as a program sets it up once, with the scratch that its operators ask for."""
    from paper_2609_34334_b200 import binding as hb

    comm = hb.Comm(R, torch.cuda.current_device())
    if scratch:
        comm.set_scratch(torch.empty(scratch, dtype=torch.uint8, device="cuda"), scratch)
    return comm


def _erfinv(x):
    return float(torch.erfinv(torch.tensor(x, dtype=torch.float64)))


def prepare(case, seed: int):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(n, scale):
        return torch.empty(n, dtype=torch.float32, device="cuda").normal_(0.0, scale, generator=g)

    op = case["op"]
    s = {"adamw": _prepare_adamw, "norm": _prepare_norm, "sharded": _prepare_sharded}.get(op, _prepare_route)(case, normal)
    s["case"] = case
    return s


# ------------------------------------------------------------------------------------------------ 8-bit states, plainly


def _hash(seed, tensor, index):
    """32 bits for each element: the finalizer of MurmurHash3 over (seed, tensor, element's index), twice.  `index` and `tensor`: int64 tensors or integers."""
    def mix(h):
        h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
        h = ((h ^ (h >> 13)) * 0xC2B2AE35) & 0xFFFFFFFF
        return h ^ (h >> 16)
    key = mix((seed + tensor * 0x9E3779B9) & 0xFFFFFFFF)
    return mix(((index & 0xFFFFFFFF) + key + (index >> 32) * 0x632BE5AB) & 0xFFFFFFFF)


def _round8(u, rnd, keep):
    """|u| <= 448 to the next e4m3 value below or above, above with the probability of the distance; rnd: 16 random bits as int32.
    keep: what is above zero stays above zero."""
    a = u.abs()
    normal = (((a.view(torch.int32) + (rnd << 4)) >> 20) << 20).view(torch.float32)
    small = torch.floor(a * 512 + rnd * (1.0 / 65536)) * (1.0 / 512)
    q = torch.where(a >= 2.0 ** -6, normal, small).clamp(max=448.0)
    if keep:
        q = torch.where((a > 0) & (q == 0), 2.0 ** -9, q)
    return torch.copysign(q, u)


def _store8_rows(x, codes, scales, seed, tensor, root, index=None):
    """x [T, multiple of BLOCK] -> codes, scales: block by block; tensor: T numbers; index: of each element in its tensor, the column if None."""
    T, n = x.shape
    top = x.view(T, -1, BLOCK).abs().amax(2)
    inv = torch.where(top > 1e-35, 448.0 / top, 0.0)
    scales.copy_(torch.where(top > 1e-35, top * (1.0 / 448.0), 0.0))
    h = _hash(seed, tensor[:, None], torch.arange(n, device=x.device)[None, :] if index is None else index)
    rnd = (h >> 16 if root else h & 0xFFFF).to(torch.int32)
    codes.copy_(_round8((x.view(T, -1, BLOCK) * inv[:, :, None]).view(T, n), rnd, root).to(torch.float8_e4m3fn))


def _scatter8(s, name, x, seed, root):
    """x [blocks, BLOCK] of all tensors -> the buffer's codes and the scales."""
    b, x = s["blocks"], torch.where(s["blocks"]["place"] < s["total"], x, 0.0)
    codes = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=x.device)
    _store8_rows(x, codes, s["flat_scales"][name + "_scale"].view(-1, 1), seed, b["tensor"], root, b["index"])
    s["wide"][name].view(torch.uint8).scatter_(0, b["place"].view(-1), codes.view(torch.uint8).view(-1))


# ------------------------------------------------------------------------------------------------ the plain forms


def _adamw_plain(case, s):
    t, lr = s["step"], _lr(case)
    if case["state"] == "8bit":
        return _adamw8_plain(case, s)
    P = s["master"] if case["master"] else [p.float() for p in s["param"]] if case["param"] == "bf16" else s["param"]
    G = torch._foreach_mul([g.float() for g in s["grad"]], s["factor"][0])
    M, V = s["m"], s["v"]
    torch._foreach_mul_(M, BETA1)
    torch._foreach_add_(M, G, alpha=1 - BETA1)
    torch._foreach_mul_(V, BETA2)
    torch._foreach_addcmul_(V, G, G, 1 - BETA2)
    below = torch._foreach_sqrt(V)
    torch._foreach_div_(below, math.sqrt(1 - BETA2 ** t))
    torch._foreach_add_(below, EPS)
    torch._foreach_mul_(P, [1 - lr * d for d in s["decays"]])
    torch._foreach_addcdiv_(P, M, below, -lr / (1 - BETA1 ** t))
    if case["param"] == "bf16":
        torch._foreach_copy_(s["param"], P)


def _adamw8_plain(case, s):
    """All tensors' blocks as the rows of one matrix."""
    t, lr, wide, b = s["step"], _lr(case), s["wide"], s["blocks"]
    place = b["place"]
    weights = wide["master" if case["master"] else "param"]
    G = wide["grad"][place].float() * s["factor"]
    M = wide["m"][place].float() * s["flat_scales"]["m_scale"][:, None]
    V = (wide["v"][place].float() * s["flat_scales"]["v_scale"][:, None]).square()
    M = M * BETA1 + G * (1 - BETA1)
    V = V * BETA2 + G * G * (1 - BETA2)
    root = V.sqrt()
    keep = 1 - lr * s["decay"][b["tensor"]][:, None]
    P = weights[place].float() * keep - M / (root / math.sqrt(1 - BETA2 ** t) + EPS) * (lr / (1 - BETA1 ** t))
    if case["master"]:
        wide["master"].scatter_(0, place.view(-1), P.view(-1))
    wide["param"].scatter_(0, place.view(-1), P.view(-1).to(wide["param"].dtype))
    _scatter8(s, "m", M, s["seed"], False)
    _scatter8(s, "v", root, s["seed"], True)


def _norm_plain(case, s):
    norms = torch.cat(s["grad"]).double().square().sum().sqrt()
    s["out"][0] = norms
    s["out"][1] = (MAX_NORM / (norms + 1e-6)).clamp(max=1.0)


def _sharded_plain(case, s):
    R, n, q, t, lr = case["R"], case["count"], s["q"], s["step"], _lr(case)
    G = torch.zeros(R * q, device="cuda")
    G[:n] = s["grad"].float().sum(0) * (1.0 / R)
    G = G.view(R, q)
    P = torch.zeros(R * q, device="cuda")
    if case["master"]:
        P = s["master"][:, :q].clone()
    else:
        P[:n] = s["param"][0].float()
        P = P.view(R, q)
    eight = case["state"] == "8bit"
    if eight:
        M, V = ((s[k].float().view(R, -1, BLOCK) * s[k + "_scale"][:, :, None]).view(R, -1) for k in ("m", "v"))
        V = V.square()
    else:
        M, V = s["m"], s["v"]
    M, V = M[:, :q], V[:, :q]
    M = M * BETA1 + G * (1 - BETA1)
    V = V * BETA2 + G * G * (1 - BETA2)
    root = V.sqrt()
    P = P * (1 - lr * DECAY) - M / (root / math.sqrt(1 - BETA2 ** t) + EPS) * (lr / (1 - BETA1 ** t))
    inside = s["inside"]
    if case["master"]:
        s["master"][:, :q] = torch.where(inside[:, :q], P, s["master"][:, :q])
    s["param"].copy_(P.reshape(-1)[:n].to(s["param"].dtype).expand(R, n))
    if eight:
        full = torch.zeros(2, R, inside.shape[1], device="cuda")
        full[0, :, :q], full[1, :, :q] = M, root
        full = full.masked_fill(~inside, 0.0)
        ranks = torch.arange(R, device="cuda")
        _store8_rows(full[0], s["m"], s["m_scale"], s["seed"], ranks, False)
        _store8_rows(full[1], s["v"], s["v_scale"], s["seed"], ranks, True)
    else:
        s["m"][:, :q] = torch.where(inside[:, :q], M, s["m"][:, :q])
        s["v"][:, :q] = torch.where(inside[:, :q], V, s["v"][:, :q])


def _probabilities(x):
    """softmax of the rows and log of their sums; rows with no open expert: zeros."""
    top = x.amax(1, keepdim=True)
    open_ = top > -math.inf
    top = torch.where(open_, top, 0.0)
    e = torch.exp(x - top)
    total = torch.where(open_, e.sum(1, keepdim=True), 1.0)
    return e / total, torch.where(open_, top + torch.log(total), 0.0), open_


def _route_plain(case, s):
    R, E, K = case["R"], case["experts"], case["topk"]
    x = s["logits"].float()
    p, lse, open_ = _probabilities(x)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :K]   # of equal logits the lowest index first
    chosen = torch.gather(x, 1, order) > -math.inf
    indices = torch.where(chosen, order, -1)
    w = torch.gather(p, 1, order) * chosen
    if case["normalize"]:
        w = w / torch.where(open_, w.sum(1, keepdim=True), 1.0)
    rank = s["rank"]
    groups = R if case["per_rank"] else 1
    group = rank if case["per_rank"] else torch.zeros_like(rank)
    flat = torch.cat([(rank[:, None] * (E + 1) + order)[chosen], (rank * (E + 1) + E)[open_[:, 0]]])
    counts = torch.bincount(flat, minlength=R * (E + 1)).view(R, E + 1)
    c = counts if case["per_rank"] else counts.sum(0, keepdim=True)
    n = c[:, E:].double().clamp(min=1)
    f = c[:, :E] / (K * n)
    P = torch.zeros(groups, E, dtype=torch.float64, device="cuda").index_add_(0, group, p.double())
    Z = torch.zeros(groups, 1, dtype=torch.float64, device="cuda").index_add_(0, group, lse.double().square())
    loss = torch.cat([BALANCE * E * (f * P / n).sum(1, keepdim=True), ZLOSS * Z / n], 1)
    saved = torch.cat([BALANCE * E * f / n, torch.where(c[:, E:] > 0, 2 * ZLOSS / n, 0.0)], 1)
    return {"indices": indices.to(torch.int32), "weights": w, "counts": counts.to(torch.int32), "loss": loss.float(), "saved": saved.float()}


def _route_backward_plain(case, s):
    E = case["experts"]
    p, lse, open_ = _probabilities(s["logits"].float())
    group = s["rank"] if case["per_rank"] else torch.zeros_like(s["rank"])
    c, z = s["saved"][:, :E][group], s["saved"][:, E:][group]
    scale = s["dloss"][group][:, None]
    chosen = s["indices"] >= 0
    at = s["indices"].clamp(min=0).long()
    dw = torch.where(chosen, s["dweights"], 0.0)
    w = torch.gather(p, 1, at) * chosen
    if case["normalize"]:
        w = w / torch.where(open_, w.sum(1, keepdim=True), 1.0)
        d = torch.zeros_like(p).scatter_add_(1, at, w * (dw - (w * dw).sum(1, keepdim=True)))
    else:
        inner = torch.zeros_like(p).scatter_add_(1, at, dw)
        d = p * (inner - (w * dw).sum(1, keepdim=True))
    d = d + scale * p * (c - (p * c).sum(1, keepdim=True) + z * lse)
    return d.to(s["logits"].dtype)


# ------------------------------------------------------------------------------------------------ one pass


def _adamw_outputs(s):
    return {**{k: v[:s["total"]] for k, v in s["wide"].items() if k != "grad"}, **s.get("flat_scales", {})}


def run(s):
    case = s["case"]
    op = case["op"]
    if op == "adamw":
        if own:
            s["comm"].adamw(s["table"], _lr(case), s["step"], beta1=BETA1, beta2=BETA2, eps=EPS, factor=s["factor"], seed=s["seed"])
        else:
            _adamw_plain(case, s)
        return _adamw_outputs(s)
    if op == "norm":
        if own:
            s["comm"].grad_norm(s["table"], s["out"], max_norm=MAX_NORM)
        else:
            _norm_plain(case, s)
        return s["out"]
    if op == "sharded":
        if own:
            s["comm"].sharded_adamw(s["grad_rows"], s["param_rows"], s["m_rows"], s["v_rows"], case["count"], case["param"], case["grad"], _lr(case), s["step"],
                                    state=case["state"], master=s.get("master_rows"), exp_avg_scale=s.get("m_scale_rows"), exp_avg_sq_scale=s.get("v_scale_rows"),
                                    beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY, grad_scale=1.0 / case["R"], seed=s["seed"])
        else:
            _sharded_plain(case, s)
        return {k: s[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale") if k in s}
    if op == "route":
        if not own:
            return _route_plain(case, s)
        s["comm"].route(s["logits_of"], s["tokens"], case["experts"], case["topk"], case["dtype"], s["indices_of"], s["weights_of"], s["counts_of"], s["loss"], s["saved"],
                        balance_coef=BALANCE, z_coef=ZLOSS, normalize=case["normalize"], per_rank=case["per_rank"])
        return {k: s[k] for k in ("indices", "weights", "counts", "loss", "saved")}
    if not own:
        return _route_backward_plain(case, s)
    s["comm"].route_backward(s["logits_of"], s["tokens"], case["experts"], case["topk"], case["dtype"], s["indices_of"], s["saved"], s["dweights_of"], s["dloss"],
                             s["dlogits_of"], normalize=case["normalize"], per_rank=case["per_rank"])
    return s["dlogits"]


def work(case):
    op = case["op"]
    if op == "norm":
        n = sum(_counts(case))
        return {"bytes": n * BYTES[case["grad"]] + 8, "flops": 2 * n}
    if op in ("adamw", "sharded"):
        R = case.get("R", 1)
        n = case["count"] if op == "sharded" else sum(_counts(case))
        state = 16 if case["state"] == "fp32" else 4 + 16 / BLOCK
        weight = R * BYTES[case["param"]] + (8 if case["master"] else BYTES[case["param"]])
        return {"bytes": n * (R * BYTES[case["grad"]] + state + weight), "flops": n * (14 + R)}
    n = sum(max(1, case["tokens"] - 3 * r) if case["tokens"] > 64 else case["tokens"] for r in range(case["R"]))
    E, K, e = case["experts"], case["topk"], BYTES[case["dtype"]]
    if op == "route":
        return {"bytes": n * (E * e + 8 * K) + case["R"] * (E + 1) * 4, "flops": 5 * n * E}
    return {"bytes": n * (2 * E * e + 8 * K), "flops": 8 * n * E}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits


def _exact_hash(seed, tensor, n):
    """As unsigned 32-bit words: h ^= h >> 16, times 85EBCA6B, h ^= h >> 13, times C2B2AE35, h ^= h >> 16, of the key and of key + index."""
    word = 2 ** 32
    h = torch.tensor((seed + tensor * 0x9E3779B9) % word, device="cuda")
    keyed = None
    for _ in range(2):
        for shift, factor in ((16, 0x85EBCA6B), (13, 0xC2B2AE35)):
            h = torch.remainder(torch.bitwise_xor(h, torch.div(h, 2 ** shift, rounding_mode="floor")) * factor, word)
        h = torch.bitwise_xor(h, torch.div(h, 65536, rounding_mode="floor"))
        if keyed is None:
            keyed = h
            h = torch.remainder(torch.arange(n, device="cuda") + keyed, word)
    return h


def _exact_store8(x, rnd, root):
    """(codes' values, scales): x in 64 bits, rnd in [0, 1)."""
    n = x.numel()
    full = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    scale = full.abs().max(1).values / 448
    u = torch.where(scale[:, None] > 0, full / scale[:, None], 0.0).reshape(-1)[:n]
    step = 2.0 ** (torch.log2(u.abs().clamp(min=2.0 ** -6)).floor() - 3)
    q = ((u.abs() / step + rnd).floor() * step).clamp(max=448)
    if root:
        q = torch.where((u > 0) & (q == 0), 2.0 ** -9, q)
    return q * u.sign(), scale


def _exact_adamw(p, g, m, v, t, lr, decay):
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    return p - lr * decay * p - lr * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS), m, v


def _exact_tensor(case, s, k, p, g, m, v, m_scale, v_scale, decay):
    """New (weights, states) of one tensor; 8-bit states come and go as codes and scales."""
    if case["state"] == "8bit":
        spread = lambda c, sc: c.double() * sc.double()[torch.arange(c.numel(), device="cuda") // BLOCK]  # noqa: E731
        m, v = spread(m, m_scale), spread(v, v_scale) ** 2
    p, m, v = _exact_adamw(p.double(), g, m.double(), v.double(), s["step"], _lr(case), decay)
    if case["state"] == "fp32":
        return p, (m, v)
    h = _exact_hash(s["seed"], k, m.numel())
    return p, (*_exact_store8(m, (h % 65536) / 65536, False), *_exact_store8(v.sqrt(), torch.div(h, 65536, rounding_mode="floor") / 65536, True))


def exact(case, seed: int):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        n = math.sqrt(sum(float((g.double() ** 2).sum()) for g in s["grad"]))
        return torch.tensor([n, min(1.0, MAX_NORM / (n + 1e-6))], dtype=torch.float64)
    if op == "adamw":
        out = {k: t.double() for k, t in _adamw_outputs(s).items()}
        offsets, _ = _offsets(s["counts"], case["odd"])
        at = 0
        for k, (o, n) in enumerate(zip(offsets, s["counts"])):
            blocks = (n + BLOCK - 1) // BLOCK
            scales = (s["m_scale"][k], s["v_scale"][k]) if case["state"] == "8bit" else (None, None)
            p, state = _exact_tensor(case, s, k, s["master" if case["master"] else "param"][k], s["grad"][k].double() * s["factor"].double(), s["m"][k], s["v"][k], *scales,
                                     s["decays"][k])
            out["param"][o:o + n] = p
            if case["master"]:
                out["master"][o:o + n] = p
            if case["state"] == "fp32":
                out["m"][o:o + n], out["v"][o:o + n] = state
            else:
                out["m"][o:o + n], out["m_scale"][at:at + blocks], out["v"][o:o + n], out["v_scale"][at:at + blocks] = state
            at += blocks
        return out
    if op == "sharded":
        R, N, q = case["R"], case["count"], s["q"]
        out = {k: s[k].double().clone() for k in ("param", "master", "m", "v", "m_scale", "v_scale") if k in s}
        for c in range(R):
            lo, hi = min(c * q, N), min((c + 1) * q, N)
            n = hi - lo
            if not n:
                continue
            g = sum(s["grad"][r, lo:hi].double() for r in range(R)) / R
            blocks = (n + BLOCK - 1) // BLOCK
            scales = (s["m_scale"][c, :blocks], s["v_scale"][c, :blocks]) if case["state"] == "8bit" else (None, None)
            p, state = _exact_tensor(case, s, c, s["master"][c, :n] if case["master"] else s["param"][c, lo:hi], g, s["m"][c, :n], s["v"][c, :n], *scales, DECAY)
            out["param"][:, lo:hi] = p
            if case["master"]:
                out["master"][c, :n] = p
            if case["state"] == "fp32":
                out["m"][c, :n], out["v"][c, :n] = state
            else:
                out["m"][c, :n], out["m_scale"][c, :blocks], out["v"][c, :n], out["v_scale"][c, :blocks] = state
        return out
    # the router, rank by rank
    R, E, K = case["R"], case["experts"], case["topk"]
    weights, parts, dx, at = [], [], [], 0
    for r, n in enumerate(s["tokens"]):
        x = s["logits"][at:at + n].double()
        real = (x > -math.inf).any(1)
        lse = torch.logsumexp(x, 1)
        p = torch.where(real[:, None], torch.exp(x - lse[:, None]), 0.0)
        lse = torch.where(real, lse, 0.0)
        # the K largest, found by counting for each logit the ones in front of it
        if op == "route":
            got = torch.topk(x, K, dim=1).values
            w = torch.where(got > -math.inf, torch.exp(got - lse[:, None]), 0.0)
            weights.append(w / w.sum(1, keepdim=True).clamp(min=1e-300) if case["normalize"] else w)
            chosen = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :K][got > -math.inf]
            parts.append((torch.bincount(chosen, minlength=E).double(), p.sum(0), (lse ** 2).sum(), real.sum().double()))
        else:
            i, dw = s["indices"][at:at + n].long(), s["dweights"][at:at + n].double()
            saved, scale = s["saved"][r if case["per_rank"] else 0].double(), s["dloss"][r if case["per_rank"] else 0].double()
            hit = torch.zeros(n, E + 1, dtype=torch.float64, device="cuda").scatter_(1, torch.where(i < 0, E, i), 1.0)[:, :E]
            up = torch.zeros(n, E + 1, dtype=torch.float64, device="cuda").scatter_(1, torch.where(i < 0, E, i), dw)[:, :E]
            wide = p * hit
            if case["normalize"]:
                wide = wide / wide.sum(1, keepdim=True).clamp(min=1e-300)
                d = wide * (up - (wide * up).sum(1, keepdim=True))
            else:
                d = p * (up - (p * up).sum(1, keepdim=True))
            dx.append(d + scale * (p * (saved[:E] - (p @ saved[:E])[:, None]) + saved[E] * lse[:, None] * p))
        at += n
    if op == "route_backward":
        return torch.cat(dx)
    if not case["per_rank"]:
        parts = [tuple(sum(x) for x in zip(*parts))]
    loss, saved = [], []
    for c, P, Z, n in parts:
        n1 = n.clamp(min=1)
        f = c / (K * n1)
        loss.append(torch.stack([BALANCE * E * (f * P).sum() / n1, ZLOSS * Z / n1]))
        saved.append(torch.cat([BALANCE * E * f / n1, (2 * ZLOSS / n1 * (n > 0)).view(1)]))
    return {"indices": None, "weights": torch.cat(weights), "counts": None, "loss": torch.stack(loss), "saved": torch.stack(saved)}
