"""The operators of tuning a router on which speed is measured: balance loss, gradients, clipping.

A case is one call of an operator on one accumulated batch, as a program makes it that tunes the gate matrix of
an MoE layer while its experts stay as they are: the balance loss with its gradient, the gradient of the router,
the gradient of the weighted combine, and the clipping of the gradients of all tuned tensors.  The shapes are the
layer shapes of workloads/configs.py.  With `own` false every operator is computed in elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

# H, F, E, k, renormalised weights, gate bias (log of a Zipf(1.1) law over a random ranking)
SHAPES = {
    "tiny": (512, 1024, 8, 2, True, False),
    "8x7b": (4096, 14336, 8, 2, True, False),
    "8x22b": (6144, 16384, 8, 2, True, False),
    "lite": (2048, 1408, 64, 6, False, False),
    "v2": (5120, 1536, 160, 6, False, True),
}


def _case(op, shape, T, **options):
    H, F, E, k, renorm, zipf = SHAPES[shape]
    case = {"op": op, "T": T, "H": H, "E": E, "k": k, "renorm": renorm, "zipf": zipf, "padding": False}
    case.update(options)
    return case


def _balance(shape, T, z=True, grad=True, **options):
    return _case("balance", shape, T, z=z, grad=grad, **options)


def _route(shape, T, dlogits=True, accumulate=False, **options):
    return _case("route", shape, T, dlogits=dlogits, accumulate=accumulate, **options)


def _combine(shape, T, y_fp32=True, dout_fp32=False, dy=True, **options):
    return _case("combine", shape, T, y_fp32=y_fp32, dout_fp32=dout_fp32, dy=dy, **options)


def _clip(layers, H, E, experts=0, F=64, ratio=0.3):
    """Gradients of `layers` gates (fp32 matrix and bias), and of `experts` experts' three matrices (bf16); the
    clipped norm is `ratio` of the norm that standard normal gradients have."""
    return {"op": "clip", "layers": layers, "H": H, "E": E, "experts": experts, "F": F, "ratio": ratio}


def listed():
    cases = [
        # One small batch: the loss and its gradient are a few microseconds of work, launches count.
        ("balance_tiny_256", _balance("tiny", 256)),
        # A ragged accumulated batch of a layer with many narrow experts, padding rows among it.
        ("balance_lite_5003", _balance("lite", 5003, padding=True)),
        # The largest batch and most experts, skewed routing: what the loss is for.
        ("balance_v2_32768", _balance("v2", 32768)),
        # The smallest layer's router: a short step in a latency-bound loop.
        ("route_tiny_256", _route("tiny", 256)),
        # Few experts under a long batch: bound by reading x and writing its gradient.
        ("route_8x22b_16384", _route("8x22b", 16384)),
        # Ragged, with padding, the gate's gradient added to that of earlier micro-batches.
        ("route_lite_3001", _route("lite", 3001, accumulate=True, padding=True)),
        # The largest router: two matrix products in which neither side is small.
        ("route_v2_32768", _route("v2", 32768)),
        # Ragged batch, six fp32 rows a token, gradient of the weights alone (frozen experts).
        ("combine_lite_3001", _combine("lite", 3001, dout_fp32=True, dy=False)),
        # Two wide rows a token and the gradient of the experts' outputs.
        ("combine_8x7b_4096", _combine("8x7b", 4096)),
        # The largest combine, expert outputs kept in bf16.
        ("combine_v2_32768", _combine("v2", 32768, y_fp32=False)),
        # The gates of a small model: few short tensors, three dependent steps.
        ("clip_tiny_gates", _clip(4, 512, 8)),
        # A layer's experts beside all gates of the model: hundreds of tensors, a gigabyte.
        ("clip_lite_experts", _clip(26, 2048, 64, experts=66, F=1408)),
    ]
    return [dict(c, name=n) for n, c in cases]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes spread over their logarithms, odd ones among them, options at random."""
    op = rng.choice(["balance", "route", "route", "combine", "combine", "clip"])
    if op == "clip":
        H, E = 64 * _log_int(rng, 1, 80), rng.randint(3, 160)
        experts = rng.choice([0, _log_int(rng, 1, 40)])
        return _clip(_log_int(rng, 1, 60), H, E, experts, 64 * _log_int(rng, 1, 24), ratio=rng.choice([0.1, 0.7, 2.0]))
    if rng.random() < 0.5:
        case = _case(op, rng.choice(sorted(SHAPES)), 1)
    else:
        case = _case(op, "lite", 1, H=64 * _log_int(rng, 2, 96), E=_log_int(rng, 4, 256), renorm=rng.random() < 0.5,
                     zipf=rng.random() < 0.3)
        case["k"] = rng.randint(2 if case["renorm"] else 1, min(8, case["E"] - 1))   # one renormalised weight has no gradient
    H, E, k = case["H"], case["E"], case["k"]
    # no more work than the largest listed case of the operator
    most = {"balance": 32768 * 160 // E, "route": min(32768 * 5120 // H, 32768 * 5120 * 160 // (H * E)),
            "combine": 32768 * 6 * 5120 // (k * H) // 2}[op]
    case["T"] = _log_int(rng, 1, min(most, 32768))
    case["padding"] = op != "combine" and rng.random() < 0.3
    if op == "balance":
        # few picks can be exactly even, and the balance loss then has no gradient
        case.update(z=rng.random() < 0.7 or case["T"] < 64, grad=rng.random() < 0.8)
    elif op == "route":
        case.update(dlogits=rng.random() < 0.7, accumulate=rng.random() < 0.3)
    else:
        case.update(y_fp32=rng.random() < 0.5, dout_fp32=rng.random() < 0.5, dy=rng.random() < 0.5)
    return case


BALANCE_COEF, Z_COEF = 1e-2, 1e-3


class _State:
    """What a program holds before the call."""


def _inputs(case, seed):
    """The inputs of a seed."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = _State()
    s.case = case

    def normal(shape, dtype=torch.float32, std=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    if case["op"] == "clip":
        gate, matrix = case["H"] * case["E"], case["H"] * case["F"]
        sizes32 = [n for _ in range(case["layers"]) for n in (gate, case["E"])]
        sizes16 = [matrix] * (3 * case["experts"])
        s.flat32, s.flat16 = normal(sum(sizes32)), normal(sum(sizes16), torch.bfloat16)
        s.grads = list(s.flat32.split(sizes32)) + (list(s.flat16.split(sizes16)) if sizes16 else [])
        s.max_norm = case["ratio"] * math.sqrt(sum(sizes32) + sum(sizes16))
        return s
    T, H, E, k = (case[n] for n in ("T", "H", "E", "k"))
    s.keep = torch.rand(T, device="cuda", generator=gen) < 0.8 if case["padding"] else None
    if case["op"] == "combine":
        y_type, dout_type = (torch.float32 if case[n] else torch.bfloat16 for n in ("y_fp32", "dout_fp32"))
        s.dout, s.y_perm = normal((T, H), dout_type), normal((T * k, H), y_type)
        s.topk_w = torch.softmax(normal((T, k)), dim=1)
        s.inv_perm = torch.randperm(T * k, device="cuda", generator=gen).int()
        return s
    # logits as a router of N(0,1) hidden states and N(0, 0.02^2) weights has them
    s.x, s.wg = normal((T, H), torch.bfloat16), normal((H, E), torch.bfloat16, 0.02)
    s.logits = normal((T, E), std=0.02 * math.sqrt(H))
    if case["zipf"]:
        s.logits -= 1.1 * torch.log(torch.randperm(E, device="cuda", generator=gen).float() + 1.0)
    s.topk_idx = s.logits.topk(k, dim=1).indices.int()
    if case["op"] == "route":
        s.dtopk_w = normal((T, k), std=1.0 / T)
        s.dlogits = normal((T, E), std=0.01 / T) if case["dlogits"] else None
        s.dwg0, s.dbias0 = (normal((H, E)), normal(E)) if case["accumulate"] else (None, None)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:   # the context, the scratch, the list of tensors and the buffers that a program keeps from step to step
        from paper_2503_09716_amd import Moe, make_shape
        s.moe = moe = Moe(0)
        if case["op"] == "clip":
            s.out32, s.out16 = torch.empty_like(s.flat32), torch.empty_like(s.flat16)
            sizes32, sizes16 = ([g.numel() for g in s.grads if g.dtype == d] for d in (torch.float32, torch.bfloat16))
            outs = list(s.out32.split(sizes32)) + (list(s.out16.split(sizes16)) if sizes16 else [])
            s.list = moe.gradient_list(s.grads, outs)
            s.norm = torch.empty(1, device="cuda")
        else:
            T, H, E, k = (case[n] for n in ("T", "H", "E", "k"))
            s.shape = make_shape(T, H, 64, E, k, 0, case["renorm"])
            f32 = dict(dtype=torch.float32, device="cuda")
            if case["op"] == "combine":
                moe.set_option("y_fp32", int(case["y_fp32"]))
                moe.set_option("out_fp32", int(case["dout_fp32"]))
                s.dtopk_w = torch.empty((T, k), **f32)
                s.dy_perm = torch.empty_like(s.y_perm) if case["dy"] else None
            else:
                s.workspace = moe.new_backward_workspace(s.shape)
            if case["op"] == "balance":
                s.counts, s.loss = torch.empty(E, dtype=torch.int32, device="cuda"), torch.empty(2, **f32)
                s.dlogits = torch.empty((T, E), **f32) if case["grad"] else None
            if case["op"] == "route":
                s.dx, s.dwg, s.dbias = torch.empty_like(s.x), torch.empty((H, E), **f32), torch.empty(E, **f32)
    torch.cuda.synchronize()
    return s


def run(s):
    return {"balance": _run_balance, "route": _run_route, "combine": _run_combine, "clip": _run_clip}[s.case["op"]](s)


def _kept(s, v):
    """v with zeros in the rows of padding tokens."""
    return v if s.keep is None else torch.where(s.keep[:, None], v, torch.zeros_like(v))


def _run_balance(s):
    case = s.case
    z_coef = Z_COEF if case["z"] else 0.0
    if own:
        s.moe.balance_loss(s.shape, s.logits, s.topk_idx, s.keep, BALANCE_COEF, z_coef, s.counts, s.loss, s.dlogits, s.workspace)
        out = {"counts": s.counts, "loss": s.loss}
        return dict(out, dlogits=s.dlogits) if case["grad"] else out
    T, E, k = case["T"], case["E"], case["k"]
    logits = _kept(s, s.logits)
    keep = torch.ones(T, device="cuda") if s.keep is None else s.keep.float()
    n = keep.sum().clamp(min=1.0)
    top = logits.amax(dim=1, keepdim=True)
    p = torch.exp(logits - top)
    z = p.sum(dim=1, keepdim=True)
    p = p / z * keep[:, None]
    lse = (top + torch.log(z)) * keep[:, None]
    picks = keep.int()[:, None].expand(T, k).reshape(-1)
    counts = torch.zeros(E, dtype=torch.int32, device="cuda").scatter_add_(0, s.topk_idx.flatten().long(), picks)
    share = counts.float() / (k * n)
    loss = torch.stack([E * (share * p.sum(dim=0)).sum() / n, lse.square().sum() / n])
    if not case["grad"]:
        return {"counts": counts, "loss": loss}
    # the shares less their mean: that is what a gradient of nearly even shares hangs on
    off = ((counts.double() * E - k * n.double()) / (k * n.double())).float()
    dlogits = p * ((off - (p * off).sum(dim=1, keepdim=True)) * (BALANCE_COEF / n) + lse * (2.0 * z_coef / n))
    return {"counts": counts, "loss": loss, "dlogits": dlogits}


def _run_route(s):
    case = s.case
    if own:
        if case["accumulate"]:   # a program adds to its own sums; here they start from the same values every time
            s.dwg.copy_(s.dwg0)
            s.dbias.copy_(s.dbias0)
        s.moe.route_backward(s.shape, s.x, s.wg, s.logits, s.topk_idx, s.dtopk_w, s.dlogits, s.keep, s.dx, s.dwg, s.dbias,
                             case["accumulate"], s.workspace)
        return {"dx": s.dx, "dwg": s.dwg, "dbias": s.dbias}
    logits, x = _kept(s, s.logits), _kept(s, s.x).float()
    idx = s.topk_idx.long()
    g = torch.zeros_like(logits).scatter_(1, idx, s.dtopk_w)
    if case["renorm"]:   # weights are a softmax over the picks
        picked = torch.zeros_like(logits).scatter_(1, idx, 1.0)
        logits = torch.where(picked > 0, logits, torch.full_like(logits, -math.inf))
    p = torch.exp(logits - logits.amax(dim=1, keepdim=True))
    p = p / p.sum(dim=1, keepdim=True)
    dl = p * (g - (g * p).sum(dim=1, keepdim=True))
    dl = _kept(s, dl if s.dlogits is None else dl + s.dlogits)
    dx = (dl @ s.wg.float().t()).to(s.x.dtype)
    dwg, dbias = x.t() @ dl, dl.sum(dim=0)
    if case["accumulate"]:
        dwg, dbias = s.dwg0 + dwg, s.dbias0 + dbias
    return {"dx": dx, "dwg": dwg, "dbias": dbias}


def _run_combine(s):
    case = s.case
    if own:
        s.moe.combine_backward(s.shape, s.dout, s.y_perm, s.inv_perm, s.topk_w, s.dtopk_w, s.dy_perm)
        return {"dtopk_w": s.dtopk_w, "dy_perm": s.dy_perm} if case["dy"] else {"dtopk_w": s.dtopk_w}
    T, H, k = case["T"], case["H"], case["k"]
    rows = s.inv_perm.long()
    dout = s.dout.float()[:, None, :]
    out = {"dtopk_w": (s.y_perm[rows].view(T, k, H).float() * dout).sum(dim=2)}
    if case["dy"]:
        out["dy_perm"] = torch.empty_like(s.y_perm)
        out["dy_perm"][rows] = (s.topk_w[:, :, None] * dout).to(s.y_perm.dtype).view(T * k, H)
    return out


def _run_clip(s):
    if own:
        s.moe.clip_gradients(s.list, s.max_norm, s.norm)
        return {"norm": s.norm, "fp32": s.out32, "bf16": s.out16}
    norm = torch.stack([g.float().square().sum() for g in s.grads]).double().sum().sqrt().float().view(1)
    scale = torch.where(norm > s.max_norm, s.max_norm / norm, torch.ones_like(norm))
    scaled = [(g.float() * scale).to(g.dtype) for g in s.grads]
    by_type = [[g for g in scaled if g.dtype == d] for d in (torch.float32, torch.bfloat16)]
    return {"norm": norm, "fp32": torch.cat(by_type[0]), "bf16": torch.cat(by_type[1]) if by_type[1] else s.flat16}


def exact(case, seed):
    """The same from the definitions in 64 bits: the losses and the layer's formulas differentiated by autograd."""
    s = _inputs(case, seed)
    if case["op"] == "clip":
        norm = (s.flat32.double().square().sum() + s.flat16.double().square().sum()).sqrt()
        scale = min(1.0, s.max_norm / norm.item())
        return {"norm": norm.view(1), "fp32": s.flat32.double() * scale, "bf16": s.flat16.double() * scale}
    T, E, k = case["T"], case["E"], case["k"]
    if case["op"] == "combine":
        y, w = s.y_perm.double().requires_grad_(), s.topk_w.double().requires_grad_()
        out = sum(w[:, j, None] * y[s.inv_perm.view(T, k)[:, j].long()] for j in range(k))
        dw, dy = torch.autograd.grad(out, (w, y), s.dout.double())
        return {"dtopk_w": dw, "dy_perm": dy} if case["dy"] else {"dtopk_w": dw}
    kept = torch.arange(T, device="cuda") if s.keep is None else s.keep.nonzero().flatten()
    n, idx = kept.numel(), s.topk_idx[kept].long()
    leaf = s.logits.double().requires_grad_()
    logits = leaf[kept]
    if case["op"] == "balance":
        counts = torch.bincount(idx.flatten(), minlength=E)
        probs = torch.softmax(logits, dim=1)
        balance = E * ((counts.double() / max(k * n, 1)) * (probs.sum(dim=0) / max(n, 1))).sum()
        z = torch.logsumexp(logits, dim=1).square().sum() / max(n, 1)
        out = {"counts": counts, "loss": torch.stack([balance, z]).detach()}
        if case["grad"]:
            total = BALANCE_COEF * balance + (Z_COEF if case["z"] else 0.0) * z
            out["dlogits"] = torch.autograd.grad(total, leaf)[0]
        return out
    w = torch.softmax(logits, dim=1).gather(1, idx)
    if case["renorm"]:
        w = w / w.sum(dim=1, keepdim=True)
    value = (w * s.dtopk_w[kept].double()).sum()
    if s.dlogits is not None:
        value = value + (logits * s.dlogits[kept].double()).sum()
    dl = torch.autograd.grad(value, leaf)[0]
    dx = dl @ s.wg.double().t()
    dwg, dbias = s.x[kept].double().t() @ dl[kept], dl.sum(dim=0)
    if case["accumulate"]:
        dwg, dbias = dwg + s.dwg0.double(), dbias + s.dbias0.double()
    return {"dx": dx, "dwg": dwg, "dbias": dbias}


def work(case):
    """Inputs read once, outputs written once; multiply-adds of the two products, a few operations an element elsewhere."""
    if case["op"] == "clip":
        n32, n16 = case["layers"] * (case["H"] + 1) * case["E"], 3 * case["experts"] * case["H"] * case["F"]
        return {"bytes": 2 * (4 * n32 + 2 * n16), "flops": 3 * (n32 + n16)}
    T, H, E, k = (case[n] for n in ("T", "H", "E", "k"))
    if case["op"] == "combine":
        y, d = (4 if case[n] else 2 for n in ("y_fp32", "dout_fp32"))
        return {"bytes": T * H * (d + k * y * (2 if case["dy"] else 1)) + 12 * T * k, "flops": (3 if case["dy"] else 2) * T * k * H}
    if case["op"] == "balance":
        return {"bytes": 4 * T * E * (2 if case["grad"] else 1) + 4 * T * k + 4 * E + 8 + (T if case["padding"] else 0),
                "flops": 10 * T * E}
    reads = 2 * T * H + 2 * H * E + 4 * T * E * (2 if case["dlogits"] else 1) + 8 * T * k + (T if case["padding"] else 0)
    sums = 4 * (H * E + E)
    return {"bytes": reads + 2 * T * H + sums * (2 if case["accumulate"] else 1), "flops": 4 * T * H * E}
