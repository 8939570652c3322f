"""The operators of 4-bit expert weights on which speed is measured: quantisation, grouped products, the layer for few tokens.

A case is one call of an operator as a program makes it that keeps the experts of an MoE layer in MXFP4: quantising
rows or a weight matrix and reading back the values, the experts' products on a batch of quantised rows, and the
whole layer for a few tokens (there with bf16 weights, too).  The shapes are the layer shapes of
workloads/configs.py.  With `own` false every operator is computed in elementary torch operations.

MXFP4: 32 neighbours along the contraction share a scale 2^s, s = floor(log2 of their largest magnitude) - 2, and
each is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives times that scale, ties to the even code.
"""
from __future__ import annotations

import math

import torch

own = False

# H, F, E, k, shared experts, renormalised weights
SHAPES = {
    "tiny": (512, 1024, 8, 2, 0, True),
    "8x7b": (4096, 14336, 8, 2, 0, True),
    "8x22b": (6144, 16384, 8, 2, 0, True),
    "lite": (2048, 1408, 64, 6, 2, False),
    "v2": (5120, 1536, 160, 6, 2, False),
}


def _rows(rows, cols, fp32=False):
    return {"op": "rows", "rows": rows, "cols": cols, "fp32": fp32}


def _weight(K, N):
    return {"op": "weight", "K": K, "N": N}


def _product(T, E, k, K, N, gated, fp32=False, skew=False):
    """Products of the rows of T tokens, each in k of E groups.  gated: silu(x Wa) * (x Wb) in bf16, the rows gathered from
    the tokens; otherwise x W of rows in the groups' order, in bf16 or fp32."""
    return {"op": "product", "T": T, "E": E, "k": k, "K": K, "N": N, "gated": gated, "fp32": fp32, "skew": skew}


def _gate_up(shape, T, **options):
    H, F, E, k, _, _ = SHAPES[shape]
    return _product(T, E, k, H, F, True, **options)


def _down(shape, T, **options):
    H, F, E, k, _, _ = SHAPES[shape]
    return _product(T, E, k, F, H, False, **options)


def _few(shape, T, fp4=True, bias=False):
    H, F, E, k, shared, renorm = SHAPES[shape]
    return {"op": "few", "T": T, "H": H, "F": F, "E": E, "k": k, "shared": shared, "renorm": renorm, "fp4": fp4, "bias": bias}


def listed():
    cases = [
        # The hidden states of one decode step: two launches, their latency counts.
        ("rows_tiny_16", _rows(16, 512)),
        # A ragged accumulated batch in fp32, as a norm leaves it.
        ("rows_lite_5003", _rows(5003, 2048, fp32=True)),
        # Loading a model: one expert matrix of the widest kind into the form that the products read, and its values back.
        ("weight_8x7b", _weight(4096, 14336)),
        # The smallest layer's gate and up products: few tiles, a latency-bound step.
        ("gate_up_tiny_256", _gate_up("tiny", 256)),
        # Ragged, many narrow experts: about one tile an expert.
        ("gate_up_lite_3001", _gate_up("lite", 3001)),
        # A long prefill on few wide experts: bound by the matrix units.
        ("gate_up_8x7b_4096", _gate_up("8x7b", 4096)),
        # Skewed routing over many experts, some with a handful of rows: weights dominate.
        ("down_v2_2000", _down("v2", 2000, skew=True)),
        # The largest batch, a short contraction and fp32 outputs, as the weighted combine takes them.
        ("down_lite_16384", _down("lite", 16384, fp32=True)),
        # One token of a decode step through a layer with shared experts: launches and the router count.
        ("few_lite_1", _few("lite", 1)),
        # A small layer in bf16: everything in caches, latency alone.
        ("few_tiny_16_bf16", _few("tiny", 16, fp4=False)),
        # A few sequences on wide experts, every expert read: bound by the weights.
        ("few_8x7b_7", _few("8x7b", 7)),
        # Most tokens and most experts, biased gate.
        ("few_v2_16", _few("v2", 16, bias=True)),
    ]
    return [dict(c, name=n) for n, c in cases]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes spread over their logarithms, odd ones among them, options at random."""
    op = rng.choice(["rows", "weight", "product", "product", "few", "few"])
    if op == "rows":
        cols = 32 * _log_int(rng, 1, 512)
        return _rows(_log_int(rng, 1, min(200000, 2 ** 26 // cols)), cols, fp32=rng.random() < 0.5)
    if op == "weight":
        K = 32 * _log_int(rng, 1, 512)
        return _weight(K, 32 * _log_int(rng, 1, min(512, 2 ** 21 // K)))
    if op == "product":
        if rng.random() < 0.5:
            case = rng.choice([_gate_up, _down])(rng.choice(sorted(SHAPES)), 1)
        else:
            E = _log_int(rng, 1, 200)
            case = _product(1, E, rng.randint(1, min(8, E)), 32 * _log_int(rng, 1, 256), 32 * _log_int(rng, 2, 256), rng.random() < 0.5)
        # no more work than the largest listed case
        most = 8192 * 4096 * 14336 // (case["k"] * case["K"] * case["N"])
        case["T"] = _log_int(rng, 1, max(1, min(16384, most)))
        case.update(fp32=not case["gated"] and rng.random() < 0.5, skew=rng.random() < 0.4)
        return case
    case = _few(rng.choice(sorted(SHAPES)), rng.randint(1, 16), fp4=rng.random() < 0.7, bias=rng.random() < 0.4)
    if rng.random() < 0.5:
        H, E = 64 * _log_int(rng, 1, 96), _log_int(rng, 2, 128)
        case.update(H=H, E=E, F=64 * _log_int(rng, 1, 8192 // H + 16), k=rng.randint(1, min(8, E)), shared=rng.randint(0, 2),
                    renorm=rng.random() < 0.5)
    return case


class _State:
    """What a program holds before the call."""


def _to_fp4(x):
    """The MXFP4 values, in fp32, of x [rows, cols], blocks of 32 along the columns."""
    v = x.float().view(x.shape[0], -1, 32)
    amax = v.abs().amax(dim=2, keepdim=True)
    s = (torch.frexp(amax).exponent - 3).clamp(min=-127)
    s = torch.where(amax > 0, s, torch.full_like(s, -127))
    a = torch.ldexp(v.abs(), -s)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = (torch.round(a / step) * step).clamp(max=6.0)
    return torch.ldexp(torch.copysign(q, v), s).view(x.shape)


def _inputs(case, seed, values=True):
    """The inputs of a seed; values: matrices in MXFP4 as the values they stand for, otherwise as they were before."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = _State()
    s.case = case

    def normal(shape, dtype=torch.float32, std=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    def weight(K, N):
        w = normal((K, N), torch.bfloat16, 0.02)
        return _to_fp4(w.t().contiguous()).t().bfloat16().contiguous() if values and case.get("fp4", True) else w

    if case["op"] == "rows":
        s.x = normal((case["rows"], case["cols"]), torch.float32 if case["fp32"] else torch.bfloat16)
    elif case["op"] == "weight":
        s.w = normal((case["K"], case["N"]), torch.bfloat16, 0.02)
    elif case["op"] == "product":
        T, E, k, K, N = (case[n] for n in ("T", "E", "k", "K", "N"))
        logits = normal((T, E))
        if case["skew"]:
            logits -= 1.1 * torch.log(torch.randperm(E, device="cuda", generator=gen).float() + 1.0)
        picks = logits.topk(k, dim=1).indices.flatten()
        s.counts = torch.bincount(picks, minlength=E).tolist()
        s.offsets = torch.tensor([0] + s.counts, device="cuda").cumsum(0).int()
        s.row_token = (picks.sort(stable=True).indices // k).int() if case["gated"] else None
        if case["gated"]:
            s.x = normal((T, K), torch.bfloat16)
        else:   # what the gate and up products leave
            g, u = normal((T * k, K)), normal((T * k, K))
            s.x = (g * torch.sigmoid(g) * u).bfloat16()
        if values:
            s.x = _to_fp4(s.x).bfloat16()
        s.weights = [[weight(K, N) for _ in range(E)] for _ in range(2 if case["gated"] else 1)]
    else:
        T, H, F, E = (case[n] for n in ("T", "H", "F", "E"))
        s.x, s.wg = normal((T, H), torch.bfloat16), normal((H, E), torch.bfloat16, 0.02)
        s.bias = normal((E,), std=0.5) if case["bias"] else None
        experts = E + case["shared"]
        s.weights = [[weight(*kn) for _ in range(experts)] for kn in ((H, F), (H, F), (F, H))]
    return s


def prepare(case, seed):
    s = _inputs(case, seed, values=not own)
    if own:   # the context, the packed weights, the workspace and the buffers that a program keeps from step to step
        from paper_2503_09716_amd import Moe, make_shape
        s.moe = moe = Moe(0)
        if case["op"] == "rows":
            s.q, s.out = moe.new_mx_rows(case["rows"], case["cols"]), torch.empty(s.x.shape, dtype=torch.bfloat16, device="cuda")
        elif case["op"] == "weight":
            s.packed, s.out = moe.new_mx_weight(case["K"], case["N"]), torch.empty_like(s.w)
        elif case["op"] == "product":
            rows = case["T"] * case["k"]
            s.q = moe.new_mx_rows(*s.x.shape)
            moe.mx_quantize(s.x, s.q)
            s.weights = [[moe.mx_pack_weight(w) for w in ws] for ws in s.weights]
            s.list = moe.weight_list(*s.weights)
            s.out = torch.empty((rows, case["N"]), dtype=torch.float32 if case["fp32"] else torch.bfloat16, device="cuda")
            s.workspace = moe.new_mx_workspace(rows, case["E"])
        else:
            T, H, F, E, k = (case[n] for n in ("T", "H", "F", "E", "k"))
            s.shape = make_shape(T, H, F, E, k, case["shared"], case["renorm"])
            moe.set_option("gate_packed", 1)
            s.wg = moe.pack_gate(s.shape, s.wg)
            pack = moe.mx_pack_weight if case["fp4"] else moe.pack_weight
            s.weights = [[pack(w) for w in ws] for ws in s.weights]
            s.list = moe.weight_list(*s.weights)
            s.out, s.workspace = torch.empty_like(s.x), moe.new_few_workspace(s.shape)
    elif case["op"] == "few":
        s.weights = [torch.stack(ws) for ws in s.weights]
    torch.cuda.synchronize()
    return s


def run(s):
    return {"rows": _run_rows, "weight": _run_weight, "product": _run_product, "few": _run_few}[s.case["op"]](s)


def _run_rows(s):
    if own:
        s.moe.mx_quantize(s.x, s.q)
        s.moe.mx_dequantize(s.q, s.out)
        return {"values": s.out}
    return {"values": _to_fp4(s.x).bfloat16()}


def _run_weight(s):
    if own:
        s.moe.mx_pack_weight(s.w, s.packed)
        s.moe.mx_unpack_weight(s.packed, s.out)
        return {"values": s.out}
    return {"values": _to_fp4(s.w.t().contiguous()).t().bfloat16().contiguous()}


def _silu(g):
    return g / (1.0 + torch.exp(-g))


def _run_product(s):
    case = s.case
    if own:
        s.moe.mx_grouped_product(s.q, s.row_token, s.offsets, s.list, s.out, s.workspace, gated=case["gated"])
        return {"out": s.out}
    out, at = [], 0
    for e, n in enumerate(s.counts):
        rows = s.x[at:at + n] if s.row_token is None else s.x[s.row_token[at:at + n].long()]
        at += n
        if n:
            y = [rows.float() @ ws[e].float() for ws in s.weights]
            y = _silu(y[0]) * y[1] if case["gated"] else y[0]
            out.append(y if case["fp32"] else y.bfloat16())
    return {"out": torch.cat(out)}


def _run_few(s):
    case = s.case
    if own:
        s.moe.layer_few(s.shape, s.x, s.wg, s.bias, s.list, s.out, s.workspace)
        return {"out": s.out}
    x = s.x.float()
    logits = x @ s.wg.float()
    if s.bias is not None:
        logits = logits + s.bias
    p = torch.exp(logits - logits.amax(dim=1, keepdim=True))
    p = p / p.sum(dim=1, keepdim=True)
    idx = logits.topk(case["k"], dim=1).indices
    w = p.gather(1, idx)
    if case["renorm"]:
        w = w / w.sum(dim=1, keepdim=True)
    w1, w3, w2 = s.weights
    out = torch.zeros_like(x)
    for j in range(case["k"]):
        g, u = (torch.bmm(x[:, None, :], m.index_select(0, idx[:, j]).float()) for m in (w1, w3))
        y = torch.bmm(_silu(g) * u, w2.index_select(0, idx[:, j]).float())[:, 0]
        out += w[:, j, None] * y
    for e in range(case["E"], case["E"] + case["shared"]):
        out += (_silu(x @ w1[e].float()) * (x @ w3[e].float())) @ w2[e].float()
    return {"out": out.bfloat16()}


def _nearest_fp4(x):
    """_to_fp4 from the definition: how many midpoints of the grid a magnitude passes, in 64 bits."""
    v = x.double().unflatten(1, (-1, 32))
    amax = v.abs().amax(dim=2, keepdim=True)
    scale = torch.exp2(torch.where(amax > 0, torch.floor(torch.log2(amax)) - 2, -127.0).clamp(min=-127))
    a = v.abs() / scale
    code = sum((a >= m if up else a > m).long() for m, up in
               ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)))
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    return (grid[code] * scale * v.sign()).flatten(1)


def exact(case, seed):
    """The same from the definitions in 64 bits."""
    if case["op"] in ("rows", "weight"):
        s = _inputs(case, seed)
        return {"values": _nearest_fp4(s.x) if case["op"] == "rows" else _nearest_fp4(s.w.t()).t()}
    s = _inputs(case, seed, values=False)

    def held(w):   # a weight matrix as the layer has it
        return _nearest_fp4(w.t()).t() if case.get("fp4", True) else w.double()

    if case["op"] == "product":
        x = _nearest_fp4(s.x)
        out = torch.empty((case["T"] * case["k"], case["N"]), dtype=torch.float64, device="cuda")
        for e in range(case["E"]):
            lo, hi = s.offsets[e].item(), s.offsets[e + 1].item()
            rows = x[lo:hi] if s.row_token is None else x[s.row_token[lo:hi].long()]
            if case["gated"] and hi > lo:
                out[lo:hi] = torch.nn.functional.silu(rows @ held(s.weights[0][e])) * (rows @ held(s.weights[1][e]))
            elif hi > lo:
                out[lo:hi] = rows @ held(s.weights[0][e])
        return {"out": out}
    x, E = s.x.double(), case["E"]
    logits = x @ s.wg.double() + (0.0 if s.bias is None else s.bias.double())
    probs = torch.softmax(logits, dim=1)
    picked = torch.zeros_like(probs).scatter_(1, logits.argsort(dim=1, descending=True, stable=True)[:, :case["k"]], 1.0)
    share = probs * picked
    if case["renorm"]:
        share = share / share.sum(dim=1, keepdim=True)
    out = torch.zeros_like(x)
    for e in range(E + case["shared"]):
        tokens = picked[:, e].nonzero().flatten() if e < E else torch.arange(case["T"], device="cuda")
        if tokens.numel():
            w1, w3, w2 = (held(ws[e]) for ws in s.weights)
            y = (torch.nn.functional.silu(x[tokens] @ w1) * (x[tokens] @ w3)) @ w2
            out[tokens] += y * (share[tokens, e, None] if e < E else 1.0)
    return {"out": out}


def work(case):
    """Inputs read once, outputs written once; a weight in MXFP4 is 17/32 bytes; multiply-adds of the products."""
    if case["op"] == "rows":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (4 if case["fp32"] else 2) + 2 * n, "flops": 4 * n}
    if case["op"] == "weight":
        n = case["K"] * case["N"]
        return {"bytes": 4 * n, "flops": 4 * n}
    if case["op"] == "product":
        T, E, k, K, N = (case[n] for n in ("T", "E", "k", "K", "N"))
        mats = 2 if case["gated"] else 1
        read = E * (1.0 - (1.0 - k / E) ** T)   # experts with rows, as even routing has them
        rows = (T if case["gated"] else T * k) * K * 17 // 32 + (4 * T * k if case["gated"] else 0)
        return {"bytes": rows + int(read * mats * K * N) * 17 // 32 + T * k * N * (4 if case["fp32"] else 2),
                "flops": 2 * mats * T * k * K * N}
    T, H, F, E, k, shared = (case[n] for n in ("T", "H", "F", "E", "k", "shared"))
    read = E * (1.0 - (1.0 - k / E) ** T) + shared
    return {"bytes": int(3 * read * H * F * (17 / 32 if case["fp4"] else 2.0)) + 2 * H * E + 4 * T * H,
            "flops": 6 * T * (k + shared) * H * F + 2 * T * H * E}
