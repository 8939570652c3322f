"""Balance loss, gradients of the router and of the combine, and clipping, against plain implementations in 64 bits.

Bounds count roundings: U is half a step of fp32.  A softmax value of E logits that span `span` below their largest is off by at most
SOFT = (span + E / 16 + 16) U relative to itself: the difference to the largest logit (a rounding of at most span U, which the
exponential makes relative), exponential, sums along a lane and across 16 lanes, reciprocal, product."""
import math

import pytest
import torch

from paper_2503_09716_amd import MoeError, backward_workspace_bytes, make_shape

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16 = torch.finfo(torch.bfloat16).eps / 2


@pytest.fixture(scope="module")
def moe():
    from paper_2503_09716_amd import Moe
    m = Moe(0)
    yield m
    m.close()


def say(*a):
    print(*a, flush=True)


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(gen, shape, dtype=torch.float32, std=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def within(name, got, want, bound):
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert torch.isfinite(got.double()).all(), name
    off = (got.double() - want).abs() - bound
    worst = off.argmax()
    assert off.max() <= 0, "%s: %g instead of %g, bound %g" % (name, got.flatten()[worst], want.flatten()[worst],
                                                               bound.expand_as(want).flatten()[worst])


def softmax_error(logits, E):
    top = logits.amax(dim=1, keepdim=True)
    near = logits > top - 104          # what is further off is 0 in fp32, or next to it
    span = torch.where(near, top - logits, torch.zeros_like(logits)).amax(dim=1, keepdim=True)
    return (span + E / 16 + 16) * U


# ---- balance loss -------------------------------------------------------------------------------
def balance_ref(logits, idx, keep, bc, zc):
    """counts, loss, dlogits and bounds for the latter two."""
    T, E = logits.shape
    k = idx.shape[1]
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if keep is None else keep
    rows = keep.nonzero().flatten()
    n = rows.numel()
    picks = idx[rows].long().flatten()
    counts = torch.bincount(picks[(picks >= 0) & (picks < E)], minlength=E)
    l = logits[rows].double()
    p = torch.softmax(l, dim=1)
    lse = torch.logsumexp(l, dim=1)
    share = counts.double() / max(k * n, 1)
    loss = torch.stack([E * (share * p.sum(dim=0)).sum(), lse.square().sum()]) / max(n, 1)
    off = E * share - 1
    s = (p * off).sum(dim=1, keepdim=True)
    d = torch.zeros((T, E), dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(d)
    if n == 0:
        return counts, loss, d, torch.zeros_like(loss), bound
    d[rows] = p * ((off - s) * bc / n + 2 * zc / n * lse[:, None])
    eps = softmax_error(l, E)
    s_abs = (p * off.abs()).sum(dim=1, keepdim=True)
    lse_off = eps + 2 * U * lse.abs()[:, None]
    s_off = s_abs * (2 * eps + (E / 16 + 8) * U)
    bound[rows] = p * (abs(bc) / n * ((off.abs() + s_abs) * (eps + 6 * U) + s_off)
                       + 2 * abs(zc) / n * (lse.abs()[:, None] * (eps + 6 * U) + lse_off)) + 1e-44
    loss_off = torch.stack([s_off.mean() + loss[0] * U, (2 * lse.abs()[:, None] * lse_off).mean() + loss[1] * 3 * U])
    return counts, loss, d, loss_off, bound


def balance_inputs(T, E, k, seed, std=1.3, skew=0.0, padding=None):
    gen = generator(seed)
    logits = normal(gen, (T, E), std=std)
    if skew:
        logits -= skew * torch.log(torch.randperm(E, device="cuda", generator=gen).float() + 1.0)
    idx = logits.topk(k, dim=1).indices.int()
    keep = None if padding is None else torch.rand(T, device="cuda", generator=gen) >= padding
    return logits, idx, keep


def run_balance(moe, logits, idx, keep, bc=1e-2, zc=1e-3, grad=True):
    T, E = logits.shape
    shape = make_shape(T, 64, 64, E, idx.shape[1])
    ws = moe.new_backward_workspace(shape)
    ws.fill_(0xa5)
    counts = torch.full((E,), -7, dtype=torch.int32, device="cuda")
    loss = torch.full((2,), float("nan"), device="cuda")
    d = torch.full((T, E), float("nan"), device="cuda") if grad else None
    moe.balance_loss(shape, logits, idx, keep, bc, zc, counts, loss, d, ws)
    torch.cuda.synchronize()
    return counts, loss, d


BALANCE = [(1, 1, 1), (1, 8, 2), (2, 5, 3), (33, 8, 2), (256, 8, 2), (513, 8, 2), (515, 16, 4), (700, 17, 5), (301, 33, 6), (1000, 64, 6),
           (129, 65, 4), (77, 100, 64), (2000, 160, 6), (999, 163, 8), (130, 192, 8), (64, 255, 7), (4099, 256, 8), (20011, 60, 4)]


@pytest.mark.parametrize("T,E,k", BALANCE)
@pytest.mark.parametrize("padding", [None, 0.25])
def test_balance_loss(moe, T, E, k, padding):
    say("balance", T, E, k, padding)
    logits, idx, keep = balance_inputs(T, E, k, T * 1000 + E, skew=1.1 if E > 100 else 0.0, padding=padding)
    counts, loss, d = run_balance(moe, logits, idx, keep)
    r_counts, r_loss, r_d, loss_off, bound = balance_ref(logits, idx, keep, 1e-2, 1e-3)
    assert torch.equal(counts.long(), r_counts)
    within("loss", loss, r_loss, loss_off)
    within("dlogits", d, r_d, bound)
    again = run_balance(moe, logits, idx, keep)
    assert torch.equal(loss, again[1]) and torch.equal(d, again[2])
    counts, loss2, _ = run_balance(moe, logits, idx, keep, grad=False)
    assert torch.equal(counts.long(), r_counts) and torch.equal(loss2, loss)


@pytest.mark.parametrize("T,E", [(40, 8), (3000, 64), (2500, 97)])
def test_balance_loss_padding_rows_may_hold_anything(moe, T, E):
    logits, idx, keep = balance_inputs(T, E, 3, 5, padding=0.4)
    clean = run_balance(moe, logits, idx, keep)
    for value in (float("nan"), float("inf"), -float("inf"), torch.finfo(torch.float32).min, torch.finfo(torch.float32).max):
        dirty, ids = logits.clone(), idx.clone()
        dirty[~keep] = value
        ids[~keep] = -(2 ** 31)
        for a, b in zip(clean, run_balance(moe, dirty, ids, keep)):
            assert torch.equal(a, b), value
    assert (clean[2][~keep] == 0).all()


@pytest.mark.parametrize("T,E", [(40, 8), (3000, 64)])
def test_balance_loss_no_token_kept(moe, T, E):
    logits, idx, _ = balance_inputs(T, E, 2, 6)
    counts, loss, d = run_balance(moe, logits * float("nan"), idx, torch.zeros(T, dtype=torch.bool, device="cuda"))
    assert (counts == 0).all() and (loss == 0).all() and (d == 0).all()


@pytest.mark.parametrize("E", [12, 64, 130])
def test_balance_loss_masked_experts(moe, E):
    """Experts that a mask takes out, by -inf or by the lowest value: probability 0, gradient 0."""
    logits, _, _ = balance_inputs(900, E, 4, 7)
    for value in (-float("inf"), torch.finfo(torch.float32).min):
        masked = logits.clone()
        masked[:, 1::3] = value
        masked[5, :] = value
        masked[5, 2:8:3] = 1.0      # a row of two experts
        idx = masked.topk(2, dim=1).indices.int()
        counts, loss, d = run_balance(moe, masked, idx, None)
        r_counts, r_loss, r_d, loss_off, bound = balance_ref(masked, idx, None, 1e-2, 1e-3)
        assert torch.equal(counts.long(), r_counts)
        within("loss", loss, r_loss, loss_off)
        within("dlogits", d, r_d, bound)
        assert (d[:, 1::3][masked[:, 1::3] == value] == 0).all()


def test_balance_loss_empty_batch_and_ids_out_of_range(moe):
    shape = make_shape(0, 64, 64, 12, 2)
    counts, loss = torch.full((12,), 3, dtype=torch.int32, device="cuda"), torch.full((2,), 5.0, device="cuda")
    none = torch.empty(0, device="cuda")
    moe.balance_loss(shape, none, none.int(), None, 1.0, 1.0, counts, loss, None, moe.new_backward_workspace(shape))
    assert (counts == 0).all() and (loss == 0).all()
    for T in (30, 3000):
        logits, idx, _ = balance_inputs(T, 20, 3, 8)
        idx[::7, 1] = 20
        idx[::5, 2] = -1
        counts, loss, d = run_balance(moe, logits, idx, None)
        r_counts, r_loss, r_d, loss_off, bound = balance_ref(logits, idx, None, 1e-2, 1e-3)
        assert torch.equal(counts.long(), r_counts)
        within("loss", loss, r_loss, loss_off)
        within("dlogits", d, r_d, bound)


def test_balance_loss_gradient_against_differences(moe):
    """Both losses, moved along random directions in 64 bits, against the product of the direction with dlogits.  Counts are constants.
    A central difference of step h is off by h^2 / 6 times the third derivative, here under 1e-6 of the slope."""
    logits, idx, keep = balance_inputs(600, 48, 4, 9, padding=0.2)
    share = None
    for bc, zc in ((1.0, 0.0), (0.0, 1.0), (0.3, -0.7)):
        _, _, d = run_balance(moe, logits, idx, keep, bc, zc)
        share = torch.bincount(idx[keep].long().flatten(), minlength=48).double() / (4 * keep.sum())

        def value(l):
            l = l[keep]
            return bc * 48 * (share * torch.softmax(l, 1).mean(0)).sum() + zc * torch.logsumexp(l, 1).square().mean()
        gen = generator(10)
        for _ in range(3):
            v = normal(gen, logits.shape).double()
            h = 1e-4
            slope = (value(logits.double() + h * v) - value(logits.double() - h * v)) / (2 * h)
            assert abs(slope - (d.double() * v).sum()) <= 1e-5 * (d.double() * v).abs().sum()


# ---- gradient of the router ---------------------------------------------------------------------
def route_inputs(T, H, E, k, seed, dlogits=True, padding=None, std=1.0):
    gen = generator(seed)
    s = {"x": normal(gen, (T, H), torch.bfloat16), "wg": normal(gen, (H, E), torch.bfloat16, 0.05), "logits": normal(gen, (T, E), std=std)}
    s["idx"] = s["logits"].topk(k, dim=1).indices.int()
    s["dw"] = normal(gen, (T, k))
    s["dlogits"] = normal(gen, (T, E), std=0.1) if dlogits else None
    s["keep"] = None if padding is None else torch.rand(T, device="cuda", generator=gen) >= padding
    return s


def route_ref(s, renorm, scale):
    """dx, dwg, dbias from the formulas in 64 bits, and what bounds them hang on: dl, its bound."""
    T, E = s["logits"].shape
    on = torch.ones(T, dtype=torch.bool, device="cuda") if s["keep"] is None else s["keep"]
    idx = s["idx"].long()
    l = torch.where(on[:, None], s["logits"], torch.zeros_like(s["logits"])).double()
    g = torch.zeros((T, E), dtype=torch.float64, device="cuda").scatter_(1, idx, s["dw"].double() * scale)
    picked = torch.zeros((T, E), dtype=torch.bool, device="cuda").scatter_(1, idx, True)
    if renorm:
        l = torch.where(picked, l, torch.full_like(l, -math.inf))
    p = torch.softmax(l, dim=1)
    sums = (p * g).sum(dim=1, keepdim=True)
    dl = p * (g - sums)
    eps = softmax_error(l, E)
    s_abs = (p * g.abs()).sum(dim=1, keepdim=True)
    # g carries a rounding of the product with scale; the sum E / 16 + 4 more; difference, product, addition of dlogits one each
    bound = p * ((g.abs() + s_abs) * (eps + 4 * U) + s_abs * (2 * eps + (E / 16 + 8) * U)) + 1e-44
    if s["dlogits"] is not None:
        dl = dl + s["dlogits"].double()
        bound = bound + dl.abs() * U
    dl[~on] = 0
    bound[~on] = 0
    x = torch.where(on[:, None], s["x"], torch.zeros_like(s["x"])).double()
    return x, dl, bound


def run_route_backward(moe, s, renorm, scale=1.0, dx=True, dbias=True, start=None, ws=None):
    T, H = s["x"].shape
    E, k = s["logits"].shape[1], s["idx"].shape[1]
    shape = make_shape(T, H, 64, E, k, 0, renorm, scale)
    if ws is None:
        ws = moe.new_backward_workspace(shape)
        ws.fill_(0xff)        # NaN wherever something is read that was not written
    nan = float("nan")
    dx = torch.full((T, H), nan, dtype=torch.bfloat16, device="cuda") if dx else None
    dwg = torch.full((H, E), nan, device="cuda") if start is None else start[0].clone()
    db = None if not dbias else torch.full((E,), nan, device="cuda") if start is None else start[1].clone()
    moe.route_backward(shape, s["x"], s["wg"], s["logits"], s["idx"], s["dw"], s["dlogits"], s["keep"], dx, dwg, db, start is not None, ws)
    torch.cuda.synchronize()
    return dx, dwg, db


def check_route(s, renorm, scale, dx, dwg, db, start=None):
    x, dl, bound = route_ref(s, renorm, scale)
    T, E = dl.shape
    # dx: two bf16 pieces hold dl to 2^-16 of itself (half a step of the second, U for what is left), 2 E products added up in fp32
    wg = s["wg"].double()
    if dx is not None:
        want = dl @ wg.t()
        off = (bound + dl.abs() * (2.0 ** -16 + (2 * E + 8) * U)) @ wg.abs().t()
        within("dx", dx, want, off * (1 + BF16) + want.abs() * BF16 + 1e-38)
    # dWg, dbias: three pieces hold dl to 2^-24 of itself; 3 T products and as many sums as there are parts of the tokens
    many = (3 * T + 600) * U
    want, off = x.t() @ dl, x.abs().t() @ (bound + dl.abs() * (many + 2 * U))
    want_b, off_b = dl.sum(0), (bound + dl.abs() * (many + 2 * U)).sum(0)
    if start is not None:
        want, want_b = want + start[0].double(), want_b + start[1].double()
    within("dwg", dwg, want, off + want.abs() * U + 1e-38)
    if db is not None:
        within("dbias", db, want_b, off_b + want_b.abs() * U + 1e-38)
    if start is None:
        # The roundings of the sums are as good as independent: each is at most U of a partial sum, which is about as large as the
        # root of the sum of squares at most.
        rms = lambda v: v.square().mean().sqrt()
        root = (x.square().t() @ dl.square()).sqrt()
        slack = (x.square().t() @ bound.square()).sqrt()
        assert rms(dwg.double() - want) <= rms(root) * U * math.sqrt(3 * T + 16) + rms(slack)


ROUTE = [(1, 64, 2, 1), (1, 512, 8, 2), (3, 64, 3, 3), (31, 128, 8, 2), (32, 64, 16, 4), (33, 320, 17, 5), (97, 192, 31, 4), (256, 512, 8, 2),
         (300, 256, 33, 6), (515, 576, 64, 6), (130, 320, 65, 4), (200, 256, 96, 5), (77, 128, 100, 64), (150, 192, 128, 8), (1000, 2048, 64, 6),
         (640, 512, 160, 6), (333, 832, 161, 7), (90, 448, 192, 8), (120, 256, 250, 3), (1025, 1088, 256, 8), (5003, 256, 8, 2)]


@pytest.mark.parametrize("T,H,E,k", ROUTE)
@pytest.mark.parametrize("renorm", [True, False])
def test_route_backward(moe, T, H, E, k, renorm):
    say("route backward", T, H, E, k, renorm)
    s = route_inputs(T, H, E, k, T * 7 + E, dlogits=(T + E) % 2 == 0, padding=0.2 if T % 3 == 1 and T > 1 else None)
    scale = 1.0 if T % 2 else 2.5
    dx, dwg, db = run_route_backward(moe, s, renorm, scale)
    check_route(s, renorm, scale, dx, dwg, db)
    start = (torch.randn_like(dwg), torch.randn_like(db))
    dx2, dwg2, db2 = run_route_backward(moe, s, renorm, scale, start=start)
    assert torch.equal(dx, dx2)
    check_route(s, renorm, scale, dx2, dwg2, db2, start)
    _, dwg3, _ = run_route_backward(moe, s, renorm, scale, dx=False, dbias=False)
    assert torch.equal(dwg, dwg3)


@pytest.mark.parametrize("E", [7, 30, 48, 64, 70, 130, 160])
@pytest.mark.parametrize("shift", [0, 1])
def test_route_backward_one_block_of_tokens(moe, E, shift):
    """Up to 32 tokens there is nothing to add up: dWg and dbias are written, or added to, in the products' launch, by 16 or by 4 bytes."""
    for T, H in ((1, 64), (17, 576), (32, 320)):
        s = route_inputs(T, H, E, 3, T + E)
        shape = make_shape(T, H, 64, E, 3)
        ws = moe.new_backward_workspace(shape)
        at = lambda *n: torch.randn(math.prod(n) + shift, device="cuda")[shift:].view(n)
        for accumulate in (False, True):
            dx, dwg, db = torch.empty_like(s["x"]), at(H, E), at(E)
            start = (dwg.clone(), db.clone()) if accumulate else None
            moe.route_backward(shape, s["x"], s["wg"], s["logits"], s["idx"], s["dw"], s["dlogits"], None, dx, dwg, db, accumulate, ws)
            check_route(s, True, 1.0, dx, dwg, db, start)
        before = dwg.clone()
        moe.route_backward(shape, s["x"], s["wg"], s["logits"], s["idx"], s["dw"], s["dlogits"], None, None, dwg, None, True, ws)
        check_route(s, True, 1.0, None, dwg, None, (before, torch.zeros(E, device="cuda")))


@pytest.mark.parametrize("T,H,E", [(64, 512, 8), (128, 576, 20), (97, 320, 30), (127, 2112, 64), (96, 1088, 72), (95, 448, 160), (70, 192, 45), (66, 320, 63),
                                   (128, 1088, 49), (129, 320, 64), (97, 192, 96)])
@pytest.mark.parametrize("padding", [None, 0.3])
def test_route_backward_few_blocks_of_tokens(moe, T, H, E, padding):
    """Two to five blocks of tokens, of which one part is made or several, at once or to what is there, odd rows among them."""
    say("few blocks", T, H, E, padding)
    s = route_inputs(T, H, E, 2, T + E, padding=padding)
    for start in (None, (torch.randn(H, E, device="cuda"), torch.randn(E, device="cuda"))):
        out = run_route_backward(moe, s, False, 1.5, start=start)
        check_route(s, False, 1.5, *out, start)
        assert all(torch.equal(a, b) for a, b in zip(out, run_route_backward(moe, s, False, 1.5, start=start)))


@pytest.mark.parametrize("T,H,E", [(3801, 2048, 64), (3201, 2112, 40), (1281, 5120, 61), (2500, 2048, 128), (2399, 2112, 80), (900, 5120, 160), (777, 4160, 121), (3001, 2048, 96)])
def test_route_backward_parts_of_a_few_blocks(moe, T, H, E):
    """The longest parts for which the products' workgroups compute dl, and parts one block longer, with and without dx."""
    say("parts", T, H, E)
    s = route_inputs(T, H, E, 6, T, padding=0.05)
    first = run_route_backward(moe, s, True, 0.5)
    check_route(s, True, 0.5, *first)
    assert all(torch.equal(a, b) for a, b in zip(first, run_route_backward(moe, s, True, 0.5)))
    without = run_route_backward(moe, s, True, 0.5, dx=False)
    assert torch.equal(without[1], first[1]) and torch.equal(without[2], first[2])


def test_route_backward_many_tokens(moe):
    """Long sums: each part of the tokens over several rounds of the ring, parts that end inside a block."""
    for T, H, E, k in ((20011, 320, 40, 4), (40003, 64, 8, 2), (12345, 256, 144, 6)):
        say("many tokens", T, H, E, k)
        s = route_inputs(T, H, E, k, T, padding=0.1)
        check_route(s, False, 1.0, *run_route_backward(moe, s, False))


@pytest.mark.parametrize("T,H,E,k", [(20000, 4096, 8, 2), (9001, 4096, 24, 2), (9000, 4160, 60, 6), (7003, 2112, 90, 6), (6000, 1984, 128, 8), (9002, 1088, 160, 6),
                                     (5001, 2112, 192, 8), (4001, 1088, 256, 8)])
def test_route_backward_rounds_of_the_ring(moe, T, H, E, k):
    """Every width of the products with parts of many blocks of tokens, H that ends inside a tile, and the same bits every time."""
    say("rounds", T, H, E, k)
    s = route_inputs(T, H, E, k, T, padding=0.05)
    first = run_route_backward(moe, s, True, 0.5)
    check_route(s, True, 0.5, *first)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, run_route_backward(moe, s, True, 0.5)))
    without = run_route_backward(moe, s, True, 0.5, dx=False)
    assert torch.equal(without[1], first[1]) and torch.equal(without[2], first[2])


@pytest.mark.parametrize("E", [20, 64, 160])
def test_misaligned_rows(moe, E):
    """Logits, their gradients and sums at addresses that are aligned to their elements only."""
    T, H, k = 333, 192, 4
    s = route_inputs(T, H, E, k, 30, padding=0.2)

    def shifted(t):
        out = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape)
        return out.copy_(t)
    want = run_route_backward(moe, s, False)
    for name in ("logits", "dlogits", "dw", "idx", "wg", "keep"):
        s[name] = shifted(s[name])
    got = run_route_backward(moe, s, False)
    check_route(s, False, 1.0, *got)
    assert all(torch.allclose(a.float(), b.float(), rtol=1e-2, atol=1e-4) for a, b in zip(want, got))
    shape = make_shape(T, H, 64, E, k, 0, False)
    dwg, db = shifted(torch.zeros(H, E, device="cuda")), shifted(torch.zeros(E, device="cuda"))
    moe.route_backward(shape, s["x"], s["wg"], s["logits"], s["idx"], s["dw"], s["dlogits"], s["keep"], None, dwg, db, False, moe.new_backward_workspace(shape))
    assert torch.equal(dwg, got[1]) and torch.equal(db, got[2])
    counts, loss, d = run_balance(moe, s["logits"], s["idx"], s["keep"])
    r_counts, r_loss, r_d, loss_off, bound = balance_ref(s["logits"], s["idx"], s["keep"], 1e-2, 1e-3)
    assert torch.equal(counts.long(), r_counts)
    within("loss", loss, r_loss, loss_off)
    within("dlogits", d, r_d, bound)


@pytest.mark.parametrize("T,H,E", [(70, 128, 8), (700, 320, 64), (300, 192, 160)])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_backward_padding_rows_may_hold_anything(moe, T, H, E, renorm):
    s = route_inputs(T, H, E, 4, 3, padding=0.3)
    clean = run_route_backward(moe, s, renorm)
    off = ~s["keep"]
    assert (clean[0][off] == 0).all()
    for value in (float("nan"), float("inf"), -float("inf"), torch.finfo(torch.float32).min):
        d = dict(s)
        for name in ("x", "logits", "dw", "dlogits"):
            d[name] = s[name].clone()
            d[name][off] = value
        d["idx"] = s["idx"].clone()
        d["idx"][off] = 2 ** 31 - 1
        for a, b in zip(clean, run_route_backward(moe, d, renorm)):
            assert torch.equal(a, b), value
    s["keep"] = torch.zeros(T, dtype=torch.bool, device="cuda")
    for v in run_route_backward(moe, s, renorm):
        assert (v == 0).all()


@pytest.mark.parametrize("E", [12, 64, 130])
def test_route_backward_masked_experts(moe, E):
    """-inf and the lowest value in logits of experts that nobody picks."""
    for value in (-float("inf"), torch.finfo(torch.float32).min):
        for renorm in (True, False):
            s = route_inputs(200, 128, E, 3, 11)
            s["logits"][:, 1::3] = value
            s["idx"] = s["logits"].topk(3, dim=1).indices.int()
            check_route(s, renorm, 1.0, *run_route_backward(moe, s, renorm))


def test_route_backward_far_apart_logits(moe):
    """Rows in which one expert has nearly all the weight, and logits of hundreds."""
    for std in (8.0, 100.0):
        for renorm in (True, False):
            s = route_inputs(400, 128, 48, 4, 12, std=std)
            check_route(s, renorm, 1.0, *run_route_backward(moe, s, renorm))


def test_route_backward_gradient_not_finite_stays_visible(moe):
    s = route_inputs(100, 128, 24, 3, 13)
    s["dw"][17, 1] = float("nan")
    dx, dwg, db = run_route_backward(moe, s, False)
    assert not torch.isfinite(dx[17].float()).any() and torch.isfinite(dx[16].float()).all()
    assert not torch.isfinite(dwg).any() and not torch.isfinite(db).any()


def test_route_backward_empty_batch(moe):
    e = lambda *n, dtype=torch.float32: torch.empty(n, dtype=dtype, device="cuda")
    shape = make_shape(0, 128, 64, 8, 2)
    dwg, db = torch.ones(128, 8, device="cuda"), torch.ones(8, device="cuda")
    args = (e(0, 128, dtype=torch.bfloat16), e(128, 8, dtype=torch.bfloat16), e(0, 8), e(0, 2, dtype=torch.int32), e(0, 2), None, None, None)
    ws = moe.new_backward_workspace(shape)
    moe.route_backward(shape, *args, dwg, db, True, ws)
    assert (dwg == 1).all() and (db == 1).all()
    moe.route_backward(shape, *args, dwg, db, False, ws)
    assert (dwg == 0).all() and (db == 0).all()


@pytest.mark.parametrize("renorm", [True, False])
def test_route_backward_against_differences(moe, renorm):
    """The value whose gradient it is, moved along random directions of x, Wg and bias in 64 bits, picks kept.  dx is rounded to bf16:
    2^-8 of each of its elements."""
    T, H, E, k, scale = 50, 64, 20, 3, 1.7
    s = route_inputs(T, H, E, k, 14)
    bias = normal(generator(15), (E,))
    s["logits"] = (s["x"].double() @ s["wg"].double() + bias.double()).float()
    s["idx"] = s["logits"].topk(k, dim=1).indices.int()
    dx, dwg, db = run_route_backward(moe, s, renorm, scale)
    idx = s["idx"].long()

    def value(x, wg, b):
        l = x @ wg + b
        w = torch.softmax(l, 1).gather(1, idx)
        if renorm:
            w = w / w.sum(1, keepdim=True)
        return (scale * w * s["dw"].double()).sum() + (l * s["dlogits"].double()).sum()
    gen = generator(16)
    at = (s["x"].double(), s["wg"].double(), bias.double())
    for moved in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 1)):
        way = [normal(gen, a.shape).double() * m for a, m in zip(at, moved)]
        h = 1e-4
        slope = (value(*[a + h * v for a, v in zip(at, way)]) - value(*[a - h * v for a, v in zip(at, way)])) / (2 * h)
        got = sum((d.double() * v).sum() for d, v in zip((dx, dwg, db), way))
        size = sum((d.double() * v).abs().sum() for d, v in zip((dx, dwg, db), way))
        assert abs(slope - got) <= (BF16 if moved[0] else 1e-5) * size


def test_gradient_of_the_gate_through_the_layer(moe):
    """Route, permute, FFN, combine and back: dWg and dbias of <out, R> against 64-bit differentiation of the weighted sum of the
    experts' outputs that the layer itself produced."""
    from workloads import make_layer_inputs, scaled_config
    import parity as P
    cfg = scaled_config("C4", T=300, H=256, F=192, E=24, top_k=4)
    gl = P.GpuLayer(moe, make_layer_inputs(cfg, device="cuda"), host_weights=False)
    shape, T, H, E, k = gl.shape, cfg.T, cfg.H, cfg.E, cfg.top_k
    ws, back = moe.new_workspace(shape), moe.new_backward_workspace(shape)
    i32 = lambda *n: torch.empty(n, dtype=torch.int32, device="cuda")
    f32 = lambda *n: torch.empty(n, device="cuda")
    idx, w, logits = i32(T, k), f32(T, k), f32(T, E)
    moe.route(shape, gl.x, gl.wg, gl.bias, idx, w, logits, ws)
    offsets, perm, inv = i32(E + 1), i32(T * k), i32(T * k)
    rows = i32(T * k)
    moe.permute(shape, gl.x, idx, None, offsets, perm, inv, rows, ws)
    y, ys = f32(T * k, H), f32(T, H)
    moe.grouped_ffn(shape, None, rows, gl.x, offsets, gl.w1p, gl.w3p, gl.w2p, moe.new_h_scratch(shape), y, ys, ws)
    dout = normal(generator(17), (T, H), torch.bfloat16)
    dw, dx, dwg, db = f32(T, k), torch.empty_like(gl.x), f32(H, E), f32(E)
    moe.combine_backward(shape, dout, y, inv, w, dw, None)
    moe.route_backward(shape, gl.x, gl.wg, logits, idx, dw, None, None, dx, dwg, db, False, back)
    torch.cuda.synchronize()
    x, wg = gl.x.double(), gl.wg.double().requires_grad_()
    b = (torch.zeros(E, device="cuda") if gl.bias is None else gl.bias).double().requires_grad_()
    weights = torch.softmax(x @ wg + b, 1).gather(1, idx.long())
    if cfg.renormalize:
        weights = weights / weights.sum(1, keepdim=True)
    out = (weights[:, :, None] * cfg.routed_scale * y.double()[inv.long()].view(T, k, H)).sum(1)
    r_wg, r_b = torch.autograd.grad((out * dout.double()).sum(), (wg, b))
    # fp32 throughout: logits of H terms carry the largest error, (H / 4) U of a few units
    for got, want in ((dwg, r_wg), (db, r_b)):
        assert (got.double() - want).norm() <= 1e-4 * want.norm()


# ---- gradient of the combine --------------------------------------------------------------------
def combine_inputs(T, H, k, seed, y32, d32):
    gen = generator(seed)
    f = {True: torch.float32, False: torch.bfloat16}
    return (normal(gen, (T, H), f[d32]), normal(gen, (T * k, H), f[y32]), torch.randperm(T * k, device="cuda", generator=gen).int(),
            torch.softmax(normal(gen, (T, k)), 1))


def run_combine_backward(moe, dout, y, inv, w, dy=True, E=64):
    (T, H), k = dout.shape, w.shape[1]
    moe.set_option("y_fp32", int(y.dtype == torch.float32))
    moe.set_option("out_fp32", int(dout.dtype == torch.float32))
    try:
        dw = torch.full((T, k), float("nan"), device="cuda")
        dy = torch.full_like(y, float("nan")) if dy else None
        moe.combine_backward(make_shape(T, H, 64, max(E, k), k), dout, y, inv, w, dw, dy)
        torch.cuda.synchronize()
        return dw, dy
    finally:
        moe.set_option("y_fp32", 1)
        moe.set_option("out_fp32", 0)


COMBINE = [(1, 64, 1), (1, 6144, 2), (2, 192, 3), (7, 128, 64), (33, 1024, 5), (70, 2112, 17), (301, 320, 4), (600, 5120, 6), (1200, 4096, 2),
           (2501, 640, 1), (50, 64, 8), (3, 16384, 7)]


@pytest.mark.parametrize("T,H,k", COMBINE)
@pytest.mark.parametrize("y32", [True, False])
@pytest.mark.parametrize("d32", [True, False])
def test_combine_backward(moe, T, H, k, y32, d32):
    say("combine backward", T, H, k, y32, d32)
    dout, y, inv, w = combine_inputs(T, H, k, T + H, y32, d32)
    dw, dy = run_combine_backward(moe, dout, y, inv, w)
    rows = inv.long()
    terms = y.double()[rows].view(T, k, H) * dout.double()[:, None, :]
    # H / 64 terms along a lane at most, then across 64 lanes and up to 16 wavefronts
    within("dtopk_w", dw, terms.sum(2), terms.abs().sum(2) * (H / 64 + 24) * U + 1e-38)
    want = torch.empty(y.shape, dtype=torch.float64, device="cuda")
    want[rows] = (w.double()[:, :, None] * dout.double()[:, None, :]).view(T * k, H)
    within("dy_perm", dy, want, want.abs() * (U if y32 else BF16 + 2 * U) + 1e-38)
    only, _ = run_combine_backward(moe, dout, y, inv, w, dy=False)
    assert torch.equal(only, dw)


def test_combine_backward_rows_past_two_gib(moe):
    """Rows whose offsets pass 32 bits (fp32: 4.4 GB), at the first and the last tokens."""
    T, H, k = 34000, 16384, 2
    gen = generator(19)
    y = torch.empty((T * k, H), device="cuda")
    y[:200].normal_(generator=gen)
    y[-200:].normal_(generator=gen)
    y[200:-200] = 0
    dout = normal(gen, (T, H), torch.bfloat16)
    inv = torch.arange(T * k, device="cuda", dtype=torch.int32).flip(0).contiguous()
    w = torch.rand((T, k), device="cuda", generator=gen)
    dw, dy = run_combine_backward(moe, dout, y, inv, w)
    for part in (slice(0, 100), slice(T - 100, T)):
        rows = inv.view(T, k)[part].long()
        terms = y[rows].double() * dout[part].double()[:, None, :]
        within("dtopk_w", dw[part], terms.sum(2), terms.abs().sum(2) * (H / 64 + 24) * U)
        want = w[part].double()[:, :, None] * dout[part].double()[:, None, :]
        within("dy_perm", dy[rows], want, want.abs() * U)


def test_combine_backward_not_finite(moe):
    """An infinity in a row of y reaches that pair's weight alone; a weight of zero gives rows of zeros."""
    for y32 in (True, False):
        dout, y, inv, w = combine_inputs(40, 256, 3, 20, y32, False)
        y[5, 7] = float("inf")
        w[4, 1] = 0
        dw, dy = run_combine_backward(moe, dout, y, inv, w)
        hit = inv.view(40, 3) == 5
        assert torch.isinf(dw[hit]).all() and torch.isfinite(dw[~hit]).all()
        assert (dy[inv.view(40, 3)[4, 1].long()] == 0).all() and torch.isfinite(dy.float()).all()


# ---- clipping -----------------------------------------------------------------------------------
def tensors(gen, sizes, dtypes, shift=0):
    """Views of one buffer per type that start `shift` elements into it."""
    out = []
    for dtype in (torch.float32, torch.bfloat16):
        mine = [n for n, d in zip(sizes, dtypes) if d == dtype]
        flat = normal(gen, (sum(mine) + shift + 1,), dtype)
        out.append(iter(flat[shift:shift + sum(mine)].split(mine)) if mine else iter(()))
    return [next(out[0] if d == torch.float32 else out[1]) for d in dtypes]


def check_clip(grads, outs, before, norm, max_norm):
    want_norm = math.sqrt(sum(float(g.double().square().sum()) for g in before))
    assert abs(float(norm) - want_norm) <= 2 * U * want_norm
    scale = min(1.0, max_norm / want_norm) if want_norm > 0 else 1.0
    for g, o in zip(before, outs):
        if scale == 1.0:
            assert torch.equal(g, o)
        else:
            want = g.double() * scale
            within("out", o, want, want.abs() * (3 * U if o.dtype == torch.float32 else BF16 + 3 * U) + 1e-38)


F, B = torch.float32, torch.bfloat16
CLIP = [([1], [F]), ([1], [B]), ([0, 3], [F, B]), ([5, 7, 64, 1], [F, B, B, F]), ([4096, 8] * 4, [F] * 8), ([8191, 1], [F, F]), ([8192], [F]), ([8193], [F]),
        ([16384], [B]), ([16383, 16385], [B, B]), ([100000, 33, 70001], [F, F, B]), ([2048 * 64, 64] * 13 + [2048 * 512] * 9, [F] * 26 + [B] * 9),
        ([30000001], [B]), ([17] * 1500, [F, B, F] * 500)]


@pytest.mark.parametrize("sizes,dtypes", CLIP)
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("shift", [0, 1])
def test_clip_gradients(moe, sizes, dtypes, in_place, shift):
    say("clip", len(sizes), sum(sizes), in_place, shift)
    gen = generator(sum(sizes))
    norm = torch.full((1,), float("nan"), device="cuda")
    root = math.sqrt(sum(sizes))
    for ratio in (0.3, 3.0):
        grads = tensors(gen, sizes, dtypes, shift)
        before = [g.clone() for g in grads]
        outs = grads if in_place else tensors(gen, sizes, dtypes, 2 if shift else 0)
        made = moe.gradient_list(grads, outs)
        norm.fill_(float("nan"))
        moe.clip_gradients(made, ratio * root, norm)
        torch.cuda.synchronize()
        if sum(sizes) > 10 or ratio > 1:
            check_clip(grads, outs, before, norm, ratio * root)
        if not in_place:
            first = [o.clone() for o in outs] + [norm.clone()]
            moe.clip_gradients(made, ratio * root, norm)
            assert all(torch.equal(a, b) for a, b in zip(first, outs + [norm]))
            assert all(torch.equal(g, b) for g, b in zip(grads, before))


def test_clip_gradients_leaves_the_neighbours_alone(moe):
    for dtype in (F, B):
        flat = torch.ones(100, dtype=dtype, device="cuda")
        out = torch.full((100,), 7.0, dtype=dtype, device="cuda")
        made = moe.gradient_list([flat[3:50], flat[50:61]], [out[5:52], out[60:71]])
        moe.clip_gradients(made, 0.0, torch.empty(1, device="cuda"))
        torch.cuda.synchronize()
        zero = torch.zeros(100, dtype=torch.bool, device="cuda")
        zero[5:52] = True
        zero[60:71] = True
        assert (out[zero] == 0).all() and (out[~zero] == 7).all()


def test_clip_gradients_far_values(moe):
    """Squares that pass the range of fp32 both ways, zeros, infinities, NaN, and limits of 0 and infinity."""
    norm = torch.empty(1, device="cuda")

    def clip(g, limit):
        out = torch.empty_like(g)
        moe.clip_gradients(moe.gradient_list([g], [out]), limit, norm)
        torch.cuda.synchronize()
        return out
    for dtype in (F, B):
        for size in (1e30, 1e-30):
            g = torch.full((4096,), size, dtype=dtype, device="cuda")
            out = clip(g, 32 * size)
            want = g.double().norm().item()
            assert abs(norm.item() - want) <= 2 * U * want
            within("far", out, g.double() * (32 * size / want), g.double() * (BF16 + 3 * U))
        g = torch.zeros(777, dtype=dtype, device="cuda")
        assert (clip(g, 0.0) == 0).all() and norm.item() == 0
        g = torch.ones(777, dtype=dtype, device="cuda")
        assert (clip(g, 0.0) == 0).all()
        assert torch.equal(clip(g, float("inf")), g)
        g[5] = float("inf")
        out = clip(g, 1.0)
        assert math.isinf(norm.item()) and torch.isnan(out[5]) and (out[:5] == 0).all()
        g[5] = float("nan")
        out = clip(g, 1.0)
        assert math.isnan(norm.item()) and torch.isnan(out[5]) and (out[:5] == 1).all()
    empty = moe.gradient_list([], [])
    norm.fill_(3.0)
    moe.clip_gradients(empty, 1.0, norm)
    assert norm.item() == 0


# ---- refusals, streams, graphs ------------------------------------------------------------------
def refused(status, call):
    with pytest.raises(MoeError) as e:
        call()
    assert e.value.status == status, str(e.value)
    torch.cuda.synchronize()


def test_refusals(moe):
    T, H, E, k = 40, 128, 8, 2
    shape = make_shape(T, H, 64, E, k)
    s = route_inputs(T, H, E, k, 1)
    ws = moe.new_backward_workspace(shape)
    small = torch.empty(backward_workspace_bytes(shape) - 1, dtype=torch.uint8, device="cuda")
    counts, loss, d = torch.zeros(E, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros((T, E), device="cuda")
    nan, inf = float("nan"), float("inf")
    bal = lambda sh=shape, logits=s["logits"], bc=1.0, zc=1.0, c=counts, d=d, w=ws: moe.balance_loss(sh, logits, s["idx"], None, bc, zc, c, loss, d, w)
    refused(1, lambda: bal(logits=None))
    refused(1, lambda: bal(c=None))
    refused(1, lambda: bal(bc=nan))
    refused(1, lambda: bal(zc=-inf))
    refused(1, lambda: bal(d=s["logits"]))
    refused(3, lambda: bal(w=small))
    refused(1, lambda: bal(w=torch.empty(ws.numel() + 256, dtype=torch.uint8, device="cuda")[1:]))
    refused(2, lambda: bal(sh=make_shape(T, H, 65, E, k)))
    refused(1, lambda: bal(sh=make_shape(T, H, 64, E, k, -1)))
    dx, dwg, db = torch.zeros((T, H), dtype=torch.bfloat16, device="cuda"), torch.zeros((H, E), device="cuda"), torch.zeros(E, device="cuda")

    def route(x=s["x"], wg=s["wg"], dw=s["dw"], dx=dx, dwg=dwg, w=ws):
        moe.route_backward(shape, x, wg, s["logits"], s["idx"], dw, None, None, dx, dwg, db, False, w)
    refused(1, lambda: route(x=None))
    refused(1, lambda: route(wg=None))
    refused(1, lambda: route(dw=None))
    refused(1, lambda: route(dwg=None))
    refused(1, lambda: route(dx=s["x"]))
    refused(3, lambda: route(w=small))
    odd = torch.zeros(T * H + 1, dtype=torch.bfloat16, device="cuda")[1:].view(T, H)
    refused(1, lambda: route(x=odd))
    refused(1, lambda: route(dx=odd))
    with pytest.raises(AssertionError):
        route(dwg=dwg.t())
    with pytest.raises(AssertionError):
        route(x=s["x"].float())
    big = make_shape(1 << 23, 64, 64, 256, 1)
    assert backward_workspace_bytes(big) == 0 and backward_workspace_bytes(make_shape(1 << 22, 64, 64, 128, 1)) > 0
    dout, y, inv, w = combine_inputs(T, H, k, 2, True, False)
    dtw = torch.empty_like(w)
    com = lambda dout=dout, y=y, inv=inv, w=w, dw=dtw, dy=None: moe.combine_backward(shape, dout, y, inv, w, dw, dy)
    refused(1, lambda: com(dout=None))
    refused(1, lambda: com(y=None))
    refused(1, lambda: com(dw=None))
    refused(1, lambda: com(w=None, dy=torch.empty_like(y)))
    refused(1, lambda: com(dy=y))
    refused(1, lambda: com(dw=w))
    refused(1, lambda: com(dout=odd))
    com(w=None)                                      # the weights are read for dy_perm only
    with pytest.raises(AssertionError):
        com(dy=y.bfloat16())
    norm = torch.empty(1, device="cuda")
    a = torch.zeros(100, device="cuda")
    refused(1, lambda: moe.gradient_list([a[:60]], [a[40:]]))
    refused(1, lambda: moe.gradient_list([a[:60], a[50:]], [torch.empty(60, device="cuda"), torch.empty(50, device="cuda")]))
    refused(1, lambda: moe.gradient_list([a[:50], a[:50]], [a[:50], a[:50]]))
    refused(1, lambda: moe.gradient_list([a[:50], a[50:]], [a[50:], a[:50]]))
    for limit in (nan, -1.0, -inf):
        refused(1, lambda: moe.clip_gradients(moe.gradient_list([a], [a]), limit, norm))
    refused(1, lambda: moe.clip_gradients(moe.gradient_list([a], [a]), 1.0, None))


def step(moe, shape, s, bufs, made):
    moe.combine_backward(shape, bufs["dout"], bufs["y"], bufs["inv"], bufs["w"], bufs["dw"], bufs["dy"])
    moe.balance_loss(shape, s["logits"], s["idx"], s["keep"], 1e-2, 1e-3, bufs["counts"], bufs["loss"], bufs["dlogits"], bufs["ws"])
    moe.route_backward(shape, s["x"], s["wg"], s["logits"], s["idx"], bufs["dw"], bufs["dlogits"], s["keep"], bufs["dx"], bufs["dwg"], bufs["db"], False,
                       bufs["ws"])
    moe.clip_gradients(made, 1e-3, bufs["norm"])


def step_buffers(moe, T, H, E, k, seed):
    s = route_inputs(T, H, E, k, seed, padding=0.1)
    dout, y, inv, w = combine_inputs(T, H, k, seed, True, False)
    shape = make_shape(T, H, 64, E, k, 0, False)
    f = lambda *n: torch.zeros(n, device="cuda")
    b = {"dout": dout, "y": y, "inv": inv, "w": w, "dw": f(T, k), "dy": torch.zeros_like(y), "counts": f(E).int(), "loss": f(2), "dlogits": f(T, E),
         "dx": torch.zeros_like(s["x"]), "dwg": f(H, E), "db": f(E), "norm": f(1), "out_g": f(H, E), "out_b": f(E),
         "ws": moe.new_backward_workspace(shape)}
    return shape, s, b, moe.gradient_list([b["dwg"], b["db"]], [b["out_g"], b["out_b"]])


OUTS = ("dw", "dy", "counts", "loss", "dlogits", "dx", "dwg", "db", "norm", "out_g", "out_b")


def test_another_stream_and_a_graph(moe):
    """A whole step on a stream of its own, then captured and replayed with eager steps in between: the same bits every time."""
    for T, H, E, k in ((64, 128, 8, 2), (1500, 320, 48, 4)):
        shape, s, b, made = step_buffers(moe, T, H, E, k, 21)
        step(moe, shape, s, b, made)
        torch.cuda.synchronize()
        want = {n: b[n].clone() for n in OUTS}
        side = torch.cuda.Stream()
        for n in OUTS:
            b[n].zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(moe, shape, s, b, made)
        torch.cuda.synchronize()
        assert all(torch.equal(b[n], want[n]) for n in OUTS)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(moe, shape, s, b, made)
        for _ in range(3):
            for n in OUTS:
                b[n].zero_()
            b["ws"].fill_(0x5a)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(b[n], want[n]) for n in OUTS)
            step(moe, shape, s, b, made)
            torch.cuda.synchronize()
            assert all(torch.equal(b[n], want[n]) for n in OUTS)


def test_the_example_learns():
    """examples/tune_router.py: the layer's output nears the target and the tokens spread."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import tune_router
    history = tune_router.tune(steps=30, tokens=1000, say=say)
    assert torch.isfinite(history).all()
    assert history[-1, 0] < 0.5 * history[0, 0] and history[-1, 1] < 0.7 * history[0, 1]
