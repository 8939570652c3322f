"""Edges of the calls that train a router: what shows fewer bits than fp32, values at the ends of their types, ids that name no expert,
and the variants that only large inputs take.  Bounds as in test_gpu_training.py."""
import pytest
import torch

from paper_2503_09716_amd import make_shape

from test_gpu_training import (BF16, U, balance_inputs, balance_ref, check_clip, check_route, combine_inputs, generator, moe, normal, route_inputs, run_balance,  # noqa: F401
                               run_combine_backward, run_route_backward, say, within)

pytestmark = pytest.mark.gpu


# ---- balance loss -------------------------------------------------------------------------------
@pytest.mark.parametrize("T,E,k", [(384, 64, 42), (384, 63, 43), (385, 8, 2), (384, 33, 2), (256, 128, 32), (256, 65, 33), (320, 85, 8), (170, 129, 1),
                                   (171, 191, 1), (128, 256, 64), (129, 255, 30)])
@pytest.mark.parametrize("padding", [None, 0.25])
def test_balance_loss_at_the_limit_of_one_workgroup(moe, T, E, k, padding):
    """Tokens, and logits with picks, for which one workgroup does all, and a few more."""
    say("balance", T, E, k, padding)
    logits, idx, keep = balance_inputs(T, E, k, T + E, padding=padding)
    counts, loss, d = run_balance(moe, logits, idx, keep)
    r_counts, r_loss, r_d, loss_off, bound = balance_ref(logits, idx, keep, 1e-2, 1e-3)
    assert torch.equal(counts.long(), r_counts)
    within("loss", loss, r_loss, loss_off)
    within("dlogits", d, r_d, bound)


# ---- gradient of the router ---------------------------------------------------------------------
@pytest.mark.parametrize("T,H,E", [(33, 128, 8), (70, 192, 30), (100, 320, 64), (64, 576, 90), (90, 256, 128), (64, 128, 160), (45, 64, 192), (64, 192, 250),
                                   (5300, 4096, 8), (5301, 4160, 27), (5300, 4096, 64), (5303, 4096, 90), (5300, 4096, 128), (5300, 4096, 160)])
def test_dx_of_gradients_that_cancel_but_for_their_last_bits(moe, T, H, E):
    """Two experts whose columns of the gate matrix are equal get dl and -dl rounded to 16 bits: dx is the rest, 2^-17 of dl at most, times
    the column.  Six products and as many additions, each off by 2 U of the larger terms at most."""
    say("cancelling", T, H, E)
    gen = generator(T + E)
    dl = normal(gen, (T,))
    first = torch.randint(E, (T,), device="cuda", generator=gen)
    second = (first + 1 + torch.randint(E - 1, (T,), device="cuda", generator=gen)) % E
    hi = dl.bfloat16().float()
    most = hi + (dl - hi).bfloat16().float()
    d = torch.zeros((T, E), device="cuda")
    d[torch.arange(T), first] = dl
    d[torch.arange(T), second] = -most
    column = normal(gen, (H,), torch.bfloat16)
    s = {"x": normal(gen, (T, H), torch.bfloat16), "wg": column[:, None].expand(H, E).contiguous(), "logits": normal(gen, (T, E)),
         "idx": torch.zeros((T, 1), dtype=torch.int32, device="cuda"), "dw": torch.zeros((T, 1), device="cuda"), "dlogits": d, "keep": None}
    dx, _, _ = run_route_backward(moe, s, False)
    rest = dl.double() - most.double()
    assert (rest != 0).sum() > T // 4
    size = dl.double().abs()[:, None] * column.double().abs()
    want = rest[:, None] * column.double()
    within("dx", dx, want, size * 12 * U + want.abs() * BF16 + 1e-38)


@pytest.mark.parametrize("T,H,E", [(40, 128, 8), (70, 192, 60), (64, 192, 250), (5300, 4096, 8)])
def test_route_backward_of_gradients_at_the_ends_of_fp32(moe, T, H, E):
    """dl next to the largest number, and below the smallest normal one, which is held to 2^-134; a token each, so that nothing is added up."""
    say("ends of fp32", T, H, E)
    gen = generator(T + E)
    most = torch.finfo(torch.float32).max
    s = {"x": torch.full((T, H), 2.0 ** -30, dtype=torch.bfloat16, device="cuda"), "wg": torch.full((H, E), 2.0 ** -30, dtype=torch.bfloat16, device="cuda"),
         "logits": normal(gen, (T, E)), "idx": torch.zeros((T, 1), dtype=torch.int32, device="cuda"), "dw": torch.zeros((T, 1), device="cuda"),
         "dlogits": torch.zeros((T, E), device="cuda"), "keep": None}
    values = torch.tensor([most, -most, 3.395e38, -3.3895e38, 3.38e38, 1.0], device="cuda")
    s["dlogits"][torch.arange(6), torch.arange(6)] = values
    dx, dwg, db = run_route_backward(moe, s, False)
    want = values.double() * 2.0 ** -30
    within("dwg", dwg[:, :6], want.expand(H, 6), want.abs() * 2 * U)
    within("dbias", db[:6], values.double(), values.double().abs() * 2 * U)
    within("dx", dx[:6], want[:, None].expand(6, H), want.abs()[:, None] * (BF16 + 2 * U))
    assert (dwg[:, 6:] == 0).all() and (db[6:] == 0).all() and (dx[6:] == 0).all()
    s["x"].fill_(1.0)
    s["dlogits"].zero_()
    small = torch.tensor([1.0, -1.9999999, 1.5, 1.0000001], device="cuda") * torch.tensor([2.0 ** -e for e in (109, 112, 120, 126)], device="cuda")
    s["dlogits"][torch.arange(4), torch.arange(4)] = small
    _, dwg, db = run_route_backward(moe, s, False)
    within("small dwg", dwg[:, :4], small.double().expand(H, 4), torch.full((1,), 2.0 ** -134, dtype=torch.float64, device="cuda"))
    within("small dbias", db[:4], small.double(), torch.full((1,), 2.0 ** -134, dtype=torch.float64, device="cuda"))


# tiles that compute dl by themselves, then those that do not, in every width
PADDED = [(70, 128, 8), (333, 320, 27), (700, 320, 64), (300, 576, 90), (200, 192, 128), (300, 192, 160), (120, 128, 192), (200, 192, 250),
          (5300, 4096, 8), (5301, 4160, 27), (2100, 4096, 64), (5303, 4096, 90), (2100, 4096, 128), (2100, 4160, 160)]


@pytest.mark.parametrize("T,H,E", PADDED)
def test_dx_of_padding_tokens_where_the_gate_matrix_is_not_finite(moe, T, H, E):
    """Rows of padding tokens are zero whatever the gate matrix holds; elsewhere its columns keep to themselves."""
    say("gate not finite", T, H, E)
    s = route_inputs(T, H, E, 3, T + E, padding=0.3)
    clean = run_route_backward(moe, s, True)
    bad = torch.zeros(H, dtype=torch.bool, device="cuda")
    s["wg"][::7, 1] = float("inf")
    s["wg"][1::9, E - 1] = float("nan")
    bad[::7] = True
    bad[1::9] = True
    dx, dwg, db = run_route_backward(moe, s, True)
    off = ~s["keep"]
    assert (dx[off] == 0).all()
    assert torch.equal(dx[:, ~bad], clean[0][:, ~bad]) and not torch.isfinite(dx[s["keep"]][:, bad].float()).any()
    assert torch.equal(dwg, clean[1]) and torch.equal(db, clean[2])


@pytest.mark.parametrize("T,H,E", [(2560, 2048, 64), (2561, 2048, 40), (2560, 2048, 96), (2561, 2048, 96), (4096, 4096, 8), (4097, 4096, 24), (9500, 640, 33),
                                   (3584, 2048, 64)])
@pytest.mark.parametrize("padding", [None, 0.1])
def test_route_backward_longest_parts_without_a_launch_for_dl(moe, T, H, E, padding):
    """As many blocks of tokens to a part as workgroups compute dl for, and one more."""
    say("longest parts", T, H, E, padding)
    s = route_inputs(T, H, E, 4, T, padding=padding)
    first = run_route_backward(moe, s, True, 0.5)
    check_route(s, True, 0.5, *first)
    assert all(torch.equal(a, b) for a, b in zip(first, run_route_backward(moe, s, True, 0.5)))


@pytest.mark.parametrize("T,H,E,k", [(50, 128, 8, 2), (400, 192, 40, 6), (300, 128, 130, 20), (90, 64, 200, 5), (5300, 4096, 8, 2)])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dlogits", [True, False])
def test_route_backward_ids_out_of_range(moe, T, H, E, k, renorm, dlogits):
    """Ids that name no expert have no weight: the softmax over the picks is that over the others, and a row without any has the gradient
    dlogits alone."""
    say("ids out of range", T, H, E, k, renorm, dlogits)
    s = route_inputs(T, H, E, k, T + E, dlogits=dlogits)
    ref = {n: v if v is None else v.clone() for n, v in s.items()}
    gen = generator(T)
    some, none = torch.arange(T, device="cuda") % 3 == 0, torch.arange(T, device="cuda") % 5 == 0
    out = torch.tensor([-1, E, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    wrong = out[torch.randint(4, (T, k), device="cuda", generator=gen)]
    lost = torch.rand((T, k), device="cuda", generator=gen) < 0.4
    lost &= some[:, None]
    lost[:, 0] = False
    lost |= none[:, None]
    s["idx"] = torch.where(lost, wrong, s["idx"])
    # the same picks in ids that exist: the row's first in place of a lost one, and weights without a gradient where all are lost
    ref["idx"] = torch.where(lost, ref["idx"][:, :1], ref["idx"])
    ref["dw"] = torch.where(lost, ref["dw"][:, :1], ref["dw"])
    ref["dw"][none] = 0
    check_route(ref, renorm, 1.5, *run_route_backward(moe, s, renorm, 1.5))


# ---- gradient of the combine --------------------------------------------------------------------
@pytest.mark.parametrize("y32", [True, False])
@pytest.mark.parametrize("d32", [True, False])
@pytest.mark.parametrize("dy", [True, False])
def test_combine_backward_small_terms_behind_large_ones(moe, y32, d32, dy):
    """Terms of 1 in the first elements of a row and small ones behind them, which a single sum along a lane loses one by one.  As many sums
    to a lane as it has elements to a load, N: (H / 64 / N + 24) U of the sum of the terms."""
    T, H, k = 700, 16384, 3
    say("small terms", y32, d32, dy)
    N = 4 if y32 or d32 else 8
    f = {True: torch.float32, False: torch.bfloat16}
    dout = torch.full((T, H), (2 if N == 4 else 6) * U, dtype=f[d32], device="cuda")
    dout[:, :64 * N] = 1
    y = torch.ones((T * k, H), dtype=f[y32], device="cuda")
    inv = torch.randperm(T * k, device="cuda", generator=generator(1)).int()
    dw, _ = run_combine_backward(moe, dout, y, inv, torch.ones((T, k), device="cuda"), dy=dy)
    want = dout.double().sum(1, keepdim=True).expand(T, k)
    within("dtopk_w", dw, want, want * (H / 64 / N + 24) * U)


@pytest.mark.parametrize("d32", [True, False])
@pytest.mark.parametrize("T,H,k", [(1501, 5120, 5), (40001, 192, 5)])
def test_combine_backward_of_bf16_rows_past_the_cache(moe, T, H, k, d32):
    """y in bf16 of more than 64 MiB, which is read past the caches, with the rows' gradient, which is written past them, and without."""
    say("bf16 rows", T, H, k, d32)
    dout, y, inv, w = combine_inputs(T, H, k, 5, False, d32)
    assert y.numel() * 2 > 64 << 20
    dw, dy = run_combine_backward(moe, dout, y, inv, w)
    rows = inv.long()
    terms = y.double()[rows].view(T, k, H) * dout.double()[:, None, :]
    within("dtopk_w", dw, terms.sum(2), terms.abs().sum(2) * (H / 64 + 24) * U + 1e-38)
    want = torch.empty(y.shape, dtype=torch.float64, device="cuda")
    want[rows] = (w.double()[:, :, None] * dout.double()[:, None, :]).view(T * k, H)
    within("dy_perm", dy, want, want.abs() * (BF16 + 2 * U) + 1e-38)
    only, _ = run_combine_backward(moe, dout, y, inv, w, dy=False)
    assert torch.equal(only, dw)


# ---- clipping -----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [4096, 200001])
@pytest.mark.parametrize("in_place", [False, True])
def test_clip_gradients_by_factors_below_the_range_of_fp32(moe, dtype, n, in_place):
    """The norm passes the range of fp32 and max_norm / norm falls below it; the gradients scaled by it do not."""
    say("small factors", dtype, n, in_place)
    norm = torch.zeros(1, device="cuda")
    for size, limit in ((3e38, 1.0), (3e38, 1e-6), (1e37, 1e-12), (1e30, 1e-25), (3e38, 1e-33)):
        g = torch.full((n,), size, dtype=dtype, device="cuda")
        g[1::2] = -g[1::2]
        g[5::16] = 1e-3
        before = g.double()
        out = g if in_place else torch.empty_like(g)
        moe.clip_gradients(moe.gradient_list([g], [out]), limit, norm)
        want = before.norm().item()
        assert norm.item() == float("inf") if want > 3.5e38 else abs(norm.item() - want) <= 2 * U * want
        want = before * (limit / want)
        # products below 2^-126 are held to a step of 2^-149 (fp32) or 2^-133 (bf16), or are zero
        within("out", out, want, want.abs() * (3 * U if dtype == torch.float32 else BF16 + 3 * U) + 2.0 ** -126)

@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("first", [torch.float32, torch.bfloat16])
def test_clip_gradients_of_lists_past_the_cache(moe, in_place, first):
    """More chunks than what is kept in the memory-side cache between the passes (245 MB of 32 KiB each), of both types on both sides of
    that border, with odd lengths and starts."""
    say("long list", in_place, first)
    second = torch.bfloat16 if first == torch.float32 else torch.float32
    gen = generator(3)
    sizes = [3000001, 777, 5000003, 45000007, 30000001, 1, 3000005, 40000003]
    dtypes = [first, second, second, torch.float32, torch.bfloat16, first, second, first]
    shifted = lambda n, dtype, by: torch.empty(n + by, dtype=dtype, device="cuda")[by:]
    grads = [shifted(n, d, 1 + i % 3).normal_(generator=gen) for i, (n, d) in enumerate(zip(sizes, dtypes))]
    before = [g.clone() for g in grads]
    outs = grads if in_place else [shifted(n, d, i % 2) for i, (n, d) in enumerate(zip(sizes, dtypes))]
    made = moe.gradient_list(grads, outs)
    assert made.struct.chunks > 9500
    norm = torch.zeros(1, device="cuda")
    for ratio in (3.0, 0.3):
        limit = ratio * sum(sizes) ** 0.5
        moe.clip_gradients(made, limit, norm)
        check_clip(grads, outs, before, norm, limit)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("in_place", [False, True])
def test_clip_gradients_of_a_few_elements(moe, dtype, in_place):
    """Lists of one to nine elements whose norm is known, scaled and not."""
    for n in (1, 2, 3, 9):
        for share in (0.3, 0.999, 1.0, 1.5):
            g = torch.arange(1, n + 1, device="cuda").to(dtype) * -0.75
            before = g.clone()
            out = g if in_place else torch.empty_like(g)
            made, norm = moe.gradient_list([g], [out]), torch.zeros(1, device="cuda")
            limit = share * before.double().norm().item()
            moe.clip_gradients(made, limit, norm)
            check_clip([g], [out], [before], norm, limit)
            assert share >= 1 or not torch.equal(out, before) or (dtype == torch.bfloat16 and share > 0.99)


# ---- refusals -----------------------------------------------------------------------------------
def test_transposed_shapes_are_refused(moe):
    """A matrix of as many elements whose rows have another length."""
    T, H, E, k = 40, 128, 8, 2
    s = route_inputs(T, H, E, k, 1)
    shape, ws = make_shape(T, H, 64, E, k), moe.new_backward_workspace(make_shape(T, H, 64, E, k))
    dwg = torch.zeros((H, E), device="cuda")
    call = lambda s, dwg: moe.route_backward(shape, s["x"], s["wg"], s["logits"], s["idx"], s["dw"], None, None, None, dwg, None, False, ws)
    call(s, dwg)
    call(s, dwg.view(-1))
    for name in ("x", "wg", "logits", "idx", "dw"):
        wrong = dict(s)
        wrong[name] = s[name].t().contiguous()
        with pytest.raises(AssertionError):
            call(wrong, dwg)
    with pytest.raises(AssertionError):
        call(s, dwg.view(E, H))
    with pytest.raises(AssertionError):
        moe.balance_loss(shape, s["logits"].t().contiguous(), s["idx"], None, 1.0, 0.0, torch.zeros(E, dtype=torch.int32, device="cuda"),
                         torch.zeros(2, device="cuda"), None, ws)
