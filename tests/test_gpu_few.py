"""The whole layer for up to 16 tokens, on bf16 and MXFP4 weights, against the definition in 64 bits."""
import pytest
import torch

from paper_2503_09716_amd import Moe, MoeError, make_shape

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def moe():
    m = Moe(0)
    yield m
    m.close()


@pytest.fixture(autouse=True)
def options(moe):
    yield
    moe.set_option("out_fp32", 0)
    moe.set_option("gate_packed", 0)


class Layer:
    def __init__(self, moe, T, H, F, E, k, shared=0, renorm=True, fp4=True, bias=None, seed=0, scale=1.0, spoil=None):
        gen = torch.Generator().manual_seed(seed)
        self.moe, self.T, self.k, self.E, self.shared, self.fp4 = moe, T, k, E, shared, fp4
        self.shape = make_shape(T, H, F, E, k, shared, renorm, scale)
        self.x = torch.randn((T, H), generator=gen).bfloat16().to(DEV)
        self.wg = (torch.randn((H, E), generator=gen) * 2 / H ** 0.5).bfloat16().to(DEV)
        self.bias = None if bias is None else (torch.randn(E, generator=gen) * bias).to(DEV)
        n = E + shared
        w = [[(torch.randn(s, generator=gen) * 0.05).bfloat16().to(DEV) for _ in range(n)] for s in ((H, F), (H, F), (F, H))]
        if spoil:
            spoil(self, w)
        if fp4:
            packed = [[moe.mx_pack_weight(m) for m in ms] for ms in w]
            self.w = [[moe.mx_unpack_weight(p, torch.empty_like(m)).double() for p, m in zip(ps, ms)] for ps, ms in zip(packed, w)]
        else:
            packed, self.w = [[moe.pack_weight(m) for m in ms] for ms in w], [[m.double() for m in ms] for ms in w]
        self.packed = packed
        self.list = moe.weight_list(*packed)
        self.workspace = moe.new_few_workspace(self.shape)
        self.workspace.fill_(0xFF)   # NaN in whatever the call reads before it writes

    def run(self, fp32=True, packed_gate=False, out=None):
        self.moe.set_option("out_fp32", int(fp32))
        self.moe.set_option("gate_packed", int(packed_gate))
        wg = self.moe.pack_gate(self.shape, self.wg) if packed_gate else self.wg
        if out is None:
            out = torch.full(self.x.shape, 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device=DEV)
        self.moe.layer_few(self.shape, self.x, wg, self.bias, self.list, out, self.workspace)
        return out

    def picks(self):
        logits = self.x.double() @ self.wg.double() + (0.0 if self.bias is None else self.bias.double())
        order = logits.argsort(dim=1, descending=True, stable=True)
        if self.k < self.E:
            top = logits.gather(1, order)
            gap = top[:, self.k - 1] - top[:, self.k]
            assert not ((gap > 0) & (gap < 1e-5)).any(), "a near tie: take another seed"
        p = torch.softmax(logits, dim=1).gather(1, order[:, :self.k])
        if self.shape.renormalize:
            p = p / p.sum(dim=1, keepdim=True)
        return order[:, :self.k], p * self.shape.routed_scale

    def expected(self):
        """(values, bound of the error in fp32).  A sum of n exact products is off by at most n half steps of the sum of magnitudes, twice that where
        additions cut; that holds for logits (and so for the weights, relatively), gate, up and the sum over experts and F; h is held
        to 2^-17, and exponentials and divisions add a few steps."""
        x, (T, H) = self.x.double(), self.x.shape
        idx, weight = self.picks()
        want, bound = torch.zeros_like(x), torch.zeros_like(x)
        magnitude = torch.zeros_like(x)
        off_logit = (x.abs() @ self.wg.double().abs()).amax() * (H * 2.0 ** -23)
        terms = 0
        for e in range(self.E + self.shared):
            if e < self.E:
                hit = (idx == e)
                tokens = hit.any(dim=1).nonzero().flatten()
                w = (weight * hit).sum(dim=1)[tokens, None]
            else:
                tokens, w = torch.arange(T, device=DEV), torch.ones((T, 1), dtype=torch.float64, device=DEV)
            if not tokens.numel():
                continue
            terms += 1
            w1, w3, w2 = (ws[e] for ws in self.w)
            t = x[tokens]
            g, u = t @ w1, t @ w3
            og, ou = (t.abs() @ w1.abs()) * (H * 2.0 ** -23), (t.abs() @ w3.abs()) * (H * 2.0 ** -23)
            s = torch.nn.functional.silu(g)
            h = w * s * u
            oh = w * (1.1 * og * (u.abs() + ou) + s.abs() * ou) + h.abs() * (2.0 ** -17 + (16 + g.abs()) * 2.0 ** -23 + 2 * off_logit)
            want[tokens] += h @ w2
            bound[tokens] += oh @ w2.abs()
            magnitude[tokens] += h.abs() @ w2.abs()
        return want, bound + magnitude * ((terms * self.shape.F) * 2.0 ** -23)

    def check(self, packed_gate=False):
        want, bound = self.expected()
        got = self.run(True, packed_gate).double()
        error = (got - want).abs()
        assert (error <= bound).all(), (error / bound).max()
        rms = (error.square().mean() / want.square().mean()).sqrt().item()
        assert rms <= 2.0 ** -15, rms    # h to 2^-17 each, sums as rounding errors add up
        out16 = self.run(False, packed_gate)
        assert torch.equal(out16, got.float().bfloat16())   # the same sums, rounded once


@pytest.mark.parametrize("fp4", [True, False])
@pytest.mark.parametrize("T,H,F,E,k,shared,renorm", [
    (1, 64, 64, 1, 1, 0, True),
    (1, 64, 64, 4, 2, 0, True),
    (16, 512, 1024, 8, 2, 0, True),
    (7, 192, 320, 16, 4, 1, False),
    (3, 576, 704, 17, 3, 0, True),
    (16, 256, 192, 64, 6, 2, False),
    (1, 2048, 1408, 64, 6, 2, False),
    (5, 832, 64, 60, 16, 8, True),
    (13, 64, 1472, 130, 7, 3, False),
    (16, 1088, 128, 248, 16, 8, True),
    (16, 640, 64, 256, 16, 0, False),
    (2, 4160, 192, 31, 5, 1, True),
    (16, 4160, 128, 8, 8, 0, True),
])
def test_layer(moe, T, H, F, E, k, shared, renorm, fp4):
    Layer(moe, T, H, F, E, k, shared, renorm, fp4, bias=0.3 if E % 2 else None, seed=T + E, scale=1.5 if shared else 1.0).check()


@pytest.mark.parametrize("T", range(1, 17))
def test_every_number_of_tokens(moe, T):
    Layer(moe, T, 320, 192, 12, 3, 1, seed=T).check()


@pytest.mark.parametrize("E,H", [(8, 256), (64, 2048), (65, 2048), (200, 1536)])
def test_packed_and_logical_gate_give_the_same_bits(moe, E, H):
    a = Layer(moe, 9, H, 128, E, 4, seed=E)
    a.check(packed_gate=True)
    assert torch.equal(a.run(True, False), a.run(True, True))


@pytest.mark.parametrize("fp4", [True, False])
def test_agrees_with_the_layer_for_any_batch(moe, fp4):
    """moe_layer on the same values rounds h to bf16: half a step of 2^-8 of each term, and of the output."""
    a = Layer(moe, 11, 512, 448, 20, 4, 1, False, fp4, seed=4)
    weights = [[moe.pack_weight(m.bfloat16()) for m in ms] for ms in a.w]
    from paper_2503_09716_amd import workspace_bytes
    moe.set_option("out_fp32", 1)
    out = torch.empty(a.x.shape, device=DEV)
    moe.layer(a.shape, a.x, a.wg, a.bias, *weights, out, torch.empty(workspace_bytes(a.shape), dtype=torch.uint8, device=DEV))
    mine = a.run(True)
    want, _ = a.expected()
    assert (mine.double() - want).square().mean() < (out.double() - want).square().mean()
    assert ((out - mine).square().mean() / mine.square().mean()).sqrt().item() < 2.0 ** -8


def test_same_bits_every_time_and_in_a_replayed_graph(moe):
    for E, H in ((8, 512), (96, 2048)):
        a = Layer(moe, 16, H, 704, E, 4, 1, seed=E)
        want = a.run(True).clone()
        for _ in range(3):
            assert torch.equal(a.run(True), want)
        wg = moe.pack_gate(a.shape, a.wg)
        moe.set_option("gate_packed", 1)
        out = torch.empty_like(want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            moe.layer_few(a.shape, a.x, wg, a.bias, a.list, out, a.workspace)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            moe.layer_few(a.shape, a.x, wg, a.bias, a.list, out, a.workspace)
        x0 = a.x.clone()
        for i in range(3):
            a.x.copy_(x0.flip(0) if i == 1 else x0)   # other tokens, other picks
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            eager = a.run(True)
            assert torch.equal(out, eager) and torch.equal(eager, want) == (i != 1)
            moe.set_option("gate_packed", 1)


def test_equal_logits_pick_the_lowest_experts(moe):
    def spoil(a, w):
        a.x.zero_()
        a.x[2:] = 1.0
        a.wg.zero_()
    a = Layer(moe, 5, 128, 128, 24, 5, 1, spoil=spoil, seed=1)
    want, bound = a.expected()
    assert torch.equal(a.picks()[0][0].cpu(), torch.arange(5))
    assert ((a.run(True).double() - want).abs() <= bound).all()


def test_experts_masked_by_the_bias(moe):
    a = Layer(moe, 16, 128, 192, 16, 3, bias=0.1, seed=2)
    a.bias[[0, 3, 4, 5, 9, 15]] = float("-inf")
    want, bound = a.expected()
    assert ((a.run(True).double() - want).abs() <= bound).all()


@pytest.mark.parametrize("fp4", [True, False])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_what_is_not_a_number_stays_with_its_token_or_expert(moe, fp4, value):
    """A token's reaches its own row alone, an expert's those of the tokens that picked it."""
    def spoil_expert(matrix):
        def spoil(a, w):
            w[matrix][3][10, 20] = value
        return spoil
    for matrix in range(3):
        a = Layer(moe, 16, 256, 192, 16, 2, 1, fp4=fp4, seed=6)
        clean, idx = a.run(True).clone(), a.picks()[0]
        b = Layer(moe, 16, 256, 192, 16, 2, 1, fp4=fp4, seed=6, spoil=spoil_expert(matrix))
        hit = (idx == 3).any(dim=1)
        assert hit.any() and not hit.all()
        out = b.run(True)
        assert torch.equal(out[~hit], clean[~hit])
        assert not torch.isfinite(out[hit]).all(dim=1).any()
    a = Layer(moe, 16, 256, 192, 16, 2, 1, fp4=fp4, seed=6)
    want, bound = a.expected()
    a.x[5, 77] = value
    out = a.run(True)
    # the token's picks are others now, and with the set of experts changes the order in which the other tokens' sums are formed
    ok = (out.double() - want).abs() <= bound
    ok[5] = True
    assert ok.all() and not torch.isfinite(out[5]).any()


def test_large_values_of_h(moe):
    """h beyond the range of fp32 is infinite, not NaN from what the infinity leaves."""
    def spoil(a, w):
        for ms in w[:2]:
            for m in ms:
                m.fill_(2.0 ** 60)
        for m in w[2]:
            m.fill_(1.0)
        a.x.fill_(1.0)
    a = Layer(moe, 2, 64, 64, 1, 1, fp4=False, spoil=spoil)
    assert torch.isinf(a.run(True)).all()


def test_no_tokens_and_refusals(moe):
    def refused(status, a, x=None, list_=None, ws=None, shape=None):
        with pytest.raises(MoeError) as e:
            s = shape or a.shape
            moe.layer_few(s, a.x if x is None else x, a.wg[:, :s.E].contiguous(), None, list_ or a.list, torch.empty((s.T, s.H), dtype=torch.bfloat16, device=DEV),
                          a.workspace if ws is None else ws)
        assert e.value.status == status, e.value
    a = Layer(moe, 4, 128, 64, 6, 2)
    none = make_shape(0, 128, 64, 6, 2)
    moe.layer_few(none, a.x[:0], a.wg, None, a.list, torch.empty((0, 128), dtype=torch.bfloat16, device=DEV), moe.new_few_workspace(none))
    for bad in (make_shape(17, 128, 64, 6, 2), make_shape(4, 128, 64, 40, 17), make_shape(4, 100, 64, 6, 2), make_shape(4, 65536, 64, 6, 2)):
        with pytest.raises(MoeError):
            moe.new_few_workspace(bad)
    refused(2, a, torch.zeros((17, 128), dtype=torch.bfloat16, device=DEV), shape=make_shape(17, 128, 64, 6, 2))
    refused(1, a, shape=make_shape(4, 128, 64, 5, 2))                          # a list of six experts for five
    refused(3, a, ws=a.workspace[:256])
    refused(1, a, ws=a.workspace[16:])
    with pytest.raises(AssertionError):
        refused(1, a, list_=moe.weight_list(a.packed[0], a.packed[1]))
    with pytest.raises(AssertionError):
        refused(1, a, x=a.x[:3])


@pytest.mark.parametrize("T,H,F,E,k,shared", [
    (1, 32768, 64, 3, 2, 0),
    (16, 32768, 64, 2, 1, 1),
    (16, 64, 65536, 2, 2, 0),
    (16, 2560, 192, 16, 3, 1),     # the most x that LDS takes
    (15, 2752, 192, 16, 3, 1),     # and a little more
    (1, 4096, 64, 16, 2, 0),       # the largest gate matrix of the gate/up launch
    (1, 4096, 64, 17, 2, 0),
])
@pytest.mark.parametrize("fp4", [True, False])
def test_largest_sizes_and_both_sides_of_the_rules(moe, T, H, F, E, k, shared, fp4):
    Layer(moe, T, H, F, E, k, shared, True, fp4, seed=H + F).check()


def test_calls_at_the_same_time(moe):
    """One list on two streams, with workspaces of their own, over and over."""
    a = Layer(moe, 16, 1024, 704, 16, 4, 1, seed=9)
    want = a.run(True).clone()
    flipped = a.x.flip(0).contiguous()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(want) for _ in range(8)] for _ in streams]
    spaces = [moe.new_few_workspace(a.shape) for _ in streams]
    torch.cuda.synchronize()
    for i in range(8):
        for s, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                moe.layer_few(a.shape, flipped if s else a.x, a.wg, None, a.list, outs[s][i], spaces[s])
    torch.cuda.synchronize()
    for i in range(8):
        assert torch.equal(outs[0][i], want)
        assert torch.equal(outs[1][i], outs[1][0])
    want64, bound = a.expected()
    assert ((outs[1][0].flip(0).double() - want64).abs() <= bound).all()


def test_two_graphs_share_a_workspace(moe):
    a, b = Layer(moe, 5, 512, 320, 12, 3, seed=3), Layer(moe, 16, 512, 320, 12, 4, 1, seed=4)
    want = [a.run(True).clone(), b.run(True).clone()]
    shared = b.workspace if b.workspace.numel() > a.workspace.numel() else a.workspace
    outs, graphs = [torch.empty_like(w) for w in want], []
    for layer, out in zip((a, b), outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            moe.layer_few(layer.shape, layer.x, layer.wg, None, layer.list, out, shared)
        graphs.append(graph)
    for _ in range(3):
        for out in outs:
            out.zero_()
        for graph in graphs:
            graph.replay()
        shared.fill_(0xFF)
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            assert torch.equal(out, w)


@pytest.mark.parametrize("shared", [0, 1])
@pytest.mark.parametrize("fp4", [True, False])
def test_h_between_the_largest_bf16_and_the_largest_fp32(moe, fp4, shared):
    """h = 2^64 (2^64 - 2^54) rounds to no finite bf16, and is finite in fp32.  Exact throughout: one value of h meets ones, the others zeros."""
    def spoil(a, w):
        a.x.zero_()
        a.x[:, 0], a.x[:, 1], a.x[:, 2] = 1.0, 1.0, -2.0 ** -8
        for e in range(1 + shared):
            for ms in w:
                ms[e].zero_()
            w[0][e][0], w[1][e][1], w[1][e][2] = 2.0 ** 64, 2.0 ** 64, 2.0 ** 62
        w[2][shared][3] = 1.0
    a = Layer(moe, 3, 64, 64, 1, 1, shared, fp4=fp4, spoil=spoil)
    want, _ = a.expected()
    assert (want == 2.0 ** 128 * (1 - 2.0 ** -10)).all()
    assert torch.equal(a.run(True).double(), want)
