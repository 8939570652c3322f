"""MXFP4: quantisation of rows and weights, the layouts, and the grouped products, against 64-bit references."""
import numpy as np
import pytest
import torch

from paper_2503_09716_amd import Moe, MoeError

pytestmark = pytest.mark.gpu
DEV = "cuda"
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
MIDPOINTS = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))   # True: a tie goes up


@pytest.fixture(scope="module")
def moe():
    m = Moe(0)
    yield m
    m.close()


def reference(x):
    """(codes 0..15, scale bytes) of x [rows, cols], on the CPU in 64 bits, from the definition."""
    v = x.detach().cpu().double().unflatten(1, (-1, 32))
    finite = torch.isfinite(v).all(dim=2)
    v = torch.where(finite[..., None], v, torch.zeros_like(v))
    amax = v.abs().amax(dim=2)
    s = torch.where(amax > 0, torch.floor(torch.log2(amax)) - 2, torch.tensor(-127.0, dtype=torch.float64)).clamp(min=-127)
    a = v.abs() / torch.exp2(s)[..., None]
    code = sum((a >= m if up else a > m).int() for m, up in MIDPOINTS) + 8 * torch.signbit(v).int()
    byte = torch.where(finite, s.int() + 127, torch.full_like(s.int(), 255))
    return torch.where(finite[..., None], code, torch.zeros_like(code)).flatten(1), byte


def values(code, byte):
    v = GRID[(code & 7).long()] * torch.where(code & 8 > 0, -1.0, 1.0).double()
    scale = torch.where(byte == 255, torch.tensor(float("nan"), dtype=torch.float64), torch.exp2(byte.double() - 127))
    return (v.unflatten(1, (-1, 32)) * scale[..., None]).flatten(1)


def held(x):
    return values(*reference(x))


def same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=1e300), torch.nan_to_num(b, nan=1e300))


def inputs(kind, rows, cols, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    if kind == "normal":
        return torch.randn((rows, cols), generator=gen).to(dtype)
    if kind == "bits":   # any pattern of bits: all exponents, infinities and NaN among them
        t = torch.randint(-2 ** 31, 2 ** 31, (rows, cols), generator=gen, dtype=torch.int64).int()
        return t.view(torch.float32) if dtype is torch.float32 else (t & 0xffff).to(torch.int16).view(torch.bfloat16)
    if kind == "ties":   # multiples of 1/8 up to 8 times a power of two: every midpoint and its neighbours
        x = torch.randint(-64, 65, (rows, cols), generator=gen).float() / 8
        return (x * torch.exp2(torch.randint(-20, 20, (rows, 1), generator=gen).float())).to(dtype)
    if kind == "tiny":   # around the smallest scale, subnormal numbers among them
        return (torch.randn((rows, cols), generator=gen).double() * torch.exp2(torch.randint(-140, -118, (rows, cols // 32, 1), generator=gen).double())
                .expand(-1, -1, 32).reshape(rows, cols)).to(dtype)
    if kind == "large":
        return (torch.rand((rows, cols), generator=gen).double() * 2 - 1).mul(torch.finfo(dtype).max).to(dtype)
    assert kind == "zeros"
    return torch.zeros((rows, cols), dtype=dtype)


SIZES = [(1, 32), (3, 64), (5, 480), (2, 512), (7, 544), (17, 1408), (33, 4096)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["normal", "bits", "ties", "tiny", "large", "zeros"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rows_come_back_as_the_nearest_values(moe, rows, cols, kind, dtype):
    x = inputs(kind, rows, cols, dtype, seed=rows)
    want = held(x)
    q = moe.new_mx_rows(rows, cols)
    moe.mx_quantize(x.to(DEV), q)
    for out_type in (torch.bfloat16, torch.float32):
        out = torch.full((rows, cols), 7.0, dtype=out_type, device=DEV)
        moe.mx_dequantize(q, out)
        assert same(out.cpu().double(), want), (kind, out_type)


def test_every_bf16_under_every_scale_that_it_can_have(moe):
    """Each finite value next to a largest one of its own exponent and of up to eight more."""
    bits = torch.arange(0, 0x7f80, dtype=torch.int32)
    bits = torch.cat([bits, bits | 0x8000])
    for up in range(9):
        top = (((bits & 0x7fff) >> 7) + up).clamp(max=254) << 7 | 0x55
        x = torch.stack([bits, torch.maximum(top, bits & 0x7fff)] + [bits] * 30, dim=1).to(torch.int16).view(torch.bfloat16)
        q, out = moe.new_mx_rows(*x.shape), torch.empty(x.shape, dtype=torch.bfloat16, device=DEV)
        moe.mx_quantize(x.to(DEV), q)
        moe.mx_dequantize(q, out)
        assert same(out.cpu().double(), held(x)), up


@pytest.mark.parametrize("rows,cols", SIZES)
def test_layout_of_quantised_rows(moe, rows, cols):
    x = inputs("normal", rows, cols, torch.bfloat16)
    q = moe.new_mx_rows(rows, cols)
    q.buffer.fill_(0xAB)
    moe.mx_quantize(x.to(DEV), q)
    got = q.buffer.cpu().numpy()
    code, byte = (t.numpy() for t in reference(x))
    subs, groups = -(-cols // 128), -(-cols // 512)
    at = (rows * subs * 64 + 255) // 256 * 256
    assert got.size == at + rows * groups * 16
    codes = np.zeros((rows, subs * 128), dtype=np.uint8)
    codes[:, :cols] = code
    assert np.array_equal(got[:rows * subs * 64].reshape(rows, -1), codes[:, 0::2] | codes[:, 1::2] << 4)
    scales = np.full((rows, groups * 16), 127, dtype=np.uint8)
    for b in range(cols // 32):
        scales[:, 16 * (b // 16) + 4 * (b % 4) + b // 4 % 4] = byte[:, b]
    assert np.array_equal(got[at:].reshape(rows, -1), scales)


WEIGHTS = [(32, 32), (64, 96), (160, 64), (512, 160), (544, 32), (1408, 288), (4096, 64)]


@pytest.mark.parametrize("kind", ["normal", "bits", "tiny"])
@pytest.mark.parametrize("K,N", WEIGHTS)
def test_weights_come_back_as_the_nearest_values(moe, K, N, kind):
    w = inputs(kind, N, K, torch.bfloat16, seed=K).t().contiguous()
    out = torch.empty((K, N), dtype=torch.bfloat16, device=DEV)
    packed = moe.mx_pack_weight(w.to(DEV))
    assert same(moe.mx_unpack_weight(packed, out).cpu().double(), held(w.t()).t())
    again = moe.mx_pack_weight(out)
    assert same(moe.mx_unpack_weight(again, torch.empty_like(out)).double(), out.double())


@pytest.mark.parametrize("K,N", WEIGHTS)
def test_layout_of_packed_weights(moe, K, N):
    w = inputs("normal", K, N, torch.bfloat16)
    packed = moe.new_mx_weight(K, N).fill_(0xAB)
    got = moe.mx_pack_weight(w.to(DEV), packed).cpu().numpy()
    code, byte = (t.numpy() for t in reference(w.t()))
    subs, groups = -(-K // 128), -(-K // 512)
    codes = np.zeros((N, subs * 128), dtype=np.uint8)
    codes[:, :K] = code
    nibbles = codes[:, 0::2] | codes[:, 1::2] << 4
    blocks = np.zeros((N // 16, subs, 16, 4, 16), dtype=np.uint8)
    scales = np.full((N // 16, groups, 16, 16), 127, dtype=np.uint8)
    for n in range(N):
        r = n % 16
        for t in range(subs):
            for c in range(4):
                blocks[n // 16, t, r, c ^ ((4 - r // 4) & 3)] = nibbles[n, t * 64 + c * 16:t * 64 + c * 16 + 16]
        for b in range(K // 32):
            scales[n // 16, b // 16, r, 4 * (b % 4) + b // 4 % 4] = byte[n, b]
    at = (blocks.size + 255) // 256 * 256
    assert got.size == at + scales.size
    assert np.array_equal(got[:blocks.size], blocks.ravel()) and np.array_equal(got[at:], scales.ravel())


def test_values_under_scales_that_another_program_chose_are_kept(moe):
    """Codes under scales larger than this library's: quantising their values changes nothing."""
    gen = torch.Generator().manual_seed(3)
    for top in range(1, 8):
        code = torch.randint(0, top + 1, (64, 32), generator=gen)
        sign = torch.randint(0, 2, (64, 32), generator=gen) * 2 - 1
        x = (GRID[code] * sign * torch.exp2(torch.randint(-90, 90, (64, 1), generator=gen).double())).to(torch.bfloat16)
        q, out = moe.new_mx_rows(64, 32), torch.empty((64, 32), dtype=torch.bfloat16, device=DEV)
        moe.mx_quantize(x.to(DEV), q)
        moe.mx_dequantize(q, out)
        assert torch.equal(out.cpu(), x)


# ---- grouped products ------------------------------------------------------------------------------------------------------

class Product:
    """Quantised rows, expert matrices and their values in 64 bits."""

    def __init__(self, moe, counts, K, N, gated, tokens=0, seed=0, spoil=None):
        gen = torch.Generator().manual_seed(seed)
        self.moe, self.K, self.N, self.gated, self.counts = moe, K, N, gated, counts
        E, self.rows = len(counts), sum(counts)
        n = tokens or self.rows
        x = torch.randn((n, K), generator=gen).bfloat16()
        w = (torch.randn((2 if gated else 1, E, K, N), generator=gen) * 0.05).bfloat16()
        if spoil:
            spoil(x, w)
        self.index = torch.randint(0, n, (self.rows,), generator=gen).int() if tokens else None
        self.offsets = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device=DEV)
        self.q = moe.new_mx_rows(n, K)
        moe.mx_quantize(x.to(DEV), self.q)
        self.list = moe.weight_list(*[[moe.mx_pack_weight(m.to(DEV)) for m in ms] for ms in w])
        self.x, self.w = held(x).to(DEV), [[held(m.t()).t().to(DEV) for m in ms] for ms in w]
        self.workspace = moe.new_mx_workspace(self.rows, E)

    def run(self, dtype, out=None):
        out = torch.full((self.rows, self.N), 7.0, dtype=dtype, device=DEV) if out is None else out
        index = None if self.index is None else self.index.to(DEV)
        self.moe.mx_grouped_product(self.q, index, self.offsets, self.list, out, self.workspace, gated=self.gated)
        return out

    def expected(self):
        """(values, bound of the error in fp32): a sum of K products, exact each, is off by at most K half steps of the sum of
        magnitudes, twice that where additions cut instead of rounding; the gate's exponential and reciprocal add a few steps."""
        want = torch.empty((self.rows, self.N), dtype=torch.float64, device=DEV)
        bound = torch.empty_like(want)
        at = 0
        for e, n in enumerate(self.counts):
            rows = slice(at, at + n)
            at += n
            x = self.x[rows] if self.index is None else self.x[self.index[rows].long().to(DEV)]
            y = [x @ ws[e] for ws in self.w]
            off = [(x.abs() @ ws[e].abs()) * (self.K * 2.0 ** -23) for ws in self.w]
            if self.gated:
                s = torch.nn.functional.silu(y[0])
                want[rows] = s * y[1]
                bound[rows] = 1.1 * off[0] * (y[1].abs() + off[1]) + s.abs() * off[1] + want[rows].abs() * (8 + y[0].abs()) * 2.0 ** -23
            else:
                want[rows], bound[rows] = y[0], off[0]
        return want, bound

    def check(self, dtype):
        got = self.run(dtype).double()
        want, bound = self.expected()
        if dtype is torch.bfloat16:
            bound = bound * (1 + 2.0 ** -8) + want.abs() * 2.0 ** -8
        error = (got - want).abs()
        assert (error <= bound).all(), (error / bound.clamp(min=1e-300)).max()
        if dtype is torch.float32 and want.numel() >= 4096:   # and on the whole as rounding errors add up
            rms = (error.square().mean() / want.square().mean()).sqrt().item()
            assert rms <= 2.0 ** -22 * max(self.K, 16) ** 0.5, rms


COUNTS = [[1], [16], [3, 0, 1], [0, 64, 65, 0], [33, 130, 7], [257, 1, 300], [0, 0, 5], [700, 90]]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("K,N", [(32, 32), (64, 96), (96, 288), (512, 160), (544, 64), (1408, 544), (2176, 96)])
@pytest.mark.parametrize("counts", COUNTS)
def test_products(moe, counts, K, N, gated):
    p = Product(moe, counts, K, N, gated, seed=K + N)
    p.check(torch.float32)
    p.check(torch.bfloat16)


@pytest.mark.parametrize("gated,N", [(True, 4128), (False, 8224)])
@pytest.mark.parametrize("K", [32, 160, 288, 416, 544, 672, 1152, 2080])
def test_products_of_long_batches(moe, K, N, gated):
    """Several tiles to a workgroup, of all heights, with contractions from one sub-tile on."""
    p = Product(moe, [1500, 0, 250, 230, 180, 2100, 3, 33, 70, 100, 150, 770], K, N, gated, seed=K, tokens=2000 if gated else 0)
    p.check(torch.float32 if K % 64 else torch.bfloat16)


def test_products_of_few_rows_with_a_long_contraction(moe):
    for counts in ([3, 0, 120], [128, 256]):
        Product(moe, counts, 5152, 320, False).check(torch.float32)
        Product(moe, counts, 4096, 160, True).check(torch.float32)


def test_outputs_larger_than_the_caches(moe):
    """256 MiB and more are stored past the caches."""
    Product(moe, [9000, 7500], 96, 4352, False).check(torch.float32)
    Product(moe, [20000, 12000], 64, 4352, True).check(torch.bfloat16)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("counts,tokens", [([5, 0, 9], 6), ([300, 280], 200), ([1], 1)])
def test_products_of_gathered_rows(moe, counts, tokens, gated):
    Product(moe, counts, 640, 192, gated, tokens=tokens).check(torch.float32)


def test_products_of_many_groups_with_few_rows(moe):
    gen = torch.Generator().manual_seed(5)
    counts = torch.randint(0, 9, (256,), generator=gen).tolist()
    Product(moe, counts, 256, 64, True).check(torch.float32)


@pytest.mark.parametrize("E,high,K,N,gated", [
    (256, 60, 64, 1088, True),     # short tiles, too many for workgroups to find theirs
    (200, 300, 96, 544, True),     # long ones that workgroups find, groups in every slot
    (130, 700, 64, 288, False),
    (65, 40, 160, 320, False),     # short ones that workgroups find
])
def test_products_of_many_groups(moe, E, high, K, N, gated):
    gen = torch.Generator().manual_seed(E)
    counts = torch.randint(0, high, (E,), generator=gen)
    counts[torch.randint(0, E, (E // 5,), generator=gen)] = 0
    counts[[0, E - 1]] = torch.tensor([0, high])
    Product(moe, counts.tolist(), K, N, gated, tokens=500 if gated else 0, seed=E).check(torch.float32)


@pytest.mark.parametrize("gated", [False, True])
def test_blocks_that_are_not_a_number_spoil_their_rows_and_columns_alone(moe, gated):
    def spoil(x, w):
        x[3, 40] = float("inf")
        x[70, 639] = float("nan")
        w[0, 1, 100, 5] = float("nan")
    p = Product(moe, [64, 100], 640, 96, gated, spoil=spoil)
    got = p.run(torch.float32)
    nan = torch.zeros((164, 96), dtype=torch.bool, device=DEV)
    nan[3] = nan[70] = True
    nan[64:, 5] = True
    assert torch.equal(torch.isnan(got), nan)


def test_rows_behind_the_last_group_stay_as_they_were(moe):
    p = Product(moe, [40, 3], 256, 64, False)
    out = torch.full((43, 64), 7.0, device=DEV)
    whole = p.run(torch.float32).clone()
    p.offsets = torch.tensor([0, 40, 41], dtype=torch.int32, device=DEV)
    p.run(torch.float32, out)
    assert torch.equal(out[:41], whole[:41]) and (out[41:] == 7.0).all()
    p.offsets.zero_()
    out.fill_(7.0)
    p.run(torch.float32, out)
    assert (out == 7.0).all()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("ends", [[0, 0, 0, 0], [0, 0, 300, 300], [7, 7, 2000, 2001], [0, 5000, 5000, 9000], [8000, 8500, 8500, 9000]])
def test_long_launches_with_fewer_rows_than_they_have_room_for(moe, ends, gated):
    p = Product(moe, [3000, 3000, 3000], 96, 8224, gated, seed=3)
    whole = p.run(torch.float32).clone()
    p.offsets = torch.tensor(ends, dtype=torch.int32, device=DEV)
    out = torch.full_like(whole, 7.0)
    p.run(torch.float32, out)
    assert (out[:ends[0]] == 7.0).all() and (out[ends[3]:] == 7.0).all()
    for e in range(3):   # rows that are in the same group as before have the same bits
        a, b = max(ends[e], 3000 * e), min(ends[e + 1], 3000 * (e + 1))
        if a < b:
            assert torch.equal(out[a:b], whole[a:b])
    assert torch.isfinite(out).all()


def test_rows_in_front_of_the_first_group_stay_as_they_were(moe):
    p = Product(moe, [40, 300], 256, 64, False)
    whole = p.run(torch.float32).clone()
    p.offsets = torch.tensor([5, 40, 340], dtype=torch.int32, device=DEV)
    out = torch.full_like(whole, 7.0)
    p.run(torch.float32, out)
    assert torch.equal(out[5:], whole[5:]) and (out[:5] == 7.0).all()


@pytest.mark.parametrize("gated", [False, True])
def test_outputs_above_4_gib(moe, gated):
    """Tiles behind the 32-bit border are those of the same rows alone."""
    rows, N = 70016, 32768
    gen = torch.Generator().manual_seed(1)
    w = [[moe.mx_pack_weight((torch.randn((32, N), generator=gen) * 0.05).bfloat16().to(DEV))] for _ in range(1 + gated)]
    x = torch.randn((rows, 32), generator=gen).bfloat16().to(DEV)
    lst, ws = moe.weight_list(*w), moe.new_mx_workspace(rows, 1)
    q, out = moe.new_mx_rows(rows, 32), torch.empty((rows, N), dtype=torch.bfloat16, device=DEV)
    moe.mx_quantize(x, q)
    moe.mx_grouped_product(q, None, torch.tensor([0, rows], dtype=torch.int32, device=DEV), lst, out, ws, gated=gated)
    for at in (0, 65500, rows - 100):
        q2, part = moe.new_mx_rows(100, 32), torch.empty((100, N), dtype=torch.bfloat16, device=DEV)
        moe.mx_quantize(x[at:at + 100], q2)
        moe.mx_grouped_product(q2, None, torch.tensor([0, 100], dtype=torch.int32, device=DEV), lst, part, ws, gated=gated)
        assert torch.equal(part, out[at:at + 100])


def test_out_must_not_be_the_quantised_rows(moe):
    q = moe.new_mx_rows(4, 512)
    moe.mx_quantize(torch.zeros((4, 512), dtype=torch.bfloat16, device=DEV), q)
    lst = moe.weight_list([moe.mx_pack_weight(torch.zeros((512, 32), dtype=torch.bfloat16, device=DEV))])
    with pytest.raises(MoeError) as e:
        moe.mx_grouped_product(q, None, torch.tensor([0, 4], dtype=torch.int32, device=DEV), lst, q.buffer[:256].view(torch.bfloat16).view(4, 32), moe.new_mx_workspace(4, 1))
    assert e.value.status == 1


def test_one_list_for_a_layer(moe):
    """Gate, up and down matrices in one list: `first` picks."""
    gen = torch.Generator().manual_seed(7)
    w = [[(torch.randn(s, generator=gen) * 0.05).bfloat16().to(DEV) for _ in range(2)] for s in ((128, 192), (128, 192), (192, 128))]
    packed = [[moe.mx_pack_weight(m) for m in ms] for ms in w]
    whole, down = moe.weight_list(*packed), moe.weight_list(packed[2])
    x = torch.randn((9, 192), generator=gen).bfloat16().to(DEV)
    q = moe.new_mx_rows(9, 192)
    moe.mx_quantize(x, q)
    offsets, ws = torch.tensor([0, 4, 9], dtype=torch.int32, device=DEV), moe.new_mx_workspace(9, 2)
    a, b = torch.empty((9, 128), device=DEV), torch.empty((9, 128), device=DEV)
    moe.mx_grouped_product(q, None, offsets, whole, a, ws, first=2)
    moe.mx_grouped_product(q, None, offsets, down, b, ws)
    assert torch.equal(a, b)


def test_products_in_a_replayed_graph_and_on_another_stream(moe):
    p = Product(moe, [70, 0, 300], 384, 160, True)
    want = p.run(torch.bfloat16).clone()
    out = torch.zeros_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.run(torch.bfloat16, out)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run(torch.bfloat16, out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        p.run(torch.bfloat16)


def test_two_graphs_share_a_workspace_and_two_streams_do_not(moe):
    gen = torch.Generator().manual_seed(11)
    cases = [Product(moe, torch.randint(0, 40, (256,), generator=gen).tolist(), 64, 1088, True, seed=s) for s in (1, 2)]   # with a list of tiles in the workspace
    want = [p.run(torch.bfloat16).clone() for p in cases]
    outs = [torch.zeros_like(w) for w in want]
    own = [p.workspace for p in cases]
    shared = max(own, key=lambda w: w.numel())
    graphs = []
    for p, out in zip(cases, outs):
        p.workspace = shared
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            p.run(torch.bfloat16, out)
        graphs.append(graph)
    for _ in range(3):
        for out in outs:
            out.zero_()
        for graph in graphs:
            graph.replay()
        shared.fill_(0xFF)
        torch.cuda.synchronize()
        assert all(torch.equal(out, w) for out, w in zip(outs, want))
    streams = [torch.cuda.Stream() for _ in cases]
    many = [[torch.zeros_like(w) for _ in range(6)] for w in want]
    torch.cuda.synchronize()
    for i in range(6):
        for p, stream, out, ws in zip(cases, streams, many, own):
            p.workspace = ws
            with torch.cuda.stream(stream):
                p.run(torch.bfloat16, out[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for out, w in zip(many, want) for o in out)


def test_refusals(moe):
    def refused(status, call, *args, **kw):
        with pytest.raises(MoeError) as e:
            call(*args, **kw)
        assert e.value.status == status, e.value
    q = moe.new_mx_rows(4, 64)
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    refused(1, moe.new_mx_rows, 4, 48)
    refused(1, moe.new_mx_rows, -1, 64)
    refused(1, moe.new_mx_weight, 64, 40)
    refused(1, moe.new_mx_workspace, 4, 257)
    for bad in (x[:3], x.half(), x.cpu(), x.t()):
        with pytest.raises(AssertionError):
            moe.mx_quantize(bad, q)
    flat = torch.zeros(4 * 64 + 8, dtype=torch.bfloat16, device=DEV)
    refused(1, moe.mx_quantize, flat[4:260].view(4, 64), q)   # 8 bytes off
    moe.mx_quantize(x, q)
    w = [moe.mx_pack_weight(torch.zeros((64, 32), dtype=torch.bfloat16, device=DEV)) for _ in range(2)]
    offsets, ws = torch.tensor([0, 2, 4], dtype=torch.int32, device=DEV), moe.new_mx_workspace(4, 2)
    out, lst = torch.empty((4, 32), device=DEV), moe.weight_list(w)
    refused(1, moe.mx_grouped_product, q, None, offsets, lst, out, ws, gated=True)
    refused(1, moe.mx_grouped_product, q, None, offsets, lst, out, ws, first=-1)
    refused(1, moe.mx_grouped_product, q, None, offsets, lst, torch.empty((5, 32), device=DEV), ws)   # more rows than xq has
    refused(3, moe.mx_grouped_product, q, None, offsets, lst, out, ws[:256])
    with pytest.raises(AssertionError):
        moe.mx_grouped_product(q, None, offsets, lst, torch.empty((4, 64), device=DEV), ws)           # matrices of another size
    bf16 = moe.weight_list([torch.zeros_like(w[0][:moe.new_mx_weight(64, 32).numel() // 2 * 2]).view(torch.bfloat16) for _ in range(2)])
    refused(1, moe.mx_grouped_product, q, None, offsets, bf16, out, ws)
    empty = moe.new_mx_rows(0, 64)
    moe.mx_quantize(x[:0], empty)
    moe.mx_dequantize(empty, x[:0])
    moe.mx_grouped_product(empty, None, offsets, lst, out[:0], moe.new_mx_workspace(0, 2))


# ---- the operators together --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("T,k,shared", [(700, 4, 2), (33, 1, 0), (1, 3, 1)])
def test_a_layer_stage_by_stage(moe, T, k, shared):
    """route, permute, quantise, gate and up, quantise, down, combine against 64 bits.  Each stage is held to its own inputs as the stage before left
    them (h is quantised again: where a value sits at a border, one step of h is no error of a product)."""
    H, F, E = 320, 192, 12
    gen = torch.Generator().manual_seed(T)
    x = torch.randn((T, H), generator=gen).bfloat16().to(DEV)
    wg = (torch.randn((H, E), generator=gen) * 0.1).bfloat16().to(DEV)
    w = [[(torch.randn(s, generator=gen) * 0.06).bfloat16().to(DEV) for _ in range(E)] for s in ((H, F), (H, F), (F, H))]
    ws_shared = [(torch.randn(s, generator=gen) * 0.06).bfloat16().to(DEV) for s in ((H, F * shared), (H, F * shared), (F * shared, H))] if shared else None
    from paper_2503_09716_amd import make_shape
    s = make_shape(T, H, F, E, k, 0)
    i32 = dict(dtype=torch.int32, device=DEV)
    idx, weight = torch.empty((T, k), **i32), torch.empty((T, k), device=DEV)
    offsets, perm, inv_perm, row_token = (torch.empty(n, **i32) for n in (E + 1, T * k, T * k, T * k))
    ws = moe.new_workspace(s)
    moe.route(s, x, wg, None, idx, weight, None, ws)
    moe.permute(s, x, idx, None, offsets, perm, inv_perm, row_token, ws)
    q = moe.new_mx_rows(T, H)
    moe.mx_quantize(x, q)
    xv = held(x).to(DEV)

    def ffn(row_index, at, matrices, rows, width):
        """(y, expected y, bound) of the experts' matrices, [3][experts]."""
        listed = moe.weight_list(*[[moe.mx_pack_weight(m) for m in ms] for ms in matrices])
        space = moe.new_mx_workspace(rows, len(matrices[0]))
        h = torch.empty((rows, width), dtype=torch.bfloat16, device=DEV)
        moe.mx_grouped_product(q, row_index, at, listed, h, space, gated=True)
        hq = moe.new_mx_rows(rows, width)
        moe.mx_quantize(h, hq)
        y = torch.empty((rows, H), device=DEV)
        moe.mx_grouped_product(hq, None, at, listed, y, space, first=2)
        hv, want, bound = held(h).to(DEV), torch.empty((rows, H), dtype=torch.float64, device=DEV), torch.empty((rows, H), dtype=torch.float64, device=DEV)
        cuts = at.tolist()
        for e, (m1, m3, m2) in enumerate(zip(*matrices)):
            lo, hi = cuts[e], cuts[e + 1]
            v1, v3, v2 = (held(m.t()).t().to(DEV) for m in (m1, m3, m2))
            rows_e = xv[row_index[lo:hi].long()] if row_index is not None else xv[lo:hi]
            g, u = rows_e @ v1, rows_e @ v3
            og, ou = (rows_e.abs() @ v1.abs()) * H * 2.0 ** -23, (rows_e.abs() @ v3.abs()) * H * 2.0 ** -23
            sg = torch.nn.functional.silu(g)
            off = 1.1 * og * (u.abs() + ou) + sg.abs() * ou + (sg * u).abs() * (2.0 ** -8 + (8 + g.abs()) * 2.0 ** -23)
            assert ((h[lo:hi].double() - sg * u).abs() <= off * (1 + 2.0 ** -8)).all()
            want[lo:hi], bound[lo:hi] = hv[lo:hi] @ v2, (hv[lo:hi].abs() @ v2.abs()) * width * 2.0 ** -23
        assert ((y.double() - want).abs() <= bound).all()
        return y, want, bound

    y, y_want, y_bound = ffn(row_token, offsets, w, T * k, F)
    y_shared, want, bound = None, 0.0, 0.0
    if shared:
        y_shared, want, bound = ffn(None, torch.tensor([0, T], **i32), [[m] for m in ws_shared], T, F * shared)
    moe.set_option("out_fp32", 1)
    out = torch.empty((T, H), device=DEV)
    moe.combine(s, y, inv_perm, weight, y_shared, out)
    moe.set_option("out_fp32", 0)
    terms = weight.double()[:, :, None] * y_want[inv_perm.long()].view(T, k, H)
    want = want + terms.sum(dim=1)
    bound = bound + (weight.double()[:, :, None] * y_bound[inv_perm.long()].view(T, k, H)).sum(dim=1) + (terms.abs().sum(dim=1) + want.abs()) * (k + 2) * 2.0 ** -23
    assert ((out.double() - want).abs() <= bound).all()


def test_the_example_runs():
    """examples/quantized_experts.py.  Its layer for few tokens rounds nothing that the layer on the values does not round, and a bf16 output by 2^-8 at
    most on either side; h is rounded there to 2^-8 of each term."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import quantized_experts
    result = quantized_experts.main(["--tokens", "300", "--steps", "2"])
    assert 0.0 <= result["few"] < 3 * 2.0 ** -8 and result["long"] == result["long"] and result["long_us"] > 0
