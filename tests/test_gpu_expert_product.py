"""GPU parity of eb_expert_product with its definition in 64 bits.

Bound: a block's 128 products are exact in fp32; their sum, its scale's product
and the sum over the blocks take at most 128 + 2 + blocks additions and
multiplications, each within 2^-23 (a matrix instruction may truncate) of the
sum of magnitudes, the bias one more.  Then the activation (exp, a sum, a
division, two products: 8 roundings), and one rounding to the output's type.
16-bit outputs may come from the 8-bit matrix unit, which cuts each of eight
products 13 bits below the largest of them: 8 * 2^-13 of that one for each eight,
at most 2^-10 of the sum of magnitudes.
"""
import pytest
import torch

from paper_2512_05831_amd import eb, experts as ex

pytestmark = pytest.mark.gpu
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}


def blocks(n):
    return -(-n // 128)


def fp8(shape, gen, device, pitch=None):
    """Random e4m3 values of all sizes; the bytes between the columns and the pitch are NaNs."""
    rows, cols = shape[-2:]
    pitch = -(-cols // 16) * 16 if pitch is None else pitch
    whole = torch.full((*shape[:-1], pitch), 0x7F, dtype=torch.uint8)
    whole[..., :cols] = (torch.randn(*shape, generator=gen) * 40).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return whole.to(device).view(torch.float8_e4m3fn)[..., :cols]


class Case:
    def __init__(self, M, N, K, device, E=1, act=ex.EB_ACT_NONE, bias=False, counts=None, gather=None, seed=0, x_pitch=None):
        g = torch.Generator().manual_seed(seed + M + 3 * N + 7 * K + 11 * E)
        self.M, self.N, self.K, self.E, self.act = M, N, K, E, act
        self.gate = act == ex.EB_ACT_SILU_GATE
        self.width = N // 2 if self.gate else N
        rows = M if gather is None else gather
        self.x = fp8((rows, K), g, device, x_pitch)
        self.xs = (torch.rand(blocks(K), rows, generator=g) + 0.1).mul_(0.02).to(device).t()
        w = fp8((E, N, K), g, device)
        ws = (torch.rand(E, (2 if self.gate else 1) * blocks(self.width), blocks(K), generator=g) + 0.1).mul_(0.02 / K ** 0.5).to(device)
        self.bias = torch.randn(E, N, generator=g).to(device) if bias else None
        self.tokens = None if gather is None else torch.randint(0, max(gather, 1), (M,), generator=g, dtype=torch.int32).to(device)
        self.offsets = None
        if counts is not None:
            off = [0]
            for c in counts:
                off.append(off[-1] + c)
            self.offsets = torch.tensor(off, dtype=torch.int32, device=device)
        self.w, self.ws = (w, ws) if E > 1 or counts is not None else (w[0], ws[0])

    def run(self, **kw):
        return ex.product(self.x, self.xs, self.w, self.ws, offsets=self.offsets, tokens=self.tokens, bias=self.bias,
                          act=self.act, **kw)

    def exact(self, cut=0.0):
        """The outputs of all slots in 64 bits, how far fp32 may be from them, and which slots are written."""
        dev, K = self.x.device, self.K
        col = torch.arange(K, device=dev) // 128
        row = torch.arange(self.width, device=dev) // 128
        row = torch.cat([row, row + blocks(self.width)]) if self.gate else row
        y = torch.zeros(self.M, self.N, dtype=torch.float64, device=dev)
        size = torch.zeros_like(y)
        written = torch.zeros(self.M, dtype=torch.bool, device=dev)
        bounds = [0, self.M] if self.offsets is None else self.offsets.tolist()
        for e in range(self.E):
            a, b = bounds[e], bounds[e + 1]
            w = (self.w if self.w.dim() == 2 else self.w[e]).double()
            w = w * (self.ws if self.w.dim() == 2 else self.ws[e]).double()[row][:, col]
            t = torch.arange(a, b, device=dev) if self.tokens is None else self.tokens[a:b].long()
            fit = (t >= 0) & (t < self.x.shape[0])
            t = torch.where(fit, t, 0)
            x = self.x.double()[t] * self.xs.double()[t][:, col]
            y[a:b], size[a:b], written[a:b] = x @ w.t(), x.abs() @ w.abs().t(), fit
            if self.bias is not None:
                y[a:b] += self.bias.view(self.E, -1)[e].double()
                size[a:b] += self.bias.view(self.E, -1)[e].double().abs()
        off = ((128 + 3 + blocks(K)) * 2.0 ** -23 + cut) * size
        if self.act == ex.EB_ACT_RELU:
            y = y.clamp(min=0)
        if self.gate:
            g, u = y[:, :self.width], y[:, self.width:]
            dg, du = off[:, :self.width], off[:, self.width:]
            s = g * torch.sigmoid(g)
            y = s * u
            off = 1.1 * dg * (u.abs() + du) + s.abs() * du + 8 * 2.0 ** -23 * y.abs()  # |silu'| < 1.1
        return y, off, written


def close(got, case, dtype):
    y, off, written = case.exact(2.0 ** -10 if dtype in (torch.float16, torch.bfloat16) else 0.0)
    off = off + UNIT[dtype] * (y.abs() + off) + TINY[dtype]
    bad = ((got.double() - y).abs() > off)[written]
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outputs, worst {float(((got.double() - y).abs() / off)[written].max()):.2f} bounds off"


def close_fp8(q, s, case):
    y, off, written = case.exact()
    pad = torch.zeros(case.M, blocks(case.width) * 128, dtype=torch.float64, device=y.device)
    pad[:, :case.width] = y.abs()
    most = pad.view(case.M, -1, 128).amax(2)
    far = torch.zeros_like(pad)
    far[:, :case.width] = off
    far = far.view(case.M, -1, 128).amax(2)
    assert ((s.double() - most / 448).abs() <= far / 448 + most / 448 * 2.0 ** -22 + 2.0 ** -126)[written].all()
    each = s.double().repeat_interleave(128, 1)[:, :case.width]
    wrong = (q.double() * each - y).abs()
    assert (wrong <= (y.abs() + off) * 2.0 ** -4 * (1 + 2.0 ** -20) + each * 2.0 ** -10 + off)[written].all()


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 64, 65, 130, 300])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (3, 130), (128, 16), (130, 127), (257, 400), (1000, 1512), (640, 1024)])
def test_plain_product(M, N, K, device):
    case = Case(M, N, K, device, bias=M % 2 == 0)
    close(case.run(out_dtype=torch.float32), case, torch.float32)


@pytest.mark.parametrize("M,N,K", [(513, 384, 700), (1500, 1024, 1024), (2048, 1000, 1512), (1025, 515, 3328), (4100, 256, 256)])
@pytest.mark.parametrize("act", [ex.EB_ACT_NONE, ex.EB_ACT_RELU, ex.EB_ACT_SILU_GATE])
def test_large_product(M, N, K, act, device):
    case = Case(M, N + N % 2, K, device, act=act, bias=act == ex.EB_ACT_RELU)
    close(case.run(out_dtype=torch.float32), case, torch.float32)
    close_fp8(*case.run(out_dtype=torch.float8_e4m3fn), case)


@pytest.mark.parametrize("out", [torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("act", [ex.EB_ACT_NONE, ex.EB_ACT_RELU, ex.EB_ACT_SILU_GATE])
@pytest.mark.parametrize("M,N,K", [(1, 256, 256), (7, 128, 200), (20, 514, 384), (50, 1002, 520), (200, 290, 640), (700, 770, 300)])
@pytest.mark.parametrize("bias", [False, True])
def test_outputs(out, act, M, N, K, bias, device):
    case = Case(M, N, K, device, act=act, bias=bias)
    got = case.run(out_dtype=out)
    if out == torch.float8_e4m3fn:
        close_fp8(*got, case)
    else:
        close(got, case, out)


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("act", [ex.EB_ACT_NONE, ex.EB_ACT_SILU_GATE])
@pytest.mark.parametrize("M,N,K,counts", [(6000, 2900, 300, None), (8200, 2050, 520, None), (8200, 4100, 129, None),
                                          (8003, 2304, 640, [1000, 3, 2000, 0, 5000]), (3000, 4096, 400, [500] * 6), (1700, 2560, 256, [100, 103] * 8)])
def test_every_size_of_tile(out, act, M, N, K, counts, device):
    """Calls that large and medium tiles take, with tiles that are cut on either side."""
    case = Case(M, N, K, device, E=1 if counts is None else len(counts), act=act, bias=True, counts=counts, gather=None if counts is None else 777)
    got = case.run(out_dtype=out)
    if out == torch.float8_e4m3fn:
        close_fp8(*got, case)
    else:
        close(got, case, out)


COUNTS = {"even": [20] * 9, "ragged": [0, 1, 130, 17, 0, 0, 64, 5, 300], "one": [0, 0, 0, 0, 500, 0, 0, 0, 0], "empty": [0] * 9,
          "long": [700, 3, 257, 0, 1400, 129, 128, 127, 1]}


@pytest.mark.parametrize("counts", list(COUNTS))
@pytest.mark.parametrize("gather", [None, 77])
@pytest.mark.parametrize("act", [ex.EB_ACT_NONE, ex.EB_ACT_SILU_GATE])
@pytest.mark.parametrize("N,K", [(256, 256), (300, 456)])
def test_experts(counts, gather, act, N, K, device):
    n = sum(COUNTS[counts])
    case = Case(n + 13, N, K, device, E=9, act=act, bias=True, counts=COUNTS[counts], gather=gather)  # 13 slots of no expert
    out = torch.full((n + 13, case.width), 7.0, device=device)
    close(case.run(out=out), case, torch.float32)
    assert (out[n:] == 7.0).all()
    close_fp8(*case.run(out_dtype=torch.float8_e4m3fn), case)


def test_many_experts(device):
    g = torch.Generator().manual_seed(3)
    counts = torch.randint(0, 5, (300,), generator=g).tolist()
    case = Case(sum(counts), 130, 260, device, E=300, counts=counts, gather=50)
    close(case.run(out_dtype=torch.float32), case, torch.float32)


def test_tokens_out_of_range_are_not_written(device):
    for M in (40, 900):
        case = Case(M, 200, 300, device, E=3, counts=[M // 2, 0, M - M // 2], gather=30)
        case.tokens[::7] = -1
        case.tokens[3::11] = 30
        out = torch.full((M, 200), 7.0, device=device)
        case.run(out=out)
        y, off, written = case.exact()
        assert (out[~written] == 7.0).all()
        close(out, case, torch.float32)


def test_offsets_out_of_range_are_clamped(device):
    case = Case(50, 64, 128, device, E=2, counts=[20, 30])
    want = case.run(out_dtype=torch.float32)
    case.offsets[0], case.offsets[2] = -5, 1000
    assert torch.equal(case.run(out_dtype=torch.float32), want)


@pytest.mark.parametrize("M", [9, 700])
def test_strides(M, device):
    """Rows of x far apart, an output with a pitch and at an odd column, scales in any order."""
    case = Case(M, 190, 330, device, x_pitch=1024)
    big = torch.full((M, 400), 7.0, device=device)
    case.run(out=big[:, 3:193])
    close(big[:, 3:193], case, torch.float32)
    assert (big[:, :3] == 7.0).all() and (big[:, 193:] == 7.0).all()
    want = case.run(out_dtype=torch.float32)
    case.xs = case.xs.contiguous()
    assert torch.equal(case.run(out_dtype=torch.float32), want)


@pytest.mark.parametrize("M", [5, 600])
def test_integers_are_exact(M, device):
    """Small integers under scales of powers of two: every sum is exact, so every output is."""
    g = torch.Generator().manual_seed(1)
    x = torch.randint(-4, 5, (M, 640), generator=g).float().to(device)
    w = torch.randint(-4, 5, (384, 640), generator=g).float().to(device)
    xs = torch.full((5, M), 0.5, device=device).t()
    ws = torch.full((3, 5), 4.0, device=device)
    got = ex.product(x.to(torch.float8_e4m3fn), xs, w.to(torch.float8_e4m3fn), ws, out_dtype=torch.float32)
    assert torch.equal(got.double(), 2 * x.double() @ w.double().t())


@pytest.mark.parametrize("M", [3, 600])
def test_not_a_number_stays_in_its_row(M, device):
    case = Case(M, 256, 256, device)
    want = case.run(out_dtype=torch.float32)
    case.x.view(torch.uint8)[1, 200] = 0x7F
    got = case.run(out_dtype=torch.float32)
    assert got[1].isnan().all()
    keep = torch.arange(M, device=device) != 1
    assert torch.equal(got[keep], want[keep])
    q, s = case.run(out_dtype=torch.float8_e4m3fn)
    assert s[1].isnan().all() and q[1].float().isnan().all() and not s[keep].isnan().any()


def test_equal_calls_give_equal_bits(device):
    for M, counts in ((60, [10, 0, 50]), (3000, [1000, 1, 1999])):
        case = Case(M, 512, 1024, device, E=3, act=ex.EB_ACT_SILU_GATE, counts=counts, gather=100)
        a, b = case.run(out_dtype=torch.float32), case.run(out_dtype=torch.float32)
        assert torch.equal(a, b)


def test_row_offsets_past_32_bits(device):
    """x and out with rows far apart: byte offsets past 2^32."""
    case = Case(300, 128, 256, device, x_pitch=256)
    wide = torch.zeros(300, 1 << 24, dtype=torch.uint8, device=device)
    wide[:, :256] = case.x.contiguous().view(torch.uint8)
    case.x = wide.view(torch.float8_e4m3fn)[:, :256]
    out = torch.zeros(300, 1 << 23, device=device)[:, :128]
    case.run(out=out)
    close(out, case, torch.float32)


def test_captured_into_a_graph(device):
    for M, counts in ((40, [20, 20]), (1200, [300, 900])):
        case = Case(M, 256, 512, device, E=2, counts=counts, gather=64)
        case.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = case.run()
        for seed in range(4):
            case.tokens.copy_(torch.randint(0, 64, (M,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, case.run())


def test_no_slots(device):
    case = Case(0, 64, 128, device, E=2, counts=[0, 0], gather=5)
    assert case.run().shape == (0, 64)


def test_refusals(device):
    case = Case(8, 64, 128, device)
    for kw in (dict(act=9), dict(out_dtype=torch.int32), dict(bias=torch.zeros(3, device=device)), dict(out=torch.zeros(8, 63, device=device)),
               dict(tokens=torch.zeros(8, dtype=torch.int64, device=device)), dict(offsets=torch.zeros(3, dtype=torch.int32, device=device))):
        with pytest.raises((eb.EbError, ValueError)):
            ex.product(case.x, case.xs, case.w, case.ws, **kw)
    with pytest.raises(ValueError):
        ex.product(case.x, case.xs[:, :0], case.w, case.ws)
    with pytest.raises(ValueError):
        ex.product(case.x.cpu(), case.xs, case.w, case.ws)
    with pytest.raises(ValueError):
        ex.product(case.x.float(), case.xs, case.w, case.ws)
    with pytest.raises(eb.EbError) as e:  # rows no multiple of 16 bytes apart
        odd = torch.zeros(8, 130, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)[:, :128]
        ex.product(odd, case.xs, case.w, case.ws)
    assert e.value.code == eb.EB_ERR_INVALID
    with pytest.raises(eb.EbError) as e:  # a gate over an odd number of rows
        three = Case(8, 63, 128, device)
        ex.product(three.x, three.xs, three.w, torch.zeros(2, 1, device=device), act=ex.EB_ACT_SILU_GATE)
    assert e.value.code == eb.EB_ERR_INVALID


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("act", [ex.EB_ACT_NONE, ex.EB_ACT_SILU_GATE])
@pytest.mark.parametrize("M,N,K,counts", [(8200, 4200, 640, None), (8193, 4100, 424, None), (4097, 8300, 128, None),
                                          (12400, 3050, 300, [4000, 8299, 101])])
def test_tiles_of_256_slots(out, act, M, N, K, counts, device):
    """Calls with many slots per expert, whose last tiles are cut on either side."""
    case = Case(M, N, K, device, E=1 if counts is None else len(counts), act=act, bias=K != 640, counts=counts, gather=None if counts is None else 1000)
    got = case.run(out_dtype=out)
    if out == torch.float8_e4m3fn:
        close_fp8(*got, case)
    else:
        close(got, case, out)


@pytest.mark.parametrize("out", [torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("act", [ex.EB_ACT_NONE, ex.EB_ACT_RELU, ex.EB_ACT_SILU_GATE])
@pytest.mark.parametrize("M,N,K,counts", [(1601, 2050, 300, None), (1990, 1672, 385, None), (4500, 716, 520, [1501, 0, 1400, 90, 1509]), (1000, 130, 1050, None)])
def test_tiles_of_64_and_32_slots(out, act, M, N, K, counts, device):
    case = Case(M, N, K, device, E=1 if counts is None else len(counts), act=act, bias=N != 716, counts=counts, gather=None if counts is None else 900)
    got = case.run(out_dtype=out)
    if out == torch.float8_e4m3fn:
        close_fp8(*got, case)
    else:
        close(got, case, out)


@pytest.mark.parametrize("act", [ex.EB_ACT_NONE, ex.EB_ACT_RELU, ex.EB_ACT_SILU_GATE])
def test_gathered_rows_past_32_bits(act, device):
    """Tokens at byte offsets past 2^32, every type of output."""
    case = Case(90, 420, 300, device, E=3, act=act, bias=True, counts=[33, 0, 50], gather=280, x_pitch=304)
    case.tokens[::9] = -1
    wide = torch.full((280, 1 << 24), 0x7F, dtype=torch.uint8, device=device)
    wide[:, :300] = case.x.contiguous().view(torch.uint8)
    case.x = wide.view(torch.float8_e4m3fn)[:, :300]
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        close(case.run(out_dtype=dtype), case, dtype)
    close_fp8(*case.run(out_dtype=torch.float8_e4m3fn), case)
