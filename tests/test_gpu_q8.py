"""Products with 8-bit weights and rows quantized on the way (lcsm_q8.h) against
the oracle on the GPU (needs an MI355X).

The codes and their sums are whole numbers and the same on both sides.  What is
rounded: the sum to fp32, its products with two scales, the bias, and the output
to its type: four roundings of 2^-24 of the value before the bias and one of the
sum with it, and half an ulp of the type (2^-24, 2^-8, 2^-11, in fp16 2^-25 below
its normal numbers)."""
import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod, say
from oracle import lin as oracle

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


class Matrix:
    def __init__(self, N, K, max_rows, bias=True, M=1, layer=0, seed=0, stream=None):
        r = np.random.default_rng(seed)
        self.N, self.K, self.layer, self.rng = N, K, layer, r
        self.codes = r.integers(-128, 128, (M, N, K)).astype(np.int8)
        self.scales = ((0.5 + r.random((M, N))) / (73 * np.sqrt(K))).astype(np.float32)
        self.bias = r.standard_normal((M, N)).astype(np.float32) if bias else None
        up = lambda v: None if v is None else torch.from_numpy(v).to(dev())  # noqa: E731
        self.ctx = lcsm_mod().Q8(up(self.codes), up(self.scales), max_rows, bias=up(self.bias), stream=stream)

    def rows(self, R, dtype, pad=0):
        return torch.from_numpy(self.rng.standard_normal((R, self.K + 2 * pad)).astype(np.float32)).to(TYPES[dtype]).to(
            dev())[:, pad:pad + self.K]

    def check(self, y, x, dtype):
        m = self.layer
        want, size = oracle.q8(x.double().cpu().numpy(), self.codes[m], self.scales[m], None if self.bias is None else self.bias[m])
        torch.cuda.synchronize()
        got = y.double().cpu().numpy()
        # (rounding to a type takes what is beyond its largest number to infinity)
        fine = np.isfinite(want) & (np.abs(np.nan_to_num(want)) <= torch.finfo(TYPES[dtype]).max)
        assert np.array_equal(fine, np.isfinite(got))
        room = ULP[dtype] * np.abs(want) + 2.0 ** -24 * (3 * size + 2 * np.abs(want)) + (2.0 ** -25 if dtype == "f16" else 1e-38)
        far = np.abs(got - want) - (1 + 1e-3) * room
        assert far[fine].max(initial=-1.0) <= 0, (far[fine].max(), room[fine].max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", [(1, 1), (16, 64), (17, 65), (33, 63), (100, 200), (64, 773), (257, 128), (130, 1029), (512, 384),
                                 (300, 2048)])
def test_sizes(N, K, dtype):
    m = Matrix(N, K, 300, seed=N + K)
    for R in (1, 2, 3, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 300):
        say(f"[q8] {R} x {K} -> {N} {dtype}")
        x = m.rows(R, dtype)
        m.check(m.ctx.matmul(0, x), x, dtype)


@pytest.mark.parametrize("R,N,K", [(1, 8192, 2048), (4, 2048, 4096), (40, 5000, 640), (256, 256, 256), (257, 513, 1000), (513, 1025, 130),
                                   (1024, 768, 512), (2000, 300, 700), (700, 2000, 90), (128, 4096, 1024), (512, 2048, 300)])
def test_large(R, N, K):
    m = Matrix(N, K, R, bias=False, seed=R)
    for dtype in ("bf16", "f32"):
        say(f"[q8] {R} x {K} -> {N} {dtype}")
        x = m.rows(R, dtype)
        m.check(m.ctx.matmul(0, x), x, dtype)


@pytest.mark.parametrize("R,N", [(3500, 3600), (2500, 2600), (1300, 2600), (700, 1500), (90, 2400), (40, 4500)])
@pytest.mark.parametrize("K", [70, 300])
def test_every_size_of_pieces(R, N, K):
    """Pieces of each size, whole ones and such that end inside, with and without a bias, an odd and an even number of stages."""
    for dtype, bias in (("f16", True), ("f32", False)):
        say(f"[q8] {R} x {K} -> {N} {dtype}")
        m = Matrix(N, K, R, bias=bias, seed=R + K)
        x = m.rows(R, dtype)
        m.check(m.ctx.matmul(0, x), x, dtype)


def test_longest_sums():
    """Every code at its end, over the longest rows: the sums reach 2^31."""
    K = 1 << 17
    m = Matrix(3, K, 20, seed=1)
    codes = torch.tensor([[-128] * K, [127] * K, [-128, 127] * (K // 2)], dtype=torch.int8, device=dev())[None]
    m.codes = codes.cpu().numpy()
    m.ctx = lcsm_mod().Q8(codes, torch.from_numpy(m.scales).to(dev()), 20, bias=torch.from_numpy(m.bias).to(dev()))
    x = torch.ones((20, K), device=dev())
    x[1] = -1.0
    for R in (2, 20):
        m.check(m.ctx.matmul(0, x[:R]), x[:R], "f32")


@pytest.mark.parametrize("dtype", TYPES)
def test_codes_of_borders(dtype):
    """Values half way between two codes go to the even one, and their neighbours to their own side: weights of one
    show the code itself."""
    K = 512
    big = {"f32": 127.0, "bf16": 127.0, "f16": 127.0}[dtype]
    m = Matrix(K, K, 40, bias=False, seed=2)
    m.codes = np.eye(K, dtype=np.int8)[None]
    m.scales = np.ones((1, K), np.float32)
    m.ctx = lcsm_mod().Q8(*(torch.from_numpy(v).to(dev()) for v in (m.codes, m.scales)), 40)
    half = (torch.arange(K) % 254 - 127 + 0.5).clamp(-126.5, 126.5)
    for factor in (1.0, 2.0 ** -10, 3.0, 0.7, 1e-30, 1e30) if dtype != "f16" else (1.0, 2.0 ** -10, 3.0, 0.7):
        v = (half * factor).to(TYPES[dtype])
        v[0] = big * factor
        ints = v.view(torch.int32 if dtype == "f32" else torch.int16).clone()
        rows = torch.stack([v] + [(ints + d).view(TYPES[dtype]) for d in (-1, 1, -2, 2)]).to(dev())
        rows[:, 0] = big * factor
        m.check(m.ctx.matmul(0, rows), rows, dtype)


def test_smallest_and_largest_values():
    m = Matrix(40, 100, 40, bias=False, seed=3)
    x = m.rows(40, "f32")
    x[0] = 0.0
    x[1] *= 1e-38
    x[2] = 1e-44
    x[3] *= 3e37
    x[4] = 0.0
    x[4, 7] = 1e-45
    x[5] *= 1e-42
    x[6] = 3.4e38
    m.check(m.ctx.matmul(0, x), x, "f32")


def test_rows_apart():
    m = Matrix(70, 200, 40, seed=4)
    for R in (5, 40):
        x = m.rows(R, "bf16")
        x[1, 3], x[3, 199], x[4, 0] = float("nan"), float("inf"), float("-inf")
        y = m.ctx.matmul(0, x)
        m.check(y, x, "bf16")
        fine = torch.isfinite(y).all(-1).tolist()
        assert fine[:5] == [True, False, True, False, False] and all(fine[5:])


@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("R", [2, 50, 300])
def test_slices_and_layers(R, pad):
    m = Matrix(90, 150, 300, M=3, layer=2, seed=pad)
    for dtype in TYPES:
        x = m.rows(R, dtype, pad)
        wide = torch.full((R, 90 + 2 * pad), 7.0, dtype=TYPES[dtype], device=dev())
        m.check(m.ctx.matmul(2, x, y=wide[:, pad:pad + 90]), x, dtype)
        assert bool((wide[:, :pad] == 7).all()) and bool((wide[:, pad + 90:] == 7).all())


def test_rows_beyond_two_to_the_31_elements():
    m = Matrix(32, 64, 140, seed=5)
    x = m.rows(130, "bf16")
    stride = 1 << 24
    far = torch.empty(129 * stride + 64, dtype=torch.bfloat16, device=dev()).as_strided((130, 64), (stride, 1))
    far.copy_(x)
    m.check(m.ctx.matmul(0, far), x, "bf16")
    y = torch.empty(129 * stride + 64, dtype=torch.bfloat16, device=dev()).as_strided((130, 32), (stride, 1))
    m.check(m.ctx.matmul(0, x, y=y), x, "bf16")


def test_calls_in_turn_and_again():
    """Calls of different sizes over one workspace leave nothing behind, and repeat bit for bit."""
    m = Matrix(200, 333, 400, seed=6)
    xs = [m.rows(R, "f32") for R in (400, 1, 17, 400, 130, 2)]
    first = [m.ctx.matmul(0, x) for x in xs]
    again = [m.ctx.matmul(0, x) for x in xs]
    for x, a, b in zip(xs, first, again):
        assert torch.equal(a, b)
        m.check(a, x, "f32")


@pytest.mark.parametrize("R", [1, 20, 200])
def test_another_stream_and_a_graph(R):
    stream = torch.cuda.Stream(dev())
    m = Matrix(100, 300, 200, seed=7, stream=stream)
    x = m.rows(R, "bf16")
    m.check(m.ctx.matmul(0, x), x, "bf16")
    with torch.cuda.stream(stream):
        y = torch.empty((R, 100), dtype=torch.bfloat16, device=dev())
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            m.ctx.matmul(0, x, y=y)
        for _ in range(3):
            y.fill_(float("nan"))
            x.neg_()
            m.ctx.matmul(0, x)
            g.replay()
            m.check(y, x, "bf16")


@pytest.mark.parametrize("K", [9, 1100])
def test_very_many_rows(K):
    """Rows whose codes take more than one line of workgroups: the first, those around the line's end and the last."""
    R, line = 600_000, 4096 * 128
    m = Matrix(7, K, R, seed=K)
    x = torch.randn((1000, K), generator=torch.Generator().manual_seed(3)).bfloat16().to(dev()).repeat(R // 1000, 1)
    x *= torch.exp2((torch.arange(R, device=dev()) % 7).float())[:, None].bfloat16()
    say(f"[q8] {R} x {K}")
    y = m.ctx.matmul(0, x)
    for a, b in ((0, 300), (line - 150, line + 150), (R - 300, R)):
        m.check(y[a:b], x[a:b], "bf16")


def test_quantize():
    lcsm = lcsm_mod()
    r = np.random.default_rng(8)
    for shape in ((5, 1), (2, 3, 130), (64, 1000)):
        w = r.standard_normal(shape).astype(np.float32)
        w.reshape(-1, shape[-1])[0] = 0.0
        w.reshape(-1, shape[-1])[1, 0] = np.inf
        codes, scales = lcsm.Q8.quantize(torch.from_numpy(w).to(dev()))
        want, s = oracle.codes(w.reshape(-1, shape[-1]))
        assert np.array_equal(codes.cpu().numpy().reshape(want.shape), want)
        assert np.array_equal(scales.cpu().numpy().reshape(-1), s.astype(np.float32), equal_nan=True)
    codes, scales = lcsm.Q8.quantize(torch.empty((0, 4), device=dev()))
    assert codes.shape == (0, 4) and scales.shape == (0,)


def test_quantize_very_many_rows():
    rows = (1 << 26) + 70  # more waves than a launch has
    w = torch.ones((rows, 1), device=dev())
    w[-3], w[5] = -2.0, 0.0
    codes, scales = lcsm_mod().Q8.quantize(w)
    want = torch.full_like(codes, 127)
    want[-3], want[5] = -127, 0
    assert torch.equal(codes, want)
    assert torch.equal(scales, w.abs().squeeze(1) / 127)


def test_refusals():
    lcsm = lcsm_mod()
    m = Matrix(20, 30, 8, seed=9)
    x = m.rows(4, "f32")
    for bad in (dict(x=x[:, :29]), dict(x=x.double()), dict(x=x.t().contiguous().t()), dict(x=x.cpu()), dict(y=x), dict(
            y=torch.empty((4, 20), dtype=torch.bfloat16, device=dev()))):
        with pytest.raises(ValueError):
            m.ctx.matmul(0, **{"x": x, **bad})
    for layer, R in ((1, 4), (-1, 4), (2 ** 32, 4), (0, 9)):
        with pytest.raises(lcsm.LcsmError) as e:
            m.ctx.matmul(layer, m.rows(R, "f32"))
        assert e.value.code == lcsm.LCSM_EINVAL
    m.check(m.ctx.matmul(0, x), x, "f32")  # no refusal faults the context
    assert m.ctx.matmul(0, x[:0]).shape == (0, 20)
    codes, scales = torch.ones((1, 4, 8), dtype=torch.int8, device=dev()), torch.ones((1, 4), device=dev())
    for args, kw in (((codes.int(), scales, 4), {}), ((codes, scales[:, :3], 4), {}), ((codes, scales.double(), 4), {}),
                     ((codes, scales, 4 + 2 ** 32), {}), ((codes.cpu(), scales, 4), {}), ((codes[0], scales, 4), {}),
                     ((codes, scales, 4), dict(bias=scales.cpu()))):
        with pytest.raises(ValueError):
            lcsm.Q8(*args, **kw)
    for rows in (0, -1, (1 << 24) + 1):
        with pytest.raises(lcsm.LcsmError):
            lcsm.Q8(codes, scales, rows)
    with pytest.raises(ValueError):
        lcsm.Q8.quantize(torch.ones((4, 8), dtype=torch.bfloat16, device=dev()))
