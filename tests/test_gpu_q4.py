"""Products with 4-bit weights (lcsm_q4.h) against the fp64 oracle on the GPU
(needs an MI355X).

Tolerances, as a share of the largest output: it is rounded once to its type
(half an ulp: 2^-24, 2^-8, 2^-11).  Before that, products are exact and summed
in fp32 as (16 + code) x, from which (16 + zero) x comes off again: terms of up
to 31 |x| where the result's are 4.6 |x| on average, so a rounding of 2^-24 of
a running sum counts seven times; K / 32 such sums a row give 7 sqrt(K / 32)
2^-24 of a typical output, below 1e-5 up to K = 16384 (32 sums of a step are
rounded once more each)."""
import ctypes

import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod, say
from oracle import ssm as oracle

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SUMS = 1e-5


class Case:
    def __init__(self, N, K, group, sdtype="f32", zeros=False, bias=False, M=1, seed=0, stream=None):
        r = np.random.default_rng(seed)
        ng = -(-K // group)
        self.N, self.K, self.group, self.rng = N, K, group, r
        codes = r.integers(0, 256, (M, N, (K + 1) // 2), dtype=np.uint8)
        scales = torch.from_numpy(((0.5 + r.random((M, N, ng))) / np.sqrt(K)).astype(np.float32)).to(TYPES[sdtype])
        z = r.integers(0, 256, (M, N, ng), dtype=np.uint8) if zeros else None
        self.bias = r.standard_normal((M, N)).astype(np.float32) if bias else None
        up = lambda v: None if v is None else torch.from_numpy(v).to(dev())  # noqa: E731
        self.ctx = lcsm_mod().Q4(up(codes), scales.to(dev()), K, group, zeros=up(z), bias=up(self.bias), stream=stream)
        self.w = [oracle.q4_weights(codes[m].astype(np.int64), scales[m].double().numpy(), None if z is None else z[m], K, group)
                  for m in range(M)]

    def x(self, R, dtype, pad=0):
        t = torch.from_numpy(self.rng.standard_normal((R, self.K + 2 * pad)).astype(np.float32)).to(TYPES[dtype]).to(dev())
        return t[:, pad:pad + self.K]

    def want(self, x, m=0):
        y = x.double().cpu().numpy() @ self.w[m].T
        return y if self.bias is None else y + self.bias[m]

    def check(self, y, x, dtype, m=0):
        want = self.want(x, m)
        torch.cuda.synchronize()
        got = y.double().cpu().numpy()
        assert got.shape == want.shape
        err = np.abs(got - want).max() / np.abs(want).max()
        assert err <= SUMS + ULP[dtype], err


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K,group", [(1, 1, 32), (16, 128, 128), (17, 129, 32), (100, 32, 32), (33, 1000, 64), (64, 770, 128),
                                       (256, 1536, 256), (1543, 773, 32), (48, 4096, 4096), (2048, 4096, 64), (5, 16384, 128)])
def test_sizes(N, K, group, dtype):
    c = Case(N, K, group, "f32" if dtype == "f32" else dtype, zeros=N % 2 == 1, bias=N % 3 == 0, seed=N + K)
    for R in (1, 2, 5, 16, 17, 33, 64, 65):
        say(f"[q4] {R} rows x {N} x {K} group {group} {dtype}")
        x = c.x(R, dtype)
        c.check(c.ctx.matvec(0, x), x, dtype)


@pytest.mark.parametrize("sdtype", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
def test_scales_zeros_and_layers(sdtype, zeros):
    c = Case(70, 300, 64, sdtype, zeros=zeros, bias=True, M=3, seed=3)
    for m in (2, 0, 1):
        x = c.x(3, "f32")
        c.check(c.ctx.matvec(m, x), x, "f32", m)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad", [1, 3, 8])
def test_strides_and_starts(dtype, pad):
    c = Case(40, 256, 128, seed=4)
    x = c.x(6, dtype, pad)
    wide = torch.full((6, 40 + 2 * pad), 7.0, dtype=TYPES[dtype], device=dev())
    c.check(c.ctx.matvec(0, x, wide[:, pad:pad + 40]), x, dtype)
    assert bool((wide[:, :pad] == 7.0).all()) and bool((wide[:, pad + 40:] == 7.0).all())


def test_exact_for_whole_numbers():
    """Codes, scales of one and whole x: every output is exact."""
    K, N = 512, 32
    r = np.random.default_rng(5)
    codes = torch.from_numpy(r.integers(0, 256, (1, N, K // 2), dtype=np.uint8)).to(dev())
    ctx = lcsm_mod().Q4(codes, torch.ones((1, N, 4), device=dev()), K, 128)
    x = torch.from_numpy(r.integers(-8, 9, (9, K)).astype(np.float32)).to(dev())
    w = oracle.q4_weights(codes[0].cpu().numpy().astype(np.int64), np.ones((N, 4)), None, K, 128)
    for dtype in TYPES.values():
        y = ctx.matvec(0, x.to(dtype))
        want = torch.from_numpy(x.double().cpu().numpy() @ w.T).to(dtype)
        assert torch.equal(y.cpu(), want)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_apart(dtype):
    """Rows of zeros, tiny, large and not finite values beside ordinary ones."""
    c = Case(48, 384, 128, seed=6)
    x = c.x(6, dtype)
    x[0] = 0.0
    x[1] *= 1e-3
    x[2] *= 1e3
    x[3, 7], x[4, 200] = float("nan"), float("inf")
    y = c.ctx.matvec(0, x)
    torch.cuda.synchronize()
    assert not torch.isfinite(y[3:5]).any()
    for k in (0, 1, 2, 5):
        want, got = c.want(x[k:k + 1])[0], y[k].double().cpu().numpy()
        assert np.abs(got - want).max() <= (SUMS + ULP[dtype]) * np.abs(want).max(), k


def test_no_rows_streams_and_a_graph():
    stream = torch.cuda.Stream(dev())
    c = Case(100, 640, 64, "bf16", seed=7, stream=stream)
    assert c.ctx.matvec(0, c.x(0, "bf16")).shape == (0, 100)
    x = c.x(4, "bf16")
    c.check(c.ctx.matvec(0, x), x, "bf16")
    with torch.cuda.stream(stream):
        y = torch.empty((4, 100), dtype=torch.bfloat16, device=dev())
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            c.ctx.matvec(0, x, y)
        for _ in range(3):
            y.fill_(float("nan"))
            g.replay()
            c.check(y, x, "bf16")


def test_rows_beyond_two_to_the_31_elements():
    c = Case(20, 64, 32, seed=8)
    stride = 1 << 24
    x = c.x(130, "bf16")
    big = torch.empty(129 * stride + 64, dtype=torch.bfloat16, device=dev()).as_strided((130, 64), (stride, 1))
    big.copy_(x)
    c.check(c.ctx.matvec(0, big), x, "bf16")


@pytest.mark.parametrize("sdtype", TYPES)
@pytest.mark.parametrize("K,group", [(128, 128), (257, 64), (31, 32), (1000, 256), (1, 32)])
def test_quantize(K, group, sdtype):
    """Codes and scales by the rule, bit for bit, and weights within half a
    step of what they stand for."""
    r = np.random.default_rng(K)
    w = r.standard_normal((2, 9, K)).astype(np.float32)
    w[0, 3] = 0.0
    w[1, 2, ::3] = -7.0
    codes, scales = lcsm_mod().Q4.quantize(torch.from_numpy(w).to(dev()), group, TYPES[sdtype])
    torch.cuda.synchronize()
    ng = -(-K // group)
    padded = np.zeros((2, 9, ng * group), np.float32)
    padded[..., :K] = w
    most = np.abs(padded).reshape(2, 9, ng, group).max(-1)
    want = torch.from_numpy(most / np.float32(7)).to(TYPES[sdtype])
    assert torch.equal(scales.cpu(), want)
    s = want.float().numpy()[..., np.arange(K) // group]
    with np.errstate(invalid="ignore", divide="ignore"):
        q = np.where(s == 0, 8, np.clip(np.rint(w / s) + 8, 0, 15)).astype(np.int64)
    if K % 2:
        q = np.concatenate([q, np.full(q.shape[:-1] + (1,), 8)], -1)
    assert np.array_equal(codes.cpu().numpy(), (q[..., 0::2] | q[..., 1::2] << 4).astype(np.uint8))
    ctx = lcsm_mod().Q4(codes, scales, K, group)
    y = ctx.matvec(1, torch.eye(K, device=dev())).cpu().numpy()
    # a scale rounded down by its type can leave the largest weights half a step and its rounding short
    assert np.abs(y - w[1].T).max() <= (0.5 + 7 * ULP[sdtype] + SUMS) * most[1].max() / 7 * (1 + ULP[sdtype])


def test_a_library_workspace_and_refusals():
    lcsm = lcsm_mod()
    lib = lcsm.raw()
    codes = torch.zeros((1, 8, 16), dtype=torch.uint8, device=dev())
    scales = torch.ones((1, 8, 1), device=dev())
    shape, ctx = lcsm.Q4Shape(1, 8, 32, 32, 0), ctypes.c_void_p()
    st = torch.cuda.current_stream().cuda_stream
    init = lambda sh, c, s, ws=None, n=0: lib.lcsm_q4_init(ctypes.byref(ctx), ctypes.byref(sh), c, s, None, None, st, ws, n)  # noqa: E731
    assert init(shape, codes.data_ptr(), scales.data_ptr()) == 0
    x, y = torch.ones((3, 32), device=dev()), torch.zeros((3, 8), device=dev())
    run = lambda *a: lib.lcsm_q4_matvec(ctx, *a)  # noqa: E731
    assert run(0, 3, 0, x.data_ptr(), 32, y.data_ptr(), 8) == 0
    torch.cuda.synchronize()
    assert bool((y == -256.0).all())
    bad = [run(1, 3, 0, x.data_ptr(), 32, y.data_ptr(), 8), run(-1, 3, 0, x.data_ptr(), 32, y.data_ptr(), 8),
           run(0, -1, 0, x.data_ptr(), 32, y.data_ptr(), 8), run(0, 3, 3, x.data_ptr(), 32, y.data_ptr(), 8),
           run(0, 3, 0, None, 32, y.data_ptr(), 8), run(0, 3, 0, x.data_ptr(), 32, None, 8),
           run(0, 3, 0, x.data_ptr(), 31, y.data_ptr(), 8), run(0, 3, 0, x.data_ptr(), 32, y.data_ptr(), 7)]
    assert bad == [lcsm.LCSM_EINVAL] * len(bad)
    lib.lcsm_q4_destroy(ctx)
    assert init(shape, codes.data_ptr(), scales.data_ptr(), codes.data_ptr(), 1) == lcsm.LCSM_ENOMEM
    assert init(shape, None, scales.data_ptr()) == lcsm.LCSM_EINVAL
    with pytest.raises(lcsm.LcsmError):
        lcsm.Q4(codes, torch.ones((1, 8, 1), device=dev()), 32, 48)
    for args in ((codes, scales[:, :, :0], 32, 32), (codes, scales, 40, 32), (codes.float(), scales, 32, 32), (codes[0], scales, 32, 32)):
        with pytest.raises(ValueError):
            lcsm.Q4(*args)
    q = lcsm.Q4(codes, scales, 32, 32)
    for a in ((x[:, :31],), (x.double(),), (x.cpu(),), (x, y.bfloat16()), (x, y[:2]), (x.t().contiguous().t(),)):
        with pytest.raises(ValueError):
            q.matvec(0, *a)
    with pytest.raises(lcsm.LcsmError):
        q.matvec(1, x)
    with pytest.raises(lcsm.LcsmError):
        lcsm.Q4.quantize(x, 48)
