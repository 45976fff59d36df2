"""The norms around a block (lcsm_norm.h) against the fp64 oracle on the GPU
(needs an MI355X).

Tolerances: an output is rounded once to its type, by at most half an ulp of
itself (2^-24, 2^-8, 2^-11 of the largest value); before that a value has gone
through a dozen fp32 roundings and two sums over the row of error below 2^-20
(sums of up to 32768 terms, tens of them in a chain): 4e-6 of the largest."""
import ctypes

import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod, say
from oracle import ssm as oracle

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SUMS = 4e-6


def close(got, want, tol, what=""):
    got = got.double().cpu().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), what
    if fine.any():
        err = np.abs(got[fine] - want[fine]).max() / np.abs(want[fine]).max()
        assert err <= tol, (what, err, tol)


class Case:
    def __init__(self, R, D, dtype="f32", rdtype=None, post="rms", pre="rms", act="none", groups=1, alpha=1.0, weights=True,
                 block=True, M=1, layer=0, seed=0, pad=0, stream=None):
        r = np.random.default_rng(seed)
        self.dtype, self.rdtype = dtype, rdtype or dtype
        rows = lambda t, on=True: (torch.from_numpy(r.standard_normal((R, D + 2 * pad)).astype(np.float32)).to(  # noqa: E731
            TYPES[t]).to(dev())[:, pad:pad + D] if on else None)
        self.o, self.g, self.r = rows(dtype, block), rows(dtype, block and act != "none"), rows(self.rdtype)
        vec = lambda mid: (mid + 0.1 * r.standard_normal((M, D))).astype(np.float32) if weights else None  # noqa: E731
        self.w = [vec(1.0), vec(0.0), vec(0.3), vec(1.0), vec(0.0)]
        names = ("post_weight", "post_bias", "scale", "pre_weight", "pre_bias")
        kw = {n: torch.from_numpy(v).to(dev()) for n, v in zip(names, self.w) if v is not None}
        self.kw = dict(post=post, pre=pre, act=act, groups=groups, alpha=alpha, eps=1e-5)
        self.layer = layer
        self.ctx = lcsm_mod().Norm(D, dtype=TYPES[dtype], res_dtype=TYPES[self.rdtype], layers=M, stream=stream, **self.kw, **kw)

    def want(self):
        n = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
        w = [None if v is None else v[self.layer].astype(np.float64) for v in self.w]
        return oracle.block_norm(n(self.o), n(self.g), n(self.r), *(self.kw[k] for k in ("post", "pre", "act", "groups", "alpha",
                                                                                         "eps")), *w)

    def check(self, got, want=None):
        res, out = self.want() if want is None else want
        torch.cuda.synchronize()
        close(got[0], res, SUMS + ULP[self.rdtype], "residual")
        close(got[1], out, SUMS + ULP[self.dtype], "norm")


@pytest.mark.parametrize("dtype,rdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("D", [1, 5, 64, 512, 520, 771, 2048, 2056, 4099, 8192, 12288, 20001, 32768])
def test_widths(D, dtype, rdtype):
    for R in (1, 3, 9):
        say(f"[norm] {R} x {D} {dtype} {rdtype}")
        c = Case(R, D, dtype, rdtype, post="layer" if D > 1 else "rms", act="silu", seed=D)
        c.check(c.ctx.block(0, c.o, c.r, gate=c.g))


@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("act", ["none", "silu", "sigmoid"])
@pytest.mark.parametrize("weights", [True, False])
def test_kinds(post, pre, act, weights):
    c = Case(7, 768, "bf16", "f32", post, pre, act, alpha=2.25, weights=weights, M=3, layer=2, seed=1)
    c.check(c.ctx.block(2, c.o, c.r, gate=c.g))


@pytest.mark.parametrize("D,groups", [(768, 8), (768, 768), (6, 3), (4096, 64), (4098, 3), (12288, 1024), (32768, 2)])
@pytest.mark.parametrize("post", ["rms", "layer"])
def test_groups(D, groups, post):
    c = Case(5, D, "f16", "f32", post, "rms", "silu", groups=groups, seed=D)
    c.check(c.ctx.block(0, c.o, c.r, gate=c.g))


@pytest.mark.parametrize("D,pad", [(512, 1), (512, 8), (100, 3), (8200, 4)])
def test_strides_and_starts(D, pad):
    """Slices of wider rows, some of which begin between two vectors."""
    for dtype, rdtype in (("bf16", "f32"), ("f32", "f32"), ("f16", "f16")):
        c = Case(6, D, dtype, rdtype, act="sigmoid", pad=pad, seed=pad)
        want = c.want()
        wide = torch.full((6, D + 2 * pad), 7.0, dtype=TYPES[dtype], device=dev())
        c.check(c.ctx.block(0, c.o, c.r, gate=c.g, out=wide[:, pad:pad + D]), want)
        assert bool((wide[:, :pad] == 7.0).all()) and bool((wide[:, pad + D:] == 7.0).all())
        c.check(c.ctx.block(0, c.o, c.r, gate=c.g, res_out=c.r, out=c.o), want)  # in place


@pytest.mark.parametrize("D", [768, 4096])
def test_first_and_last_block(D):
    """No block before (the norm alone), and no norm after (the sum alone)."""
    c = Case(4, D, "bf16", "f32", block=False, seed=2)
    res, out = c.ctx.block(0, None, c.r, res_out=False)
    assert res is None
    torch.cuda.synchronize()
    close(out, c.want()[1], SUMS + ULP["bf16"])
    c = Case(4, D, "bf16", "f32", seed=3)
    res, out = c.ctx.block(0, c.o, c.r, out=False)
    assert out is None
    torch.cuda.synchronize()
    close(res, c.want()[0], SUMS)


@pytest.mark.parametrize("D", [768, 4096])
def test_rows_apart(D):
    """Rows of zeros, of one value, of large values, and one with a value that
    is not finite: each is what it is alone."""
    c = Case(6, D, "f32", post="layer", pre="layer", seed=4)
    c.o[0], c.r[0] = 0.0, 0.0
    c.o[1] = 3.0
    c.o[2] *= 1e15
    c.r[3, D // 2] = float("nan")
    c.o[4, 5] = float("inf")
    got = c.ctx.block(0, c.o, c.r)
    with np.errstate(invalid="ignore"):
        want = c.want()
    torch.cuda.synchronize()
    for k in range(6):
        for a, b, tol in zip(got, want, (SUMS, SUMS)):
            if k == 1:
                # the differences from the mean are roundings of 3.0: 2^-24 of it, measured against eps = 1e-5
                tol = 1e-3
            close(a[k], b[k], tol, f"row {k}")


def test_many_rows_and_none():
    c = Case(3001, 130, "f16", post="rms", pre="layer", act="silu", seed=5)
    c.check(c.ctx.block(0, c.o, c.r, gate=c.g))
    res, out = c.ctx.block(0, c.o[:0], c.r[:0], gate=c.g[:0])
    assert res.shape == out.shape == (0, 130)


def test_rows_beyond_two_to_the_31_elements():
    c = Case(130, 64, "bf16", "bf16", seed=6)
    stride = 1 << 24
    big = torch.empty(129 * stride + 64, dtype=torch.bfloat16, device=dev()).as_strided((130, 64), (stride, 1))
    big.copy_(c.o)
    c.check(c.ctx.block(0, big, c.r))


def test_another_stream_and_a_graph():
    stream = torch.cuda.Stream(dev())
    c = Case(33, 768, "bf16", "f32", act="silu", seed=7, stream=stream)
    want = c.want()
    c.check(c.ctx.block(0, c.o, c.r, gate=c.g), want)
    with torch.cuda.stream(stream):
        res, out = torch.empty_like(c.r), torch.empty_like(c.o)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            c.ctx.block(0, c.o, c.r, gate=c.g, res_out=res, out=out)
        for _ in range(3):
            res.fill_(float("nan"))
            out.fill_(float("nan"))
            g.replay()
            c.check((res, out), want)


def test_refusals():
    lcsm = lcsm_mod()
    lib = lcsm.raw()
    for k, v in (("D", 0), ("D", 32769), ("groups", 3), ("groups", 0), ("eps", -1.0), ("eps", float("nan")), ("alpha", float("inf"))):
        args = dict(D=16)
        args[k] = v
        with pytest.raises(lcsm.LcsmError):
            lcsm.Norm(**args)
    with pytest.raises(lcsm.LcsmError):
        lcsm.Norm(16, dtype=torch.bfloat16, res_dtype=torch.float16)
    with pytest.raises(KeyError):
        lcsm.Norm(16, post="batch")
    c = Case(4, 16, act="silu", seed=8)
    for args in (dict(o=c.o[:3]), dict(o=c.o.double()), dict(res=c.r.cpu()), dict(gate=c.g.t().contiguous().t()),
                 dict(out=c.o.bfloat16()), dict(res_out=c.r[:, :8])):
        kw = dict(o=c.o, res=c.r, gate=c.g)
        kw.update(args)
        with pytest.raises(ValueError):
            c.ctx.block(0, **kw)
    for kw in (dict(gate=None), dict(o=None), dict(layer=1), dict(layer=-1), dict(res_out=False, out=False)):
        args = dict(layer=0, o=c.o, res=c.r, gate=c.g)
        args.update(kw)
        with pytest.raises(lcsm.LcsmError) as e:
            c.ctx.block(**args)
        assert e.value.code == lcsm.LCSM_EINVAL
    p = c.o.data_ptr()
    io = lcsm.NormIo(p, p, p, p, p, 15, 16, 16, 16, 16)
    assert lib.lcsm_norm_block(c.ctx._ctx, 0, 4, ctypes.byref(io)) == lcsm.LCSM_EINVAL
    assert lib.lcsm_norm_block(c.ctx._ctx, 0, 4, None) == lcsm.LCSM_EINVAL
    assert lib.lcsm_norm_block(c.ctx._ctx, 0, -1, ctypes.byref(io)) == lcsm.LCSM_EINVAL
    assert lib.lcsm_norm_block(None, 0, 4, ctypes.byref(io)) == lcsm.LCSM_EINVAL


@pytest.mark.parametrize("D,groups", [(24, 4), (64, 4), (512, 512), (300, 100), (510, 5), (513, 27), (1025, 41), (2047, 23), (1001, 1),
                                      (8191, 1), (9001, 1)])
@pytest.mark.parametrize("dtype,rdtype", [("bf16", "f32"), ("f16", "f16")])
def test_parts_and_tails_stay_in_their_rows(D, groups, dtype, rdtype):
    """Short parts, rows that end inside a vector and begin at odd places: nothing beside a row is written."""
    c = Case(6, D, dtype, rdtype, "layer", "rms", "silu", groups=groups, pad=1, seed=D)
    res = torch.full((6, D + 9), 7.0, dtype=TYPES[rdtype], device=dev())
    out = torch.full((6, D + 9), 7.0, dtype=TYPES[dtype], device=dev())
    c.check(c.ctx.block(0, c.o, c.r, gate=c.g, res_out=res[:, 3:3 + D], out=out[:, 5:5 + D]))
    assert bool((res[:, :3] == 7).all()) and bool((res[:, 3 + D:] == 7).all())
    assert bool((out[:, :5] == 7).all()) and bool((out[:, 5 + D:] == 7).all())
