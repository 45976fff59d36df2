"""The norms of queries and keys for each head with their rotation (lcsm_rot.h)
against the fp64 oracle on the GPU (needs an MI355X).

Tolerances, as a share of the largest value of a row: an output is rounded once
to its type (2^-24, 2^-8, 2^-11); before that stand two sums over a head (up to
512 terms, a dozen of them in a chain), a division, a weight, and sine and cosine
of an angle rounded to fp32 (pi 2^-25) with their products: thirty roundings of
2^-24, 2e-6.  A head that the norm takes apart into differences from its mean
loses what those lose, which the test of such rows says."""
import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod, say
from oracle import lin as oracle

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
WORK = 2e-6


def close(got, want, tol, what=""):
    got = got.double().cpu().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), what
    for a, b, ok in zip(got, want, fine):
        if ok.any():
            assert np.abs(a[ok] - b[ok]).max() <= tol * np.abs(b[ok]).max(), (what, np.abs(a[ok] - b[ok]).max() / np.abs(b[ok]).max())


class Case:
    def __init__(self, T, P, H, G, rotary=None, pairs="half", norm="rms", dtype="f32", weights=True, M=1, layer=0, pad=0, seed=0,
                 base=10000.0, far=4096, stream=None, eps=1e-5):
        r = np.random.default_rng(seed)
        self.P, self.dtype, self.layer = P, dtype, layer
        self.rotary = P // 2 * 2 if rotary is None else rotary
        rows = lambda n: torch.from_numpy(r.standard_normal((T, n * P + 2 * pad)).astype(np.float32)).to(  # noqa: E731
            TYPES[dtype]).to(dev())[:, pad:pad + n * P]
        self.q, self.k = rows(H), rows(G) if G else None
        self.pos = r.integers(0, far, T).astype(np.int32)
        self.positions = torch.from_numpy(self.pos).to(dev())
        self.w = [(1 + 0.1 * r.standard_normal((M, P))).astype(np.float32) if weights else None for _ in "qk"]
        self.freqs = np.array([base ** (-2.0 * j / self.rotary) for j in range(self.rotary // 2)])
        self.kw = dict(norm=norm, pairs=pairs)
        self.eps = eps
        up = lambda v: None if v is None else torch.from_numpy(v).to(dev())  # noqa: E731
        self.ctx = lcsm_mod().Rot(P, H, G, rotary=rotary, base=base, eps=eps, q_weight=up(self.w[0]), k_weight=up(self.w[1]),
                                  dtype=TYPES[dtype], layers=M, stream=stream, **self.kw)

    def want(self):
        return [None if x is None else oracle.heads(x.double().cpu().numpy(), self.P, self.kw["norm"],
                                                    None if w is None else w[self.layer], np.float32(self.eps), self.pos,
                                                    self.freqs, self.kw["pairs"]) for x, w in zip((self.q, self.k), self.w)]

    def check(self, got, want=None, tol=None):
        torch.cuda.synchronize()
        for a, b, name in zip(got, self.want() if want is None else want, "qk"):
            if b is None:
                assert a is None
            else:
                close(a, b, (WORK if tol is None else tol) + ULP[self.dtype], name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairs", ["half", "adjacent"])
@pytest.mark.parametrize("P,rotary", [(1, None), (2, None), (3, None), (8, 4), (16, None), (40, 18), (50, 18), (64, None), (64, 32),
                                      (72, 8), (99, 98), (128, None), (128, 116), (130, 0), (200, 160), (256, None), (257, 6),
                                      (512, None), (511, 0), (509, 508)])
def test_heads(P, rotary, pairs, dtype):
    for T, H, G, norm in ((1, 1, 1, "rms"), (5, 3, 2, "layer" if P > 1 else "rms"), (3, 2, 0, "none")):
        say(f"[rot] {T} x {H}+{G} x {P} turned {rotary} {pairs} {norm} {dtype}")
        # (two values are two roundings of their mean apart where they are alike: eps keeps that within a tenth)
        c = Case(T, P, H, G, rotary, pairs, norm, dtype, seed=P, eps=1e-5)
        if norm == "layer" and P < 8:
            for x in (c.q, c.k):
                x.copy_((torch.arange(x.shape[1], device=dev()) % P % 2 * 2.0 - 1.0 + 0.125 * torch.arange(T, device=dev())[:, None]))
        c.check(c.ctx.apply(0, c.q, c.k, c.positions))


@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
@pytest.mark.parametrize("weights", [True, False])
def test_layers_and_weights(norm, weights):
    c = Case(9, 64, 4, 2, norm=norm, weights=weights, M=3, layer=2, dtype="bf16", seed=1)
    c.check(c.ctx.apply(2, c.q, c.k, c.positions))


@pytest.mark.parametrize("far", [1 << 16, 1 << 24, 2 ** 31 - 1])
def test_far_positions(far):
    """Angles of far positions keep their fraction of a turn: fp64 leaves 2^31 2^-53 of a radian."""
    c = Case(40, 64, 2, 2, dtype="f32", far=far, seed=2)
    c.pos[:4] = [0, far - 1, -5, -far + 1]
    c.positions.copy_(torch.from_numpy(c.pos))
    c.check(c.ctx.apply(0, c.q, c.k, c.positions))


def test_many_rows():
    """Enough of them that a team goes through several heads of its token, odd counts of heads among them."""
    for H, G, P, dtype in ((7, 4, 64, "bf16"), (3, 0, 128, "f32"), (13, 13, 50, "f16")):
        T = 70000 // (H + G) * 8 // (8 if P < 64 else 1)
        c = Case(T, P, H, G, dtype=dtype, seed=3)
        c.check(c.ctx.apply(0, c.q, c.k, c.positions))


@pytest.mark.parametrize("P,pad", [(64, 1), (50, 3), (128, 8)])
def test_slices_and_in_place(P, pad):
    for dtype in TYPES:
        c = Case(6, P, 3, 2, dtype=dtype, pad=pad, seed=pad)
        want = c.want()
        wide = [torch.full((6, n * P + 2 * pad), 7.0, dtype=TYPES[dtype], device=dev()) for n in (3, 2)]
        outs = [w[:, pad:w.shape[1] - pad] for w in wide]
        got = c.ctx.apply(0, c.q, c.k, c.positions, q_out=outs[0], k_out=outs[1])
        c.check(got, want)
        for w in wide:
            assert bool((w[:, :pad] == 7).all()) and bool((w[:, w.shape[1] - pad:] == 7).all())
        c.check(c.ctx.apply(0, c.q, c.k, c.positions, q_out=c.q, k_out=c.k), want)


def test_one_projection_in_place():
    """Queries and keys as slices of one wide row, turned where they are; what lies beside them stays."""
    P, H, G, T = 32, 4, 2, 11
    c = Case(T, P, H, G, dtype="bf16", seed=5)
    row = torch.randn((T, 3 * 256), device=dev()).bfloat16()
    q, k = row[:, 16:16 + H * P], row[:, 300:300 + G * P]
    q.copy_(c.q)
    k.copy_(c.k)
    before = row.clone()
    want = c.want()
    c.check(c.ctx.apply(0, q, k, c.positions, q_out=q, k_out=k), want)
    before[:, 16:16 + H * P], before[:, 300:300 + G * P] = q, k
    assert torch.equal(before, row)


def test_heads_apart():
    """Values that are not finite, and large ones, touch their own head only."""
    c = Case(4, 64, 3, 2, dtype="f32", seed=6)
    c.q[0, 5] = float("nan")
    c.q[1, 64 + 9] = float("inf")
    c.q[2, 128:192] *= 1e15
    c.k[3, 3] = float("-inf")
    got = c.ctx.apply(0, c.q, c.k, c.positions)
    torch.cuda.synchronize()
    for x, want in zip(got, c.want()):
        x = x.double().cpu().numpy().reshape(-1, 64)
        want = want.reshape(-1, 64)
        fine = np.isfinite(want).all(-1)
        # (a head with inf is NaN there and zero elsewhere where the definition says so; it is its own)
        assert np.isfinite(x[fine]).all() and np.abs(x[fine] - want[fine]).max() <= (WORK + ULP["f32"]) * np.abs(want[fine]).max()
        assert not np.isfinite(x[~fine]).all(-1).any()
    # what is not turned is not made of products: a value that is not finite stays alone
    c = Case(2, 8, 1, 1, rotary=4, norm="none", dtype="f32", seed=7)
    c.q[0, 6] = float("inf")
    q, _ = c.ctx.apply(0, c.q, c.k, c.positions)
    assert np.array_equal(np.isfinite(q.cpu().numpy()), np.isfinite(c.q.cpu().numpy()))


def test_rows_beyond_two_to_the_31_elements():
    c = Case(130, 16, 2, 2, dtype="bf16", seed=8)
    stride = 1 << 24
    far = torch.empty(129 * stride + 64, dtype=torch.bfloat16, device=dev()).as_strided((130, 32), (stride, 1))
    far.copy_(c.q)
    c.check(c.ctx.apply(0, far, c.k, c.positions, q_out=far))


def test_another_stream_and_a_graph():
    stream = torch.cuda.Stream(dev())
    c = Case(33, 64, 4, 4, dtype="bf16", seed=9, stream=stream)
    want = c.want()
    c.check(c.ctx.apply(0, c.q, c.k, c.positions), want)
    with torch.cuda.stream(stream):
        outs = torch.empty_like(c.q), torch.empty_like(c.k)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            c.ctx.apply(0, c.q, c.k, c.positions, q_out=outs[0], k_out=outs[1])
        for _ in range(3):
            for o in outs:
                o.fill_(float("nan"))
            g.replay()
            c.check(outs, want)


def test_given_frequencies():
    lcsm = lcsm_mod()
    f = torch.tensor([1.0, 0.3, 1e-3], dtype=torch.float64, device=dev())
    c = Case(5, 16, 2, 1, rotary=6, norm="none", dtype="f32", weights=False, seed=10)
    ctx = lcsm.Rot(16, 2, 1, freqs=f, norm="none", dtype=torch.float32)
    assert ctx.rotary == 6
    c.freqs = f.cpu().numpy()
    c.check(ctx.apply(0, c.q, c.k, c.positions))


def test_refusals():
    lcsm = lcsm_mod()
    good = dict(P=16, q_heads=2, k_heads=1)
    for k, v in (("P", 0), ("P", 513), ("q_heads", 0), ("k_heads", -1), ("rotary", 3), ("rotary", 18), ("rotary", -2), ("eps", -1.0),
                 ("eps", float("nan"))):
        with pytest.raises((lcsm.LcsmError, ValueError)):
            lcsm.Rot(**{**good, k: v})
    for k in good:
        with pytest.raises(ValueError):
            lcsm.Rot(**{**good, k: good[k] + 2 ** 32})
    with pytest.raises(KeyError):
        lcsm.Rot(**good, pairs="thirds")
    with pytest.raises(KeyError):
        lcsm.Rot(**good, norm="batch")
    with pytest.raises(ValueError):
        lcsm.Rot(**good, freqs=torch.ones(4, device=dev()))  # fp32
    with pytest.raises(ValueError):
        lcsm.Rot(**good, q_weight=torch.ones((1, 15), device=dev()))
    c = Case(4, 16, 2, 1, dtype="f32", seed=11)
    bad = [dict(q=c.q[:, :16]), dict(q=c.q.double()), dict(k=c.k[:3]), dict(k=c.k.cpu()), dict(positions=c.positions.long()),
           dict(positions=c.positions[:3]), dict(q=c.q.t().contiguous().t()), dict(q_out=c.q.bfloat16()), dict(k_out=c.k[:2])]
    for more in bad:
        kw = dict(q=c.q, k=c.k, positions=c.positions)
        kw.update(more)
        with pytest.raises(ValueError):
            c.ctx.apply(0, **kw)
    for layer in (1, -1, 2 ** 32, -2 ** 32):
        with pytest.raises(lcsm.LcsmError) as e:
            c.ctx.apply(layer, c.q, c.k, c.positions)
        assert e.value.code == lcsm.LCSM_EINVAL
    with pytest.raises(lcsm.LcsmError):
        c.ctx.apply(0, c.q, c.k, None)
    q, k = c.ctx.apply(0, c.q[:0], c.k[:0], c.positions[:0])
    assert q.shape == (0, 32) and k.shape == (0, 16)
    only = lcsm.Rot(16, 2, 0, dtype=torch.float32)
    with pytest.raises(ValueError):
        only.apply(0, c.q, c.k, c.positions)
    assert only.apply(0, c.q, None, c.positions)[1] is None
