"""The selective state space mixer (lcsm_ssm.h) against the fp64 oracle on the
GPU (needs an MI355X).

Tolerances, as a share of the largest value: an output is rounded once to its
type (half an ulp: 2^-24, 2^-8, 2^-11), and what is summed in fp32 before that
(the states too) may be off by 2e-5: some hundred roundings of 2^-24 along the
decays and over the states, or products of values held to 2^-17."""
import ctypes

import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod, say
from oracle import ssm as oracle

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SUMS = 2e-5
TOL = {"f32": SUMS, "bf16": SUMS + 2.0 ** -8, "f16": SUMS + 2.0 ** -11}


def close(got, want, tol, what=""):
    """|got - want| <= tol max|want|, not finite in the same places."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape
    if not got.size:
        return
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), what
    if fine.any():
        err = np.abs(got[fine] - want[fine]).max() / max(np.abs(want[fine]).max(), 1e-30)
        assert err <= tol, (what, err, tol)


class Layer:
    """Weights of M layers, the context and the oracle's states."""

    def __init__(self, H, P, N, G, W, dtype="f32", slots=4, max_tokens=1024, M=1, seed=0, skip=True, decay=16.0, **more):
        r = np.random.default_rng(seed)
        self.H, self.P, self.N, self.G, self.W, self.M = H, P, N, G, W, M
        self.D, self.C, self.dtype, self.slots, self.rng = H * P, H * P + 2 * G * N, dtype, slots, r
        f = lambda *s: r.standard_normal(s).astype(np.float32)  # noqa: E731
        self.conv_w, self.conv_b = f(M, self.C, W) / np.float32(np.sqrt(W)), f(M, self.C) * np.float32(0.1)
        self.A = -(1 + (decay - 1) * r.random((M, H))).astype(np.float32)
        self.skip = f(M, H) if skip else np.zeros((M, H), np.float32)
        self.dt_bias = np.log(np.expm1(np.exp(r.uniform(np.log(1e-3), np.log(1e-1), (M, H))))).astype(np.float32)
        up = lambda v: torch.from_numpy(v).to(dev())  # noqa: E731
        self.ctx = lcsm_mod().Ssm(up(self.conv_w), up(self.A), slots=slots, groups=G, states=N, conv_bias=up(self.conv_b),
                                  skip=up(self.skip) if skip else None, dt_bias=up(self.dt_bias), dtype=TYPES[dtype],
                                  max_tokens=max_tokens, **more)
        self.state = np.zeros((M, slots, H, P, N))
        self.window = np.zeros((M, slots, W - 1, self.C))

    def rows(self, T, width, scale=1.0):
        """Values in the layer's type, on the GPU and as the oracle takes them."""
        t = torch.from_numpy((self.rng.standard_normal((T, width)) * scale).astype(np.float32)).to(TYPES[self.dtype])
        return t.to(dev()), t.double().numpy()

    def inputs(self, T, gate=True):
        a, b, c = self.rows(T, self.C), self.rows(T, self.H, 0.5), self.rows(T, self.D)
        return (a[0], b[0], c[0] if gate else None), (a[1], b[1], c[1] if gate else None)

    def want(self, x, offsets, src=None, dst=None, m=0):
        """The oracle's outputs for sequences at these offsets; its states move on."""
        y = np.zeros((x[0].shape[0], self.D))
        before_s, before_w = self.state[m].copy(), self.window[m].copy()
        for i in range(len(offsets) - 1):
            s, d = (i if src is None else src[i]), (i if dst is None else dst[i])
            a, b = offsets[i], offsets[i + 1]
            s0 = before_s[s] if s >= 0 else np.zeros_like(before_s[0])
            w0 = before_w[s] if s >= 0 else np.zeros_like(before_w[0])
            y[a:b], s1, w1 = oracle.scan(x[0][a:b], x[1][a:b], None if x[2] is None else x[2][a:b], self.conv_w[m],
                                         self.conv_b[m], self.A[m], self.skip[m], self.dt_bias[m], self.G, self.N, s0, w0)
            if d >= 0:
                self.state[m, d], self.window[m, d] = s1, w1
        return y

    def check(self, y, want, what="", m=0):
        torch.cuda.synchronize()
        close(y.double().cpu().numpy(), want, TOL[self.dtype], what + " y")
        close(self.ctx.state(m).double().cpu().numpy(), self.state[m], SUMS, what + " state")
        got = self.ctx.window(m).double().cpu().numpy()
        assert np.array_equal(got, self.window[m], equal_nan=True), what + " window"


def ints(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32, device=dev())


# (H, P, N, G, W): ordinary heads, every tail (channels, states, groups), the largest states, one of everything
SHAPES = [(4, 64, 128, 1, 4), (6, 48, 40, 3, 3), (3, 41, 23, 3, 2), (2, 16, 16, 1, 4), (2, 7, 256, 1, 4), (1, 1, 1, 1, 1),
          (2, 130, 33, 2, 2), (8, 32, 64, 2, 4), (5, 33, 200, 1, 3)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_prompts_and_steps_follow_the_oracle(shape, dtype):
    """Ragged prompts with an empty and a one-token sequence, then single
    tokens, then more prompts that go on from there."""
    lay = Layer(*shape, dtype=dtype, slots=6, seed=sum(shape))
    lens = [65, 0, 1, 130, 64, 3]
    offs = np.concatenate([[0], np.cumsum(lens)]).tolist()
    say(f"[ssm] {shape} {dtype} prompts of {lens}")
    x, xr = lay.inputs(offs[-1])
    y = lay.ctx.prompt(0, x[0], x[1], z=x[2], offsets=ints(offs))
    lay.check(y, lay.want(xr, offs), "first prompts")
    for k in range(2):
        x, xr = lay.inputs(6, gate=k == 0)
        y = lay.ctx.step(0, x[0], x[1], z=x[2])
        lay.check(y, lay.want(xr, list(range(7))), f"step {k}")
    lens = [2, 5, 190, 0, 1, 63]
    offs = np.concatenate([[0], np.cumsum(lens)]).tolist()
    x, xr = lay.inputs(offs[-1], gate=False)
    y = lay.ctx.prompt(0, x[0], x[1], offsets=ints(offs))
    lay.check(y, lay.want(xr, offs), "more prompts")


@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 127, 128, 129, 1000, 4097])
def test_lengths_around_the_pieces(T):
    lay = Layer(3, 64, 64, 1, 4, slots=1, max_tokens=T, seed=T)
    x, xr = lay.inputs(T)
    say(f"[ssm] one prompt of {T}")
    lay.check(lay.ctx.prompt(0, x[0], x[1], z=x[2]), lay.want(xr, [0, T]))


@pytest.mark.parametrize("dtype", TYPES)
def test_one_long_prompt_of_one_head(dtype):
    """Few sequences and heads: the work is split along the tokens."""
    lay = Layer(1, 64, 128, 1, 4, dtype=dtype, slots=2, max_tokens=9000, seed=3, decay=1.5)
    x, xr = lay.inputs(9000)
    y = lay.ctx.prompt(0, x[0], x[1], z=x[2], offsets=ints([0, 8200, 9000]))
    lay.check(y, lay.want(xr, [0, 8200, 9000]))


def test_slots_are_read_and_written_as_named():
    """Copies, new sequences, ones that are not kept, values out of range, in
    prompts and steps; slots that are not named keep what they hold."""
    lay = Layer(2, 16, 24, 2, 4, slots=5, seed=9)
    x, xr = lay.inputs(50)
    offs = [0, 10, 20, 30, 40, 50]
    lay.check(lay.ctx.prompt(0, x[0], x[1], offsets=ints(offs)), lay.want((xr[0], xr[1], None), offs), "fill")
    for k, (src, dst) in enumerate([([3, -1, 0], [1, 2, 0]), ([0, 1, 2], [-1, 4, 2]), ([4, 99, -7], [4, 99, 1])]):
        seen = [s if 0 <= s < 5 else -1 for s in src], [d if 0 <= d < 5 else -1 for d in dst]
        x, xr = lay.inputs(3)
        y = lay.ctx.step(0, x[0], x[1], z=x[2], src=ints(src), dst=ints(dst))
        lay.check(y, lay.want(xr, [0, 1, 2, 3], *seen), f"step {k}")
        offs = [0, 70, 70, 75]
        x, xr = lay.inputs(75)
        y = lay.ctx.prompt(0, x[0], x[1], z=x[2], offsets=ints(offs), src=ints(src), dst=ints(dst))
        lay.check(y, lay.want(xr, offs, *seen), f"prompt {k}")


def test_a_prompt_in_pieces_is_the_prompt():
    """One prompt, the same in two pieces and the same token by token."""
    T, lay = 150, Layer(2, 32, 16, 1, 4, slots=3, seed=4)
    x, xr = lay.inputs(T)
    want = lay.want(xr, [0, T], dst=[0])
    y = lay.ctx.prompt(0, x[0], x[1], z=x[2])
    cut = [t[:77] for t in x], [t[77:] for t in x]
    for part in cut:
        one = lay.ctx.prompt(0, part[0], part[1], z=part[2], src=ints([1]), dst=ints([1]))
    for t in range(T):
        last = lay.ctx.step(0, x[0][t:t + 1], x[1][t:t + 1], z=x[2][t:t + 1], src=ints([2]), dst=ints([2]))
    torch.cuda.synchronize()
    close(y.cpu().numpy(), want, SUMS)
    close(one[-1:].cpu().numpy(), want[-1:], SUMS)
    close(last.cpu().numpy(), want[-1:], SUMS)
    s = lay.ctx.state(0).double().cpu().numpy()
    for k in range(3):
        close(s[k], lay.state[0, 0], SUMS)


@pytest.mark.parametrize("shape", [(1, 64, 64, 1, 4), (8, 64, 128, 1, 4), (40, 64, 16, 1, 4), (3, 20, 9, 3, 3)], ids=str)
def test_long_prompts_continued_in_place(shape):
    """Sequences long enough to be cut, each read from and written to its own
    slot: whoever finishes first must not change what the others begin from."""
    lay = Layer(*shape, slots=3, max_tokens=5000, seed=15, decay=1.1)
    for lens in ([2000, 1, 300], [3000, 700, 0], [640, 64, 4100]):
        offs = [0, lens[0], lens[0] + lens[1], sum(lens)]
        x, xr = lay.inputs(offs[-1], gate=False)
        lay.check(lay.ctx.prompt(0, x[0], x[1], offsets=ints(offs)), lay.want(xr, offs), str(lens))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_one_wide_projection(dtype):
    """xbc, z and dt as slices of the rows of one projection (strides, starts
    that are not aligned), the outputs written over the gate."""
    lay = Layer(3, 16, 12, 1, 4, dtype=dtype, slots=2, seed=5)
    T, wide = 97, lay.D + lay.C + lay.H + 3
    t, tr = lay.rows(T, wide)
    z, zr = t[:, 1:1 + lay.D], tr[:, 1:1 + lay.D]
    xbc, xr = t[:, 1 + lay.D:1 + lay.D + lay.C], tr[:, 1 + lay.D:1 + lay.D + lay.C]
    dt, dr = t[:, 1 + lay.D + lay.C:1 + lay.D + lay.C + lay.H], tr[:, 1 + lay.D + lay.C:1 + lay.D + lay.C + lay.H]
    want = lay.want((xr, dr, zr), [0, 40, 97])
    before = t.clone()
    y = lay.ctx.prompt(0, xbc, dt, z=z, y=z, offsets=ints([0, 40, 97]))
    lay.check(y, want, "prompt")
    before[:, 1:1 + lay.D] = y
    assert torch.equal(before, t)
    t, tr = lay.rows(2, wide)
    args = [(v[:, 1:1 + lay.D], v[:, 1 + lay.D:1 + lay.D + lay.C], v[:, 1 + lay.D + lay.C:1 + lay.D + lay.C + lay.H])
            for v in (t, tr)]
    want = lay.want((args[1][1], args[1][2], args[1][0]), [0, 1, 2])
    lay.check(lay.ctx.step(0, args[0][1], args[0][2], z=args[0][0], y=args[0][0]), want, "step")


@pytest.mark.parametrize("shape", [(2, 64, 128, 1, 4), (2, 7, 12, 2, 3)], ids=str)
@pytest.mark.parametrize("what", ["x", "B", "C", "dt", "z"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite_stay_where_they_act(shape, what, value):
    """A value in one token of one sequence: everything that does not depend on
    it is what it is without it."""
    H, P, N, G, W = shape
    T, at = 150, 97
    plain = Layer(*shape, slots=2, seed=6)
    x, _ = plain.inputs(2 * T)
    offs = ints([0, T, 2 * T])
    y0 = plain.ctx.prompt(0, x[0], x[1], z=x[2], offsets=offs).clone()
    s0 = plain.ctx.state(0).clone()
    lay = Layer(*shape, slots=2, seed=6)
    t = {"x": x[0], "B": x[0], "C": x[0], "dt": x[1], "z": x[2]}[what]
    col = {"x": 3, "B": H * P + 2, "C": H * P + G * N + 2, "dt": 1, "z": 3}[what]
    t[at, col] = value
    y1 = lay.ctx.prompt(0, x[0], x[1], z=x[2], offsets=offs)
    s1 = lay.ctx.state(0)
    torch.cuda.synchronize()
    same = lambda a, b: torch.allclose(a, b, rtol=0, atol=float(SUMS * b.abs().max()))  # noqa: E731
    assert same(y1[:at], y0[:at]) and same(y1[T:], y0[T:]) and same(s1[1], s0[1])
    if what == "z":
        assert same(s1[0], s0[0])
        rest = torch.ones_like(y1[:T], dtype=torch.bool)
        rest[at, col] = False
        assert same(y1[:T][rest], y0[:T][rest])
    if what == "x":
        rest = torch.arange(H * P, device=dev()) != col
        assert same(y1[:T, rest], y0[:T, rest])
        if value == value and value < 0:
            assert not torch.isfinite(y1[at, col])  # silu(-inf) is not a number
    if what == "dt":
        head = slice(0, P)  # the other head
        assert same(y1[:T, head], y0[:T, head]) and same(s1[0, 0], s0[0, 0])
        if value > 0:
            assert not torch.isfinite(y1[at:T, P:2 * P]).any() and not torch.isfinite(s1[0, 1]).any()
    if what == "C":
        assert same(s1[0], s0[0])
        if value > 0:
            last = min(at + W, T)
            assert same(y1[last:T], y0[last:T])
    if value != value and what in ("x", "B"):
        assert not torch.isfinite(s1[0]).all()


def test_large_values_and_strong_decays():
    """Steps of 30 and decays that leave nothing, inputs of 1e15: no overflow
    where the definition has none."""
    lay = Layer(2, 24, 16, 1, 4, slots=1, seed=8)
    x, xr = lay.inputs(200)
    x[0][:, :lay.D] *= 1e15
    xr[0][:, :lay.D] = x[0][:, :lay.D].double().cpu().numpy()
    x[1][50:60] = 30.0
    xr[1][50:60] = 30.0
    y = lay.ctx.prompt(0, x[0], x[1], z=x[2])
    want = lay.want(xr, [0, 200])
    lay.check(y, want)
    # per row: a row's error is measured by the row's own size
    for t in range(0, 200, 7):
        close(y[t].double().cpu().numpy(), want[t], 10 * SUMS, f"row {t}")


def test_layers_streams_reset_and_bad_offsets():
    stream = torch.cuda.Stream(dev())
    lay = Layer(2, 16, 16, 1, 4, M=3, slots=2, seed=11, stream=stream)
    for m in (2, 0):
        x, xr = lay.inputs(30)
        y = lay.ctx.prompt(m, x[0], x[1], z=x[2], offsets=ints([0, 12, 30]))
        lay.check(y, lay.want(xr, [0, 12, 30], m=m), f"layer {m}", m=m)
    assert float(lay.ctx.state(1).abs().max()) == 0.0
    # offsets out of range or falling: nothing outside the rows is touched
    guard = torch.full((40, lay.D), 7.0, device=dev())
    x, _ = lay.inputs(30)
    lay.ctx.prompt(0, x[0], x[1], y=guard[5:35], offsets=ints([-5, 1000, 3]))
    torch.cuda.synchronize()
    assert bool((guard[:5] == 7.0).all()) and bool((guard[35:] == 7.0).all())
    lay.ctx.reset()
    torch.cuda.synchronize()
    assert all(float(lay.ctx.state(m).abs().max()) == 0.0 and float(lay.ctx.window(m).abs().max()) == 0.0 for m in range(3))


def test_rows_beyond_two_to_the_31_elements():
    """A stride that puts the last rows past 2^31 elements."""
    lay = Layer(1, 8, 8, 1, 4, dtype="bf16", slots=1, max_tokens=130, seed=12)
    T, stride = 130, 1 << 24
    big = torch.empty((T - 1) * stride + 64, dtype=torch.bfloat16, device=dev())
    x, xr = lay.inputs(T)
    wide = big.as_strided((T, lay.C), (stride, 1))
    wide.copy_(x[0])
    lay.check(lay.ctx.prompt(0, wide, x[1], z=x[2]), lay.want(xr, [0, T]))


def test_a_recorded_generation_replays():
    """A prompt and steps in one graph, replayed with other work in between."""
    stream = torch.cuda.Stream(dev())
    lay = Layer(2, 16, 24, 1, 4, slots=2, seed=13, stream=stream)
    x, _ = lay.inputs(80)
    ys = torch.empty((80, lay.D), device=dev())
    fresh, zero = ints([-1]), ints([0])

    def generation():
        lay.ctx.prompt(0, x[0][:70], x[1][:70], z=x[2][:70], y=ys[:70], src=fresh, dst=zero)
        for t in range(70, 80):
            lay.ctx.step(0, x[0][t:t + 1], x[1][t:t + 1], z=x[2][t:t + 1], y=ys[t:t + 1], src=zero, dst=zero)

    with torch.cuda.stream(stream):
        generation()
        torch.cuda.synchronize()
        eager, state = ys.clone(), lay.ctx.state(0).clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            generation()
        for k in range(3):
            ys.fill_(float("nan"))
            lay.ctx.state(0).fill_(5.0)
            x2, _ = lay.inputs(3)
            lay.ctx.step(0, x2[0][:1], x2[1][:1], src=ints([1]), dst=ints([1]))
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(ys, eager) and torch.equal(lay.ctx.state(0)[0], state[0])


def test_repeated_calls_give_the_same_bits():
    lay = Layer(4, 64, 128, 1, 4, dtype="bf16", slots=2, max_tokens=3000, seed=14)
    x, _ = lay.inputs(3000)
    got = [lay.ctx.prompt(0, x[0], x[1], z=x[2], src=ints([-1]), dst=ints([1])).clone() for _ in range(3)]
    s = [lay.ctx.step(0, x[0][:2], x[1][:2], src=ints([1, 1]), dst=ints([-1, -1])).clone() for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(got[0], g) for g in got) and all(torch.equal(s[0], g) for g in s)


def test_a_library_workspace_and_raw_errors():
    """The C entry points without the binding: the library's own workspace,
    every refusal before any work."""
    lcsm = lcsm_mod()
    lib = lcsm.raw()
    shape = lcsm.SsmShape(1, 2, 2, 4, 4, 1, 4, 0, 8)
    w, A = torch.randn((1, 16, 4), device=dev()), -torch.ones((1, 2), device=dev())
    ctx = ctypes.c_void_p()
    assert lib.lcsm_ssm_init(ctypes.byref(ctx), ctypes.byref(shape), w.data_ptr(), None, A.data_ptr(), None, None,
                             torch.cuda.current_stream().cuda_stream, None, 0) == 0
    x, dt, y = (torch.randn((8, n), device=dev()) for n in (16, 2, 8))
    io = lcsm.SsmIo(x.data_ptr(), dt.data_ptr(), None, y.data_ptr(), 16, 2, 0, 8, None, None)
    ref = ctypes.byref(io)
    assert lib.lcsm_ssm_prompt_layer(ctx, 0, 8, 1, None, ref) == 0
    assert lib.lcsm_ssm_step_layer(ctx, 0, 2, ref) == 0
    assert lib.lcsm_ssm_step_layer(ctx, 0, 0, ref) == 0
    bad = [lib.lcsm_ssm_step_layer(ctx, 1, 1, ref), lib.lcsm_ssm_step_layer(ctx, -1, 1, ref),
           lib.lcsm_ssm_step_layer(ctx, 0, 3, ref), lib.lcsm_ssm_step_layer(ctx, 0, -1, ref),
           lib.lcsm_ssm_step_layer(ctx, 0, 1, None), lib.lcsm_ssm_step_layer(None, 0, 1, ref),
           lib.lcsm_ssm_prompt_layer(ctx, 0, 9, 1, None, ref), lib.lcsm_ssm_prompt_layer(ctx, 0, -1, 1, None, ref),
           lib.lcsm_ssm_prompt_layer(ctx, 0, 8, 2, None, ref)]
    assert bad == [lcsm.LCSM_EINVAL] * len(bad)
    assert b"offsets" in lib.lcsm_ssm_last_error(ctx)
    for k, v in (("xbc", None), ("dt", None), ("y", None), ("xbc_stride", 15), ("dt_stride", 1), ("y_stride", 7)):
        o = lcsm.SsmIo(x.data_ptr(), dt.data_ptr(), None, y.data_ptr(), 16, 2, 0, 8, None, None)
        setattr(o, k, v)
        assert lib.lcsm_ssm_step_layer(ctx, 0, 1, ctypes.byref(o)) == lcsm.LCSM_EINVAL, k
    torch.cuda.synchronize()
    assert bool(torch.isfinite(y).all())
    lib.lcsm_ssm_destroy(ctx)
    small = torch.empty(256, dtype=torch.uint8, device=dev())
    assert lib.lcsm_ssm_init(ctypes.byref(ctx), ctypes.byref(shape), w.data_ptr(), None, A.data_ptr(), None, None,
                             None, small.data_ptr(), 256) == lcsm.LCSM_ENOMEM
    assert not ctx.value


def test_the_binding_refuses():
    lay = Layer(2, 4, 4, 1, 4, slots=2, max_tokens=8, seed=1)
    x, _ = lay.inputs(2)
    bad = [dict(xbc=x[0][:, :-1]), dict(xbc=x[0].double()), dict(xbc=x[0].cpu()), dict(dt=x[1].bfloat16()),
           dict(z=x[2][:1]), dict(y=x[0]), dict(src=torch.zeros(2, dtype=torch.int64, device=dev())),
           dict(dst=torch.zeros(1, dtype=torch.int32, device=dev())), dict(xbc=x[0].t().contiguous().t())]
    for b in bad:
        args = dict(xbc=x[0], dt=x[1], z=x[2])
        args.update(b)
        with pytest.raises(ValueError):
            lay.ctx.step(0, **args)
    with pytest.raises(lcsm_mod().LcsmError):
        lay.ctx.step(1, x[0], x[1])
    x, _ = lay.inputs(9)
    with pytest.raises(lcsm_mod().LcsmError):
        lay.ctx.prompt(0, x[0], x[1])
    with pytest.raises(lcsm_mod().LcsmError):
        lay.ctx.prompt(0, x[0][:0].expand(0, lay.C), x[1][:0], offsets=ints([0, 0, 0, 0]))
