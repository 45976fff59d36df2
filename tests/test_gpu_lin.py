"""Linear attention with decays (lcsm_lin.h) against the fp64 oracle on the GPU
(needs an MI355X).

Tolerances.  With A what the formula gives for the magnitudes of queries, keys,
values and states, an output is off by half an ulp of its type and by a share of
A: in fp32 and for the states the products that are left out (three of 2^-24) and
at most some three hundred roundings of 2^-24 in a chain (products of a chunk,
the states of up to forty chunks, exponents): 2e-5; where outputs have 16 bits
their scores and states are rounded to 2^-16 besides, twice."""
import ctypes

import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod, say
from oracle import lin as oracle

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SUMS = 2e-5
LOST = {"f32": 0.0, "bf16": 2.0 ** -15, "f16": 2.0 ** -15}


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=dev())


def close(got, want, room, what=""):
    """|got - want| <= room, not finite in the same places."""
    got = got.double().cpu().numpy()
    assert got.shape == want.shape
    if not got.size:
        return
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), what
    over = (np.abs(got - want) - room)[fine]
    assert over.max(initial=-1.0) <= 0.0, (what, float(over.max()), float(room[fine].max()))


class Layer:
    """Decays of M layers, the context and the oracle's states."""

    def __init__(self, H, G, K, V, dtype="f32", slots=4, max_tokens=1024, M=1, seed=0, decay=None, scale=0.25, **more):
        r = np.random.default_rng(seed)
        self.H, self.G, self.K, self.V, self.M, self.dtype, self.slots, self.rng, self.scale = H, G, K, V, M, dtype, slots, r, scale
        self.decay = (-np.exp2(-8 * r.random((M, G))) if decay is None else np.broadcast_to(np.asarray(decay), (M, G))).astype(np.float32)
        self.ctx = lcsm_mod().Lin(torch.from_numpy(self.decay.copy()).to(dev()), slots=slots, heads=H, keys=K, values=V, scale=scale,
                                  dtype=TYPES[dtype], max_tokens=max_tokens, **more)
        self.state = np.zeros((M, slots, G, K, V))
        self.size = np.zeros((M, slots, G, K, V))  # of the magnitudes

    def widths(self):
        return self.H * self.K, self.G * self.K, self.G * self.V

    def inputs(self, T, pad=0):
        """(q, k, v) in the layer's type on the GPU."""
        return [torch.from_numpy(self.rng.standard_normal((T, w + 2 * pad)).astype(np.float32)).to(TYPES[self.dtype]).to(
            dev())[:, pad:pad + w] for w in self.widths()]

    def set_states(self, layer=0):
        s = self.rng.standard_normal(self.state[layer].shape).astype(np.float32)
        self.ctx.state(layer).copy_(torch.from_numpy(s))
        self.state[layer], self.size[layer] = s, np.abs(s)

    def want(self, x, offs, layer=0, src=None, dst=None):
        """(y, room) of the rows that sequences have, zeros elsewhere; moves the oracle's states."""
        q, k, v = (a.double().cpu().numpy().reshape(len(a), n, -1) for a, n in zip(x, (self.H, self.G, self.G)))
        n = len(offs) - 1
        src, dst = (list(range(n)) if s is None else s for s in (src, dst))
        y, room, after = np.zeros((len(q), self.H, self.V)), np.zeros((len(q), self.H, self.V)), []
        for i in range(n):
            a, b = offs[i], offs[i + 1]
            old = [s[layer, src[i]] if 0 <= src[i] < self.slots else np.zeros(self.state.shape[2:]) for s in (self.state, self.size)]
            y[a:b], S = oracle.attend(q[a:b], k[a:b], v[a:b], self.decay[layer], np.float32(self.scale), old[0])
            big, Z = oracle.attend(*(np.abs(t[a:b]) for t in (q, k, v)), self.decay[layer], abs(self.scale), old[1])
            room[a:b] = ULP[self.dtype] * np.abs(y[a:b]) + (SUMS + LOST[self.dtype]) * big + (1e-38 if self.dtype != "f16" else 2.0 ** -25)
            after.append((S, Z))
        for i in range(n):
            if 0 <= dst[i] < self.slots:
                self.state[layer, dst[i]], self.size[layer, dst[i]] = after[i]
        return y.reshape(len(q), -1), room.reshape(len(q), -1)

    def check(self, y, want, layer=0):
        torch.cuda.synchronize()
        close(y, want[0], want[1], "outputs")
        close(self.ctx.state(layer), self.state[layer], SUMS * self.size[layer] + 1e-38, "states")


SHAPES = [(1, 1, 1, 1), (2, 2, 8, 8), (3, 1, 5, 7), (4, 2, 16, 33), (2, 2, 32, 32), (6, 3, 33, 31), (2, 1, 64, 130), (3, 3, 40, 72),
          (2, 2, 100, 96), (1, 1, 128, 128), (2, 1, 128, 260), (1, 1, 129, 64), (2, 2, 200, 20), (1, 1, 256, 128), (1, 1, 255, 257)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_prompts(shape, dtype):
    """Lengths around the borders of tiles and chunks, states taken up, begun and not kept."""
    lay = Layer(*shape, dtype=dtype, slots=9, seed=sum(shape))
    lens = [1, 17, 0, 31, 64, 65, 130, 33]
    offs = [0]
    for n in lens:
        offs.append(offs[-1] + n)
    say(f"[lin] {shape} {dtype} {lens}")
    lay.set_states()
    x = lay.inputs(offs[-1])
    # (a slot that is written is read by its own sequence only)
    src, dst = [0, -1, 2, 3, 4, -1, 6, 99], [0, 1, 8, 3, 4, -1, 6, 7]
    y = lay.ctx.prompt(0, *x, offsets=ints(offs), src=ints(src), dst=ints(dst))
    lay.check(y, lay.want(x, offs, src=src, dst=dst))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(2, 2, 16, 16), (3, 1, 40, 40), (2, 2, 64, 100), (1, 1, 128, 64), (2, 1, 160, 32)], ids=str)
def test_cut_prompts(shape, dtype):
    """Long calls, cut into segments: one sequence, several, in place and in a copy, the same bits every time."""
    lay = Layer(*shape, dtype=dtype, slots=4, max_tokens=1600, seed=sum(shape), decay=[-0.004, -0.3, -0.02][:shape[1]])
    lay.set_states()
    x = lay.inputs(1500)
    lay.check(lay.ctx.prompt(0, *x), lay.want(x, [0, 1500]))
    # (slot 1 is read by two and written by none)
    offs, src, dst = [0, 700, 700, 1420, 1500], [0, 1, -1, 1], [0, 2, 3, -1]
    before = lay.ctx.state(0).clone()
    got = []
    for _ in range(3):
        lay.ctx.state(0).copy_(before)
        got.append((lay.ctx.prompt(0, *x, offsets=ints(offs), src=ints(src), dst=ints(dst)).clone(), lay.ctx.state(0).clone()))
    lay.check(got[0][0], lay.want(x, offs, src=src, dst=dst))
    for y, s in got[1:]:
        assert torch.equal(y, got[0][0]) and torch.equal(s, got[0][1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_steps(shape, dtype):
    lay = Layer(*shape, dtype=dtype, slots=6, seed=sum(shape), max_tokens=0, M=2)
    lay.set_states(1)
    for src, dst in ((None, None), ([1, -1, 0], [1, 2, 4]), ([5, 5, 77], [-1, 3, -4])):
        n = 4 if src is None else 3
        x = lay.inputs(n)
        y = lay.ctx.step(1, *x, src=None if src is None else ints(src), dst=None if dst is None else ints(dst))
        lay.check(y, lay.want(x, list(range(n + 1)), layer=1, src=src, dst=dst), layer=1)
    assert not lay.ctx.state(0).any()


def test_many_steps_at_once():
    """As many sequences as take the form for large batches, of odd widths too."""
    for H, G, K, V, n in ((4, 4, 128, 128, 300), (6, 2, 40, 73, 600), (2, 2, 200, 36, 520)):
        lay = Layer(H, G, K, V, dtype="bf16", slots=n, max_tokens=0, seed=n)
        lay.set_states()
        x = lay.inputs(n)
        lay.check(lay.ctx.step(0, *x), lay.want(x, list(range(n + 1))))


@pytest.mark.parametrize("dtype", TYPES)
def test_many_short_prompts(dtype):
    lay = Layer(2, 1, 24, 24, dtype=dtype, slots=700, max_tokens=3000, seed=3)
    lens = lay.rng.integers(0, 8, 700)
    offs = [0] + np.cumsum(lens).tolist()
    lay.set_states()
    x = lay.inputs(offs[-1])
    lay.check(lay.ctx.prompt(0, *x, offsets=ints(offs)), lay.want(x, offs))


@pytest.mark.parametrize("dtype", TYPES)
def test_prompt_pieces_and_tokens_agree(dtype):
    """A prompt at once, in pieces, and token by token end in the same states and outputs, within what each may be off."""
    lay = Layer(4, 2, 48, 40, dtype=dtype, slots=3, seed=4)
    x = lay.inputs(150)
    want = lay.want(x, [0, 150])
    none = ints([-1])
    y0 = lay.ctx.prompt(0, *x, src=none, dst=ints([0]))
    pieces = []
    for a, b in ((0, 1), (1, 70), (70, 70), (70, 150)):
        pieces.append(lay.ctx.prompt(0, *(t[a:b] for t in x), src=none if a == 0 else ints([1]), dst=ints([1])))
    tokens = [lay.ctx.step(0, *(t[i:i + 1] for t in x), src=none if i == 0 else ints([2]), dst=ints([2])) for i in range(150)]
    torch.cuda.synchronize()
    for slot, y in enumerate((y0, torch.cat(pieces), torch.cat(tokens))):
        close(y, want[0], want[1], f"way {slot}")
        close(lay.ctx.state(0)[slot], lay.state[0, 0], SUMS * lay.size[0, 0], f"way {slot}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("decay", [0.0, -1e-7, -5.0, -60.0, -1e4, float("-inf"), 0.01])
def test_decays(decay, dtype):
    """From none at all to one that leaves nothing (and a growing one)."""
    lay = Layer(2, 2, 20, 20, dtype=dtype, slots=2, seed=5, decay=decay)
    lay.set_states()
    x = lay.inputs(300)
    with np.errstate(invalid="ignore"):
        want = lay.want(x, [0, 300])
    lay.check(lay.ctx.prompt(0, *x), want)
    x = lay.inputs(1)
    lay.check(lay.ctx.step(0, *x), lay.want(x, [0, 1]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(2, 2, 40, 72), (4, 2, 128, 64), (1, 1, 160, 40)], ids=str)
def test_values_that_are_not_finite(shape, dtype):
    """They reach what depends on them: no earlier token, no other sequence, head or value."""
    H, G, K, V = shape
    for which, at in (("v", 0), ("v", 37), ("v", 64 + 31), ("k", 50), ("q", 20), ("v2", 40)):
        lay = Layer(*shape, dtype=dtype, slots=2, seed=6)
        lay.set_states()
        x = lay.inputs(260)
        if which == "v2":  # two values of one token, one of them NaN
            x[2][at, 1], x[2][at, V - 1] = float("nan"), float("inf")
        else:
            x["qkv".index(which)][at, 2] = float("-inf")
        offs = [0, 130, 260]
        with np.errstate(invalid="ignore"):
            want = lay.want(x, offs)
        y = lay.ctx.prompt(0, *x, offsets=ints(offs))
        say(f"[lin] not finite: {which} {at} {shape} {dtype}")
        lay.check(y, want)
        assert np.isfinite(want[0][:at]).all() and np.isfinite(want[0][130:]).all()


def test_slices_of_one_projection():
    """Queries, keys and values side by side in one row, odd starts, outputs into a wider one; rows that no sequence has
    keep what they hold."""
    for dtype in TYPES:
        lay = Layer(4, 2, 24, 40, dtype=dtype, slots=3, seed=7)
        a, b, c = lay.widths()
        row = torch.randn((230, a + b + c + 9), device=dev()).to(TYPES[dtype])
        x = [row[:, 3:3 + a], row[:, 3 + a:3 + a + b], row[:, 5 + a + b:5 + a + b + c]]
        wide = torch.full((230, 4 * 40 + 6), 7.0, dtype=TYPES[dtype], device=dev())
        y = wide[:, 5:5 + 160]
        offs = [20, 100, 100, 200]
        lay.ctx.prompt(0, *x, y=y, offsets=ints(offs))
        want = lay.want(x, offs)
        torch.cuda.synchronize()
        close(y[20:200], want[0][20:200], want[1][20:200])
        assert bool((wide[:, :5] == 7).all()) and bool((wide[:, 165:] == 7).all())
        assert bool((wide[:20] == 7).all()) and bool((wide[200:] == 7).all())
        close(lay.ctx.state(0), lay.state[0], SUMS * lay.size[0] + 1e-38)
        lay.ctx.step(0, *(t[:3] for t in x), y=y[:3])
        want = lay.want([t[:3] for t in x], [0, 1, 2, 3])
        torch.cuda.synchronize()
        close(y[:3], *want)
        assert bool((wide[:3, :5] == 7).all()) and bool((wide[:3, 165:] == 7).all())


def test_rows_beyond_two_to_the_31_elements():
    lay = Layer(1, 1, 16, 16, dtype="bf16", slots=1, seed=8)
    x = lay.inputs(130)
    stride = 1 << 24
    far = torch.empty(129 * stride + 64, dtype=torch.bfloat16, device=dev())
    xs = [far[16 * i:].as_strided((130, 16), (stride, 1)) for i in range(4)]
    for a, b in zip(xs, x):
        a.copy_(b)
    lay.check(lay.ctx.prompt(0, *xs[:3], y=xs[3]), lay.want(x, [0, 130]))


def test_wrong_offsets_and_slots_stay_in_bounds():
    """Offsets that do not rise or leave the rows give wrong values; what lies around the rows keeps its."""
    lay = Layer(2, 2, 16, 16, dtype="f32", slots=4, max_tokens=700, seed=9)
    a, b, c = lay.widths()
    around = [torch.zeros((900, w), device=dev()) for w in (a, b, c, 32)]
    for t in around[:3]:
        t[100:800] = torch.randn_like(t[100:800])
    around[3].fill_(7.0)
    x, y = [t[100:800] for t in around[:3]], around[3][100:800]
    states = lay.ctx.state(0)
    for offs in ([0, 700, 0, 700, 700], [500, 20, 400, 100, 650], [-5, 2 ** 31 - 1, -2 ** 31, 300, 900], [700, 700, 0, 0, 0],
                 [0, 1, 699, 2, 2000]):
        lay.ctx.prompt(0, *x, y=y, offsets=ints(offs), src=ints([-7, 4, 2 ** 31 - 1, 0]), dst=ints([-2 ** 31, 1, 4, 2]))
        torch.cuda.synchronize()
        assert bool((around[3][:100] == 7).all()) and bool((around[3][800:] == 7).all())
        assert not states[3].any() and not states[0].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_segments_of_many_chunks(dtype):
    """Many states, so that a long prompt is cut in two or three pieces of tens of chunks, under all kinds of decays: what a
    piece adds to the state is summed over all of them at once."""
    G = 200
    lay = Layer(G, G, 8, 12, dtype=dtype, slots=2, max_tokens=3100, seed=12, decay=-np.exp2(-16 + 18 * np.arange(G) / G))
    lay.set_states()
    x = lay.inputs(3100)
    say(f"[lin] long segments {dtype}")
    lay.check(lay.ctx.prompt(0, *x), lay.want(x, [0, 3100]))


def test_two_graphs_of_one_context():
    """Two prompts' graphs share the context's workspace: replayed one after another, in either order, each is right."""
    stream = torch.cuda.Stream(dev())
    lay = Layer(4, 2, 64, 32, dtype="bf16", slots=2, seed=13, max_tokens=1500, stream=stream)
    xs = [lay.inputs(T) for T in (1500, 900)]
    src, nowhere = ints([-1]), ints([-1])
    wants = [lay.want(x, [0, len(x[0])], src=[-1], dst=[-1]) for x in xs]
    with torch.cuda.stream(stream):
        ys = [torch.empty((len(x[0]), 4 * 32), dtype=torch.bfloat16, device=dev()) for x in xs]
        torch.cuda.synchronize()
        graphs = []
        for x, y in zip(xs, ys):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=stream):
                lay.ctx.prompt(0, *x, y=y, src=src, dst=nowhere)
        for order in ((0, 1), (1, 0), (1, 1), (0, 1)):
            for y in ys:
                y.zero_()
            for i in order:
                graphs[i].replay()
            torch.cuda.synchronize()
            for i in set(order):
                close(ys[i], *wants[i])


@pytest.mark.parametrize("T", [60, 1500])
def test_another_stream_and_a_graph(T):
    stream = torch.cuda.Stream(dev())
    lay = Layer(2, 2, 32, 32, dtype="bf16", slots=2, seed=10, max_tokens=1500, stream=stream)
    x, x1 = lay.inputs(T), lay.inputs(2)
    y0 = lay.ctx.prompt(0, *x, src=ints([-1]))
    want = lay.want(x, [0, T], src=[-1])
    lay.check(y0, want)
    with torch.cuda.stream(stream):
        y, y1 = torch.empty_like(y0), torch.empty((2, 64), dtype=torch.bfloat16, device=dev())
        src, at = ints([-1]), ints([0, -1])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            lay.ctx.prompt(0, *x, y=y, src=src)
            lay.ctx.step(0, *x1, y=y1, src=at, dst=at)
        first = lay.want(x, [0, T], src=[-1]), lay.want(x1, [0, 1, 2], src=[0, -1], dst=[0, -1])
        for _ in range(3):
            y.fill_(float("nan"))
            y1.fill_(float("nan"))
            lay.ctx.reset()
            lay.ctx.step(0, *x1)
            lay.ctx.state(0)[1].zero_()
            g.replay()
            torch.cuda.synchronize()
            close(y, *first[0])
            lay.check(y1, first[1])


def test_reset_and_layers():
    lay = Layer(2, 2, 16, 16, slots=2, M=3, seed=11)
    x = lay.inputs(70)
    for m in (0, 2):
        lay.check(lay.ctx.prompt(m, *x), lay.want(x, [0, 70], layer=m), layer=m)
    assert not lay.ctx.state(1).any()
    lay.ctx.reset()
    torch.cuda.synchronize()
    assert not any(lay.ctx.state(m).any() for m in range(3))


def test_refusals():
    lcsm = lcsm_mod()
    lib = lcsm.raw()
    d = torch.zeros((1, 2), device=dev())
    good = dict(slots=2, heads=4, keys=16, values=8)
    for k, v in (("slots", 0), ("slots", 32769), ("heads", 3), ("heads", 0), ("keys", 0), ("keys", 257), ("values", 0), ("values", 4097),
                 ("max_tokens", -1), ("max_tokens", (1 << 26) + 1), ("scale", float("inf"))):
        with pytest.raises(lcsm.LcsmError):
            lcsm.Lin(d, **{**good, k: v})
    for k in ("slots", "heads", "keys", "values", "max_tokens"):
        with pytest.raises(ValueError):
            lcsm.Lin(d, **{**good, "max_tokens": 8, k: {**good, "max_tokens": 8}[k] + 2 ** 32})
    for bad in (d.double(), d.cpu(), d[0]):
        with pytest.raises(ValueError):
            lcsm.Lin(bad, **good)
    lay = Layer(4, 2, 16, 8, slots=2, max_tokens=10, seed=12)
    q, k, v = lay.inputs(2)
    for more in (dict(q=q[:, :63]), dict(k=k.double()), dict(v=v[:1]), dict(q=q.cpu()), dict(y=q), dict(src=ints([0])), dict(
            dst=torch.zeros(2, dtype=torch.int64, device=dev())), dict(q=q.t().contiguous().t())):
        kw = dict(q=q, k=k, v=v)
        kw.update(more)
        with pytest.raises(ValueError):
            lay.ctx.step(0, **kw)
    big = lay.inputs(11)
    calls = [lambda: lay.ctx.step(1, q, k, v), lambda: lay.ctx.step(-1, q, k, v), lambda: lay.ctx.step(2 ** 32, q, k, v),
             lambda: lay.ctx.step(0, *(t[:3] for t in big)), lambda: lay.ctx.prompt(0, *big),
             lambda: lay.ctx.prompt(0, q, k, v, offsets=ints([0, 1, 1, 2])), lambda: lay.ctx.prompt(2 ** 32, q, k, v)]
    for call in calls:
        with pytest.raises(lcsm.LcsmError) as e:
            call()
        assert e.value.code == lcsm.LCSM_EINVAL
    p = q.data_ptr()
    io = lcsm.LinIo(p, p, p, p, 63, 32, 16, 32)
    assert lib.lcsm_lin_step_layer(lay.ctx._ctx, 0, 2, ctypes.byref(io)) == lcsm.LCSM_EINVAL
    assert lib.lcsm_lin_step_layer(lay.ctx._ctx, 0, 2, None) == lcsm.LCSM_EINVAL
    assert lib.lcsm_lin_prompt_layer(lay.ctx._ctx, 0, 2, 2, None, ctypes.byref(io)) == lcsm.LCSM_EINVAL
    assert lay.ctx.step(0, q[:0], k[:0], v[:0]).shape == (0, 32)
    assert lay.ctx.prompt(0, q[:0], k[:0], v[:0], src=ints([-1])).shape == (0, 32)
    lay.check(lay.ctx.step(0, q, k, v), lay.want((q, k, v), [0, 1, 2]))  # no refusal faults the context
