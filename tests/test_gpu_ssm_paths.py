"""The state space mixer's ways through a call that depend on how many sequences
and heads there are, or how long they are (needs an MI355X): single tokens of many
sequences, prompts of so many sequences that none is cut, and values that are not
finite position by position and in single tokens.

`each` measures every value by itself.  A state: against the largest of its head,
2e-6 (a term goes through some ten fp32 roundings in convolution, SiLU, step and
decay, and the three parts of a product leave 2^-24 of a factor: 30 x 2^-24 where
terms cancel to a third).  An output: against the magnitude of what it is summed
from, taken through the recurrence (`magnitudes`), beside its own rounding (2^-24,
2^-8, 2^-11 of it, or half of the type's least value).  x is good to 8 x 2^-24 of its convolution's terms, B and C, which are
taken as they come out of theirs, to twice that on the average over the states; all
three together, and a dozen roundings of step, decay and gate, are below 64 x 2^-24
= 2^-18."""
import numpy as np
import pytest
import torch

from gpu_harness import dev
from oracle import ssm as oracle
from test_gpu_ssm import TYPES, Layer, ints

pytestmark = pytest.mark.gpu

ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}  # half of what the least values are apart
STATES, OUTPUTS = 2e-6, 2.0 ** -18


def magnitudes(lay, x, offsets, state, window):
    """What the outputs [T, D] are summed from, without signs: |C| |S| and skip x, where S adds up |x| |B| and the states
    before, and x stands for the terms of its convolution."""
    H, P, N, G, D = lay.H, lay.P, lay.N, lay.G, lay.D
    w, b = np.abs(lay.conv_w[0]).astype(np.float64), np.abs(lay.conv_b[0])
    out, group = np.zeros((x[0].shape[0], D)), np.arange(H) // (H // G)
    for i in range(len(offsets) - 1):
        S, rows = np.abs(state[i]), np.concatenate([window[i], x[0][offsets[i]:offsets[i + 1]]])
        for t in range(offsets[i], offsets[i + 1]):
            near = rows[t - offsets[i]:t - offsets[i] + lay.W]
            xs = (w * np.abs(near.T)).sum(1)[:D] + b[:D]
            u = np.abs(oracle.silu((lay.conv_w[0] * near.T).sum(1) + lay.conv_b[0]))
            s = np.logaddexp(0.0, x[1][t] + lay.dt_bias[0])
            B, C = u[D:D + G * N].reshape(G, N)[group], u[D + G * N:].reshape(G, N)[group]
            S = np.exp(s * lay.A[0])[:, None, None] * S + (s[:, None] * xs.reshape(H, P))[:, :, None] * B[:, None]
            out[t] = ((S * C[:, None]).sum(-1) + np.abs(lay.skip[0])[:, None] * xs.reshape(H, P)).reshape(D)
    return out if x[2] is None else out * np.abs(oracle.silu(x[2]))


def each(lay, call, x, offsets, src=None, dst=None, what=""):
    """call() is the layer's pass over x; sequence i is rows offsets[i] .. offsets[i + 1]."""
    n = len(offsets) - 1
    slots = list(range(n)) if src is None else src
    before = [(lay.state[0][s], lay.window[0][s]) if s >= 0 else (0 * lay.state[0][0], 0 * lay.window[0][0]) for s in slots]
    most = magnitudes(lay, x, offsets, [v[0] for v in before], [v[1] for v in before])
    want = lay.want(x, offsets, src, dst)
    y = call().double().cpu().numpy()
    err = np.abs(y - want) - np.maximum(ULP[lay.dtype] * np.abs(want), LEAST[lay.dtype])
    assert (err <= OUTPUTS * most).all(), (what, "y", (err / most).max())
    got = lay.ctx.state(0).double().cpu().numpy()
    err, most = np.abs(got - lay.state[0]).max((-1, -2)), np.abs(lay.state[0]).max((-1, -2))
    assert (err <= STATES * most).all(), (what, "state", (err / most).max())
    assert np.array_equal(lay.ctx.window(0).double().cpu().numpy(), lay.window[0]), (what, "window")


def seed_states(lay):
    """Every slot with a state and a window of its own."""
    s = lay.rng.standard_normal(lay.state[0].shape).astype(np.float32)
    w = torch.from_numpy(lay.rng.standard_normal(lay.window[0].shape).astype(np.float32)).to(TYPES[lay.dtype])
    lay.state[0], lay.window[0] = s, w.double().numpy()
    lay.ctx.state(0).copy_(torch.from_numpy(s))
    lay.ctx.window(0).copy_(w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(18, 41, 10, 3, 4), (18, 41, 24, 6, 4), (16, 64, 32, 1, 3), (9, 72, 40, 9, 4), (16, 64, 64, 2, 2),
                                   (16, 50, 100, 4, 4), (17, 64, 128, 1, 4), (16, 33, 200, 8, 4), (8, 130, 256, 1, 4)], ids=str)
def test_tokens_of_many_sequences(shape, dtype):
    """n H ceil(P / 64) >= 1024: 64 channels a workgroup.  In place, then slots moved about."""
    n = 66
    assert n * shape[0] * -(-shape[1] // 64) >= 1024
    lay = Layer(*shape, dtype=dtype, slots=n + 9, max_tokens=0, seed=sum(shape))
    seed_states(lay)
    x, xr = lay.inputs(n)
    each(lay, lambda: lay.ctx.step(0, x[0], x[1], z=x[2]), xr, list(range(n + 1)), what="in place")
    slots = lay.rng.permutation(n + 9).tolist()
    src = slots[:n]
    dst = slots[9:n] + slots[n:n + 9]  # (a slot that is written to is read by nobody else of the call)
    dst = [d if d not in src or d == src[i] else -1 for i, d in enumerate(dst)]
    dst = [src[i] if d == -1 and i % 2 else d for i, d in enumerate(dst)]
    src = [-1 if i % 11 == 5 and dst[i] != src[i] else s for i, s in enumerate(src)]
    x, xr = lay.inputs(n, gate=False)
    each(lay, lambda: lay.ctx.step(0, x[0], x[1], src=ints(src), dst=ints(dst)), xr, list(range(n + 1)), src, dst, "moved")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(64, 32, 70, 1, 4), (64, 32, 16, 4, 3), (32, 64, 40, 32, 4), (16, 33, 200, 2, 2)], ids=str)
def test_prompts_of_many_sequences_are_not_cut(shape, dtype):
    """More sequences than there is room for workgroups: each goes through in one piece, continued in its own slot."""
    H, P, N, G, W = shape
    n = 130
    lay = Layer(*shape, dtype=dtype, slots=n, seed=sum(shape), decay=6.0)
    items = H // G * -(-P // 32)
    waves = min(items, 8 if 64 < N <= 128 else 4)
    assert (512 if N <= 64 else 256) // (G * -(-items // waves)) <= n
    seed_states(lay)
    lens = lay.rng.integers(0, 4, n)
    lens[[0, 63, 64, 65, n - 1]] = [65, 0, 70, 1, 130]
    for part in range(2):
        offs = np.concatenate([[0], np.cumsum(lens)]).tolist()
        assert 192 < offs[-1] <= 1024
        x, xr = lay.inputs(offs[-1], gate=part == 0)
        each(lay, lambda: lay.ctx.prompt(0, x[0], x[1], z=x[2], offsets=ints(offs)), xr, offs, what=f"part {part}")
        lens = np.roll(lens, 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(4, 64, 128, 1, 4), (6, 48, 40, 3, 3), (3, 40, 16, 1, 4), (2, 33, 200, 1, 4)], ids=str)
def test_every_head_of_a_long_prompt(shape, dtype):
    """Two sequences that are cut, from states of their own; decays that forget within 50 tokens and ones that hardly do."""
    lay = Layer(*shape, dtype=dtype, slots=2, max_tokens=1300, seed=sum(shape))
    seed_states(lay)
    x, xr = lay.inputs(1300)
    offs = [0, 1003, 1300]
    each(lay, lambda: lay.ctx.prompt(0, x[0], x[1], z=x[2], offsets=ints(offs)), xr, offs)


@pytest.mark.parametrize("shape", [(2, 64, 128, 1, 4), (2, 7, 12, 2, 3), (2, 33, 64, 1, 4), (2, 20, 200, 1, 2)], ids=str)
@pytest.mark.parametrize("what", ["x", "B", "C", "dt", "z"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite_position_by_position(shape, what, value):
    """One value in a token of one of two sequences, in a prompt of up to 192 tokens and in single tokens: what does not
    depend on it is what it is without it, bit for bit (the same operations in the same order)."""
    H, P, N, G, W = shape
    T, at = 90, 47
    col = {"x": 3, "B": H * P + 2, "C": H * P + G * N + 2, "dt": 1, "z": 3}[what]
    hit = {"x": 0, "B": 0, "C": 0, "dt": 1, "z": 2}[what]

    def run(layer, change, steps):
        x, _ = layer.inputs(2 * T)
        row = at
        if steps:  # token t of the two sequences side by side
            x = [torch.stack([v[:T], v[T:]], 1).reshape(2 * T, -1).contiguous() for v in x]
            row = 2 * at
        if change:
            x[hit][row, col] = value
        if not steps:
            y = layer.ctx.prompt(0, x[0], x[1], z=x[2], offsets=ints([0, T, 2 * T]))
            return y[:T], y[T:], layer.ctx.state(0)
        y = torch.stack([layer.ctx.step(0, *(v[2 * t:2 * t + 2] for v in x)) for t in range(T)])
        return y[:, 0], y[:, 1], layer.ctx.state(0)

    for steps in (False, True):
        y0, other0, s0 = run(Layer(*shape, slots=2, seed=6), False, steps)
        y1, other1, s1 = run(Layer(*shape, slots=2, seed=6), True, steps)
        torch.cuda.synchronize()
        assert torch.equal(other1, other0) and torch.equal(s1[1], s0[1]) and torch.equal(y1[:at], y0[:at])
        if what == "z":
            rest = torch.ones_like(y1, dtype=torch.bool)
            rest[at, col] = False
            assert torch.equal(s1, s0) and torch.equal(y1[rest], y0[rest]) and (value > 0 or not torch.isfinite(y1[at, col]))
        if what == "x":
            rest = torch.arange(H * P, device=dev()) != col
            assert torch.equal(y1[:, rest], y0[:, rest])
            assert value > 0 or not torch.isfinite(y1[at, col])
        if what == "dt":
            assert torch.equal(y1[:, :P], y0[:, :P]) and torch.equal(s1[0, 0], s0[0, 0])
            if not value < 0:
                assert not torch.isfinite(y1[at:, P:]).any() and not torch.isfinite(s1[0, 1]).any()
        if what == "C":
            assert torch.equal(s1[0], s0[0]) and torch.equal(y1[at + W:], y0[at + W:])
        if what == "B":
            mine = torch.zeros((H, 1, N), dtype=torch.bool, device=dev())
            mine[:H // G, :, 2] = True
            keep = ~mine.expand(H, P, N)
            assert torch.equal(s1[0][keep], s0[0][keep])
