"""The state space mixer's two ways through a prompt, where each can go wrong:
calls of up to 192 tokens position by position, longer ones in chunks (needs an
MI355X).  Tolerances are those of test_gpu_ssm.py, and derived there."""
import ctypes

import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod
from test_gpu_ssm import SHAPES, SUMS, TYPES, Layer, close, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_ragged_short_prompts(shape, dtype):
    """Position by position: blocks of 32 that end inside, an empty sequence, and on from there."""
    lay = Layer(*shape, dtype=dtype, slots=5, seed=1 + sum(shape))
    for lens in ([33, 0, 1, 130, 64], [2, 31, 32, 3, 0], [256, 0, 0, 0, 0], [33, 0, 1, 94, 64], [192, 0, 0, 0, 0]):
        offs = np.concatenate([[0], np.cumsum(lens)]).tolist()
        x, xr = lay.inputs(offs[-1])
        y = lay.ctx.prompt(0, x[0], x[1], z=x[2], offsets=ints(offs))
        lay.check(y, lay.want(xr, offs), str(lens))


@pytest.mark.parametrize("T", [191, 192, 193, 255, 256, 257, 320, 321])
def test_lengths_around_the_change(T):
    lay = Layer(3, 40, 64, 1, 4, slots=1, max_tokens=T, seed=T)
    x, xr = lay.inputs(T)
    lay.check(lay.ctx.prompt(0, x[0], x[1], z=x[2]), lay.want(xr, [0, T]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(6, 64, 128, 1, 4), (4, 32, 64, 2, 4), (3, 24, 16, 1, 3), (2, 16, 200, 1, 4)], ids=str)
def test_strong_decays_in_chunks(shape, dtype):
    """Heads that forget within a position beside ones that do not, and steps of 30 that leave nothing in any."""
    lay = Layer(*shape, dtype=dtype, slots=2, seed=21, decay=4000.0)
    x, _ = lay.inputs(700)
    x[1][100:110] = 30.0
    x[1][400:402] = 30.0
    xr = tuple(t.double().cpu().numpy() for t in x)
    offs = [0, 610, 700]
    lay.check(lay.ctx.prompt(0, x[0], x[1], z=x[2], offsets=ints(offs)), lay.want(xr, offs))


def test_large_values_in_chunks():
    """Inputs of 1e15 with steps that leave nothing: every row within its own size."""
    lay = Layer(2, 24, 16, 1, 4, slots=1, seed=22)
    x, _ = lay.inputs(500)
    x[0][:, :lay.D] *= 1e15
    x[1][250:260] = 30.0
    xr = tuple(t.double().cpu().numpy() for t in x)
    y = lay.ctx.prompt(0, x[0], x[1], z=x[2])
    want = lay.want(xr, [0, 500])
    lay.check(y, want)
    for t in range(0, 500, 11):
        close(y[t].double().cpu().numpy(), want[t], 10 * SUMS, f"row {t}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape,first", [((4, 64, 128, 1, 4), 8), ((4, 64, 64, 1, 4), 1), ((5, 33, 20, 1, 2), 3)], ids=str)
def test_slices_of_one_projection_in_chunks(shape, first, dtype):
    """xbc, z and dt from one projection's rows at even and odd starts, the outputs over the gate."""
    lay = Layer(*shape, dtype=dtype, slots=2, seed=23)
    T, D, C, H = 600, lay.D, lay.C, lay.H
    t, tr = lay.rows(T, first + D + C + H + 5)
    cut = lambda v: (v[:, first:first + D], v[:, first + D:first + D + C], v[:, first + D + C:first + D + C + H])  # noqa: E731
    (z, xbc, dt), (zr, xr, dr) = cut(t), cut(tr)
    before = t.clone()
    y = lay.ctx.prompt(0, xbc, dt, z=z, y=z, offsets=ints([0, 401, T]))
    lay.check(y, lay.want((xr, dr, zr), [0, 401, T]))
    before[:, first:first + D] = y
    assert torch.equal(before, t)


def test_slots_as_named_in_chunks():
    lay = Layer(2, 16, 24, 2, 4, slots=5, seed=24, decay=1.2)
    x, xr = lay.inputs(500)
    offs = [0, 100, 200, 300, 400, 500]
    lay.check(lay.ctx.prompt(0, x[0], x[1], z=x[2], offsets=ints(offs)), lay.want(xr, offs), "fill")
    for k, (src, dst) in enumerate([([3, -1, 0], [1, 2, 0]), ([0, 1, 2], [-1, 4, 2]), ([4, 99, -7], [4, 99, 1])]):
        seen = [s if 0 <= s < 5 else -1 for s in src], [d if 0 <= d < 5 else -1 for d in dst]
        offs = [0, 700, 700, 775]
        x, xr = lay.inputs(775)
        y = lay.ctx.prompt(0, x[0], x[1], z=x[2], offsets=ints(offs), src=ints(src), dst=ints(dst))
        lay.check(y, lay.want(xr, offs, *seen), f"prompt {k}")


def test_strides_at_the_limit_and_beyond():
    """Rows 2^24 elements apart, far past 2^31 elements, for inputs and outputs; one more is refused."""
    lay = Layer(1, 8, 8, 1, 4, dtype="bf16", slots=1, max_tokens=300, seed=25)
    T, stride = 300, 1 << 24
    big = torch.empty((T - 1) * stride + 128, dtype=torch.bfloat16, device=dev())
    x, xr = lay.inputs(T)
    wide, out = big.as_strided((T, lay.C), (stride, 1)), big.as_strided((T, lay.D), (stride, 1), 64)
    wide.copy_(x[0])
    lay.check(lay.ctx.prompt(0, wide, x[1], z=x[2], y=out), lay.want(xr, [0, T]))
    far = big.as_strided((2, lay.C), (stride + 1, 1))
    with pytest.raises(lcsm_mod().LcsmError, match="2\\^24"):
        lay.ctx.prompt(0, far, x[1][:2])


def test_layers_and_bad_offsets_in_chunks():
    lay = Layer(2, 16, 16, 1, 4, M=3, slots=4, seed=26)
    for m in (2, 0):
        x, xr = lay.inputs(400)
        y = lay.ctx.prompt(m, x[0], x[1], z=x[2], offsets=ints([0, 12, 400]))
        lay.check(y, lay.want(xr, [0, 12, 400], m=m), f"layer {m}", m=m)
    assert float(lay.ctx.state(1).abs().max()) == 0.0
    # offsets out of range, falling, and rows that several sequences claim: nothing outside the rows is touched
    guard = torch.full((420, lay.D), 7.0, device=dev())
    x, _ = lay.inputs(400)
    for offs in ([-5, 1000, 3], [400, 0, 400, 0, 400], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1]):
        lay.ctx.prompt(1, x[0], x[1], y=guard[10:410], offsets=ints(offs))
        torch.cuda.synchronize()
        assert bool((guard[:10] == 7.0).all()) and bool((guard[410:] == 7.0).all()), offs
    for m in (0, 2):
        close(lay.ctx.state(m).double().cpu().numpy(), lay.state[m], SUMS, "another layer")


def test_a_recorded_long_prompt_replays():
    stream = torch.cuda.Stream(dev())
    lay = Layer(2, 32, 64, 1, 4, slots=2, max_tokens=900, seed=27, stream=stream)
    x, _ = lay.inputs(900)
    ys = torch.empty((900, lay.D), device=dev())
    fresh, zero = ints([-1]), ints([0])
    run = lambda: lay.ctx.prompt(0, x[0], x[1], z=x[2], y=ys, src=fresh, dst=zero)  # noqa: E731
    with torch.cuda.stream(stream):
        run()
        torch.cuda.synchronize()
        eager, state = ys.clone(), lay.ctx.state(0).clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            run()
        for k in range(3):
            ys.fill_(float("nan"))
            x2, _ = lay.inputs(300)
            lay.ctx.prompt(0, x2[0], x2[1], src=ints([0]), dst=ints([1]))
            lay.ctx.state(0)[0].fill_(5.0)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(ys, eager) and torch.equal(lay.ctx.state(0)[0], state[0]), k


def test_more_rows_than_the_products_take_are_refused():
    lcsm = lcsm_mod()
    codes, scales = lcsm.Q4.quantize(torch.ones((1, 2, 32), device=dev()), 32, torch.float32)
    q = lcsm.Q4(codes, scales, 32, 32)
    x = torch.ones((1, 32), device=dev())
    y = torch.empty((1, 2), device=dev())
    lib = lcsm.raw()
    for rows in (65535 * 16 + 1, 2 ** 31 - 1, -1):
        assert lib.lcsm_q4_matvec(q._ctx, 0, rows, 0, x.data_ptr(), 32, y.data_ptr(), 2) == lcsm.LCSM_EINVAL
    assert lib.lcsm_q4_matvec(q._ctx, 0, 1, 0, x.data_ptr(), ctypes.c_size_t(32), y.data_ptr(), ctypes.c_size_t(2)) == 0
    torch.cuda.synchronize()
    assert torch.allclose(y, torch.full_like(y, 32.0))
