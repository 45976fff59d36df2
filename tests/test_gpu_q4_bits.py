"""Products with 4-bit weights (lcsm_q4.h): nothing is summed that the result
does not have, and no bit of a row is lost on the way (needs an MI355X).  The
outputs here are exact in fp32 sums, so every comparison is for equality."""
import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def pack(codes):
    """[1, N, ceil(K/2)] bytes of codes [N, K]."""
    n, k = codes.shape
    c = np.concatenate([codes, np.zeros((n, k % 2), np.int64)], 1)
    return torch.from_numpy((c[:, 0::2] | c[:, 1::2] << 4).astype(np.uint8)[None]).to(dev())


def product(codes, x, group, scale=1.0, zeros=None):
    n, k = codes.shape
    s = torch.full((1, n, -(-k // group)), scale, device=dev())
    ctx = lcsm_mod().Q4(pack(codes), s, k, group, zeros=zeros)
    return ctx.matvec(0, x)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("R,N", [(1, 40), (20, 40), (40, 40), (2, 8208)])
def test_weights_of_zero_add_nothing(R, N, group, dtype):
    """One weight of a row is not zero, and its input is small beside the others:
    the output is that product."""
    K = 300
    r = np.random.default_rng(R + group)
    codes = np.full((N, K), 8)
    at = r.integers(0, K, N)
    codes[np.arange(N), at] = 9
    x = torch.from_numpy((2.0 ** r.uniform(-10, 1, (R, K))).astype(np.float32)).to(TYPES[dtype])
    want = x.float().numpy()[:, at]
    assert np.array_equal(product(codes, x.to(dev()), group).float().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 128])
def test_large_rows_of_one_sign_stay_finite(group, zeros, dtype):
    """Inputs of 1.5e35 (6e4 in fp16), scales that bring the sums back: 128 products
    with whole numbers up to 15 are within fp32."""
    N, K = 24, 256
    r = np.random.default_rng(group)
    codes = r.integers(0, 16, (N, K))
    value = 6e4 if dtype == "f16" else 1.5e35
    x = torch.full((3, K), value, device=dev()).to(TYPES[dtype])
    z = torch.from_numpy(r.integers(0, 16, (1, N, K // group), dtype=np.uint8)).to(dev()) if zeros else None
    y = product(codes, x, group, 2.0 ** -12, z).double().cpu().numpy()
    zero = 8 if z is None else z[0].cpu().numpy().astype(np.int64)[:, np.arange(K) // group]
    want = (codes - zero).sum(1) * 2.0 ** -12 * x[0, 0].double().item()
    # sums of whole multiples of one value: fp32 keeps them but for the roundings of the multiples and of y
    tol = 1e-6 + {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dtype]
    terms = np.abs(codes - zero).sum(1) * 2.0 ** -12 * x[0, 0].double().item()
    assert np.isfinite(y).all() and (np.abs(y - want) <= 1e-6 * terms + tol * np.abs(want)).all()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("R", [1, 20, 40])
def test_fp32_rows_keep_all_their_bits(R, group):
    """One value of 24 significant bits a row times powers of two."""
    K, N = 128, 32
    r = np.random.default_rng(group)
    codes = 8 + r.choice([-8, -4, -2, -1, 1, 2, 4], (N, K))
    x = np.zeros((R, K), np.float32)
    at = r.integers(0, K, R)
    x[np.arange(R), at] = (2.0 ** 23 + r.integers(0, 2 ** 23, R) // 2 * 2 + 1) * 2.0 ** r.integers(-40, 20, R).astype(float)
    want = x[np.arange(R), at].astype(np.float64)[:, None] * (codes - 8).T[at]
    got = product(codes, torch.from_numpy(x).to(dev()), group).double().cpu().numpy()
    assert np.array_equal(got, want)
