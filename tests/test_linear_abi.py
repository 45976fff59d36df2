"""Argument checks of the linear attention layer's operators that touch no device,
the structs of their binding, and their oracle (CPU only)."""
import ctypes

import numpy as np
import pytest

import paper_2410_12982_amd.lcsm as lcsm
from oracle import lin as oracle
from test_operators_abi import _fields

lib = lcsm.raw()


@pytest.mark.parametrize("header,name,struct", [
    ("lcsm_rot.h", "lcsm_rot_shape", lcsm.RotShape), ("lcsm_rot.h", "lcsm_rot_io", lcsm.RotIo),
    ("lcsm_q8.h", "lcsm_q8_shape", lcsm.Q8Shape), ("lcsm_lin.h", "lcsm_lin_shape", lcsm.LinShape),
    ("lcsm_lin.h", "lcsm_lin_io", lcsm.LinIo)])
def test_structs_match_the_headers(header, name, struct):
    want = _fields(header, name)
    assert [f for f, _ in want] == [f[0] for f in struct._fields_]
    for (f, d), (_, t) in zip(want, struct._fields_):
        kind = {"int": ctypes.c_int, "float": ctypes.c_float, "size_t": ctypes.c_size_t}.get(d, ctypes.c_void_p)
        assert t is kind or (f == "reserved" and t._type_ is ctypes.c_int), f


def size_of(kind, struct, good, **over):
    n = ctypes.c_size_t(0)
    reserved = over.pop("reserved", None)
    s = struct(**{**good, **over})
    if reserved is not None:
        s.reserved[reserved] = 1
    return getattr(lib, f"lcsm_{kind}_workspace_bytes")(ctypes.byref(s), ctypes.byref(n)), n.value


ROT = dict(M=2, P=64, q_heads=4, k_heads=2, rotary=32, pairs=0, norm=1, dtype=1, eps=1e-5)
Q8 = dict(M=2, N=100, K=200, max_rows=33)
LIN = dict(M=2, slots=3, H=4, G=2, K=16, V=24, dtype=1, max_tokens=1000, scale=1.0)


@pytest.mark.parametrize("over", [dict(M=0), dict(M=16385), dict(P=0), dict(P=513), dict(q_heads=0), dict(q_heads=65537), dict(
    k_heads=-1), dict(k_heads=65537), dict(rotary=31), dict(rotary=66), dict(rotary=-2), dict(pairs=2), dict(pairs=-1), dict(norm=3),
    dict(norm=-1), dict(dtype=3), dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")), dict(reserved=2)], ids=str)
def test_rot_shapes_refused(over):
    assert size_of("rot", lcsm.RotShape, ROT)[0] == 0
    assert size_of("rot", lcsm.RotShape, ROT)[1] >= 16 * 8 + 2 * 2 * 64 * 4
    assert size_of("rot", lcsm.RotShape, ROT, **over)[0] == lcsm.LCSM_EINVAL


@pytest.mark.parametrize("over", [dict(M=0), dict(M=16385), dict(N=0), dict(N=(1 << 24) + 1), dict(K=0), dict(K=(1 << 17) + 1),
                                  dict(max_rows=0), dict(max_rows=(1 << 24) + 1), dict(N=1 << 24, K=1 << 17), dict(reserved=3)], ids=str)
def test_q8_shapes_refused(over):
    r, n = size_of("q8", lcsm.Q8Shape, Q8)
    assert r == 0 and n >= 2 * 112 * 256 + 2 * 2 * 100 * 4 + 48 * 256 + 33 * 4 and n % 256 == 0
    assert size_of("q8", lcsm.Q8Shape, Q8, **over)[0] == lcsm.LCSM_EINVAL


@pytest.mark.parametrize("over", [dict(M=0), dict(M=16385), dict(slots=0), dict(slots=32769), dict(H=0), dict(H=65536, G=1), dict(G=0),
                                  dict(G=3), dict(K=0), dict(K=257), dict(V=0), dict(V=4097), dict(dtype=3), dict(dtype=-1),
                                  dict(max_tokens=-1), dict(max_tokens=(1 << 26) + 1), dict(scale=float("nan")), dict(
                                      H=32768, G=32768, K=256, V=257), dict(M=16384, slots=32768, H=8192, G=8192, K=256, V=256),
                                  dict(reserved=0)], ids=str)
def test_lin_shapes_refused(over):
    r, n = size_of("lin", lcsm.LinShape, LIN)
    assert r == 0 and n >= 2 * 3 * 2 * 16 * 24 * 4 and n % 256 == 0
    assert size_of("lin", lcsm.LinShape, LIN, max_tokens=0)[1] <= n <= size_of("lin", lcsm.LinShape, LIN, max_tokens=100000)[1]
    assert size_of("lin", lcsm.LinShape, LIN, **over)[0] == lcsm.LCSM_EINVAL


def test_null_arguments():
    ctx, fake, n = ctypes.c_void_p(1), ctypes.c_void_p(4096), ctypes.c_size_t()
    shapes = dict(rot=lcsm.RotShape(**ROT), q8=lcsm.Q8Shape(**Q8), lin=lcsm.LinShape(**LIN))
    for kind, s in shapes.items():
        bytes_of = getattr(lib, f"lcsm_{kind}_workspace_bytes")
        assert bytes_of(None, ctypes.byref(n)) == lcsm.LCSM_EINVAL and bytes_of(ctypes.byref(s), None) == lcsm.LCSM_EINVAL
        assert getattr(lib, f"lcsm_{kind}_reset")(None) == lcsm.LCSM_EINVAL
        assert getattr(lib, f"lcsm_{kind}_last_error")(None) == b""
        getattr(lib, f"lcsm_{kind}_destroy")(None)
    rot = lambda c, s, f, ws, size: lib.lcsm_rot_init(c, s, f, None, None, None, ws, size)  # noqa: E731
    q8 = lambda c, s, f, ws, size: lib.lcsm_q8_init(c, s, f, f, None, None, ws, size)  # noqa: E731
    lin = lambda c, s, f, ws, size: lib.lcsm_lin_init(c, s, f, None, ws, size)  # noqa: E731
    for init, kind in ((rot, "rot"), (q8, "q8"), (lin, "lin")):
        s = ctypes.byref(shapes[kind])
        assert init(None, s, fake, fake, 1 << 30) == lcsm.LCSM_EINVAL
        for args, code in (((None, fake, fake, 1 << 30), lcsm.LCSM_EINVAL), ((s, None, fake, 1 << 30), lcsm.LCSM_EINVAL),
                           ((s, fake, ctypes.c_void_p(4097), 1 << 30), lcsm.LCSM_EINVAL), ((s, fake, fake, 255), lcsm.LCSM_ENOMEM)):
            ctx.value = 1
            assert init(ctypes.byref(ctx), *args) == code
            assert not ctx.value
    assert lib.lcsm_q8_init(ctypes.byref(ctx), ctypes.byref(shapes["q8"]), fake, None, None, None, fake, 1 << 30) == lcsm.LCSM_EINVAL
    assert lib.lcsm_rot_apply(None, 0, 1, ctypes.byref(lcsm.RotIo())) == lcsm.LCSM_EINVAL
    assert lib.lcsm_q8_matmul(None, 0, 1, 0, fake, 1, fake, 1) == lcsm.LCSM_EINVAL
    assert lib.lcsm_lin_step_layer(None, 0, 1, ctypes.byref(lcsm.LinIo())) == lcsm.LCSM_EINVAL
    assert lib.lcsm_lin_prompt_layer(None, 0, 1, 1, None, ctypes.byref(lcsm.LinIo())) == lcsm.LCSM_EINVAL
    p = ctypes.c_void_p()
    assert lib.lcsm_lin_state(None, 0, ctypes.byref(p)) == lcsm.LCSM_EINVAL
    for args in ((None, 1, 8, fake, fake), (fake, 1, 8, None, fake), (fake, 1, 8, fake, None), (fake, -1, 8, fake, fake),
                 (fake, 1, 0, fake, fake), (fake, 1, (1 << 24) + 1, fake, fake)):
        assert lib.lcsm_q8_quantize(*args, None) == lcsm.LCSM_EINVAL
    assert lib.lcsm_q8_quantize(None, 0, 8, None, None, None) == 0


def test_oracle_by_hand():
    """Two tokens of linear attention, a quarter turn, and codes of a row."""
    y, S = oracle.attend([[[2.0]], [[3.0]]], [[[5.0]], [[7.0]]], [[[1.0]], [[-1.0]]], [np.log(0.5)], 0.1, [[[4.0]]])
    assert np.allclose(y[:, 0, 0], [0.2 * 7.0, 0.3 * (3.5 - 7.0)]) and np.allclose(S, -3.5)
    r = np.random.default_rng(0)
    q, k, v, g = r.standard_normal((9, 6, 4)), r.standard_normal((9, 3, 4)), r.standard_normal((9, 3, 5)), -r.random(3)
    s0 = r.standard_normal((3, 4, 5))
    whole, one = oracle.attend(q, k, v, g, 1.0, s0), oracle.attend(q[:4], k[:4], v[:4], g, 1.0, s0)
    two = oracle.attend(q[4:], k[4:], v[4:], g, 1.0, one[1])
    assert np.allclose(whole[0], np.concatenate([one[0], two[0]])) and np.allclose(whole[1], two[1])
    direct = sum(np.exp(g[1]) ** (8 - j) * (q[8, 3] @ k[j, 1]) * v[j, 1] for j in range(9)) + np.exp(g[1]) ** 9 * (q[8, 3] @ s0[1])
    assert np.allclose(whole[0][8, 3], direct)  # heads 2 and 3 read state 1
    x = [[1.0, 2.0, 3.0, 4.0, 9.0]]
    turned = oracle.heads(x, 5, "none", None, 0.0, [1], [np.pi / 2, np.pi], "half")
    assert np.allclose(turned, [[-3.0, -2.0, 1.0, -4.0, 9.0]])
    turned = oracle.heads(x, 5, "none", None, 0.0, [1], [np.pi / 2, np.pi], "adjacent")
    assert np.allclose(turned, [[-2.0, 1.0, -3.0, -4.0, 9.0]])
    n = oracle.heads(r.standard_normal((2, 12)), 6, "rms", None, 0.0, [3, 4], [0.5], "half").reshape(4, 6)
    assert np.allclose((n * n).mean(-1), 1)
    c, s = oracle.codes([[127.0, 0.5, 1.5, -2.5, -127.0], [0.0] * 5, [np.inf, 1.0, 0.0, 0.0, 0.0]])
    assert c.tolist() == [[127, 0, 2, -2, -127], [0] * 5, [0] * 5] and s[:2].tolist() == [1.0, 0.0] and np.isnan(s[2])
    y, size = oracle.q8([[127.0, 1.0]], [[2, -3]], [0.5], [10.0])
    assert y.tolist() == [[(254 - 3) * 0.5 + 10.0]] and size.tolist() == [[125.5]]
