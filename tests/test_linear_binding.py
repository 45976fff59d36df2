"""What the binding of the linear attention layer's operators does before it calls
the library (CPU only: contexts without a handle, which the library refuses)."""
import pytest
import torch

import paper_2410_12982_amd.lcsm as lcsm


def bare(cls, monkeypatch, **fields):
    """A context of `cls` on the CPU, with no handle behind it."""
    monkeypatch.setattr(lcsm, "_current_device", lambda: -1)
    ctx = object.__new__(cls)
    ctx._ctx, ctx._index, ctx.device, ctx.M = lcsm._vp(), -1, torch.device("cpu"), 1
    ctx._order, ctx._last_error = lambda: False, lambda handle: b""
    for k, v in fields.items():
        setattr(ctx, k, v)
    return ctx


def one_value(rows):
    """A tensor [rows, 1] whose rows are one value's memory."""
    return torch.zeros((1, 1), dtype=torch.bfloat16).expand(rows, 1)


@pytest.mark.parametrize("rows", [2 ** 31, 2 ** 32, 2 ** 32 + 4])
def test_rotations_of_more_rows_than_an_int(rows, monkeypatch):
    """Refused, not taken modulo 2^32: a call of 2^32 + 4 rows would turn four."""
    io = lcsm.RotIo()
    ctx = bare(lcsm.Rot, monkeypatch, P=1, q_heads=1, k_heads=0, dtype=torch.bfloat16, _io=io, _io_ref=lcsm.ctypes.byref(io))
    with pytest.raises(ValueError, match="rows"):
        ctx.apply(0, one_value(rows), None, None, q_out=one_value(rows))


@pytest.mark.parametrize("cls", [lcsm.Lin, lcsm.Rot, lcsm.Q8, lcsm.Ssm, lcsm.Norm, lcsm.Q4])
def test_resets_on_their_own_device(cls, monkeypatch):
    """A reset queues work on the context's stream: with another device current it goes to the context's."""
    current = ["another"]

    class Device:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            current.append(self.device)

        def __exit__(self, *exc):
            current.pop()

    monkeypatch.setattr(lcsm.torch.cuda, "device", Device)
    at = []
    ctx = bare(cls, monkeypatch, _reset=lambda handle: at.append(current[-1]) or 0)
    ctx.reset()
    assert at == [ctx.device] and current == ["another"]
