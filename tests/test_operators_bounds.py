"""Sizes that the gated layer's operators cannot serve are refused before any
work (CPU only)."""
import ctypes

import paper_2410_12982_amd.lcsm as lcsm

lib = lcsm.raw()


def ssm(**over):
    s = dict(M=1, slots=1, H=65535, P=1, N=1, G=65535, W=1, dtype=0, max_tokens=193)
    s.update(over)
    return lib.lcsm_ssm_workspace_bytes(ctypes.byref(lcsm.SsmShape(**s)), ctypes.byref(ctypes.c_size_t()))


def test_groups_beyond_a_prompts_launch():
    assert ssm() == lcsm.LCSM_EINVAL
    assert ssm(max_tokens=192) == 0 and ssm(G=21845) == 0
    assert ssm(H=63550, G=63550) == lcsm.LCSM_EINVAL and ssm(H=63548, G=63548) == 0
