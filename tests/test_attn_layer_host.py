"""Refusals of the attention calls and of AttentionLayer, without a GPU."""
import ctypes

import pytest
import torch

A = 0x1000  # any 16-byte aligned address, never dereferenced: every call below fails its checks first
vp = ctypes.c_void_p
INVALID, UNSUPPORTED, OK, BF16 = 1, 2, 0, 1


@pytest.fixture(scope="module")
def at():
    from paper_2608_20961_b200 import attention, build
    build.build()
    attention.load_library()
    return attention


def z(*s, dt=torch.bfloat16):
    return torch.zeros(s, dtype=dt)


def i32(*s):
    return torch.zeros(s, dtype=torch.int32)


def test_rope_rows_refusals(at):
    rope = at.RopeStruct(cos_sin=A, positions=A, pair_axis=None, n_axes=1, max_positions=16, rot_dim=64, interleaved=0)

    def call(B=2, T=3, off=A, x=A, ld_x=256, y=A, ld_y=256, H=4, d=64, io=BF16, status=None):
        return at.load_library().treewy_rope_rows(ctypes.byref(rope), B, T, vp(off), vp(x), ld_x, vp(y), ld_y, H, d, 0, io, vp(status), None)
    for bad in (dict(B=-1), dict(T=-1), dict(off=None), dict(off=A + 4), dict(x=None), dict(y=A + 2), dict(ld_x=255), dict(H=0),
                dict(status=A + 4)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(io=7), dict(d=63)):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(T=0, off=None, x=None, y=None) == OK and call(B=0, off=None) == OK
    handle = at.Rope(z(16, 64, dt=torch.float32), i32(6))
    for off, x in ((i32(3), z(5, 4, 64)), (i32(3).long(), z(6, 4, 64)), (i32(0), z(6, 4, 64)), (i32(3), z(6, 4, 64, dt=torch.float16))):
        with pytest.raises(ValueError):
            at.treewy_rope_rows(handle, off, x, x)
