"""The numbers of positions up to which layer norm's calls can be launched.  No
kernel is launched."""
import ctypes

import paper_2003_12621_amd as fs
from paper_2003_12621_amd import attention as at


def status(**kw):
    base = dict(batch=1, positions=1, channels=16, x_dtype=1, y_dtype=1, x_layout=0, y_layout=0, eps=1e-5)
    base.update(kw)
    need = ctypes.c_size_t()
    return fs.lib().fftsplit_layer_norm_workspace(ctypes.byref(at.LayerNorm(**base)), ctypes.byref(need))


def test_channels_first():
    """The narrowest kernel (bf16 rows that 4 does not divide, above 512
    channels) takes 8 positions by 1024 threads: 2^22 of them would make 2^32."""
    first = dict(x_layout=1, y_layout=1, channels=513)
    for s in (9, 15, 25):
        tiles = (s + 15) // 16
        most = ((1 << 21) - 1) // tiles
        assert status(batch=most, positions=s, **first) == fs.SUCCESS
        assert most * ((s + 7) // 8) * 1024 < 1 << 32
        assert status(batch=most + 1, positions=s, **first) == fs.ERROR_NOT_SUPPORTED


def test_channels_last():
    """Below 2^25 rows up to 1024 channels, in several launches where need be, 2^23 above."""
    for c, most in ((8, 25), (257, 25), (1024, 25), (1025, 23), (8192, 23)):
        assert status(positions=(1 << most) - 1, channels=c) == fs.SUCCESS
        assert status(positions=1 << most, channels=c) == fs.ERROR_NOT_SUPPORTED
