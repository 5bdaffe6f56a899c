"""Host-side checks of the paged cache in 4-bit floats (no GPU): its descriptor, the
binding, and the reference the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

import _cache_ref as R
import _fp4_ref as F


def test_descriptor_and_pools():
    from paper_2606_03075_gb300 import _lib, api, build
    build.build()
    lib = _lib.load()
    for d in (64, 128):
        cd = api.make_cache_desc(2, 8, 2, d, 16, 64, 8, "fp4")
        assert cd.format == 4
        assert lib.tgvkv_cache_workspace_size(ctypes.byref(cd)) > 0
        cache = api.alloc_cache(cd, device="meta")
        assert cache.k.shape == (64, 16, d // 2) and cache.k.dtype == torch.uint8
        assert cache.v_scale.shape == (64, 16, d // 32)
    cd.format = 5
    assert lib.tgvkv_cache_workspace_size(ctypes.byref(cd)) == 0
    # the scale pools are not optional
    fake = ctypes.c_void_p(0x10000)
    cd.format = 4
    pools = ctypes.byref(_lib.CachePools(fake, fake, None, None))
    rc = lib.tgvkv_cache_read(ctypes.byref(cd), pools, fake, None, fake, fake, fake, 3, fake, None)
    assert rc == 1 and b"scale" in lib.tgvkv_last_error()


def test_reference_format():
    """The reference's own pins: the scale is the smallest that holds, codes are the
    nearest, ties go to the even code, packing is reversible."""
    rng = np.random.default_rng(1)
    x = R.bf16_values(R.bf16_bits(rng.standard_normal((50, 64)) * 2.0 ** rng.integers(-9, 9, (50, 1))))
    code, byte = F.encode(x)
    s = 2.0 ** (byte.astype(float) - 127)
    top = np.abs(x).reshape(50, 2, 32).max(-1)
    assert (top <= 6 * s).all() and (top > 3 * s).all()
    y, step = F.decode(code, byte), np.repeat(s, 32, axis=1)
    levels = np.concatenate([-F.LEVELS, F.LEVELS])
    best = np.abs(x[..., None] - levels * step[..., None]).min(-1)
    assert np.array_equal(np.abs(y - x), best)
    assert np.array_equal(F.unpack(F.pack(code)), code)
    t = np.zeros((1, 32))
    t[0, :10] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -5]
    code, byte = F.encode(t)
    assert byte[0, 0] == 127 and code[0, :10].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 14]
    t[0, 0] = 6.03125
    assert F.encode(t)[1][0, 0] == 128
    t[0, 0] = 2.0 ** 80                     # beyond the largest scale: saturates
    assert F.encode(t)[1][0, 0] == 127 + 56 and F.round_trip(t)[0, 0] == 6 * 2.0 ** 56
    t[0] = 2.0 ** -61                       # half a step of the smallest scale: a tie
    assert F.encode(t)[1][0, 0] == 127 - 60 and (F.encode(t)[0] == 1).all()
    t[0] = 2.0 ** -62
    assert (F.encode(t)[0] == 0).all()
    t[0, 9] = np.nan
    code, byte = F.encode(t)
    assert byte[0, 0] == 255 and (code == 0).all() and np.isnan(F.decode(code, byte)).all()


def test_outliers_cost_less_than_in_equal_steps():
    """Why the format is there: a group with one large value keeps the small ones better."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((2000, 32))
    x[:, 5] *= 8
    x = R.bf16_values(R.bf16_bits(x))
    err = [np.sqrt(np.mean((y - x) ** 2)) for y in (F.round_trip(x), R.round_trip(x, "int4"))]
    assert err[0] < 0.8 * err[1]
