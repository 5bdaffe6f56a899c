"""Plain fp64 numpy reference of the paged cache's 4-bit floats, written from the definition
in include/tgvkv.h; shares no code with the CUDA path."""
import numpy as np

from _cache_ref import GROUP

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E_MIN, E_MAX = -60, 56


def encode(x):
    """Rows x (fp64 [..., d]) -> (codes 0 .. 15, scale bytes)."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    top = np.abs(g).max(-1)
    fine = np.isfinite(top)
    e = np.full(top.shape, E_MIN)
    for _ in range(E_MAX - E_MIN):          # smallest e with top <= 6 2^e, one step at a time
        up = fine & (top > 6 * 2.0 ** e.astype(np.float64))
        if not up.any():
            break
        e += up
    a = np.abs(np.where(fine[..., None], g, 0.0)) / 2.0 ** e[..., None].astype(np.float64)
    away = np.abs(np.minimum(a, 6.0)[..., None] - LEVELS)
    near = away == away.min(-1, keepdims=True)
    first = near.argmax(-1)                 # one level, or two of a tie: the even one
    tie = near.sum(-1) == 2
    code = np.where(tie & (first % 2 == 1), first + 1, first)
    code = code + 8 * (np.signbit(g) & fine[..., None])
    return code.reshape(x.shape).astype(np.uint8), np.where(fine, e + 127, 255).astype(np.uint8)


def decode(code, byte):
    """Codes and scale bytes -> fp64 values (a NaN group reads as NaN)."""
    s = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    v = np.where(code >= 8, -1.0, 1.0) * LEVELS[code & 7]
    g = v.reshape(*code.shape[:-1], code.shape[-1] // GROUP, GROUP) * s[..., None]
    return g.reshape(code.shape)


def round_trip(x):
    return decode(*encode(x))


def pack(code):
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def unpack(stored):
    u = stored.astype(np.uint8)
    return np.stack([u & 15, u >> 4], -1).reshape(*u.shape[:-1], 2 * u.shape[-1])
