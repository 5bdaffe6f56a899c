"""Plain fp64 numpy reference of the paged cache: its formats, its addressing, and
attention of a chunk of new tokens over it.  Written from the definitions in
include/tgvkv.h; shares no code with the CUDA path."""
import numpy as np

GROUP = 32
Q_MAX = {"int8": 127, "int4": 7}
E_MAX = {"int8": 122, "int4": 120}


def bf16_bits(x):
    """fp32 -> bf16 bits, round to nearest even (NaN kept a NaN)."""
    x = np.asarray(x, np.float32)
    u = x.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r)


def bf16_values(bits):
    """bf16 bits -> fp64 values."""
    return (np.asarray(bits).astype(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def encode(x, fmt):
    """Rows x (fp64 [..., d]) -> (codes int, scale bytes)."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    top = np.abs(g).max(-1)
    fine = np.isfinite(top)
    e = np.full(top.shape, -126)
    for _ in range(E_MAX[fmt] + 126):       # smallest e with top <= Q 2^e, one step at a time
        up = fine & (top > Q_MAX[fmt] * 2.0 ** e.astype(np.float64))
        if not up.any():
            break
        e += up
    q = np.rint(np.where(fine[..., None], g, 0.0) / 2.0 ** e[..., None].astype(np.float64))
    q = np.clip(q, -Q_MAX[fmt], Q_MAX[fmt]).astype(np.int64)
    return q.reshape(x.shape), np.where(fine, e + 127, 255).astype(np.uint8)


def decode(q, byte):
    """Codes and scale bytes -> fp64 values (a NaN group reads as NaN)."""
    s = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    g = q.astype(np.float64).reshape(*q.shape[:-1], q.shape[-1] // GROUP, GROUP) * s[..., None]
    return g.reshape(q.shape)


def round_trip(x, fmt):
    """What rows read back as."""
    if fmt == "bf16":
        return np.asarray(x, np.float64)
    return decode(*encode(x, fmt))


def pack(q, fmt):
    if fmt == "int8":
        return q.astype(np.int8)
    u = (q + 8).astype(np.uint8)
    return u[..., 0::2] | (u[..., 1::2] << 4)


def unpack(stored, fmt):
    if fmt == "int8":
        return stored.astype(np.int64)
    u = stored.astype(np.int64)
    return np.stack([u % 16, u // 16], -1).reshape(*u.shape[:-1], 2 * u.shape[-1]) - 8


def attention(q, k, v, n, scale):
    """One sequence and KV head: q fp64 [n, G, d] the last n of k, v [len, d].
    Returns o [n, G, d], 0 where a token sees nothing."""
    ln = k.shape[0]
    o = np.zeros(q.shape)
    for i in range(n):
        seen = ln - n + i + 1
        if seen <= 0:
            continue
        x = scale * (q[i] @ k[:seen].T)
        p = np.exp(x - x.max(-1, keepdims=True))
        o[i] = (p / p.sum(-1, keepdims=True)) @ v[:seen]
    return o
