"""Attention over 4-bit floats at logits far beyond those of a model: the weights of a set's
slots depend on differences of logits alone, and V reads back exactly where one slot has all
the weight, however large the logits are.

The logits are exact in fp32 (products of powers of two whose sum has at most 24 bits), and
softmax_scale is the float next to ln 2, so that a logit in units of log2 is the product
q k itself, to within 3e-9 of differences.  Tolerances: one visible slot, or one whose
weight is 1 beside weights below 2^-126, reads back as its V, which is exact in bf16; else those
of test_fp4_cache_gpu.py, 2^-7 sum_j A_ij |v_j| + 1e-6."""
import numpy as np
import pytest

import _cache_ref as R
from test_fp4_cache_gpu import Box, api  # noqa: F401
from test_paged_cache_gpu import Box as FlatBox

pytestmark = pytest.mark.gpu

LN2 = float(np.float32(np.log(2.0)))


def q_and_k(d, n, slots, top, step):
    """Queries [n, 1, d] and keys [slots, d] whose products are top + step[j] at slot j
    (top a power of two, step[j] in {0, 4, 64, 68})."""
    q, k = np.zeros((n, 1, d)), np.zeros((slots, d))
    q[..., 0], q[..., 1], q[..., 2] = top, 64.0, 4.0
    k[:, 0] = 1.0
    k[:, 1], k[:, 2] = np.asarray(step) >= 64, np.asarray(step) % 64 >= 4
    return q, k


# up to 32 rows by the row streams, 40 by the tile kernel
@pytest.mark.parametrize("n", [1, 9, 24, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_one_slot_reads_back_exactly(api, d, n):
    """The first token sees one slot of every scale, the others equal rows."""
    B = 117                                  # e = -60 .. 56
    box = Box(api, B, 1, 1, d, 16, n, scale=LN2)
    v = np.tile(np.where(np.arange(d) % 2, -1.5, 3.0), (B, 1))
    v[:, ::32] = 6.0                         # a group's scale is 2^e
    v = v * 2.0 ** np.arange(-60, 57)[:, None]
    for top in (2.0 ** 24, 2.0 ** 29, 2.0 ** 30, 2.0 ** 31, 2.0 ** 34, -2.0 ** 31):
        q, k = q_and_k(d, n, n, top, np.zeros(n))
        box.put(np.tile(k, (B, 1)), np.repeat(v, n, axis=0), [n] * B)
        q, got = box.attend([n] * B, q=np.tile(q, (B, 1, 1)))
        got = got.reshape(B, n, d)
        assert np.array_equal(got[:, 0], v), top
        # weights rounded to bf16 and the output too, each within 2^-8 at most
        assert (np.abs(got - v[:, None]) <= 2.0 ** -7 * np.abs(v[:, None])).all(), top


@pytest.mark.parametrize("n", [1, 9, 24, 40])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("top", [2.0 ** 20, 2.0 ** 25, 2.0 ** 27, -2.0 ** 26])
def test_neighbouring_logits_keep_their_ratio(api, d, n, top):
    """Halves of a set whose logits differ by 4 (64 at 2^27, where 4 is no step of fp32): weights 1
    and 1/16 (2^-64) whichever warp, CTA or chunk has which half."""
    slots, up = 700, 4 if top < 2.0 ** 27 else 64
    for sign in (1, -1):                     # the larger logits last, or first
        half = np.arange(slots)[::sign] >= slots // 2
        q, k = q_and_k(d, n, slots, top, 64 * (up == 4) + up * half)
        v = np.where(half, -1.0, 1.0)[:, None] * np.where(np.arange(d) % 2, 1.0, 0.5)
        box = Box(api, 1, 1, 1, d, 16, slots, scale=LN2)
        box.put(k, v, [slots])
        q, got = box.attend([n], q=q)
        box.check([n], q, got)


@pytest.mark.parametrize("fmt", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("n", [1, 40])
def test_the_other_formats_at_the_same_logits(api, fmt, n):
    """What the 4-bit floats are held to, of pages whose values are exact in every format."""
    d, slots = 64, 700
    for top in (2.0 ** 20, 2.0 ** 25):
        half = np.arange(slots) >= slots // 2
        q, k = q_and_k(d, n, slots, top, 64 + 4 * half)
        v = np.where(half, -1.0, 1.0)[:, None] * np.ones(d)
        box = FlatBox(api, 1, 1, 1, d, 16, fmt, slots, scale=LN2)
        rows = iter((k, v))
        box.values = lambda *_, **__: R.bf16_values(R.bf16_bits(next(rows)))
        box.fill([slots])
        q, got = box.attend([n], q=q)
        box.check([n], q, got)
