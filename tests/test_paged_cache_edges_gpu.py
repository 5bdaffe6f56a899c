"""GPU tests of the paged cache's attention at its edges: faults in the offsets, chunks
longer than the caller said, every slot counted once, many query heads per KV head,
and the range of the values.

Tolerances.  The weights of one output, relative to the largest, are rounded to bf16
for the value product (a relative error d_j of at most 2^-9 each) and summed unrounded;
the output is rounded to bf16 (at most 2^-9).  So for every element
    |error| <= 2^-9 sum_j A_j |v_j| + 2^-9 |o| <= 2^-8 sum_j A_j |v_j|,
of which twice is allowed (the fp32 accumulation has its room in it), and for a whole
output row, over values v_j whose signs are independent of the d_j,
    E |error - output rounding|^2 = sum_j A_j^2 d_j^2 |v_j|^2 <= 2^-18 sum_j A_j^2 |v_j|^2,
of whose root four times is allowed, plus 2^-8 |o| for the output's rounding and the
accumulation.  A lost slot moves the row by A_j |v_j|, which is more up to thousands of
slots of equal weight."""
import numpy as np
import pytest
import torch

import _cache_ref as R
from test_paged_cache_gpu import FORMATS, Box, api, dev_bf16, host_bits  # noqa: F401 (api: the fixture)

pytestmark = pytest.mark.gpu
INDEX = 0x08


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def weights(q, k, seen, scale):
    """fp64 attention weights [G, seen] of one token's heads."""
    x = scale * (q @ k[:seen].T)
    p = np.exp(x - x.max(-1, keepdims=True))
    return p / p.sum(-1, keepdims=True)


def check_rows(box, news, q, got, t0=0):
    """Both bounds of the module's comment, for every output row."""
    G = box.H_q // box.H_kv
    for b, n in enumerate(news):
        for g in range(box.H_kv):
            s = b * box.H_kv + g
            for i in range(n):
                o, seen = got[t0 + i, g * G:(g + 1) * G], box.lens[s] - n + i + 1
                if seen <= 0:
                    assert (o == 0).all()
                    continue
                a = weights(q[t0 + i, g * G:(g + 1) * G], box.k[s], seen, box.scale)
                v = box.v[s][:seen]
                ref = a @ v
                err = o - ref
                top = np.abs(v).max()
                assert (np.abs(err) <= 2.0 ** -7 * (a @ np.abs(v)) + 1e-9 * top).all(), (b, g, i)
                spread = np.sqrt((a * a) @ (v * v).sum(-1))
                norm = np.linalg.norm(ref, axis=-1)
                assert (np.linalg.norm(err, axis=-1) <= 2.0 ** -7 * spread + 2.0 ** -8 * norm).all(), (b, g, i)
        t0 += n


# ---------------------------------------------------------------- faults in the offsets
@pytest.mark.parametrize("fmt", ["bf16", "int8"])
@pytest.mark.parametrize("news", [[1, 2], [2, 1], [40, 17]])
def test_offsets_that_do_not_start_at_zero_are_reported(api, fmt, news):
    """The status says so, in both kernels; the tokens there are get their attention and
    the rows before them stay as they were."""
    box = Box(api, 2, 4, 2, 64, 16, fmt, 90)
    box.fill([70, 90, 45, 66])
    T, skip = sum(news) + 1, 1
    q = R.bf16_values(R.bf16_bits(box.rng.standard_normal((T, 4, 64))))
    out = torch.full((T, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    off = ints([skip, skip + news[0], T])
    api.tgvkv_chunk_attention(box.desc, box.cache, box.table, box.lens_t(box.lens),
                              dev_bf16(R.bf16_bits(q)).view(T, 4, 64), off, max(news), out, box.ws)
    assert api.tgvkv_status(box.ws) == INDEX
    got = R.bf16_values(host_bits(out)).reshape(T, 4, 64)
    assert (got[:skip] == 3).all()
    check_rows(box, news, q[skip:], got[skip:])


@pytest.mark.parametrize("fmt", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("H_q,news,most", [(4, [5, 2], 3), (4, [2, 7], 2), (8, [70, 20], 33), (2, [200, 3], 150)])
def test_a_chunk_longer_than_the_caller_said(api, fmt, H_q, news, most):
    """The status says so; its first max_q tokens get their attention (each up to its own
    slot, also where the set has fewer slots than the chunk has tokens), the rest no row."""
    box = Box(api, 2, H_q, 2, 128, 16, fmt, 400)
    box.fill([400, news[0] - 1, 333, 1])
    T = sum(news)
    q = R.bf16_values(R.bf16_bits(box.rng.standard_normal((T, H_q, 128))))
    out = torch.full((T, H_q, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    api.tgvkv_chunk_attention(box.desc, box.cache, box.table, box.lens_t(box.lens),
                              dev_bf16(R.bf16_bits(q)).view(T, H_q, 128), ints([0, news[0], T]), most, out, box.ws)
    assert api.tgvkv_status(box.ws) == INDEX
    got = R.bf16_values(host_bits(out)).reshape(T, H_q, 128)
    lens, t0 = box.lens, 0
    for b, n in enumerate(news):
        done = min(n, most)
        # the computed tokens are the last of the slots before the ones left out
        box.lens = [x - (n - done) for x in lens]
        alone = [done if x == b else 0 for x in range(2)]
        check_rows(box, alone, q[t0:t0 + done], got[t0:t0 + done])
        assert (got[t0 + done:t0 + n] == 3).all()
        t0 += n


# ---------------------------------------------------------------- every slot, once
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H_q,H_kv,page,longest,news", [
    (1, 2, 2, 64, 9001, [1]), (1, 2, 1, 16, 9001, [8]), (1, 14, 2, 256, 8193, [1]), (2, 4, 4, 32, 4100, [5, 5]),
    (1, 2, 2, 64, 9001, [70]), (2, 7, 1, 16, 5003, [90, 300]), (6, 16, 16, 64, 700, [96, 17, 128, 1, 40, 0]),
    (40, 8, 8, 64, 900, [1] * 40), (8, 2, 2, 16, 500, [1, 2, 0, 4, 3, 1, 1, 2])])
def test_every_slot_counts_once(api, fmt, d, B, H_q, H_kv, page, longest, news):
    """Keys of zero weigh every visible slot alike, and slot j's value is 1 in dim j mod d
    alone: output c is (slots seen of residue c) / (slots seen), a quotient of integers.
    Sums of ones are exact and so is P; one slot more or less changes a count below 142
    by more than 2^-7.2, and the output is rounded once (2^-9)."""
    box = Box(api, B, H_q, H_kv, d, page, fmt, longest)
    lens = [longest - (s * 7919) % (longest // 2) for s in range(box.S)]
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    v = np.zeros((int(off[-1]), d))
    at = np.concatenate([np.arange(n) for n in lens])
    v[np.arange(len(at)), at % d] = 1
    k_t, v_t = torch.zeros(len(at), d, dtype=torch.bfloat16, device="cuda"), dev_bf16(R.bf16_bits(v)).view(-1, d)
    api.tgvkv_cache_write_rows(box.desc, box.cache, box.table, ints([0] * box.S), k_t, v_t,
                               torch.from_numpy(off).cuda(), ints([0] * box.S), box.ws)
    box.lens = lens
    _, got = box.attend(news)
    G, t0 = H_q // H_kv, 0
    for b, n in enumerate(news):
        for g in range(H_kv):
            for i in range(n):
                seen = lens[b * H_kv + g] - n + i + 1
                want = np.bincount(np.arange(max(seen, 0)) % d, minlength=d) / max(seen, 1)
                o = got[t0 + i, g * G:(g + 1) * G]
                assert (np.abs(o - want) <= 2.0 ** -8 * want).all(), (b, g, i)
        t0 += n


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,H_q,H_kv,d,longest,news", [
    (1, 4, 2, 128, 9001, [1]), (1, 4, 2, 128, 9001, [4]), (1, 4, 2, 64, 9001, [20]), (4, 8, 8, 64, 2000, [3] * 4),
    (4, 16, 8, 128, 600, [40, 1, 0, 33]), (1, 7, 1, 128, 3000, [150])])
def test_rows_within_their_spread(api, fmt, B, H_q, H_kv, d, longest, news):
    """Random values: every element, and every row as a whole."""
    box = Box(api, B, H_q, H_kv, d, 64, fmt, longest)
    box.fill([longest - (s * 911) % (longest // 3) for s in range(box.S)])
    q, got = box.attend(news)
    check_rows(box, news, q, got)


# ---------------------------------------------------------------- many heads a KV head
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [32, 33, 65, 100, 128])
@pytest.mark.parametrize("H_kv,page,lens,news", [
    (1, 16, [300, 77, 1, 0], [1, 1, 1, 1]), (2, 64, [130, 129, 3, 128, 257, 60], [2, 0, 3]),
    (1, 256, [1400, 20], [29, 30]), (2, 32, [6000, 5500], [1])])
def test_many_query_heads(api, fmt, d, G, H_kv, page, lens, news):
    """17 to 128 query heads a KV head: row tiles of one to four tokens, partly filled
    warps, one token as a tile, items over several CTAs."""
    box = Box(api, len(news), G * H_kv, H_kv, d, page, fmt, max(lens))
    box.fill(lens)
    q, got = box.attend(news)
    check_rows(box, news, q, got)
    assert np.array_equal(got, box.attend(news, q=q)[1])


def test_thousands_of_sets_with_few_tokens(api):
    """2050 sequences of which one has a token, then every third one or two."""
    B = 2050
    box = Box(api, B, 2, 2, 64, 16, "int8", 40)
    box.fill([(s * 7) % 41 for s in range(2 * B)])
    for news in ([int(b == 1371) for b in range(B)], [(b + 1) % 3 for b in range(B)]):
        q, got = box.attend(news)
        box.check(news, q, got)


# ---------------------------------------------------------------- the range of the values
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("exponent", [-100, -60, 60, 100])
def test_values_of_any_magnitude(api, fmt, d, exponent):
    """Values of magnitudes around 2^-100 to 2^100, beside logits that rise along the
    cache (so that weights above the running reference occur), in both kernels."""
    box = Box(api, 2, 8, 4, d, 32, fmt, 900)
    box.fill([900 - 100 * s for s in range(8)])
    v, off = [], np.concatenate([[0], np.cumsum(box.lens)]).astype(np.int64)
    for s in range(8):
        v.append(R.bf16_values(R.bf16_bits(box.values(box.lens[s]).astype(np.float32))) * 2.0 ** exponent)
        box.k[s] = box.k[s] * np.linspace(0, 4, box.lens[s])[:, None]
    k = R.bf16_values(R.bf16_bits(np.concatenate(box.k)))
    api.tgvkv_cache_write_rows(box.desc, box.cache, box.table, ints([0] * 8), dev_bf16(R.bf16_bits(k)).view(-1, d),
                               dev_bf16(R.bf16_bits(np.concatenate(v))).view(-1, d),
                               torch.from_numpy(off).cuda(), ints([0] * 8), box.ws)
    kk, vv = R.round_trip(k, fmt), R.round_trip(np.concatenate(v), fmt)
    box.k, box.v = ([x[off[s]:off[s + 1]] for s in range(8)] for x in (kk, vv))
    for news in ([1, 1], [2, 3], [40, 70]):
        q, got = box.attend(news)
        check_rows(box, news, q, got)
