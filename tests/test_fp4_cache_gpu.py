"""GPU parity of the paged cache in 4-bit floats: quantising writes, reads and attention
through the C ABI, against the fp64 reference of _fp4_ref.py.

Stored codes, scale bytes and rows read back are exact.  The attention's tolerance is that
of the other formats, whose arithmetic it shares (products of bf16 operands, which the
stored values are exactly): weights rounded to bf16 and an output rounded to bf16, 2^-8
relative each, are off by at most 2^-7 sum_j A_ij |v_j|, plus 1e-6 for the fp32 sums."""
import numpy as np
import pytest
import torch

import _cache_ref as R
import _fp4_ref as F
from test_paged_cache_gpu import Box as FlatBox
from test_paged_cache_gpu import dev_bf16, host_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "the GPU tests need a CUDA device"
    from paper_2606_03075_gb300 import build
    build.build()
    from paper_2606_03075_gb300 import api as _api
    return _api


class Box(FlatBox):
    def __init__(self, api, B, H_q, H_kv, d, page, max_len, **kw):
        super().__init__(api, B, H_q, H_kv, d, page, "fp4", max_len, **kw)

    def put(self, k, v, total):
        """Rows k, v (fp64 values of bf16, set after set) into the sets' first slots."""
        off = np.concatenate([[0], np.cumsum(total)]).astype(np.int64)
        out = torch.empty(self.S, dtype=torch.int32, device="cuda")
        self.api.tgvkv_cache_write_rows(
            self.desc, self.cache, self.table, self.lens_t([0] * self.S),
            dev_bf16(R.bf16_bits(k)).view(-1, self.d), dev_bf16(R.bf16_bits(v)).view(-1, self.d),
            torch.from_numpy(off).cuda(), out, self.ws)
        assert self.api.tgvkv_status(self.ws) == 0
        assert out.cpu().tolist() == list(total)
        kk, vv = F.round_trip(k), F.round_trip(v)
        self.k = [kk[off[s]:off[s + 1]] for s in range(self.S)]
        self.v = [vv[off[s]:off[s + 1]] for s in range(self.S)]
        self.lens = list(total)

    def fill(self, total):
        n = int(sum(total))
        self.put(self.values(n, keys=True), self.values(n), total)

    def stored(self, name, s, n):
        """The pool's bytes of set s's first n slots: codes, scale bytes."""
        rows = self.rows_of(s, 0, n)
        code = getattr(self.cache, name).cpu().numpy().reshape(self.n_pages * self.page, -1)[rows]
        byte = getattr(self.cache, name + "_scale").cpu().numpy().reshape(self.n_pages * self.page, -1)[rows]
        return F.unpack(code), byte


@pytest.mark.parametrize("d,page", [(64, 16), (128, 16), (128, 64), (64, 256)])
def test_rows_stored_and_read_back(api, d, page):
    total = [0, 1, 15, 16, 17, 33, 0, 70, 129, 5, 64, 2]
    box = Box(api, 3, 8, 4, d, page, max(total))
    n = sum(total)
    k, v = box.values(n, keys=True), box.values(n)
    box.put(k, v, total)
    off = np.concatenate([[0], np.cumsum(total)])
    touched = np.zeros(box.n_pages * page, bool)
    for s in range(box.S):
        touched[box.rows_of(s, 0, total[s])] = True
        for name, x in (("k", k), ("v", v)):
            code, byte = F.encode(x[off[s]:off[s + 1]])
            got = box.stored(name, s, total[s])
            assert np.array_equal(got[0], code) and np.array_equal(got[1], byte)
    for t in (box.cache.k, box.cache.v, box.cache.k_scale, box.cache.v_scale):
        assert (t.cpu().numpy().reshape(box.n_pages * page, -1)[~touched] == 255).all()
    out = [torch.full((n + 2, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    api.tgvkv_cache_read(box.desc, box.cache, box.table, None, torch.from_numpy(off.astype(np.int64)).cuda(),
                         *out, box.ws)
    assert api.tgvkv_status(box.ws) == 0
    for t, x in zip(out, (k, v)):
        got = R.bf16_values(host_bits(t))
        assert np.array_equal(got[:n], F.round_trip(x)) and (got[n:] == 7).all()


def test_every_value_and_the_ends_of_the_range(api):
    """Each bf16 magnitude class beside the ties, both zeros, saturation, flushing, and
    groups with an infinity or a NaN."""
    rng = np.random.default_rng(5)
    rows = [np.concatenate([np.arange(32) / 4 - 4, np.arange(32) / 8 + 2]),      # ties of both signs
            np.full(64, -0.0), np.zeros(64)]
    for e in (-133, -126, -70, -63, -62, -61, -60, -59, -1, 0, 1, 54, 55, 56, 57, 58, 60, 90, 120):
        x = rng.choice([1.0, 1.25, 1.5, 1.75, 1.9921875], 64) * 2.0 ** e
        rows.append(x * rng.choice([-1, 1], 64))
        rows.append(x * 2.0 ** -rng.integers(0, 6, 64))
    for bad in (np.nan, np.inf, -np.inf):
        x = rng.standard_normal(64)
        x[17] = bad
        rows.append(x)
    x = R.bf16_values(R.bf16_bits(np.array(rows)))
    n = len(rows)
    box = Box(api, 1, 1, 1, 64, 16, n)
    box.put(x, x[::-1].copy(), [n])
    for name, y in (("k", x), ("v", x[::-1])):
        code, byte = F.encode(y)
        got = box.stored(name, 0, n)
        assert np.array_equal(got[1], byte), np.argwhere(got[1] != byte)[:5]
        assert np.array_equal(got[0], code), (y[got[0] != code][:5], got[0][got[0] != code][:5])
    out = [torch.empty((n, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    api.tgvkv_cache_read(box.desc, box.cache, box.table, None,
                         torch.tensor([0, n], device="cuda"), *out, box.ws)
    got = R.bf16_values(host_bits(out[0]))
    assert np.array_equal(got, F.round_trip(x), equal_nan=True)
    assert np.array_equal(np.signbit(got[1:3]), np.signbit(x[1:3]))


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_every_code_of_every_scale_through_the_attention(api, d, n):
    """Sets of one visible slot: the output is its V, whatever K is (n = 40: the tile kernel,
    whose first token alone sees one slot).  V of code c at scale 2^e is exact in bf16."""
    B = 117                                 # e = -60 .. 56
    box = Box(api, B, 1, 1, d, 16, n, scale=2.0 ** -20)
    e = np.arange(-60, 57)
    code = np.concatenate([np.arange(16), np.arange(15, -1, -1)])
    row = F.decode(np.tile(code.astype(np.uint8), d // 32)[None], np.full((1, d // 32), 127, np.uint8))
    v = np.repeat(row * 2.0 ** e[:, None].astype(float), n, axis=0)
    k = box.values(B * n)
    box.put(k, v, [n] * B)
    assert np.array_equal(box.v[3], v[3 * n:4 * n])
    q, got = box.attend([n] * B)
    assert np.array_equal(got[::n, 0], v[::n])
    # later tokens see several equal rows: a convex combination of equal values, whose
    # weights are rounded to bf16 (their sum is off by 2^-8 at most), and the output too
    for b in range(B):
        assert (np.abs(got[b * n:(b + 1) * n, 0] - v[b * n]) <= 2.0 ** -7 * np.abs(v[b * n])).all(), e[b]


@pytest.mark.parametrize("n", [1, 40])
def test_keys_of_every_scale(api, n):
    """K times 2^e against q times 2^-e gives the logits of e = 0, for every scale."""
    B, d, ln = 117, 128, 70
    box = Box(api, B, 1, 1, d, 32, ln)
    e = np.arange(-60, 57)
    rng = np.random.default_rng(2)
    base = R.bf16_values(R.bf16_bits(rng.standard_normal((ln, d))))
    base[:, ::32] = 5.0                     # every group's scale is 2^0
    k = (base[None] * 2.0 ** e[:, None, None].astype(float)).reshape(-1, d)
    box.put(k, np.tile(box.values(ln), (B, 1)), [ln] * B)
    q = R.bf16_values(R.bf16_bits(rng.standard_normal((1, n, 1, d))))
    q = (q * 2.0 ** -e[:, None, None, None].astype(float)).reshape(B * n, 1, d)
    q, got = box.attend([n] * B, q=q)
    box.check([n] * B, q, got)


# rows of a set (n G): 1 .. 8, .. 16, .. 24, .. 32 (the row streams' sizes), then the tile
# kernel's one and two row tiles; lengths of zero, one, around chunks, tiles and pages
@pytest.mark.parametrize("H_q,H_kv,d,page,n", [
    (1, 1, 64, 16, 1), (8, 8, 128, 16, 1), (28, 4, 128, 64, 1), (12, 1, 64, 32, 1), (16, 1, 128, 256, 1),
    (8, 2, 64, 32, 5), (8, 2, 128, 32, 6), (4, 1, 64, 16, 8), (32, 1, 64, 64, 1), (32, 1, 128, 64, 1),
    (8, 8, 64, 16, 33), (28, 4, 128, 32, 20), (8, 8, 128, 128, 96), (2, 2, 64, 64, 300), (14, 2, 128, 16, 41)])
def test_attention(api, H_q, H_kv, d, page, n):
    news = [n, max(1, n - 1), 0, n, 1, n, (n + 1) // 2]
    lens = [n, 0, 5, 4 * page + 1, 1, 777, 130]
    B = len(news)
    box = Box(api, B, H_q, H_kv, d, page, max(lens) + 8, seed=n)
    # every set its own length, from none (a token that sees nothing) on
    box.fill([max(0, lens[s // H_kv] - (s % H_kv) * 3) for s in range(box.S)])
    q, got = box.attend(news)
    box.check(news, q, got)
    again = box.attend(news, q=q)[1]
    assert np.array_equal(got, again)


@pytest.mark.parametrize("n", [1, 3, 64])
def test_one_long_set_and_short_ones(api, n):
    box = Box(api, 5, 4, 1, 128, 64, 9000)
    total = [8900, 3, 64, 0, 2049]
    box.fill(total)
    q, got = box.attend([n, min(n, 3), n, 0, n])
    box.check([n, min(n, 3), n, 0, n], q, got)


def test_tokens_appended_then_attended_in_a_graph(api):
    """cache_write of new tokens, then their attention, captured and replayed."""
    B, H_q, H_kv, d, n, ln = 3, 8, 2, 128, 2, 50
    box = Box(api, B, H_q, H_kv, d, 16, ln + n)
    box.fill([ln + 2 * (s % 3) for s in range(box.S)])
    T = B * n
    qkv = dev_bf16(R.bf16_bits(box.rng.standard_normal((T, H_q + 2 * H_kv, d)))).view(T, -1, d)
    q, k, v = qkv.split([H_q, H_kv, H_kv], dim=1)
    off = torch.arange(0, T + 1, n, dtype=torch.int32, device="cuda")
    lens, grown = box.lens_t(box.lens), torch.empty(box.S, dtype=torch.int32, device="cuda")
    out = torch.empty(T, H_q, d, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        api.tgvkv_cache_write(box.desc, box.cache, box.table, lens, k, v, off, grown, box.ws)
        api.tgvkv_chunk_attention(box.desc, box.cache, box.table, grown, q, off, n, out, box.ws)
    for _ in range(2):
        out.fill_(float("nan"))
        graph.replay()
    assert api.tgvkv_status(box.ws) == 0
    kk, vv = (R.bf16_values(host_bits(t)).reshape(T, H_kv, d) for t in (k, v))
    for s in range(box.S):
        b, g = divmod(s, H_kv)
        box.k[s] = np.concatenate([box.k[s], F.round_trip(kk[b * n:(b + 1) * n, g])])
        box.v[s] = np.concatenate([box.v[s], F.round_trip(vv[b * n:(b + 1) * n, g])])
        box.lens[s] += n
    box.check([n] * B, R.bf16_values(host_bits(q)).reshape(T, H_q, d),
              R.bf16_values(host_bits(out)).reshape(T, H_q, d))
