"""GPU parity of the paged cache: quantising writes, reads, and attention of a
chunk of new tokens over it, through the C ABI, against the fp64 reference of
_cache_ref.py.

Tolerances.  Stored codes, scale bytes, lengths and rows read back are exact.
An attention output is a convex combination of value rows, computed with the
weights rounded to bf16 (relative error <= 2^-9) and rounded to bf16 itself
(<= 2^-9): |error| <= 2^-9 sum_j A_ij |v_j| + 2^-9 |o| <= 2^-8 sum_j A_ij |v_j|.
The bound tested is twice that, 2^-7 sum_j A_ij |v_jc|, plus 1e-6, leaving the
fp32 accumulation its room."""
import numpy as np
import pytest
import torch

import _cache_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "the GPU tests need a CUDA device"
    from paper_2606_03075_gb300 import build
    build.build()
    from paper_2606_03075_gb300 import api as _api
    return _api


def dev_bf16(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def host_bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class Box:
    """A paged cache with shuffled pages whose unused rows hold NaN patterns."""

    def __init__(self, api, B, H_q, H_kv, d, page, fmt, max_len, seed=0, spare=3, scale=0.0):
        rng = np.random.default_rng([seed, B, H_q, H_kv, d, page])
        self.api, self.fmt, self.page, self.d = api, fmt, page, d
        self.B, self.H_q, self.H_kv, self.S = B, H_q, H_kv, B * H_kv
        self.max_pages = max(1, -(-max_len // page)) + 1
        need = self.S * self.max_pages
        self.n_pages = need + spare
        self.scale = scale if scale > 0 else 1 / np.sqrt(d)
        self.desc = api.make_cache_desc(B, H_q, H_kv, d, page, self.n_pages, self.max_pages, fmt,
                                        softmax_scale=scale)
        self.cache = api.alloc_cache(self.desc)
        for name in ("k", "v", "k_scale", "v_scale"):
            t = getattr(self.cache, name)
            if t is not None:      # all ones: NaN in bf16, a NaN scale, code -1 / 7
                t.view(torch.uint8).fill_(255)
        self.table_np = rng.permutation(self.n_pages)[:need].reshape(self.S, -1).astype(np.int32)
        self.table = torch.from_numpy(self.table_np).cuda()
        self.ws = api.new_cache_workspace(self.desc)
        self.rng = rng

    def values(self, rows, keys=False):
        x = self.rng.standard_normal((rows, self.d)).astype(np.float32)
        if keys:
            x[:, self.rng.permutation(self.d)[:4]] *= 8
        return R.bf16_values(R.bf16_bits(x))

    def lens_t(self, lens):
        return torch.tensor(lens, dtype=torch.int32, device="cuda")

    def rows_of(self, s, lo, hi):
        j = np.arange(lo, hi)
        return self.table_np[s, j // self.page].astype(np.int64) * self.page + j % self.page

    def fill(self, total):
        """Fill every set's first total[s] slots through tgvkv_cache_write_rows;
        returns the fp64 values each set then holds."""
        off = np.concatenate([[0], np.cumsum(total)]).astype(np.int64)
        k, v = self.values(int(off[-1]), keys=True), self.values(int(off[-1]))
        out = torch.empty(self.S, dtype=torch.int32, device="cuda")
        self.api.tgvkv_cache_write_rows(
            self.desc, self.cache, self.table, self.lens_t([0] * self.S),
            dev_bf16(R.bf16_bits(k)).view(-1, self.d), dev_bf16(R.bf16_bits(v)).view(-1, self.d),
            torch.from_numpy(off).cuda(), out, self.ws)
        assert self.api.tgvkv_status(self.ws) == 0
        assert out.cpu().tolist() == list(total)
        kk, vv = R.round_trip(k, self.fmt), R.round_trip(v, self.fmt)
        self.k = [kk[off[s]:off[s + 1]] for s in range(self.S)]
        self.v = [vv[off[s]:off[s + 1]] for s in range(self.S)]
        self.lens = list(total)

    def attend(self, news, q=None, max_q=None, out=None):
        T = sum(news)
        off = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        if q is None:
            q = R.bf16_values(R.bf16_bits(self.rng.standard_normal((T, self.H_q, self.d))))
        qt = dev_bf16(R.bf16_bits(q)).view(T, self.H_q, self.d)
        if out is None:
            out = torch.full((T, self.H_q, self.d), float("nan"), dtype=torch.bfloat16,
                             device="cuda")
        self.api.tgvkv_chunk_attention(self.desc, self.cache, self.table, self.lens_t(self.lens), qt,
                                       torch.from_numpy(off).cuda(),
                                       max(news) if max_q is None else max_q, out, self.ws)
        assert self.api.tgvkv_status(self.ws) == 0
        return q, R.bf16_values(host_bits(out)).reshape(T, self.H_q, self.d)

    def check(self, news, q, got):
        G, t0 = self.H_q // self.H_kv, 0
        for b, n in enumerate(news):
            for g in range(self.H_kv):
                s = b * self.H_kv + g
                qs = q[t0:t0 + n, g * G:(g + 1) * G]
                ref = R.attention(qs, self.k[s], self.v[s], n, self.scale)
                mass = R.attention(qs, self.k[s], np.abs(self.v[s]), n, self.scale)
                o = got[t0:t0 + n, g * G:(g + 1) * G]
                bad = ~(np.abs(o - ref) <= 2.0 ** -7 * mass + 1e-6)
                assert not bad.any(), (b, g, np.argwhere(bad)[:3], o[bad][:3], ref[bad][:3])
            t0 += n


FORMATS = ["bf16", "int8", "int4"]
TIMEOUT = 0x20


# ---- writing and reading -------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 16), (128, 64), (64, 256)])
def test_write_rows_stores_the_format_and_reads_back(api, fmt, d, page):
    total = [0, 1, 15, 16, 17, 33, 0, 70, 129, 5, 64, 2]
    box = Box(api, 3, 8, 4, d, page, fmt, max(total))
    box.fill(total)
    # the stored bytes themselves, slot by slot; pages never written keep theirs
    pool = {n: getattr(box.cache, n) for n in ("k", "v", "k_scale", "v_scale")}
    touched = np.zeros(box.n_pages * page, bool)
    for s in range(box.S):
        rows = box.rows_of(s, 0, total[s])
        touched[rows] = True
        for n, ref in (("k", box.k[s]), ("v", box.v[s])):
            if fmt == "bf16":
                got = host_bits(pool[n]).reshape(-1, d)[rows]
                assert np.array_equal(got, R.bf16_bits(ref))
            else:
                codes, byte = R.encode(ref, fmt)
                st = pool[n].cpu().numpy().reshape(box.n_pages * page, -1)[rows]
                sb = pool[n + "_scale"].cpu().numpy().reshape(box.n_pages * page, -1)[rows]
                assert np.array_equal(R.decode(R.unpack(st, fmt), sb), ref)
    for n, t in pool.items():
        if t is not None:
            raw = t.view(torch.uint8).cpu().numpy().reshape(box.n_pages * page, -1)
            assert (raw[~touched] == 255).all(), n
    # read everything, then a slice from the middle of every set
    for first, count in (([0] * box.S, total),
                         ([t // 3 for t in total], [t - t // 3 - t // 5 for t in total])):
        off = np.concatenate([[0], np.cumsum(count)]).astype(np.int64)
        rows = int(off[-1])
        k = torch.zeros(rows + 2, d, dtype=torch.bfloat16, device="cuda")
        v = torch.zeros(rows + 2, d, dtype=torch.bfloat16, device="cuda")
        api.tgvkv_cache_read(box.desc, box.cache, box.table,
                             box.lens_t(first) if any(first) else None,
                             torch.from_numpy(off).cuda(), k, v, box.ws)
        assert api.tgvkv_status(box.ws) == 0
        for t, ref in ((k, box.k), (v, box.v)):
            want = np.concatenate([ref[s][first[s]:first[s] + count[s]] for s in range(box.S)])
            got = R.bf16_values(host_bits(t)).reshape(-1, d)
            assert np.array_equal(got[:rows], want)
            assert (got[rows:] == 0).all()         # rows past the offsets' end stay


def _codes(box, s, lo, hi, name):
    rows = box.rows_of(s, lo, hi)
    st = getattr(box.cache, name).cpu().numpy().reshape(box.n_pages * box.page, -1)[rows]
    sb = getattr(box.cache, name + "_scale").cpu().numpy().reshape(box.n_pages * box.page, -1)[rows]
    return R.unpack(st, box.fmt), sb


@pytest.mark.parametrize("fmt", ["int8", "int4"])
@pytest.mark.parametrize("d", [64, 128])
def test_quantisation_edges(api, fmt, d):
    """Code for code and byte for byte: groups at and around the scale's steps,
    ties, zeros, subnormals, the largest bf16, infinities and NaN."""
    rng = np.random.default_rng(5)
    top = R.bf16_values(np.uint16(0x7F7F))
    rows = []
    for m in (127, 126, 128, 254, 255, 7, 6, 6.9375, 7.0625, 8, 1, 0.0):   # group maxima
        for e in (-8, 0, 5):
            r = rng.uniform(-1, 1, d) * m * 2.0 ** e
            r[::GR] = m * 2.0 ** e * np.where(np.arange(len(r[::GR])) % 2, -1, 1)
            rows.append(r)
    rows.append((np.arange(d) % 17 - 8) * 0.5)                  # exact ties
    rows.append(np.arange(d) * 2.0 ** -133)                     # subnormal bf16
    rows.append(np.where(np.arange(d) % 3, 2.0 ** -126, -2.0 ** -125))
    rows.append(np.where(np.arange(d) % 5 == 0, top, 1.0))
    for bad in (np.inf, -np.inf, np.nan):
        r = rng.standard_normal(d)
        r[37 % d] = bad                                          # one group of the row only
        rows.append(r)
    rows.append(np.zeros(d))
    x = R.bf16_values(R.bf16_bits(np.array(rows)))
    n = x.shape[0]
    box = Box(api, 1, 2, 1, d, 16, fmt, n)
    out = torch.empty(1, dtype=torch.int32, device="cuda")
    bits = dev_bf16(R.bf16_bits(x))
    off = torch.tensor([0, n], dtype=torch.int64, device="cuda")
    api.tgvkv_cache_write_rows(box.desc, box.cache, box.table, box.lens_t([0]), bits, bits.flip(0),
                               off, out, box.ws)
    assert api.tgvkv_status(box.ws) == 0
    for name, ref in (("k", x), ("v", x[::-1])):
        codes, byte = R.encode(ref, fmt)
        got, gb = _codes(box, 0, 0, n, name)
        assert np.array_equal(gb, byte), name
        assert np.array_equal(got, codes), name
    k = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    api.tgvkv_cache_read(box.desc, box.cache, box.table, None, off, k, v, box.ws)
    want = R.round_trip(x, fmt)
    # the largest values may round up past bf16's range: then they read as infinity
    want = np.where(np.abs(want) >= 2.0 ** 128, np.sign(want) * np.inf, want)
    got = R.bf16_values(host_bits(k)).reshape(n, d)
    assert np.array_equal(got, want, equal_nan=True)


GR = 32


@pytest.mark.parametrize("fmt", FORMATS)
def test_write_tokens_strided_over_existing_lengths(api, fmt):
    """Chunks appended behind existing rows from slices of a fused projection:
    sequences without new tokens, pages crossed, every row in its place."""
    B, H_kv, d, page = 4, 3, 64, 16
    box = Box(api, B, 6, H_kv, d, page, fmt, 90)
    start = [int(x) for x in box.rng.integers(0, 40, B * H_kv)]
    box.fill(start)
    news = [5, 0, 33, 1]
    T = sum(news)
    fused = R.bf16_values(R.bf16_bits(box.rng.standard_normal((T, 2 * H_kv + 2, d))))
    ft = dev_bf16(R.bf16_bits(fused)).view(T, 2 * H_kv + 2, d)
    off = torch.tensor([0] + list(np.cumsum(news)), dtype=torch.int32, device="cuda")
    lens_out = torch.empty(box.S, dtype=torch.int32, device="cuda")
    # K with head stride d, V taken from every other head slot (stride 2 d) of its own tensor
    v2 = torch.zeros(T, 2 * H_kv, d, dtype=torch.bfloat16, device="cuda")
    v2[:, ::2] = ft[:, H_kv + 1:2 * H_kv + 1]
    api.tgvkv_cache_write(box.desc, box.cache, box.table, box.lens_t(start), ft[:, 1:H_kv + 1],
                          v2[:, ::2], off, lens_out, box.ws)
    assert api.tgvkv_status(box.ws) == 0
    total = [start[s] + news[s // H_kv] for s in range(box.S)]
    assert lens_out.cpu().tolist() == total
    offs = np.concatenate([[0], np.cumsum(total)]).astype(np.int64)
    k = torch.empty(int(offs[-1]), d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    api.tgvkv_cache_read(box.desc, box.cache, box.table, None, torch.from_numpy(offs).cuda(), k, v,
                         box.ws)
    kn, vn = R.bf16_values(host_bits(k)).reshape(-1, d), R.bf16_values(host_bits(v)).reshape(-1, d)
    t0 = 0
    for b, n in enumerate(news):
        for g in range(H_kv):
            s = b * H_kv + g
            got = kn[offs[s]:offs[s + 1]], vn[offs[s]:offs[s + 1]]
            assert np.array_equal(got[0][:start[s]], box.k[s])
            assert np.array_equal(got[0][start[s]:], R.round_trip(fused[t0:t0 + n, 1 + g], fmt))
            assert np.array_equal(got[1][start[s]:],
                                  R.round_trip(fused[t0:t0 + n, H_kv + 1 + g], fmt))
        t0 += n


def test_many_sets_search(api):
    """More sets than a CTA has threads, most of them empty."""
    S = 1500
    total = [0] * S
    for s in (0, 3, 255, 256, 700, 701, 1499):
        total[s] = 1 + s % 7
    box = Box(api, S // 4, 4, 4, 64, 16, "int8", 8)
    box.fill(total)
    off = np.concatenate([[0], np.cumsum(total)]).astype(np.int64)
    k = torch.empty(int(off[-1]), 64, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    api.tgvkv_cache_read(box.desc, box.cache, box.table, None, torch.from_numpy(off).cuda(), k, v,
                         box.ws)
    assert np.array_equal(R.bf16_values(host_bits(k)).reshape(-1, 64), np.concatenate(box.k))


# ---- attention -----------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H_q,H_kv,page", [(4, 4, 16), (7, 1, 64), (32, 2, 32), (6, 2, 256)])
def test_single_token(api, fmt, d, H_q, H_kv, page):
    """One token per sequence: lengths around tiles, chunks and pages, an empty set."""
    B = 6
    lens = [1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200, 0, 2, 257, 300, 48, 80, 5, 96, 128, 255,
            8, 70][:B * H_kv]
    box = Box(api, B, H_q, H_kv, d, page, fmt, max(lens))
    box.fill(lens)
    q, got = box.attend([1] * B)
    box.check([1] * B, q, got)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_drafted_tokens_and_idle_sequences(api, fmt, d):
    """A few tokens a sequence (at most 16 query rows a set), some sequences idle,
    some with fewer slots than tokens (their first tokens see nothing)."""
    news = [3, 0, 4, 1, 2, 4]
    box = Box(api, 6, 8, 2, d, 32, fmt, 310)
    lens = [40, 3, 10, 0, 2, 4, 300, 1, 2, 1, 310, 3]
    box.fill(lens)
    q, got = box.attend(news)
    box.check(news, q, got)
    t = 3 + 4                                   # sequence 3: one token; sequence 4 follows
    assert (got[t + 1, 4:] == 0).all()          # set 9 holds 1 slot, its first of 2 tokens sees none
    q2, again = box.attend(news, q=q)
    assert np.array_equal(got, again)           # the same bits on every call


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H_q,H_kv,page", [(2, 2, 16), (7, 1, 128), (8, 2, 64)])
def test_chunks(api, fmt, d, H_q, H_kv, page):
    """Chunks of up to a few hundred tokens beside short ones: several row tiles,
    ragged last tiles, chunks that are the whole cache, and sets shorter than their chunk."""
    news = [1, 150, 0, 37, 261]
    base = [90, 0, 11, 300, 140]
    box = Box(api, 5, H_q, H_kv, d, page, fmt, 420)
    lens = [base[b] + news[b] + 3 * g for b in range(5) for g in range(H_kv)]
    lens[3 * H_kv] = 20                          # fewer slots than its 37 tokens
    box.fill(lens)
    q, got = box.attend(news)
    box.check(news, q, got)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,longest", [(2, 300), (6, 1500)])
def test_one_row_tile_per_set(api, fmt, d, B, longest):
    """Chunks of one row tile (more than 16 query rows): a few key tiles in all, so
    that a CTA gets one or none, then shares of several sets, parts of sets and
    single tiles in one CTA."""
    H = 16
    box = Box(api, B, H, H, d, 64, fmt, longest)
    lens = [1 + (s * 7919) % longest for s in range(B * H)]
    box.fill(lens)
    news = [(96, 17, 128, 1, 40, 0)[b % 6] for b in range(B)]
    for _ in range(3):                           # back to back, no wait in between
        q, got = box.attend(news)
    box.check(news, q, got)


@pytest.mark.parametrize("fmt", FORMATS)
def test_long_sets_split_over_the_whole_gpu(api, fmt):
    """Few sets, long caches: every set is split over many streams and joined."""
    box = Box(api, 1, 4, 2, 128, 64, fmt, 9001)
    box.fill([9001, 4444])
    for news in ([1], [4], [70]):
        q, got = box.attend(news)
        box.check(news, q, got)


def test_more_sets_than_the_plan_holds(api):
    """4100 sets (several per plan entry), ragged, with empty ones."""
    S = 4100
    box = Box(api, S // 2, 2, 2, 64, 16, "int8", 40)
    lens = [(s * 7) % 41 for s in range(S)]
    box.fill(lens)
    for news in ([(b * 3) % 3 for b in range(S // 2)], [b % 3 for b in range(S // 2)]):
        q, got = box.attend(news)                # no token at all, then 0, 1 or 2 each
        box.check(news, q, got)


@pytest.mark.parametrize("fmt", FORMATS)
def test_large_logits_and_scale(api, fmt):
    """Saturated softmax rows (logits of a thousand) and a given softmax scale."""
    box = Box(api, 2, 4, 2, 64, 16, fmt, 150, scale=3.0)
    lens = [150, 33, 64, 149]
    box.fill(lens)
    for news in ([2, 3], [40, 33]):
        q, got = box.attend(news)
        # logits this far apart make the weights one-hot or ties; the bound holds as it is,
        # but the fp32 logits' own error (2^-22 of 1000) moves a weight by 1e-3 at most
        G, t0 = 2, 0
        for b, n in enumerate(news):
            for g in range(2):
                s = b * 2 + g
                qs = q[t0:t0 + n, g * G:(g + 1) * G]
                ref = R.attention(qs, box.k[s], box.v[s], n, 3.0)
                mass = R.attention(qs, box.k[s], np.abs(box.v[s]), n, 3.0)
                o = got[t0:t0 + n, g * G:(g + 1) * G]
                assert (np.abs(o - ref) <= (2.0 ** -7 + 4e-3) * mass + 1e-6).all()
            t0 += n


def test_strided_queries_and_a_shared_prefix(api):
    """Queries sliced out of a fused projection; two sequences whose tables share
    their first pages."""
    H_q, H_kv, d, page = 8, 2, 128, 16
    box = Box(api, 2, H_q, H_kv, d, page, "bf16", 80)
    box.fill([80, 80, 80, 80])
    for g in range(H_kv):                        # sequence 1 takes over sequence 0's 3 first pages
        box.table_np[H_kv + g, :3] = box.table_np[g, :3]
        box.k[H_kv + g][:48], box.v[H_kv + g][:48] = box.k[g][:48], box.v[g][:48]
    box.table = torch.from_numpy(box.table_np).cuda()
    for news in ([1, 1], [20, 31]):
        T = sum(news)
        fused = R.bf16_values(R.bf16_bits(box.rng.standard_normal((T, H_q + 5, d))))
        ft = dev_bf16(R.bf16_bits(fused)).view(T, H_q + 5, d)
        out = torch.empty(T, H_q, d, dtype=torch.bfloat16, device="cuda")
        off = torch.tensor([0, news[0], T], dtype=torch.int32, device="cuda")
        api.tgvkv_chunk_attention(box.desc, box.cache, box.table, box.lens_t(box.lens),
                                  ft[:, 3:3 + H_q], off, max(news), out, box.ws)
        assert api.tgvkv_status(box.ws) == 0
        got = R.bf16_values(host_bits(out)).reshape(T, H_q, d)
        box.check(news, fused[:, 3:3 + H_q], got)


def test_device_faults_set_the_status_and_touch_nothing(api):
    INDEX = 0x08
    box = Box(api, 2, 4, 2, 64, 16, "bf16", 40)
    box.fill([20, 30, 10, 40])
    q = torch.randn(4, 4, 64, device="cuda").bfloat16()
    out = torch.zeros(4, 4, 64, dtype=torch.bfloat16, device="cuda")
    good = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")

    def attend(lens=(20, 30, 10, 40), off=good, max_q=2, table=None):
        api.tgvkv_chunk_attention(box.desc, box.cache, box.table if table is None else table,
                                  box.lens_t(list(lens)), q, off, max_q, out, box.ws)
        return api.tgvkv_status(box.ws)

    cap = box.max_pages * box.page
    assert attend() == 0
    assert attend(lens=(20, 30, -1, 40)) == INDEX
    assert attend(lens=(20, cap + 1, 10, 40)) & INDEX
    assert attend(off=torch.tensor([0, 3, 2], dtype=torch.int32, device="cuda")) == INDEX
    assert attend(off=torch.tensor([0, 2, 9], dtype=torch.int32, device="cuda")) == INDEX
    assert attend(max_q=1) == INDEX
    bad = box.table.clone()
    bad[1, 0] = box.n_pages
    assert attend(table=bad) == INDEX
    bad[1, 0] = -5
    assert attend(table=bad) == INDEX
    assert attend() == 0
    # writes: a set that would grow past its pages, bad pages, bad offsets
    before = box.cache.k.clone()
    k = torch.ones(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    lens_out = torch.empty(4, dtype=torch.int32, device="cuda")

    def write(lens, off=good, table=None):
        api.tgvkv_cache_write(box.desc, box.cache, box.table if table is None else table,
                              box.lens_t(lens), k, k, off, lens_out, box.ws)
        return api.tgvkv_status(box.ws)

    assert write([cap, cap, cap, cap]) == INDEX
    assert lens_out.cpu().tolist() == [cap] * 4
    none = torch.full_like(box.table, -1)
    assert write([0, 0, 0, 0], table=none) == INDEX
    assert write([0] * 4, off=torch.tensor([0, 0, 0], dtype=torch.int32, device="cuda")) == 0
    assert torch.equal(before.view(torch.int16), box.cache.k.view(torch.int16))
    assert write([0] * 4, off=torch.tensor([0, 9, 9], dtype=torch.int32, device="cuda")) == INDEX
    o = torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([0, 2, 4, 6, 8], dtype=torch.int64, device="cuda")
    api.tgvkv_cache_read(box.desc, box.cache, none, None, off, o, o.clone(), box.ws)
    assert api.tgvkv_status(box.ws) == INDEX and (o == 0).all()


def test_another_stream_and_graph_replay(api):
    """The calls run on the stream they are given, and a captured decode step
    (write, then attention) replays."""
    B, H_q, H_kv, d = 3, 4, 2, 128
    box = Box(api, B, H_q, H_kv, d, 16, "int8", 100)
    box.fill([50, 60, 17, 80, 31, 64])
    lens = box.lens_t(box.lens)
    lens2 = torch.empty_like(lens)
    off = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    kv = [R.bf16_values(R.bf16_bits(box.rng.standard_normal((B, H_kv, d)))) for _ in range(2)]
    kt, vt = (dev_bf16(R.bf16_bits(x)).view(B, H_kv, d) for x in kv)
    q = R.bf16_values(R.bf16_bits(box.rng.standard_normal((B, H_q, d))))
    qt = dev_bf16(R.bf16_bits(q)).view(B, H_q, d)
    out = torch.empty(B, H_q, d, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()

    def step(stream):
        api.tgvkv_cache_write(box.desc, box.cache, box.table, lens, kt, vt, off, lens2, box.ws,
                              stream=stream)
        api.tgvkv_chunk_attention(box.desc, box.cache, box.table, lens2, qt, off, 1, out, box.ws,
                                  stream=stream)

    step(st)
    st.synchronize()
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(None)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert api.tgvkv_status(box.ws) == 0
    assert torch.equal(out.view(torch.int16), first.view(torch.int16))
    for s in range(box.S):
        b, g = divmod(s, H_kv)
        box.k[s] = np.concatenate([box.k[s], R.round_trip(kv[0][b:b + 1, g], "int8")])
        box.v[s] = np.concatenate([box.v[s], R.round_trip(kv[1][b:b + 1, g], "int8")])
    box.check([1] * B, q, R.bf16_values(host_bits(out)).reshape(B, H_q, d))


def test_a_workspace_that_was_not_initialised_is_reported(api):
    """Counters that are not at zero give no CTA a share: nothing is read or written out
    of range, the status says so, and an initialisation makes the workspace good."""
    box = Box(api, 3, 8, 2, 128, 32, "int8", 400)
    box.fill([300, 250, 400, 90, 200, 333])
    news = [40, 40, 40]
    q = torch.randn(120, 8, 128, device="cuda").bfloat16()
    off = torch.tensor([0, 40, 80, 120], dtype=torch.int32, device="cuda")
    out = torch.zeros(120, 8, 128, dtype=torch.bfloat16, device="cuda")
    box.ws.fill_(0x7F)
    box.ws[:4] = 0
    api.tgvkv_chunk_attention(box.desc, box.cache, box.table, box.lens_t(box.lens), q, off, 40, out,
                              box.ws)
    assert api.tgvkv_status(box.ws) == TIMEOUT
    assert (out == 0).all()
    api.tgvkv_cache_workspace_init(box.desc, box.ws)
    q, got = box.attend(news)
    box.check(news, q, got)


@pytest.mark.parametrize("fmt,page_bytes", [("bf16", 65536), ("int8", 32768), ("int4", 16384)])
def test_pools_past_32_bits(api, fmt, page_bytes):
    """Pages on either side of byte 2^32 (and element 2^31) of a pool."""
    d, page = 128, 256
    edge = 2 ** 32 // page_bytes
    box = Box(api, 2, 16, 2, d, page, fmt, 700, spare=edge + 16)
    far = np.arange(box.S * box.max_pages).reshape(box.S, -1)
    box.table_np = np.where(far % 3 == 0, far, edge + far).astype(np.int32)
    box.table = torch.from_numpy(box.table_np).cuda()
    box.fill([700, 300, 513, 256])
    for news in ([1, 1], [2, 0], [30, 41]):
        q, got = box.attend(news)
        box.check(news, q, got)
    off = torch.tensor([0, 700, 1000, 1513, 1769], dtype=torch.int64, device="cuda")
    k, v = (torch.empty(1769, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    api.tgvkv_cache_read(box.desc, box.cache, box.table, None, off, k, v, box.ws)
    assert api.tgvkv_status(box.ws) == 0
    assert np.array_equal(R.bf16_values(host_bits(k)), np.concatenate(box.k).astype(np.float32))
    assert np.array_equal(R.bf16_values(host_bits(v)), np.concatenate(box.v).astype(np.float32))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H_q,H_kv,most", [(8, 2, 6), (8, 2, 8), (7, 1, 3), (2, 2, 17), (2, 2, 25), (2, 2, 33),
                                           (16, 1, 2), (12, 1, 2)])
def test_a_few_tokens_of_17_to_33_rows(api, fmt, d, H_q, H_kv, most):
    """Around the largest calls of the kernel for few rows: ragged tokens, idle
    sequences, sets shorter than their tokens, and sets split over many streams."""
    news = [most, 0, 1, most - 1, most, 2]
    box = Box(api, 6, H_q, H_kv, d, 16, fmt, 3000)
    lens = [1700, most - 1, 1, 65, most // 2, 3000, 90, 0, 128, 400, most, 2][:6 * H_kv]
    box.fill(lens)
    q, got = box.attend(news)
    box.check(news, q, got)
    q2, again = box.attend(news, q=q)
    assert np.array_equal(got, again)


@pytest.mark.parametrize("fmt,n", [("bf16", 1), ("int8", 1), ("int4", 9), ("int8", 40)])
def test_steps_in_a_row_see_what_the_step_before_wrote(api, fmt, n):
    """Writes, attention and reads queued without a pause: the kernels may start
    before the ones ahead of them have finished, and wait for what they read."""
    B, H_q, H_kv, d, steps = 4, 8, 2, 64, 24
    box = Box(api, B, H_q, H_kv, d, 16, fmt, 40 + n * steps)
    box.fill([5, 17, 0, 33, 40, 12, 1, 8])
    off = torch.arange(0, B * n + 1, n, dtype=torch.int32, device="cuda")
    lens, grown = box.lens_t(box.lens), box.lens_t(box.lens)
    kv = [[box.values(B * n * H_kv, keys=i == 0).reshape(B * n, H_kv, d) for i in (0, 1)]
          for _ in range(steps)]
    qs = [R.bf16_values(R.bf16_bits(box.rng.standard_normal((B * n, H_q, d)))) for _ in range(steps)]
    kv_t = [[dev_bf16(R.bf16_bits(x)).view(B * n, H_kv, d) for x in pair] for pair in kv]
    qs_t = [dev_bf16(R.bf16_bits(q)).view(B * n, H_q, d) for q in qs]
    outs = [torch.empty(B * n, H_q, d, dtype=torch.bfloat16, device="cuda") for _ in range(steps)]
    back = [torch.empty(B * H_kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rows = torch.arange(B * H_kv + 1, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    for i in range(steps):
        api.tgvkv_cache_write(box.desc, box.cache, box.table, lens, *kv_t[i], off, grown, box.ws)
        api.tgvkv_chunk_attention(box.desc, box.cache, box.table, grown, qs_t[i], off, n, outs[i], box.ws)
        lens, grown = grown, lens
    api.tgvkv_cache_read(box.desc, box.cache, box.table, lens - 1, rows, *back, box.ws)
    assert api.tgvkv_status(box.ws) == 0
    for i in range(steps):
        for s in range(B * H_kv):
            b, g = divmod(s, H_kv)
            new = [R.round_trip(x[b * n:(b + 1) * n, g], fmt) for x in kv[i]]
            box.k[s], box.v[s] = np.concatenate([box.k[s], new[0]]), np.concatenate([box.v[s], new[1]])
        box.check([n] * B, qs[i], R.bf16_values(host_bits(outs[i])).reshape(B * n, H_q, d))
    for t, held in zip(back, (box.k, box.v)):
        assert np.array_equal(R.bf16_values(host_bits(t)), np.stack([x[-1] for x in held]).astype(np.float32))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [200, 513, 1100, 2200, 9000])
def test_few_rows_for_short_and_long_page_tables(api, fmt, d, cap):
    """The same small sets under page tables of several sizes (short ones have a kernel
    that takes a set a CTA), a full set, empty ones, and sets at chunk boundaries."""
    box = Box(api, 8, 8, 2, d, 64, fmt, cap)
    lens = [box.max_pages * box.page, 64, 65, 0, 1, 127, 128, 129, 16, 15, 0, 3, min(cap, 511), 200, 33, 2]
    box.fill(lens)
    for news in ([1] * 8, [2, 0, 1, 2, 1, 2, 1, 1], [4, 3, 0, 4, 1, 4, 2, 3]):
        q, got = box.attend(news)
        box.check(news, q, got)
        assert np.array_equal(got, box.attend(news, q=q)[1])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H_q,H_kv,most", [(8, 8, 96), (8, 8, 130), (16, 8, 40)])
def test_many_sets_that_each_span_several_ctas(api, fmt, H_q, H_kv, most):
    """Sets whose parts lie in four CTAs or more, with many rows in all: the second
    kernel joins several rows a CTA."""
    box = Box(api, 4, H_q, H_kv, 64, 64, fmt, 4100)
    box.fill([4100 - 37 * s for s in range(4 * H_kv)])
    for news in ([most] * 4, [most, 0, most - 1, 33]):
        q, got = box.attend(news)
        box.check(news, q, got)
        assert np.array_equal(got, box.attend(news, q=q)[1])
