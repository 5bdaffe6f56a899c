"""GPU tests of tgvkv_rope_write (queries turned, keys turned and stored, values stored) and
of a serving step's calls together: pages, turned keys into them, attention over them."""
import numpy as np
import pytest
import torch

import _cache_ref as R
import _fp4_ref
import _rope_ref as F

pytestmark = pytest.mark.gpu
INDEX = 0x08
FORMATS = ["bf16", "int8", "int4", "fp4"]


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "the GPU tests need a CUDA device"
    from paper_2606_03075_gb300 import build
    build.build()
    from paper_2606_03075_gb300 import api as _api
    return _api


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def host_bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def pools_of(cache):
    return [t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]


def step(api, fmt, d, H_q, H_kv, news, lens, page=16, pad=0, seed=0):
    """A cache whose pages are filled with 0xFF, the slots of new tokens, and the tokens."""
    B, T = len(news), int(sum(news)) + pad
    gen = torch.Generator("cuda").manual_seed(seed)
    max_pages = -(-(max(lens) + max(news) + 1) // page)
    desc = api.make_cache_desc(B, H_q, H_kv, d, page, B * H_kv * max_pages + 2, max_pages, fmt)
    cache, ws = api.alloc_cache(desc), api.new_cache_workspace(desc)
    for t in pools_of(cache):
        t.view(torch.uint8).fill_(255)
    order = torch.randperm(desc.n_pages, generator=gen, device="cuda")[:B * H_kv * max_pages]
    table = order.to(torch.int32).view(B * H_kv, max_pages)
    off = ints(np.concatenate([[0], np.cumsum(news)]))
    ln = ints(np.repeat(lens, H_kv))
    slots = torch.empty((T, H_kv), dtype=torch.int32, device="cuda")
    api.tgvkv_page_slots(desc, table, ln, off, slots, ws)
    assert api.tgvkv_status(ws) == 0
    qkv = torch.randn((T, H_q + 2 * H_kv, d), generator=gen, device="cuda")
    qkv[:, H_q:H_q + H_kv, 1:4] *= 8
    return desc, cache, ws, table, ln, off, slots, qkv.bfloat16()


CASES = [(128, 128, "half"), (128, 128, "interleaved"), (64, 64, "half"), (128, 64, "half"), (64, 32, "interleaved"),
         (128, 96, "half"), (128, 32, "half"), (64, 20, "half"), (128, 12, "interleaved"), (64, 62, "half"),
         (128, 2, "half")]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,rot,layout", CASES)
@pytest.mark.parametrize("H_q,H_kv,news", [(8, 2, [5, 0, 33]), (7, 7, [1]), (28, 4, [64, 1, 300])])
def test_the_same_as_turning_then_writing(api, fmt, d, rot, layout, H_q, H_kv, news):
    desc, cache, ws, table, ln, off, slots, qkv = step(api, fmt, d, H_q, H_kv, news, [3 + 17 * b for b in range(len(news))])
    q, k, v = qkv.split([H_q, H_kv, H_kv], dim=1)
    T = qkv.shape[0]
    pos = ints(np.random.default_rng(rot).integers(0, 50000, (3, T)))
    third = rot // 2 // 3
    plan = api.make_rope(d, rot_dim=rot, layout=layout, sections=[rot // 2 - 2 * third, third, third],
                         attention=1.25)
    qo, ko = torch.empty_like(q.contiguous()), torch.empty_like(k.contiguous())
    api.tgvkv_rope(plan, pos, q, qo, k, ko)
    grown = torch.empty_like(ln)
    api.tgvkv_cache_write(desc, cache, table, ln, ko, v, off, grown, ws)
    want = [t.clone() for t in pools_of(cache)]
    for t in pools_of(cache):
        t.view(torch.uint8).fill_(255)
    got = torch.full((T, 2 * H_q, d), 7.0, dtype=torch.bfloat16, device="cuda")
    api.tgvkv_rope_write(desc, cache, plan, pos, slots, q, k, v, got[:, ::2], ws)
    assert api.tgvkv_status(ws) == 0
    assert torch.equal(got[:, ::2].view(torch.int16), qo.view(torch.int16)) and (got[:, 1::2] == 7).all()
    for a, b in zip(pools_of(cache), want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # keys and values alone; then queries in place
    for t in pools_of(cache):
        t.view(torch.uint8).fill_(255)
    api.tgvkv_rope_write(desc, cache, plan, pos, slots, None, k, v, None, ws)
    for a, b in zip(pools_of(cache), want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    own = qkv.clone()
    q, k, v = own.split([H_q, H_kv, H_kv], dim=1)
    api.tgvkv_rope_write(desc, cache, plan, pos, slots, q, k, v, q, ws)
    assert torch.equal(q.contiguous().view(torch.int16), qo.view(torch.int16))
    assert torch.equal(own[:, H_q:], qkv[:, H_q:]) and api.tgvkv_status(ws) == 0


@pytest.mark.parametrize("fmt", FORMATS)
def test_padding_and_slots_past_the_pool(api, fmt):
    """Negative slots go nowhere; those past the pool are reported; the others are stored."""
    desc, cache, ws, table, ln, off, slots, qkv = step(api, fmt, 128, 8, 2, [20, 9], [0, 40], pad=7)
    q, k, v = qkv.split([8, 2, 2], dim=1)
    assert (slots[29:] == -1).all()
    pos, plan = ints(np.arange(36)), api.make_rope(128)
    qo = torch.empty((36, 8, 128), dtype=torch.bfloat16, device="cuda")
    api.tgvkv_rope_write(desc, cache, plan, pos, slots, q, k, v, qo, ws)
    assert api.tgvkv_status(ws) == 0
    rows = desc.n_pages * desc.page_size
    touched = torch.zeros(rows, dtype=torch.bool, device="cuda")
    touched[slots[:29].flatten().long()] = True
    want = [t.clone().view(torch.uint8).view(rows, -1) for t in pools_of(cache)]
    for w in want:
        assert (w[~touched] == 255).all()
    bad = slots.clone()
    bad[3, 1], bad[7, 0], bad[20, 0], bad[21, 1] = rows, 2 ** 31 - 1, -(2 ** 31), -7
    for t in pools_of(cache):
        t.view(torch.uint8).fill_(255)
    api.tgvkv_rope_write(desc, cache, plan, pos, bad, q, k, v, qo, ws)
    assert api.tgvkv_status(ws) == INDEX
    for s in (slots[3, 1], slots[7, 0], slots[20, 0], slots[21, 1]):
        touched[s.long()] = False
    for t, w in zip(pools_of(cache), want):
        got = t.view(torch.uint8).view(rows, -1)
        assert torch.equal(got[touched], w[touched]) and (got[~touched] == 255).all()


def test_keys_against_the_reference(api):
    """bf16 pages against the definition in 64 bits (tolerance of test_rope_gpu.py)."""
    desc, cache, ws, table, ln, off, slots, qkv = step(api, "bf16", 64, 4, 2, [9, 30], [5, 0])
    q, k, v = qkv.split([4, 2, 2], dim=1)
    pos = np.random.default_rng(0).integers(0, 100000, (1, 39))
    o = dict(scaling="parts", factor=4.0, original=2048)
    qo = torch.empty((39, 4, 64), dtype=torch.bfloat16, device="cuda")
    api.tgvkv_rope_write(desc, cache, api.make_rope(64, rot_dim=48, **o), ints(pos), slots, q, k, v, qo, ws)
    f = F.frequencies(48, **o)
    at = slots.long()
    for got, x in ((qo, q), (cache.k.view(-1, 64)[at], k)):
        got, x = (R.bf16_values(host_bits(t)) for t in (got, x))
        ref = F.turned(x, pos, f, 48)
        room = (2.0 ** -21 + 2.0 ** -50 * pos.max()) * F.partner_magnitude(x, 48)
        assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + room).all()
    assert torch.equal(cache.v.view(-1, 64)[at], v)


@pytest.mark.parametrize("fmt", ["bf16", "int8", "fp4"])
@pytest.mark.parametrize("H_q,H_kv,d,rot,T", [(8, 1, 64, 64, 5000), (1, 1, 128, 128, 3001), (33, 3, 64, 20, 2500),
                                             (28, 4, 128, 128, 9000), (130, 2, 128, 64, 700)])
def test_long_prompts_the_same_as_turning_then_writing(api, fmt, H_q, H_kv, d, rot, T):
    """CTAs of many tiles of every tensor, queries in place."""
    desc, cache, ws, table, ln, off, slots, qkv = step(api, fmt, d, H_q, H_kv, [T // 3, 2 * T // 3 + 1], [100, 7], page=64)
    q, k, v = qkv.split([H_q, H_kv, H_kv], dim=1)
    pos, plan = torch.arange(qkv.shape[0], dtype=torch.int32, device="cuda"), api.make_rope(d, rot_dim=rot)
    qo, ko = torch.empty_like(q.contiguous()), torch.empty_like(k.contiguous())
    api.tgvkv_rope(plan, pos, q, qo, k, ko)
    api.tgvkv_cache_write(desc, cache, table, ln, ko, v, off, torch.empty_like(ln), ws)
    want = [t.clone() for t in pools_of(cache)]
    for t in pools_of(cache):
        t.view(torch.uint8).fill_(255)
    api.tgvkv_rope_write(desc, cache, plan, pos, slots, q, k, v, q, ws)
    assert api.tgvkv_status(ws) == 0
    assert torch.equal(q.contiguous().view(torch.int16), qo.view(torch.int16))
    for a, b in zip(pools_of(cache), want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_no_tokens(api):
    desc, cache, ws, table, ln, off, slots, qkv = step(api, "int8", 64, 4, 2, [3], [0])
    none = qkv[:0]
    api.tgvkv_rope_write(desc, cache, api.make_rope(64), ints([]), slots[:0], none[:, :4], none[:, 4:6],
                         none[:, 6:], none[:, :4], ws)
    assert api.tgvkv_status(ws) == 0
    assert all((t.view(torch.uint8) == 255).all() for t in pools_of(cache))


# ---- a serving step's calls together ------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H_q,H_kv,d,page", [(8, 2, 128, 16), (4, 4, 64, 32)])
def test_serving_steps(api, fmt, H_q, H_kv, d, page):
    """Prompts of three requests, decode steps replayed from a graph, one request ended and
    another admitted in its pages: pages, turned tokens into them, attention over them.
    The attention's tolerance is 2^-7 sum_j A_ij |v_j| + 1e-6 (weights and output in bf16,
    2^-8 each) for the stored rows, which are read back and compared with the reference
    before (a turned key lies within the fp32 arithmetic of the exact one, test_rope_gpu.py;
    next to a border of the rounding it may fall on either side)."""
    B, L = 3, 90
    max_pages = -(-L // page)
    desc = api.make_cache_desc(B, H_q, H_kv, d, page, 2 * H_kv * max_pages + 4, max_pages, fmt)
    cache, pages, ws = api.alloc_cache(desc), api.alloc_pages(desc), api.new_cache_workspace(desc)
    for t in pools_of(cache):
        t.view(torch.uint8).fill_(255)
    plan = api.make_rope(d, base=1e5)
    gen = torch.Generator("cuda").manual_seed(d)
    lens, grown = ints(np.zeros(B * H_kv)), ints(np.zeros(B * H_kv))
    turned = [[] for _ in range(B)]        # reference: every sequence's turned keys and values
    stored = {"bf16": lambda x: x, "fp4": _fp4_ref.round_trip}.get(fmt, lambda x: R.round_trip(x, fmt))

    def tokens(T):
        x = torch.randn((T, H_q + 2 * H_kv, d), generator=gen, device="cuda").bfloat16()
        return x.split([H_q, H_kv, H_kv], dim=1)

    def run(q, k, v, pos, off, max_q, qt, slots, out):
        api.tgvkv_pages_append(desc, pages, lens, off, slots, grown, ws)
        api.tgvkv_rope_write(desc, cache, plan, pos, slots, q, k, v, qt, ws)
        api.tgvkv_chunk_attention(desc, cache, pages.page_table, grown, qt, off, max_q, out, ws)
        lens.copy_(grown)

    def note(news, first, k, v):
        t = 0
        for b, n in enumerate(news):
            kk, vv = (R.bf16_values(host_bits(x[t:t + n])).reshape(n, H_kv, d) for x in (k, v))
            pos = np.arange(first[b], first[b] + n)[None]
            turned[b] += list(zip(F.turned(kk, pos, F.frequencies(d, base=1e5), d), vv,
                                  2.0 ** -21 * F.partner_magnitude(kk, d)))
            t += n

    def check(news, qt, out):
        assert api.tgvkv_status(ws) == 0
        total = lens.cpu().numpy().astype(np.int64)
        off = torch.tensor(np.concatenate([[0], np.cumsum(total)]), device="cuda")
        rows = [torch.empty((int(off[-1]), d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        api.tgvkv_cache_read(desc, cache, pages.page_table, None, off, *rows, ws)
        kr, vr = (R.bf16_values(host_bits(x)) for x in rows)
        o = R.bf16_values(host_bits(out)).reshape(-1, H_q, d)
        qv = R.bf16_values(host_bits(qt)).reshape(-1, H_q, d)
        G, t, seen = H_q // H_kv, 0, []
        for b, n in enumerate(news):
            for g in range(H_kv):
                s = b * H_kv + g
                lo, hi = int(off[s]), int(off[s + 1])
                assert hi - lo == len(turned[b])
                if hi > lo:
                    want_v = stored(np.array([x[1][g] for x in turned[b]]))
                    assert np.array_equal(vr[lo:hi], want_v)
                    exact, room = (np.array([x[i][g] for x in turned[b]]) for i in (0, 2))
                    # the turned value lies within `room` of the exact one, and rounding to bf16
                    # is monotone: where both ends round alike, the stored group is known
                    ends = [R.bf16_values(R.bf16_bits(exact + sign * room)) for sign in (-1, 1)]
                    known = (ends[0] == ends[1]).reshape(hi - lo, -1, 32).all(-1).repeat(32, -1)
                    seen.append(known.flatten())
                    assert np.array_equal(kr[lo:hi][known], stored(ends[0])[known])
                    if fmt == "bf16":
                        assert ((kr[lo:hi] >= ends[0]) & (kr[lo:hi] <= ends[1])).all()
                qs = qv[t:t + n, g * G:(g + 1) * G]
                ref = R.attention(qs, kr[lo:hi], vr[lo:hi], n, 1 / np.sqrt(d))
                mass = R.attention(qs, kr[lo:hi], np.abs(vr[lo:hi]), n, 1 / np.sqrt(d))
                got = o[t:t + n, g * G:(g + 1) * G]
                assert (np.abs(got - ref) <= 2.0 ** -7 * mass + 1e-6).all(), (b, g)
            t += n
        assert np.concatenate(seen).mean() > 0.8      # borders are rare: most groups are known

    def prompts(news, first):
        T = sum(news)
        q, k, v = tokens(T)
        off = ints(np.concatenate([[0], np.cumsum(news)]))
        pos = ints(np.concatenate([np.arange(f, f + n) for f, n in zip(first, news)]))
        qt, out = torch.empty((T, H_q, d), dtype=torch.bfloat16, device="cuda"), torch.empty((T, H_q, d), dtype=torch.bfloat16, device="cuda")
        run(q, k, v, pos, off, max(news), qt, torch.empty((T, H_kv), dtype=torch.int32, device="cuda"), out)
        note(news, first, k, v)
        check(news, qt, out)

    prompts([40, 1, 17], [0, 1000, 5])
    # a decode step, captured: new tokens and positions are written into its inputs
    q, k, v = (x.contiguous() for x in tokens(B))
    pos, off = ints([40, 1001, 22]), ints([0, 1, 2, 3])
    qt, out = torch.empty_like(q), torch.empty_like(q)
    slots = torch.empty((B, H_kv), dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        run(q, k, v, pos, off, 1, qt, slots, out)
        pos += 1
    first = [40, 1001, 22]
    for i in range(20):
        for dst, src in zip((q, k, v), tokens(B)):
            dst.copy_(src)
        note([1] * B, [f + i for f in first], k, v)
        graph.replay()
        if i % 7 == 0 or i == 19:
            check([1] * B, qt, out)
    # the first request ends, another takes its place
    end = lens.clone()
    end[:H_kv] = 0
    api.tgvkv_pages_shrink(desc, pages, lens, end, ws)
    lens.copy_(end)
    turned[0] = []
    prompts([25, 0, 2], [0, 0, 42])
    held = (lens + page - 1) // page
    assert int(pages.n_free) == desc.n_pages - int(held.sum())
    used = pages.page_table[pages.page_table >= 0].cpu().tolist() + pages.free[:int(pages.n_free)].cpu().tolist()
    assert sorted(used) == list(range(desc.n_pages))
