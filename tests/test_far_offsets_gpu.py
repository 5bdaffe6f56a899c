"""Rows that lie beyond 2^31 elements or 2^32 bytes, for the rotary calls and the paged cache
in every format, compared bit for bit with the same rows near the start; infinities and NaN
that stay in their pair; one workspace shared by graphs that follow one another."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "the GPU tests need a CUDA device"
    from paper_2606_03075_gb300 import build
    build.build()
    from paper_2606_03075_gb300 import api as _api
    return _api


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of free device memory")
    yield
    torch.cuda.empty_cache()


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("heads", [1, 3])
def test_tokens_far_apart(api, heads):
    """Three tokens 2^31 elements from one another, in place and into another tensor."""
    d, far = 128, 2 ** 31
    x = torch.randn((3, heads, d), device="cuda").bfloat16()
    plan, pos, want = api.make_rope(d), ints([5, 77, 30000]), torch.empty_like(x)
    api.tgvkv_rope(plan, pos, x, want)
    wide = [torch.empty(2 * far + heads * d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    a, b = (t.as_strided((3, heads, d), (far, d, 1)) for t in wide)
    a.copy_(x)
    api.tgvkv_rope(plan, pos, a, b)
    assert same(a, x) and same(b, want)
    api.tgvkv_rope(plan, pos, a, a)
    assert same(a, want)


@pytest.mark.parametrize("T,H_q,H_k", [(300001, 56, 4), (20000003, 1, 0)])
def test_more_than_two_to_the_31_elements(api, T, H_q, H_k):
    d, part = 128, 50000
    gen = torch.Generator("cuda").manual_seed(3)
    plan, pos = api.make_rope(d, layout="interleaved"), torch.arange(T, dtype=torch.int32, device="cuda")
    base = torch.randn((part, H_q + H_k, d), generator=gen, device="cuda").bfloat16()
    x = torch.empty((T, H_q + H_k, d), dtype=torch.bfloat16, device="cuda")
    for t in range(0, T, part):
        x[t:t + part] = base[:T - t]
    q, k = x.split([H_q, H_k], dim=1)
    api.tgvkv_rope(plan, pos, q, q, *((k, k) if H_k else ()))
    for t in (0, part, T // part // 2 * part, T // part * part):
        want = base[:T - t].clone()
        q, k = want.split([H_q, H_k], dim=1)
        api.tgvkv_rope(plan, pos[t:t + part], q, q, *((k, k) if H_k else ()))
        assert same(x[t:t + part], want), t


@pytest.mark.parametrize("fmt,n_pages", [("bf16", 1 << 17), ("int8", 1 << 18), ("int4", 1 << 19), ("fp4", 1 << 19)])
@pytest.mark.parametrize("n", [1, 300])
def test_pages_beyond_four_gigabytes(api, fmt, n_pages, n):
    """The last pages of pools of 8 GB each, taken first: stored, attended to, read back."""
    B, H_q, H_kv, d, page, max_pages = 2, 8, 2, 128, 256, 4
    gen = torch.Generator("cuda").manual_seed(n)
    first = [301, 700]
    results = []
    qkv = [torch.randn((sum(c), H_q + 2 * H_kv, d), generator=gen, device="cuda").bfloat16() for c in (first, [n, n])]
    plan = api.make_rope(d)
    for pages_of in (n_pages, 24):
        desc = api.make_cache_desc(B, H_q, H_kv, d, page, pages_of, max_pages, fmt)
        cache, pages, ws = api.alloc_cache(desc), api.alloc_pages(desc), api.new_cache_workspace(desc)
        pages.free.copy_(torch.arange(pages_of, dtype=torch.int32, device="cuda"))    # the last on top
        lens, got = torch.zeros(B * H_kv, dtype=torch.int32, device="cuda"), []
        at = [0, 0]
        for news, x in zip((first, [n, n]), qkv):
            q, k, v = x.split([H_q, H_kv, H_kv], dim=1)
            off, T = ints(np.concatenate([[0], np.cumsum(news)])), sum(news)
            pos = ints(np.concatenate([np.arange(a, a + c) for a, c in zip(at, news)]))
            at = [a + c for a, c in zip(at, news)]
            slots, grown = torch.empty((T, H_kv), dtype=torch.int32, device="cuda"), torch.empty_like(lens)
            api.tgvkv_pages_append(desc, pages, lens, off, slots, grown, ws)
            assert int(slots.min()) >= (pages_of - 24) * page
            qt, out = (torch.empty((T, H_q, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            api.tgvkv_rope_write(desc, cache, plan, pos, slots, q, k, v, qt, ws)
            api.tgvkv_chunk_attention(desc, cache, pages.page_table, grown, qt, off, max(news), out, ws)
            lens = grown
            got += [qt, out]
        rows_off = torch.cat([lens.new_zeros(1, dtype=torch.int64), lens.long().cumsum(0)])
        rows = [torch.empty((int(rows_off[-1]), d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        api.tgvkv_cache_read(desc, cache, pages.page_table, None, rows_off, *rows, ws)
        assert api.tgvkv_status(ws) == 0
        results.append(got + rows)
        del cache
    for a, b in zip(*results):
        assert same(a, b)


@pytest.mark.parametrize("layout,rot", [("half", 64), ("half", 20), ("interleaved", 64), ("interleaved", 20)])
@pytest.mark.parametrize("H", [1, 4])
def test_infinities_and_nan_stay_in_their_pair(api, layout, rot, H):
    d, T = 64, 40
    x = torch.randn((T, H, d), device="cuda").bfloat16()
    plan, pos = api.make_rope(d, rot_dim=rot, layout=layout), torch.arange(T, dtype=torch.int32, device="cuda")
    clean = torch.empty_like(x)
    api.tgvkv_rope(plan, pos, x, clean)
    dirty, touched = x.clone(), torch.zeros_like(x, dtype=torch.bool)
    for t, (c, value) in enumerate([(0, float("nan")), (rot - 1, float("inf")), (3, float("-inf")), (d - 1, float("nan"))]):
        dirty[7 * t + 1, H - 1, c] = value
        partner = c if c >= rot else (c + rot // 2) % rot if layout == "half" else c ^ 1
        touched[7 * t + 1, H - 1, c] = touched[7 * t + 1, H - 1, partner] = True
    out = torch.empty_like(x)
    api.tgvkv_rope(plan, pos, dirty, out)
    assert same(out[~touched], clean[~touched])
    assert not torch.isfinite(out[touched]).any()
    # the fused write: bf16 pages
    desc = api.make_cache_desc(1, H, H, d, 16, 3 * H, 3)
    cache, pages, ws = api.alloc_cache(desc), api.alloc_pages(desc), api.new_cache_workspace(desc)
    lens, grown = torch.zeros(H, dtype=torch.int32, device="cuda"), torch.empty(H, dtype=torch.int32, device="cuda")
    slots = torch.empty((T, H), dtype=torch.int32, device="cuda")
    api.tgvkv_pages_append(desc, pages, lens, ints([0, T]), slots, grown, ws)
    qt = torch.empty_like(x)
    api.tgvkv_rope_write(desc, cache, plan, pos, slots, dirty, dirty, x, qt, ws)
    for got in (qt, cache.k.view(-1, d)[slots.long()]):
        assert same(got[~touched], clean[~touched]) and not torch.isfinite(got[touched]).any()
    assert same(cache.v.view(-1, d)[slots.long()], x) and api.tgvkv_status(ws) == 0


def test_graphs_that_share_a_workspace(api):
    """Two captured decode steps of different lists and formats, one workspace, replayed in
    turn on two streams ordered by events."""
    B, H_q, H_kv, d, page, max_pages, steps = 5, 4, 2, 64, 16, 8, 40
    ws, graphs, outs = None, [], []
    for fmt in ("fp4", "int8"):
        desc = api.make_cache_desc(B, H_q, H_kv, d, page, B * H_kv * max_pages, max_pages, fmt)
        ws = api.new_cache_workspace(desc) if ws is None else ws
        cache, pages = api.alloc_cache(desc), api.alloc_pages(desc)
        gen = torch.Generator("cuda").manual_seed(1)
        x = torch.randn((B, H_q + 2 * H_kv, d), generator=gen, device="cuda").bfloat16()
        q, k, v = x.split([H_q, H_kv, H_kv], dim=1)
        lens, grown = (torch.zeros(B * H_kv, dtype=torch.int32, device="cuda") for _ in range(2))
        pos, off = ints(np.arange(B)), ints(np.arange(B + 1))
        slots = torch.empty((B, H_kv), dtype=torch.int32, device="cuda")
        qt, out = (torch.empty((B, H_q, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        plan = api.make_rope(d)

        def step():
            api.tgvkv_pages_append(desc, pages, lens, off, slots, grown, ws)
            api.tgvkv_rope_write(desc, cache, plan, pos, slots, q, k, v, qt, ws)
            api.tgvkv_chunk_attention(desc, cache, pages.page_table, grown, qt, off, 1, out, ws)
            lens.copy_(grown)
            pos.add_(1)

        start = [t.clone() for t in (lens, pos)]
        want = []
        for _ in range(steps):
            step()
            want.append(out.clone())
        lens.copy_(start[0]), pos.copy_(start[1])
        api.tgvkv_pages_init(desc, pages)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            step()
        graphs.append((graph, out, want, (desc, cache, pages, x, lens, grown, pos, off, slots, qt)))
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    done, seen = None, [[], []]
    for i in range(steps):
        for j, (graph, out, _, _) in enumerate(graphs):
            with torch.cuda.stream(streams[j]):
                if done is not None:
                    streams[j].wait_event(done)
                graph.replay()
                seen[j].append(out.clone())
                done = torch.cuda.Event()
                done.record()
    torch.cuda.synchronize()
    assert api.tgvkv_status(ws) == 0
    for (_, _, want, _), got in zip(graphs, seen):
        assert all(same(a, b) for a, b in zip(got, want))
