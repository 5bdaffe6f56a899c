"""Calls queued one after another without a pause see what the ones before wrote, where the
page lists and rotary calls are among them: each chain is run with the GPU waited for after
every call, then as a graph and behind a busy GPU, and compared bit for bit."""
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


def compare(reset, steps, outputs):
    """reset() restores the inputs; outputs: tensors."""
    def run(wait):
        for f in steps:
            f()
            if wait:
                torch.cuda.synchronize()

    def taken():
        torch.cuda.synchronize()
        return [t.clone().view(torch.uint8) for t in outputs]

    reset()
    torch.cuda.synchronize()
    run(True)
    want = taken()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        reset()
        run(False)
    for _ in range(4):
        graph.replay()
    for a, b in zip(taken(), want):
        assert torch.equal(a, b)
    busy = torch.randn(4096, 4096, device="cuda").bfloat16()
    for _ in range(3):
        busy = busy @ busy * 1e-3
        reset()
        run(False)
    for a, b in zip(taken(), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T,H_q,H_k", [(1, 4, 1), (700, 8, 2), (9000, 1, 0), (5000, 28, 4)])
def test_turned_again_and_again(api, T, H_q, H_k):
    """In place, call after call: a row read too early misses a turn."""
    d = 128
    gen = torch.Generator("cuda").manual_seed(T)
    plan = api.make_rope(d)
    q0, k0 = (torch.randn((T, h, d), generator=gen, device="cuda").bfloat16() for h in (H_q, H_k))
    q, k = torch.empty_like(q0), torch.empty_like(k0)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    kk = (k, k) if H_k else ()
    compare(lambda: (q.copy_(q0), k.copy_(k0)), [lambda: api.tgvkv_rope(plan, pos, q, q, *kk)] * 6, [q, k])


@pytest.mark.parametrize("fmt,B,n,H_q,H_kv", [("bf16", 3, 1, 8, 2), ("fp4", 2, 700, 8, 8), ("int8", 40, 1, 28, 4),
                                              ("int8", 2, 3000, 16, 2)])
def test_a_layer_of_calls(api, fmt, B, n, H_q, H_kv):
    """Pages and slots, tokens turned and stored, attention, rows read back, moved, and the
    pages given back for the next round; buffers hold other values before."""
    d, page = 128, 32
    S, T, rounds = B * H_kv, B * n, 3
    max_pages = -(-2 * n // page) + 2
    desc = api.make_cache_desc(B, H_q, H_kv, d, page, S * max_pages, max_pages, fmt)
    cache, pages, ws = api.alloc_cache(desc), api.alloc_pages(desc), api.new_cache_workspace(desc)
    gen = torch.Generator("cuda").manual_seed(n)
    plan = api.make_rope(d, sections=[20, 22, 22])
    ints = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")
    lens, grown, first = ints([n // 2] * S), ints([0] * S), ints([n // 2] * S)
    off = ints(np.arange(0, T + 1, n))
    pos = torch.arange(3 * T, dtype=torch.int32, device="cuda").view(3, T)
    qkv = torch.randn((T, H_q + 2 * H_kv, d), generator=gen, device="cuda").bfloat16()
    q, k, v = qkv.split([H_q, H_kv, H_kv], dim=1)
    slots = torch.empty((T, H_kv), dtype=torch.int32, device="cuda")
    qt, out = (torch.empty((T, H_q, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = torch.arange(0, S * n + 1, n, dtype=torch.int64, device="cuda")
    kr, vr, km = (torch.empty((S * n, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    back = -torch.arange(S * n, dtype=torch.int32, device="cuda")
    move = api.make_rope(d)
    start = [t.clone() for t in (pages.page_table, pages.free, pages.n_free)]
    pools = [t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]

    def reset():
        for t, s in zip((pages.page_table, pages.free, pages.n_free), start):
            t.copy_(s)
        for t in pools:
            t.view(torch.uint8).zero_()
        for t in (slots, grown):
            t.fill_(-1)
        for t in (qt, out, kr, vr, km):
            t.fill_(3.0)

    zeros = ints([0] * S)
    steps = [lambda: api.tgvkv_pages_grow(desc, pages, zeros, first, ws)]
    for _ in range(rounds):
        steps += [lambda: api.tgvkv_pages_append(desc, pages, lens, off, slots, grown, ws),
                  lambda: api.tgvkv_rope_write(desc, cache, plan, pos, slots, q, k, v, qt, ws),
                  lambda: api.tgvkv_chunk_attention(desc, cache, pages.page_table, grown, qt, off, n, out, ws),
                  lambda: api.tgvkv_cache_read(desc, cache, pages.page_table, lens, rows, kr, vr, ws),
                  lambda: api.tgvkv_rope(move, back, kr.view(-1, 1, d), km.view(-1, 1, d), mode="move"),
                  lambda: api.tgvkv_rope(plan, pos, qt, qt, mode="gradient"),
                  lambda: api.tgvkv_pages_shrink(desc, pages, grown, lens, ws)]
    compare(reset, steps, [qt, out, kr, vr, km, slots, grown, pages.page_table, pages.free, pages.n_free] + pools)
    assert api.tgvkv_status(ws) == 0
