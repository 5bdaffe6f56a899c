"""Calls queued one after another without a pause see what the ones before wrote,
where a paged-cache call or an eviction makes the rows that the next eviction reads.

The kernels of both may start before those ahead of them have finished, so the
rows' buffer holds other (finite) values before each step, and the outputs are
compared bit for bit with the same calls made one at a time."""
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


class Rig:
    """A paged cache of L x H_kv sets of N slots, in shuffled pages, and the eviction
    whose dense K and V those sets are."""

    def __init__(self, api, L, H_q, H_kv, d, N, fmt, n_win=8, n_vision=None, seed=0, shuffled=True):
        self.api, self.L, self.N, self.S, self.d = api, L, N, L * H_kv, d
        self.gen = torch.Generator("cuda").manual_seed(seed)
        page = 16
        max_pages = -(-N // page)
        n_pages = self.S * max_pages
        self.cdesc = api.make_cache_desc(L, H_q, H_kv, d, page, n_pages, max_pages, fmt)
        self.cache = api.alloc_cache(self.cdesc)
        order = torch.randperm(n_pages, generator=self.gen, device="cuda") if shuffled else \
            torch.arange(n_pages, device="cuda")
        self.table = order.to(torch.int32).view(self.S, max_pages)
        self.cws = api.new_cache_workspace(self.cdesc)
        n_vision = N - 2 * n_win if n_vision is None else n_vision
        self.desc = api.make_desc(L, H_q, H_kv, d, N, n_vision, n_win)
        self.ws = api.new_workspace(self.desc)
        self.modality = torch.zeros(N, dtype=torch.uint8, device="cuda")
        self.modality[3:3 + n_vision] = 1
        self.text_pos = torch.arange(N - n_win, N, dtype=torch.int32, device="cuda")
        self.w = torch.full((L, n_win), 1.0 / n_win, device="cuda")
        self.q = self.values(L, H_q, n_win, d)
        self.offsets = torch.arange(0, self.S * N + 1, N, dtype=torch.int64, device="cuda")
        self.zeros = torch.zeros(self.S, dtype=torch.int32, device="cuda")
        self.lens = torch.empty_like(self.zeros)

    def values(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda").bfloat16()

    def write_rows(self, k, v):
        self.api.tgvkv_cache_write_rows(self.cdesc, self.cache, self.table, self.zeros, k, v, self.offsets,
                                        self.lens, self.cws)

    def read(self, k, v):
        self.api.tgvkv_cache_read(self.cdesc, self.cache, self.table, None, self.offsets, k, v, self.cws)

    def evict(self, k, v, out, ratio=0.25):
        self.api.tgvkv_evict(self.desc, self.q, k, v, self.modality, self.text_pos, self.w, ratio, out,
                             self.ws)

    def clean(self):
        assert self.api.tgvkv_status(self.ws) == 0 and self.api.tgvkv_status(self.cws) == 0


def fields(out):
    return [out.scores, out.tvb_stat, out.budgets, out.offsets, out.idx, out.k_out, out.v_out]


def same(a, b):
    for x, y in zip(fields(a), fields(b)):
        x, y = (t.view(torch.int16) if t.dtype == torch.bfloat16 else t for t in (x, y))
        assert torch.equal(x, y)


def in_a_graph(steps):
    """The steps as one graph, replayed a few times."""
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        for step in steps:
            step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()


# (layers, query heads, KV heads, d, slots): fewer CTAs of the read than SMs, about as
# many, and many times as many
SIZES = [(1, 2, 2, 64, 100), (1, 8, 8, 128, 113), (2, 8, 2, 128, 700), (8, 8, 8, 64, 1500), (4, 28, 4, 128, 2304)]


@pytest.mark.parametrize("L,H_q,H_kv,d,N", SIZES)
@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_rows_read_back_then_evicted(api, L, H_q, H_kv, d, N, fmt):
    """tgvkv_cache_read into K and V, then tgvkv_evict on them."""
    rig = Rig(api, L, H_q, H_kv, d, N, fmt)
    rig.write_rows(rig.values(rig.S * N, d), rig.values(rig.S * N, d))
    k, v = (torch.empty(rig.S * N, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    old_k, old_v = rig.values(rig.S * N, d), rig.values(rig.S * N, d)
    want = api.alloc_outputs(rig.desc, 0.25)
    rig.read(k, v)
    torch.cuda.synchronize()
    rig.evict(k, v, want)
    rig.clean()
    outs = [api.alloc_outputs(rig.desc, 0.25) for _ in range(4)]

    def step(out):
        k.copy_(old_k)
        v.copy_(old_v)
        rig.read(k, v)
        rig.evict(k, v, out)

    in_a_graph([lambda o=o: step(o) for o in outs])
    rig.clean()
    for out in outs:
        same(out, want)
    for out in outs:                   # and queued behind a pause of the GPU, not captured
        for t in fields(out):
            t.zero_()
    busy = torch.randn(8192, 8192, device="cuda").bfloat16()
    busy = busy @ busy
    for out in outs:
        step(out)
    rig.clean()
    for out in outs:
        same(out, want)


@pytest.mark.parametrize("L,H_q,H_kv,d,N", SIZES[:4])
def test_rows_read_back_then_scored_and_gathered(api, L, H_q, H_kv, d, N):
    """tgvkv_cache_read, then tgvkv_score, or tgvkv_select_compact, on the rows."""
    rig = Rig(api, L, H_q, H_kv, d, N, "int8")
    rig.write_rows(rig.values(rig.S * N, d), rig.values(rig.S * N, d))
    k, v = (torch.empty(rig.S * N, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    old = rig.values(rig.S * N, d)
    want, got = api.alloc_outputs(rig.desc, 0.25), api.alloc_outputs(rig.desc, 0.25)
    rig.read(k, v)
    torch.cuda.synchronize()
    rig.evict(k, v, want)
    rig.clean()
    text = torch.zeros(L, H_kv, N - rig.desc.N_v, device="cuda")

    def score():
        k.copy_(old)
        rig.read(k, v)
        api.tgvkv_score(rig.desc, rig.q, k, rig.modality, rig.text_pos, rig.w, got.scores, got.tvb_stat,
                        rig.ws)

    def gather():
        k.copy_(old)
        v.copy_(old)
        rig.read(k, v)
        api.tgvkv_select_compact(rig.desc, want.scores, text, want.budgets, rig.modality, k, v, got.offsets,
                                 got.idx, got.k_out, got.v_out, rig.ws)

    in_a_graph([score, gather, score, gather])
    rig.clean()
    got.budgets.copy_(want.budgets)
    same(got, want)


@pytest.mark.parametrize("L,H_q,H_kv,d,N", [(1, 2, 2, 64, 96), (2, 8, 2, 128, 704), (4, 28, 4, 128, 2304)])
@pytest.mark.parametrize("between", [False, True])
def test_a_pool_that_is_the_dense_cache(api, L, H_q, H_kv, d, N, between):
    """Rows written into a bf16 pool whose pages lie in order, which is the eviction's
    K and V; with another paged-cache call in between, which starts early too."""
    rig = Rig(api, L, H_q, H_kv, d, N, "bf16", shuffled=False)
    k, v = rig.values(rig.S * N, d), rig.values(rig.S * N, d)
    old = rig.values(rig.S * N, d)
    want = api.alloc_outputs(rig.desc, 0.25)
    torch.cuda.synchronize()
    rig.evict(k, v, want)
    rig.clean()
    pk, pv = rig.cache.k.view(-1, d), rig.cache.v.view(-1, d)
    small = Rig(api, 1, 2, 2, 64, 32, "int8", n_win=4)
    sk, sv = small.values(64, 64), small.values(64, 64)
    outs = [api.alloc_outputs(rig.desc, 0.25) for _ in range(4)]

    def step(out):
        pk.copy_(old)
        pv.copy_(old)
        rig.write_rows(k, v)
        if between:
            small.write_rows(sk, sv)
        rig.evict(pk, pv, out)

    in_a_graph([lambda o=o: step(o) for o in outs])
    rig.clean()
    for out in outs:
        same(out, want)


@pytest.mark.parametrize("H_q,H_kv,d,N", [(2, 2, 64, 100), (28, 4, 128, 2304), (32, 32, 128, 675)])
def test_evicted_rows_evicted_again(api, H_q, H_kv, d, N):
    """One layer's sets have one length: the rows an eviction kept are the dense K and V
    of the next, queued right behind it."""
    ratio, n_win = 0.25, 8
    first = Rig(api, 1, H_q, H_kv, d, N, "bf16", n_win=n_win)
    rows = api.tgvkv_retained_rows(first.desc, ratio)
    N2 = rows // H_kv
    assert N2 * H_kv == rows
    second = Rig(api, 1, H_q, H_kv, d, N2, "bf16", n_win=n_win, n_vision=N2 - 2 * n_win, seed=1)
    k, v = first.values(H_kv * N, d), first.values(H_kv * N, d)
    mid = api.alloc_outputs(first.desc, ratio)
    want = api.alloc_outputs(second.desc, ratio)
    first.evict(k, v, mid, ratio)
    torch.cuda.synchronize()
    second.evict(mid.k_out, mid.v_out, want, ratio)
    first.clean()
    second.clean()
    old = first.values(rows, d)
    outs = [api.alloc_outputs(second.desc, ratio) for _ in range(4)]

    def step(out):
        mid.k_out.copy_(old)
        mid.v_out.copy_(old)
        first.evict(k, v, mid, ratio)
        second.evict(mid.k_out, mid.v_out, out, ratio)

    in_a_graph([lambda o=o: step(o) for o in outs])
    first.clean()
    second.clean()
    for out in outs:
        same(out, want)
