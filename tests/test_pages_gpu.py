"""GPU tests of the page list (tables and slot maps built on the device) through the C ABI,
against the list operations of _rope_ref.py.  Whole numbers: everything is compared exactly."""
import numpy as np
import pytest
import torch

import _rope_ref as F

pytestmark = pytest.mark.gpu
INDEX, PAGES = 0x08, 0x80


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "the GPU tests need a CUDA device"
    from paper_2606_03075_gb300 import build
    build.build()
    from paper_2606_03075_gb300 import api as _api
    return _api


class Rig:
    def __init__(self, api, B, H_kv, page, max_pages, n_pages):
        self.api, self.B, self.H_kv, self.S = api, B, H_kv, B * H_kv
        self.desc = api.make_cache_desc(B, H_kv, H_kv, 64, page, n_pages, max_pages)
        self.pages, self.ws = api.alloc_pages(self.desc), api.new_cache_workspace(self.desc)
        self.ref = F.Pages(self.S, max_pages, n_pages, page)
        self.lens = np.zeros(self.S, np.int64)
        self.same()

    def ints(self, a):
        return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")

    def same(self):
        assert np.array_equal(self.pages.page_table.cpu().numpy(), self.ref.table)
        n = int(self.pages.n_free)
        assert n == len(self.ref.stack)
        assert self.pages.free[:n].cpu().tolist() == self.ref.stack

    def grow(self, new):
        self.api.tgvkv_pages_grow(self.desc, self.pages, self.ints(self.lens), self.ints(new), self.ws)
        assert self.api.tgvkv_status(self.ws) == (0 if self.ref.grow(self.lens, new) else PAGES)
        self.same()

    def shrink(self, new):
        self.api.tgvkv_pages_shrink(self.desc, self.pages, self.ints(self.lens), self.ints(new), self.ws)
        assert self.api.tgvkv_status(self.ws) == 0
        self.ref.shrink(self.lens, new)
        self.same()

    def append(self, news, pad=0, slots=True):
        off, T = np.concatenate([[0], np.cumsum(news)]), int(sum(news)) + pad
        out = torch.full((self.S,), 99, dtype=torch.int32, device="cuda")
        got = torch.full((T, self.H_kv), 99, dtype=torch.int32, device="cuda") if slots else None
        self.api.tgvkv_pages_append(self.desc, self.pages, self.ints(self.lens), self.ints(off), got, out, self.ws,
                                    n_tokens=T)
        new = self.lens + np.repeat(news, self.H_kv)
        ok = self.ref.grow(self.lens, new)
        assert self.api.tgvkv_status(self.ws) == (0 if ok else PAGES)
        self.same()
        assert out.cpu().tolist() == (new if ok else self.lens).tolist()
        if slots:
            want = self.ref.slots(self.lens, news if ok else [0] * self.B, self.H_kv, T)
            assert np.array_equal(got.cpu().numpy(), want)
            again = torch.full_like(got, 99)
            if ok:
                self.api.tgvkv_page_slots(self.desc, self.pages.page_table, self.ints(self.lens), self.ints(off),
                                          again, self.ws)
                assert self.api.tgvkv_status(self.ws) == 0 and torch.equal(again, got)
        if ok:
            self.lens = new
        return ok


@pytest.mark.parametrize("B,H_kv,page,max_pages", [(1, 1, 16, 1), (1, 1, 256, 40), (3, 4, 16, 9), (64, 4, 16, 12),
                                                   (7, 128, 32, 5), (300, 3, 64, 4)])
def test_a_life_of_requests(api, B, H_kv, page, max_pages):
    """Prompts, decode steps, evictions and ends at random, the list compared after each."""
    rng = np.random.default_rng([B, H_kv, page])
    rig = Rig(api, B, H_kv, page, max_pages, B * H_kv * max_pages)
    cap = max_pages * page
    for step in range(12):
        room = cap - rig.lens.reshape(B, H_kv).max(1)
        kind = step % 4
        if kind == 0:      # prompts of any size, for some requests
            rig.append(np.where(rng.random(B) < 0.7, rng.integers(0, room + 1), 0), pad=step)
        elif kind == 1:    # a decode step
            rig.append(np.minimum(room, 1), pad=3, slots=step != 5)
        elif kind == 2:    # an eviction: every set its own length
            new = rng.integers(0, rig.lens + 1)
            rig.shrink(new)
            rig.lens = new
        else:              # some requests end, others are admitted
            end = np.repeat(rng.random(B) < 0.5, H_kv)
            rig.shrink(np.where(end, 0, rig.lens))
            rig.lens = np.where(end, 0, rig.lens)
            new = np.minimum(rig.lens + rng.integers(0, cap, rig.S), cap)
            rig.grow(new)
            rig.lens = new


@pytest.mark.parametrize("B,H_kv,page", [(64, 4, 16), (300, 7, 32), (33, 1, 64)])
def test_longer_sequences_beside_decode_steps(api, B, H_kv, page):
    """A token for most, none for some, tens for a few: under 4 a sequence in all."""
    rng = np.random.default_rng(B)
    rig = Rig(api, B, H_kv, page, 20, B * H_kv * 20)
    new = rng.integers(0, 5 * page, rig.S)
    rig.grow(new)
    rig.lens = new
    for step in range(4):
        news = np.where(rng.random(B) < 0.8, 1, 0)
        news[rng.permutation(B)[:4]] = [3 * B // 2, B // 2, 5, 4]
        assert news.sum() <= 4 * B
        rig.append(news, pad=step % 2, slots=step != 3)


def test_taking_and_giving_back_leaves_the_list_as_it_was(api):
    rig = Rig(api, 5, 3, 16, 8, 200)
    rig.append([3, 40, 0, 100, 16])
    before = [t.clone() for t in (rig.pages.page_table, rig.pages.free, rig.pages.n_free)]
    lens = rig.lens
    rig.append([17, 1, 5, 28, 0])
    rig.shrink(lens)
    for a, b in zip(before, (rig.pages.page_table, rig.pages.free, rig.pages.n_free)):
        assert torch.equal(a, b)


# granules of 2, 4 and 8 sets, several CTAs; few new tokens a sequence, and more
@pytest.mark.parametrize("B,H_kv,max_pages,most", [(9001, 1, 3, 3), (5000, 4, 2, 2), (65535, 1, 2, 3),
                                                   (9001, 1, 4, 25), (2050, 5, 3, 20), (65535, 1, 3, 18),
                                                   (9001, 1, 3, 0), (4500, 3, 3, 0)])
def test_many_sets(api, B, H_kv, max_pages, most):
    page, rng = 16, np.random.default_rng(B)
    S = B * H_kv
    desc = api.make_cache_desc(B, H_kv, H_kv, 64, page, S * max_pages, max_pages)
    pages, ws = api.alloc_pages(desc), api.new_cache_workspace(desc)
    lens = rng.integers(0, 20, S)
    ints = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")
    zeros, out = ints(np.zeros(S)), torch.empty(S, dtype=torch.int32, device="cuda")
    api.tgvkv_pages_grow(desc, pages, zeros, ints(lens), ws)
    held = (lens + page - 1) // page
    first = np.cumsum(held) - held
    table = np.full((S, max_pages), -1)
    for j in range(max_pages):
        table[:, j] = np.where(held > j, first + j, -1)
    assert np.array_equal(pages.page_table.cpu().numpy(), table)
    assert int(pages.n_free) == S * max_pages - held.sum()
    # (0: a few tokens for some, less than 2048 in all)
    news = rng.integers(0, most + 1, B) if most else np.where(rng.random(B) < 0.05, rng.integers(1, 9, B), 0)
    off, T = np.concatenate([[0], np.cumsum(news)]), int(news.sum())
    slots = torch.empty((T, H_kv), dtype=torch.int32, device="cuda")
    api.tgvkv_pages_append(desc, pages, ints(lens), ints(off), slots, out, ws)
    new = lens + np.repeat(news, H_kv)
    more = (new + page - 1) // page - held
    first = held.sum() + np.cumsum(more) - more
    for j in range(max_pages):
        table[:, j] = np.where((j >= held) & (j < held + more), first + j - held, table[:, j])
    assert np.array_equal(pages.page_table.cpu().numpy(), table)
    assert np.array_equal(out.cpu().numpy(), new)
    seq = np.repeat(np.arange(B), news)
    sets = seq[:, None] * H_kv + np.arange(H_kv)
    j = lens[sets] + (np.arange(T) - off[seq])[:, None]
    assert np.array_equal(slots.cpu().numpy(), table[sets, j // page] * page + j % page)
    api.tgvkv_pages_shrink(desc, pages, out, zeros, ws)
    assert (pages.page_table == -1).all() and int(pages.n_free) == S * max_pages
    assert sorted(pages.free.cpu().tolist()) == list(range(S * max_pages))
    assert api.tgvkv_status(ws) == 0


def test_long_sets_of_small_pages(api):
    """Entries and slots shared out over many CTAs: one set of 200000 slots beside short ones."""
    rig = Rig(api, 3, 2, 16, 12800, 40000)
    rig.append([5, 200000, 1])
    rig.append([0, 4000, 300])
    rig.shrink([0] * rig.S)
    rig.lens = np.zeros(rig.S, np.int64)


def test_too_few_pages_changes_nothing(api):
    rig = Rig(api, 4, 2, 16, 6, 20)
    assert rig.append([30, 17, 0, 16])                       # 4 + 4 + 2 of 20
    assert not rig.append([50, 40, 33, 1], pad=2)
    rig.grow([96] * rig.S)                                   # refused, compared inside
    assert rig.append([2, 15, 16, 0])                        # fits


def test_nonsense_is_reported_and_changes_nothing(api):
    rig = Rig(api, 3, 2, 16, 4, 24)
    rig.append([20, 0, 64])
    ints, d, pg, ws = rig.ints, rig.desc, rig.pages, rig.ws
    good = rig.lens
    out, slots = ints(np.full(6, 99)), torch.full((4, 2), 99, dtype=torch.int32, device="cuda")

    def bad(lens, new):
        for fn in (api.tgvkv_pages_grow, api.tgvkv_pages_shrink):
            fn(d, pg, ints(lens), ints(new), ws)
            assert api.tgvkv_status(ws) == INDEX
            rig.same()

    for s, n in ((0, -1), (5, 65), (3, 1 << 30)):
        wrong = good.copy()
        wrong[s] = n
        bad(wrong, good)
        bad(good, wrong)
    for off in ([1, 2, 3, 4], [0, 2, 1, 4], [0, 1, 2, 5], [0, 1, 1, 2], [0, -1, 0, 1], [0, 0, 0, 1 << 30]):
        # [0, 1, 1, 2]: the last sequence is at its table's end
        slots.fill_(99)
        api.tgvkv_pages_append(d, pg, ints(good), ints(off), slots, out, ws)
        assert api.tgvkv_status(ws) == INDEX, off
        rig.same()
        assert out.cpu().tolist() == good.tolist() and (slots == -1).all()
    for n in (-1, 25):
        keep = pg.n_free.clone()
        pg.n_free.fill_(n)
        api.tgvkv_pages_grow(d, pg, ints(good), ints(good + (good < 64)), ws)
        assert api.tgvkv_status(ws) == INDEX and int(pg.n_free) == n
        pg.n_free.copy_(keep)
    rig.same()
    # more given back than the pool has
    pg.n_free.fill_(23)
    api.tgvkv_pages_shrink(d, pg, ints(good), ints([0] * 6), ws)
    assert api.tgvkv_status(ws) == INDEX and int(pg.n_free) == 23


def test_entries_that_name_no_page(api):
    """They move as -1 and are reported; their slots are -1."""
    rig = Rig(api, 2, 1, 16, 4, 8)
    ints, d, pg, ws = rig.ints, rig.desc, rig.pages, rig.ws
    pg.free[7], pg.free[6] = 8, -5                           # the top two of the stack
    slots, out = torch.empty((40, 1), dtype=torch.int32, device="cuda"), ints([0, 0])
    api.tgvkv_pages_append(d, pg, ints([0, 0]), ints([0, 20, 40]), slots, out, ws)
    assert api.tgvkv_status(ws) == INDEX
    assert pg.page_table.cpu().tolist() == [[-1, -1, -1, -1], [2, 3, -1, -1]] and int(pg.n_free) == 4
    assert (slots[:20] == -1).all() and slots[20:].flatten().cpu().tolist() == list(range(32, 52))
    pg.page_table[1, 1] = 77
    api.tgvkv_pages_shrink(d, pg, ints([20, 20]), ints([20, 0]), ws)
    assert api.tgvkv_status(ws) == INDEX
    assert pg.free[:6].cpu().tolist() == [7, 6, 5, 4, -1, 2] and int(pg.n_free) == 6
    # a table from elsewhere: pages outside the pool, slots past the table
    table = ints([[0, 9, 1, 2], [3, 4, 5, 6]])
    got = torch.empty((30, 1), dtype=torch.int32, device="cuda")
    api.tgvkv_page_slots(d, table, ints([12, 50]), ints([0, 10, 28]), got, ws)
    assert api.tgvkv_status(ws) == INDEX
    want = [12, 13, 14, 15] + [-1] * 6 + [98 + i for i in range(14)] + [-1] * 6
    assert got.flatten().cpu().tolist() == want


def test_no_tokens_and_no_growth(api):
    rig = Rig(api, 2, 2, 32, 3, 12)
    rig.append([0, 0])
    rig.append([0, 0], pad=5)
    rig.append([7, 64])
    rig.grow(rig.lens)
    rig.shrink(rig.lens)
    rig.grow(rig.lens // 2)                                  # would shrink: stays
    rig.shrink(np.minimum(rig.lens + 9, 96))                 # would grow: stays


def test_a_graph_of_decode_steps(api):
    """Captured once: every replay takes the pages of its own step."""
    B, H_kv, page, steps = 6, 2, 16, 40
    rig = Rig(api, B, H_kv, page, 6, B * H_kv * 6)
    rig.append([1, 15, 16, 17, 40, 0])
    lens, out = rig.ints(rig.lens), torch.empty(rig.S, dtype=torch.int32, device="cuda")
    off = rig.ints(np.arange(B + 1))
    slots = torch.empty((B, H_kv), dtype=torch.int32, device="cuda")
    log, at = torch.empty((steps, B, H_kv), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        api.tgvkv_pages_append(rig.desc, rig.pages, lens, off, slots, out, rig.ws)
        lens.copy_(out)
        log.index_copy_(0, at, slots[None])
        at += 1
    for _ in range(steps):
        graph.replay()
    assert api.tgvkv_status(rig.ws) == 0
    for i in range(steps):
        new = rig.lens + 1
        assert rig.ref.grow(rig.lens, new)
        assert np.array_equal(log[i].cpu().numpy(), rig.ref.slots(rig.lens, [1] * B, H_kv, B)), i
        rig.lens = new
    rig.same()
