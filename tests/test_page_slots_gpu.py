"""The slot map alone (tgvkv_page_slots) where a set's length or a sequence's offsets are wrong:
reported, no slot for them, and the other sets' slots are as ever.  Whole numbers, compared
exactly."""
import numpy as np
import pytest
import torch

from test_pages_gpu import INDEX, Rig, api  # noqa: F401

pytestmark = pytest.mark.gpu


def made(rig, lens, off, T):
    got = torch.full((T, rig.H_kv), 99, dtype=torch.int32, device="cuda")
    rig.api.tgvkv_page_slots(rig.desc, rig.pages.page_table, rig.ints(lens), rig.ints(off), got, rig.ws)
    return got.cpu().numpy(), rig.api.tgvkv_status(rig.ws)


@pytest.mark.parametrize("wrong", [-1, -70, 65, 1 << 30, -(1 << 31)])
def test_a_set_of_a_wrong_length_has_no_slots(api, wrong):
    rig = Rig(api, 3, 2, 16, 4, 24)
    rig.grow([64] * 6)
    lens, news = np.array([20, 0, 13, 40, 1, 59]), [5, 0, 3]
    want = rig.ref.slots(lens, news, 2, 11)
    for s in range(6):
        bad = lens.copy()
        bad[s] = wrong
        expect = want.copy()
        b, g = divmod(s, 2)
        first = sum(news[:b])
        expect[first:first + news[b], g] = -1
        got, status = made(rig, bad, [0, 5, 5, 8], 11)
        assert status == INDEX and np.array_equal(got, expect), s
    assert made(rig, lens, [0, 5, 5, 8], 11)[1] == 0


@pytest.mark.parametrize("off", [[1, 2, 3, 4], [0, 2, 1, 4], [0, 1, 2, 5], [0, -1, 0, 1], [0, 0, 0, 1 << 30],
                                 [-3, 0, 2, 4], [0, 4, 4, 3], [2, 2, 2, 2]])
def test_sequences_of_wrong_offsets_have_no_slots(api, off):
    """A slot is that of the token's place in a sequence whose offsets have it, or -1."""
    rig = Rig(api, 3, 2, 16, 4, 24)
    rig.grow([64] * 6)
    lens, T = np.array([20, 0, 13, 40, 1, 59]), 4
    got, status = made(rig, lens, off, T)
    assert status == INDEX
    fine = [0 <= lo <= hi <= T and (b > 0 or lo == 0) for b, (lo, hi) in enumerate(zip(off, off[1:]))]
    ordered = all(a <= b for a, b in zip(off, off[1:]))
    for t in range(T):
        for g in range(2):
            may = set()
            for b in range(3):
                if fine[b] and off[b] <= t < off[b + 1]:
                    j = int(lens[2 * b + g]) + t - off[b]
                    may.add(int(rig.ref.table[2 * b + g, j // 16]) * 16 + j % 16)
            if not may or not ordered:       # decreasing offsets: whose it is, is not defined
                may.add(-1)
            assert int(got[t, g]) in may, (t, g, got[t, g], may)


@pytest.mark.parametrize("B,H_kv,T", [(65535, 1, 3), (512, 127, 700), (1, 1, 0)])
def test_wrong_lengths_are_found_among_many_sets(api, B, H_kv, T):
    """Sets without a token, too, and whichever it is; right ones report nothing."""
    d = api.make_cache_desc(B, H_kv, H_kv, 64, 16, 4, 2)
    ws, S = api.new_cache_workspace(d), B * H_kv
    table = torch.zeros(S, 2, dtype=torch.int32, device="cuda")
    lens = torch.zeros(S, dtype=torch.int32, device="cuda")
    off = torch.clamp(torch.arange(B + 1, device="cuda"), max=T).to(torch.int32)
    slots = torch.empty(T, H_kv, dtype=torch.int32, device="cuda")
    api.tgvkv_page_slots(d, table, lens, off, slots, ws)
    assert api.tgvkv_status(ws) == 0 and (slots[:min(T, B)] == 0).all()
    for s in {0, S // 3, S - 1}:
        lens[s] = 33
        api.tgvkv_page_slots(d, table, lens, off, slots, ws)
        assert api.tgvkv_status(ws) == INDEX, s
        lens[s] = 0
