"""Host-side checks of the page list and of rotary positions (no GPU): plans hold the
frequencies of their definition, bad arguments are refused before any launch, and the
references' own pins."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import _rope_ref as F

P = ctypes.c_void_p
FAKE, FAKE2, ODD, ODD4 = P(0x10000), P(0x200000), P(0x10008), P(0x10002)   # never dereferenced
NULL = P(0)


@pytest.fixture(scope="module")
def lib():
    from paper_2606_03075_gb300 import build
    build.build()
    from paper_2606_03075_gb300 import _lib
    return _lib.load()


@pytest.fixture(scope="module")
def api(lib):
    from paper_2606_03075_gb300 import api as _api
    return _api


# ---- plans ----------------------------------------------------------------------
@pytest.mark.parametrize("rot", [2, 6, 20, 64, 128])
@pytest.mark.parametrize("o", [dict(), dict(base=1e6), dict(scaling="linear", factor=4.0),
                               dict(scaling="base", factor=8.0, base=5e5),
                               dict(scaling="parts", factor=8.0, original=8192, low=1.0, high=4.0),
                               dict(scaling="parts", factor=16.0, original=4096, base=1e6)])
def test_plan_frequencies(api, rot, o):
    plan = api.make_rope(128, rot_dim=rot, **o)
    for i, f in enumerate(F.frequencies(rot, **o)):
        got = plan.turns[i] / 2 ** 64
        # pow and a few operations in double, 2^-52 each; a fraction of 2^64
        assert abs(got - f / F.TWO_PI) <= 8 * 2.0 ** -52 * f / F.TWO_PI + 2.0 ** -63
        assert plan.axis[i] == 0
    assert (plan.d, plan.rot_dim, plan.layout, plan.axes, plan.attention) == (128, rot, 0, 1, 1.0)


def test_plan_sections_and_given_frequencies(api):
    plan = api.make_rope(128, sections=[16, 0, 40, 8], layout="interleaved", attention=1.25)
    assert list(plan.axis[:64]) == [0] * 16 + [2] * 40 + [3] * 8
    assert (plan.layout, plan.axes, plan.attention) == (1, 4, 1.25)
    assert set(api.make_rope(64, sections=[0, 32]).axis[:32]) == {1}
    f = [0.0, 1.0, -1.0, 7.5, 1e-9, 2.0 ** 30, -2.0 ** 33, 1e-40]
    plan = api.make_rope(16, freqs=f)
    for i, x in enumerate(f):
        want = Fraction(x / F.TWO_PI) % 1
        assert abs(Fraction(int(plan.turns[i]), 2 ** 64) - want) <= Fraction(1, 2 ** 63), x


def test_plan_refusals(lib, api):
    from paper_2606_03075_gb300 import _lib
    plan = _lib.RopePlan()

    def init(pl=plan, **kw):
        base = dict(d=128, rot_dim=128, layout=0, axes=1, scaling=0, base=1e4, factor=2.0, original=100,
                    low=1.0, high=4.0, attention=1.0)
        sections = (ctypes.c_int32 * 4)(*kw.pop("sections", (0, 0, 0, 0)))
        base.update(kw)
        return lib.tgvkv_rope_init(pl and ctypes.byref(pl),
                                   ctypes.byref(_lib.RopeDesc(sections=sections, **base)))

    assert init() == 0 and plan.ready != 0
    nan, inf = float("nan"), float("inf")
    for bad in (dict(d=0), dict(d=4, rot_dim=4), dict(d=100), dict(rot_dim=0), dict(rot_dim=7),
                dict(rot_dim=130), dict(layout=2), dict(layout=-1), dict(axes=0), dict(axes=5),
                dict(axes=2, sections=(32, 31, 1, 0)), dict(axes=2, sections=(65, -1, 0, 0)),
                dict(axes=2, sections=(2 ** 31 - 1, 2 ** 31 - 1, 0, 0)),
                dict(scaling=4), dict(scaling=-1), dict(base=0.0), dict(base=-2.0), dict(base=nan),
                dict(base=inf), dict(scaling=1, factor=0.0), dict(scaling=1, factor=nan),
                dict(scaling=2, factor=inf), dict(scaling=3, low=-1.0), dict(scaling=3, high=1.0),
                dict(scaling=3, high=inf), dict(scaling=3, original=0), dict(scaling=3, low=nan),
                dict(attention=-1.0), dict(attention=nan), dict(attention=inf),
                dict(base=1e-300), dict(freqs=(ctypes.c_double * 64)(*[nan] * 64)),
                dict(freqs=(ctypes.c_double * 64)(*[2.0 ** 40] * 64))):
        assert init(**bad) == 1, bad
        assert plan.ready == 0 and lib.tgvkv_last_error() != b""
    assert init(d=264, rot_dim=64) == 2
    assert init(pl=None) == 1 and lib.tgvkv_rope_init(ctypes.byref(plan), None) == 1
    for bad in (dict(sections=[30, 30]), dict(sections=[]), dict(sections=[8] * 8), dict(sections=[3]),
                dict(freqs=[1.0]), dict(attention=0.0)):
        with pytest.raises((ValueError, api.TgvkvError)):
            api.make_rope(128, **bad)
    with pytest.raises(KeyError):
        api.make_rope(128, layout="both")


# ---- refusals of the calls -----------------------------------------------------------
def test_rope_refusals(lib, api):
    plan = api.make_rope(128)
    made = ctypes.byref(plan)
    raw = ctypes.byref(type(plan)())

    def rope(pl=made, mode=0, pos=FAKE, ps=9, n=3, q=FAKE, qt=1024, qh=128, H=8, o=FAKE2, ot=1024, oh=128,
             k=NULL, kt=0, kh=0, Hk=0, l=NULL, lt=0, lh=0):
        return lib.tgvkv_rope(pl, mode, pos, ps, n, q, qt, qh, H, o, ot, oh, k, kt, kh, Hk, l, lt, lh, None)

    for kw in (dict(pl=None), dict(pl=raw), dict(mode=3), dict(mode=-1), dict(pos=NULL), dict(pos=ODD4),
               dict(n=-1), dict(q=NULL), dict(q=ODD), dict(o=NULL), dict(o=ODD), dict(qt=1020), dict(qh=4),
               dict(qh=-128), dict(qh=64), dict(ot=4), dict(oh=120), dict(H=0), dict(H=-1), dict(H=65536),
               dict(Hk=-1), dict(Hk=2), dict(Hk=2, k=FAKE, kt=256, kh=128, l=NULL, lt=256, lh=128),
               dict(Hk=2, k=FAKE, kt=256, kh=128, l=ODD, lt=256, lh=128),
               dict(o=FAKE, ot=2048), dict(o=FAKE, oh=256)):
        assert rope(**kw) == 1, kw
        assert lib.tgvkv_last_error() != b"", kw
    assert rope(n=1 << 31) == 2 and rope(n=1 << 28) == 2        # 2^31 rows
    axes = ctypes.byref(api.make_rope(128, sections=[32, 32]))
    assert rope(pl=axes, ps=-1) == 1 and rope(pl=axes, ps=1 << 38) == 1
    assert rope(n=0, q=NULL, o=NULL, pos=NULL) == 0             # nothing to do
    assert lib.tgvkv_last_error() == b""


def cache_desc(**kw):
    from paper_2606_03075_gb300 import _lib
    base = dict(B=2, H_q=8, H_kv=2, d=128, page_size=16, n_pages=64, max_pages=8, format=1,
                softmax_scale=0.0)
    base.update(kw)
    return ctypes.byref(_lib.CacheDesc(**base))


def test_rope_write_refusals(lib, api):
    from paper_2606_03075_gb300 import _lib
    plan, small = ctypes.byref(api.make_rope(128)), ctypes.byref(api.make_rope(64))

    def pools(k=FAKE, v=FAKE, ks=FAKE, vs=FAKE):
        return ctypes.byref(_lib.CachePools(k, v, ks, vs))

    def write(d=cache_desc(), pl=pools(), plan=plan, pos=FAKE, ps=9, slots=FAKE, n=3, q=FAKE, qt=1024,
              qh=128, k=FAKE, kt=256, kh=128, v=FAKE, vt=256, vh=128, o=FAKE2, ot=1024, oh=128, ws=FAKE):
        return lib.tgvkv_rope_write(d, pl, plan, pos, ps, slots, n, q, qt, qh, k, kt, kh, v, vt, vh, o, ot,
                                    oh, ws, None)

    for kw in (dict(d=None), dict(pl=None), dict(pl=pools(k=NULL)), dict(pl=pools(vs=NULL)), dict(plan=None),
               dict(plan=small), dict(plan=ctypes.byref(_lib.RopePlan())), dict(pos=NULL), dict(slots=NULL),
               dict(slots=ODD4), dict(n=-1), dict(q=NULL), dict(o=NULL), dict(q=ODD), dict(o=ODD),
               dict(k=NULL), dict(v=NULL), dict(k=ODD), dict(qt=1020), dict(kt=4), dict(vh=-8),
               dict(oh=120), dict(o=FAKE, ot=2048), dict(ws=NULL), dict(ws=ODD)):
        assert write(**kw) == 1, kw
        assert lib.tgvkv_last_error() != b"", kw
    assert write(n=1 << 31) == 2
    assert write(n=0, q=NULL, o=NULL, k=NULL, v=NULL, slots=NULL, pos=NULL) == 0


def test_page_refusals(lib):
    from paper_2606_03075_gb300 import _lib
    d = cache_desc()

    def pages(t=FAKE, f=FAKE, n=FAKE):
        return ctypes.byref(_lib.PageListPointers(t, f, n))

    bad_lists = [None, pages(t=NULL), pages(f=NULL), pages(n=NULL), pages(t=ODD4), pages(f=ODD4),
                 pages(n=ODD4)]
    for pg in bad_lists:
        assert lib.tgvkv_pages_init(d, pg, None) == 1
        assert lib.tgvkv_pages_grow(d, pg, FAKE, FAKE, FAKE, None) == 1
        assert lib.tgvkv_pages_shrink(d, pg, FAKE, FAKE, FAKE, None) == 1
        assert lib.tgvkv_pages_append(d, pg, FAKE, FAKE, 3, FAKE, FAKE2, FAKE, None) == 1
    bad = cache_desc(page_size=17)
    assert lib.tgvkv_pages_init(bad, pages(), None) == 2
    for fn in (lib.tgvkv_pages_grow, lib.tgvkv_pages_shrink):
        for args in ((bad, pages(), FAKE, FAKE, FAKE), (d, pages(), NULL, FAKE, FAKE),
                     (d, pages(), FAKE, ODD4, FAKE), (d, pages(), FAKE, FAKE, NULL),
                     (d, pages(), FAKE, FAKE, ODD)):
            assert fn(*args, None) != 0, args

    def append(lens=FAKE, off=FAKE, n=3, slots=FAKE, out=FAKE2, ws=FAKE):
        return lib.tgvkv_pages_append(d, pages(), lens, off, n, slots, out, ws, None)

    for kw in (dict(lens=NULL), dict(off=NULL), dict(off=ODD4), dict(n=-1), dict(slots=ODD4), dict(out=NULL),
               dict(out=FAKE), dict(ws=NULL), dict(ws=ODD)):
        assert append(**kw) == 1, kw
    assert append(n=1 << 30) == 2              # 2^31 slots

    def slots(table=FAKE, lens=FAKE, off=FAKE, n=3, out=FAKE, ws=FAKE):
        return lib.tgvkv_page_slots(d, table, lens, off, n, out, ws, None)

    for kw in (dict(table=NULL), dict(lens=ODD4), dict(off=NULL), dict(n=-1), dict(out=NULL), dict(ws=NULL)):
        assert slots(**kw) == 1, kw
    assert slots(n=1 << 30) == 2


def test_binding_refusals(api):
    """The Python binding's own checks, on CPU tensors and wrong shapes."""
    cd = api.make_cache_desc(2, 8, 2, 64, 16, 8, 4)
    pages = api.alloc_pages(cd, device="meta")
    assert pages.page_table.shape == (4, 4) and pages.free.shape == (8,) and pages.n_free.shape == (1,)
    ints = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        api.tgvkv_pages_grow(cd, pages, ints, ints, None)
    with pytest.raises(ValueError, match="columns"):
        api.tgvkv_pages_grow(cd, api.PageList(torch.zeros(4, 5, dtype=torch.int32), pages.free, pages.n_free),
                             ints, ints, None)
    with pytest.raises(TypeError, match="n_tokens"):
        api.tgvkv_pages_append(cd, pages, ints, ints, None, ints, None)
    with pytest.raises(ValueError, match="slots"):
        api.tgvkv_page_slots(cd, pages.page_table, ints, ints, torch.zeros(3, 3, dtype=torch.int32), None)
    plan = api.make_rope(64)
    x = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        api.tgvkv_rope(plan, ints, x, x)
    with pytest.raises(TypeError):
        api.tgvkv_rope(plan, ints, None, x)


# ---- the references -------------------------------------------------------------------
def test_reference_turns():
    """A turn keeps a pair's length, undoes itself, and depends on the difference of
    positions alone in a product of two rows."""
    rng = np.random.default_rng(0)
    for layout in ("half", "interleaved"):
        f = F.frequencies(16, scaling="parts", factor=4.0, original=64)
        x, y = rng.standard_normal((2, 5, 1, 24))
        pos = np.array([[0, 1, 7, 100, 1 << 20]])
        a = F.turned(x, pos, f, 16, layout)
        assert np.allclose((a ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(a[..., 16:], x[..., 16:])
        assert np.allclose(F.turned(a, -pos, f, 16, layout), x)
        assert np.allclose(F.turned(a, pos, f, 16, layout, mode="gradient"), x)
        b = F.turned(y, pos + 3, f, 16, layout)
        c = F.turned(y, np.full((1, 5), 3), f, 16, layout)
        assert np.allclose((a * b).sum(-1), (x * c).sum(-1))
    z = np.array([[[1.0, 0.0]]])
    assert np.allclose(F.turned(z, [[2]], [0.5], 2), [[[math.cos(1.0), math.sin(1.0)]]])
    assert F.angle(-1, 1.0) == pytest.approx(F.TWO_PI - 1)


def test_reference_pages():
    p = F.Pages(3, 4, 9, 2)
    assert p.grow([0, 0, 0], [3, 0, 1])
    assert p.table.tolist() == [[0, 1, -1, -1], [-1] * 4, [2, -1, -1, -1]]
    assert p.slots([2, 0, 0], [1, 0, 1], 1, 3).tolist() == [[2], [4], [-1]]
    before = (p.table.copy(), list(p.stack))
    assert not p.grow([3, 0, 1], [8, 8, 8]) and p.grow([3, 0, 1], [5, 7, 2])
    p.shrink([5, 7, 2], [3, 0, 1])
    assert np.array_equal(p.table, before[0]) and p.stack == before[1]
