"""Host-side checks of the paged-cache calls (no GPU): every bad argument is
refused before any launch, and the descriptor's limits hold at their bounds."""
import ctypes

import numpy as np
import pytest
import torch

import _cache_ref as R

P = ctypes.c_void_p
FAKE, ODD = P(0x10000), P(0x10008)     # never dereferenced
FAKE2 = P(0x200000)


@pytest.fixture(scope="module")
def lib(repo_root):
    from paper_2606_03075_gb300 import build
    build.build()
    from paper_2606_03075_gb300 import _lib
    return _lib.load()


def desc(**kw):
    from paper_2606_03075_gb300 import _lib
    base = dict(B=2, H_q=8, H_kv=2, d=128, page_size=16, n_pages=64, max_pages=8, format=1,
                softmax_scale=0.0)
    base.update(kw)
    return _lib.CacheDesc(**base)


def pools(k=FAKE, v=FAKE, ks=FAKE, vs=FAKE):
    from paper_2606_03075_gb300 import _lib
    return ctypes.byref(_lib.CachePools(k, v, ks, vs))


def test_descriptor(lib):
    def ws(**kw):
        return lib.tgvkv_cache_workspace_size(ctypes.byref(desc(**kw)))

    assert lib.tgvkv_cache_workspace_size(None) == 0
    for good in (dict(), dict(B=1, H_q=1, H_kv=1), dict(d=64), dict(H_q=256), dict(page_size=256),
                 dict(format=0), dict(format=2), dict(B=65535, H_q=1, H_kv=1), dict(max_pages=1),
                 dict(softmax_scale=-1.0), dict(n_pages=(1 << 27) - 1),
                 dict(B=1, H_q=1, H_kv=1, max_pages=1 << 26)):
        assert ws(**good) > 0, good
    for bad in (dict(B=0), dict(H_q=0), dict(H_kv=0), dict(n_pages=0), dict(max_pages=0), dict(B=-1),
                dict(H_q=7), dict(d=96), dict(d=256), dict(H_q=258), dict(page_size=8),
                dict(page_size=48), dict(page_size=512), dict(page_size=0), dict(format=3),
                dict(format=-1), dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")),
                dict(B=32768), dict(n_pages=1 << 27), dict(max_pages=(1 << 26) + 1),
                dict(B=1024, H_kv=2, max_pages=1 << 20)):
        assert ws(**bad) == 0, bad


def test_refusals(lib):
    d = ctypes.byref(desc())
    flat = ctypes.byref(desc(format=0))

    def write(d=d, pl=pools(), table=FAKE, lens=FAKE, k=FAKE, kt=256, kh=128, v=FAKE, vt=256, vh=128,
              n=3, off=FAKE, out=FAKE2, ws=FAKE):
        return lib.tgvkv_cache_write(d, pl, table, lens, k, kt, kh, v, vt, vh, n, off, out, ws, None)

    for kw in (dict(d=None), dict(pl=None), dict(pl=pools(k=P(0))), dict(pl=pools(v=ODD)),
               dict(pl=pools(ks=P(0))), dict(pl=pools(vs=ODD)), dict(table=P(0)), dict(lens=P(0)),
               dict(k=P(0)), dict(k=ODD), dict(v=ODD), dict(kt=252), dict(kh=4), dict(kh=64),
               dict(vt=-8), dict(vh=-128), dict(kt=1 << 38), dict(n=-1), dict(off=P(0)),
               dict(out=P(0)), dict(out=FAKE), dict(out=P(0x10000 + 12)), dict(ws=P(0)),
               dict(ws=ODD), dict(d=ctypes.byref(desc(d=32)))):
        assert write(**kw) in (1, 2), kw
        assert lib.tgvkv_last_error() != b"", kw
    assert write(n=1 << 31) == 2
    assert write(lens=FAKE, out=FAKE) == 1 and b"overlap" in lib.tgvkv_last_error()

    def rows(d=d, pl=pools(), k=FAKE, v=FAKE, n=3, off=FAKE, out=FAKE2):
        return lib.tgvkv_cache_write_rows(d, pl, FAKE, FAKE, k, v, n, off, out, FAKE, None)

    for kw in (dict(d=None), dict(k=P(0)), dict(v=ODD), dict(n=-1), dict(off=P(0)),
               dict(off=P(0x10004)), dict(out=FAKE)):
        assert rows(**kw) == 1, kw
    assert rows(n=1 << 31) == 2

    def read(d=d, pl=pools(), table=FAKE, off=FAKE, k=FAKE, v=FAKE, n=3, ws=FAKE):
        return lib.tgvkv_cache_read(d, pl, table, None, off, k, v, n, ws, None)

    for kw in (dict(d=None), dict(pl=pools(ks=P(0))), dict(table=P(0)), dict(off=P(0)), dict(k=P(0)),
               dict(v=ODD), dict(n=-2), dict(ws=P(0))):
        assert read(**kw) == 1, kw

    def attend(d=d, pl=pools(), table=FAKE, lens=FAKE, q=FAKE, qt=1024, qh=128, n=3, off=FAKE,
               max_q=2, out=FAKE, ws=FAKE):
        return lib.tgvkv_chunk_attention(d, pl, table, lens, q, qt, qh, n, off, max_q, out, ws, None)

    for kw in (dict(d=None), dict(pl=pools(vs=P(0))), dict(table=P(0)), dict(lens=P(0)), dict(q=P(0)),
               dict(q=ODD), dict(qt=1020), dict(qh=-8), dict(qh=120), dict(n=-1), dict(off=P(0)),
               dict(max_q=-1), dict(out=P(0)), dict(out=ODD), dict(ws=P(0)), dict(ws=ODD)):
        assert attend(**kw) == 1, kw
    # nothing to compute: accepted without a launch; bf16 pools need no scales
    assert attend(n=0, q=P(0), out=P(0)) == 0 and attend(max_q=0) == 0
    assert attend(d=flat, pl=pools(ks=P(0), vs=P(0)), max_q=0) == 0
    assert lib.tgvkv_last_error() == b""


def test_binding_checks(lib):
    """The Python binding's own refusals, on CPU tensors and wrong shapes."""
    from paper_2606_03075_gb300 import api
    cd = api.make_cache_desc(2, 8, 2, 64, 16, 8, 4, "int4", softmax_scale=0.5)
    assert (cd.format, cd.page_size, cd.softmax_scale) == (2, 16, 0.5)
    with pytest.raises(KeyError):
        api.make_cache_desc(2, 8, 2, 64, 16, 8, 4, "fp8")
    cache = api.alloc_cache(cd, device="meta")
    assert cache.k.shape == (8, 16, 32) and cache.k.dtype == torch.uint8
    assert cache.v_scale.shape == (8, 16, 2)
    flat = api.alloc_cache(api.make_cache_desc(2, 8, 2, 64, 16, 8, 4), device="meta")
    assert flat.k.dtype == torch.bfloat16 and flat.k.shape == (8, 16, 64) and flat.k_scale is None
    q = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        api.tgvkv_chunk_attention(cd, cache, None, None, q, None, 1, None, None)
    with pytest.raises(TypeError):
        api.tgvkv_cache_write(cd, cache, None, None, None, None, None, None, None)
    with pytest.raises(api.TgvkvError):
        api.tgvkv_cache_workspace_size(api.make_cache_desc(2, 8, 2, 64, 17, 8, 4))


@pytest.mark.parametrize("fmt", ["int8", "int4"])
def test_reference_format(fmt):
    """The reference's own pins: the scale is the smallest that holds, codes are
    nearest (ties to even), packing is reversible, the error is at most half a step."""
    rng = np.random.default_rng(1)
    x = R.bf16_values(R.bf16_bits(rng.standard_normal((50, 64)) * 2.0 ** rng.integers(-9, 9, (50, 1))))
    q, byte = R.encode(x, fmt)
    step = np.repeat(2.0 ** (byte.astype(float) - 127), 32, axis=1)
    top = np.abs(x).reshape(50, 2, 32).max(-1)
    s = 2.0 ** (byte.astype(float) - 127)
    assert (top <= R.Q_MAX[fmt] * s).all() and (top > R.Q_MAX[fmt] * s / 2).all()
    assert (np.abs(q * step - x) <= step / 2).all()
    assert np.array_equal(R.unpack(R.pack(q, fmt), fmt), q)
    t = np.zeros((1, 32))
    t[0, :4] = [R.Q_MAX[fmt], 0.5, 1.5, -2.5]
    assert R.encode(t, fmt)[0][0, :4].tolist() == [R.Q_MAX[fmt], 0, 2, -2]
    t[0, 0] += 0.5                          # above Q: the next power of two
    assert R.encode(t, fmt)[1][0, 0] == 128
    t[0, 9] = np.nan
    q, byte = R.encode(t, fmt)
    assert byte[0, 0] == 255 and (q == 0).all() and np.isnan(R.decode(q, byte)).all()


def test_reference_attention_against_scalar_loops():
    rng = np.random.default_rng(2)
    n, G, ln, d = 3, 2, 5, 4
    q, k, v = rng.standard_normal((n, G, d)), rng.standard_normal((ln, d)), rng.standard_normal((ln, d))
    o = R.attention(q, k, v, n, 0.7)
    for i in range(n):
        for h in range(G):
            w = [np.exp(0.7 * sum(q[i, h, c] * k[j, c] for c in range(d))) for j in range(ln - n + i + 1)]
            for c in range(d):
                want = sum(w[j] * v[j, c] for j in range(len(w))) / sum(w)
                assert abs(o[i, h, c] - want) < 1e-12
    o = R.attention(q, k[:2], v[:2], n, 0.7)
    assert (o[0] == 0).all() and np.allclose(o[1], v[0])
