"""Rotary calls over the ways a row is cut and held: parts of a head that end inside a vector of 8
values (narrow units beside wide copies), many tokens of head counts that leave groups of
threads idle, and the fused write of a part of a head in halves.  Tolerance: test_rope_gpu.py's,
2^-8 |y| + (2^-21 + 2^-50 |p| f_max) (|x1| + |x2|); what does not turn keeps its bits."""
import numpy as np
import pytest
import torch

import _rope_ref as F
from test_rope_write_gpu import FORMATS, ints, pools_of, step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "the GPU tests need a CUDA device"
    from paper_2606_03075_gb300 import build
    build.build()
    from paper_2606_03075_gb300 import api as _api
    return _api


def check(x, y, pos, rot, layout):
    """y against x turned, in 64 bits, a few thousand tokens at a time."""
    f = torch.tensor(F.frequencies(rot), dtype=torch.float64, device="cuda")
    for t in range(0, x.shape[0], 8000):
        xs, ys = x[t:t + 8000], y[t:t + 8000]
        th = pos[t:t + 8000].double()[:, None, None] * f
        far = th.abs().max(-1, keepdim=True).values
        part = xs[..., :rot].double()
        x1, x2 = part.chunk(2, -1) if layout == "half" else (part[..., ::2], part[..., 1::2])
        y1, y2 = x1 * th.cos() - x2 * th.sin(), x2 * th.cos() + x1 * th.sin()
        got = ys[..., :rot].double()
        g1, g2 = got.chunk(2, -1) if layout == "half" else (got[..., ::2], got[..., 1::2])
        room = (2.0 ** -21 + 2.0 ** -50 * far) * (x1.abs() + x2.abs())
        for g, ref in ((g1, y1), (g2, y2)):
            assert ((g - ref).abs() <= 2.0 ** -8 * ref.abs() + room).all()
        assert torch.equal(ys[..., rot:].contiguous().view(torch.int16), xs[..., rot:].contiguous().view(torch.int16))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot", [(80, 20), (80, 40), (96, 24), (72, 6), (256, 4), (16, 14), (128, 96), (64, 32)])
@pytest.mark.parametrize("T,H_q,H_k", [(1, 3, 1), (77, 1, 0), (300, 12, 1), (1201, 28, 4)])
def test_parts_of_a_head(api, layout, d, rot, T, H_q, H_k):
    """Into another tensor with gaps, and in place."""
    gen = torch.Generator("cuda").manual_seed(d + rot)
    plan, pos = api.make_rope(d, rot_dim=rot, layout=layout), torch.arange(T, dtype=torch.int32, device="cuda") * 31
    wide = torch.randn((T, H_q + H_k + 1, d), generator=gen, device="cuda").bfloat16()
    x = wide.clone()
    q, k = wide[:, :H_q], wide[:, H_q:H_q + H_k]
    out = torch.full((T, 2 * (H_q + H_k), d), 7.0, dtype=torch.bfloat16, device="cuda")
    qo, ko = out[:, :2 * H_q:2], out[:, 2 * H_q::2]
    api.tgvkv_rope(plan, pos, q, qo, *((k, ko) if H_k else ()))
    assert torch.equal(wide, x) and (out[:, 1::2] == 7).all()
    check(q, qo, pos, rot, layout)
    if H_k:
        check(k, ko, pos, rot, layout)
    api.tgvkv_rope(plan, pos, q, q, *((k, k) if H_k else ()))
    assert torch.equal(q, qo) and torch.equal(wide[:, -1], x[:, -1])
    if H_k:
        assert torch.equal(k, ko)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot", [(64, 32), (128, 64), (96, 96), (80, 40), (80, 20), (128, 128)])
@pytest.mark.parametrize("T,H_q,H_k", [(30011, 28, 4), (60007, 12, 1), (44444, 22, 5)])
def test_many_tokens_of_any_heads(api, layout, d, rot, T, H_q, H_k):
    """Token counts at which a token's rows are cut into smaller parts; in place, so that a row
    turned twice or not at all shows."""
    gen = torch.Generator("cuda").manual_seed(T)
    plan, pos = api.make_rope(d, rot_dim=rot, layout=layout), torch.arange(T, dtype=torch.int32, device="cuda") - 7
    both = torch.randn((T, H_q + H_k, d), generator=gen, device="cuda").bfloat16()
    x = both.clone()
    q, k = both.split([H_q, H_k], dim=1)
    api.tgvkv_rope(plan, pos, q, q, k, k)
    check(x, both, pos, rot, layout)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,rot", [(64, 16), (64, 32), (64, 48), (128, 16), (128, 48), (128, 80), (128, 112)])
@pytest.mark.parametrize("H_q,H_kv,news", [(8, 2, [5, 0, 33]), (28, 4, [64, 1, 3300])])
def test_stored_parts_of_a_head_in_halves(api, fmt, d, rot, H_q, H_kv, news):
    """The same, bit for bit, as turning and then writing; queries in place; padding."""
    desc, cache, ws, table, ln, off, slots, qkv = step(api, fmt, d, H_q, H_kv, news, [9, 0, 40], pad=5)
    T = qkv.shape[0]
    pos, plan = ints(np.random.default_rng(rot).integers(-9, 90000, T)), api.make_rope(d, rot_dim=rot)
    q, k, v = qkv.split([H_q, H_kv, H_kv], dim=1)
    qo, ko = torch.empty((T, H_q, d), dtype=torch.bfloat16, device="cuda"), torch.empty((T, H_kv, d), dtype=torch.bfloat16, device="cuda")
    api.tgvkv_rope(plan, pos, q, qo, k, ko)
    n = sum(news)
    api.tgvkv_cache_write(desc, cache, table, ln, ko[:n], v[:n], off, torch.empty_like(ln), ws)
    want = [t.clone() for t in pools_of(cache)]
    for t in pools_of(cache):
        t.view(torch.uint8).fill_(255)
    kv = qkv[:, H_q:].clone()
    api.tgvkv_rope_write(desc, cache, plan, pos, slots, q, k, v, q, ws)
    assert api.tgvkv_status(ws) == 0
    assert torch.equal(q, qo) and torch.equal(qkv[:, H_q:], kv)
    for a, b in zip(pools_of(cache), want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
