"""GPU parity of rotary positions through the C ABI, against the fp64 reference of
_rope_ref.py.

Tolerance.  An output is a (x1 c -+ x2 s) rounded to bf16: half a step, 2^-8 of the value.
Before that, c and s are within 2^-23 (the series 2^-25, their fp32 operations 2 x 2^-24
near 1) and 2^-51 of p f (the frequency's double), the products and their sum are fp32
(2^-24 each, of products at most |x1| + |x2| in all), and a is within 2^-24:
  |error| <= 2^-8 |y| + (2^-21 + 2^-50 |p| f_max) a (|x1| + |x2|).
Values that do not turn are bit copies."""
import numpy as np
import pytest
import torch

import _cache_ref as R
import _rope_ref as F

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


def values(rng, *shape):
    return R.bf16_values(R.bf16_bits(rng.standard_normal(shape)))


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def check(got, x, positions, rot, layout="half", sections=None, mode="forward", attention=1.0, freqs=None,
          **scaling):
    freqs = F.frequencies(rot, **scaling) if freqs is None else freqs
    ref = F.turned(x, positions, freqs, rot, layout, sections, attention, mode)
    a = 1.0 if mode == "move" else attention
    far = np.abs(np.asarray(positions, np.float64)).max(0)[:, None, None] * max(abs(f) for f in freqs)
    room = (2.0 ** -21 + 2.0 ** -50 * far) * a * F.partner_magnitude(x, rot, layout)
    bad = ~(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + room)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])
    assert np.array_equal(got[..., rot:], x[..., rot:])


CASES = [  # d, rot, layout: vectors of 8, 4, 2 and 1 values, whole heads and parts
    (128, 128, "half"), (128, 128, "interleaved"), (64, 64, "half"), (64, 32, "interleaved"),
    (128, 64, "half"), (128, 96, "half"), (256, 256, "half"), (256, 128, "interleaved"), (80, 80, "half"),
    (80, 40, "half"), (96, 24, "half"), (96, 24, "interleaved"), (64, 20, "half"), (64, 20, "interleaved"),
    (128, 10, "half"), (128, 2, "half"), (128, 2, "interleaved"), (8, 8, "half"), (8, 6, "half"),
    (8, 6, "interleaved"), (256, 2, "half"), (256, 254, "half")]


@pytest.mark.parametrize("d,rot,layout", CASES)
@pytest.mark.parametrize("T,H_q,H_k", [(1, 1, 0), (3, 5, 2), (37, 28, 4)])
def test_forward(api, d, rot, layout, T, H_q, H_k):
    rng = np.random.default_rng([d, rot, T])
    q, k = values(rng, T, H_q, d), values(rng, T, H_k, d)
    pos = rng.integers(0, 40000, T)
    qo = torch.full((T, H_q, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ko = torch.full((T, H_k, d), 7.0, dtype=torch.bfloat16, device="cuda")
    kk = (dev_bf16(R.bf16_bits(k)), ko) if H_k else (None, None)
    api.tgvkv_rope(api.make_rope(d, rot_dim=rot, layout=layout), ints(pos), dev_bf16(R.bf16_bits(q)), qo, *kk)
    check(R.bf16_values(host_bits(qo)), q, pos[None], rot, layout)
    if H_k:
        check(R.bf16_values(host_bits(ko)), k, pos[None], rot, layout)


@pytest.mark.parametrize("mode", ["forward", "gradient", "move"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("scaling", [dict(), dict(scaling="linear", factor=4.0),
                                     dict(scaling="base", factor=8.0, base=1e6),
                                     dict(scaling="parts", factor=8.0, original=4096, high=4.0)])
def test_modes_scalings_and_axes(api, mode, layout, scaling):
    """Three position axes, negative and large positions, an attention factor."""
    d, rot, T, H = 128, 96, 21, 3
    rng = np.random.default_rng(7)
    x, sections = values(rng, T, H, d), [8, 20, 20]
    pos = rng.integers(-(1 << 20), 1 << 20, (3, T))
    pos[:, 0] = 0
    out = torch.empty((T, H, d), dtype=torch.bfloat16, device="cuda")
    plan = api.make_rope(d, rot_dim=rot, layout=layout, sections=sections, attention=1.125, **scaling)
    api.tgvkv_rope(plan, ints(pos), dev_bf16(R.bf16_bits(x)), out, mode=mode)
    check(R.bf16_values(host_bits(out)), x, pos, rot, layout, sections, mode, 1.125, **scaling)


def test_positions_to_the_ends_of_int32_and_given_frequencies(api):
    d = 64
    rng = np.random.default_rng(3)
    pos = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30, 123456789, -987654321])
    x = values(rng, len(pos), 2, d)
    for freqs in (None, [3.0 * rng.standard_normal() for _ in range(32)]):
        out = torch.empty((len(pos), 2, d), dtype=torch.bfloat16, device="cuda")
        api.tgvkv_rope(api.make_rope(d, freqs=freqs), ints(pos), dev_bf16(R.bf16_bits(x)), out)
        check(R.bf16_values(host_bits(out)), x, pos[None], d, freqs=freqs or F.frequencies(d))


def test_quarter_turns(api):
    """Frequencies of a quarter turn: cos and sin are 0 and +-1 to within 2^-23."""
    T = 9
    x = np.zeros((T, 1, 8))
    x[..., :4], x[..., 4:] = 1.0, 3.0
    out = torch.empty((T, 1, 8), dtype=torch.bfloat16, device="cuda")
    api.tgvkv_rope(api.make_rope(8, freqs=[F.TWO_PI / 4] * 4), ints(np.arange(T) - 4),
                   dev_bf16(R.bf16_bits(x)), out)
    got = R.bf16_values(host_bits(out))
    for t in range(T):
        c, s = [(1, 0), (0, 1), (-1, 0), (0, -1)][(t - 4) % 4]
        want = np.array([c - 3 * s] * 4 + [3 * c + s] * 4, float)
        assert (np.abs(got[t, 0] - want) <= 2.0 ** -20).all(), t


def test_strides_in_place_and_untouched_neighbours(api):
    """Slices of one projection: turned into another tensor's slices, and in place."""
    T, H_q, H_k, d = 19, 6, 2, 128
    rng = np.random.default_rng(5)
    both = values(rng, T, H_q + 2 * H_k + 1, d)
    fused = dev_bf16(R.bf16_bits(both))
    pos = rng.integers(0, 9000, T)
    for layout, rot in (("half", 128), ("half", 20), ("half", 32), ("interleaved", 64), ("interleaved", 12)):
        plan = api.make_rope(d, rot_dim=rot, layout=layout)
        into = torch.full((T, 2 * H_q + H_k, d), 7.0, dtype=torch.bfloat16, device="cuda")
        q, k = fused[:, :H_q], fused[:, H_q:H_q + H_k]
        api.tgvkv_rope(plan, ints(pos), q, into[:, 0:2 * H_q:2], k, into[:, 2 * H_q:])
        got = R.bf16_values(host_bits(into))
        check(got[:, 0:2 * H_q:2], both[:, :H_q], pos[None], rot, layout)
        check(got[:, 2 * H_q:], both[:, H_q:H_q + H_k], pos[None], rot, layout)
        assert (got[:, 1:2 * H_q:2] == 7).all()
        own = fused.clone()
        q, k = own[:, :H_q], own[:, H_q:H_q + H_k]
        api.tgvkv_rope(plan, ints(pos), q, q, k, k)
        assert torch.equal(own[:, :H_q].view(torch.int16), into[:, 0:2 * H_q:2].view(torch.int16))
        assert torch.equal(own[:, H_q:H_q + H_k].view(torch.int16), into[:, 2 * H_q:].view(torch.int16))
        assert torch.equal(own[:, H_q + H_k:].view(torch.int16), fused[:, H_q + H_k:].view(torch.int16))


def test_axes_that_share_positions_and_spread_strides(api):
    """Positions expanded over the axes (stride 0), rows far apart."""
    T, H, d = 21, 3, 64
    rng = np.random.default_rng(8)
    x = values(rng, T, H, d)
    wide = torch.full((T, 5000, d), 7.0, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 2400, 4800], device="cuda")
    wide[:, at] = dev_bf16(R.bf16_bits(x)).view(T, H, d)
    src = wide[:, ::2400]
    pos = rng.integers(0, 5000, T)
    shared = ints(pos).expand(3, T)
    out = torch.full((T, 5000, d), 7.0, dtype=torch.bfloat16, device="cuda")
    plan = api.make_rope(d, sections=[4, 14, 14])
    api.tgvkv_rope(plan, shared, src, out[:, ::2400])
    got = R.bf16_values(host_bits(out[:, at]))
    check(got, x, np.broadcast_to(pos, (3, T)), d, sections=[4, 14, 14])
    out[:, at] = 7.0
    assert (out == 7).all()


@pytest.mark.parametrize("T", [1, 151, 152, 153, 609, 1217, 3650, 7301])
@pytest.mark.parametrize("H_q,H_k", [(1, 1), (2, 1), (4, 0), (33, 5), (130, 1)])
def test_tiles_of_every_depth(api, T, H_q, H_k):
    """Token counts around the tiles' depths and the CTAs' rounds; in place, so that a row
    turned twice or not at all shows."""
    d = 64
    gen = torch.Generator("cuda").manual_seed(T)
    plan, pos = api.make_rope(d, rot_dim=32), torch.arange(T, dtype=torch.int32, device="cuda") - 7
    f = torch.tensor(F.frequencies(32), dtype=torch.float64, device="cuda")
    th = pos.double()[:, None, None] * f
    c, s = th.cos(), th.sin()
    xs = [torch.randn((T, h, d), generator=gen, device="cuda").bfloat16() for h in (H_q, H_k)]
    ys = [x.clone() for x in xs]
    api.tgvkv_rope(plan, pos, ys[0], ys[0], *((ys[1], ys[1]) if H_k else ()))
    for x, y in zip(xs, ys):
        x1, x2 = x[..., :16].double(), x[..., 16:32].double()
        ref = torch.cat([x1 * c - x2 * s, x2 * c + x1 * s, x[..., 32:].double()], -1)
        room = torch.cat([(x1.abs() + x2.abs()).repeat(1, 1, 2), torch.zeros_like(ref[..., 32:])], -1) * 2.0 ** -21
        assert ((y.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + room).all()


def test_head_major_rows(api):
    """A prefill's layout [heads][T][d], as a view with the head stride above the token's."""
    T, H, d = 50, 4, 64
    rng = np.random.default_rng(6)
    x = values(rng, H, T, d)
    t, pos = dev_bf16(R.bf16_bits(x)), np.arange(T)
    out = torch.empty_like(t)
    api.tgvkv_rope(api.make_rope(d), ints(pos), t.transpose(0, 1), out.transpose(0, 1))
    check(R.bf16_values(host_bits(out)).transpose(1, 0, 2), x.transpose(1, 0, 2), pos[None], d)


@pytest.mark.parametrize("layout,rot", [("half", 64), ("half", 20), ("interleaved", 20)])
def test_values_that_do_not_turn_keep_their_bits(api, layout, rot):
    """NaN patterns, infinities and -0 past rot_dim are copied and touch nothing else; a NaN
    that turns reaches its pair alone."""
    d = 64 if rot < 64 else 128
    bits = R.bf16_bits(values(np.random.default_rng(1), 3, 2, d))
    bits[..., rot:] = [0x7FC1, 0xFFFF, 0x7F80, 0x8000][0]
    bits[0, :, rot:rot + 4] = [0x7F81, 0xFFFF, 0xFF80, 0x8000]
    bits[1, 1, 3] = 0x7FC0
    out = torch.empty((3, 2, d), dtype=torch.bfloat16, device="cuda")
    api.tgvkv_rope(api.make_rope(d, rot_dim=rot, layout=layout), ints([5, 6, 7]), dev_bf16(bits).view(3, 2, d), out)
    got = host_bits(out)
    assert np.array_equal(got[..., rot:], bits[..., rot:])
    nan = np.argwhere(np.isnan(R.bf16_values(got[..., :rot])))
    pair = [3, 3 + rot // 2] if layout == "half" else [2, 3]
    assert nan.tolist() == [[1, 1, c] for c in pair]


@pytest.mark.parametrize("layout,rot", [("half", 64), ("interleaved", 32), ("half", 12)])
def test_gradient_against_differences(api, layout, rot):
    """The map is linear: its columns are the turned unit rows.  The gradient of g is their
    products with g; an entry of a column is off by 2^-8 of itself, the gradient likewise."""
    d, p = 64, 777
    plan = api.make_rope(d, rot_dim=rot, layout=layout, attention=1.25)
    unit = torch.eye(d, device="cuda").bfloat16().view(1, d, d)
    cols = torch.empty_like(unit)
    api.tgvkv_rope(plan, ints([p]), unit, cols)
    less = torch.empty_like(unit)
    api.tgvkv_rope(plan, ints([p]), -unit, less)
    jac = (cols.double() - less.double())[0].cpu().numpy() / 2        # [j][i] = dy_i / dx_j
    g = values(np.random.default_rng(2), 1, 1, d)
    grad = torch.empty((1, 1, d), dtype=torch.bfloat16, device="cuda")
    api.tgvkv_rope(plan, ints([p]), dev_bf16(R.bf16_bits(g)).view(1, 1, d), grad, mode="gradient")
    got, want = R.bf16_values(host_bits(grad))[0, 0], jac @ g[0, 0]
    room = 2.0 ** -8 * (np.abs(jac) @ np.abs(g[0, 0]) + np.abs(got)) + 2.0 ** -20
    assert (np.abs(got - want) <= room).all()


def test_rows_moved_are_rows_turned_there(api):
    """Turned at p, moved by q - p: what turning at q gives, but for two roundings."""
    T, d = 300, 128
    rng = np.random.default_rng(4)
    x = values(rng, T, 1, d)
    p, q = rng.integers(0, 30000, T), rng.integers(0, 3000, T)
    plan = api.make_rope(d, attention=1.5)
    a, b, c = (torch.empty((T, 1, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    api.tgvkv_rope(plan, ints(p), dev_bf16(R.bf16_bits(x)), a)
    api.tgvkv_rope(plan, ints(q - p), a, b, mode="move")
    api.tgvkv_rope(plan, ints(q), dev_bf16(R.bf16_bits(x)), c)
    got, want = R.bf16_values(host_bits(b)), R.bf16_values(host_bits(c))
    # a's two values are off by 2^-8 of themselves, b and c by 2^-8 of theirs
    pair = F.partner_magnitude(R.bf16_values(host_bits(a)), d)
    assert (np.abs(got - want) <= 2.0 ** -8 * (pair * (1 + 2.0 ** -8) + np.abs(got) + np.abs(want)) + 2.0 ** -19).all()


@pytest.mark.parametrize("T,H_q,H_k", [(8704, 28, 4), (20001, 1, 0), (700, 64, 64), (5, 2000, 0)])
def test_many_rows(api, T, H_q, H_k):
    """Grids of every shape against torch's arithmetic in 64 bits."""
    d = 128
    gen = torch.Generator("cuda").manual_seed(T)
    plan, pos = api.make_rope(d, base=1e6), torch.arange(T, dtype=torch.int32, device="cuda") + 11
    f = torch.tensor(F.frequencies(d, base=1e6), dtype=torch.float64, device="cuda")
    th = pos.double()[:, None, None] * f
    c, s = th.cos(), th.sin()
    xs = [torch.randn((T, h, d), generator=gen, device="cuda").bfloat16() for h in (H_q, H_k)]
    ys = [torch.full_like(x, float("nan")) for x in xs]
    api.tgvkv_rope(plan, pos, xs[0], ys[0], *((xs[1], ys[1]) if H_k else ()))
    for x, y in zip(xs, ys):
        x1, x2 = x.double().chunk(2, -1)
        ref = torch.cat([x1 * c - x2 * s, x2 * c + x1 * s], -1)
        room = (x1.abs() + x2.abs()).repeat(1, 1, 2) * 2.0 ** -21
        assert ((y.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + room).all()


def test_no_tokens_other_streams_and_graphs(api):
    plan = api.make_rope(64)
    empty = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    api.tgvkv_rope(plan, ints([]), empty, empty)
    x = dev_bf16(R.bf16_bits(values(np.random.default_rng(0), 33, 4, 64)))
    pos, want = ints(np.arange(33)), torch.empty_like(x)
    api.tgvkv_rope(plan, pos, x, want)
    side, out = torch.cuda.Stream(), torch.zeros_like(x)
    side.wait_stream(torch.cuda.current_stream())
    api.tgvkv_rope(plan, pos, x, out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph, src = torch.cuda.CUDAGraph(), torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        api.tgvkv_rope(plan, pos, src, out)
    plan = None                        # the launch holds its own copy
    src.copy_(x)
    out.zero_()
    graph.replay()
    assert torch.equal(out, want)
