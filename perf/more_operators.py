"""Cases that measure a serving step around the paged cache: pages for new tokens, rotary
positions, keys and values rotated into the pages, and pages that hold 4-bit floats.

Pages.  Set s = b * H_kv + g (sequence b, KV head g) holds ceil(lens[s] / page) pages of a pool,
named by the first entries of its table row; the free pages are a stack of which n_free are left.
n tokens of sequence b take the pages they lack from the top of the stack, set after set; token t
of head g then has the slot table[s][j // page] * page + j % page, j = lens[s] + its place among the
sequence's new tokens.  Giving pages back puts them on the stack in the opposite order.

Rotary positions.  A pair (x1, x2) of a row at position p turns by the angle p * f:
(x1 c - x2 s, x2 c + x1 s), times an attention factor.  Pair i of a rotated part of r values is
values (i, i + r / 2) or (2 i, 2 i + 1); f_i = base^(-2 i / r), or that scaled for long contexts;
pairs may follow different position axes (time, height, width).  Modes: "forward"; "gradient", the
transposed map; "move", a forward turn by differences of positions, without the factor.

4-bit floats.  32 consecutive values share a scale 2^e, the smallest with max |x| <= 6 * 2^e and
-60 <= e <= 56, stored as the byte e + 127; codes are the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a
sign (ties to the even code), two to a byte, the even element in the low half.

Attention: token i of the n new tokens of sequence b (the last n of the set's len slots) attends to
slots 0 .. len - n + i.
"""
import math

import torch

own = False

GROUP = 32


# ---------------------------------------------------------------------------- cases
def listed():
    return [
        # a decode step of 64 requests (qwen25 heads): one token each, a page for every 16th of
        # them, and the slots to write; latency only
        dict(name="pages_token", kind="pages", B=64, H_kv=4, page=16, n=1, len=461, ragged=True),
        # a batch of 64 long prompts admitted at once, tables and slots built from their lengths
        dict(name="pages_prompts", kind="pages", B=64, H_kv=4, page=64, n=8704, len=0, ragged=True),
        # the smallest rotary call: one token's queries and keys
        dict(name="rope_token", kind="rope", T=1, H_q=28, H_kv=4, d=128, rot=128, layout="half",
             axes=1, scaling="none", mode="forward", strided=True, far=40000),
        # a video prompt's queries and keys on three position axes, as slices of one projection
        dict(name="rope_prompt_axes", kind="rope", T=8704, H_q=28, H_kv=4, d=128, rot=128,
             layout="half", axes=3, scaling="none", mode="forward", strided=True, far=20000),
        # kept rows of an eviction (llava15: 32 x 32 sets) moved to their places in the cache
        dict(name="rope_rows_moved", kind="rope", T=220161, H_q=1, H_kv=0, d=128, rot=128,
             layout="half", axes=1, scaling="none", mode="move", strided=False, far=3000),
        # gradients of an odd-length batch, neighbouring pairs in half of the head, a long context
        dict(name="rope_gradient_part", kind="rope", T=16381, H_q=32, H_kv=8, d=128, rot=64,
             layout="interleaved", axes=1, scaling="parts", mode="gradient", strided=False,
             far=1000000),
        # a decode step of 64 requests: queries rotated, keys and values into bf16 pages
        dict(name="rope_append_token", kind="rope_append", B=64, H_q=28, H_kv=4, d=128, page=16,
             fmt="bf16", n=1, len=461, ragged=True, rot=128, layout="half", axes=3,
             scaling="none", far=20000),
        # sixteen prompts rotated into 8-bit pages, which are read back
        dict(name="rope_store_int8", kind="rope_store", B=16, H_q=32, H_kv=8, d=128, page=64,
             fmt="int8", n=4099, len=0, ragged=True, rot=128, layout="half", axes=1,
             scaling="parts", far=100000),
        # a video prompt's K and V of all 28 layers stored as 4-bit floats and read back
        dict(name="store_prompt_fp4", kind="store", B=28, H_q=28, H_kv=4, d=128, page=128,
             fmt="fp4", n=8704, len=0, ragged=False),
        # a batch of decode steps over long video caches in 4-bit floats
        dict(name="token_batch_fp4", kind="attend", B=64, H_q=28, H_kv=4, d=128, page=64,
             fmt="fp4", n=1, len=8705, ragged=True),
        # five drafted tokens a sequence checked at once, d = 64
        dict(name="draft_fp4", kind="attend", B=32, H_q=32, H_kv=8, d=64, page=32, fmt="fp4",
             n=5, len=4101, ragged=True),
        # a serving batch with prompt chunks of up to 500 tokens, single tokens and idle sequences
        dict(name="mixed_fp4", kind="attend", B=16, H_q=28, H_kv=4, d=128, page=32, fmt="fp4",
             n=500, len=8900, ragged=True),
    ]


_HEADS = ((8, 8), (32, 32), (28, 4), (32, 8), (16, 2), (12, 1), (6, 2))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.8e12, w["flops"] / 1.9e15)


def _draw_rotary(rng, d):
    rot = rng.choice([d, d, d, d // 2, d // 4, 3 * d // 4 // 16 * 16])
    return dict(rot=rot, layout=rng.choice(["half", "interleaved"]), axes=rng.choice([1, 1, 2, 3]),
                scaling=rng.choice(["none", "linear", "base", "parts"]),
                far=rng.choice([1000, 40000, 1000000]))


def draw(rng):
    def log(lo, hi):
        return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))

    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["pages", "rope", "rope", "rope_append", "rope_store", "store", "attend",
                           "attend"])
        H_q, H_kv = rng.choice(_HEADS)
        B, page = log(1, 64), rng.choice([16, 32, 64, 128, 256])
        ragged, d = rng.random() < 0.7, rng.choice([64, 128, 128])
        ln = rng.choice([0, log(1, 9000)])
        if kind == "pages":
            case = dict(kind=kind, B=B, H_kv=H_kv, page=page, n=log(1, 9000), len=ln, ragged=ragged)
        elif kind == "rope":
            d = rng.choice([64, 80, 96, 128, 128, 256])
            case = dict(kind=kind, T=log(1, 200000), H_q=H_q, H_kv=rng.choice([0, H_kv, H_kv]), d=d,
                        mode=rng.choice(["forward", "forward", "gradient", "move"]),
                        strided=rng.random() < 0.5, **_draw_rotary(rng, d))
        elif kind in ("rope_append", "rope_store"):
            case = dict(kind=kind, B=B, H_q=H_q, H_kv=H_kv, d=d, page=page,
                        fmt="bf16" if kind == "rope_append" else rng.choice(["bf16", "int8"]),
                        n=log(1, 300) if kind == "rope_append" else log(1, 9000), len=ln,
                        ragged=ragged, **_draw_rotary(rng, d))
        elif kind == "store":
            case = dict(kind=kind, B=B, H_q=H_q, H_kv=H_kv, d=d, page=page, fmt="fp4",
                        n=log(1, 9000), len=ln, ragged=ragged)
        else:
            n = rng.choice([1, 1, log(2, 12), log(13, 2048)])
            case = dict(kind=kind, B=B, H_q=H_q, H_kv=H_kv, d=d, page=page, fmt="fp4", n=n,
                        len=n + log(1, 33000), ragged=ragged)
        # no costlier than the largest listed case, and its plain form fits the card several times
        rows = sum(_news(case)) * (H_q + 2 * H_kv) if kind != "rope" else case["T"] * (H_q + H_kv)
        plain = 40 * rows * d
        if kind == "attend":
            plain += 24 * B * H_kv * case["len"] * d + 14 * B * H_q * n * case["len"]
        if _cost(case) <= most and plain < 48e9:
            return case


def _lens(case):
    """Slots of every set before the call, or in all (attend)."""
    S, ln = case["B"] * case["H_kv"], case["len"]
    if not case["ragged"]:
        return [ln] * S
    return [ln - (s * 40503 % 65536) * (ln // 2) // 65536 for s in range(S)]


def _news(case):
    """New tokens of every sequence."""
    if case["kind"] == "rope":
        return [case["T"]]
    B, n = case["B"], case["n"]
    if not case["ragged"]:
        return [n] * B
    if case["kind"] == "attend":
        if n <= 12:     # decode steps and drafts: every sequence has its tokens
            return [n] * B
        # full chunks, shorter ones, single tokens and an idle sequence
        return [(n, n - n // 3, 1, n // 2 + 1, 0, n - 1)[b % 6] for b in range(B)]
    return [n - (b * 30011 % 65536) * (n // 2) // 65536 for b in range(B)]


def _sizes(case):
    S, H_kv = case["B"] * case["H_kv"], case["H_kv"]
    lens, news = _lens(case), _news(case)
    per_set = [news[s // H_kv] for s in range(S)]
    total = lens if case["kind"] == "attend" else [a + b for a, b in zip(lens, per_set)]
    max_pages = max(1, -(-max(total) // case["page"]))
    return S, lens, news, per_set, total, max_pages


def _row_bytes(d, fmt):
    return {"bf16": 2 * d, "int8": d + d // GROUP, "fp4": d // 2 + d // GROUP}[fmt]


def work(case):
    kind = case["kind"]
    if kind == "rope":
        rows, pairs = case["T"] * (case["H_q"] + case["H_kv"]), case["rot"] // 2
        return {"bytes": 4 * rows * case["d"] + 4 * case["axes"] * case["T"],
                "flops": rows * pairs * 6}
    S, lens, news, per_set, total, _ = _sizes(case)
    ps, T = case["page"], sum(news)
    if kind == "pages":
        taken = sum(-(-t // ps) - -(-ln // ps) for t, ln in zip(total, lens))
        # lengths in and out, free pages read, tables and slots written; and the way back
        return {"bytes": 4 * (3 * S + 2 * taken + T * case["H_kv"]) + 4 * (2 * S + 3 * taken),
                "flops": 4 * T * case["H_kv"]}
    d, G, row = case["d"], case["H_q"] // case["H_kv"], _row_bytes(case["d"], case["fmt"])
    pages = sum(-(-t // ps) for t in total)
    if kind == "attend":
        kv, pairs = 0, 0
        for n, t in zip(per_set, total):
            if n == 0:
                continue
            kv += t
            low, vis = max(0, t - n), min(n, t)
            pairs += G * (vis * low + vis * (vis + 1) // 2)
        return {"bytes": 2 * kv * row + 2 * T * case["H_q"] * d * 2 + 4 * (S + pages),
                "flops": 4 * d * pairs}
    rows = sum(per_set)
    back = 0 if kind == "rope_append" else rows * (row + 2 * d)      # the store is read back
    move = 2 * (rows * (2 * d + row) + back) + 4 * (S + pages)
    if kind == "store":
        return {"bytes": move, "flops": 6 * rows * d}
    return {"bytes": move + T * case["H_q"] * d * 4 + 4 * T * (case["axes"] + case["H_kv"]),
            "flops": 3 * (T * case["H_q"] + rows) * case["rot"] + 6 * rows * d}


# ---------------------------------------------------------------------------- rotary
_BASE = 1000000.0
# kind -> what a caller states of it: positions scaled by 4, a base enlarged for 4 times the
# length, or the slow pairs alone scaled (fewer than 32 turns over 4096 positions: in part, fewer
# than 1: in full), with an attention factor
_SCALING = {"none": {}, "linear": dict(factor=4.0), "base": dict(factor=4.0),
            "parts": dict(factor=8.0, original=4096, low=1.0, high=32.0,
                          attention=0.1 * math.log(8.0) + 1.0)}


def _sections(case):
    """Pairs of every position axis."""
    half, a = case["rot"] // 2, case["axes"]
    first = half // (a + 1) if a > 1 else half       # fewer for time than for height and width
    rest = half - first
    return [first] + [rest // (a - 1) + (1 if i < rest % (a - 1) else 0) for i in range(a - 1)]


def _frequencies(case, device="cuda"):
    """Radians a position of every pair (fp64), and the factor of the rotated values."""
    rot, kind = case["rot"], case["scaling"]
    o, base = _SCALING[kind], _BASE
    if kind == "base":
        base = base * o["factor"] ** (rot / (rot - 2)) if rot > 2 else base
    i = torch.arange(rot // 2, dtype=torch.float64, device=device)
    f = torch.pow(torch.tensor(base, dtype=torch.float64, device=device), -2.0 * i / rot)
    if kind == "linear":
        f = f / o["factor"]
    if kind == "parts":
        turns = o["original"] * f / (2 * math.pi)
        keep = ((turns - o["low"]) / (o["high"] - o["low"])).clamp(0.0, 1.0)
        f = f * keep + f / o["factor"] * (1.0 - keep)
    return f, o.get("attention", 1.0)


# ---------------------------------------------------------------------------- formats
def _pow2(e):
    """2^e in fp32, exactly, for integers e in [-126, 127]."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


_TOP = {"int8": (127, 7, -126, 122), "fp4": (6, 3, -60, 56)}     # largest code, its bits, e's range


def _encode(x, fmt):
    """fp32 rows [..., d] as stored rows and scale bytes (uint8 [..., d / 32])."""
    q_max, bits, e_min, e_max = _TOP[fmt]
    g = x.unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    m, e = torch.frexp(top)                                   # top = m 2^e, m in [0.5, 1)
    e = (e - bits + (m > q_max / 2 ** bits).to(e.dtype)).clamp(e_min, e_max)
    y = (g * _pow2(-e).unsqueeze(-1)).clamp(-q_max, q_max).flatten(-2)
    byte = (e + 127).to(torch.uint8)
    if fmt == "int8":
        return y.round().to(torch.int8), byte
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (a / step).round() * step
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = code + 8 * torch.signbit(y).to(torch.uint8)
    code = code.unflatten(-1, (-1, 2))
    return code[..., 0] | (code[..., 1] << 4), byte


def _decode(rows, byte, fmt):
    """Stored rows as fp32 values."""
    if fmt == "bf16":
        return rows.float()
    if fmt == "int8":
        y = rows.float()
    else:
        code = torch.stack((rows & 15, rows >> 4), -1).flatten(-2)
        m = (code & 7).float()
        a = torch.where(m < 4, m / 2, torch.where(m < 6, m - 2, 2 * m - 8))
        y = torch.where(code > 7, -a, a)
    return (y.unflatten(-1, (-1, GROUP)) * _pow2(byte.to(torch.int32) - 127).unsqueeze(-1)).flatten(-2)


# ---------------------------------------------------------------------------- inputs
def _values(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _keys(gen, rows, d):
    """Keys with a few large channels, as real key caches have."""
    k = _values(gen, rows, d)
    k[:, torch.randperm(d, generator=gen, device="cuda")[:4]] *= 8.0
    return k


def _positions(gen, case, news):
    """int32 [axes, T]: every sequence goes on from a place of its own; later axes vary slower."""
    T, far = sum(news), case["far"]
    if case.get("mode") == "move":       # differences of positions: rows move down
        return -torch.randint(0, far, (case["axes"], T), generator=gen, device="cuda", dtype=torch.int32)
    n = torch.tensor(news, device="cuda")
    start = torch.randint(0, far, (len(news),), generator=gen, device="cuda")
    first = (start - (n.cumsum(0) - n)).repeat_interleave(n)
    p = torch.arange(T, device="cuda") + first
    return torch.stack([p - p % (a * 7 + 1) for a in range(case["axes"])]).to(torch.int32).contiguous()


def _prepare_rope(s, case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T, H_q, H_kv, d = case["T"], case["H_q"], case["H_kv"], case["d"]
    if case["strided"]:
        fused = _values(gen, T, H_q + 2 * max(H_kv, 1), d).bfloat16()
        s["q"] = fused[:, :H_q]
        s["k"] = fused[:, H_q:H_q + H_kv] if H_kv else None
    else:
        s["q"] = _values(gen, T, H_q, d).bfloat16()
        s["k"] = _values(gen, T, H_kv, d).bfloat16() if H_kv else None
    s["positions"] = _positions(gen, case, [T])
    s["q_out"] = torch.empty(T, H_q, d, dtype=torch.bfloat16, device="cuda")
    s["k_out"] = torch.empty(T, H_kv, d, dtype=torch.bfloat16, device="cuda") if H_kv else None


def _rotary(s, case):
    s["d"], s["rot"], s["layout"] = case["d"], case["rot"], case["layout"]
    s["freqs"], s["attention"] = _frequencies(case)
    s["axis"] = torch.tensor([a for a, n in enumerate(_sections(case)) for _ in range(n)], device="cuda")
    if own:
        from paper_2606_03075_gb300 import api
        o = dict(_SCALING[case["scaling"]])
        s["rope"] = api.make_rope(case["d"], rot_dim=case["rot"], base=_BASE, layout=case["layout"],
                                  sections=_sections(case), scaling=case["scaling"], **o)


def prepare(case, seed):
    kind = case["kind"]
    s = {"kind": kind, "mode": case.get("mode", "forward")}
    if "rot" in case:
        _rotary(s, case)
    if kind == "rope":
        _prepare_rope(s, case, seed)
        return s
    gen = torch.Generator(device="cuda").manual_seed(seed)
    S, lens, news, per_set, total, max_pages = _sizes(case)
    B, H_kv, ps = case["B"], case["H_kv"], case["page"]
    T, n_pages = sum(news), S * max_pages
    i32 = dict(dtype=torch.int32, device="cuda")
    s |= {"page": ps, "H_kv": H_kv, "lens": torch.tensor(lens, **i32), "max_len": max(total),
          "n_max": max(news)}
    off = torch.tensor([0] + news, dtype=torch.int64, device="cuda").cumsum(0)
    s["tok_offsets"] = off.to(torch.int32)
    pages = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    if kind == "pages":
        # the pages of what the sets hold, and the others free
        table = pages.view(S, max_pages)
        free = torch.arange(max_pages, device="cuda") >= ((s["lens"] + ps - 1) // ps)[:, None]
        s["n_free"] = free.sum().to(torch.int32).view(1)
        s["free"] = torch.cat([table[free], table[~free]])
        s["page_table"] = torch.where(free, -1, table).to(torch.int32)
        s["slots"] = torch.empty(T, H_kv, **i32)
        s["lens_out"] = torch.empty(S, **i32)
        if own:
            from paper_2606_03075_gb300 import api
            s["desc"] = api.make_cache_desc(B, H_kv, H_kv, 128, ps, n_pages, max_pages)
            s["pages"] = api.PageList(s["page_table"], s["free"], s["n_free"])
            s["ws"] = api.new_cache_workspace(s["desc"])
        return s
    H_q, d, fmt = case["H_q"], case["d"], case["fmt"]
    s |= {"H_q": H_q, "d": d, "fmt": fmt, "page_table": pages.view(S, max_pages), "cache": {}}
    # the pool: random rows where the call reads them, zeros where it writes them
    words = {"bf16": (d, torch.bfloat16), "int8": (d, torch.int8), "fp4": (d // 2, torch.uint8)}[fmt]
    for name in ("k", "v"):
        if kind == "attend":
            rows = _keys(gen, n_pages * ps, d) if name == "k" else _values(gen, n_pages * ps, d)
            pool, byte = _encode(rows, fmt)
            del rows
        else:
            pool = torch.zeros(n_pages * ps, words[0], dtype=words[1], device="cuda")
            byte = None if fmt == "bf16" else torch.zeros(n_pages * ps, d // GROUP,
                                                          dtype=torch.uint8, device="cuda")
        s["cache"][name] = pool.view(n_pages, ps, words[0])
        s["cache"][name + "_scale"] = None if byte is None else byte.view(n_pages, ps, d // GROUP)
    if kind == "attend":
        s["q"] = _values(gen, T, H_q, d).bfloat16()
        s["out"] = torch.empty(T, H_q, d, dtype=torch.bfloat16, device="cuda")
    else:
        # Q, K and V as slices of one fused projection's output
        fused = _values(gen, T, H_q + 2 * H_kv, d)
        fused[:, H_q:H_q + H_kv, :4] *= 4.0
        s["q"], s["k_new"], s["v_new"] = fused.bfloat16().split([H_q, H_kv, H_kv], dim=1)
        s["lens_out"] = torch.empty(S, **i32)
    if kind in ("rope_append", "rope_store"):
        s["positions"] = _positions(gen, case, news)
        s["q_out"] = torch.empty(T, H_q, d, dtype=torch.bfloat16, device="cuda")
        s["slots"] = _slots(s)
    if kind in ("store", "rope_store"):
        s["rows"] = sum(per_set)
        s["read_offsets"] = torch.tensor([0] + per_set, dtype=torch.int64, device="cuda").cumsum(0)
        s["k_out"] = torch.empty(s["rows"], d, dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.empty(s["rows"], d, dtype=torch.bfloat16, device="cuda")
    if own:
        from paper_2606_03075_gb300 import api
        s["desc"] = api.make_cache_desc(B, H_q, H_kv, d, ps, n_pages, max_pages, format=fmt)
        s["paged"] = api.PagedCache(**s["cache"])
        s["ws"] = api.new_cache_workspace(s["desc"])
    return s


# ---------------------------------------------------------------------------- plain forms
def _csr(offsets, rows):
    """Set and position in the set of each of the CSR's rows."""
    r = torch.arange(rows, device="cuda")
    sets = torch.searchsorted(offsets, r, right=True) - 1
    return sets, r - offsets[sets]


def _slots(s):
    """Pool row of every new token and KV head [T, H_kv]."""
    H_kv, ps, T = s["H_kv"], s["page"], s["slots"].shape[0] if "slots" in s else s["q"].shape[0]
    seq, at = _csr(s["tok_offsets"].long(), T)
    sets = seq[:, None] * H_kv + torch.arange(H_kv, device="cuda")
    j = s["lens"][sets].long() + at[:, None]
    return (s["page_table"][sets, j // ps].long() * ps + j % ps).to(torch.int32)


def _plain_pages(s):
    table, free, ps, H_kv = s["page_table"], s["free"], s["page"], s["H_kv"]
    n_pages = free.shape[0]
    new = s["lens"] + s["tok_offsets"].diff().repeat_interleave(H_kv)
    held, want = (s["lens"] + ps - 1) // ps, (new + ps - 1) // ps
    take = (want - held).clamp(min=0).long()
    before, left = take.cumsum(0) - take, s["n_free"].long()
    col = torch.arange(table.shape[1], device="cuda")
    mine = (col >= held[:, None]) & (col < want[:, None])
    at = left - 1 - (before[:, None] + col - held[:, None])
    table.copy_(torch.where(mine, free[at.clamp(0, n_pages - 1)], table))
    s["n_free"].sub_(take.sum().to(torch.int32))
    s["slots"].copy_(_slots(s))
    s["lens_out"].copy_(new)
    # ... and when the tokens are done with
    left = s["n_free"].long()
    at = left + take.sum() - 1 - (before[:, None] + col - held[:, None])
    more = torch.cat([free, free[:1]])               # one entry more, for what is not given back
    more[torch.where(mine, at, n_pages).flatten()] = table.flatten()
    free.copy_(more[:n_pages])
    table.masked_fill_(mine, -1)
    s["n_free"].add_(take.sum().to(torch.int32))


def _plain_rotate(s, x):
    """Rows [T, heads, d] rotated, in fp32."""
    half, x = s["rot"] // 2, x.float()
    angle = s["positions"][s["axis"]].double().T * s["freqs"]                 # [T, rot / 2]
    sign, factor = (-1.0 if s["mode"] == "gradient" else 1.0), (1.0 if s["mode"] == "move" else s["attention"])
    c = (angle.cos() * factor).float().unsqueeze(1)
    t = (angle.sin() * (factor * sign)).float().unsqueeze(1)
    y, part = x.clone(), x[..., :s["rot"]]
    if s["layout"] == "half":
        x1, x2 = part[..., :half], part[..., half:]
        y[..., :half], y[..., half:s["rot"]] = x1 * c - x2 * t, x2 * c + x1 * t
    else:
        x1, x2 = part[..., 0::2], part[..., 1::2]
        y[..., 0:s["rot"]:2], y[..., 1:s["rot"]:2] = x1 * c - x2 * t, x2 * c + x1 * t
    return y


def _plain_write(s, k):
    """Rows k and s["v_new"], [T, H_kv, d], into the pages."""
    rows, c, fmt = _slots(s).long().flatten(), s["cache"], s["fmt"]
    for name, x in (("k", k), ("v", s["v_new"])):
        x = x.flatten(0, 1)
        if fmt == "bf16":
            c[name].flatten(0, 1)[rows] = x
        else:
            code, byte = _encode(x.float(), fmt)
            c[name].flatten(0, 1)[rows] = code
            c[name + "_scale"].flatten(0, 1)[rows] = byte


def _values_at(s, name, rows):
    c, byte = s["cache"][name].flatten(0, 1)[rows], s["cache"][name + "_scale"]
    return _decode(c, None if byte is None else byte.flatten(0, 1)[rows], s["fmt"])


def _plain_read(s):
    sets, at = _csr(s["read_offsets"], s["rows"])
    j = at + s["lens"][sets]
    rows = s["page_table"][sets, j // s["page"]].long() * s["page"] + j % s["page"]
    s["k_out"].copy_(_values_at(s, "k", rows))
    s["v_out"].copy_(_values_at(s, "v", rows))


def _plain_attend(s):
    H_q, H_kv, d, ps = s["H_q"], s["H_kv"], s["d"], s["page"]
    S, M, n_max = s["lens"].shape[0], s["max_len"], s["n_max"]
    B, G = S // H_kv, H_q // H_kv
    slots = torch.arange(M, device="cuda")
    rows = s["page_table"][:, slots // ps].long() * ps + slots % ps                # [S, M]
    off = s["tok_offsets"].long()
    n = off.diff()
    seq, at = _csr(off, s["q"].shape[0])
    q = torch.zeros(B, n_max, H_q, d, device="cuda")
    q[seq, at] = s["q"].float()
    q = q.view(B, n_max, H_kv, G, d).permute(0, 2, 1, 3, 4).reshape(S, n_max * G, d)
    x = torch.bmm(q, _values_at(s, "k", rows).transpose(1, 2))                     # [S, n G, M]
    x.mul_(1.0 / d ** 0.5)
    last = s["lens"].view(B, H_kv, 1) - n.view(B, 1, 1) + torch.arange(n_max, device="cuda")
    hidden = slots > last.reshape(S, n_max, 1)
    x.view(S, n_max, G, M).masked_fill_(hidden.unsqueeze(2), float("-inf"))
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(torch.isfinite(top), top, torch.zeros_like(top))).exp_()
    mass = x.sum(-1, keepdim=True)
    o = torch.bmm(x, _values_at(s, "v", rows)) / torch.where(mass > 0, mass, torch.ones_like(mass))
    o = o.view(B, H_kv, n_max, G, d).permute(0, 2, 1, 3, 4).reshape(B, n_max, H_q, d)
    s["out"].copy_(o[seq, at])


def run(s):
    kind = s["kind"]
    if own:
        from paper_2606_03075_gb300 import api
        if kind == "pages":
            api.tgvkv_pages_append(s["desc"], s["pages"], s["lens"], s["tok_offsets"], s["slots"],
                                   s["lens_out"], s["ws"])
            api.tgvkv_pages_shrink(s["desc"], s["pages"], s["lens_out"], s["lens"], s["ws"])
        if kind == "rope":
            api.tgvkv_rope(s["rope"], s["positions"], s["q"], s["q_out"], s["k"], s["k_out"],
                           mode=s["mode"])
        if kind in ("rope_append", "rope_store"):
            api.tgvkv_rope_write(s["desc"], s["paged"], s["rope"], s["positions"], s["slots"],
                                 s["q"], s["k_new"], s["v_new"], s["q_out"], s["ws"])
        if kind == "store":
            api.tgvkv_cache_write(s["desc"], s["paged"], s["page_table"], s["lens"], s["k_new"],
                                  s["v_new"], s["tok_offsets"], s["lens_out"], s["ws"])
        if kind in ("store", "rope_store"):
            api.tgvkv_cache_read(s["desc"], s["paged"], s["page_table"], s["lens"],
                                 s["read_offsets"], s["k_out"], s["v_out"], s["ws"])
        if kind == "attend":
            api.tgvkv_chunk_attention(s["desc"], s["paged"], s["page_table"], s["lens"], s["q"],
                                      s["tok_offsets"], s["n_max"], s["out"], s["ws"])
    else:
        if kind == "pages":
            _plain_pages(s)
        if kind == "rope":
            s["q_out"].copy_(_plain_rotate(s, s["q"]))
            if s["k"] is not None:
                s["k_out"].copy_(_plain_rotate(s, s["k"]))
        if kind in ("rope_append", "rope_store"):
            s["q_out"].copy_(_plain_rotate(s, s["q"]))
            _plain_write(s, _plain_rotate(s, s["k_new"]).bfloat16())   # a key enters the cache in bf16
        if kind == "store":
            _plain_write(s, s["k_new"])
            s["lens_out"].copy_(s["lens"] + s["tok_offsets"].diff().repeat_interleave(s["H_kv"]))
        if kind in ("store", "rope_store"):
            _plain_read(s)
        if kind == "attend":
            _plain_attend(s)
    if kind == "pages":
        return {n: s[n] for n in ("page_table", "free", "n_free", "slots", "lens_out")}
    if kind == "rope":
        return {n: s[n] for n in ("q_out", "k_out") if s[n] is not None}
    if kind == "rope_append":
        return {"q": s["q_out"], "k": s["cache"]["k"], "v": s["cache"]["v"]}
    if kind == "rope_store":
        return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
    if kind == "store":
        return {"k": s["k_out"], "v": s["v_out"], "lens": s["lens_out"]}
    return {"out": s["out"]}


# ---------------------------------------------------------------------------- in 64 bits
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_turned(case, x, positions, mode):
    """Rows [T, heads, d] turned by complex numbers, in float64."""
    T, heads, d = x.shape
    half = case["rot"] // 2
    f, factor = _frequencies(case)
    turn = torch.empty(T, half, dtype=torch.complex128, device="cuda")
    first = 0
    for a, n in enumerate(_sections(case)):
        turn[:, first:first + n] = torch.polar(
            torch.ones(T, n, dtype=torch.float64, device="cuda"),
            positions[a].double()[:, None] * f[None, first:first + n])
        first += n
    if mode == "gradient":
        turn = turn.conj()
    turn = turn * (1.0 if mode == "move" else factor)
    y = x.double().clone()
    for h in range(heads):
        r = x[:, h, :case["rot"]].double()
        z = torch.complex(*((r[:, :half], r[:, half:]) if case["layout"] == "half" else
                            (r[:, ::2].contiguous(), r[:, 1::2].contiguous()))) * turn
        if case["layout"] == "half":
            y[:, h, :half], y[:, h, half:2 * half] = z.real, z.imag
        else:
            y[:, h, :2 * half] = torch.view_as_real(z).reshape(T, 2 * half)
    return y


def _exact_stored(x, fmt):
    """What a row of bf16 values (float64 here) reads back as."""
    if fmt == "bf16":
        return x
    most, _, e_min, e_max = _TOP[fmt]
    g = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    top = g.abs().max(dim=-1, keepdim=True).values
    e = torch.full_like(top, float(e_max))
    guess = torch.ceil(torch.log2(top / most)).nan_to_num(neginf=float(e_min))
    for t in (guess + 1, guess, guess - 1):      # from above: the smallest that holds
        t = t.clamp(e_min, e_max)
        e = torch.where(top <= most * torch.exp2(t), t, e)
    y = (g / torch.exp2(e)).clamp(-most, most)
    if fmt == "int8":
        y = y.round()
    else:
        levels = torch.tensor(_E2M1, dtype=torch.float64, device="cuda")
        a = y.abs()
        hi = torch.bucketize(a, levels).clamp(max=7)          # the first level not below
        lo = (hi - 1).clamp(min=0)
        up, down = levels[hi] - a, a - levels[lo]
        pick = torch.where(up < down, hi, torch.where(down < up, lo, torch.where(hi % 2 == 0, hi, lo)))
        y = torch.where(y < 0, -levels[pick], levels[pick])
    return (y * torch.exp2(e)).reshape(x.shape)


def exact(case, seed):
    kind = case["kind"]
    if kind == "pages":
        return None                              # whole numbers only
    if kind in ("rope_store", "rope_append", "rope", "store") and work(case)["bytes"] > 12e9:
        return None
    s = prepare(case, seed)
    if kind == "rope":
        got = {"q_out": _exact_turned(case, s["q"], s["positions"], s["mode"])}
        if s["k"] is not None:
            got["k_out"] = _exact_turned(case, s["k"], s["positions"], s["mode"])
        return got
    S, lens, news, per_set, total, _ = _sizes(case)
    H_kv, G, d, ps = case["H_kv"], case["H_q"] // case["H_kv"], case["d"], case["page"]
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    if kind == "attend":
        if work(case)["flops"] > 2e12 or sum(total) > 4_000_000:
            return None
        signed = torch.tensor(_E2M1 + [-x for x in _E2M1], dtype=torch.float64, device="cuda")

        def stored(name, i):
            j = torch.arange(total[i], device="cuda")
            page, row = s["page_table"][i, j // ps].long(), j % ps
            u = s["cache"][name][page, row].long()
            q = torch.empty(total[i], d, dtype=torch.float64, device="cuda")
            q[:, 0::2], q[:, 1::2] = signed[u % 16], signed[u // 16]
            e = s["cache"][name + "_scale"][page, row].double() - 127
            return q * torch.exp2(e).repeat_interleave(GROUP, dim=1)

        out = torch.zeros(sum(news), case["H_q"], d, dtype=torch.float64, device="cuda")
        for i in range(S):
            b, g = divmod(i, H_kv)
            n, t0 = news[b], starts[b]
            if n == 0:
                continue
            k, v = stored("k", i), stored("v", i)
            seen = total[i] - n + 1 + torch.arange(n, device="cuda")
            hide = torch.arange(total[i], device="cuda")[None, :] >= seen[:, None]
            for h in range(g * G, (g + 1) * G):
                x = s["q"][t0:t0 + n, h].double() @ k.T / math.sqrt(d)
                p = torch.softmax(x.masked_fill_(hide, float("-inf")), dim=-1)
                out[t0:t0 + n, h] = torch.where((seen > 0)[:, None], p @ v, 0.0)
        return {"out": out}
    k, v = s["k_new"].double(), s["v_new"].double()
    got = {}
    if kind != "store":
        got["q"] = _exact_turned(case, s["q"], s["positions"], "forward")
        # a key is rounded to bf16 before it is stored
        k = _exact_turned(case, s["k_new"], s["positions"], "forward")
        k = k if case["fmt"] == "bf16" else k.bfloat16().double()
    for name, x in (("k", _exact_stored(k, case["fmt"])), ("v", _exact_stored(v, case["fmt"]))):
        if kind == "rope_append":
            got[name] = s["cache"][name].double()
            for i in range(S):
                b, g = divmod(i, H_kv)
                j = torch.arange(lens[i], total[i], device="cuda")
                got[name][s["page_table"][i, j // ps].long(), j % ps] = x[starts[b]:starts[b + 1], g]
        else:       # token-major in, set after set out
            got[name] = torch.cat([x[starts[i // H_kv]:starts[i // H_kv + 1], i % H_kv]
                                   for i in range(S)])
    if kind == "store":
        got["lens"] = None
    return got
