"""A follow-up question over a compacted, quantised, paged cache.

    python examples/follow_up.py [--config llava15] [--ratio 0.2] [--format int8]

The request of a workload (synthetic inputs) is evicted after its prefill; the
retained rows go into pages taken for them on the GPU, one sequence per layer, quantised
on the way.  Then a question arrives: its tokens take the pages they lack, its queries and
keys are turned by their positions, which go on from the whole prompt's (a retained row
keeps the position it had), its keys and values are stored, and it attends over the cache,
all layers in one call of each.  An answer follows, one token at a time.  At the end the
cache is read back as bf16 rows, and the decode step over those rows must agree with the
last token's attention over the pages.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

PAGE = 64


def follow_up(wl, ratio, fmt="int8", question=48, answer=8, seed=0):
    """Returns (bytes of the cache, bytes of its rows in bf16, largest difference
    between the two attentions of the last token relative to the largest output)."""
    import torch

    from paper_2606_03075_gb300 import api, synth

    inp = synth.generate(wl, seed=seed)

    def dev(a):
        return torch.from_numpy(a).cuda()

    def status(ws):
        bits = api.tgvkv_status(ws)
        if bits:
            raise RuntimeError(f"device status bits {bits:#x}")

    # ---- the eviction at the end of the prefill
    desc = api.desc_for_workload(wl)
    ws = api.new_workspace(desc)
    out = api.alloc_outputs(desc, ratio)
    api.tgvkv_evict(desc, dev(inp["q"]).view(torch.bfloat16), dev(inp["k"]).view(torch.bfloat16),
                    dev(inp["v"]).view(torch.bfloat16), dev(inp["modality"]), dev(inp["text_pos"]),
                    dev(inp["w"]), ratio, out, ws)
    status(ws)

    # ---- pages for the retained rows: a set is a (layer, KV head), each of its own length
    L, S = wl.L, wl.L * wl.H_kv
    kept = out.offsets.diff().to(torch.int32)
    most = int(kept.max()) + question + answer
    n_pages = int(((kept + question + answer + PAGE - 1) // PAGE).sum())
    cdesc = api.make_cache_desc(L, wl.H_q, wl.H_kv, wl.d, PAGE, n_pages, -(-most // PAGE), fmt)
    cache, pages, cws = api.alloc_cache(cdesc), api.alloc_pages(cdesc), api.new_cache_workspace(cdesc)
    lens = torch.zeros(S, dtype=torch.int32, device="cuda")
    grown = torch.empty_like(lens)
    api.tgvkv_pages_grow(cdesc, pages, lens, kept, cws)
    api.tgvkv_cache_write_rows(cdesc, cache, pages.page_table, lens, out.k_out, out.v_out, out.offsets,
                               grown, cws)
    lens, grown = grown, lens

    # ---- the question, then the answer's tokens: pages, turned keys into them, attention
    # (layer l's are rows tok_offsets[l] .. tok_offsets[l + 1] of q, k and v)
    gen = torch.Generator("cuda").manual_seed(seed)
    rope = api.make_rope(wl.d, base=1e6)
    position = wl.N

    def attend(n):
        nonlocal lens, grown, position
        qkv = torch.randn((L * n, wl.H_q + 2 * wl.H_kv, wl.d), generator=gen, device="cuda").bfloat16()
        q, k, v = qkv.split([wl.H_q, wl.H_kv, wl.H_kv], dim=1)       # strided views: no copies
        tok_offsets = torch.arange(0, L * n + 1, n, dtype=torch.int32, device="cuda")
        positions = torch.arange(position, position + n, dtype=torch.int32, device="cuda").repeat(L)
        slots = torch.empty((L * n, wl.H_kv), dtype=torch.int32, device="cuda")
        turned, o = (torch.empty((L * n, wl.H_q, wl.d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        api.tgvkv_pages_append(cdesc, pages, lens, tok_offsets, slots, grown, cws)
        lens, grown = grown, lens
        api.tgvkv_rope_write(cdesc, cache, rope, positions, slots, q, k, v, turned, cws)
        api.tgvkv_chunk_attention(cdesc, cache, pages.page_table, lens, turned, tok_offsets, n, o, cws)
        position += n
        return turned, o

    attend(question)
    for _ in range(answer):
        q, o = attend(1)

    # ---- the rows as the pages hold them, and the decode step over those
    offsets = torch.zeros(S + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.cumsum(lens, 0)
    k_rows, v_rows = (torch.empty((int(offsets[-1]), wl.d), dtype=torch.bfloat16, device="cuda")
                      for _ in range(2))
    api.tgvkv_cache_read(cdesc, cache, pages.page_table, None, offsets, k_rows, v_rows, cws)
    status(cws)
    want = torch.empty((L, wl.H_q, wl.d), dtype=torch.float32, device="cuda")
    api.tgvkv_decode(desc, q.contiguous(), k_rows, v_rows, offsets, want, ws)
    status(ws)
    err = float((o.float() - want).abs().max() / want.abs().max())
    held = sum(t.numel() * t.element_size() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)
               if t is not None)
    return held, 2 * k_rows.numel() * 2, err


def main():
    from paper_2606_03075_gb300 import synth

    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--config", default="llava15", choices=sorted(synth.WORKLOADS))
    ap.add_argument("--ratio", type=float, default=None, help="retained share (default: the workload's first)")
    ap.add_argument("--format", default="int8", choices=("bf16", "int8", "int4", "fp4"))
    args = ap.parse_args()
    wl = synth.WORKLOADS[args.config]
    held, rows, err = follow_up(wl, args.ratio or wl.ratios[0], args.format)
    print(f"{args.config}, {args.format}: cache of {held / 1e6:.2f} MB for {rows / 1e6:.2f} MB of bf16 rows; "
          f"last token against the decode over the rows read back: {err:.1e}")


if __name__ == "__main__":
    main()
