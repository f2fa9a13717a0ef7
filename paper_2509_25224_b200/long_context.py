"""Decoding over long contexts of which little matters, with everything that it asks of the cache done on the device:

    python -m paper_2509_25224_b200.long_context [--sequences 16] [--heads 128] [--prompt 32000] [--steps 32] [--keep 32] [--cache bf16|e4m3|fp4]

Prompts go into a paged cache in chunks: their latents are normed, their position columns rotated, the pages that they fill get their means
(cache_append, page_means).  A step then lets every sequence grow by a token (pages_reserve), stores it and rotates its queries (cache_append), brings the
means up to date (page_means) and attends to `keep` pages of each (mla_decode_sparse).  The step is recorded in a CUDA graph and replayed:
lengths, tables and counts are read and written on the device alone.

Tokens and queries are synthetic: a few pages of every prompt hold what the queries look for.  What is checked: those pages are chosen; the attention is that of
the plain decode call up to the share that went to pages which were left out; the means are those of what the pages hold.
"""
from __future__ import annotations

import argparse

PAGE, D_V, D_QK, ROPE = 64, 512, 576, 64
FORMATS = ("bf16", "e4m3", "fp4")
CHUNK = 2048


def serve(sequences: int = 16, heads: int = 128, prompt: int = 32000, steps: int = 32, keep: int = 32, cache: str = "bf16", sink: int = 1, recent: int = 2, needles: int = 3, seed: int = 0):
    """Runs the steps and returns what there is to check and to report, as a dict of tensors and numbers."""
    import torch

    from . import binding, paging, sparse

    if sequences < 1 or heads < 1 or prompt < 1 or steps < 1 or cache not in FORMATS:
        raise ValueError("a run needs a sequence, a head, a prompt, a step and one of the formats " + ", ".join(FORMATS))
    if needles < 0 or sink < 0 or recent < 1 or sink + recent + needles > keep:
        raise ValueError("keep has to have room for the first, the last and the planted pages")
    if needles and prompt // PAGE < sink + recent + needles:
        raise ValueError("the prompt has no room for the planted pages")
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev).manual_seed(seed)
    int32 = dict(dtype=torch.int32, device=dev)
    normal = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    longest = prompt + steps
    width = -(-longest // PAGE)
    num_blocks = sequences * width + 3
    kv_scale = {"bf16": 1.0, "e4m3": 1.0 / 32, "fp4": 0.25}[cache]
    shape = (num_blocks, paging.FP4_PAGE_BYTES) if cache == "fp4" else (num_blocks, PAGE, D_QK)
    pages = torch.zeros(shape, dtype=torch.bfloat16 if cache == "bf16" else torch.uint8, device=dev)
    means = torch.zeros((num_blocks, D_QK), dtype=torch.bfloat16, device=dev)
    table, lens, refs = torch.full((sequences, width), -1, **int32), torch.zeros(sequences, **int32), torch.zeros(num_blocks, **int32)
    scratch = torch.empty(paging.workspace_size(num_blocks, sequences), dtype=torch.uint8, device=dev)
    failed = torch.zeros(1, **int32)

    angle = torch.arange(longest, device=dev, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(ROPE // 2, device=dev, dtype=torch.float64) / (ROPE // 2))
    cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float()
    weight = (1.0 + 0.1 * normal(D_V)).bfloat16()
    look = normal(D_V)
    look = look / look.norm()

    # where in the prompts the queries' direction is to be found: whole pages behind the first and in front of the last ones
    free = prompt // PAGE - sink - recent
    planted = sink + torch.rand((sequences, max(free, 0)), generator=gen, device=dev).argsort(1)[:, :needles].sort(1).values
    holds = torch.zeros((sequences, width), dtype=torch.bool, device=dev)
    holds.scatter_(1, planted, True)

    def tokens(first, count):
        """What a model would hand over for positions first .. first + count - 1 of all sequences: [sequences * count, 576]."""
        x = normal(sequences, count, D_QK)
        x[..., :D_V] += 32.0 * holds[:, torch.arange(first, first + count, device=dev) // PAGE, None] * look
        return x.bfloat16().view(-1, D_QK)

    # prompts, a chunk at a time
    for first in range(0, prompt, CHUNK):
        count = min(CHUNK, prompt - first)
        failed += (paging.pages_reserve(table, lens, refs, torch.full_like(lens, first + count), workspace=scratch) == 0).sum()
        starts = torch.arange(0, sequences * count + 1, count, **int32)
        paging.cache_append(tokens(first, count), starts, pages, kv_scale, table, lens, cos_sin, norm_weight=weight)
        paging.page_means(pages, kv_scale, table, lens, starts, sequences * count, means)

    # a step, on tensors that stay where they are
    kv, q_pe = torch.empty((sequences, D_QK), dtype=torch.bfloat16, device=dev), torch.empty((sequences, heads, ROPE), dtype=torch.bfloat16, device=dev)
    q = torch.empty((sequences, 1, heads, D_QK), dtype=torch.bfloat16, device=dev)
    out, lse = torch.empty((sequences, 1, heads, D_V), dtype=torch.bfloat16, device=dev), torch.empty((sequences, 1, heads), device=dev)
    each, granted = torch.arange(sequences + 1, **int32), torch.empty(sequences, **int32)
    work = torch.empty(sparse.sparse_workspace_size(sequences, 1, heads, width, keep, dev.index), dtype=torch.uint8, device=dev)
    scale = 192 ** -0.5

    def step():
        paging.pages_reserve(table, lens, refs, lens + 1, granted, scratch)
        failed.add_((granted == 0).sum())
        # (a row that was refused has not grown: its token would land on its last key)
        paging.cache_append(kv, each, pages, kv_scale, table, lens * granted, cos_sin, norm_weight=weight, q_pe=q_pe, q=q.view(sequences, heads, D_QK))
        paging.page_means(pages, kv_scale, table, lens * granted, each, sequences, means)
        sparse.mla_decode_sparse(q, pages, kv_scale, means, table, lens, scale, keep, sink, recent, out, lse, work)

    graph, times = None, []
    for i in range(steps):
        q.copy_(normal(sequences, 1, heads, D_QK))
        q[..., :D_V] += 12.0 * look
        q_pe.copy_(normal(sequences, heads, ROPE))
        kv.copy_(tokens(prompt + i, 1))
        if i == 1:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        began, ended = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        began.record()
        if graph is None:
            step()
        else:
            graph.replay()
        ended.record()
        times.append((began, ended))
    sparse.check_status(work)

    # the same attention by the plain call, and which pages the last step attended to
    plain = {"bf16": lambda *a: binding.mla_decode(q, pages, *a), "e4m3": lambda *a: binding.mla_decode_fp8(q, pages, kv_scale, *a), "fp4": lambda *a: binding.mla_decode_fp4(q, pages, kv_scale, *a)}[cache]
    began, ended = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    whole = plain(table, lens, scale)
    began.record()
    whole = plain(table, lens, scale, *whole)
    ended.record()
    scores = sparse.page_scores(q, means, table, lens, scale)
    chosen = sparse.pages_select(scores, table, lens, keep, sink, recent)[2]
    torch.cuda.synchronize(dev)
    spent = sorted(a.elapsed_time(b) * 1e3 for a, b in times[2:])
    return dict(cache=pages, kv_scale=kv_scale, format=cache, means=means, table=table, lens=lens, out=out, lse=lse, whole=whole, chosen=chosen, planted=planted, failed=int(failed),
                step_us=spent[len(spent) // 2] if spent else None, plain_us=began.elapsed_time(ended) * 1e3, prompt=prompt, steps=steps)


def keys_of(r, page_numbers):
    """FP32 [..., 64, 576]: what pages of a run's cache hold."""
    import torch

    from . import paging

    pages = r["cache"][page_numbers.long()]
    if r["format"] == "bf16":
        return pages.float()
    if r["format"] == "e4m3":
        return pages.view(torch.float8_e4m3fn).float() * r["kv_scale"]
    n = page_numbers.numel()
    table, lens = page_numbers.view(n, 1).int().contiguous(), torch.full((n,), PAGE, dtype=torch.int32, device=pages.device)
    out = torch.empty((n * PAGE, D_QK), dtype=torch.bfloat16, device=pages.device)
    paging.cache_load_fp4(r["cache"], r["kv_scale"], table, lens, torch.arange(0, n * PAGE + 1, PAGE, dtype=torch.int32, device=pages.device), out)
    return out.float().view(*page_numbers.shape, PAGE, D_QK)


def faults(r) -> list[str]:
    """What is wrong with a run: nothing, it is to be hoped."""
    import torch

    wrong = []
    if r["failed"]:
        wrong.append("%d requests found no page" % r["failed"])
    if not bool((r["lens"] == r["prompt"] + r["steps"]).all()):
        wrong.append("a sequence has the wrong length")
    if not bool((r["planted"][:, :, None] == r["chosen"][:, None, :]).any(-1).all()):
        wrong.append("a page that the queries look for was left out")
    # the share of attention that went to the pages left out bounds how far the two are apart: twice the largest value, and the roundings of both results to bf16
    left = 1.0 - (r["lse"] - r["whole"][1]).exp()
    if not bool((left >= -1e-3).all()) or not bool((left <= 0.2).all()):
        wrong.append("the pages that were left out have a share of attention of %.3g .. %.3g" % (float(left.min()), float(left.max())))
    top = r["whole"][0].float().abs().amax()
    largest = max(float(keys_of(r, r["table"][b, : int(r["lens"][b]) // PAGE])[..., :D_V].abs().amax()) for b in range(r["table"].shape[0]))
    apart = (r["out"].float() - r["whole"][0].float()).abs().amax(-1)
    if not bool((apart <= 2.0 * left.clamp(min=0.0) * largest + 2.0 ** -6 * top).all()):
        wrong.append("the attention is further from the plain one than what was left out explains")
    for b in range(r["table"].shape[0]):
        full = r["table"][b, : int(r["lens"][b]) // PAGE]
        if full.numel():
            keys = keys_of(r, full)
            # (what a 4-bit cache reads back as is rounded to bf16; the mean itself is too)
            if not bool(((r["means"][full.long()].float() - keys.mean(1)).abs() <= 2.0 ** -7 * keys.abs().mean(1) + 1e-6).all()):
                wrong.append("the means of sequence %d are not those of its pages" % b)
    return wrong


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("sequences", 16), ("heads", 128), ("prompt", 32000), ("steps", 32), ("keep", 32)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--cache", choices=FORMATS, default="bf16")
    a = ap.parse_args()
    r = serve(a.sequences, a.heads, a.prompt, a.steps, a.keep, a.cache)
    if r["step_us"] is not None:
        print("step of %d sequences (reserve, append, means, attend to %d pages of %d): %.1f us; the plain decode call alone: %.1f us" % (
            a.sequences, a.keep, r["table"].shape[1], r["step_us"], r["plain_us"]))
    left = 1.0 - (r["lse"] - r["whole"][1]).exp()
    print("attention that the pages left out would have had: %.2g on average, %.2g at most" % (float(left.mean()), float(left.max())))
    wrong = faults(r)
    print("; ".join(wrong) if wrong else "the planted pages are found, and the attention is the plain one's but for that")
    return 1 if wrong else 0


if __name__ == "__main__":
    raise SystemExit(main())
