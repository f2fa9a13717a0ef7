"""Beam search on a 4-bit cache, with everything that it asks of the cache done on the device:

    python -m paper_2509_25224_b200.beam_search [--groups 8] [--beams 8] [--heads 128] [--prompt 1000] [--steps 64]

A prompt is stored once and forked to the beams of its group.  A step then lets every row grow by a token (pages_reserve), stores it
(cache_store_fp4), attends (mla_decode_fp4), and replaces the group's worst beam by a second continuation of its best (pages_free,
pages_fork).  The step is recorded in a CUDA graph and replayed: lengths, tables and counts are read and written on the device alone.
At the end the cache is compacted.

Queries, tokens and scores are synthetic; what is checked is the cache: the attention before and after compaction is the same to the
bit, and every row reads back as the tokens of its own history, to the format's error.
"""
from __future__ import annotations

import argparse

PAGE = 64
GROUP_ERROR = 1 / 6 + 1 / 16         # half of E2M1's widest gap, and the rounding of its scale, of the largest magnitude of 16 columns


def search(groups: int = 8, beams: int = 8, heads: int = 128, prompt: int = 1000, steps: int = 64, kv_scale: float = 0.05, seed: int = 0, num_blocks: int | None = None):
    """Runs the search and returns what there is to check and to report, as a dict of tensors and numbers."""
    import torch

    from . import binding, paging

    if beams < 2 or groups < 1 or prompt < 1 or steps < 1:
        raise ValueError("a search needs a prompt, a step, a group and two beams")
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev).manual_seed(seed)
    rows, longest = groups * beams, prompt + steps
    width = -(-longest // PAGE)
    if num_blocks is None:
        num_blocks = rows * width
    int32 = dict(dtype=torch.int32, device=dev)
    cache = torch.empty((num_blocks, paging.FP4_PAGE_BYTES), dtype=torch.uint8, device=dev)
    table, lens, refs = torch.full((rows, width), -1, **int32), torch.zeros(rows, **int32), torch.zeros(num_blocks, **int32)
    first = torch.arange(0, rows, beams, **int32)                      # a group's first row
    scratch = torch.empty(paging.workspace_size(num_blocks, rows), dtype=torch.uint8, device=dev)
    work = torch.empty(binding.fp4_workspace_size(rows, 1, heads, width, dev.index), dtype=torch.uint8, device=dev)
    failed = torch.zeros(1, **int32)

    # prompts: into the first row of each group, and from there to the others
    tokens = torch.randn((groups, prompt, 576), generator=gen, device=dev).bfloat16()
    wanted = torch.zeros(rows, **int32)
    wanted[first.long()] = prompt
    failed += (paging.pages_reserve(table, lens, refs, wanted, workspace=scratch) == 0).sum()
    starts = torch.zeros(rows + 1, **int32)
    starts[1:] = (wanted > 0).int().cumsum(0) * prompt
    paging.cache_store_fp4(tokens.view(-1, 576), starts, cache, kv_scale, table, lens)
    others = torch.tensor([r for r in range(rows) if r % beams], **int32)
    failed += (paging.pages_fork(cache, table, lens, refs, (others // beams * beams).int(), others, workspace=scratch) == 0).sum()

    # a step, on tensors that stay where they are
    q, kv = torch.empty((rows, 1, heads, 576), dtype=torch.bfloat16, device=dev), torch.empty((rows, 576), dtype=torch.bfloat16, device=dev)
    out, lse = torch.empty((rows, 1, heads, 512), dtype=torch.bfloat16, device=dev), torch.empty((rows, 1, heads), dtype=torch.float32, device=dev)
    granted, served, each = torch.empty(rows, **int32), torch.empty(groups, **int32), torch.arange(rows + 1, **int32)
    worst, best = torch.empty(groups, **int32), torch.empty(groups, **int32)
    score = torch.zeros((groups, beams), device=dev)
    scale = 576 ** -0.5

    def attend():
        binding.mla_decode_fp4(q, cache, kv_scale, table, lens, scale, out, lse, work)

    def step():
        paging.pages_reserve(table, lens, refs, lens + 1, granted, scratch)
        # a row that was refused has not grown: its token would land on its last key, in a page that others may hold too
        paging.cache_store_fp4(kv, each, cache, kv_scale, table, lens * granted)
        attend()
        score.add_(lse.mean((1, 2)).view(groups, beams))
        order = score.argsort(1)
        worst.copy_(order[:, 0] + first)
        best.copy_(order[:, -1] + first)
        score.scatter_(1, order[:, :1], score.gather(1, order[:, -1:]))
        paging.pages_free(table, lens, refs, worst)
        paging.pages_fork(cache, table, lens, refs, best, worst, served, scratch)
        failed.add_((granted == 0).sum() + (served == 0).sum())

    # what every row should hold: its tokens from the left, zeros behind them (a row that found no page has fewer than the others)
    history, row, had = torch.zeros((rows, longest, 576), dtype=torch.bfloat16, device=dev), torch.arange(rows, device=dev), torch.empty_like(lens)
    history[:, :prompt] = tokens.repeat_interleave(beams, 0) * (lens == prompt)[:, None, None]

    def inputs():
        q.normal_(generator=gen)
        kv.normal_(generator=gen)
        had.copy_(lens)

    def remember():
        at = row, had.long()
        history[at] = torch.where(granted[:, None] > 0, kv, history[at])
        history[worst.long()] = history[best.long()] * (served > 0)[:, None, None]

    graph, times = None, []
    for i in range(steps):
        inputs()
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
        remember()

    # compaction changes where pages are, and nothing else
    q.normal_(generator=gen)
    attend()
    before = out.clone(), lse.clone()
    live = paging.pages_compact(cache, table, lens, refs, workspace=scratch)
    attend()
    read = torch.empty((rows * longest, 576), dtype=torch.bfloat16, device=dev)
    paging.cache_load_fp4(cache, kv_scale, table, lens, torch.arange(0, (rows + 1) * longest, longest, **int32), read)
    # (the last tokens of a row end at the right)
    at = torch.arange(longest, device=dev) + (longest - lens.long())[:, None]
    read = read.view(rows, longest, 576)[row[:, None], at.clamp(max=longest - 1)] * (at < longest)[..., None]
    binding.check_status(work)
    spent = sorted(a.elapsed_time(b) * 1e3 for a, b in times[2:])
    return dict(cache=cache, kv_scale=kv_scale, scale=scale, q=q, out=out, lse=lse, before=before, table=table, lens=lens, refs=refs, history=history,
                read=read, live=int(live), failed=int(failed), step_us=spent[len(spent) // 2] if spent else None, width=width)


def faults(r) -> list[str]:
    """What is wrong with a search's cache: nothing, it is to be hoped."""
    import torch

    wrong = []
    if r["failed"]:
        wrong.append("%d requests found no page" % r["failed"])
    if not (torch.equal(r["out"], r["before"][0]) and torch.equal(r["lse"], r["before"][1])):
        wrong.append("compaction changed the attention")
    if not bool((r["lens"] == r["history"].shape[1]).all()):
        wrong.append("a row has the wrong length")
    held, refs = r["table"][r["table"] >= 0].long(), r["refs"]
    if not (torch.equal(torch.bincount(held, minlength=refs.numel()).int(), refs) and bool((refs[: r["live"]] > 0).all()) and not bool((refs[r["live"]:] != 0).any())):
        wrong.append("the counts of references are wrong")
    # in chunks of tokens: the histories are long
    for i in range(0, r["history"].shape[1], 256):
        kept = r["history"][:, i:i + 256].float()
        top = kept.abs().unflatten(-1, (36, 16)).amax(-1).repeat_interleave(16, -1)
        # (and the rounding of what is read to bf16)
        if not bool(((r["read"][:, i:i + 256].float() - kept).abs() <= top * (GROUP_ERROR + 2 ** -8)).all()):
            wrong.append("tokens %d.. do not read back" % i)
            break
    return wrong


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("groups", 8), ("beams", 8), ("heads", 128), ("prompt", 1000), ("steps", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    r = search(a.groups, a.beams, a.heads, a.prompt, a.steps)
    rows, longest = r["history"].shape[:2]
    if r["step_us"] is not None:
        print("step of %d rows (reserve, store, attend, free, fork): %.1f us" % (rows, r["step_us"]))
    alone = rows * r["width"]
    print("pages: %d, of %d if no row shared any; %.1f MB in 4 bits, %.1f in bf16" % (r["live"], alone, r["live"] * r["cache"].shape[1] / 1e6, r["live"] * PAGE * 576 * 2 / 1e6))
    wrong = faults(r)
    print("; ".join(wrong) if wrong else "every row reads back, and attends after compaction as before")
    return 1 if wrong else 0


if __name__ == "__main__":
    raise SystemExit(main())
