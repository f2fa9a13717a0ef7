"""What a serving program does with long contexts in a paged latent cache, as measurable cases: new tokens go into the cache (normed and
rotated on the way), the pages that they fill get a summary, and attention goes to the pages whose summaries say that they matter.

A cache is pages of 64 keys of 576 columns (512 latent, 64 of position): bf16, E4M3 bytes with one factor, or E2M1 numbers with an E4M3
scale for each 16 columns.  Sequence b has seqlens[b] keys in the pages of row b of a block table.

A case's "op" names the operator:

  append   cache_append: the latent part of new tokens is normed, the position part rotated, both are stored; the position part of their
           queries is rotated into place
  means    page_means: every page that new tokens fill gets the mean of its keys
  scores   page_scores: for every query token and page in front of its own, the share of the heads' attention that the page's mean
           draws among the pages' means, summed over the heads
  select   pages_select: the first pages, the last pages and those of the largest scores, as a block table and lengths
  sparse   mla_decode_sparse: scores, selection and attention to what is selected, in one call

"fmt" is what the pages hold: "bf16", "e4m3" or "fp4".  Pages lie in random order, as after some time of serving.
"""
import math
import random

import torch

own = False

PAGE, D_QK, D_V, ROPE, GROUP = 64, 576, 512, 64, 16
CODE_BYTES, SCALE_BYTES = PAGE * D_QK // 2, PAGE * D_QK // GROUP
TOKEN_BYTES = {"bf16": 2 * D_QK, "e4m3": D_QK, "fp4": D_QK // 2 + D_QK // GROUP}
SCALE = 1.0 / math.sqrt(192.0)
KV_SCALE = {"bf16": 1.0, "e4m3": 1.0 / 64, "fp4": 0.25}
EPS = 1e-6
MAX_PAGES = 48 * 1024                # most pages of a drawn cache (3.6 GB of bf16)


def append_case(name, fmt, B, n_new, H, n_lo, n_hi, n_seed, interleaved):
    return named(name, {"op": "append", "fmt": fmt, "B": B, "n_new": n_new, "H": H, "n_lo": n_lo, "n_hi": n_hi, "n_seed": n_seed, "interleaved": interleaved})


def means_case(name, fmt, B, n_new, n_lo, n_hi, n_seed):
    return named(name, {"op": "means", "fmt": fmt, "B": B, "n_new": n_new, "n_lo": n_lo, "n_hi": n_hi, "n_seed": n_seed})


def scores_case(name, B, Sq, H, n_lo, n_hi, n_seed):
    return named(name, {"op": "scores", "B": B, "Sq": Sq, "H": H, "n_lo": n_lo, "n_hi": n_hi, "n_seed": n_seed})


def select_case(name, B, Sq, n_lo, n_hi, n_seed, keep, sink, recent):
    return named(name, {"op": "select", "B": B, "Sq": Sq, "n_lo": n_lo, "n_hi": n_hi, "n_seed": n_seed, "keep": keep, "sink": sink, "recent": recent})


def sparse_case(name, fmt, B, Sq, H, n_lo, n_hi, n_seed, keep, sink, recent):
    return named(name, {"op": "sparse", "fmt": fmt, "B": B, "Sq": Sq, "H": H, "n_lo": n_lo, "n_hi": n_hi, "n_seed": n_seed, "keep": keep, "sink": sink, "recent": recent})


def named(name, c):
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # the smallest call: one token of one sequence of a model sharded by heads; launch and host work are all there is
        append_case("append-one", "e4m3", 1, 1, 16, 199, 199, 1, False),
        # the cache's part of a decode step of a medium batch
        append_case("append-step", "bf16", 96, 1, 128, 0, 1000, 41, False),
        # the next chunk of four prompts, sixteen heads left of a model sharded over eight GPUs
        append_case("append-chunk", "fp4", 4, 2048, 16, 0, 2000, 42, True),
        # a decode step: one sequence in 64 has filled a page
        means_case("means-step", "bf16", 96, 1, 1, 2047, 43),
        # a chunk of a few prompts: nearly every page of it is full
        means_case("means-chunk", "e4m3", 5, 1900, 0, 3000, 44),
        # contexts of ordinary length, few heads
        scores_case("scores-short", 8, 1, 16, 1500, 4000, 45),
        # a medium batch of long contexts
        scores_case("scores-long", 32, 1, 128, 65536, 65536, 46),
        # speculative decoding with two query tokens over very long, ragged contexts
        scores_case("scores-spec2-ragged", 12, 2, 128, 9000, 262144, 47),
        # a step of a medium batch
        select_case("select-step", 64, 1, 10000, 32768, 48, 32, 1, 2),
        # contexts of a million tokens, two query tokens
        select_case("select-million", 4, 2, 800000, 1048576, 49, 256, 1, 4),
        # the attention of a decode step over long contexts
        sparse_case("sparse-step", "bf16", 32, 1, 128, 8192, 65536, 50, 32, 1, 2),
        # speculative decoding, more pages kept
        sparse_case("sparse-spec2", "e4m3", 16, 2, 128, 65536, 65536, 51, 64, 1, 2),
    ]


def log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choices(["append", "means", "scores", "select", "sparse"], [3, 2, 3, 2, 3])[0]
    fmt = rng.choice(["bf16", "e4m3", "fp4"])
    seed = rng.randrange(1 << 20)
    H = rng.choices([128, 64, 32, 16, rng.randint(1, 128)], [4, 2, 1, 2, 2])[0]
    if op in ("append", "means"):
        n_new = log_uniform(rng, 1, 8) if rng.random() < 0.5 else log_uniform(rng, 8, 2048)
        n_hi = log_uniform(rng, 1, 8192)
        B = log_uniform(rng, 1, max(1, min(256, 8192 // n_new, 65536 // (n_hi + n_new))))
        n_lo = rng.randint(0, n_hi)
        if op == "means":
            return means_case(None, fmt, B, n_new, n_lo, n_hi, seed)
        H = H if B * n_new * H <= 160000 else min(H, 16)
        return append_case(None, fmt, B, n_new, H, n_lo, n_hi, seed, rng.random() < 0.5)
    Sq = rng.choices([1, 2, rng.randint(3, 8)], [6, 3, 1])[0]
    if op == "select":
        n_hi = log_uniform(rng, 64, 1048576)
        B = log_uniform(rng, 1, max(1, min(256, 400000 // (pages_of(n_hi) * Sq))))
    else:
        n_hi = log_uniform(rng, 300, 262144)
        most = (32768 if op == "scores" else MAX_PAGES) * 128 / max(128, Sq * H)
        B = log_uniform(rng, 1, max(1, min(128, int(most) // (pages_of(n_hi) + 1))))
    n_lo = n_hi if rng.random() < 0.3 else rng.randint(0, n_hi)
    if op == "scores":
        return scores_case(None, B, Sq, H, n_lo, n_hi, seed)
    sink, recent = rng.randint(0, 2), rng.randint(1, 4)
    if op == "select":
        return select_case(None, B, Sq, n_lo, n_hi, seed, sink + recent + log_uniform(rng, 1, 512), sink, recent)
    keep = sink + recent + log_uniform(rng, 1, max(1, min(128, 2048 // (B * Sq))))
    return sparse_case(None, fmt, B, Sq, H, n_lo, n_hi, seed, keep, sink, recent)


def lengths(case):
    """Per sequence: what is in the cache before the new tokens (append, means), else the lengths."""
    r = random.Random(case["n_seed"])
    return [r.randint(case["n_lo"], case["n_hi"]) for _ in range(case["B"])]


def pages_of(n):
    return (n + PAGE - 1) // PAGE


# ---------------------------------------------------------------------------------------------- inputs

def scattered(lens, blocks, gen, dev):
    """A block table [B, pages of the longest] whose sequences' pages are entries of a permutation of the cache's pages; -1 elsewhere."""
    count = [pages_of(n) for n in lens]
    place = torch.randperm(blocks, generator=gen, device=dev).to(torch.int32)
    count_d = torch.tensor(count, device=dev)
    owner = torch.repeat_interleave(torch.arange(len(lens), device=dev), count_d, output_size=sum(count))
    index = torch.arange(sum(count), device=dev) - (count_d.cumsum(0) - count_d)[owner]
    table = torch.full((len(lens), max(max(count), 1)), -1, dtype=torch.int32, device=dev)
    table[owner, index] = place[: sum(count)]
    return table


def held(x, fmt):
    """FP32 keys [pages, 64, 576] -> pages of the format."""
    if fmt == "bf16":
        return x.to(torch.bfloat16)
    if fmt == "e4m3":
        return (x / KV_SCALE[fmt]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    codes, scales = quantise(x)
    return torch.cat([codes.view(x.shape[0], -1), scales.view(x.shape[0], -1)], 1)


def empty_cache(blocks, fmt, dev):
    if fmt == "fp4":
        return torch.empty((blocks, CODE_BYTES + SCALE_BYTES), dtype=torch.uint8, device=dev)
    return torch.empty((blocks, PAGE, D_QK), dtype=torch.bfloat16 if fmt == "bf16" else torch.uint8, device=dev)


def random_pages(fmt, count, gen, dev):
    out = empty_cache(count, fmt, dev)
    for i in range(0, count, 2048):
        part = out[i:i + 2048]
        part.copy_(held(torch.randn((part.shape[0], PAGE, D_QK), generator=gen, device=dev), fmt))
    return out


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev).manual_seed(seed)
    op, B, before = case["op"], case["B"], lengths(case)
    normal = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    if op in ("append", "means"):
        fmt, n_new = case["fmt"], case["n_new"]
        lens = [n + n_new for n in before]
        blocks, n = sum(map(pages_of, lens)), B * n_new
        state = {"op": op, "fmt": fmt, "cache": random_pages(fmt, blocks, gen, dev), "table": scattered(lens, blocks, gen, dev),
                 "seqlens": torch.tensor(lens, dtype=torch.int32, device=dev), "starts": torch.arange(0, n + 1, n_new, dtype=torch.int32, device=dev), "n": n}
        if op == "means":
            return {**state, "means": normal(blocks, D_QK).to(torch.bfloat16)}
        H = case["H"]
        angle = torch.arange(max(lens), device=dev, dtype=torch.float64)[:, None] * (10000.0 ** (-torch.arange(ROPE // 2, device=dev, dtype=torch.float64) / (ROPE // 2)))
        q_full = normal(n, H, 128 + ROPE).to(torch.bfloat16)           # what the projection leaves: 128 columns to be absorbed, 64 of position
        return {**state, "interleaved": case["interleaved"], "kv": (normal(n, D_QK) * 3.0).to(torch.bfloat16),
                "weight": (1.0 + 0.2 * normal(D_V)).to(torch.bfloat16), "cos_sin": torch.cat([angle.cos(), angle.sin()], 1).float(),
                "q_pe": q_full[..., 128:], "q": normal(n, H, D_QK).to(torch.bfloat16), "out": torch.empty((n, D_QK), dtype=torch.bfloat16, device=dev)}
    width = max(1, max(map(pages_of, before)))
    seqlens = torch.tensor(before, dtype=torch.int32, device=dev)
    if op == "select":
        # shares of attention: few pages have much, most have little; some are equal
        scores = (3.0 * normal(B, case["Sq"], width)).exp()
        scores = torch.where(scores < 0.01, torch.zeros_like(scores), scores)
        blocks = sum(map(pages_of, before))
        return {"op": op, "scores": scores, "table": scattered(before, max(blocks, 1), gen, dev), "seqlens": seqlens,
                "keep": case["keep"], "sink": case["sink"], "recent": case["recent"]}
    Sq, H = case["Sq"], case["H"]
    blocks = max(1, sum(map(pages_of, before)))
    table = scattered(before, blocks, gen, dev)
    state = {"op": op, "table": table, "seqlens": seqlens, "shape": (B, Sq, H, width)}
    if op == "scores":
        # means of neighbouring keys are smaller than the keys and differ from page to page; some pages suit some heads
        means = (0.5 * normal(blocks, D_QK)).to(torch.bfloat16)
        return {**state, "means": means, "q": normal(B, Sq, H, D_QK).to(torch.bfloat16), "out": torch.empty((B, Sq, width), device=dev)}
    # as many pages of every sequence as are kept beside the first and last ones hold what the queries look for
    fmt, keep, sink, recent = case["fmt"], case["keep"], case["sink"], case["recent"]
    look = normal(D_QK)
    look = look / look.norm()
    wanted = torch.zeros(blocks, dtype=torch.bool, device=dev)
    count = (seqlens.long() + PAGE - 1) // PAGE
    slot = torch.arange(table.shape[1], device=dev)[None, :]
    # (in front of all of the query tokens' last pages)
    free = (slot >= sink) & (slot < ((seqlens.long() - Sq).clamp(min=0) // PAGE + 1 - recent)[:, None])
    order = torch.where(free, torch.rand(free.shape, generator=gen, device=dev), torch.full(free.shape, 2.0, device=dev)).argsort(1)[:, : keep - sink - recent]
    wanted[table.gather(1, order)[free.gather(1, order)].long()] = True
    cache, means = empty_cache(blocks, fmt, dev), torch.empty((blocks, D_QK), dtype=torch.bfloat16, device=dev)
    for i in range(0, blocks, 2048):
        x = normal(min(2048, blocks - i), PAGE, D_QK) + (8.0 * wanted[i:i + 2048])[:, None, None] * look
        cache[i:i + 2048] = held(x, fmt)
        means[i:i + 2048] = values(cache[i:i + 2048], fmt).mean(1).to(torch.bfloat16)
    return {**state, "fmt": fmt, "cache": cache, "means": means, "q": (normal(B, Sq, H, D_QK) + 6.0 * look).to(torch.bfloat16), "keep": keep, "sink": sink, "recent": recent,
            "out": torch.empty((B, Sq, H, D_V), dtype=torch.bfloat16, device=dev), "lse": torch.empty((B, Sq, H), device=dev)}


# ---------------------------------------------------------------------------------------------- the framework's operators

_workspaces = {}


def workspace(s, size):
    """The calls' scratch, kept by a program from call to call."""
    key = (s["op"], s.get("fmt"), s["shape"], s.get("keep"))
    if key not in _workspaces:
        _workspaces[key] = torch.empty(size(), dtype=torch.uint8, device=s["q"].device)
    return _workspaces[key]


def run(state):
    s = state
    if not own:
        return {"append": plain_append, "means": plain_means, "scores": plain_scores, "select": plain_select, "sparse": plain_sparse}[s["op"]](s)
    from paper_2509_25224_b200 import paging, sparse
    if s["op"] == "append":
        paging.cache_append(s["kv"], s["starts"], s["cache"], KV_SCALE[s["fmt"]], s["table"], s["seqlens"], s["cos_sin"], norm_weight=s["weight"], eps=EPS,
                            interleaved=s["interleaved"], q_pe=s["q_pe"], q=s["q"])
        if s["fmt"] == "fp4":
            return s["q"], paging.cache_load_fp4(s["cache"], KV_SCALE["fp4"], s["table"], s["seqlens"], s["starts"], s["out"])
        return s["q"], s["cache"] if s["fmt"] == "bf16" else s["cache"].view(torch.float8_e4m3fn)
    if s["op"] == "means":
        return paging.page_means(s["cache"], KV_SCALE[s["fmt"]], s["table"], s["seqlens"], s["starts"], s["n"], s["means"])
    if s["op"] == "scores":
        return sparse.page_scores(s["q"], s["means"], s["table"], s["seqlens"], SCALE, s["out"],
                                  workspace(s, lambda: sparse.scores_workspace_size(*s["shape"], s["q"].device.index)))
    if s["op"] == "select":
        return sparse.pages_select(s["scores"], s["table"], s["seqlens"], s["keep"], s["sink"], s["recent"])
    return sparse.mla_decode_sparse(s["q"], s["cache"], KV_SCALE[s["fmt"]], s["means"], s["table"], s["seqlens"], SCALE, s["keep"], s["sink"], s["recent"], s["out"], s["lse"],
                                    workspace(s, lambda: sparse.sparse_workspace_size(*s["shape"], s["keep"], s["q"].device.index)))


# ---------------------------------------------------------------------------------------------- plain forms

def quantise(x):
    """FP32 [..., 576] -> (E2M1 pairs uint8 [..., 288], E4M3 bytes uint8 [..., 36])."""
    g = x.unflatten(-1, (D_QK // GROUP, GROUP))
    scale = (g.abs().amax(-1) / torch.tensor(6.0 * KV_SCALE["fp4"], device=x.device)).clamp(max=448.0).to(torch.float8_e4m3fn)
    step = scale.float().unsqueeze(-1) * KV_SCALE["fp4"]
    y = torch.where(step > 0, g.abs() / torch.where(step > 0, step, torch.ones_like(step)), torch.zeros_like(g))
    # how many of E2M1's midpoints a magnitude is beyond (a tie goes to the even code)
    code = (y > 0.25).byte() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)
    code = (code + 8 * (g < 0)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale.view(torch.uint8)


def widen(codes, scales):
    """E2M1 pairs [..., 288] and E4M3 bytes [..., 36] -> FP32 [..., 576]."""
    e2m1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    x = e2m1[torch.stack([codes & 15, codes >> 4], -1).int()].flatten(-2).unflatten(-1, (D_QK // GROUP, GROUP))
    return (x * (scales.contiguous().view(torch.float8_e4m3fn).float() * KV_SCALE["fp4"]).unsqueeze(-1)).flatten(-2)


def values(pages, fmt):
    """Pages of a cache [..., ] -> FP32 [..., 64, 576]."""
    if fmt == "bf16":
        return pages.float()
    if fmt == "e4m3":
        return pages.view(torch.float8_e4m3fn).float() * KV_SCALE[fmt]
    return widen(pages[..., :CODE_BYTES].unflatten(-1, (PAGE, D_QK // 2)), pages[..., CODE_BYTES:].unflatten(-1, (PAGE, D_QK // GROUP)))


def places(s):
    """(position, page, row) of the call's tokens: the last of every sequence, in order."""
    token = torch.arange(s["n"], device=s["starts"].device)
    b = torch.searchsorted(s["starts"][1:].contiguous(), token.int(), right=True)
    at = s["seqlens"].long()[b] - s["starts"].long()[b + 1] + token
    return at, s["table"][b, at // PAGE].long(), at % PAGE


def rotated(x, cos, sin, interleaved):
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., : ROPE // 2], x[..., ROPE // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)


def plain_append(s):
    at, page, row = places(s)
    angles = s["cos_sin"][at]
    cos, sin = angles[:, : ROPE // 2], angles[:, ROPE // 2:]
    x = s["kv"].float()
    c = x[:, :D_V]
    r = torch.rsqrt((c.double().square().sum(-1, keepdim=True) / D_V + EPS).float())
    x = torch.cat([c * r * s["weight"].float(), rotated(x[:, D_V:], cos, sin, s["interleaved"])], 1)
    s["q"][..., D_V:] = rotated(s["q_pe"].float(), cos[:, None], sin[:, None], s["interleaved"]).to(torch.bfloat16)
    if s["fmt"] == "fp4":
        codes, scales = quantise(x)
        s["cache"][:, :CODE_BYTES].unflatten(1, (PAGE, D_QK // 2))[page, row] = codes
        s["cache"][:, CODE_BYTES:].unflatten(1, (PAGE, D_QK // GROUP))[page, row] = scales
        return s["q"], widen(codes, scales).to(torch.bfloat16)
    s["cache"][page, row] = held(x, s["fmt"])
    return s["q"], s["cache"] if s["fmt"] == "bf16" else s["cache"].view(torch.float8_e4m3fn)


def plain_means(s):
    at, page, row = places(s)
    full = page[row == PAGE - 1]
    s["means"][full] = values(s["cache"][full], s["fmt"]).mean(1).to(torch.bfloat16)
    return s["means"]


def sees(seqlens, Sq, width):
    """Keys that query token t sees: [B, Sq]."""
    n = seqlens.long().clamp(max=width * PAGE)[:, None] - Sq + 1 + torch.arange(Sq, device=seqlens.device)
    return n.clamp(min=0)


def plain_scores(s):
    q, table = s["q"], s["table"]
    B, Sq, H, _ = q.shape
    width = table.shape[1]
    means = s["means"][table.clamp(min=0).long()].float()
    logits = torch.bmm(q.float().flatten(1, 2), means.transpose(1, 2)).view(B, Sq, H, width) * SCALE
    candidate = torch.arange(width, device=q.device) < ((sees(s["seqlens"], Sq, width) + PAGE - 1) // PAGE - 1)[..., None]
    logits = logits.masked_fill_(~candidate[:, :, None], -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = (logits - torch.where(top == -math.inf, torch.zeros_like(top), top)).exp()
    total = p.sum(-1, keepdim=True)
    return (p / torch.where(total > 0, total, torch.ones_like(total))).sum(2)


def plain_select(s, scores=None):
    """(block table, lengths, positions of the pages) of what every query token attends to."""
    scores = s["scores"] if scores is None else scores
    table, keep = s["table"], s["keep"]
    B, Sq, width = scores.shape
    n = sees(s["seqlens"], Sq, width)
    page, count = torch.arange(width, device=scores.device), ((n + PAGE - 1) // PAGE)[..., None]
    forced = ((page < s["sink"]) | (page >= count - s["recent"])) & (page < count)
    others = (page < count) & ~forced
    order = torch.sort(torch.where(others, scores, torch.full_like(scores, -math.inf)), dim=-1, descending=True, stable=True).indices
    of_others = others.gather(-1, order)
    best = of_others & (of_others.cumsum(-1) <= keep - forced.sum(-1, keepdim=True))
    chosen = forced | torch.zeros_like(forced).scatter(-1, order, best)
    to = torch.where(chosen, chosen.cumsum(-1) - 1, torch.full_like(order, keep))          # (column `keep` is thrown away)
    empty = torch.full((B, Sq, keep + 1), -1, dtype=torch.int32, device=scores.device)
    pages = empty.scatter(-1, to, table[:, None].expand(B, Sq, width))[..., :keep]
    where = empty.scatter(-1, to, page.int().expand(B, Sq, width))[..., :keep]
    held_back = (count[..., 0] - chosen.sum(-1)) * PAGE
    return pages.reshape(-1, keep), (n - held_back).int().view(-1), where.reshape(-1, keep)


def plain_sparse(s):
    q = s["q"]
    B, Sq, H, _ = q.shape
    pages, lens, _ = plain_select(s, plain_scores(s))
    keys = values(s["cache"][pages.clamp(min=0).long()], s["fmt"]).flatten(1, 2)
    seen = torch.arange(keys.shape[1], device=q.device) < lens[:, None]
    logits = torch.bmm(q.float().view(B * Sq, H, D_QK), keys.transpose(1, 2)) * SCALE
    logits = logits.masked_fill_(~seen[:, None], -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.bmm(p, keys[..., :D_V]) / torch.where(total > 0, total, torch.ones_like(total))
    return out.to(torch.bfloat16).view(B, Sq, H, D_V), (total.log() + top).view(B, Sq, H)


# ---------------------------------------------------------------------------------------------- 64 bits

def grid_e4m3(byte):
    """E4M3 bytes -> FP64, from their fields."""
    b = byte.long()
    e, m = (b // 8) % 16, b % 8
    return torch.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * torch.exp2((e - 7).double())) * (1.0 - 2.0 * (b // 128))


def exact_values(pages, fmt):
    """Pages -> FP64 keys [keys, 576]."""
    if fmt == "bf16":
        return pages.double().reshape(-1, D_QK)
    if fmt == "e4m3":
        return grid_e4m3(pages).reshape(-1, D_QK) * KV_SCALE[fmt]
    codes, scales = pages[:, :CODE_BYTES].reshape(-1, D_QK // 2), pages[:, CODE_BYTES:].reshape(-1, D_QK // GROUP)
    nibble = torch.stack([codes % 16, codes // 16], -1).flatten(-2).long()
    e, m = (nibble // 2) % 4, nibble % 2
    x = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.exp2((e - 1).double())) * (1.0 - 2.0 * (nibble // 8))
    return x * grid_e4m3(scales).repeat_interleave(GROUP, -1) * KV_SCALE[fmt]


def nearest(v, grid):
    """The grid's numbers nearest to v >= 0, ties to the even index."""
    hi = torch.bucketize(v, grid).clamp(1, grid.shape[0] - 1)
    lo = hi - 1
    down = (v - grid[lo] < grid[hi] - v) | ((v - grid[lo] == grid[hi] - v) & (lo % 2 == 0))
    return grid[torch.where(down, lo, hi)]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "append":
        q, cache = s["q"].double(), None if s["fmt"] == "fp4" else s["cache"].view(torch.float8_e4m3fn).double() if s["fmt"] == "e4m3" else s["cache"].double()
        rows, n_new, half = [], case["n_new"], ROPE // 2
        even = torch.arange(half, device=q.device) * (2 if s["interleaved"] else 1)
        odd = even + (1 if s["interleaved"] else half)
        for b, before in enumerate(lengths(case)):
            i, at = slice(b * n_new, (b + 1) * n_new), torch.arange(before, before + n_new, device=q.device)
            turn = torch.complex(s["cos_sin"][at, :half].double(), s["cos_sin"][at, half:].double())
            x = s["kv"][i].double()
            x[:, :D_V] *= (x[:, :D_V].square().mean(1, keepdim=True) + EPS) ** -0.5 * s["weight"].double()
            z = torch.complex(x[:, D_V + even], x[:, D_V + odd]) * turn
            x[:, D_V + even], x[:, D_V + odd] = z.real, z.imag
            y = s["q_pe"][i].double()
            z = torch.complex(y[..., even], y[..., odd]) * turn[:, None]
            part = q[i]
            part[..., D_V + even], part[..., D_V + odd] = z.real, z.imag
            if cache is not None:
                cache[s["table"][b, at // PAGE].long(), at % PAGE] = (x / KV_SCALE["e4m3"]).clamp(-448.0, 448.0) if s["fmt"] == "e4m3" else x
            rows.append(x)
        if cache is not None:
            return q, cache
        x = torch.cat(rows).view(-1, D_QK // GROUP, GROUP) / KV_SCALE["fp4"]
        step = nearest((x.abs().amax(-1) / 6.0).clamp(max=448.0), grid_e4m3(torch.arange(127, device=x.device)))[..., None]
        grid4 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
        x = torch.where(step > 0, nearest((x.abs() / torch.where(step > 0, step, 1.0)).clamp(max=6.0), grid4) * step, 0.0) * x.sign() * KV_SCALE["fp4"]
        return q, x.flatten(1)
    if op == "means":
        means = s["means"].double()
        for b, before in enumerate(lengths(case)):
            pages = s["table"][b, before // PAGE: (before + case["n_new"]) // PAGE].long()
            means[pages] = exact_values(s["cache"][pages], s["fmt"]).view(-1, PAGE, D_QK).mean(1)
        return means
    if op == "select":
        return None
    B, Sq, H = case["B"], case["Sq"], case["H"]
    width = s["table"].shape[1]
    scores = torch.zeros((B, Sq, width), dtype=torch.float64, device=s["q"].device)
    for b, n in enumerate(lengths(case)):
        for t in range(Sq):
            own_page = (n - Sq + t) // PAGE
            if own_page > 0:
                logits = s["q"][b, t].double() @ s["means"][s["table"][b, :own_page].long()].double().T * SCALE
                scores[b, t, :own_page] = torch.softmax(logits, -1).sum(0)
    if op == "scores":
        return scores
    out = torch.zeros((B, Sq, H, D_V), dtype=torch.float64, device=s["q"].device)
    lse = torch.full((B, Sq, H), -math.inf, dtype=torch.float64, device=s["q"].device)
    for b, n in enumerate(lengths(case)):
        for t in range(Sq):
            seen = n - Sq + t + 1
            if seen <= 0:
                continue
            count = pages_of(seen)
            pages = list(range(count))
            if count > s["keep"]:
                ends = set(range(s["sink"])) | set(range(count - s["recent"], count))
                ranked = sorted((p for p in pages if p not in ends), key=lambda p, v=scores[b, t].tolist(): (-v[p], p))
                pages = sorted(ends | set(ranked[: s["keep"] - len(ends)]))
            keys = exact_values(s["cache"][s["table"][b, pages].long()], s["fmt"])[: seen - (count - len(pages)) * PAGE]
            logits = s["q"][b, t].double() @ keys.T * SCALE
            lse[b, t] = torch.logsumexp(logits, -1)
            out[b, t] = torch.softmax(logits, -1) @ keys[:, :D_V]
    return out, lse


def work(case):
    """Inputs once, outputs once; the means of a sequence's candidates and what its query tokens select (the same pages, where they agree) once."""
    op, before = case["op"], lengths(case)
    if op in ("append", "means"):
        n, n_new, token = case["B"] * case["n_new"], case["n_new"], TOKEN_BYTES[case["fmt"]]
        if op == "append":
            return {"bytes": n * (2 * D_QK + 4 * ROPE + token + 4 * ROPE * case["H"]) + 8 * case["B"], "flops": 0.0}
        full = sum((m + n_new) // PAGE - m // PAGE for m in before)
        return {"bytes": full * (PAGE * token + 2 * D_QK) + 12 * case["B"], "flops": 0.0}
    Sq = case["Sq"]
    width = max(1, max(map(pages_of, before)))
    if op == "select":
        return {"bytes": sum(Sq * 4 * pages_of(n) + Sq * min(case["keep"], pages_of(n)) * 4 for n in before) + case["B"] * Sq * (8 * case["keep"] + 4), "flops": 0.0}
    rows, front = Sq * case["H"], [max(0, pages_of(n) - 1) for n in before]
    score = {"bytes": sum(front) * (2 * D_QK + 4) + case["B"] * (rows * 2 * D_QK + Sq * width * 4), "flops": 2.0 * rows * sum(front) * D_QK}
    if op == "scores":
        return score
    keys = sum(min(n, case["keep"] * PAGE) for n in before)
    return {"bytes": score["bytes"] - case["B"] * Sq * width * 4 + keys * TOKEN_BYTES[case["fmt"]] + case["B"] * rows * (2 * D_V + 4),
            "flops": score["flops"] + 2.0 * rows * keys * (D_QK + D_V)}
