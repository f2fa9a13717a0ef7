"""Attention to the pages of a long context that matter: scores from the pages' means (paging.page_means), the choice, and decode on what is chosen.
Argument checks and marshalling only; the work is done by the library's kernels, on the current stream, and nothing is read back to the host.

``include/amla.h`` has the rules in full.  pages_select leaves a block table and lengths that any decode call takes, on B * Sq sequences of
one query token; mla_decode_sparse does all of it in one call.
"""
from __future__ import annotations

import ctypes

from . import binding, paging
from .binding import AMLA_OK, AmlaError

_sizes: dict = {}                    # workspace bytes by shape


def _size(entry: str, *shape) -> int:
    size = _sizes.get((entry, shape))
    if size is None:
        n = ctypes.c_size_t(0)
        rc = getattr(binding.lib(), entry)(*shape, ctypes.byref(n))
        if rc != AMLA_OK:
            raise AmlaError(rc, entry)
        if len(_sizes) > 256:
            _sizes.clear()
        size = _sizes[entry, shape] = int(n.value)
    return size


def scores_workspace_size(B: int, Sq: int, H: int, max_blocks: int, device: int = 0) -> int:
    """Bytes that page_scores needs."""
    return _size("amla_page_scores_workspace_size", int(B), int(Sq), int(H), int(max_blocks), int(device or 0))


def sparse_workspace_size(B: int, Sq: int, H: int, max_blocks: int, keep: int, device: int = 0) -> int:
    """Bytes that mla_decode_sparse needs, for a cache of any format."""
    return _size("amla_mla_decode_sparse_workspace_size", int(B), int(Sq), int(H), int(max_blocks), int(keep), int(device or 0))


def _queries(q, block_table, seqlens):
    """(device index, B, Sq, H, entries a row)"""
    torch = paging._torch
    on = q.get_device()
    if on < 0:
        raise ValueError("the decode entries take CUDA tensors, not tensors on " + str(q.device))
    if q.dtype is not torch.bfloat16 or q.dim() != 4 or q.shape[3] != 576 or not q.is_contiguous():
        raise ValueError("q must be a contiguous bfloat16 [B, Sq, H, 576]")
    paging._int32(block_table, on, "block_table")
    paging._int32(seqlens, on, "seqlens")
    B, Sq, H, _ = q.shape
    shape = block_table.shape
    if len(shape) != 2 or shape[0] != B or seqlens.dim() != 1 or seqlens.numel() != B:
        raise ValueError("block_table is [B, max_blocks], seqlens [B]")
    return on, B, Sq, H, shape[1]


def _given(t, shape, dtype, on, like, name):
    """`t`, or a new tensor where it is None."""
    if t is None:
        return like.new_empty(shape, dtype=dtype)
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != on:
        raise ValueError("%s must be a contiguous %s %s on the device of the others" % (name, str(dtype).replace("torch.", ""), list(shape)))
    return t


def _means(means, on):
    if means.dtype is not paging._torch.bfloat16 or means.dim() != 2 or means.shape[1] != 576 or not means.is_contiguous() or means.get_device() != on:
        raise ValueError("means must be a contiguous bfloat16 [num_blocks, 576] on the device of q")
    return means.shape[0]


def _scratch(workspace, size, on, like):
    if workspace is None:
        return like.new_empty(size(), dtype=paging._torch.uint8)
    if workspace.get_device() != on or not workspace.is_contiguous():
        raise ValueError(binding._WORKSPACE)
    return workspace


def page_scores(q, means, block_table, seqlens, softmax_scale: float, scores=None, workspace=None):
    """fp32 [B, Sq, max_blocks]: the share of attention of every page in front of a query token's own, were its keys their mean, summed over the heads; 0 for the other pages."""
    L = paging._ready()
    on, B, Sq, H, width = _queries(q, block_table, seqlens)
    blocks = _means(means, on)
    torch = paging._torch
    scores = _given(scores, (B, Sq, width), torch.float32, on, q, "scores")
    workspace = _scratch(workspace, lambda: scores_workspace_size(B, Sq, H, width, on), on, q)
    paging._call(on, L.amla_page_scores,
                 (q.data_ptr(), means.data_ptr(), block_table.data_ptr(), seqlens.data_ptr(), float(softmax_scale), B, Sq, H, blocks, width, scores.data_ptr(), workspace.data_ptr(),
                  workspace.numel() * workspace.element_size()), "amla_page_scores")
    return scores


def pages_select(scores, block_table, seqlens, keep: int, sink: int = 1, recent: int = 1, table=None, lens=None, chosen=None):
    """(table int32 [B * Sq, keep], lens int32 [B * Sq], chosen int32 [B * Sq, keep]): for every query token the first `sink` pages, the last `recent` and
    those of the largest scores (fp32 [B, Sq, max_blocks]), `keep` in all, as a block table and lengths, and where they are in the sequence; -1 beyond."""
    L = paging._ready()
    torch = paging._torch
    on = scores.get_device()
    if on < 0:
        raise ValueError("paging works on CUDA tensors, not tensors on " + str(scores.device))
    if scores.dtype is not torch.float32 or scores.dim() != 3 or not scores.is_contiguous():
        raise ValueError("scores must be a contiguous float32 [B, Sq, max_blocks]")
    paging._int32(block_table, on, "block_table")
    paging._int32(seqlens, on, "seqlens")
    B, Sq, width = scores.shape
    if block_table.shape != (B, width) or seqlens.dim() != 1 or seqlens.numel() != B:
        raise ValueError("block_table is [B, max_blocks], seqlens [B]")
    keep = int(keep)
    if keep < 1:
        raise ValueError("keep is at least 1")
    n, int32 = B * Sq, torch.int32
    table = block_table.new_empty(n, keep) if table is None else _given(table, (n, keep), int32, on, scores, "table")
    lens = block_table.new_empty(n) if lens is None else _given(lens, (n,), int32, on, scores, "lens")
    chosen = block_table.new_empty(n, keep) if chosen is None else _given(chosen, (n, keep), int32, on, scores, "chosen")
    paging._call(on, L.amla_pages_select,
                 (scores.data_ptr(), block_table.data_ptr(), seqlens.data_ptr(), B, Sq, width, keep, int(sink), int(recent), table.data_ptr(), lens.data_ptr(), chosen.data_ptr()),
                 "amla_pages_select")
    return table, lens, chosen


def mla_decode_sparse(q, kv_cache, kv_scale: float, means, block_table, seqlens, softmax_scale: float, keep: int, sink: int = 1, recent: int = 1, out=None, lse=None, workspace=None):
    """Decode that attends to `keep` pages of every sequence: page_scores, pages_select and the decode call for the cache's format (paging.cache_format; kv_scale is
    not used by bf16) in one.  Returns (out bf16 [B, Sq, H, 512], lse fp32 [B, Sq, H])."""
    L = paging._ready()
    on, B, Sq, H, width = _queries(q, block_table, seqlens)
    torch = paging._torch
    fmt = paging.cache_format(kv_cache)
    if not kv_cache.is_contiguous() or kv_cache.get_device() != on:
        raise ValueError("the cache must be contiguous, on the device of q")
    blocks = kv_cache.shape[0]
    if means is not None and _means(means, on) != blocks:
        raise ValueError("means must have a row for each page of the cache")
    out = _given(out, (B, Sq, H, 512), torch.bfloat16, on, q, "out")
    lse = _given(lse, (B, Sq, H), torch.float32, on, q, "lse")
    workspace = _scratch(workspace, lambda: sparse_workspace_size(B, Sq, H, width, keep, on), on, q)
    paging._call(on, L.amla_mla_decode_sparse,
                 (fmt, q.data_ptr(), kv_cache.data_ptr(), float(kv_scale), 0 if means is None else means.data_ptr(), block_table.data_ptr(), seqlens.data_ptr(), float(softmax_scale), B, Sq, H,
                  blocks, width, int(keep), int(sink), int(recent), out.data_ptr(), lse.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size()),
                 "amla_mla_decode_sparse")
    return out, lse


def check_status(workspace, stream: int = 0) -> None:
    """Raises AmlaError(-5) if a bounded wait expired during the last mla_decode_sparse call on this workspace.  (For page_scores: binding.check_status.)"""
    rc = binding.lib().amla_sparse_check_status(workspace.data_ptr(), stream)
    if rc != AMLA_OK:
        raise AmlaError(rc, "amla_sparse_check_status")
