"""A paged cache's upkeep on the device: tokens into and out of a 4-bit cache, and copying, forking, freeing, reserving and
compacting pages of any cache.  Argument checks and marshalling only; the work is done by the library's kernels, on the current
stream, and nothing is read back to the host.

The books of a cache are int32 tensors: block_table [B, max_blocks], seqlens [B] and refs [num_blocks] (in how many table
entries a page is named; 0: free).  ``include/amla.h`` has the rules in full.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import AMLA_OK, AmlaError

FP4_PAGE_BYTES = binding._FP4_PAGE_SHAPE[0]


def workspace_size(num_blocks: int, B: int) -> int:
    """Bytes that pages_fork, pages_reserve and pages_compact need for a cache of num_blocks pages and a table of B rows."""
    n = ctypes.c_size_t(0)
    rc = binding.lib().amla_pages_workspace_size(int(num_blocks), int(B), ctypes.byref(n))
    if rc != AMLA_OK:
        raise AmlaError(rc, "amla_pages_workspace_size")
    return int(n.value)


def _int32(dev, **tensors):
    import torch
    for name, t in tensors.items():
        if t.dtype is not torch.int32 or not t.is_contiguous() or t.device != dev:
            raise ValueError(name + " must be a contiguous int32 tensor on the device of the others")


def _books(block_table, seqlens, refs):
    dev = block_table.device
    if dev.type != "cuda":
        raise ValueError("paging works on CUDA tensors, not tensors on " + str(dev))
    _int32(dev, block_table=block_table, seqlens=seqlens, refs=refs)
    if block_table.dim() != 2 or seqlens.shape != (block_table.shape[0],) or refs.dim() != 1:
        raise ValueError("block_table is [B, max_blocks], seqlens [B], refs [num_blocks]")
    return dev


def _pages(cache, num_blocks=None):
    """(address, bytes of a page, pages) of a cache of any element type whose first axis counts pages."""
    if cache.device.type != "cuda" or not cache.is_contiguous() or cache.dim() < 2 or cache.shape[0] == 0:
        raise ValueError("the cache must be a contiguous CUDA tensor [num_blocks, ...]")
    if num_blocks is not None and cache.shape[0] != num_blocks:
        raise ValueError("refs must have one count for each page of the cache")
    return cache.data_ptr(), cache.numel() // cache.shape[0] * cache.element_size(), cache.shape[0]


def _workspace(workspace, num_blocks, B, dev):
    if workspace is None:
        import torch
        workspace = torch.empty(workspace_size(num_blocks, B), dtype=torch.uint8, device=dev)
    elif workspace.device != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the device of the others")
    return workspace


def _flags(t, n, dev, name):
    import torch
    if t is None:
        return torch.empty(n, dtype=torch.int32, device=dev)
    _int32(dev, **{name: t})
    if t.shape != (n,):
        raise ValueError("%s must be [%d]" % (name, n))
    return t


def _tokens(rows, starts, cache, block_table, seqlens):
    import torch
    dev = cache.device
    if dev.type != "cuda":
        raise ValueError("paging works on CUDA tensors, not tensors on " + str(dev))
    if cache.dtype is not torch.uint8 or cache.dim() != 2 or cache.shape[1] != FP4_PAGE_BYTES or not cache.is_contiguous():
        raise ValueError("the cache must be contiguous uint8 [num_blocks, %d]" % FP4_PAGE_BYTES)
    _int32(dev, starts=starts, block_table=block_table, seqlens=seqlens)
    B = block_table.shape[0]
    if block_table.dim() != 2 or starts.shape != (B + 1,) or seqlens.shape != (B,):
        raise ValueError("block_table is [B, max_blocks], seqlens [B], starts [B + 1]")
    if rows.dtype is not torch.bfloat16 or rows.dim() != 2 or rows.shape[1] != 576 or rows.device != dev or (rows.numel() and rows.stride(1) != 1):
        raise ValueError("tokens are bfloat16 [n, 576] whose columns are contiguous")
    if rows.shape[0] > 1 and rows.stride(0) < 576:
        raise ValueError("rows of tokens must not overlap")
    return dev, B


def _lib():
    return binding._lib if binding._lib is not None else binding.lib()


def cache_store_fp4(kv, starts, kv_cache_fp4, kv_scale: float, block_table, seqlens) -> None:
    """Quantises tokens kv bf16 [n, 576] (rows may be a slice of wider ones) into the 4-bit cache: rows starts[b] .. starts[b+1] - 1
    are the last tokens of sequence b, whose length seqlens[b] already counts them."""
    dev, B = _tokens(kv, starts, kv_cache_fp4, block_table, seqlens)
    binding._on_device(dev, _lib().amla_cache_store_fp4,
                       (kv.data_ptr(), kv.stride(0) if kv.shape[0] > 1 else 576, kv.shape[0], starts.data_ptr(), kv_cache_fp4.data_ptr(), float(kv_scale),
                        block_table.data_ptr(), seqlens.data_ptr(), B, kv_cache_fp4.shape[0], block_table.shape[1]), (), "amla_cache_store_fp4")


def cache_load_fp4(kv_cache_fp4, kv_scale: float, block_table, seqlens, starts, out):
    """The inverse: out[starts[b] .. starts[b+1] - 1] (bf16 [n, 576]) = the last tokens of sequence b, as the decode call sees them."""
    dev, B = _tokens(out, starts, kv_cache_fp4, block_table, seqlens)
    binding._on_device(dev, _lib().amla_cache_load_fp4,
                       (kv_cache_fp4.data_ptr(), float(kv_scale), block_table.data_ptr(), seqlens.data_ptr(), starts.data_ptr(), B, kv_cache_fp4.shape[0],
                        block_table.shape[1], out.data_ptr(), out.stride(0) if out.shape[0] > 1 else 576, out.shape[0]), (), "amla_cache_load_fp4")
    return out


def pages_copy(cache, src, dst) -> None:
    """cache[dst[i]] = cache[src[i]] for all i; a pair with an index outside the cache is skipped."""
    address, page_bytes, num_blocks = _pages(cache)
    _int32(cache.device, src=src, dst=dst)
    if src.dim() != 1 or src.shape != dst.shape:
        raise ValueError("src and dst are lists of the same length")
    binding._on_device(cache.device, _lib().amla_pages_copy, (address, page_bytes, num_blocks, src.data_ptr(), dst.data_ptr(), src.shape[0]), (), "amla_pages_copy")


def pages_free(block_table, seqlens, refs, rows) -> None:
    """The listed rows give up their pages and are left empty."""
    dev = _books(block_table, seqlens, refs)
    _int32(dev, rows=rows)
    if rows.dim() != 1:
        raise ValueError("rows is a list")
    binding._on_device(dev, _lib().amla_pages_free,
                       (block_table.data_ptr(), seqlens.data_ptr(), refs.data_ptr(), rows.data_ptr(), rows.shape[0], block_table.shape[0], refs.shape[0],
                        block_table.shape[1]), (), "amla_pages_free")


def pages_fork(cache, block_table, seqlens, refs, parents, children, served=None, workspace=None):
    """Row children[i] becomes a copy of row parents[i] that shares its full pages.  Returns served int32 [n]: 0 where no page was left."""
    dev = _books(block_table, seqlens, refs)
    address, page_bytes, num_blocks = _pages(cache, refs.shape[0])
    _int32(dev, parents=parents, children=children)
    if cache.device != dev or parents.dim() != 1 or parents.shape != children.shape:
        raise ValueError("parents and children are lists of the same length, the cache is on the device of the books")
    served = _flags(served, parents.shape[0], dev, "served")
    B = block_table.shape[0]
    workspace = _workspace(workspace, num_blocks, B, dev)
    binding._on_device(dev, _lib().amla_pages_fork,
                       (address, page_bytes, block_table.data_ptr(), seqlens.data_ptr(), refs.data_ptr(), parents.data_ptr(), children.data_ptr(), parents.shape[0], B,
                        num_blocks, block_table.shape[1], served.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size()), (), "amla_pages_fork")
    return served


def pages_reserve(block_table, seqlens, refs, new_lens, granted=None, workspace=None):
    """Rows grow to new_lens [B], with free pages where they need them.  Returns granted int32 [B]: 0 where the row stays as it was."""
    dev = _books(block_table, seqlens, refs)
    _int32(dev, new_lens=new_lens)
    B, num_blocks = block_table.shape[0], refs.shape[0]
    if new_lens.shape != (B,):
        raise ValueError("new_lens is [B]")
    granted = _flags(granted, B, dev, "granted")
    workspace = _workspace(workspace, num_blocks, B, dev)
    binding._on_device(dev, _lib().amla_pages_reserve,
                       (block_table.data_ptr(), seqlens.data_ptr(), refs.data_ptr(), new_lens.data_ptr(), B, num_blocks, block_table.shape[1], granted.data_ptr(),
                        workspace.data_ptr(), workspace.numel() * workspace.element_size()), (), "amla_pages_reserve")
    return granted


def pages_compact(cache, block_table, seqlens, refs, live=None, workspace=None):
    """Moves the pages in use to the front of the cache.  Returns live int32 [1]: how many there are; the pages from there on are free."""
    dev = _books(block_table, seqlens, refs)
    address, page_bytes, num_blocks = _pages(cache, refs.shape[0])
    if cache.device != dev:
        raise ValueError("the cache is on the device of the books")
    live = _flags(live, 1, dev, "live")
    B = block_table.shape[0]
    workspace = _workspace(workspace, num_blocks, B, dev)
    binding._on_device(dev, _lib().amla_pages_compact,
                       (address, page_bytes, block_table.data_ptr(), seqlens.data_ptr(), refs.data_ptr(), B, num_blocks, block_table.shape[1], live.data_ptr(),
                        workspace.data_ptr(), workspace.numel() * workspace.element_size()), (), "amla_pages_compact")
    return live
