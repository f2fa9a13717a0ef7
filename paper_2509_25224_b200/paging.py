"""A paged cache's upkeep on the device: tokens into and out of a 4-bit cache, and copying, forking, freeing, reserving and
compacting pages of any cache.  Argument checks and marshalling only; the work is done by the library's kernels, on the current
stream, and nothing is read back to the host.

The books of a cache are int32 tensors: block_table [B, max_blocks], seqlens [B] and refs [num_blocks] (in how many table
entries a page is named; 0: free).  ``include/amla.h`` has the rules in full.

The checks are written out for speed: a step of a serving loop is a handful of these calls, of a few microseconds each on the GPU.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import AMLA_OK, AmlaError

FP4_PAGE_BYTES = binding._FP4_PAGE_SHAPE[0]

_torch = _int = None
_sizes: dict = {}                    # workspace bytes by (num_blocks, B)


def _ready():
    """The loaded library (and torch, for the checks)."""
    global _torch, _int
    if _int is None:
        import torch
        _torch, _int = torch, torch.int32
    return binding._lib if binding._lib is not None else binding.lib()


def _call(on, entry, args, what):
    """entry(*args, stream) on the current stream of device `on`.  (Where that is the current device, which is cheap to ask for once a tensor of
    it exists, without the wrappers that binding._on_device has; 0.5 us of a call that takes 7.)"""
    if on == _torch._C._cuda_getDevice():
        rc = entry(*args, _torch._C._cuda_getCurrentRawStream(on))
        if rc != AMLA_OK:
            raise AmlaError(rc, what)
    else:
        binding._on_device(_torch.device("cuda", on), entry, args, (), what)


def workspace_size(num_blocks: int, B: int) -> int:
    """Bytes that pages_fork, pages_reserve and pages_compact need for a cache of num_blocks pages and a table of B rows."""
    n = ctypes.c_size_t(0)
    rc = binding.lib().amla_pages_workspace_size(int(num_blocks), int(B), ctypes.byref(n))
    if rc != AMLA_OK:
        raise AmlaError(rc, "amla_pages_workspace_size")
    return int(n.value)


def _int32(t, on, name):
    if t.dtype is not _int or not t.is_contiguous() or t.get_device() != on:
        raise ValueError(name + " must be a contiguous int32 tensor on the device of the others")


def _books(block_table, seqlens, refs):
    """(device index, rows, entries a row, pages) of consistent books."""
    on = block_table.get_device()
    if on < 0:
        raise ValueError("paging works on CUDA tensors, not tensors on " + str(block_table.device))
    _int32(block_table, on, "block_table")
    _int32(seqlens, on, "seqlens")
    _int32(refs, on, "refs")
    if block_table.dim() != 2 or seqlens.dim() != 1 or refs.dim() != 1 or seqlens.numel() != block_table.shape[0]:
        raise ValueError("block_table is [B, max_blocks], seqlens [B], refs [num_blocks]")
    B, width = block_table.shape
    return on, B, width, refs.numel()


def _page_bytes(cache, on=None, num_blocks=None):
    """Bytes of a page of a cache of any element type whose first axis counts pages."""
    if cache.get_device() < 0 or not cache.is_contiguous() or cache.dim() < 2 or cache.numel() == 0:
        raise ValueError("the cache must be a contiguous CUDA tensor [num_blocks, ...]")
    blocks = cache.shape[0]
    if num_blocks is not None and (blocks != num_blocks or cache.get_device() != on):
        raise ValueError("refs must have one count for each page of the cache, on its device")
    return cache.numel() // blocks * cache.element_size()


def _scratch(workspace, num_blocks, B, on, like):
    """(tensor, bytes); the tensor is the caller's, or one that lives until the call is enqueued (the allocator keeps the stream's order)."""
    if workspace is None:
        key = (num_blocks, B)
        size = _sizes.get(key)
        if size is None:
            if len(_sizes) > 64:
                _sizes.clear()
            size = _sizes[key] = workspace_size(num_blocks, B)
        return like.new_empty((size + 3) // 4), size
    if workspace.get_device() != on or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the device of the others")
    return workspace, workspace.numel() * workspace.element_size()


def _answers(t, n, on, like, name):
    if t is None:
        return like.new_empty(n)
    _int32(t, on, name)
    if t.dim() != 1 or t.numel() != n:
        raise ValueError("%s must be [%d]" % (name, n))
    return t


def _tokens(rows, starts, cache, block_table, seqlens):
    """(device index, sequences, entries a row, pages, tokens, elements from one token to the next)"""
    on = cache.get_device()
    if on < 0:
        raise ValueError("paging works on CUDA tensors, not tensors on " + str(cache.device))
    shape = cache.shape
    if cache.dtype is not _torch.uint8 or len(shape) != 2 or shape[1] != FP4_PAGE_BYTES or not cache.is_contiguous():
        raise ValueError("the cache must be contiguous uint8 [num_blocks, %d]" % FP4_PAGE_BYTES)
    _int32(starts, on, "starts")
    _int32(block_table, on, "block_table")
    _int32(seqlens, on, "seqlens")
    if block_table.dim() != 2 or starts.dim() != 1 or seqlens.dim() != 1:
        raise ValueError("block_table is [B, max_blocks], seqlens [B], starts [B + 1]")
    B, width = block_table.shape
    if starts.numel() != B + 1 or seqlens.numel() != B:
        raise ValueError("block_table is [B, max_blocks], seqlens [B], starts [B + 1]")
    if rows.dtype is not _torch.bfloat16 or rows.dim() != 2 or rows.get_device() != on:
        raise ValueError("tokens are bfloat16 [n, 576] on the device of the cache")
    n, d = rows.shape
    step, inner = rows.stride()
    if d != 576 or (n > 0 and inner != 1):
        raise ValueError("tokens are bfloat16 [n, 576] whose columns are contiguous")
    if n <= 1:
        step = 576
    elif step < 576:
        raise ValueError("rows of tokens must not overlap")
    return on, B, width, shape[0], n, step


def cache_store_fp4(kv, starts, kv_cache_fp4, kv_scale: float, block_table, seqlens) -> None:
    """Quantises tokens kv bf16 [n, 576] (rows may be a slice of wider ones) into the 4-bit cache: rows starts[b] .. starts[b+1] - 1
    are the last tokens of sequence b, whose length seqlens[b] already counts them."""
    L = _ready()
    on, B, width, blocks, n, step = _tokens(kv, starts, kv_cache_fp4, block_table, seqlens)
    _call(on, L.amla_cache_store_fp4,
          (kv.data_ptr(), step, n, starts.data_ptr(), kv_cache_fp4.data_ptr(), float(kv_scale), block_table.data_ptr(), seqlens.data_ptr(), B, blocks, width),
          "amla_cache_store_fp4")


def cache_load_fp4(kv_cache_fp4, kv_scale: float, block_table, seqlens, starts, out):
    """The inverse: out[starts[b] .. starts[b+1] - 1] (bf16 [n, 576]) = the last tokens of sequence b, as the decode call sees them."""
    L = _ready()
    on, B, width, blocks, n, step = _tokens(out, starts, kv_cache_fp4, block_table, seqlens)
    _call(on, L.amla_cache_load_fp4,
          (kv_cache_fp4.data_ptr(), float(kv_scale), block_table.data_ptr(), seqlens.data_ptr(), starts.data_ptr(), B, blocks, width, out.data_ptr(), step, n),
          "amla_cache_load_fp4")
    return out


def pages_copy(cache, src, dst) -> None:
    """cache[dst[i]] = cache[src[i]] for all i; a pair with an index outside the cache is skipped."""
    L = _ready()
    page_bytes = _page_bytes(cache)
    on = cache.get_device()
    _int32(src, on, "src")
    _int32(dst, on, "dst")
    if src.dim() != 1 or dst.dim() != 1 or src.numel() != dst.numel():
        raise ValueError("src and dst are lists of the same length")
    _call(on, L.amla_pages_copy, (cache.data_ptr(), page_bytes, cache.shape[0], src.data_ptr(), dst.data_ptr(), src.numel()), "amla_pages_copy")


def pages_free(block_table, seqlens, refs, rows) -> None:
    """The listed rows give up their pages and are left empty."""
    L = _ready()
    on, B, width, blocks = _books(block_table, seqlens, refs)
    _int32(rows, on, "rows")
    if rows.dim() != 1:
        raise ValueError("rows is a list")
    _call(on, L.amla_pages_free,
          (block_table.data_ptr(), seqlens.data_ptr(), refs.data_ptr(), rows.data_ptr(), rows.numel(), B, blocks, width), "amla_pages_free")


def pages_fork(cache, block_table, seqlens, refs, parents, children, served=None, workspace=None):
    """Row children[i] becomes a copy of row parents[i] that shares its full pages.  Returns served int32 [n]: 0 where no page was left."""
    L = _ready()
    on, B, width, blocks = _books(block_table, seqlens, refs)
    page_bytes = _page_bytes(cache, on, blocks)
    _int32(parents, on, "parents")
    _int32(children, on, "children")
    n = parents.numel()
    if parents.dim() != 1 or children.dim() != 1 or children.numel() != n:
        raise ValueError("parents and children are lists of the same length")
    served = _answers(served, n, on, refs, "served")
    workspace, size = _scratch(workspace, blocks, B, on, refs)
    _call(on, L.amla_pages_fork,
          (cache.data_ptr(), page_bytes, block_table.data_ptr(), seqlens.data_ptr(), refs.data_ptr(), parents.data_ptr(), children.data_ptr(), n, B, blocks, width,
           served.data_ptr(), workspace.data_ptr(), size), "amla_pages_fork")
    return served


def pages_reserve(block_table, seqlens, refs, new_lens, granted=None, workspace=None):
    """Rows grow to new_lens [B], with free pages where they need them.  Returns granted int32 [B]: 0 where the row stays as it was
    (which takes no page from the rows behind it)."""
    L = _ready()
    on, B, width, blocks = _books(block_table, seqlens, refs)
    _int32(new_lens, on, "new_lens")
    if new_lens.dim() != 1 or new_lens.numel() != B:
        raise ValueError("new_lens is [B]")
    granted = _answers(granted, B, on, refs, "granted")
    workspace, size = _scratch(workspace, blocks, B, on, refs)
    _call(on, L.amla_pages_reserve,
          (block_table.data_ptr(), seqlens.data_ptr(), refs.data_ptr(), new_lens.data_ptr(), B, blocks, width, granted.data_ptr(), workspace.data_ptr(), size),
          "amla_pages_reserve")
    return granted


def pages_compact(cache, block_table, seqlens, refs, live=None, workspace=None):
    """Moves the pages in use to the front of the cache.  Returns live int32 [1]: how many there are; the pages from there on are free."""
    L = _ready()
    on, B, width, blocks = _books(block_table, seqlens, refs)
    page_bytes = _page_bytes(cache, on, blocks)
    live = _answers(live, 1, on, refs, "live")
    workspace, size = _scratch(workspace, blocks, B, on, refs)
    _call(on, L.amla_pages_compact,
          (cache.data_ptr(), page_bytes, block_table.data_ptr(), seqlens.data_ptr(), refs.data_ptr(), B, blocks, width, live.data_ptr(), workspace.data_ptr(), size),
          "amla_pages_compact")
    return live
