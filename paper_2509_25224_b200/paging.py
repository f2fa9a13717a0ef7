"""A paged cache's upkeep on the device: tokens into a cache of any format (normed and rotated on the way, or as they are) and out of a 4-bit one, the
means of full pages, and copying, forking, freeing, reserving and compacting pages of any cache.  Argument checks and marshalling only; the work is done by the library's kernels, on the current
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
CACHE_BF16, CACHE_E4M3, CACHE_FP4 = 0, 1, 2

_torch = _int = None
_sizes: dict = {}                    # workspace bytes by (num_blocks, B)


def _types():
    """torch, for the checks."""
    global _torch, _int
    if _int is None:
        import torch
        _torch, _int = torch, torch.int32


def _ready():
    """The loaded library (and torch)."""
    if _int is None:
        _types()
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


def cache_format(cache) -> int:
    """What a cache's pages hold (AMLA_CACHE_*), told from its shape and type: bf16 [num_blocks, 64, 576], uint8 of that shape (E4M3), uint8 [num_blocks, 20736] (4 bits)."""
    if _torch is None:
        _types()
    shape = cache.shape
    if len(shape) == 3 and shape[1] == 64 and shape[2] == 576:
        if cache.dtype is _torch.bfloat16:
            return CACHE_BF16
        if cache.dtype is _torch.uint8:
            return CACHE_E4M3
    elif len(shape) == 2 and shape[1] == FP4_PAGE_BYTES and cache.dtype is _torch.uint8:
        return CACHE_FP4
    raise ValueError("the cache must be bfloat16 or uint8 [num_blocks, 64, 576], or uint8 [num_blocks, %d]" % FP4_PAGE_BYTES)


def _batch(cache, starts, block_table, seqlens):
    """(device index, format, sequences, entries a row, pages)"""
    on = cache.get_device()
    if on < 0:
        raise ValueError("paging works on CUDA tensors, not tensors on " + str(cache.device))
    fmt = cache_format(cache)
    if not (cache.is_contiguous() and starts.dtype is _int and starts.is_contiguous() and starts.get_device() == on and block_table.dtype is _int and block_table.is_contiguous()
            and block_table.get_device() == on and seqlens.dtype is _int and seqlens.is_contiguous() and seqlens.get_device() == on):
        raise ValueError("the cache must be contiguous, and starts, block_table and seqlens contiguous int32 tensors on its device")
    shape = block_table.shape
    if len(shape) != 2 or starts.dim() != 1 or seqlens.dim() != 1 or starts.numel() != shape[0] + 1 or seqlens.numel() != shape[0]:
        raise ValueError("block_table is [B, max_blocks], seqlens [B], starts [B + 1]")
    return on, fmt, shape[0], shape[1], cache.shape[0]


def cache_append(kv, starts, cache, kv_scale: float, block_table, seqlens, cos_sin, positions=None, norm_weight=None, eps: float = 1e-6, interleaved: bool = False, q_pe=None, q=None) -> None:
    """New tokens into a cache of any format (cache_format), and their queries' position columns into place.

    Rows starts[b] .. starts[b+1] - 1 of kv (bf16 [n, 576], perhaps a slice of wider rows) are the last tokens of sequence b, whose length seqlens[b] already
    counts them.  Columns 0 .. 511 are normed where norm_weight (bf16 or fp32 [512]) is given, c * rsqrt(mean(c^2) + eps) * norm_weight; columns
    512 .. 575 are rotated by the angles of the token's position (positions int32 [n]; None: its place in the sequence), whose cosines and sines
    are a row of cos_sin (fp32 [n_positions, 64]).  interleaved: columns 2i, 2i+1 are a pair, else i, i+32.  q_pe (bf16 [n, H, 64], any strides)
    is rotated into columns 512 .. 575 of q (bf16 [n, H, 576]).  ``include/amla.h`` says what happens to tokens without a place or a position."""
    L = _ready()
    on, fmt, B, width, blocks = _batch(cache, starts, block_table, seqlens)
    bf16 = _torch.bfloat16
    shape = kv.shape
    if kv.dtype is not bf16 or kv.get_device() != on or len(shape) != 2 or shape[1] != 576:
        raise ValueError("tokens are bfloat16 [n, 576] on the device of the cache")
    n = shape[0]
    step, inner = kv.stride()
    # (an axis of at most one entry has no stride that matters)
    if n > 0 and (inner != 1 or (n > 1 and step < 576)):
        raise ValueError("rows of tokens must have contiguous columns and not overlap")
    if cos_sin.dtype is not _torch.float32 or cos_sin.dim() != 2 or cos_sin.shape[1] != 64 or not cos_sin.is_contiguous() or cos_sin.get_device() != on:
        raise ValueError("cos_sin must be a contiguous float32 [n_positions, 64] on the device of the cache")
    at = weight = wide = H = from_q = from_token = from_head = to_q = to_token = to_head = 0
    if positions is not None:
        _int32(positions, on, "positions")
        if positions.dim() != 1 or positions.numel() != n:
            raise ValueError("positions is [n]")
        at = positions.data_ptr()
    if norm_weight is not None:
        wide = 1 if norm_weight.dtype is _torch.float32 else 0
        if not (wide or norm_weight.dtype is bf16) or norm_weight.dim() != 1 or norm_weight.numel() != 512 or not norm_weight.is_contiguous() or norm_weight.get_device() != on:
            raise ValueError("norm_weight must be a contiguous bfloat16 or float32 [512] on the device of the cache")
        weight = norm_weight.data_ptr()
    if q is not None and q_pe is not None:
        if q.dtype is not bf16 or q_pe.dtype is not bf16 or q.get_device() != on or q_pe.get_device() != on:
            raise ValueError("q_pe and q must be bfloat16, on the device of the cache")
        shape, source = q.shape, q_pe.shape
        if len(shape) != 3 or len(source) != 3 or shape[0] != n or source[0] != n or source[1] != shape[1] or shape[2] != 576 or source[2] != 64:
            raise ValueError("q_pe is [n, H, 64] and q [n, H, 576]")
        H = shape[1]
        to_token, to_head, inner = q.stride()
        from_token, from_head, columns = q_pe.stride()
        if n > 0 and H > 0 and (inner != 1 or columns != 1 or (n > 1 and to_token < 576) or (H > 1 and to_head < 576)):
            raise ValueError("rows of q and q_pe must have contiguous columns, and those of q must not overlap")
        from_q, to_q = q_pe.data_ptr(), q.data_ptr()
    elif q is not None or q_pe is not None:
        raise ValueError("q_pe and q are given together, or neither")
    _call(on, L.amla_cache_append,
          (fmt, kv.data_ptr(), step, n, starts.data_ptr(), cache.data_ptr(), float(kv_scale), block_table.data_ptr(), seqlens.data_ptr(), B, blocks, width, cos_sin.data_ptr(),
           cos_sin.shape[0], at, weight, wide, float(eps), 1 if interleaved else 0, from_q, from_token, from_head, to_q, to_token, to_head, H), "amla_cache_append")


def page_means(cache, kv_scale: float, block_table, seqlens, starts, n_tokens: int, means):
    """means[page] (bf16 [num_blocks, 576]) = the mean key of every page that is filled by one of the tokens starts[b] .. starts[b+1] - 1, the last ones of
    sequence b; n_tokens bounds starts[B].  The other pages' are left as they were.  Pages that were moved since (pages_compact, pages_copy): call it with all tokens."""
    L = _ready()
    on, fmt, B, width, blocks = _batch(cache, starts, block_table, seqlens)
    if means.dtype is not _torch.bfloat16 or means.shape != (blocks, 576) or not means.is_contiguous() or means.get_device() != on:
        raise ValueError("means must be a contiguous bfloat16 [num_blocks, 576] on the device of the cache")
    _call(on, L.amla_page_means,
          (fmt, cache.data_ptr(), float(kv_scale), block_table.data_ptr(), seqlens.data_ptr(), starts.data_ptr(), int(n_tokens), B, blocks, width, means.data_ptr()), "amla_page_means")
    return means


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
