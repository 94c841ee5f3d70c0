"""Pages of a cache under a beam search.

A pool's pages are counted in ``refs`` [pages] int32: how many page table
entries hold each, 0 for a free page.  ``kv_fork`` makes the page tables of the
hypotheses that a step has chosen from their parents', frees what no one holds
any more and gives out fresh pages; ``kv_copy`` copies what two hypotheses
would otherwise write into, in each layer's cache; ``kv_compact`` moves the
used pages of a pool together.  All enqueue their HIP kernels on the current
stream (or ``stream``) and return; the C ABI is ``include/ngpu_lm.h``.
"""

from __future__ import annotations

import ctypes

from . import _check, _torch_mod, load_library
from .serving import _cache, _Cache, _cache8, _Cache8, _device_of, _native, _need, _on, _table, _untracked, _whole

MAX_FORK = 4096                  # NGPU_LM_MAX_FORK
MAX_PAGES = 1 << 28              # NGPU_LM_MAX_PAGES

_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class _Fork(ctypes.Structure):
    _fields_ = [("G", _i64), ("W", _i64), ("K", _i64), ("pages", _vp), ("width", _i64), ("pages_stride", _i64),
                ("lengths", _vp), ("parents", _vp), ("tokens", _vp), ("T", _i64), ("page_size", _i32),
                ("num_pages", _i64), ("refs", _vp), ("out_pages", _vp), ("out_lengths", _vp), ("copies", _vp)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        p = ctypes.POINTER
        lib.ngpu_lm_kv_fork_workspace.argtypes = [_i64, _i64, _i64]
        lib.ngpu_lm_kv_fork_workspace.restype = ctypes.c_size_t
        lib.ngpu_lm_kv_fork.argtypes = [p(_Fork), _vp, ctypes.c_size_t, _vp]
        lib.ngpu_lm_kv_copy.argtypes = [p(_Cache), _vp, _i64, _vp]
        lib.ngpu_lm_kv_copy8.argtypes = [p(_Cache8), _vp, _i64, _vp]
        lib.ngpu_lm_kv_compact_workspace.argtypes = [_i64]
        lib.ngpu_lm_kv_compact_workspace.restype = ctypes.c_size_t
        lib.ngpu_lm_kv_compact.argtypes = [_vp, _i64, _i32, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        lib.ngpu_lm_kv_move.argtypes = [_vp, _i64, _i64, _i64, _vp, _i64, _vp]
        _lib = lib
    return _lib


def _pool(refs):
    torch = _torch_mod()
    dev = _device_of(refs, "refs")
    if refs.dim() != 1:
        raise ValueError("refs must be a [pages] tensor")
    return dev, _need(refs, "refs", dev, torch.int32, refs.shape), refs.shape[0]


def kv_fork(pages, lengths, parents, refs, page_size: int, tokens=0, stream=None):
    """Page tables of the hypotheses that go on, from those of the hypotheses before.

    ``pages`` [G * W, width] and ``lengths`` [G * W] int32: the tables and tokens of G groups of W
    hypotheses; ``parents`` [G, K] int32: which of its group's W each of the K new ones continues, any value
    outside [0, W) for none; ``tokens``: how many tokens each is going to append, an int or [G, K] int32.
    ``refs`` [pages of the pool] int32 counts the table entries that hold each page and is updated in place.

    A new row shares its parent's pages.  Where it is going to append into a page that is filled in part and that
    others hold too, it gets a fresh page, to which ``kv_copy`` has to copy what is filled, in each layer's
    cache, before the append; and fresh pages for the tokens behind.  Fresh pages are the lowest free ones, in
    the rows' order.  A row that finds too few, or whose tokens do not fit the table, is dropped: it holds no pages
    and its length is -1.  The caller has to end that hypothesis (a score of -inf in ``beam_step``, nothing to append),
    as a length below 0 counts as 0 in the next call.
    Entries of the old tables are given up: pages that no new row holds are free.  So ``parents`` of
    -1 free a group's pages, a shorter length gives up rejected tokens, and a new sequence is a row of -1 entries
    and length 0 that is forked with its prompt's tokens.

    Returns (pages [G * K, width], lengths [G * K] without the new tokens, copies [G * K, 3]), int32."""
    native = _native()
    if stream is None and native:
        r = native.kv_fork(pages, lengths, parents, refs, page_size, tokens)
        if r is not None:   # None: not the ordinary call, handled (or refused) below
            if r.__class__ is int:
                _check(r)
            return r
    torch = _torch_mod()
    dev, refs_at, P = _pool(refs)
    i32 = torch.int32
    if parents.dim() != 2:
        raise ValueError("parents must be a [G, K] tensor")
    G, K = parents.shape
    if pages.dim() != 2 or (G > 0 and pages.shape[0] % G != 0) or (G == 0 and pages.shape[0] > 0):
        raise ValueError("pages must be a [G * W, width] tensor")
    rows = pages.shape[0]
    a = _Fork(G, rows // G if G else 0, K, page_size=_whole(page_size, "page_size"), num_pages=P, refs=refs_at)
    a.pages, a.width, a.pages_stride = _table(pages, "pages", dev, rows)
    a.lengths = _need(lengths, "lengths", dev, i32, (rows,))
    a.parents = _need(parents, "parents", dev, i32, (G, K))
    if hasattr(tokens, "dim"):
        a.tokens = _need(tokens, "tokens", dev, i32, (G, K))
    else:
        a.T = _whole(tokens, "tokens", 64)
    lib = _library()
    with _on(dev, stream) as handle:
        new = torch.empty((G * K, a.width), dtype=i32, device=dev)
        after = torch.empty(G * K, dtype=i32, device=dev)
        copies = torch.empty((G * K, 3), dtype=i32, device=dev)
        a.out_pages, a.out_lengths, a.copies = new.data_ptr(), after.data_ptr(), copies.data_ptr()
        size = lib.ngpu_lm_kv_fork_workspace(G, K, P)
        workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        _check(lib.ngpu_lm_kv_fork(ctypes.byref(a), workspace.data_ptr(), size, handle))
    return new, after, copies


def kv_copy(k_cache, v_cache, copies, k_scale=None, v_scale=None, stream=None):
    """Copy entries of pages to other pages of a cache [pages, page size, heads, dim], in place.

    ``copies`` [n, 3] int32 of ``kv_fork`` or ``kv_compact``: {from, to, entries} a row; rows with a page outside
    the cache are skipped.  No page may be written by two rows, or written by one and read by another.  Of an
    8-bit cache all scales of a page, ``k_scale`` and ``v_scale`` [pages, blocks, heads] float32, go with it; they may be
    expanded, or one tensor for both, and must not overlap otherwise."""
    native = _native()
    eight = k_scale is not None or v_scale is not None
    if stream is None and native:
        r = native.kv_copy(k_cache, v_cache, copies, *((k_scale, v_scale) if eight else ()))
        if r is not None:
            if r.__class__ is int:
                _check(r)
            return
    torch = _torch_mod()
    dev, cache = _cache8(k_cache, v_cache, k_scale, v_scale, torch.float16) if eight else _cache(k_cache, v_cache)
    if copies.dim() != 2:
        raise ValueError("copies must be a [n, 3] tensor")
    at = _need(copies, "copies", dev, torch.int32, (copies.shape[0], 3))
    _untracked(k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale)
    lib = _library()
    with _on(dev, stream) as handle:
        _check((lib.ngpu_lm_kv_copy8 if eight else lib.ngpu_lm_kv_copy)(ctypes.byref(cache), at, copies.shape[0], handle))


def kv_compact(refs, page_size: int, tables=(), stream=None):
    """Move the used pages of a pool to its lowest numbers.

    With n pages in use (``refs`` other than 0), those from page n on move to the free ones below, in ascending
    order.  ``refs`` and the page ``tables`` (int32 [rows, width] each, all that hold the pool's pages) are
    updated in place; ``kv_copy`` then has to move the pages of each layer's cache.  Tables may be views that share rows:
    an entry that is put through ``moved`` twice stays where the first time put it.

    Returns (copies [pages // 2, 3] int32, moved [pages] int32: each page's new number)."""
    native, tables = _native(), tuple(tables)
    if stream is None and native:
        r = native.kv_compact(refs, page_size, tables)
        if r is not None:
            if r.__class__ is int:
                _check(r)
            return r
    torch = _torch_mod()
    dev, refs_at, P = _pool(refs)
    found = [_table(t, f"tables[{i}]", dev, t.shape[0]) for i, t in enumerate(tables)]
    for i, t in enumerate(tables):
        if t.shape[0] > 1 and t.stride(0) < t.shape[1]:
            raise ValueError(f"the rows of tables[{i}] must not overlap")
    # (views that share entries otherwise do no harm: a page's new place was free, and a free page's number stays)
    starts = [f[0] for f, t in zip(found, tables) if t.numel() > 0]
    if len(set(starts)) < len(starts):
        raise ValueError("a table must not be listed twice")
    page_size, lib = _whole(page_size, "page_size"), _library()
    with _on(dev, stream) as handle:
        copies = torch.empty((P // 2, 3), dtype=torch.int32, device=dev)
        moved = torch.empty(P, dtype=torch.int32, device=dev)
        size = lib.ngpu_lm_kv_compact_workspace(P)
        workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        _check(lib.ngpu_lm_kv_compact(refs_at, P, page_size, copies.data_ptr(), moved.data_ptr(),
                                      workspace.data_ptr(), size, handle))
        for (at, width, stride), t in zip(found, tables):
            _check(lib.ngpu_lm_kv_move(at, t.shape[0], width, stride, moved.data_ptr(), P, handle))
    return copies, moved
