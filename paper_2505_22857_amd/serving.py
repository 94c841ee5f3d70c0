"""Serving operators around a network that the n-gram model drafts for.

``verify`` keeps or replaces drafted tokens given the network's logits,
``kv_append`` rotates and stores new keys and values in a paged cache, and
``attend`` is attention over that cache with the prefix that the sequences of a
group share (the hypotheses of one utterance) read once.  All three enqueue
their HIP kernels on the current stream (or ``stream``) and return; the C ABI is
``include/ngpu_lm.h``.  Page tables, lengths and tokens are int32 tensors.
None has a gradient: ``kv_append`` and ``attend`` refuse tensors that require one
while gradients are recorded.
"""

from __future__ import annotations

import contextlib
import ctypes
import math

from . import _check, _fast_or_none, _stream_handle, _torch_mod, load_library

NGPU_F32, NGPU_F16, NGPU_BF16 = 0, 1, 2
NGPU_ROPE_HALF, NGPU_ROPE_INTERLEAVED = 0, 1
MAX_DRAFT = 63                   # NGPU_LM_MAX_DRAFT
MAX_HEAD_DIM = 256               # NGPU_LM_MAX_HEAD_DIM

_i32, _i64, _vp, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float


class _Verify(ctypes.Structure):
    _fields_ = [("B", _i64), ("K", _i32), ("V", _i64), ("dtype", _i32), ("logits", _vp), ("logits_stride_b", _i64),
                ("logits_stride_k", _i64), ("tokens", _vp), ("lengths", _vp), ("logprobs", _vp),
                ("logprobs_stride_b", _i64), ("logprobs_stride_k", _i64), ("uniforms", _vp), ("noise", _vp),
                ("noise_stride_b", _i64), ("temperature", _f32), ("draft_states", _vp), ("out_tokens", _vp),
                ("accepted", _vp), ("states", _vp)]


class _Cache(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("heads", _i32), ("dim", _i32), ("page_size", _i32), ("num_pages", _i64),
                ("k", _vp), ("v", _vp), ("k_stride_page", _i64), ("k_stride_token", _i64), ("k_stride_head", _i64),
                ("v_stride_page", _i64), ("v_stride_token", _i64), ("v_stride_head", _i64)]


class _Append(ctypes.Structure):
    _fields_ = [("S", _i64), ("T", _i64), ("k", _vp), ("v", _vp), ("k_stride_seq", _i64), ("k_stride_token", _i64),
                ("k_stride_head", _i64), ("v_stride_seq", _i64), ("v_stride_token", _i64), ("v_stride_head", _i64),
                ("q", _vp), ("q_heads", _i32), ("q_stride_seq", _i64), ("q_stride_token", _i64),
                ("q_stride_head", _i64), ("q_out", _vp), ("pages", _vp), ("pages_width", _i64),
                ("pages_stride", _i64), ("start", _vp), ("lengths", _vp), ("rotary", _i32), ("layout", _i32),
                ("positions", _vp), ("cos", _vp), ("sin", _vp), ("positions_count", _i64)]


class _Attend(ctypes.Structure):
    _fields_ = [("S", _i64), ("T", _i64), ("q_heads", _i32), ("q", _vp), ("q_stride_seq", _i64),
                ("q_stride_token", _i64), ("q_stride_head", _i64), ("q_lengths", _vp), ("G", _i64),
                ("prefix_pages", _vp), ("prefix_width", _i64), ("prefix_stride", _i64), ("prefix_lengths", _vp),
                ("pages", _vp), ("pages_width", _i64), ("pages_stride", _i64), ("lengths", _vp), ("scale", _f32),
                ("out", _vp), ("lse", _vp)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        p = ctypes.POINTER
        lib.ngpu_lm_verify_workspace.argtypes = [_i64, _i32, _i64]
        lib.ngpu_lm_verify_workspace.restype = ctypes.c_size_t
        lib.ngpu_lm_verify.argtypes = [p(_Verify), _vp, ctypes.c_size_t, _vp]
        lib.ngpu_lm_kv_append.argtypes = [p(_Cache), p(_Append), _vp]
        lib.ngpu_lm_attend_workspace.argtypes = [p(_Cache), p(_Attend)]
        lib.ngpu_lm_attend_workspace.restype = ctypes.c_size_t
        lib.ngpu_lm_attend.argtypes = [p(_Cache), p(_Attend), _vp, ctypes.c_size_t, _vp]
        _lib = lib
    return _lib


_native_module = None


def _native():
    """The native per-call module, False where it cannot be used (said once)."""
    global _native_module
    if _native_module is None:
        _native_module = _fast_or_none() or False
    return _native_module


def _type_code(dtype):
    torch = _torch_mod()
    return {torch.float32: NGPU_F32, torch.float16: NGPU_F16, torch.bfloat16: NGPU_BF16}.get(dtype)


@contextlib.contextmanager
def _on(device, stream):
    """Runs on the tensors' device, and allocates for the stream that the work is enqueued on: what is
    freed when the call returns is then handed out again in that stream's order."""
    torch = _torch_mod()
    if stream is not None and stream.device != device:
        raise ValueError(f"the stream belongs to {stream.device}, the tensors are on {device}")
    with contextlib.ExitStack() as stack:
        if device.index != torch.cuda.current_device():
            stack.enter_context(torch.cuda.device(device))
        if stream is not None:
            stack.enter_context(torch.cuda.stream(stream))
        yield _stream_handle(stream, device.index)


def _need(t, name, device, dtype, shape, rows=False):
    """Address of a device tensor of this type and shape; contiguous, or with ``rows`` of unit stride in
    its last dimension."""
    if t is None:
        return None
    if not hasattr(t, "is_cuda") or not t.is_cuda or t.device != device or t.dtype is not dtype:
        raise TypeError(f"{name} must be a {dtype} tensor on {device}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if rows:
        if t.shape[-1] > 1 and t.stride(-1) != 1 and t.numel() > 0:
            raise TypeError(f"{name} must have unit stride in the last dimension")
    elif not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    return t.data_ptr()


def _temperature(t):
    """A float as the library is to check it: what fp32 would round to 0, which is greedy, stays one that is refused."""
    t = float(t)
    return math.copysign(1e-30, t) if 0.0 < abs(t) < 1e-30 else t


def _untracked(**tensors):
    """Nothing here has a backward pass, and a result without its graph would be wrong in silence."""
    if _torch_mod().is_grad_enabled():
        for name, t in tensors.items():
            if t is not None and t.requires_grad:
                raise TypeError(f"{name} must not require a gradient: this call has none (torch.no_grad() or detach())")


def _device_of(t, name):
    if not hasattr(t, "is_cuda") or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    return t.device


def verify(logits, tokens, logprobs=None, uniforms=None, noise=None, temperature: float = 1.0, lengths=None,
           draft_states=None, stream=None):
    """Keep the drafted tokens that the network's distribution allows and add one token.

    ``logits`` [B, K + 1, V] (float32, float16 or bfloat16): row k scores the token at place k.
    ``tokens`` [B, K] int32: the draft (a token outside [0, V) ends it); ``lengths`` [B]: how many of
    them count.  ``logprobs`` [B, K, V] float32: the draft's log-probabilities (-inf for classes that it does
    not know, as an end of sequence), None where every drafted token had probability 1.  ``uniforms`` [B, K] in [0, 1) and ``noise`` [B, V], unit exponential,
    float32: the random numbers.  ``temperature`` 0: greedy, without the last three.
    ``draft_states`` [B, K + 1] int32 of ``NgpuLM.draft``.

    Returns (tokens [B, K + 1] int32: the kept ones, the added one, then -1; kept tokens [B] int32; the
    n-gram state [B] int32 after the kept tokens, None without ``draft_states``).  The added token is the
    next draft's ``last``."""
    native = _native()
    if stream is None and native:
        r = native.verify(logits, tokens, logprobs, uniforms, noise, float(temperature), lengths, draft_states)
        if r is not None:   # None: not the ordinary call, handled (or refused) below
            if r.__class__ is int:
                _check(r)
            return r
    torch = _torch_mod()
    dev = _device_of(logits, "logits")
    if logits.dim() != 3 or logits.shape[1] < 1:
        raise ValueError("logits must be a [B, K + 1, V] tensor")
    B, K, V = logits.shape[0], logits.shape[1] - 1, logits.shape[2]
    code = _type_code(logits.dtype)
    if code is None:
        raise TypeError("logits must be float32, float16 or bfloat16")
    temperature = _temperature(temperature)
    sample = temperature != 0.0
    if sample and (noise is None or (K > 0 and uniforms is None)):
        raise ValueError("sampling needs uniforms and noise")
    f32, i32 = torch.float32, torch.int32
    a = _Verify(B, K, V, code, _need(logits, "logits", dev, logits.dtype, (B, K + 1, V), rows=True),
                logits.stride(0), logits.stride(1), _need(tokens, "tokens", dev, i32, (B, K)),
                _need(lengths, "lengths", dev, i32, (B,)), temperature=temperature)
    if sample:
        a.uniforms = _need(uniforms, "uniforms", dev, f32, (B, K))
        a.noise, a.noise_stride_b = _need(noise, "noise", dev, f32, (B, V), rows=True), noise.stride(0)
        if logprobs is not None:
            a.logprobs = _need(logprobs, "logprobs", dev, f32, (B, K, V), rows=True)
            a.logprobs_stride_b, a.logprobs_stride_k = logprobs.stride(0), logprobs.stride(1)
    a.draft_states = _need(draft_states, "draft_states", dev, i32, (B, K + 1))
    lib = _library()
    with _on(dev, stream) as handle:
        out = torch.empty((B, K + 1), dtype=i32, device=dev)
        accepted = torch.empty(B, dtype=i32, device=dev)
        states = torch.empty(B, dtype=i32, device=dev) if draft_states is not None else None
        size = lib.ngpu_lm_verify_workspace(B, K, V)
        workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        a.out_tokens, a.accepted = out.data_ptr(), accepted.data_ptr()
        a.states = states.data_ptr() if states is not None else None
        _check(lib.ngpu_lm_verify(ctypes.byref(a), workspace.data_ptr(), size, handle))
    return out, accepted, states


def _cache(k_cache, v_cache):
    dev = _device_of(k_cache, "k_cache")
    code = _type_code(k_cache.dtype)
    if code not in (NGPU_F16, NGPU_BF16):
        raise TypeError("the cache must be float16 or bfloat16")
    if k_cache.dim() != 4:
        raise ValueError("the cache must be a [pages, page size, heads, dim] tensor")
    pages, page_size, heads, dim = k_cache.shape
    return dev, _Cache(code, heads, dim, page_size, pages,
                       _need(k_cache, "k_cache", dev, k_cache.dtype, k_cache.shape, rows=True),
                       _need(v_cache, "v_cache", dev, k_cache.dtype, k_cache.shape, rows=True),
                       *k_cache.stride()[:3], *v_cache.stride()[:3])


def _table(t, name, dev, rows):
    torch = _torch_mod()
    if t.dim() != 2:
        raise ValueError(f"{name} must be a [{rows}, width] tensor")
    return _need(t, name, dev, torch.int32, (rows, t.shape[1]), rows=True), t.shape[1], t.stride(0)


def kv_append(k, v, k_cache, v_cache, pages, start, positions=None, cos=None, sin=None,
              layout: int = NGPU_ROPE_HALF, q=None, lengths=None, stream=None):
    """Store new keys and values in a paged cache, rotating keys and queries on the way.

    ``k``, ``v`` [S, T, heads, dim] go to places ``start[s] + t`` of the sequences' own tokens, entry
    ``place % page size`` of page ``pages[s, place // page size]`` of ``k_cache`` and ``v_cache`` [pages,
    page size, heads, dim]; only the first ``lengths[s]`` of a sequence's T tokens count.  With ``cos`` and
    ``sin`` [positions, rotary / 2] (``rope_table``) the first ``rotary`` dimensions of the keys, and of
    ``q`` [S, T, q heads, dim], are rotated by row ``positions[s, t]`` (without it: the token's place).
    Returns the rotated queries (zero where a token does not count), None without ``q``."""
    native = _native()
    if stream is None and native:
        r = native.kv_append(k, v, k_cache, v_cache, pages, start, positions, cos, sin, layout, q, lengths)
        if r is not None:
            if r.__class__ is int:
                _check(r)
            return r if q is not None else None
    torch = _torch_mod()
    dev, cache = _cache(k_cache, v_cache)
    if k.dim() != 4:
        raise ValueError("k must be a [S, T, heads, dim] tensor")
    S, T = k.shape[:2]
    shape, dt, i32 = (S, T, cache.heads, cache.dim), k_cache.dtype, torch.int32
    a = _Append(S, T, _need(k, "k", dev, dt, shape, rows=True), _need(v, "v", dev, dt, shape, rows=True),
                *k.stride()[:3], *v.stride()[:3])
    a.pages, a.pages_width, a.pages_stride = _table(pages, "pages", dev, S)
    a.start = _need(start, "start", dev, i32, (S,))
    a.lengths = _need(lengths, "lengths", dev, i32, (S,))
    a.layout = int(layout)
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin come together")
    if cos is not None:
        if cos.dim() != 2:
            raise ValueError("cos must be a [positions, rotary / 2] tensor")
        a.rotary, a.positions_count = 2 * cos.shape[1], cos.shape[0]
        a.cos = _need(cos, "cos", dev, torch.float32, cos.shape)
        a.sin = _need(sin, "sin", dev, torch.float32, cos.shape)
        a.positions = _need(positions, "positions", dev, i32, (S, T))
    if q is not None:
        if q.dim() != 4:
            raise ValueError("q must be a [S, T, q heads, dim] tensor")
        a.q_heads = q.shape[2]
        a.q = _need(q, "q", dev, dt, (S, T, q.shape[2], cache.dim), rows=True)
        a.q_stride_seq, a.q_stride_token, a.q_stride_head = q.stride()[:3]
    _untracked(k=k, v=v, k_cache=k_cache, v_cache=v_cache, q=q, cos=cos, sin=sin)
    with _on(dev, stream) as handle:
        out = torch.empty(q.shape, dtype=dt, device=dev) if q is not None else None
        a.q_out = out.data_ptr() if out is not None else None
        _check(_library().ngpu_lm_kv_append(ctypes.byref(cache), ctypes.byref(a), handle))
    return out


def attend(q, k_cache, v_cache, pages=None, lengths=None, prefix_pages=None, prefix_lengths=None, q_lengths=None,
           scale=None, return_lse: bool = False, stream=None):
    """Attention of ``q`` [S, T, q heads, dim] over a paged cache [pages, page size, heads, dim].

    With ``prefix_pages`` [G, width] and ``prefix_lengths`` [G], consecutive sequences in G groups of
    S / G share their group's prefix, which is read once for all of them.  With ``pages`` [S, width] and
    ``lengths`` [S], each sequence has tokens of its own after it, the T query tokens (or the first
    ``q_lengths[s]`` of them) being the last: query t sees the whole prefix and the own tokens up to its
    own.  ``scale`` is 1 / sqrt(dim) unless given.  Dimensions and strides in multiples of 8, 16-byte alignment and
    pages that span at most 32 GiB take the matrix cores; other caches a kernel many times slower.

    Returns [S, T, q heads, dim] (zero where a row sees no key or does not count), and with
    ``return_lse`` the log of each row's softmax sum [S, T, q heads] float32 (-inf there)."""
    native = _native()
    if stream is None and native and not return_lse:
        r = native.attend(q, k_cache, v_cache, pages, lengths, prefix_pages, prefix_lengths, q_lengths,
                          scale if scale is None else float(scale))
        if r is not None:
            if r.__class__ is int:
                _check(r)
            return r
    torch = _torch_mod()
    dev, cache = _cache(k_cache, v_cache)
    if q.dim() != 4:
        raise ValueError("q must be a [S, T, q heads, dim] tensor")
    S, T, heads, dt, i32 = q.shape[0], q.shape[1], q.shape[2], k_cache.dtype, torch.int32
    a = _Attend(S, T, heads, _need(q, "q", dev, dt, (S, T, heads, cache.dim), rows=True), *q.stride()[:3],
                _need(q_lengths, "q_lengths", dev, i32, (S,)),
                scale=1.0 / math.sqrt(cache.dim) if scale is None else float(scale))
    if (prefix_pages is None) != (prefix_lengths is None) or (pages is None) != (lengths is None):
        raise ValueError("page tables and lengths come together")
    if prefix_pages is not None:
        a.G = prefix_pages.shape[0]
        a.prefix_pages, a.prefix_width, a.prefix_stride = _table(prefix_pages, "prefix_pages", dev, a.G)
        a.prefix_lengths = _need(prefix_lengths, "prefix_lengths", dev, i32, (a.G,))
        if a.G == 0 and S > 0:
            raise ValueError("prefix_pages must hold a row for every group")
    if pages is not None:
        a.pages, a.pages_width, a.pages_stride = _table(pages, "pages", dev, S)
        a.lengths = _need(lengths, "lengths", dev, i32, (S,))
        if a.pages_width == 0:
            a.pages = None   # a table without pages holds no own tokens
    _untracked(q=q, k_cache=k_cache, v_cache=v_cache)
    lib = _library()
    with _on(dev, stream) as handle:
        out = torch.empty(q.shape, dtype=dt, device=dev)
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=dev) if return_lse else None
        a.out, a.lse = out.data_ptr(), lse.data_ptr() if return_lse else None
        size = lib.ngpu_lm_attend_workspace(ctypes.byref(cache), ctypes.byref(a))
        workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        _check(lib.ngpu_lm_attend(ctypes.byref(cache), ctypes.byref(a), workspace.data_ptr(), size, handle))
    return (out, lse) if return_lse else out


def rope_table(count: int, rotary: int, base: float = 10000.0, scale: float = 1.0, frequencies=None, device="cuda"):
    """Cosines and sines [count, rotary / 2] float32 of positions 0 .. count - 1, computed in 64 bits.

    Pair i turns by position / ``scale`` times ``base ** (-2 i / rotary)`` (``scale`` > 1 stretches the
    positions for contexts longer than the model was trained on), or times ``frequencies[i]``."""
    torch = _torch_mod()
    if rotary < 0 or rotary % 2 != 0:
        raise ValueError("rotary must be even")
    if frequencies is None:
        frequencies = float(base) ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / max(rotary, 1))
    frequencies = torch.as_tensor(frequencies, dtype=torch.float64)
    if tuple(frequencies.shape) != (rotary // 2,):
        raise ValueError(f"frequencies must hold {rotary // 2} values")
    angle = torch.arange(count, dtype=torch.float64)[:, None] / float(scale) * frequencies.cpu()
    return angle.cos().float().to(device), angle.sin().float().to(device)
