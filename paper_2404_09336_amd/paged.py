"""ctypes binding of the operators on a key / value cache in pages, with the names of the C entry points of
include/span_paged.h.

Tensors are torch tensors that already live on one GPU, which has to be the current device; this module only checks their
types, shapes and contiguity, fills the descriptor, and passes raw device pointers and the current HIP stream.
"""
import ctypes

import numpy as np

from .binding import PreparedCall, SpanAttnError, _dtype_code, load_library

PAGED_DECODE, PAGED_DECODE_WEIGHTS, PAGED_SPAN_DECODE, PAGED_SPAN_DECODE_WEIGHTS, PAGED_PROMPT, PAGED_EVICT = range(6)


class _PagedDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "heads", "kv_heads", "head_dim", "dtype", "page_size", "num_pages", "table_pages",
                                              "num_tokens", "window", "sinks", "num_intervals", "num_splits", "budget", "recent")]
    _fields_ += [("tokens_per_seq", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                 ("stream", ctypes.c_void_p)]


_signed = False


def _library():
    global _signed
    lib = load_library()
    if not _signed:
        P, F, DP = ctypes.c_void_p, ctypes.c_float, ctypes.POINTER(_PagedDesc)
        for name, args in (("paged_append", [P] * 9), ("paged_decode_attn", [P] * 5 + [F, P, P]), ("paged_span_decode_attn", [P] * 7 + [F, P, P]),
                           ("paged_prompt_attn", [P] * 6 + [F, P]), ("paged_evict", [P] * 9), ("paged_workspace_init", []), ("paged_check", [])):
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = [DP] + args, ctypes.c_int
        lib.paged_workspace_bytes.argtypes, lib.paged_workspace_bytes.restype = [DP, ctypes.c_int], ctypes.c_size_t
        _signed = True
    return lib


def make_paged_desc(batch, heads, kv_heads, head_dim, dtype_code, page_size, num_pages, table_pages, *, num_tokens=0, window=0, sinks=0,
                    num_intervals=0, num_splits=0, budget=0, recent=0, tokens_per_seq=None, workspace_ptr=0, workspace_bytes=0, stream=0):
    """tokens_per_seq: host int64 numpy array [batch] or None; the descriptor keeps a reference to it."""
    for name, v in (("window", window), ("sinks", sinks), ("budget", budget), ("recent", recent), ("num_splits", num_splits)):
        if not 0 <= int(v) < 1 << 31:
            raise ValueError(f"{name} must lie in [0, 2^31)")
    d = _PagedDesc(int(batch), int(heads), int(kv_heads), int(head_dim), int(dtype_code), int(page_size), int(num_pages), int(table_pages),
                   int(num_tokens), int(window), int(sinks), int(num_intervals), int(num_splits), int(budget), int(recent), None,
                   workspace_ptr or None, int(workspace_bytes), stream or None)
    if tokens_per_seq is not None:
        tok = np.ascontiguousarray(tokens_per_seq, dtype=np.int64).reshape(-1)
        if tok.shape[0] != batch:
            raise ValueError("tokens_per_seq must have one entry per sequence")
        d._tokens_keepalive = tok
        d.tokens_per_seq = tok.ctypes.data
    return d


def paged_workspace_bytes(desc, use) -> int:
    return int(_library().paged_workspace_bytes(ctypes.byref(desc), int(use)))


def paged_workspace_init(desc) -> None:
    """Zeroes the ticket counters at the head of desc.workspace (enqueued on desc.stream)."""
    rc = _library().paged_workspace_init(ctypes.byref(desc))
    if rc != 0:
        raise SpanAttnError(rc, "paged_workspace_init")


def _on_gpu(t, name, dtype, shape, device):
    """A contiguous GPU tensor of this type and shape (None: any) on `device`, aligned to 16 bytes."""
    if t.dtype != dtype or t.device != device or not t.is_contiguous() or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape) if shape is not None else 'any'} on {device}")
    if t.data_ptr() % 16 and t.numel():
        raise ValueError(f"{name} must be aligned to 16 bytes")
    return t.data_ptr()


def _cache(k_pages, v_pages, block_table, ctx_lens):
    """What every call checks: (batch, kv_heads, page_size, head_dim, num_pages, table_pages, device)."""
    import torch
    if not k_pages.is_cuda or k_pages.dim() != 4 or block_table.dim() != 2:
        raise ValueError("expected GPU tensors k_pages / v_pages [num_pages, kv_heads, page_size, head_dim] and block_table [batch, table_pages]")
    device = k_pages.device
    if device.index != torch.cuda.current_device():
        raise ValueError(f"the tensors lie on {device}, which is not the current device")
    num_pages, kv_heads, page_size, head_dim = k_pages.shape
    batch, table_pages = block_table.shape
    _on_gpu(k_pages, "k_pages", k_pages.dtype, None, device)
    _on_gpu(v_pages, "v_pages", k_pages.dtype, k_pages.shape, device)
    _on_gpu(block_table, "block_table", torch.int32, None, device)
    if ctx_lens is not None:
        _on_gpu(ctx_lens, "ctx_lens", torch.int32, (batch,), device)
    return batch, kv_heads, page_size, head_dim, num_pages, table_pages, device


def _stream(stream, device):
    import torch
    return torch.cuda.current_stream(device).cuda_stream if stream is None else stream


def _allocations(stream, device):
    """Context in which new tensors are allocated, filled and later handed on in the order of the call's stream, whichever the current one is."""
    import contextlib
    import torch
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device))


def _take_workspace(desc, use, workspace, stream, device, counters):
    """Workspace of the call; one that the caller hands in must have been initialised (paged_workspace_init) where it has counters."""
    import torch
    need = paged_workspace_bytes(desc, use)
    if need == 0:
        return None
    fresh = workspace is None
    if fresh:
        with _allocations(stream, device):
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
    elif workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    desc.workspace = workspace.data_ptr()
    desc.workspace_bytes = workspace.numel() * workspace.element_size()
    if fresh and counters:
        paged_workspace_init(desc)
    return workspace


def _check(desc, name):
    """A descriptor that the library would refuse is refused before anything is sized by it."""
    rc = _library().paged_check(ctypes.byref(desc))
    if rc != 0:
        raise SpanAttnError(rc, name)


def prepare_paged_append(k_new, v_new, k_pages, v_pages, block_table, ctx_lens, q_offsets=None, *, positions=None, seen=None,
                         stream=None) -> PreparedCall:
    """k_new, v_new [num_tokens, kv_heads, head_dim]; ctx_lens counts the new rows already; q_offsets int32 [batch + 1], None = one token per
    sequence.  positions int32 [batch, kv_heads, table_pages * page_size] and seen int32 [batch]: see span_paged.h.  Calling it returns
    (k_pages, v_pages)."""
    import torch
    B, KV, P, D, N, TP, device = _cache(k_pages, v_pages, block_table, ctx_lens)
    T = k_new.shape[0]
    _on_gpu(k_new, "k_new", k_pages.dtype, (T, KV, D), device)
    _on_gpu(v_new, "v_new", k_pages.dtype, (T, KV, D), device)
    if q_offsets is None and T != B:
        raise ValueError("without q_offsets there is one new token per sequence")
    opt = lambda t, name, shape: None if t is None else _on_gpu(t, name, torch.int32, shape, device)  # noqa: E731
    args = (opt(q_offsets, "q_offsets", (B + 1,)), opt(positions, "positions", (B, KV, TP * P)), opt(seen, "seen", (B,)))
    desc = make_paged_desc(B, KV, KV, D, _dtype_code(k_pages), P, N, TP, num_tokens=T, stream=_stream(stream, device))
    args = (ctypes.byref(desc), k_new.data_ptr(), v_new.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), block_table.data_ptr(), ctx_lens.data_ptr(), *args)
    keep = (k_new, v_new, block_table, ctx_lens, q_offsets, positions, seen)
    return PreparedCall("paged_append", _library().paged_append, desc, args, (k_pages, v_pages), keep)


def paged_append(k_new, v_new, k_pages, v_pages, block_table, ctx_lens, q_offsets=None, **kw):
    """Writes the new tokens' K / V rows into their pages.  Returns (k_pages, v_pages)."""
    return prepare_paged_append(k_new, v_new, k_pages, v_pages, block_table, ctx_lens, q_offsets, **kw)()


def _prepare_decode(name, q, k_pages, v_pages, block_table, ctx_lens, spans, scale, out, window, sinks, weights, num_splits, workspace, stream,
                    tokens_per_seq):
    import torch
    lib = _library()
    B, KV, P, D, N, TP, device = _cache(k_pages, v_pages, block_table, ctx_lens)
    if q.dim() != 3:
        raise ValueError("expected q [batch, heads, head_dim]")
    H = q.shape[1]
    _on_gpu(q, "q", k_pages.dtype, (B, H, D), device)
    if out is None:
        with _allocations(stream, device):
            out = torch.empty((B, H, D), dtype=torch.float32, device=device)
    _on_gpu(out, "out", torch.float32, (B, H, D), device)
    weights_ptr = None if weights is None else _on_gpu(weights, "weights", torch.float32, (B, KV, TP * P), device)
    n_int = 0
    if spans is not None:
        off, st, en = spans
        n_int = int(st.numel())
        _on_gpu(off, "span_offsets", torch.int32, (B + 1,), device)
        _on_gpu(st, "span_starts", torch.int32, (n_int,), device)
        _on_gpu(en, "span_ends", torch.int32, (n_int,), device)
    desc = make_paged_desc(B, H, KV, D, _dtype_code(k_pages), P, N, TP, window=window, sinks=sinks, num_intervals=n_int, num_splits=num_splits,
                           tokens_per_seq=tokens_per_seq, stream=_stream(stream, device))
    _check(desc, name)
    use = (PAGED_DECODE if spans is None else PAGED_SPAN_DECODE) + (weights is not None)
    workspace = _take_workspace(desc, use, workspace, stream, device, True)
    lists = (ctx_lens,) if spans is None else spans
    args = (ctypes.byref(desc), q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), block_table.data_ptr(), *(t.data_ptr() for t in lists),
            float(scale), weights_ptr, out.data_ptr())
    keep = (q, k_pages, v_pages, block_table, *lists, weights, workspace)
    return PreparedCall(name, getattr(lib, name), desc, args, out, keep)


def prepare_paged_decode_attn(q, k_pages, v_pages, block_table, ctx_lens, scale, out=None, *, window=0, sinks=0, weights=None, num_splits=0,
                              workspace=None, stream=None) -> PreparedCall:
    """q [batch, heads, head_dim], ctx_lens int32 GPU tensor [batch], out fp32 shaped like q.  weights: fp32 [batch, kv_heads, table_pages *
    page_size], to which the attention weights are added."""
    return _prepare_decode("paged_decode_attn", q, k_pages, v_pages, block_table, ctx_lens, None, scale, out, window, sinks, weights, num_splits,
                           workspace, stream, None)


def paged_decode_attn(q, k_pages, v_pages, block_table, ctx_lens, scale, out=None, **kw):
    """One token per sequence attends its cache in pages: all of it, or the last `window` positions and the first `sinks`.  Returns `out`."""
    return prepare_paged_decode_attn(q, k_pages, v_pages, block_table, ctx_lens, scale, out, **kw)()


def prepare_paged_span_decode_attn(q, k_pages, v_pages, block_table, span_offsets, span_starts, span_ends, scale, out=None, *, weights=None,
                                   num_splits=0, workspace=None, stream=None, tokens_per_seq=None) -> PreparedCall:
    """The same over span lists (device int32 tensors); tokens_per_seq: host counts as span_validate returns them."""
    return _prepare_decode("paged_span_decode_attn", q, k_pages, v_pages, block_table, None, (span_offsets, span_starts, span_ends), scale, out, 0, 0,
                           weights, num_splits, workspace, stream, tokens_per_seq)


def paged_span_decode_attn(q, k_pages, v_pages, block_table, span_offsets, span_starts, span_ends, scale, out=None, **kw):
    """span_decode_attn over a cache in pages.  Returns `out`."""
    return prepare_paged_span_decode_attn(q, k_pages, v_pages, block_table, span_offsets, span_starts, span_ends, scale, out, **kw)()


def prepare_paged_prompt_attn(q, k_pages, v_pages, block_table, ctx_lens, q_offsets, scale, out=None, *, window=0, sinks=0, workspace=None,
                              stream=None) -> PreparedCall:
    """q [num_tokens, heads, head_dim], q_offsets int32 GPU tensor [batch + 1], out shaped and typed like q."""
    import torch
    lib = _library()
    B, KV, P, D, N, TP, device = _cache(k_pages, v_pages, block_table, ctx_lens)
    if q.dim() != 3:
        raise ValueError("expected q [num_tokens, heads, head_dim]")
    T, H = q.shape[:2]
    _on_gpu(q, "q", k_pages.dtype, (T, H, D), device)
    _on_gpu(q_offsets, "q_offsets", torch.int32, (B + 1,), device)
    if out is None:
        with _allocations(stream, device):
            out = torch.empty_like(q)
    _on_gpu(out, "out", q.dtype, (T, H, D), device)
    desc = make_paged_desc(B, H, KV, D, _dtype_code(k_pages), P, N, TP, num_tokens=T, window=window, sinks=sinks, stream=_stream(stream, device))
    _check(desc, "paged_prompt_attn")
    workspace = _take_workspace(desc, PAGED_PROMPT, workspace, stream, device, False)
    args = (ctypes.byref(desc), q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), block_table.data_ptr(), ctx_lens.data_ptr(), q_offsets.data_ptr(),
            float(scale), out.data_ptr())
    keep = (q, k_pages, v_pages, block_table, ctx_lens, q_offsets, workspace)
    return PreparedCall("paged_prompt_attn", lib.paged_prompt_attn, desc, args, out, keep)


def paged_prompt_attn(q, k_pages, v_pages, block_table, ctx_lens, q_offsets, scale, out=None, **kw):
    """Causal attention of the new tokens of every sequence over its cache, optionally with a window and sinks.  Returns `out`."""
    return prepare_paged_prompt_attn(q, k_pages, v_pages, block_table, ctx_lens, q_offsets, scale, out, **kw)()


def prepare_paged_evict(k_pages, v_pages, block_table, ctx_lens, weights, budget, *, sinks=0, recent=0, positions=None, weights_out=None,
                        positions_out=None, new_lens=None, workspace=None, stream=None) -> PreparedCall:
    """weights fp32 and positions int32 (or None) [batch, kv_heads, table_pages * page_size].  weights_out, positions_out and new_lens may be the
    arrays themselves; left out, they are new (zeros, -1) ones.  Calling it returns (weights_out, positions_out, new_lens)."""
    import torch
    lib = _library()
    B, KV, P, D, N, TP, device = _cache(k_pages, v_pages, block_table, ctx_lens)
    _on_gpu(weights, "weights", torch.float32, (B, KV, TP * P), device)
    with _allocations(stream, device):
        weights_out = torch.zeros_like(weights) if weights_out is None else weights_out
        new_lens = torch.empty_like(ctx_lens) if new_lens is None else new_lens
        if positions is not None and positions_out is None:
            positions_out = torch.full_like(positions, -1)
    _on_gpu(weights_out, "weights_out", torch.float32, (B, KV, TP * P), device)
    if positions is not None:
        _on_gpu(positions, "positions", torch.int32, (B, KV, TP * P), device)
        _on_gpu(positions_out, "positions_out", torch.int32, (B, KV, TP * P), device)
    elif positions_out is not None:
        raise ValueError("positions_out needs positions")
    _on_gpu(new_lens, "new_lens", torch.int32, (B,), device)
    desc = make_paged_desc(B, KV, KV, D, _dtype_code(k_pages), P, N, TP, sinks=sinks, budget=budget, recent=recent, stream=_stream(stream, device))
    _check(desc, "paged_evict")
    workspace = _take_workspace(desc, PAGED_EVICT, workspace, stream, device, True)
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    args = (ctypes.byref(desc), k_pages.data_ptr(), v_pages.data_ptr(), block_table.data_ptr(), ctx_lens.data_ptr(), weights.data_ptr(), ptr(positions),
            weights_out.data_ptr(), ptr(positions_out), new_lens.data_ptr())
    keep = (k_pages, v_pages, block_table, ctx_lens, weights, positions, workspace)
    return PreparedCall("paged_evict", lib.paged_evict, desc, args, (weights_out, positions_out, new_lens), keep)


def paged_evict(k_pages, v_pages, block_table, ctx_lens, weights, budget, **kw):
    """Cuts every cache down to `budget` rows per KV head, in place.  Returns (weights_out, positions_out, new_lens)."""
    return prepare_paged_evict(k_pages, v_pages, block_table, ctx_lens, weights, budget, **kw)()
