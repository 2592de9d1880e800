"""Binding of the rotary positions and the paged 8-bit key/value cache of include/flat_attn.h.  Same names as the C entry points; as in
binding.py, arguments are checked and marshalled and nothing is computed here."""
from __future__ import annotations

import ctypes

from . import binding as _b
from .binding import FLAT_MASK_NONE, FlatCache8Struct, _check, _load_torch, load_library

FLAT_CACHE8_BLOCK = 16
FLAT_CACHE8_E4M3 = 0
FLAT_CACHE8_INT8 = 1
FLAT_CACHE8_MAX_LISTED_PAGES = 1 << 20
FLAT_ROPE_HALF = 0
FLAT_ROPE_INTERLEAVED = 1
FLAT_ROPE_SCALE_NONE = 0
FLAT_ROPE_SCALE_LINEAR = 1
FLAT_ROPE_SCALE_BASE = 2
FLAT_ROPE_SCALE_BANDS = 3


def _lib():
    return _b._lib or load_library()


def _torch():
    return _b._torch or _load_torch()


def _stream_on(tensor, stream) -> int:
    """The handle of the stream to enqueue on.  Without one it is the current stream of the current device, which has to be the tensors' own."""
    if stream is not None:
        if stream.device_index != tensor.get_device():
            raise ValueError("the stream belongs to another device than the tensors")
        return int(stream.cuda_stream)
    device = tensor.get_device()
    if _b._device() != device:
        raise ValueError(f"the tensors live on GPU {device}, which is not the current device")
    return _b._raw_stream(device)


def _ints(name, t, device, shape):
    if t.dtype is not _b._torch.int32 or not t.is_cuda or t.get_device() != device or not t.is_contiguous() or tuple(t.shape) != shape:
        raise ValueError(f"{name} must be a contiguous int32 tensor of shape {list(shape)} on the GPU of the other tensors")
    return t.data_ptr()


class FlatCache8:
    """A paged cache of keys and values in 8 bits: `k`, `v` uint8 [n_pages, n_heads, page_tokens, d] (the bytes of a page lie in the order of
    flat_cache8 in the header), `k_scale`, `v_scale` float32 [n_pages, n_heads, page_tokens / 16], GPU tensors, kept alive by this object."""

    def __init__(self, k, v, k_scale, v_scale, format: int = FLAT_CACHE8_E4M3):
        torch = _torch()
        if k.dim() != 4 or k.dtype != torch.uint8 or v.dtype != torch.uint8 or v.shape != k.shape:
            raise ValueError("k and v must be uint8 tensors of one shape [n_pages, n_heads, page_tokens, d]")
        n_pages, n_heads, page_tokens, d = k.shape
        for t in (k_scale, v_scale):
            if t.dtype != torch.float32 or tuple(t.shape) != (n_pages, n_heads, page_tokens // FLAT_CACHE8_BLOCK):
                raise ValueError("k_scale and v_scale must be float32 tensors [n_pages, n_heads, page_tokens / 16]")
        for t in (k, v, k_scale, v_scale):
            if not t.is_cuda or not t.is_contiguous() or t.get_device() != k.get_device():
                raise ValueError("the cache's tensors must be contiguous and live on one GPU")
        self.k, self.v, self.k_scale, self.v_scale, self.format = k, v, k_scale, v_scale, int(format)
        self.n_pages, self.n_heads, self.page_tokens, self.d = n_pages, n_heads, page_tokens, d
        self._device = k.get_device()
        self._struct = FlatCache8Struct(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), n_pages, n_heads, page_tokens, d, int(format))
        self._ref = ctypes.byref(self._struct)


def flat_attn_rope_freqs(rot_d: int, base: float = 10000.0, scaling: int = FLAT_ROPE_SCALE_NONE, factor: float = 1.0, original_len: float = 0.0,
                         low: float = 1.0, high: float = 32.0):
    """Frequencies for flat_attn_rope as a float64 CPU tensor of rot_d / 2 entries."""
    torch = _torch()
    if not 2 <= int(rot_d) <= 256:
        _check(-3)
    out = torch.empty(int(rot_d) // 2, dtype=torch.float64)
    _check(_lib().flat_attn_rope_freqs(out.data_ptr(), int(rot_d), float(base), int(scaling), float(factor), float(original_len), float(low), float(high)))
    return out


def flat_attn_rope(Q, Q_out, K, K_out, freqs, positions=None, layout: int = FLAT_ROPE_HALF, magnitude: float = 1.0, transpose: bool = False,
                   stream=None) -> None:
    """Rotary positions of Q [B,Hq,N,d] and, unless None, K [B,Hk,N,d], bf16 or float32 device tensors, into Q_out and K_out (which may be Q and K).
    `freqs`: float64 device tensor of rot_d / 2 radians per position; `positions`: int32 device tensor [B,N], or None for 0 .. N - 1.
    transpose: turn the other way, which is the gradient."""
    torch = _torch()
    dtype, shape, device = Q.dtype, Q.shape, Q.get_device()
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise ValueError(f"expected bfloat16 or float32, got {dtype}")
    if (K is None) != (K_out is None):
        raise ValueError("K and K_out go together")
    if len(shape) != 4 or (K is not None and (K.dim() != 4 or K.shape[0] != shape[0] or K.shape[2:] != shape[2:])):
        raise ValueError("Q and K must be [B, H, N, d] tensors that share B, N and d")
    for t, like in ((Q, Q), (Q_out, Q)) + (((K, K), (K_out, K)) if K is not None else ()):
        if not t.is_cuda or t.dtype is not dtype or t.shape != like.shape or not t.is_contiguous() or t.get_device() != device:
            raise ValueError("tensors must be contiguous, of one dtype and on one GPU, and outputs shaped like their inputs")
    if freqs.dtype is not torch.float64 or not freqs.is_cuda or freqs.get_device() != device or not freqs.is_contiguous() or freqs.dim() != 1:
        raise ValueError("freqs must be a contiguous float64 vector on the GPU of the other tensors")
    B, Hq, N, d = shape
    status = _lib().flat_attn_rope(Q.data_ptr(), Q_out.data_ptr(), Hq, None if K is None else K.data_ptr(), None if K is None else K_out.data_ptr(),
                                   0 if K is None else K.shape[1], B, N, d, 0 if dtype is torch.bfloat16 else 1, 2 * freqs.numel(), int(layout),
                                   freqs.data_ptr(), None if positions is None else _ints("positions", positions, device, (B, N)),
                                   float(magnitude), 1 if transpose else 0, _stream_on(Q, stream))
    if status != 0:
        _check(status)


def _bf16_on(name, t, device, shape):
    if t.dtype is not _b._torch.bfloat16 or not t.is_cuda or t.get_device() != device or not t.is_contiguous() or t.shape != shape:
        raise ValueError(f"{name} must be a contiguous bfloat16 tensor of shape {list(shape)} on the GPU of the cache")
    return t.data_ptr()


def _table(page_table, device):
    if page_table.dtype is not _b._torch.int32 or page_table.dim() != 2 or not page_table.is_contiguous() or not page_table.is_cuda or page_table.get_device() != device:
        raise ValueError("page_table must be a contiguous int32 tensor [sequences, pages] on the GPU of the other tensors")
    return page_table.data_ptr(), page_table.shape[0], page_table.shape[1]


def flat_attn_cache8_write(cache: FlatCache8, K, V, page_table, lens, n_new=None, stream=None) -> None:
    """Appends K, V bf16 [B,n_heads,N,d]: row n of entry b becomes token lens[b] + n, n < n_new[b] (None: N).  page_table int32 [B,max_pages],
    lens and n_new int32 [B].  lens is not changed."""
    _torch()
    if K.dim() != 4:
        raise ValueError("K and V must be [B, n_heads, N, d] tensors")
    device, B, N = cache._device, K.shape[0], K.shape[2]
    shape = (B, cache.n_heads, N, cache.d)
    table, rows, max_pages = _table(page_table, device)
    if rows != B:
        raise ValueError("page_table must have one row per batch entry")
    status = _lib().flat_attn_cache8_write(cache._ref, _bf16_on("K", K, device, shape), _bf16_on("V", V, device, shape), B, N, table, max_pages,
                                           _ints("lens", lens, device, (B,)), None if n_new is None else _ints("n_new", n_new, device, (B,)),
                                           _stream_on(K, stream))
    if status != 0:
        _check(status)


def flat_attn_fwd_cache8_workspace_bytes(B: int, H: int, n_heads: int, Nq: int, max_tokens: int, d: int) -> int:
    return int(_lib().flat_attn_fwd_cache8_workspace_bytes(int(B), int(H), int(n_heads), int(Nq), int(max_tokens), int(d)))


def flat_attn_fwd_cache8(cache: FlatCache8, Q, O, page_table, lens, scale: float, mask_kind: int = FLAT_MASK_NONE, q_lens=None, workspace=None,
                         stream=None) -> None:
    """Attention of Q bf16 [B,H,Nq,d] over the lens[b] tokens that entry b has in the cache, into O.  q_lens: int32 [B], queries that count (None: Nq).
    `workspace`: device tensor of at least flat_attn_fwd_cache8_workspace_bytes(B, H, n_heads, Nq, max_pages * page_tokens, d) bytes (None where that is 0)."""
    _torch()
    if Q.dim() != 4:
        raise ValueError("Q and O must be [B, H, Nq, d] tensors")
    device, shape = cache._device, Q.shape
    B, H, Nq, d = shape
    if d != cache.d:
        raise ValueError("Q must have the head size of the cache")
    table, rows, max_pages = _table(page_table, device)
    if rows != B:
        raise ValueError("page_table must have one row per batch entry")
    ws, nbytes = None, 0
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous() or workspace.get_device() != device:
            raise ValueError("workspace must be a contiguous tensor on the GPU of the cache")
        ws, nbytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    status = _lib().flat_attn_fwd_cache8(cache._ref, _bf16_on("Q", Q, device, shape), _bf16_on("O", O, device, shape), B, H, Nq, table, max_pages,
                                         _ints("lens", lens, device, (B,)), None if q_lens is None else _ints("q_lens", q_lens, device, (B,)),
                                         float(scale), int(mask_kind), ws, nbytes, _stream_on(Q, stream))
    if status != 0:
        _check(status)


def flat_attn_cache8_copy_pages(cache: FlatCache8, src, dst, stream=None) -> None:
    """Copies page src[i] to page dst[i]; int32 device tensors of one length."""
    _torch()
    n = src.numel()
    status = _lib().flat_attn_cache8_copy_pages(cache._ref, _ints("src", src, cache._device, (n,)), _ints("dst", dst, cache._device, (n,)), n,
                                                _stream_on(cache.k, stream))
    if status != 0:
        _check(status)


def flat_attn_cache8_fork(cache: FlatCache8, page_table, lens, parents, children, spares, stream=None) -> None:
    """Entry children[i] becomes a copy of entry parents[i], sharing its full pages; a begun last page is copied to page spares[i].  page_table
    int32 [n_seqs,max_pages] and lens int32 [n_seqs] are updated; the lists are int32 device tensors of one length."""
    _torch()
    device = cache._device
    table, n_seqs, max_pages = _table(page_table, device)
    n = parents.numel()
    status = _lib().flat_attn_cache8_fork(cache._ref, table, max_pages, n_seqs, _ints("lens", lens, device, (n_seqs,)), _ints("parents", parents, device, (n,)),
                                          _ints("children", children, device, (n,)), _ints("spares", spares, device, (n,)), n, _stream_on(cache.k, stream))
    if status != 0:
        _check(status)


def flat_attn_cache8_free(page_table, lens, seqs, unused, n_unused, stream=None) -> None:
    """Empties the rows `seqs` of page_table and their lens; then unused[: n_unused] are the pages (of unused.numel()) that no row holds."""
    _torch()
    device = page_table.get_device()
    table, n_seqs, max_pages = _table(page_table, device)
    n, n_pages = seqs.numel(), unused.numel()
    status = _lib().flat_attn_cache8_free(table, max_pages, n_seqs, _ints("lens", lens, device, (n_seqs,)), _ints("seqs", seqs, device, (n,)) if n else None, n, n_pages,
                                          _ints("unused", unused, device, (n_pages,)), _ints("n_unused", n_unused, device, (1,)), _stream_on(page_table, stream))
    if status != 0:
        _check(status)


def flat_attn_cache8_compact_workspace_bytes(n_pages: int) -> int:
    return int(_lib().flat_attn_cache8_compact_workspace_bytes(int(n_pages)))


def flat_attn_cache8_compact(cache: FlatCache8, page_table, new_table, n_used, workspace, stream=None) -> None:
    """Moves the held pages to ids 0 .. n_used - 1 and writes the page table that names them there to new_table (which may be page_table).
    `workspace`: device tensor of at least flat_attn_cache8_compact_workspace_bytes(n_pages) bytes."""
    _torch()
    device = cache._device
    table, n_seqs, max_pages = _table(page_table, device)
    if not workspace.is_cuda or not workspace.is_contiguous() or workspace.get_device() != device:
        raise ValueError("workspace must be a contiguous tensor on the GPU of the cache")
    status = _lib().flat_attn_cache8_compact(cache._ref, table, _ints("new_table", new_table, device, (n_seqs, max_pages)), max_pages, n_seqs,
                                             _ints("n_used", n_used, device, (1,)), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                             _stream_on(cache.k, stream))
    if status != 0:
        _check(status)
