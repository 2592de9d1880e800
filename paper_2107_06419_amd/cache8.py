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


# torch's types and the library, looked up once.  A call costs the host as much as a small one costs the GPU, so every tensor gets one test, and which part of it
# failed is looked up afterwards.
_i32 = _bf16 = _f32 = _f64 = _library = None


def _load():
    global _i32, _bf16, _f32, _f64, _library
    torch = _b._torch or _load_torch()
    _i32, _bf16, _f32, _f64 = torch.int32, torch.bfloat16, torch.float32, torch.float64
    _library = load_library()
    return _library


def _stream(device, stream) -> int:
    """The handle of the stream to enqueue on.  Without one it is the current stream of the current device, which has to be the tensors' own."""
    if stream is None:
        if _b._device() != device:
            raise ValueError(f"the tensors live on GPU {device}, which is not the current device")
        return _b._raw_stream(device)
    if stream.device_index != device:
        raise ValueError("the stream belongs to another device than the tensors")
    return int(stream.cuda_stream)


def _refuse(name, t, dtype, device, shape):
    if device < 0 or t.get_device() != device:
        raise ValueError(f"{name} must live on a GPU, the one of the other tensors")
    raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {list(shape)}, got {t.dtype} {list(t.shape)}")


def _ints(name, t, device, shape):
    if t.dtype is not _i32 or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        _refuse(name, t, _i32, device, shape)
    return t.data_ptr()


def _table(page_table, device):
    shape = page_table.shape
    if page_table.dtype is not _i32 or device < 0 or page_table.get_device() != device or len(shape) != 2 or not page_table.is_contiguous():
        raise ValueError("page_table must be a contiguous int32 tensor [sequences, pages] on the GPU of the other tensors")
    return shape


def _buffer(name, t, device):
    if t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor on the GPU of the cache")
    return t.data_ptr(), t.numel() * t.element_size()


class FlatCache8:
    """A paged cache of keys and values in 8 bits: `k`, `v` uint8 [n_pages, n_heads, page_tokens, d] (the bytes of a page lie in the order of
    flat_cache8 in the header), `k_scale`, `v_scale` float32 [n_pages, n_heads, page_tokens / 16], GPU tensors, kept alive by this object."""

    def __init__(self, k, v, k_scale, v_scale, format: int = FLAT_CACHE8_E4M3):
        _load()
        torch = _b._torch
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
    lib = _library or _load()
    if not 2 <= int(rot_d) <= 256:
        _check(-3)
    out = _b._torch.empty(int(rot_d) // 2, dtype=_f64)
    _check(lib.flat_attn_rope_freqs(out.data_ptr(), int(rot_d), float(base), int(scaling), float(factor), float(original_len), float(low), float(high)))
    return out


def flat_attn_rope(Q, Q_out, K, K_out, freqs, positions=None, layout: int = FLAT_ROPE_HALF, magnitude: float = 1.0, transpose: bool = False,
                   stream=None) -> None:
    """Rotary positions of Q [B,Hq,N,d] and, unless None, K [B,Hk,N,d], bf16 or float32 device tensors, into Q_out and K_out (which may be Q and K).
    `freqs`: float64 device tensor of rot_d / 2 radians per position; `positions`: int32 device tensor [B,N], or None for 0 .. N - 1.
    transpose: turn the other way, which is the gradient."""
    lib = _library or _load()
    dtype, shape, device = Q.dtype, Q.shape, Q.get_device()
    if dtype is not _bf16 and dtype is not _f32:
        raise ValueError(f"expected bfloat16 or float32, got {dtype}")
    if len(shape) != 4 or device < 0 or not Q.is_contiguous():
        raise ValueError("Q must be a contiguous [B, H, N, d] tensor on a GPU")
    B, Hq, N, d = shape
    if Q_out is not Q and (Q_out.dtype is not dtype or Q_out.get_device() != device or Q_out.shape != shape or not Q_out.is_contiguous()):
        _refuse("Q_out", Q_out, dtype, device, shape)
    if K is not None and K_out is not None:
        shape = K.shape
        Hk = shape[1] if len(shape) == 4 else 0
        if K.dtype is not dtype or K.get_device() != device or shape != (B, Hk, N, d) or not K.is_contiguous():
            _refuse("K", K, dtype, device, (B, Hk, N, d))
        if K_out is not K and (K_out.dtype is not dtype or K_out.get_device() != device or K_out.shape != shape or not K_out.is_contiguous()):
            _refuse("K_out", K_out, dtype, device, shape)
        k, k_out = K.data_ptr(), K_out.data_ptr()
    elif K is not K_out:
        raise ValueError("K and K_out go together")
    else:
        Hk, k, k_out = 0, None, None
    if freqs.dtype is not _f64 or freqs.get_device() != device or freqs.dim() != 1 or not freqs.is_contiguous():
        _refuse("freqs", freqs, _f64, device, ["rot_d / 2"])
    status = lib.flat_attn_rope(Q.data_ptr(), Q_out.data_ptr(), Hq, k, k_out, Hk, B, N, d, 0 if dtype is _bf16 else 1, 2 * freqs.numel(), int(layout),
                                freqs.data_ptr(), None if positions is None else _ints("positions", positions, device, (B, N)),
                                float(magnitude), 1 if transpose else 0, _stream(device, stream))
    if status != 0:
        _check(status)


def flat_attn_cache8_write(cache: FlatCache8, K, V, page_table, lens, n_new=None, stream=None) -> None:
    """Appends K, V bf16 [B,n_heads,N,d]: row n of entry b becomes token lens[b] + n, n < n_new[b] (None: N).  page_table int32 [B,max_pages],
    lens and n_new int32 [B].  lens is not changed."""
    lib = _library or _load()
    device, shape = cache._device, K.shape
    B, max_pages = _table(page_table, device)
    if len(shape) != 4 or shape[0] != B or shape[1] != cache.n_heads or shape[3] != cache.d or K.dtype is not _bf16 or K.get_device() != device or not K.is_contiguous():
        _refuse("K", K, _bf16, device, (B, cache.n_heads, "N", cache.d))
    if V.dtype is not _bf16 or V.get_device() != device or V.shape != shape or not V.is_contiguous():
        _refuse("V", V, _bf16, device, shape)
    status = lib.flat_attn_cache8_write(cache._ref, K.data_ptr(), V.data_ptr(), B, shape[2], page_table.data_ptr(), max_pages, _ints("lens", lens, device, (B,)),
                                        None if n_new is None else _ints("n_new", n_new, device, (B,)), _stream(device, stream))
    if status != 0:
        _check(status)


def flat_attn_fwd_cache8_workspace_bytes(B: int, H: int, n_heads: int, Nq: int, max_tokens: int, d: int) -> int:
    return int((_library or _load()).flat_attn_fwd_cache8_workspace_bytes(int(B), int(H), int(n_heads), int(Nq), int(max_tokens), int(d)))


def flat_attn_fwd_cache8(cache: FlatCache8, Q, O, page_table, lens, scale: float, mask_kind: int = FLAT_MASK_NONE, q_lens=None, workspace=None,
                         stream=None) -> None:
    """Attention of Q bf16 [B,H,Nq,d] over the lens[b] tokens that entry b has in the cache, into O.  q_lens: int32 [B], queries that count (None: Nq).
    `workspace`: device tensor of at least flat_attn_fwd_cache8_workspace_bytes(B, H, n_heads, Nq, max_pages * page_tokens, d) bytes (None where that is 0)."""
    lib = _library or _load()
    device, shape = cache._device, Q.shape
    B, max_pages = _table(page_table, device)
    if len(shape) != 4 or shape[0] != B or shape[3] != cache.d or Q.dtype is not _bf16 or Q.get_device() != device or not Q.is_contiguous():
        _refuse("Q", Q, _bf16, device, (B, "H", "Nq", cache.d))
    if O.dtype is not _bf16 or O.get_device() != device or O.shape != shape or not O.is_contiguous():
        _refuse("O", O, _bf16, device, shape)
    ws, nbytes = (None, 0) if workspace is None else _buffer("workspace", workspace, device)
    status = lib.flat_attn_fwd_cache8(cache._ref, Q.data_ptr(), O.data_ptr(), B, shape[1], shape[2], page_table.data_ptr(), max_pages, _ints("lens", lens, device, (B,)),
                                      None if q_lens is None else _ints("q_lens", q_lens, device, (B,)), float(scale), int(mask_kind), ws, nbytes, _stream(device, stream))
    if status != 0:
        _check(status)


def flat_attn_cache8_copy_pages(cache: FlatCache8, src, dst, stream=None) -> None:
    """Copies page src[i] to page dst[i]; int32 device tensors of one length."""
    lib = _library or _load()
    device, n = cache._device, src.numel()
    status = lib.flat_attn_cache8_copy_pages(cache._ref, _ints("src", src, device, (n,)), _ints("dst", dst, device, (n,)), n, _stream(device, stream))
    if status != 0:
        _check(status)


def flat_attn_cache8_fork(cache: FlatCache8, page_table, lens, parents, children, spares, stream=None) -> None:
    """Entry children[i] becomes a copy of entry parents[i], sharing its full pages; a begun last page is copied to page spares[i].  page_table
    int32 [n_seqs,max_pages] and lens int32 [n_seqs] are updated; the lists are int32 device tensors of one length."""
    lib = _library or _load()
    device, n = cache._device, parents.numel()
    n_seqs, max_pages = _table(page_table, device)
    status = lib.flat_attn_cache8_fork(cache._ref, page_table.data_ptr(), max_pages, n_seqs, _ints("lens", lens, device, (n_seqs,)), _ints("parents", parents, device, (n,)),
                                       _ints("children", children, device, (n,)), _ints("spares", spares, device, (n,)), n, _stream(device, stream))
    if status != 0:
        _check(status)


def flat_attn_cache8_free(page_table, lens, seqs, unused, n_unused, stream=None) -> None:
    """Empties the rows `seqs` of page_table and their lens; then unused[: n_unused] are the pages (of unused.numel()) that no row holds."""
    lib = _library or _load()
    device = page_table.get_device()
    n_seqs, max_pages = _table(page_table, device)
    n, n_pages = seqs.numel(), unused.numel()
    status = lib.flat_attn_cache8_free(page_table.data_ptr(), max_pages, n_seqs, _ints("lens", lens, device, (n_seqs,)), _ints("seqs", seqs, device, (n,)), n, n_pages,
                                       _ints("unused", unused, device, (n_pages,)), _ints("n_unused", n_unused, device, (1,)), _stream(device, stream))
    if status != 0:
        _check(status)


def flat_attn_cache8_compact_workspace_bytes(n_pages: int) -> int:
    return int((_library or _load()).flat_attn_cache8_compact_workspace_bytes(int(n_pages)))


def flat_attn_cache8_compact(cache: FlatCache8, page_table, new_table, n_used, workspace, stream=None) -> None:
    """Moves the held pages to ids 0 .. n_used - 1 and writes the page table that names them there to new_table (which may be page_table).
    `workspace`: device tensor of at least flat_attn_cache8_compact_workspace_bytes(n_pages) bytes."""
    lib = _library or _load()
    device = cache._device
    shape = _table(page_table, device)
    ws, nbytes = _buffer("workspace", workspace, device)
    status = lib.flat_attn_cache8_compact(cache._ref, page_table.data_ptr(), _ints("new_table", new_table, device, shape), shape[1], shape[0],
                                          _ints("n_used", n_used, device, (1,)), ws, nbytes, _stream(device, stream))
    if status != 0:
        _check(status)
