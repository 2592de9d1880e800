"""Rotary positions and the paged 8-bit cache without a GPU: refusals of every entry point, frequencies, workspace sizes, and the numpy
implementation the GPU tests compare with against values worked out by hand."""
import ctypes
import math
import os
import shutil
import subprocess
import tempfile

import numpy as np
import pytest

import paper_2107_06419_amd as fa
from paper_2107_06419_amd.binding import FlatCache8Struct
import cache8_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = [0x10_0000_0000 * (i + 1) for i in range(12)]  # fake, aligned, far apart: never dereferenced on these paths


def cache(k=A[0], v=A[1], ks=A[2], vs=A[3], n_pages=8, n_heads=2, page_tokens=32, d=64, fmt=0):
    return FlatCache8Struct(k, v, ks, vs, n_pages, n_heads, page_tokens, d, fmt)


BAD_CACHES = [({"k": None}, -1), ({"vs": None}, -1), ({"n_pages": 0}, -2), ({"n_heads": -1}, -2), ({"page_tokens": 0}, -2), ({"page_tokens": 24}, -2),
              ({"page_tokens": 65552}, -2), ({"d": 48}, -3), ({"d": 512}, -3), ({"fmt": 2}, -3), ({"fmt": -1}, -3), ({"n_pages": 1 << 30}, -2),
              ({"k": A[0] + 8}, -4), ({"ks": A[2] + 2}, -4), ({"v": A[0] + 16}, -7), ({"vs": A[2]}, -7), ({"ks": A[1] + 64}, -7)]


def write(c=None, K=A[4], V=A[5], B=2, N=3, table=A[6], max_pages=4, lens=A[7], n_new=None, **kw):
    return fa.load_library().flat_attn_cache8_write(ctypes.byref(c if c is not None else cache(**kw)), K, V, B, N, table, max_pages, lens, n_new, None)


def attend(Q=A[4], O=A[5], B=2, H=4, Nq=1, table=A[6], max_pages=4, lens=A[7], q_lens=None, scale=1.0, mask=0, ws=A[8], ws_bytes=1 << 30, **kw):
    return fa.load_library().flat_attn_fwd_cache8(ctypes.byref(cache(**kw)), Q, O, B, H, Nq, table, max_pages, lens, q_lens, scale, mask, ws, ws_bytes, None)


def copy(src=A[4], dst=A[5], n=3, **kw):
    return fa.load_library().flat_attn_cache8_copy_pages(ctypes.byref(cache(**kw)), src, dst, n, None)


def fork(table=A[4], max_pages=4, n_seqs=3, lens=A[5], parents=A[6], children=A[7], spares=A[8], n=2, **kw):
    return fa.load_library().flat_attn_cache8_fork(ctypes.byref(cache(**kw)), table, max_pages, n_seqs, lens, parents, children, spares, n, None)


def free(table=A[0], max_pages=4, n_seqs=3, lens=A[1], seqs=A[2], n=2, n_pages=8, unused=A[3], n_unused=A[4]):
    return fa.load_library().flat_attn_cache8_free(table, max_pages, n_seqs, lens, seqs, n, n_pages, unused, n_unused, None)


def compact(table=A[4], new=A[5], max_pages=4, n_seqs=3, n_used=A[6], ws=A[7], ws_bytes=1 << 20, **kw):
    return fa.load_library().flat_attn_cache8_compact(ctypes.byref(cache(**kw)), table, new, max_pages, n_seqs, n_used, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [write, attend, copy, fork, compact])
@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_a_cache_that_is_none_is_refused_by_every_call(call, bad, status):
    assert call(**bad) == status


def test_write_refuses():
    assert fa.load_library().flat_attn_cache8_write(None, A[4], A[5], 1, 1, A[6], 1, A[7], None, None) == -1
    assert write(K=None) == -1 and write(V=None) == -1 and write(table=None) == -1 and write(lens=None) == -1
    assert write(B=0) == -2 and write(N=0) == -2 and write(max_pages=0) == -2 and write(max_pages=1 << 27) == -2
    assert write(B=1 << 20, N=1 << 20, max_pages=1) == -2
    assert write(K=A[4] + 8) == -4 and write(lens=A[7] + 2) == -4 and write(n_new=A[8] + 1) == -4
    assert write(K=A[0] + 16) == -7 and write(lens=A[3]) == -7 and write(table=A[1] + 64) == -7


def test_attend_refuses():
    assert attend(Q=None) == -1 and attend(O=None) == -1 and attend(table=None) == -1 and attend(lens=None) == -1
    assert attend(mask=2) == -3 and attend(scale=-1.0) == -3 and attend(scale=float("nan")) == -3 and attend(scale=float("inf")) == -3
    assert attend(B=0) == -2 and attend(H=3) == -2 and attend(H=0) == -2 and attend(Nq=0) == -2 and attend(max_pages=0) == -2
    assert attend(max_pages=1 << 26) == -2 and attend(Nq=1 << 25, max_pages=1) == -2 and attend(B=1 << 20, Nq=1 << 12, max_pages=1) == -2
    assert attend(Q=A[4] + 8) == -4 and attend(O=A[5] + 2) == -4 and attend(q_lens=A[9] + 2) == -4
    assert attend(O=A[4]) == -7 and attend(O=A[0] + 16) == -7 and attend(lens=A[5] + 16) == -7 and attend(q_lens=A[5] + 4) == -7
    need = fa.flat_attn_fwd_cache8_workspace_bytes(2, 4, 2, 1, 4096 * 32, 64)
    assert need > 0
    assert attend(max_pages=4096, ws=None) == -1 and attend(max_pages=4096, ws=A[8] + 4) == -4 and attend(max_pages=4096, ws_bytes=need - 1) == -5
    assert attend(max_pages=4096, ws=A[4], ws_bytes=need) == -7 and attend(max_pages=4096, ws=A[5], ws_bytes=need) == -7
    assert attend(max_pages=4096, ws=A[3], ws_bytes=need) == -7


def test_attend_workspace_sizes():
    size = fa.flat_attn_fwd_cache8_workspace_bytes
    assert size(0, 4, 2, 1, 100, 64) == 0 and size(1, 3, 2, 1, 100, 64) == 0 and size(1, 4, 2, 1, 100, 48) == 0 and size(1, 4, 2, 1, 0, 64) == 0
    assert size(1, 4, 2, 1, 64, 64) == 0                                      # a cache of a few tiles is not divided
    assert size(1, 1, 1, 1, 1 << 30, 128) == size(1, 1, 1, 1, 1 << 20, 128)   # the size does not grow with the cache
    for B, H, heads, Nq, d in ((1, 16, 16, 1, 64), (4, 64, 8, 1, 128), (3, 5, 1, 7, 256), (20, 8, 8, 4, 96)):
        assert 0 < size(B, H, heads, Nq, 1 << 17, d) < 1 << 28
    assert size(64, 64, 8, 1, 1 << 17, 128) == 0 and size(2, 16, 16, 4096, 1 << 14, 128) == 0   # entries that fill the chip are not divided either


def test_page_calls_refuse():
    assert copy(n=-1) == -2 and copy(src=None) == -1 and copy(dst=None) == -1 and copy(src=A[4] + 2) == -4 and copy(dst=A[0]) == -7
    assert copy(n=0, src=None, dst=None) == 0
    assert fork(table=None) == -1 and fork(lens=None) == -1 and fork(spares=None) == -1 and fork(n=-1) == -2 and fork(n_seqs=0) == -2
    assert fork(parents=A[6] + 1) == -4 and fork(lens=A[4] + 8) == -7 and fork(children=A[4]) == -7 and fork(spares=A[5]) == -7 and fork(table=A[2]) == -7
    assert fork(n=0, parents=None, children=None, spares=None) == 0
    assert free(table=None) == -1 and free(unused=None) == -1 and free(n_unused=None) == -1 and free(seqs=None) == -1
    assert free(n=-1) == -2 and free(n_pages=0) == -2 and free(n_pages=(1 << 20) + 1) == -2 and free(n_seqs=0) == -2
    assert free(lens=A[1] + 2) == -4 and free(unused=A[0]) == -7 and free(n_unused=A[3] + 4) == -7 and free(seqs=A[1]) == -7
    assert compact(new=None) == -1 and compact(n_used=None) == -1 and compact(ws=None) == -1 and compact(ws_bytes=8) == -5
    assert compact(n_pages=(1 << 20) + 1) == -2 and compact(n_seqs=0) == -2 and compact(ws=A[7] + 2) == -4
    assert compact(new=A[4] + 4) == -7 and compact(ws=A[5]) == -7 and compact(n_used=A[4]) == -7 and compact(new=A[0]) == -7 and compact(ws=A[2]) == -7
    assert fa.flat_attn_cache8_compact_workspace_bytes(0) == 0 and fa.flat_attn_cache8_compact_workspace_bytes((1 << 20) + 1) == 0
    assert fa.flat_attn_cache8_compact_workspace_bytes(8) == 100


def rope(Q=A[0], Qo=A[1], Hq=4, K=A[2], Ko=A[3], Hk=2, B=2, N=8, d=64, dtype=0, rot=64, layout=0, freqs=A[4], pos=A[5], mag=1.0, transpose=0):
    return fa.load_library().flat_attn_rope(Q, Qo, Hq, K, Ko, Hk, B, N, d, dtype, rot, layout, freqs, pos, mag, transpose, None)


def test_rope_refuses():
    assert rope(Q=None) == -1 and rope(Qo=None) == -1 and rope(freqs=None) == -1 and rope(K=None) == -1 and rope(Ko=None) == -1
    assert rope(Hq=0) == -2 and rope(Hk=0) == -2 and rope(B=0) == -2 and rope(N=0) == -2 and rope(B=1 << 20, N=1 << 12) == -2
    assert rope(d=48) == -3 and rope(rot=0) == -3 and rope(rot=3) == -3 and rope(rot=66) == -3 and rope(dtype=2) == -3 and rope(layout=2) == -3
    assert rope(mag=float("nan")) == -3 and rope(mag=float("inf")) == -3
    assert rope(Q=A[0] + 8) == -4 and rope(Ko=A[3] + 2) == -4 and rope(freqs=A[4] + 4) == -4 and rope(pos=A[5] + 2) == -4
    assert rope(Qo=A[0] + 16) == -7 and rope(Qo=A[2]) == -7 and rope(Ko=A[0]) == -7 and rope(Ko=A[1]) == -7 and rope(Qo=A[4]) == -7 and rope(Ko=A[5]) == -7


def test_frequencies():
    f = fa.flat_attn_rope_freqs(64).numpy()
    np.testing.assert_allclose(f, [10000.0 ** (-i / 32) for i in range(32)], rtol=1e-14)
    np.testing.assert_allclose(fa.flat_attn_rope_freqs(64, scaling=fa.FLAT_ROPE_SCALE_LINEAR, factor=4.0).numpy(), f / 4, rtol=1e-14)
    g = fa.flat_attn_rope_freqs(64, scaling=fa.FLAT_ROPE_SCALE_BASE, factor=4.0).numpy()
    assert g[0] == 1.0 and math.isclose(g[-1], f[-1] / 4, rel_tol=1e-12) and (np.diff(g) < 0).all()
    b = fa.flat_attn_rope_freqs(64, 500000.0, fa.FLAT_ROPE_SCALE_BANDS, 8.0, 8192.0, 1.0, 4.0).numpy()
    plain = fa.flat_attn_rope_freqs(64, 500000.0).numpy()
    for i in range(32):
        turns = 8192 * plain[i] / (2 * math.pi)
        keep = min(max((turns - 1) / 3, 0), 1)
        assert math.isclose(b[i], plain[i] * keep + plain[i] / 8 * (1 - keep), rel_tol=1e-13)
    assert fa.flat_attn_rope_freqs(2, scaling=fa.FLAT_ROPE_SCALE_BASE, factor=2.0).tolist() == [1.0]
    for bad in ({"rot_d": 0}, {"rot_d": 7}, {"rot_d": 258}, {"base": 1.0}, {"base": float("nan")}, {"scaling": 4}, {"scaling": 1, "factor": 0.5},
                {"scaling": 3, "factor": 2.0}, {"scaling": 3, "factor": 2.0, "original_len": 100.0, "low": 4.0, "high": 4.0}):
        with pytest.raises(fa.FlatAttnError) as e:
            fa.flat_attn_rope_freqs(**{"rot_d": 64, **bad})
        assert e.value.status == -3
    assert fa.load_library().flat_attn_rope_freqs(None, 64, 10000.0, 0, 1.0, 0.0, 1.0, 32.0) == -1


def test_binding_refuses_tensors_that_are_not_on_a_gpu():
    import torch
    k, s = torch.zeros(2, 1, 16, 32, dtype=torch.uint8), torch.zeros(2, 1, 1)
    with pytest.raises(ValueError):
        fa.FlatCache8(k, k, s, s)
    with pytest.raises(ValueError):
        fa.FlatCache8(k.int(), k, s, s)
    with pytest.raises(ValueError):
        fa.FlatCache8(k, k, s[:1], s)
    x, f = torch.zeros(1, 2, 3, 32, dtype=torch.bfloat16), torch.zeros(16, dtype=torch.float64)
    for args in ((x, x, None, None, f), (x, x, x, None, f), (x.half(), x.half(), None, None, f)):
        with pytest.raises(ValueError):
            fa.flat_attn_rope(*args)
    t = torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        fa.flat_attn_cache8_free(t, t[0].contiguous(), t[0].contiguous(), t[0].contiguous(), t[0, :1].contiguous())


def test_reference_codes_by_hand():
    v = ref.E4M3_VALUES
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[7] == 7 * 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0x38] == 1.0 and v[0x7e] == 448 and np.isnan(v[0x7f]) and v[0xb8] == -1
    x = np.array([448.0, -448.0, 17.0, 19.0, 17.1, 2.0 ** -10, 3 * 2.0 ** -10, -0.0])   # 17 lies between 16 and 18, 19 between 18 and 20
    assert ref.from_codes(ref.to_codes(x, ref.E4M3), ref.E4M3).tolist() == [448, -448, 16, 20, 18, 0, 2 * 2.0 ** -9, 0]
    assert ref.from_codes(ref.to_codes(np.array([0.5, 1.5, -2.5, 127.0, -127.0]), ref.INT8), ref.INT8).tolist() == [0, 2, -2, 127, -127]
    c = ref.Cache(1, 1, 16, 32, ref.INT8)
    c.write(np.full((1, 1, 1, 32), 3.0, np.float32), np.zeros((1, 1, 1, 32), np.float32), np.array([[0]]), [0])
    assert c.scale["k"][0, 0, 0] == 2.0 ** -5 and c.codes["k"][0, 0, 0, 0, 0] == 96 and c.scale["v"][0, 0, 0] == 0
    c.write(np.full((1, 1, 1, 32), -127.5, np.float32), np.ones((1, 1, 1, 32), np.float32), np.array([[0]]), [1])
    assert c.scale["k"][0, 0, 0] == 2.0 and c.codes["k"][0, 0, 0, :3, 0].view(np.int8).tolist() == [2, -64, 0]   # 1.5 and -63.75 to even
    o, _ = c.attend(np.zeros((1, 1, 1, 32), np.float32), np.array([[0]]), [2], 1.0, 0)
    assert o[0, 0, 0, 0] == 0.5


def test_validation_code_is_clean_under_asan_and_ubsan():
    """The argument checks and the planning of the cache's entry points as plain C++ against stub launchers, driven by sanitize/cache8_host_check.cpp."""
    if shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include/hip"):
        pytest.skip("g++ or the HIP headers not available")
    csrc = os.path.join(ROOT, "paper_2107_06419_amd", "csrc")
    with tempfile.TemporaryDirectory() as tmp:
        exe = os.path.join(tmp, "host_check")
        built = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__",
                                "-I/opt/rocm/include", "-o", exe, "-x", "c++", os.path.join(csrc, "flat_cache8_api.hip"), os.path.join(csrc, "flat_cache8_plan.hip"),
                                os.path.join(ROOT, "tests", "sanitize", "cache8_host_check.cpp")], capture_output=True, text=True)
        assert built.returncode == 0, built.stderr[-4000:]
        env = dict(os.environ, UBSAN_OPTIONS="print_stacktrace=1")
        env.pop("LD_PRELOAD", None)
        run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
        out = run.stdout + run.stderr
        assert run.returncode == 0 and "cache8 host checks passed" in out and "runtime error" not in out, out[-4000:]


def test_page_tables_whose_tokens_pass_31_bits_are_refused():
    """Token numbers are 31 bits wide, and wavefronts look at blocks up to some thousands of tokens behind an entry's last."""
    for tokens in (16, 48, 65536):
        most = (2 ** 31 - 65537) // tokens
        assert write(max_pages=most + 1, page_tokens=tokens, B=1) == -2 and attend(max_pages=most + 1, page_tokens=tokens, B=1) == -2
        assert fork(max_pages=most + 1, page_tokens=tokens, n_seqs=1) == -2 and compact(max_pages=most + 1, page_tokens=tokens, n_seqs=1) == -2
        assert attend(max_pages=most, page_tokens=tokens, B=1, lens=A[7] + 2) == -4 and write(max_pages=most, page_tokens=tokens, B=1, lens=A[7] + 2) == -4
    size = fa.flat_attn_fwd_cache8_workspace_bytes
    assert size(1, 1, 1, 1, 2 ** 31 - 65537, 128) == size(1, 1, 1, 1, 1 << 20, 128) > 0 and size(1, 1, 1, 1, 2 ** 31 - 65536, 128) == 0
