"""Rotary positions on the GPU against 64-bit numpy.  A result is off by half a step of its type, by the fp32 products and sum (each 2^-24 of
|x_a| + |x_b|), and by the sine and cosine: 2^-23 for theirs, 2 pi 2^-26 for the fraction of a turn held in fp32."""
import math

import numpy as np
import pytest

import paper_2107_06419_amd as fa
import cache8_reference as ref

pytestmark = pytest.mark.gpu


def run(q, k, freqs, positions, dtype, **kw):
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    dq, dk = (None if x is None else torch.from_numpy(x).to(t).cuda() for x in (q, k))
    oq, ok = (None if x is None else torch.full_like(x, float("nan")) for x in (dq, dk))
    pos = None if positions is None else torch.from_numpy(positions.astype(np.int32)).cuda()
    fa.flat_attn_rope(dq, oq, dk, ok, torch.from_numpy(freqs).cuda(), pos, **kw)
    torch.cuda.synchronize()
    return dq, dk, oq, ok


def close(got, x, want, mag, dtype, rot, interleaved):
    g, x = got.float().cpu().numpy().astype(np.float64), x.float().cpu().numpy().astype(np.float64)
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    size = np.zeros(x.shape)
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    off = size * mag * (4 * 2.0 ** -24 + 2.0 ** -23 + 2 * math.pi * 2.0 ** -26) + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * 1.001
    assert (np.abs(g - want) <= off + 1e-37).all(), float((np.abs(g - want) - off).max())
    assert np.array_equal(g[..., rot:], x[..., rot:])


@pytest.mark.parametrize("d,rot", [(32, 32), (64, 64), (64, 16), (96, 96), (96, 50), (128, 128), (128, 6), (128, 126), (256, 256), (256, 2), (256, 64)])
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope_matches_the_definition(d, rot, interleaved, dtype):
    rng = np.random.default_rng(d * 1000 + rot + interleaved)
    for B, Hq, Hk, N, far in ((1, 1, 1, 1, 0), (2, 5, 3, 33, 1000), (3, 4, 0, 7, 2 ** 31 - 1)):
        q, k = ref.bf16(rng.standard_normal((B, Hq, N, d))), ref.bf16(rng.standard_normal((B, max(Hk, 1), N, d)))
        positions = rng.integers(-far, far + 1, (B, N)) if far else None
        freqs = fa.flat_attn_rope_freqs(rot).numpy()
        transpose, mag = bool(N & 2), 1.0 if N == 1 else 1.25
        print(f"case rope d={d} rot={rot} {dtype} interleaved={interleaved} B={B} N={N}", flush=True)
        dq, dk, oq, ok = run(q, k if Hk else None, freqs, positions, dtype, layout=interleaved, magnitude=mag, transpose=transpose)
        pos = np.broadcast_to(np.arange(N), (B, N)) if positions is None else positions
        for x, y in ((dq, oq), (dk, ok)):
            if x is None:
                continue
            close(y, x, ref.rope(x.float().cpu().numpy(), freqs, pos, rot, interleaved, mag, transpose), mag, dtype, rot, interleaved)


@pytest.mark.parametrize("interleaved", [0, 1])
def test_rope_over_many_rows_in_place_and_with_heads_in_groups(interleaved):
    """Long enough that a thread has several heads, with a number of heads that is no multiple of what it takes at once; in place."""
    import torch
    B, Hq, Hk, N, d, rot = 2, 13, 3, 2500, 128, 96
    rng = np.random.default_rng(3)
    q, k = (ref.bf16(rng.standard_normal((B, h, N, d))) for h in (Hq, Hk))
    freqs = fa.flat_attn_rope_freqs(rot, 500000.0, fa.FLAT_ROPE_SCALE_BANDS, 8.0, 4096.0).numpy()
    dq, dk, oq, ok = run(q, k, freqs, None, "bf16", layout=interleaved)
    close(oq, dq, ref.rope(q, freqs, np.broadcast_to(np.arange(N), (B, N)), rot, interleaved, 1.0, False), 1.0, "bf16", rot, interleaved)
    fa.flat_attn_rope(dq, dq, dk, dk, torch.from_numpy(freqs).cuda(), None, layout=interleaved)
    torch.cuda.synchronize()
    assert torch.equal(dq.view(torch.int16), oq.view(torch.int16)) and torch.equal(dk.view(torch.int16), ok.view(torch.int16))


@pytest.mark.parametrize("interleaved", [0, 1])
def test_transposed_rotation_is_the_gradient(interleaved):
    """<g, R x> changes by <R^T g, dx> when x changes by dx: compared with differences, which are exact but for rounding as R is linear."""
    import torch
    rng = np.random.default_rng(9)
    B, H, N, d, rot, mag = 1, 2, 40, 64, 48, 1.5
    freqs, pos = fa.flat_attn_rope_freqs(rot).numpy(), rng.integers(0, 5000, (B, N))
    x, g, dx = (rng.standard_normal((B, H, N, d)).astype(np.float32) for _ in range(3))
    f = lambda y: run(y, None, freqs, pos, "f32", layout=interleaved, magnitude=mag)[2].double().cpu().numpy()
    back = run(g, None, freqs, pos, "f32", layout=interleaved, magnitude=mag, transpose=True)[2].double().cpu().numpy()
    moved = (x + dx).astype(np.float32)
    step = moved.astype(np.float64) - x
    difference, predicted = float((g * (f(moved) - f(x))).sum()), float((back * step).sum())
    n = B * H * N * d
    # each of the 3 n rotated values is off by at most 8 * 2^-24 of |a| + |b| < 2 * 6 * mag, times |g|, |step| < 6
    assert abs(difference - predicted) <= 3 * math.sqrt(n) * 8 * 2.0 ** -24 * 12 * mag * 6
    close(torch.from_numpy(back), torch.from_numpy(g), ref.rope(g, freqs, pos, rot, interleaved, mag, True), mag, "f32", rot, interleaved)


def test_rope_refuses_what_does_not_belong_together():
    import torch
    q = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16, device="cuda")
    f = torch.zeros(32, dtype=torch.float64, device="cuda")
    bad_pos, half = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.empty_like(q)
    for args, kw in (((q, half, None, None, f.float()), {}), ((q, half, None, None, f), {"positions": bad_pos}), ((q, half[:, :1], None, None, f), {}),
                     ((q, half.transpose(1, 2), None, None, f), {}), ((q, half, q[:, :, :2].contiguous(), half, f), {}), ((q, half, q, half.float(), f), {})):
        with pytest.raises(ValueError):
            fa.flat_attn_rope(*args, **kw)
    for kw, status in (({"layout": 2}, -3), ({"magnitude": float("nan")}, -3)):
        with pytest.raises(fa.FlatAttnError) as e:
            fa.flat_attn_rope(q, half, None, None, f, **kw)
        assert e.value.status == status
    with pytest.raises(fa.FlatAttnError) as e:
        fa.flat_attn_rope(q, q, q, half, f)      # q would be read as K while it is written as Q_out
    assert e.value.status == -7
