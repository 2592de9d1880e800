"""The paged 8-bit cache on the GPU against numpy in 64 bits: writes bit for bit, attention within a bound derived row by row
(cache8_reference.Cache.attend), pages bit for bit, and a run of all of it together."""
import numpy as np
import pytest

import paper_2107_06419_amd as fa
import cache8_reference as ref

pytestmark = pytest.mark.gpu

E4M3, INT8 = fa.FLAT_CACHE8_E4M3, fa.FLAT_CACHE8_INT8


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def i32(x):
    return dev(np.asarray(x, np.int32))


def b16(x):
    import torch
    return dev(x, torch.bfloat16)


def attend(c, q, table, lens, scale, mask, q_lens=None, out=None, poison=True, stream=None):
    import torch
    B, H, Nq, d = q.shape
    dq = b16(q)
    o = torch.full_like(dq, float("nan")) if out is None else out
    nbytes = fa.flat_attn_fwd_cache8_workspace_bytes(B, H, c.n_heads, Nq, table.shape[1] * c.page_tokens, d)
    ws = torch.full((nbytes // 4,), float("nan") if poison else 0.0, dtype=torch.float32, device="cuda") if nbytes else None
    fa.flat_attn_fwd_cache8(c, dq, o, i32(table), i32(lens), scale, mask, None if q_lens is None else i32(q_lens), ws, stream=stream)
    torch.cuda.synchronize()
    return o


def check(o, want, bound):
    got = o.float().cpu().numpy().astype(np.float64)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], bound[bad][:4])


def filled(rng, lens, heads, d, T, fmt, spare=3, extra=1):
    """A cache of anything, whose pages up to the lengths were written with normal values, with its page table."""
    n_pages = sum(-(-max(int(n), 0) // T) for n in lens) + spare
    c = ref.Cache(n_pages, heads, T, d, fmt, rng)
    table = ref.page_table(rng, lens, T, n_pages, max(-(-max(int(n), 1) // T) for n in lens) + extra)
    B, N = len(lens), max(int(n) for n in lens)
    for b in range(B):   # values straight into the codes: how they got there is another test's matter
        for blk in range(-(-int(lens[b]) // 16)):
            page, at, n = table[b, blk * 16 // T], blk % (T // 16), min(16, int(lens[b]) - 16 * blk)
            for name in "kv":
                x = rng.standard_normal((heads, n, d)) * 2.0 ** rng.integers(-2, 2)
                c.codes[name][page, :, at, :n] = ref.to_codes(np.clip(x * (ref.LARGEST[fmt] / 8), -ref.LARGEST[fmt], ref.LARGEST[fmt]), fmt)
                c.scale[name][page, :, at] = np.exp2(rng.integers(-8, -4, heads))
    return c, table


# ---- write -------------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 256])
def test_writes_leave_the_bits_that_the_definition_says(d, fmt):
    """Token by token, in chunks that begin and end inside blocks and pages, with values that raise a begun block's scale, zeros and tiny
    values; entries that write nothing, holes, and tokens behind the last page."""
    import torch
    rng = np.random.default_rng(d + fmt)
    for T, heads, N, starts, news in ((16, 3, 1, [0, 15, 16, 5, 32], None), (32, 2, 37, [0, 1, 31, 64, 11], [37, 0, 5, 1, 37]), (48, 1, 16, [16, 7, 47, 96, 3], None),
                                      (64, 2, 130, [0, 63, 0, 126, 200], [130, 130, 2, 130, -4]), (16, 1, 3, [-5, 1000, 62, 63, 64], [3, 3, 3, 3, 9])):
        B = len(starts)
        width = 4 if T == 16 and N == 3 else -(-max(s + N for s in starts) // T)
        n_pages = B * width + 2
        c = ref.Cache(n_pages, heads, T, d, fmt, rng)
        c.codes = {n: np.where((x & 127) == 127, 5, x) if fmt == E4M3 else np.where(x == 128, 1, x).astype(np.uint8) for n, x in c.codes.items()}
        c.codes = {n: x.astype(np.uint8) for n, x in c.codes.items()}
        table = rng.permutation(n_pages)[:B * width].reshape(B, width).astype(np.int32)
        table[2, -1] = n_pages if N == 3 else table[2, -1]
        table[4, 0] = -1 if N == 37 else table[4, 0]
        k, v = (ref.bf16(rng.standard_normal((B, heads, N, d)) * 2.0 ** rng.integers(-10, 11, (B, heads, N, 1))) for _ in range(2))
        k[0, 0], v[1, :, :, ::3] = 0.0, 0.0
        k[2] = ref.bf16(k[2] * 2.0 ** -120)
        v[3] = ref.bf16(np.clip(v[3].astype(np.float64) * 2.0 ** 118, -3e38, 3e38))
        print(f"case write d={d} fmt={fmt} T={T} N={N}", flush=True)
        dc = c.device()
        fa.flat_attn_cache8_write(dc, b16(k), b16(v), i32(table), i32(starts), None if news is None else i32(news))
        torch.cuda.synchronize()
        c.write(k, v, table, starts, news)
        c.like(dc).assert_same(c)


@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_a_sequence_written_token_by_token(fmt):
    import torch
    rng = np.random.default_rng(fmt)
    heads, d, T, n = 2, 64, 32, 50
    c = ref.Cache(3, heads, T, d, fmt, rng)
    dc, table, dt = c.device(), np.array([[2, 0]], np.int32), i32([[2, 0]])
    for t in range(n):
        k, v = (ref.bf16(rng.standard_normal((1, heads, 1, d)) * 2.0 ** (t % 16 - 8)) for _ in range(2))
        fa.flat_attn_cache8_write(dc, b16(k), b16(v), dt, i32([t]))
        c.write(k, v, table, [t])
    torch.cuda.synchronize()
    c.like(dc).assert_same(c)


def test_every_bf16_magnitude_is_rounded_to_the_nearest_code():
    """All finite bf16 values, sixteen neighbours in value to a token, so that every one is the largest of a block once and small beside others."""
    import torch
    bits = np.arange(0x7f80, dtype=np.uint32)
    x = np.concatenate([bits, bits | 0x8000]).astype(np.uint32) << 16
    x = x.view(np.float32)
    x = np.concatenate([x, np.random.default_rng(1).permutation(x)])
    for fmt in (E4M3, INT8):
        n = x.size // 32
        k = x[:n * 32].reshape(1, 1, n, 32)
        c = ref.Cache(-(-n // 64), 1, 64, 32, fmt)
        table = np.arange(c.n_pages, dtype=np.int32)[None]
        dc = c.device()
        fa.flat_attn_cache8_write(dc, b16(k), b16(k), i32(table), i32([0]))
        torch.cuda.synchronize()
        c.write(k, k, table, [0])
        c.like(dc).assert_same(c)


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_values_that_are_no_numbers_show_in_what_sees_them_and_nowhere_else(fmt, bad):
    import torch
    rng = np.random.default_rng(4)
    heads, d, T, n = 2, 64, 16, 40
    c = ref.Cache(4, heads, T, d, fmt, rng)
    k, v = (ref.bf16(rng.standard_normal((1, heads, n, d))) for _ in range(2))
    k[0, 0, 37, 3], v[0, 1, 20, 5] = bad, bad
    table, dc = np.array([[3, 1, 0]], np.int32), c.device()
    fa.flat_attn_cache8_write(dc, b16(k), b16(v), i32(table), i32([0]))
    torch.cuda.synchronize()
    c.write(k, v, table, [0])
    c.like(dc).assert_same(c)
    assert np.isnan(c.scale["k"][0, 0, 0]) and np.isnan(c.scale["v"][1, 1, 0]) and np.isnan(c.scale["k"]).sum() == 1
    # a later token keeps a block that is no number as it is
    more = ref.bf16(rng.standard_normal((1, heads, 2, d)))
    fa.flat_attn_cache8_write(dc, b16(more), b16(more), i32(table), i32([40]))
    torch.cuda.synchronize()
    c.write(more, more, table, [40])
    c.like(dc).assert_same(c)
    q = ref.bf16(rng.standard_normal((1, heads, n, d)))
    o = attend(dc, q, table, [n], 0.125, 1).float().cpu().numpy()
    # K's block 2 (tokens 32 ..) of head 0 and V's block 1 (tokens 16 ..) of head 1
    assert np.isnan(o[0, 0, 32:]).all() and np.isfinite(o[0, 0, :32]).all() and np.isnan(o[0, 1, 16:]).all() and np.isfinite(o[0, 1, :16]).all()


# ---- attention -----------------------------------------------------------------------------------------------------------------------------

ATTEND = [  # B lens, H, heads, Nq, T, q_lens
    ([1], 1, 1, 1, 16, None),
    ([0, 5, 33], 4, 2, 1, 16, None),
    ([31, 32, 17, 64], 6, 2, 1, 32, None),
    ([700], 16, 16, 1, 16, None),
    ([1000, 3, 513], 10, 2, 1, 48, None),
    ([300, 40, 7], 8, 1, 5, 64, [5, 5, 3]),
    ([257, 5, 0], 2, 2, 9, 32, [9, 9, 9]),          # queries that see no key: longer than the cache
    ([130, 129], 7, 1, 33, 16, [33, 0]),
    ([260], 4, 4, 200, 64, None),
    ([500, 77], 12, 3, 70, 128, [70, 64]),
]


@pytest.mark.parametrize("lens,H,heads,Nq,T,q_lens", ATTEND)
@pytest.mark.parametrize("d", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("mask", [0, 1])
def test_attention_matches_the_definition(lens, H, heads, Nq, T, q_lens, d, fmt, mask):
    rng = np.random.default_rng(sum(lens) + d + fmt)
    c, table = filled(rng, lens, heads, d, T, fmt)
    q = ref.bf16(rng.standard_normal((len(lens), H, Nq, d)))
    scale = float(np.float32(d ** -0.5))
    print(f"case attend lens={lens} H={H}/{heads} Nq={Nq} T={T} d={d} fmt={fmt} mask={mask}", flush=True)
    want, bound = c.attend(q, table, lens, scale, mask, q_lens, untouched=np.full(q.shape, 7.0))
    o = attend(c.device(), q, table, lens, scale, mask, q_lens, out=b16(np.full(q.shape, 7.0, np.float32)))
    check(o, want, bound)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("lens,H,heads,Nq,T", [([20000], 4, 2, 1, 64), ([9000, 1, 0, 3000, 700], 8, 2, 1, 16), ([5000, 4100], 6, 1, 40, 256), ([12000], 1, 1, 3, 16),
                                               ([2500, 90, 2000], 2, 2, 300, 64), ([9000, 4000, 100, 0, 7000, 2500], 32, 16, 1, 32), ([6000, 5000, 17], 64, 16, 7, 64)])
def test_attention_over_keys_divided_over_workgroups(lens, H, heads, Nq, T, d, fmt):
    """Long entries next to short ones and empty ones: parts of several workgroups are put together, and the same call gives the same bits
    whatever the workspace held."""
    import torch
    rng = np.random.default_rng(len(lens) * 7 + Nq + d)
    c, table = filled(rng, lens, heads, d, T, fmt)
    q = ref.bf16(rng.standard_normal((len(lens), H, Nq, d)) * 2)
    scale = float(np.float32(d ** -0.5))
    dc = c.device()
    for mask in (0, 1):
        print(f"case attend long lens={lens} H={H}/{heads} Nq={Nq} T={T} d={d} fmt={fmt} mask={mask}", flush=True)
        want, bound = c.attend(q, table, lens, scale, mask)
        o = attend(dc, q, table, lens, scale, mask)
        check(o, want, bound)
        assert torch.equal(o.view(torch.int16), attend(dc, q, table, lens, scale, mask, poison=False).view(torch.int16))


MANY_ROWS = [  # B, H, heads, Nq, longest, T: at least 512 blocks of 128 rows, which a kernel of their own takes
    (2, 256, 256, 33, 130, 16),
    (4, 128, 128, 40, 70, 32),          # longer than some entries: queries that see no key
    (3, 192, 64, 90, 260, 64),          # three query heads to a head of the cache: 270 rows in three blocks
    (2, 320, 64, 110, 1300, 48),        # more tiles than the blocks of one look-ahead
    (1, 128, 32, 510, 2300, 256),
]


@pytest.mark.parametrize("B,H,heads,Nq,longest,T", MANY_ROWS)
@pytest.mark.parametrize("d,fmt,mask", [(32, E4M3, 1), (64, E4M3, 0), (64, INT8, 1), (96, INT8, 1), (128, E4M3, 1), (128, INT8, 0), (256, E4M3, 1)])
def test_attention_of_many_rows(B, H, heads, Nq, longest, T, d, fmt, mask):
    """Ragged lengths and query counts, holes, keys whose logits grow along the sequence so that the reference maximum rises in later tiles, and a
    block that is no number near the end of the last entry."""
    rng = np.random.default_rng(Nq + d)
    lens = [longest] + [int(rng.integers(0, longest)) for _ in range(B - 1)]
    q_lens = [Nq] + [int(rng.integers(0, Nq + 1)) for _ in range(B - 1)]
    c, table = filled(rng, lens, heads, d, T, fmt)
    for blk in range(-(-longest // 16)):
        c.scale["k"][table[0, blk * 16 // T], :, blk % (T // 16)] *= np.float32(2.0 ** min(blk / 16, 4))
    if longest > 1000:
        table[0, 3], table[0, 9] = -1, c.n_pages + 2
    q = ref.bf16(rng.standard_normal((B, H, Nq, d)))
    scale = float(np.float32(d ** -0.5))
    print(f"case attend many rows B={B} H={H}/{heads} Nq={Nq} lens={lens} q_lens={q_lens} T={T} d={d} fmt={fmt} mask={mask}", flush=True)
    want, bound = c.attend(q, table, lens, scale, mask, q_lens, untouched=np.full(q.shape, 7.0))
    dc = c.device()
    out = b16(np.full(q.shape, 7.0, np.float32))
    check(attend(dc, q, table, lens, scale, mask, q_lens, out=out), want, bound)
    if mask and longest > 200:
        at = (longest - 17) // 16                       # a whole block that the last positions see, and the first do not
        dc.v_scale[int(table[0, at * 16 // T]), heads - 1, at % (T // 16)] = float("nan")
        o = attend(dc, q, table, lens, scale, mask, q_lens).float().cpu().numpy()
        first = 16 * at - (longest - Nq)                # the first query that sees a token of it
        hit = o[0, -(H // heads):]
        assert np.isnan(hit[:, max(first, 0):]).all() and np.isfinite(hit[:, :max(first, 0)]).all() and np.isfinite(o[0, : H - H // heads]).all()


SHARED_TILES = [  # B, H, heads, Nq, longest, T: at least 256 blocks of 256 rows (d = 256: 128), most of whose wavefronts have rows
    (2, 128, 128, 250, 130, 16),
    (4, 64, 64, 225, 70, 32),           # longer than some entries: queries that see no key
    (3, 258, 86, 250, 260, 64),         # three query heads to a head of the cache: 750 rows in three blocks
    (2, 320, 64, 100, 1300, 48),        # more tiles than the blocks of one look-ahead
    (8, 32, 32, 256, 16, 16),           # one tile, or none
    (1, 64, 64, 1000, 2111, 32),
]


@pytest.mark.parametrize("B,H,heads,Nq,longest,T", SHARED_TILES)
@pytest.mark.parametrize("d,fmt,mask,q_size", [(32, E4M3, 1, 1), (32, INT8, 0, 30), (64, E4M3, 0, 30), (64, INT8, 1, 1), (96, E4M3, 1, 30), (128, E4M3, 1, 1), (128, E4M3, 0, 30), (128, INT8, 1, 3),
                                               (256, E4M3, 1, 30)])
def test_attention_of_rows_that_share_tiles(B, H, heads, Nq, longest, T, d, fmt, mask, q_size):
    """Ragged lengths from 0 on and query counts, holes, logits of some units and of hundreds, which grow along the sequence in steps: the reference maximum
    rises a little or by more than a float holds; and a block that is no number."""
    rng = np.random.default_rng(Nq + d + q_size)
    lens = [longest] + [int(rng.integers(0, longest)) for _ in range(B - 1)]
    q_lens = [Nq] + [int(rng.integers(0, Nq + 1)) for _ in range(B - 1)]
    if B > 2:
        lens[1] = 0
    c, table = filled(rng, lens, heads, d, T, fmt)
    for blk in range(-(-longest // 16)):
        c.scale["k"][table[0, blk * 16 // T], :, blk % (T // 16)] *= np.float32(2.0 ** min(blk // 12, 4))
    if longest > 1000:
        table[0, 3], table[0, 9] = -1, c.n_pages + 2
    q = ref.bf16(rng.standard_normal((B, H, Nq, d)) * q_size)
    scale = float(np.float32(d ** -0.5))
    print(f"case attend shared tiles B={B} H={H}/{heads} Nq={Nq} lens={lens} q_lens={q_lens} T={T} d={d} fmt={fmt} mask={mask} q_size={q_size}", flush=True)
    want, bound = c.attend(q, table, lens, scale, mask, q_lens, untouched=np.full(q.shape, 7.0))
    dc = c.device()
    check(attend(dc, q, table, lens, scale, mask, q_lens, out=b16(np.full(q.shape, 7.0, np.float32))), want, bound)
    if longest > 200:
        at = (longest - 17) // 16
        dc.v_scale[int(table[0, at * 16 // T]), heads - 1, at % (T // 16)] = float("nan")
        o = attend(dc, q, table, lens, scale, mask, q_lens).float().cpu().numpy()
        first = max(16 * at - (longest - Nq), 0) if mask else 0
        hit = o[0, -(H // heads):]
        assert np.isnan(hit[:, first:]).all() and np.isfinite(hit[:, :first]).all() and np.isfinite(o[0, : H - H // heads]).all()


@pytest.mark.parametrize("d", [64, 128])
def test_logits_that_stay_somewhat_above_the_first_ones(d):
    """Rows of 256-row blocks whose first keys have logit 0 and whose later ones 2, 3, ... 9 in base 2: around what lets the reference maximum be, and sums of
    sixteen of them around what does not."""
    rng = np.random.default_rng(d)
    B, heads, Nq, n = 4, 64, 256, 640
    c = ref.Cache(B * n // 64, heads, 64, d, E4M3, rng)
    table = np.arange(B * n // 64, dtype=np.int32).reshape(B, -1)
    c.scale["k"][:], c.scale["v"][:] = 1.0, 2.0 ** -6
    c.codes["k"][:] = 0
    v = ref.to_codes(rng.standard_normal(c.codes["v"].shape) * 40, E4M3)
    c.codes["v"][:] = v
    for t in range(1, n // 64):      # channel 0 alone tells the keys apart: 1, 1.125, 1.25, ...
        c.codes["k"][t::n // 64, :, :, :, 0] = ref.to_codes(np.full(c.codes["k"][t::n // 64, :, :, :, 0].shape, 1.0 + t / 8), E4M3)
    q = np.zeros((B, heads, Nq, d))
    q[..., 0] = ref.bf16(np.log(2.0) * rng.integers(1, 9, (B, heads, Nq)) / 2)
    want, bound = c.attend(q, table, [n] * B, 2.0, 0)
    check(attend(c.device(), q, table, [n] * B, 2.0, 0), want, bound)


@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_attention_over_a_few_long_entries_among_many_short_ones(fmt):
    """More entries than a wavefront has lanes, divided by lengths that only the device knows; and a table with room for far more than the entries have."""
    rng = np.random.default_rng(15)
    lens = rng.integers(0, 200, 100)
    lens[[3, 64, 65, 99]] = [12000, 9001, 30, 11111]
    q = ref.bf16(rng.standard_normal((100, 3, 1, 64)))
    c, table = filled(rng, lens, 1, 64, 32, fmt)
    want, bound = c.attend(q, table, lens, 0.125, 1)
    check(attend(c.device(), q, table, lens, 0.125, 1), want, bound)
    few = [5, 0, 40]
    c, table = filled(rng, few, 2, 128, 16, fmt, extra=3000)
    q = ref.bf16(rng.standard_normal((3, 4, 2, 128)))
    assert fa.flat_attn_fwd_cache8_workspace_bytes(3, 4, 2, 2, table.shape[1] * 16, 128) > 0
    want, bound = c.attend(q, table, few, 0.09, 1)
    check(attend(c.device(), q, table, few, 0.09, 1), want, bound)


def test_attention_over_many_short_entries_and_lengths_out_of_range():
    """More entries than a wavefront looks over at once, and more than are ever divided; lengths below 0 and beyond the table count as the nearest that can be."""
    rng = np.random.default_rng(5)
    heads, d, T = 1, 64, 32
    for B in (130, 1100):
        lens = rng.integers(0, 400 if B < 200 else 60, B)
        c, table = filled(rng, lens, heads, d, T, E4M3, extra=0)
        said = lens.copy()
        said[lens == lens.max()] = 10 ** 6          # the row of the longest is full only if its pages are
        full = table.shape[1] * T
        lens = np.where(said > full, full, lens)
        said[3], lens[3] = -7, 0
        q = ref.bf16(rng.standard_normal((B, 2, 1, d)))
        for name in "kv":  # what lies between the end and the end of the page is seen now: make it numbers
            c.codes[name] = np.where((c.codes[name] & 127) == 127, 1, c.codes[name]).astype(np.uint8)
        want, bound = c.attend(q, table, lens, 0.125, 1)
        check(attend(c.device(), q, table, said, 0.125, 1), want, bound)


@pytest.mark.parametrize("Nq", [1, 40])
@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_holes_in_the_page_table_count_for_nothing(Nq, fmt):
    rng = np.random.default_rng(8)
    lens = [3000, 100, 64]
    c, table = filled(rng, lens, 2, 64, 16, fmt)
    table[0, ::3], table[0, 5], table[1] = -1, c.n_pages, 2 ** 31 - 1
    q = ref.bf16(rng.standard_normal((3, 4, Nq, 64)))
    for mask in (0, 1):
        want, bound = c.attend(q, table, lens, 0.125, mask)
        check(attend(c.device(), q, table, lens, 0.125, mask), want, bound)
        assert (want[1] == 0).all()


def test_extreme_logits_and_scales():
    """One key far above the others, logits that all lie far below zero, blocks of zeros (scale 0), scale 0 for the logits, and scales that are no powers of two."""
    rng = np.random.default_rng(6)
    lens, d = [400, 333], 64
    c, table = filled(rng, lens, 2, d, 32, INT8)
    q = ref.bf16(rng.standard_normal((2, 4, 2, d)))
    c.scale["v"] = (c.scale["v"] * rng.uniform(0.6, 1.9, c.scale["v"].shape)).astype(np.float32)
    c.scale["k"][table[0, 3], 0, 1] = 0.0
    c.scale["v"][table[0, 2]] = 0.0
    c.scale["k"][table[0, 4], 1, 0] = 300.0           # logits in the thousands
    c.scale["k"][table[1, :11], 1] = 3e4
    for scale in (0.125, 0.0, 1e-30, 1.0):
        for mask in (0, 1):
            want, bound = c.attend(q, table, lens, scale, mask)
            # a logit of size s is off by 2^-23 s in fp32, in the exponent: where that is not small the weight of neighbours is not settled
            check(attend(c.device(), q, table, lens, scale, mask), want, bound)
    # every key's logit is -1e5: the reference maximum follows
    c2, t2 = filled(rng, [100], 1, d, 32, INT8)
    c2.codes["k"][:] = 100
    c2.scale["k"][:] = 1.0
    want, bound = c2.attend(-np.ones((1, 1, 1, d), np.float32) * 16, t2, [100], 1.0, 0)
    check(attend(c2.device(), -np.ones((1, 1, 1, d), np.float32) * 16, t2, [100], 1.0, 0), want, bound)


def test_pools_beyond_four_gigabytes():
    import torch
    n_pages, heads, T, d = 330_000, 1, 64, 256                 # 5.4 GB of codes each
    k, v = (torch.empty(n_pages, heads, T, d, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.empty(n_pages, heads, T // 16, dtype=torch.float32, device="cuda") for _ in range(2))
    big = fa.FlatCache8(k, v, ks, vs, E4M3)
    rng = np.random.default_rng(2)
    n = 150
    x, y = (ref.bf16(rng.standard_normal((1, heads, n, d))) for _ in range(2))
    pages = [n_pages - 1, n_pages - 70000, 5]
    fa.flat_attn_cache8_write(big, b16(x), b16(y), i32([pages]), i32([0]))
    small = ref.Cache(3, heads, T, d, E4M3)
    small.write(x, y, np.array([[0, 1, 2]]), [0])
    q = ref.bf16(rng.standard_normal((1, 2, 1, d)))
    want, bound = small.attend(q, np.array([[0, 1, 2]]), [n], 0.0625, 0)
    check(attend(big, q, np.array([pages]), [n], 0.0625, 0), want, bound)
    fa.flat_attn_cache8_copy_pages(big, i32([n_pages - 1, 5]), i32([7, n_pages - 2]))
    check(attend(big, q, np.array([[7, n_pages - 70000, n_pages - 2]]), [n], 0.0625, 0), want, bound)


def test_token_numbers_near_31_bits():
    """The widest page table there is, of holes but for its first page and its last two: lengths and token numbers close to 2^31, and a write whose rows would pass it."""
    import torch
    T, d, width = 65536, 32, (2 ** 31 - 65537) // 65536
    rng = np.random.default_rng(31)
    cap = width * T
    small = ref.Cache(3, 1, T, d, E4M3)
    start, N = cap - 37, 131_200                                # the last 37 tokens there is room for, of rows that go on beyond 2^31
    x, y = (ref.bf16(rng.standard_normal((1, 1, N, d))) for _ in range(2))
    dc = small.device()
    table = np.full((1, width), -1, np.int32)
    table[0, [0, width - 2, width - 1]] = [1, 0, 2]
    fa.flat_attn_cache8_write(dc, b16(x), b16(y), i32(table), i32([start]))
    first = [ref.bf16(rng.standard_normal((1, 1, 50, d))) for _ in range(2)]
    fa.flat_attn_cache8_write(dc, b16(first[0]), b16(first[1]), i32(table), i32([0]))
    small.write(first[0], first[1], np.array([[1, 0, 2]], np.int32), [0])
    small.write(x[:, :, :37], y[:, :, :37], np.array([[1, 0, 2]], np.int32), [3 * T - 37])
    small.like(dc).assert_same(small)
    q = ref.bf16(rng.standard_normal((1, 2, 3, d)))
    for n in (cap, cap - 5):                                    # holes count for nothing: a short table with the same tokens
        want, bound = small.attend(q, np.array([[1, 0, 2]], np.int32), [3 * T - (cap - n)], 2.0, 1)
        check(attend(dc, q, table, [n], 2.0, 1), want, bound)


# ---- pages ---------------------------------------------------------------------------------------------------------------------------------

def random_cache(rng, n_pages=23, heads=3, T=32, d=32):
    return ref.Cache(n_pages, heads, T, d, E4M3, rng)


def move(c, src, dst):
    for n in "kv":
        c.codes[n][dst], c.scale[n][dst] = c.codes[n][src].copy(), c.scale[n][src].copy()


@pytest.mark.parametrize("heads,T,d", [(1, 16, 32), (3, 32, 96), (8, 256, 256)])
def test_copy_pages(heads, T, d):
    """Pairs that count, and those that do not: ids out of range, a page onto itself, a destination named again, a source that is a destination."""
    import torch
    rng = np.random.default_rng(d)
    c = random_cache(rng, 23, heads, T, d)
    src = [0, 1, 2, -1, 5, 6, 7, 7, 9, 23, 11, 3, 4]
    dst = [12, 13, 13, 14, 23, 6, 15, 16, 17, 18, 0, 4, 2147483647]
    dc = c.device()
    fa.flat_attn_cache8_copy_pages(dc, i32(src), i32(dst))
    torch.cuda.synchronize()
    # (0 -> 12) is left out: 0 is a destination; (1 -> 13) is followed by (2 -> 13); 6 stays; 7 goes to two pages
    for s, t in ((2, 13), (7, 15), (7, 16), (9, 17), (11, 0), (3, 4)):
        move(c, s, t)
    c.like(dc).assert_same(c)
    fa.flat_attn_cache8_copy_pages(dc, i32([]), i32([]))
    n = 3000                                                    # a list longer than a workgroup looks through at once
    src, dst = np.full(n, 20), np.full(n, 21)
    src[-1] = 19
    fa.flat_attn_cache8_copy_pages(dc, i32(src), i32(dst))
    torch.cuda.synchronize()
    move(c, 19, 21)
    c.like(dc).assert_same(c)


def test_fork():
    import torch
    rng = np.random.default_rng(1)
    T = 32
    lens = [70, 64, 0, 5, 0, 33, 0, 0, 96, 0, 0, 0]
    c = random_cache(rng, 40)
    table = ref.page_table(rng, lens, T, 30, 5)
    table[5, 1] = -1                                            # the begun page of 5 is a hole
    table[8, 3:] = [38, 39]                                     # pages set aside for what is to come
    before, L = table.copy(), np.array(lens, np.int32)
    parents = [0, 1, 3, 5, 8, 0, 0, 12, 0, 2, 9, 0, 1]
    children = [2, 4, 6, 7, 9, 10, 10, 11, 0, 11, 11, 11, -1]
    spares = [30, -5, 31, 99, -1, 32, 33, 1, 2, 3, 4, 40, 5]
    dc, dt, dl = c.device(), i32(table), i32(L)
    fa.flat_attn_cache8_fork(dc, dt, dl, i32(parents), i32(children), i32(spares))
    torch.cuda.synchronize()
    # left out: the first fork to 10, those with ids out of range, 0 to itself (and its being listed leaves out all whose parent is 0), 2 and 9 as parents
    # (children of others), and 0 -> 11 with a spare out of range
    for p, ch, sp in ((1, 4, None), (3, 6, 31), (5, 7, None), (8, 9, None)):
        full = L[p] // T
        table[ch] = -1
        table[ch, :full] = before[p, :full]
        if sp is not None:
            table[ch, full] = sp
            move(c, before[p, full], sp)
        L[ch] = L[p]
    assert np.array_equal(dt.cpu().numpy(), table) and np.array_equal(dl.cpu().numpy(), L)
    c.like(dc).assert_same(c)
    # without the fork onto itself they count: 0 -> 2 with page 30, 0 -> 10 with page 33 (the later one); twice the same spare: the later one
    fa.flat_attn_cache8_fork(dc, dt, dl, i32([0, 0, 0, 3]), i32([2, 10, 10, 11]), i32([30, 32, 33, 30]))
    torch.cuda.synchronize()
    for p, ch, sp in ((0, 10, 33), (3, 11, 30)):
        full = L[p] // T
        table[ch] = -1
        table[ch, :full], table[ch, full] = before[p, :full], sp
        move(c, before[p, full], sp)
        L[ch] = L[p]
    assert np.array_equal(dt.cpu().numpy(), table) and np.array_equal(dl.cpu().numpy(), L)
    c.like(dc).assert_same(c)


@pytest.mark.parametrize("n_pages", [1, 63, 64, 65, 5000, 1 << 20])
def test_free_lists_the_pages_that_nobody_holds(n_pages):
    import torch
    rng = np.random.default_rng(n_pages)
    n_seqs, width = 37, 11
    table = rng.integers(-3, n_pages + 3, (n_seqs, width)).astype(np.int32)
    lens = rng.integers(0, 100, n_seqs).astype(np.int32)
    for seqs in ([], [3, 3, 36, -1, 37, 0], list(range(n_seqs))):
        dt, dl = i32(table), i32(lens)
        unused, count = i32(np.full(n_pages, 77)), i32([77])
        fa.flat_attn_cache8_free(dt, dl, i32(seqs), unused, count)
        torch.cuda.synchronize()
        t, l = table.copy(), lens.copy()
        for s in seqs:
            if 0 <= s < n_seqs:
                t[s], l[s] = -1, 0
        free = np.setdiff1d(np.arange(n_pages), t)
        assert np.array_equal(dt.cpu().numpy(), t) and np.array_equal(dl.cpu().numpy(), l)
        assert count.item() == len(free) and np.array_equal(unused.cpu().numpy(), np.pad(free, (0, n_pages - len(free)), constant_values=-1))


@pytest.mark.parametrize("n_pages,held", [(1, 1), (1, 0), (64, 64), (65, 1), (300, 150), (300, 299), (4000, 37)])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(n_pages, held, in_place):
    import torch
    rng = np.random.default_rng(n_pages + held)
    c = random_cache(rng, n_pages, 2, 16, 32)
    ids = rng.permutation(n_pages)[:held]
    table = np.full((7, max(held, 1)), -1, np.int32)
    table[2, :held] = ids
    table[5, : held // 2] = ids[: held // 2]                    # shared pages
    table[6, 0] = n_pages + 5
    dc, dt, used = c.device(), i32(table), i32([77])
    new = dt if in_place else torch.full_like(dt, 77)
    ws = torch.full((fa.flat_attn_cache8_compact_workspace_bytes(n_pages),), 255, dtype=torch.uint8, device="cuda")
    fa.flat_attn_cache8_compact(dc, dt, new, used, ws)
    torch.cuda.synchronize()
    src, dst = sorted(p for p in ids if p >= held), sorted(set(range(held)) - set(ids.tolist()))
    name = dict(zip(src, dst))
    for s, t in name.items():
        move(c, s, t)
    assert used.item() == held
    assert np.array_equal(new.cpu().numpy(), np.vectorize(lambda p: name.get(p, p))(table))
    c.like(dc).assert_same(c)


# ---- together ------------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_a_batch_is_served(fmt):
    """Prompts rotated, written and attended to; tokens one by one; a request forked, both halves continued apart; one freed; the pool compacted, and
    the answers after it are the same bits as before."""
    import torch
    rng = np.random.default_rng(fmt)
    heads, G, d, T, B, width, n_pages = 2, 3, 64, 32, 4, 6, 30
    H, scale = heads * G, 0.125
    freqs = fa.flat_attn_rope_freqs(d)
    df = freqs.cuda()
    c = ref.Cache(n_pages, heads, T, d, fmt, rng)
    dc = c.device()
    table, lens = np.full((B, width), -1, np.int32), np.zeros(B, np.int32)
    free = list(rng.permutation(n_pages))

    def step(n_new):
        N = max(n_new)
        for b in range(B):
            while (table[b] >= 0).sum() * T < lens[b] + n_new[b]:
                table[b, (table[b] >= 0).sum()] = free.pop()
        q, k, v = (ref.bf16(rng.standard_normal((B, h, N, d))) for h in (H, heads, heads))
        pos = lens[:, None] + np.arange(N)
        dq, dk = b16(q), b16(k)
        fa.flat_attn_rope(dq, dq, dk, dk, df, i32(pos))
        fa.flat_attn_cache8_write(dc, dk, b16(v), i32(table), i32(lens), i32(n_new))
        q, k = dq.float().cpu().numpy(), dk.float().cpu().numpy()
        c.write(k, v, table, lens, n_new)
        lens[:] += np.asarray(n_new, np.int32)
        want, bound = c.attend(q, table, lens, scale, 1, n_new, untouched=np.full(q.shape, 3.0))
        o = attend(dc, q, table, lens, scale, 1, n_new, out=b16(np.full(q.shape, 3.0, np.float32)))
        check(o, want, bound)
        c.like(dc).assert_same(c)
        return q, o

    step([50, 7, 0, 33])
    for _ in range(3):
        step([1, 1, 0, 1])
    dt, dl, spare = i32(table), i32(lens), int(free.pop())
    fa.flat_attn_cache8_fork(dc, dt, dl, i32([0]), i32([2]), i32([spare]))
    move(c, table[0, 1], spare)
    table[2], lens[2] = [table[0, 0], spare, -1, -1, -1, -1], lens[0]
    assert np.array_equal(dt.cpu().numpy(), table) and np.array_equal(dl.cpu().numpy(), lens)
    step([2, 1, 5, 0])
    unused, count = torch.empty(n_pages, dtype=torch.int32, device="cuda"), i32([0])
    dt, dl = i32(table), i32(lens)
    fa.flat_attn_cache8_free(dt, dl, i32([1]), unused, count)
    table[1], lens[1] = -1, 0
    assert sorted(unused[: count.item()].tolist()) == sorted(set(range(n_pages)) - set(table.ravel().tolist()))
    q = ref.bf16(rng.standard_normal((B, H, 1, d)))
    before = attend(dc, q, table, lens, scale, 1)
    used = i32([0])
    fa.flat_attn_cache8_compact(dc, dt, dt, used, torch.empty(fa.flat_attn_cache8_compact_workspace_bytes(n_pages), dtype=torch.uint8, device="cuda"))
    after = attend(dc, q, dt.cpu().numpy(), lens, scale, 1)
    assert torch.equal(before.view(torch.int16), after.view(torch.int16)) and dt.max().item() == used.item() - 1


def test_a_step_is_captured_and_replayed():
    """Rotation, write and attention of one token in a HIP graph whose lengths and positions are updated between the replays, with eager work of
    another size between them; every replay equals an eager step on a copy of the cache, on a stream of its own."""
    import torch
    rng = np.random.default_rng(12)
    B, heads, H, d, T, width = 3, 2, 8, 128, 16, 40
    start = [600, 31, 255]
    c, table = filled(rng, [n + 16 for n in start], heads, d, T, E4M3, extra=0)
    dc, mirror = c.device(), c.device()
    dt, freqs = i32(table), fa.flat_attn_rope_freqs(d).cuda()
    q, k, v, rq, rk, o = (torch.zeros(B, h, 1, d, dtype=torch.bfloat16, device="cuda") for h in (H, heads, heads, H, heads, H))
    lens, total = i32(start), i32(np.array(start) + 1)
    pos = lens.view(B, 1)
    nbytes = fa.flat_attn_fwd_cache8_workspace_bytes(B, H, heads, 1, table.shape[1] * T, d)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")

    def step(cache, q, k, v, rq, rk, o, lens, total, pos, ws, stream=None):
        fa.flat_attn_rope(q, rq, k, rk, freqs, pos, stream=stream)
        fa.flat_attn_cache8_write(cache, rk, v, dt, lens, stream=stream)
        fa.flat_attn_fwd_cache8(cache, rq, o, dt, total, 0.09, 1, workspace=ws, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    scratch = c.device()
    step(scratch, q, k, v, rq, rk, o, lens, total, pos, ws)   # loads the kernels
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(dc, q, k, v, rq, rk, o, lens, total, pos, ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for n in range(4):
        for t, h in ((q, H), (k, heads), (v, heads)):
            t.copy_(b16(rng.standard_normal((B, h, 1, d)).astype(np.float32)))
        now = [start[b] + n for b in range(B)]
        lens.copy_(i32(now))
        total.copy_(i32(np.array(now) + 1))
        o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        e = torch.full_like(o, float("nan"))
        step(mirror, q.clone(), k.clone(), v.clone(), torch.empty_like(q), torch.empty_like(k), e, i32(now), i32(np.array(now) + 1), i32(now).view(B, 1),
             torch.empty_like(ws))
        torch.cuda.synchronize()
        assert torch.equal(o.view(torch.int16), e.view(torch.int16)), n
        assert torch.equal(dc.k, mirror.k) and torch.equal(dc.v, mirror.v) and torch.equal(dc.k_scale, mirror.k_scale)


def test_refusals_on_the_device():
    import torch
    c = ref.Cache(4, 2, 32, 64, E4M3).device()
    x = torch.zeros(2, 2, 1, 64, dtype=torch.bfloat16, device="cuda")
    t, l = i32([[0], [1]]), i32([0, 0])
    q, o = torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16, device="cuda")
    for f, args in ((fa.flat_attn_cache8_write, (c, x, x.float(), t, l)), (fa.flat_attn_cache8_write, (c, x, x, t.long(), l)), (fa.flat_attn_cache8_write, (c, x, x, t[:1].contiguous(), l)),
                    (fa.flat_attn_cache8_write, (c, x, x, t, l.cpu())), (fa.flat_attn_fwd_cache8, (c, q, o[:, :2], t, l, 1.0)), (fa.flat_attn_fwd_cache8, (c, q[..., :32].contiguous(), o, t, l, 1.0)),
                    (fa.flat_attn_fwd_cache8, (c, q, o, t, l[:1], 1.0)), (fa.flat_attn_cache8_copy_pages, (c, l, l[:1])), (fa.flat_attn_cache8_free, (t, l, l, l, l)),
                    (fa.flat_attn_cache8_compact, (c, t, t.t(), l[:1], x))):
        with pytest.raises(ValueError):
            f(*args)
    big = i32(np.zeros((2, 100)))
    for ws, status in ((None, -1), (torch.zeros(4, device="cuda"), -5)):
        with pytest.raises(fa.FlatAttnError) as e:
            fa.flat_attn_fwd_cache8(c, q, o, big, l, 1.0, workspace=ws)
        assert e.value.status == status
    with pytest.raises(fa.FlatAttnError) as e:
        fa.flat_attn_fwd_cache8(c, q[:, :3].contiguous(), o[:, :3].contiguous(), t, l, 1.0)
    assert e.value.status == -2
