"""Plain numpy implementation, in 64 bits, of the paged 8-bit cache and of rotary positions, written from the header: what the tests compare with."""
import numpy as np

BLOCK = 16
E4M3, INT8 = 0, 1
LARGEST = {E4M3: 448.0, INT8: 127.0}


def e4m3_values():
    """The value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 fraction bits; 0x7f and 0xff are NaN."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


E4M3_VALUES = e4m3_values()


def to_codes(x, fmt):
    """Codes (uint8) of the values nearest to x, ties to the even code; |x| <= the largest."""
    if fmt == INT8:
        return np.rint(x).astype(np.int8).view(np.uint8)
    grid = E4M3_VALUES[:127]                       # codes 0 .. 126 ascend from 0 to 448
    a = np.abs(x)
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    dl, dh = a - grid[lo], grid[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def from_codes(c, fmt):
    return c.view(np.int8).astype(np.float64) if fmt == INT8 else E4M3_VALUES[c]


def bf16(x):
    """x rounded to bf16, as float32."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7fff + ((b >> 16) & 1)) & 0xffff0000).astype(np.uint32)
    return r.view(np.float32).reshape(np.shape(x))


class Cache:
    """Codes and scales by block: k [pages, heads, blocks, token, channel] in the logical order, whatever their order in memory."""

    def __init__(self, n_pages, heads, page_tokens, d, fmt, rng=None):
        self.n_pages, self.heads, self.T, self.d, self.fmt = n_pages, heads, page_tokens, d, fmt
        shape = (n_pages, heads, page_tokens // BLOCK, BLOCK, d)
        if rng is None:
            self.codes = {n: np.zeros(shape, np.uint8) for n in "kv"}
            self.scale = {n: np.zeros(shape[:3], np.float32) for n in "kv"}
        else:  # anything a pool may hold, NaN codes among it
            self.codes = {n: rng.integers(0, 256, shape).astype(np.uint8) for n in "kv"}
            self.scale = {n: np.exp2(rng.integers(-6, 3, shape[:3])).astype(np.float32) for n in "kv"}

    def to_memory(self):
        p, h, b, t, d = self.codes["k"].shape
        k = self.codes["k"].reshape(p, h, b, t, d // 16, 16).transpose(0, 1, 2, 4, 3, 5).reshape(p, h, b * t, d)
        v = self.codes["v"].transpose(0, 1, 2, 4, 3).reshape(p, h, b * t, d)
        return np.ascontiguousarray(k), np.ascontiguousarray(v)

    def from_memory(self, k, v, ks, vs):
        p, h, b, t, d = self.codes["k"].shape
        self.codes["k"] = np.ascontiguousarray(k.reshape(p, h, b, d // 16, t, 16).transpose(0, 1, 2, 4, 3, 5).reshape(p, h, b, t, d))
        self.codes["v"] = np.ascontiguousarray(v.reshape(p, h, b, d, t).transpose(0, 1, 2, 4, 3))
        self.scale = {"k": ks, "v": vs}
        return self

    def device(self):
        """(FlatCache8, its tensors) on the GPU with these contents."""
        import torch
        import paper_2107_06419_amd as fa
        k, v = (torch.from_numpy(x).cuda() for x in self.to_memory())
        ks, vs = (torch.from_numpy(self.scale[n].copy()).cuda() for n in "kv")
        return fa.FlatCache8(k, v, ks, vs, self.fmt)

    def like(self, c):
        """The contents of a FlatCache8."""
        out = Cache.__new__(Cache)
        out.__dict__.update(self.__dict__)
        return out.from_memory(*(t.cpu().numpy() for t in (c.k, c.v, c.k_scale, c.v_scale)))

    def assert_same(self, other):
        for n in "kv":
            a, b = self.scale[n], other.scale[n]
            assert np.array_equal(a, b, equal_nan=True), (n, "scales", np.argwhere(~((a == b) | (np.isnan(a) & np.isnan(b))))[:5])
            assert np.array_equal(self.codes[n], other.codes[n]), (n, "codes", np.argwhere(self.codes[n] != other.codes[n])[:5])

    def write(self, k, v, table, lens, n_new=None):
        """k, v float32 [B, heads, N, d]; token by token into blocks, block by block."""
        B, H, N, _ = k.shape
        cap = table.shape[1] * self.T
        for b in range(B):
            start = min(max(int(lens[b]), 0), cap)
            n = N if n_new is None else min(max(int(n_new[b]), 0), N)
            end = min(start + n, cap)
            for blk in range(start // BLOCK, -(-end // BLOCK) if end > start else 0):
                page, at = int(table[b, blk * BLOCK // self.T]), blk % (self.T // BLOCK)
                if not 0 <= page < self.n_pages:
                    continue
                lo, hi = max(start, blk * BLOCK), min(end, (blk + 1) * BLOCK)
                kept = lo - blk * BLOCK
                for name, x in (("k", k), ("v", v)):
                    for h in range(H):
                        new = x[b, h, lo - start:hi - start].astype(np.float64)
                        old = from_codes(self.codes[name][page, h, at, :kept], self.fmt) * (np.float64(self.scale[name][page, h, at]) if kept else 1.0)
                        before = np.float64(self.scale[name][page, h, at]) if kept else 0.0
                        most = np.abs(new).max() if new.size else 0.0
                        if not np.isfinite(new).all() or np.isnan(before):
                            scale = np.nan
                        else:
                            need = 0.0
                            if most > 0:
                                e = -100
                                while most > LARGEST[self.fmt] * 2.0 ** e:
                                    e += 1
                                need = 2.0 ** e
                            scale = max(before, need)
                        block = np.zeros((BLOCK, self.d))
                        if scale > 0:
                            block[:kept] = old / scale
                            block[kept:kept + len(new)] = new / scale
                        self.codes[name][page, h, at] = to_codes(block, self.fmt)
                        self.scale[name][page, h, at] = np.float32(scale)

    def values(self, name, table_row, n):
        """[heads, n, d] values of the first n tokens of a row, and which of them are there."""
        per = self.T // BLOCK
        out, there = np.zeros((self.heads, n, self.d)), np.zeros(n, bool)
        for blk in range(-(-n // BLOCK)):
            page = int(table_row[blk // per])
            if not 0 <= page < self.n_pages:
                continue
            lo, hi = blk * BLOCK, min(n, blk * BLOCK + BLOCK)
            x = from_codes(self.codes[name][page, :, blk % per], self.fmt) * self.scale[name][page, :, blk % per].astype(np.float64)[:, None, None]
            out[:, lo:hi], there[lo:hi] = x[:, :hi - lo], True
        return out, there

    def attend(self, q, table, lens, scale, mask, q_lens=None, untouched=None):
        """(O, bound): the answer, and how far a bf16 kernel may be off: half a step of the result, half a step of every probability, and what
        fp32 products and sums of the logits are off by.  A probability times its value's scale that lies below the smallest normal number, 2^-126, may count
        as 0: a key then lacks up to 2^-126 times its code, at most 448 or 127, over a sum of probabilities that is at least 1, the largest one's."""
        lost = LARGEST[self.fmt] * 2.0 ** -126
        B, H, Nq, d = q.shape
        G = H // self.heads
        cap = table.shape[1] * self.T
        out = np.zeros(q.shape) if untouched is None else untouched.astype(np.float64).copy()
        bound = np.zeros(q.shape)
        for b in range(B):
            n = min(max(int(lens[b]), 0), cap)
            rows = Nq if q_lens is None else min(max(int(q_lens[b]), 0), Nq)
            (k, there), (v, _) = self.values("k", table[b], n), self.values("v", table[b], n)
            out[b, :, :rows] = 0.0
            k, v = k[:, there], v[:, there]            # what is not there may be anything
            j = np.arange(n)[there]
            if not len(j):
                continue
            seen = np.ones((rows, len(j)), bool) if not mask else j[None] <= np.arange(rows)[:, None] + n - rows
            for h in range(H):
                kk, vv, row = k[h // G], v[h // G], q[b, h, :rows].astype(np.float64)
                with np.errstate(invalid="ignore"):
                    x = np.where(seen, row @ kk.T * scale, -np.inf)
                top = x.max(1, keepdims=True)
                p = np.exp(x - np.where(np.isinf(top), 0.0, top))
                total = p.sum(1, keepdims=True)
                p /= np.where(total > 0, total, 1.0)
                size = np.where(seen, np.abs(row) @ np.abs(kk).T, 0.0).max(1, keepdims=True) * scale
                off = 2.0 ** -8 + 2 * size * (d + 8) * 2.0 ** -24 + seen.sum(1, keepdims=True) * 2.0 ** -24 + 2.0 ** -20
                out[b, h, :rows] = p @ vv
                bound[b, h, :rows] = 2.0 ** -8 * np.abs(out[b, h, :rows]) + off * 1.01 * (p @ np.abs(vv)) + len(j) * lost
        return out, bound


def rope(x, freqs, positions, rot, interleaved, magnitude, transpose):
    """x [B,H,N,d] in 64 bits."""
    y = x.astype(np.float64).copy()
    t = positions.astype(np.float64)[:, None, :, None] * freqs
    c, s = np.cos(t) * magnitude, np.sin(t) * magnitude * (-1.0 if transpose else 1.0)
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    xa, xb = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = xa * c - xb * s, xa * s + xb * c
    return y


def page_table(rng, lens, page_tokens, n_pages, width):
    """Scattered pages for the lengths; -1 behind them."""
    need = [-(-max(int(n), 0) // page_tokens) for n in lens]
    ids = rng.permutation(n_pages)[:sum(need)]
    table, at = np.full((len(lens), width), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table
