// Attention over the 8-bit paged cache (flat_cache8.hpp has the layout): device code shared by the kernels of flat_cache8_fwd.hip.
#pragma once
#include "flat_cache8.hpp"
#include "flat_common.hpp"
#include "flat_launch.hpp"

namespace flat {

// Kernel arguments: geometry, and quotients by launch-time divisors.
struct Cache8Args {
    const uint8_t *k, *v;
    const float *ks, *vs;
    const bf16* Q;
    bf16* O;
    const int *page_table, *lens, *q_lens;
    int2* units;  // workspace of a launch that divides entries: of every entry the units before it and its own,
    float* parts; // and the units' partial results
    int n_pages, heads, max_pages, max_tokens;
    int B, H, Nq, group;  // group = H / heads
    float scale_log2;
    int causal;
    int rows_per_block, row_blocks, entries, tile_shift, aim, limit, least_tiles;
    Divisor by_heads, by_group, by_row_blocks, by_page_blocks;
    int page_blocks;
};

// One entry of a launch: a row block of a batch entry, with the lengths it goes by.
struct CacheEntry {
    int b, row0, len, q_len;
    int rows;   // that the batch entry has in all (q_len * group)
    int tiles;  // of 2^tile_shift keys that any row of the block sees
};

__device__ __forceinline__ CacheEntry cache_entry_of(const Cache8Args& a, int e, int len, int q_len) {
    CacheEntry t;
    t.b = a.by_row_blocks.quotient(e);
    t.row0 = (e - t.b * a.row_blocks) * a.rows_per_block;
    t.len = len;
    t.q_len = q_len;
    t.rows = q_len * a.group;
    int seen = len;
    if (a.causal) {  // what the last row of the block sees
        const int last = a.by_group.quotient(max(min(t.rows, t.row0 + a.rows_per_block) - 1, 0));
        seen = min(max(last + 1 + len - q_len, 0), len);
    }
    t.tiles = (int)(((unsigned)seen + (1u << a.tile_shift) - 1u) >> a.tile_shift);
    return t;
}
__device__ __forceinline__ CacheEntry cache_entry(const Cache8Args& a, int e) {
    const int b = a.by_row_blocks.quotient(e);
    const int len = min(max(a.lens[b], 0), a.max_tokens), q_len = a.q_lens ? min(max(a.q_lens[b], 0), a.Nq) : a.Nq;
    return cache_entry_of(a, e, len, q_len);
}

__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_prefix(x), 63); }

// How the keys of the entries are divided.  Only the device knows the lengths, so every workgroup settles it for itself, all in the same way: a
// unit has at most `chunk` tiles; chunk is the tiles of all entries over the units aimed at, raised by eighths until there are no more units than
// workgroups were launched per head of the cache.  Long entries then get more units than short ones, and all units run at once.
struct CacheUnit {
    CacheEntry entry;
    int e;          // its number, -1: the launch has fewer units
    int before, n;  // the units before the entry, and its own
};
// Units of an entry with these tiles (-1: it has no rows).  Parts are made by their number alone, so a quotient off by one in its last place does no harm.
__device__ __forceinline__ int cache_units(int tiles, float per_chunk) { return tiles < 0 ? 0 : max((int)__builtin_ceilf((float)tiles * per_chunk), 1); }

__device__ __forceinline__ CacheUnit cache_find_unit(const Cache8Args& a, int u, int lane) {
    CacheUnit r;
    r.e = -1;
    auto tiles_of = [&](int e, CacheEntry* t) __attribute__((always_inline)) {
        if (e >= a.entries) return -1;
        *t = cache_entry(a, e);
        return t->row0 < t->rows ? min(t->tiles, 1 << 20) : -1;
    };
    CacheEntry t0{};
    const int tiles0 = tiles_of(lane, &t0);  // most launches have no more entries than lanes: then this is the only look at the lengths
    int total = wave_total(max(tiles0, 0));
    for (int e = 64; e < a.entries; e += 64) {
        CacheEntry t;
        total += wave_total(max(tiles_of(e + lane, &t), 0));
    }
    int chunk = max((int)(((unsigned)total + (unsigned)a.aim - 1u) / (unsigned)a.aim), a.least_tiles);
    float per_chunk;
    for (;;) {
        per_chunk = 1.0f / (float)chunk;
        int units = wave_total(cache_units(tiles0, per_chunk));
        for (int e = 64; e < a.entries; e += 64) {
            CacheEntry t;
            units += wave_total(cache_units(tiles_of(e + lane, &t), per_chunk));
        }
        if (units <= a.limit) break;  // at the latest with one unit per entry: the limit is no less than the entries
        chunk += (chunk + 7) >> 3;
    }
    int before = 0;
    for (int e0 = 0; e0 < a.entries; e0 += 64) {
        CacheEntry t = t0;
        const int n = cache_units(e0 ? tiles_of(e0 + lane, &t) : tiles0, per_chunk);
        const int upto = wave_prefix(n) + before;
        const unsigned long long found = __ballot(u < upto);
        if (found) {
            const int l = __builtin_ctzll(found);
            r.e = e0 + l;
            r.n = __builtin_amdgcn_readlane(n, l);
            r.before = __builtin_amdgcn_readlane(upto, l) - r.n;
            r.entry = cache_entry_of(a, r.e, __builtin_amdgcn_readlane(t.len, l), __builtin_amdgcn_readlane(t.q_len, l));
            return r;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return r;
}

// Tiles of part `part` of n: the first tiles % n parts have one more.  (The same for the whole wavefront, which the compiler does not see through a division.)
__device__ __forceinline__ void cache_part(int tiles, int part, int n, int* t0, int* t1) {
    const int share = (unsigned)tiles / (unsigned)n, more = tiles - share * n;
    *t0 = __builtin_amdgcn_readfirstlane(part * share + min(part, more));
    *t1 = __builtin_amdgcn_readfirstlane(*t0 + share + (part < more ? 1 : 0));
}

// What is needed of a block: its number in the pool (-1: a hole, or behind the entry's last token), how many of its tokens are there, and its scales.
// The value's scale goes into the exponent of the probabilities, 2^(ks s + vs_log2 - m), so that a logit costs one fma and the sum of a block's
// probabilities is put right by one more.  Where it is 0, the codes are cleared instead.
struct CacheBlock {
    int e, there;
    float ks, vs_log2, vs_inv;
};
__device__ __forceinline__ CacheBlock cache_block(const Cache8Args& a, int kvh, int len, int blk, int page) {
    CacheBlock x{-1, 0, 0.f, 0.f, 1.f};
    if (kCacheBlock * blk < len && (unsigned)page < (unsigned)a.n_pages) {
        x.e = (page * a.heads + kvh) * a.page_blocks + blk - a.by_page_blocks.quotient(blk) * a.page_blocks;
        x.ks = a.ks[x.e] * a.scale_log2;
        const float vs = a.vs[x.e];
        x.there = vs == 0.f ? 0 : min(len - kCacheBlock * blk, kCacheBlock);
        x.vs_log2 = vs == 0.f ? 0.f : __builtin_log2f(vs);
        x.vs_inv = vs == 0.f ? 1.f : 1.0f / vs;
    }
    return x;
}
// x of lane (byte address / 4).
__device__ __forceinline__ float value_of_lane(int at, float x) { return __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(at, __builtin_bit_cast(int, x))); }

// The running state of a row's softmax, in every lane that has it: reference maximum (log2 units), what is subtracted (0 until there is one), and the
// sum of this lane's keys.
struct RowState {
    float m, sub, l;
};
constexpr int kRescaleAbove = 8;  // log2: the reference maximum rises only when a logit is this far above it, so p stays below 2^8 and exact to rounding

// Probabilities of a tile: s holds the logits of the lane's row and block, token by token.  c: the block's key scale; the result is p * vs in
// bf16, and *l gets the sum of the block's p.  visible: tokens of the block that the row sees (all if !EDGE).  The sum is of the fp32 values, by additions: a bf16 dot product adds two
// at a time, but waits for the matrix unit; beside another wavefront's MFMAs 32 of them take 1197 cycles (without 161), 32 additions 204 (159).
// (Summing what the product's rounding left would cost two more instructions a pair; without, the error against 64 bits is 2.2e-3 instead of 2.0e-3, 2-norm.)
template <bool EDGE, typename S>
__device__ __forceinline__ void tile_probabilities(const S& s, float c, float vs_log2, float vs_inv, float sub, int visible, bf16x8* lo, bf16x8* hi, float* l) {
    const float b = vs_log2 - sub;
    uint4v plo, phi;
    float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
        float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, b)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + 1], c, b));
        if constexpr (EDGE) {  // chosen, not multiplied: logits of what is not seen, and scales of blocks that are not, may be no numbers
            p0 = r < visible ? p0 : 0.f;
            p1 = r + 1 < visible ? p1 : 0.f;
        }
        const uint32_t w = pack_bf16(p0, p1);
        sum0 += p0;
        sum1 += p1;
        if (r < 8) plo[r / 2] = w;
        else phi[r / 2 - 4] = w;
    }
    *lo = __builtin_bit_cast(bf16x8, plo);
    *hi = __builtin_bit_cast(bf16x8, phi);
    if (!EDGE || visible > 0) *l = __builtin_fmaf(sum0 + sum1, vs_inv, *l);  // a scale that is no number is none of a row that does not see the block
}

// v_mfma_f32_16x16x32_bf16:  D[16x16] += A[16x32] * B[32x16].  A: lane l holds row (l % 16), contraction indices 8 (l / 16) .. + 7; B: column (l % 16), the
// same indices; C/D: column (l % 16), register r is row 4 (l / 16) + r.
__device__ __forceinline__ floatx4 mfma_bf16_16x16x32(bf16x8 a, bf16x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Largest value, and sum, over the lanes that have a row: l and l ^ 32, and where a tile has 16 rows l ^ 16 too.
template <int ROWS>
__device__ __forceinline__ float row_max(float x) {
    x = halves_max(x);
    if constexpr (ROWS == 16) {
        const uint32_t u = __builtin_bit_cast(uint32_t, x);
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = __builtin_fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
    }
    return x;
}
template <int ROWS>
__device__ __forceinline__ float row_sum(float x) {
    x = halves_sum(x);
    if constexpr (ROWS == 16) {
        const uint32_t u = __builtin_bit_cast(uint32_t, x);
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
    }
    return x;
}

// Eight codes as bf16, exactly: e4m3 has 4 significant bits, int8 8.
template <int FMT>
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t lo, uint32_t hi) {
    if constexpr (FMT == FLAT_CACHE8_E4M3) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
        return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
        // byte by byte in the instruction that converts (SDWA); else the compiler takes the bytes apart an iteration ahead, and 50 registers with them
        asm("" : "+v"(lo), "+v"(hi));
        uint4v r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = i < 2 ? lo : hi;
            const int s = 16 * (i & 1);
            r[i] = pack_bf16((float)(int8_t)(w >> s), (float)(int8_t)(w >> (s + 8)));
        }
        return __builtin_bit_cast(bf16x8, r);
    }
}

// Codes of the tokens from n on (n < 16) of a V operand cleared: what lies behind an entry's last token may be anything, NaN codes among it.
__device__ __forceinline__ uint4v clear_behind(uint4v x, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int keep = min(max(n - 4 * i, 0), 4);
        x[i] &= keep == 4 ? 0xffffffffu : (1u << (8 * keep)) - 1u;
    }
    return x;
}

}  // namespace flat
