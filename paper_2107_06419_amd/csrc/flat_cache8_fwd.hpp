// Attention over the 8-bit paged cache (flat_cache8.hpp has the layout): device code shared by the kernels of flat_cache8_fwd.hip.
#pragma once
#include "flat_cache8.hpp"
#include "flat_common.hpp"
#include "flat_launch.hpp"

namespace flat {

constexpr int kCacheTile = 2 * kCacheBlock;  // keys of a step: one 32 x 32 logit tile

// Kernel arguments: geometry, and quotients by launch-time divisors.
struct Cache8Args {
    const uint8_t *k, *v;
    const float *ks, *vs;
    const bf16* Q;
    bf16* O;
    const int *page_table, *lens, *q_lens;
    float* ws;
    int n_pages, heads, max_pages, max_tokens;
    int B, H, Nq, group;  // group = H / heads
    float scale_log2;
    int causal;
    int rows_per_block, row_blocks, entries, target, least_tiles;
    Divisor by_heads, by_group, by_row_blocks, by_page_blocks;
    int page_blocks;
};

// One entry of a launch: a row block of a batch entry, with the lengths it goes by.
struct CacheEntry {
    int b, row0, rows, len, q_len;  // rows: that the entry has in all (q_len * group)
    int tiles;                      // of kCacheTile keys that any of its rows sees
};

__device__ __forceinline__ CacheEntry cache_entry(const Cache8Args& a, int e) {
    CacheEntry t;
    t.b = a.by_row_blocks.quotient(e);
    t.row0 = (e - t.b * a.row_blocks) * a.rows_per_block;
    t.len = min(max(a.lens[t.b], 0), a.max_tokens);
    t.q_len = a.q_lens ? min(max(a.q_lens[t.b], 0), a.Nq) : a.Nq;
    t.rows = t.q_len * a.group;
    int seen = t.len;
    if (a.causal) {  // what the last row of the block sees
        const int last = a.by_group.quotient(max(min(t.rows, t.row0 + a.rows_per_block) - 1, 0));
        seen = min(max(last + 1 + t.len - t.q_len, 0), t.len);
    }
    t.tiles = (seen + kCacheTile - 1) / kCacheTile;
    return t;
}

// Units of an entry: one at least if it has rows (they have to be written), each of `chunk` tiles at most.
__device__ __forceinline__ int cache_units(const CacheEntry& t, int chunk) {
    if (t.row0 >= t.rows) return 0;
    return chunk == 0 ? 1 : max((int)(((unsigned)t.tiles + (unsigned)chunk - 1u) / (unsigned)chunk), 1);
}

__device__ __forceinline__ unsigned long long wave_sum_u64(unsigned long long x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// Tiles of a unit: the keys of all entries over the units aimed at, so that long entries get more units than short ones whatever
// the lengths, which only the device knows; 0: entries are not divided.
__device__ __forceinline__ int cache_chunk(const Cache8Args& a, int lane) {
    if (a.target == 0) return 0;
    unsigned long long total = 0;
    for (int e = lane; e < a.entries; e += 64) {
        const CacheEntry t = cache_entry(a, e);
        total += t.row0 < t.rows ? t.tiles : 0;
    }
    total = wave_sum_u64(total) + (unsigned)a.target - 1u;
    const int chunk = total >> 32 ? (int)(total / (unsigned)a.target) : (int)((unsigned)total / (unsigned)a.target);
    return max(__builtin_amdgcn_readfirstlane(chunk), a.least_tiles);
}

// Inclusive sum over the lanes up to this one.
__device__ __forceinline__ int wave_prefix(int x, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        x += lane >= o ? y : 0;
    }
    return x;
}

// The entry that unit u belongs to, the units before it and its own number of them; entry = -1: the launch has fewer units.
struct CacheUnit {
    int entry, before, n;
};
__device__ __forceinline__ CacheUnit cache_find_unit(const Cache8Args& a, int u, int chunk, int lane) {
    int before = 0;
    for (int e0 = 0; e0 < a.entries; e0 += 64) {
        const int n = e0 + lane < a.entries ? cache_units(cache_entry(a, e0 + lane), chunk) : 0;
        const int upto = wave_prefix(n, lane) + before;
        const unsigned long long found = __ballot(u < upto);
        if (found) {
            const int l = __builtin_amdgcn_readfirstlane(__builtin_ctzll(found));
            const int mine = __builtin_amdgcn_readlane(n, l);
            return {e0 + l, __builtin_amdgcn_readlane(upto, l) - mine, mine};
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return {-1, 0, 0};
}
// The units before entry e, and its own.
__device__ __forceinline__ CacheUnit cache_units_of(const Cache8Args& a, int e, int chunk, int lane) {
    int before = 0;
    for (int e0 = 0; e0 <= e; e0 += 64) {
        const int n = e0 + lane < a.entries ? cache_units(cache_entry(a, e0 + lane), chunk) : 0;
        const int upto = wave_prefix(n, lane) + before;
        if (e < e0 + 64) {
            const int mine = __builtin_amdgcn_readlane(n, e - e0);
            return {e, __builtin_amdgcn_readlane(upto, e - e0) - mine, mine};
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return {-1, 0, 0};
}

// Eight codes as bf16, exactly: e4m3 has 4 significant bits, int8 8.
template <int FMT>
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t lo, uint32_t hi) {
    if constexpr (FMT == FLAT_CACHE8_E4M3) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
        return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
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
