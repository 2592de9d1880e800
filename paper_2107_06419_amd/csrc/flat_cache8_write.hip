// New tokens into the 8-bit paged cache: quantisation by blocks of 16 tokens of a head.
//
// One wavefront has one block of K or of V: it finds the block's largest magnitude over its lanes, settles the scale, and writes the whole
// block (16 d codes).  A block that is begun already is read first.  Scales are powers of two, so a quotient by one is exact and the only
// rounding is that to the code; codes and scales are the same whatever the order of the work.  Long calls are bound by reading bf16 and writing codes, short
// ones by a chain of three dependent loads (length, page, scale and codes so far).
#include "flat_cache8.hpp"
#include "flat_common.hpp"

namespace flat {

namespace {

constexpr int kWaves = 4;

struct WriteArgs {
    uint8_t *k, *v;
    float *ks, *vs;
    const bf16 *K, *V;
    const int *page_table, *lens, *n_new;
    int n_pages, heads, page_blocks, max_pages, max_tokens, N, blocks;  // blocks: that N tokens may touch
    int waves;
    Divisor by_heads, by_blocks, by_page_blocks;
};

// Four values to four codes, to the nearest, ties to even.  |x| <= the format's largest value.
template <int FMT>
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
    if constexpr (FMT == FLAT_CACHE8_E4M3) {
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    } else {
        return ((uint32_t)(int)__builtin_rintf(a) & 255u) | (((uint32_t)(int)__builtin_rintf(b) & 255u) << 8) |
               (((uint32_t)(int)__builtin_rintf(c) & 255u) << 16) | ((uint32_t)(int)__builtin_rintf(d) << 24);
    }
}
template <int FMT>
__device__ __forceinline__ float code_value(uint32_t word, int byte) {
    if constexpr (FMT == FLAT_CACHE8_E4M3) {
        const auto x = __builtin_amdgcn_cvt_pk_f32_fp8((int)(word >> (8 * byte)), false);
        return x[0];
    } else {
        return (float)(int8_t)(word >> (8 * byte));
    }
}

// Least power of two s >= 2^-100 with |x| <= M s for the magnitude whose bf16 bits are given; 0 for 0.
template <int FMT>
__device__ __forceinline__ float least_scale(uint32_t bf16_bits) {
    const uint32_t bits = bf16_bits << 16;
    const int exponent = (int)(bits >> 23) - 126 - (FMT == FLAT_CACHE8_E4M3 ? 9 : 7);  // M = 0.875 * 2^9, 0.9921875 * 2^7
    const bool above = (bits & 0x7fffffu) > (FMT == FLAT_CACHE8_E4M3 ? 0x600000u : 0x7e0000u);
    const int e = max(exponent + (above ? 1 : 0), -100);
    return bits ? __builtin_bit_cast(float, (uint32_t)(e + 127) << 23) : 0.f;
}

__device__ __forceinline__ uint32_t wave_max_bits(uint32_t x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, o));
    return x;
}

// The scale of the block and what its values are multiplied by (0: its codes are 0).
template <int FMT>
__device__ __forceinline__ void settle_scale(uint32_t largest, float before, float* scale, float* by) {
    float s = __builtin_fmaxf(least_scale<FMT>(largest), before);
    if (largest >= 0x7f80u || before != before) s = __builtin_nanf("");
    *scale = s;
    *by = s > 0.f ? 1.0f / s : 0.f;
}

template <int D, int FMT>
__global__ __launch_bounds__(64 * kWaves) void cache8_write_kernel(const WriteArgs a) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * kWaves + (threadIdx.x >> 6)));
    if (wave >= a.waves) return;
    // wave = ((entry * blocks + block) * heads + head) * 2 + (K, V)
    const int is_v = wave & 1, eb = a.by_heads.quotient(wave >> 1), head = (wave >> 1) - eb * a.heads;
    const int b = a.by_blocks.quotient(eb), j = eb - b * a.blocks;
    const int start = min(max(a.lens[b], 0), a.max_tokens);
    int n = a.n_new ? min(max(a.n_new[b], 0), a.N) : a.N;
    n = min(n, a.max_tokens - start);
    const int blk = start / kCacheBlock + j, tok0 = blk * kCacheBlock;
    if (n <= 0 || blk > (start + n - 1) / kCacheBlock) return;  // (by blocks: the last token numbers that N could reach may lie beyond 2^31)
    const int page = a.page_table[(size_t)b * a.max_pages + a.by_page_blocks.quotient(blk)];
    if ((unsigned)page >= (unsigned)a.n_pages) return;
    const int e = (page * a.heads + head) * a.page_blocks + blk - a.by_page_blocks.quotient(blk) * a.page_blocks;
    const int kept = max(start - tok0, 0), end = min(start + n - tok0, kCacheBlock);  // tokens kept .. end - 1 of the block are new
    const bf16* src = (is_v ? a.V : a.K) + ((size_t)b * a.heads + head) * a.N * D;
    const int row0 = tok0 - start;  // row of token 0 of the block
    uint8_t* codes = (is_v ? a.v : a.k) + (size_t)e * (16 * D);
    float* scales = (is_v ? a.vs : a.ks) + e;
    const float before = kept ? *scales : 0.f;

    if (!is_v) {
        constexpr int PIECES = (D + 63) / 64;  // of 16 channels of a token, per lane
        uint4v x[PIECES][2], old[PIECES], out[PIECES];
        uint32_t largest = 0;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int p = lane + 64 * i, tok = p & 15, ch = (p >> 4) * 16;
            x[i][0] = x[i][1] = old[i] = uint4v{0, 0, 0, 0};
            if (p < D && tok >= kept && tok < end) {
                const uint4v* s = (const uint4v*)(src + (size_t)(row0 + tok) * D + ch);
                x[i][0] = s[0];
                x[i][1] = s[1];
            }
            if (p < D && tok < kept) old[i] = *(const uint4v*)(codes + 16 * p);
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int q = 0; q < 4; ++q) largest = max(largest, max(x[i][h][q] & 0x7fffu, (x[i][h][q] >> 16) & 0x7fffu));
        largest = wave_max_bits(largest);
        float scale, by;
        settle_scale<FMT>(largest, before, &scale, &by);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int p = lane + 64 * i, tok = p & 15;
            float y[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const uint32_t w = x[i][q >> 3][(q >> 1) & 3];
                const float f = __builtin_bit_cast(float, q & 1 ? w & 0xffff0000u : w << 16);
                y[q] = tok < kept ? code_value<FMT>(old[i][q >> 2], q & 3) * before * by : f * by;
                y[q] = by > 0.f ? y[q] : 0.f;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) out[i][q] = to_codes<FMT>(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
            if (p < D) *(uint4v*)(codes + 16 * p) = out[i];
        }
        if (lane == 0) *scales = scale;
    } else {
        constexpr int C = D == 256 ? 4 : D >= 96 ? 2 : 1;  // channels of a lane
        typedef uint16_t __attribute__((ext_vector_type(C == 1 ? 2 : C))) chan_t;
        const int ch = lane * C;
        const bool mine = ch < D;
        uint16_t x[16][C];
        uint4v old[C];
        uint32_t largest = 0;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
#pragma unroll
            for (int c = 0; c < C; ++c) x[t][c] = 0;
            if (mine && t >= kept && t < end) {
                const bf16* s = src + (size_t)(row0 + t) * D + ch;
                if constexpr (C == 1) {
                    x[t][0] = *(const uint16_t*)s;
                } else {
                    const chan_t v = *(const chan_t*)s;
#pragma unroll
                    for (int c = 0; c < C; ++c) x[t][c] = v[c];
                }
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            old[c] = uint4v{0, 0, 0, 0};
            if (mine && kept) old[c] = *(const uint4v*)(codes + 16 * (ch + c));
        }
#pragma unroll
        for (int t = 0; t < 16; ++t)
#pragma unroll
            for (int c = 0; c < C; ++c) largest = max(largest, (uint32_t)x[t][c] & 0x7fffu);
        largest = wave_max_bits(largest);
        float scale, by;
        settle_scale<FMT>(largest, before, &scale, &by);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float y[16];
#pragma unroll
            for (int t = 0; t < 16; ++t) {
                const float f = __builtin_bit_cast(float, (uint32_t)x[t][c] << 16);
                y[t] = t < kept ? code_value<FMT>(old[c][t >> 2], t & 3) * before * by : f * by;
                y[t] = by > 0.f ? y[t] : 0.f;
            }
            uint4v out;
#pragma unroll
            for (int q = 0; q < 4; ++q) out[q] = to_codes<FMT>(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
            if (mine) *(uint4v*)(codes + 16 * (ch + c)) = out;
        }
        if (lane == 0) *scales = scale;
    }
}

template <int D>
hipError_t launch(const WriteArgs& a, int format, hipStream_t stream) {
    const unsigned grid = ((unsigned)a.waves + kWaves - 1) / kWaves;
    if (format == FLAT_CACHE8_E4M3) hipLaunchKernelGGL((cache8_write_kernel<D, FLAT_CACHE8_E4M3>), dim3(grid), dim3(64 * kWaves), 0, stream, a);
    else hipLaunchKernelGGL((cache8_write_kernel<D, FLAT_CACHE8_INT8>), dim3(grid), dim3(64 * kWaves), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache8_write(const flat_cache8& c, const CacheWrite& w, hipStream_t stream) {
    const int blocks = cache8_write_blocks(w.N);
    const WriteArgs a{(uint8_t*)c.k, (uint8_t*)c.v, c.k_scale, c.v_scale, (const bf16*)w.K, (const bf16*)w.V, w.page_table, w.lens, w.n_new, c.n_pages, c.n_heads,
                      c.page_tokens / kCacheBlock, w.max_pages, w.max_pages * c.page_tokens, w.N, blocks, w.B * blocks * c.n_heads * 2, Divisor(c.n_heads), Divisor(blocks),
                      Divisor(c.page_tokens / kCacheBlock)};
    switch (c.d) {
        case 32: return launch<32>(a, c.format, stream);
        case 64: return launch<64>(a, c.format, stream);
        case 96: return launch<96>(a, c.format, stream);
        case 128: return launch<128>(a, c.format, stream);
        case 256: return launch<256>(a, c.format, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace flat
