// Attention over the paged 8-bit cache.  See flat_cache8.hpp for the layout that this rests on.
//
// Few rows.  A workgroup has up to 32 of the Nq * group rows that share a head of the cache, and its four wavefronts take the unit's
// tiles of 32 keys in turn.  A tile is S^T = K Q^T and O^T += V^T P^T on the 32 x 32 x 16 bf16 MFMAs, with K and V widened from their codes in
// registers: no LDS in the loop, no barrier.  Row m of the K operand is block (m / 4) % 2, token 4 (m / 8) + m % 4, so that the accumulator of a
// lane in wave half h holds the 16 tokens of block h in order: exactly the contraction order in which the same half holds V's bytes.  The
// probabilities go from one MFMA to the other without leaving their lane, and a lane needs the scales of one block only.
#include "flat_cache8_fwd.hpp"

namespace flat {

namespace {

constexpr int kWaves = 4;
constexpr int kRescaleAbove = 8;  // log2: the reference maximum rises only when a logit is this far above it

// What a wavefront knows of the next 32 tiles it takes: lane l has block l % 2 of the (l / 2)-th of them.
struct BlockInfo {
    int e;         // block number in the pool, -1 a hole
    float ks, vs;  // its scales; 0 for a hole
};

template <int D, int FMT>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) void cache8_few_rows_kernel(const Cache8Args a) {
    constexpr int J = D / 32;        // 16-byte pieces of a K row per wave half, and 32-channel groups of V
    constexpr int RS = D + 4;        // row stride of the merge buffer, floats: spreads the rows over the banks
    extern __shared__ __align__(16) float lds[];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, col = lane & 31;
    const int id = blockIdx.x, u = a.by_heads.quotient(id), kvh = id - u * a.heads;

    const int chunk = cache_chunk(a, lane);
    CacheUnit unit{u, u, 1};
    if (a.target) unit = cache_find_unit(a, u, chunk, lane);
    if (unit.entry < 0) return;
    CacheEntry t = cache_entry(a, unit.entry);
    if (t.row0 >= t.rows) return;
    const int part = u - unit.before;
    const int share = (unsigned)t.tiles / (unsigned)unit.n, more = t.tiles - share * unit.n;  // the first `more` parts have one tile more
    const int tile0 = part * share + min(part, more), tile1 = tile0 + share + (part < more ? 1 : 0);

    // the rows: row = position * group + query head of the group
    const int row = t.row0 + col, pos = a.by_group.quotient(row), g = row - pos * a.group;
    const bool has_row = row < t.rows;
    const size_t q_at = ((size_t)(t.b * (size_t)a.H + kvh * a.group + g) * a.Nq + pos) * D;
    bf16x8 q[2 * J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            q[2 * j + i] = bf16x8{};
            if (has_row) q[2 * j + i] = *(const bf16x8*)(a.Q + q_at + 32 * j + 16 * half + 8 * i);
        }
    }
    const int seen = !has_row ? t.len : a.causal ? min(max(pos + 1 + t.len - t.q_len, 0), t.len) : t.len;  // keys that this row sees
    const int all_see = a.causal ? min(max(a.by_group.quotient(t.row0) + 1 + t.len - t.q_len, 0), t.len) : t.len;

    const int blocks = (t.len + kCacheBlock - 1) / kCacheBlock;
    const int* table = a.page_table + (size_t)t.b * a.max_pages;
    const int first = tile0 + w;  // tiles first, first + kWaves, ...
    auto page_of = [&](int group) __attribute__((always_inline)) {  // page of this lane's block in the group-th 32 tiles, -1 a hole
        const int blk = 2 * (first + kWaves * (32 * group + (lane >> 1))) + (lane & 1);
        return blk < blocks ? table[a.by_page_blocks.quotient(blk)] : -1;
    };
    auto info_of = [&](int group, int page) __attribute__((always_inline)) {
        const int blk = 2 * (first + kWaves * (32 * group + (lane >> 1))) + (lane & 1);
        BlockInfo x{-1, 0.f, 0.f};
        if (blk < blocks && (unsigned)page < (unsigned)a.n_pages) {
            x.e = (page * a.heads + kvh) * a.page_blocks + blk - a.by_page_blocks.quotient(blk) * a.page_blocks;
            x.ks = a.ks[x.e] * a.scale_log2;
            x.vs = a.vs[x.e];
        }
        return x;
    };

    const uint32_t k_lane = (4 * (col >> 3) + (col & 3)) * 16 + half * 256, v_lane = col * 16;
    const bool k_second = (col >> 2) & 1;
    uint4v kc[J], vc[J], kn[J], vn[J];
    auto load = [&](const BlockInfo& x, int at, uint4v* k, uint4v* v) __attribute__((always_inline)) {
        const int e0 = max(__builtin_amdgcn_readlane(x.e, 2 * at), 0), e1 = max(__builtin_amdgcn_readlane(x.e, 2 * at + 1), 0);
        const size_t at0 = (size_t)e0 * (16 * D), at1 = (size_t)e1 * (16 * D);
        const uint8_t* kp = a.k + (k_second ? at1 : at0) + k_lane;
        const uint8_t* vp = a.v + (half ? at1 : at0) + v_lane;
#pragma unroll
        for (int j = 0; j < J; ++j) k[j] = *(const uint4v*)(kp + 512 * j);
#pragma unroll
        for (int j = 0; j < J; ++j) v[j] = *(const uint4v*)(vp + 512 * j);
    };

    floatx16 o[J];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[j][r] = 0.f;
    float m = -INFINITY, msub = 0.f, l = 0.f;  // reference maximum (log2 units), what is subtracted (0 until there is a maximum), row sum of this half

    const int n_mine = first < tile1 ? (tile1 - first + kWaves - 1) / kWaves : 0;
    BlockInfo now{-1, 0.f, 0.f}, next{-1, 0.f, 0.f};
    int next_page = -1;
    if (n_mine > 0) {
        now = info_of(0, page_of(0));
        load(now, 0, kc, vc);
    }
    for (int i = 0; i < n_mine; ++i) {
        const int at = i & 31;
        // pages and scales of the next 32 tiles: fetched over this 32, so that their two round trips are not waited for
        if (at == 0 && i + 32 < n_mine) next_page = page_of((i >> 5) + 1);
        if (at == 16 && i + 16 < n_mine) next = info_of((i >> 5) + 1, next_page);
        const int s0 = 2 * at, s1 = 2 * at + 1;
        const int e0 = __builtin_amdgcn_readlane(now.e, s0), e1 = __builtin_amdgcn_readlane(now.e, s1);
        const int ks0 = __builtin_amdgcn_readlane(__builtin_bit_cast(int, now.ks), s0), ks1 = __builtin_amdgcn_readlane(__builtin_bit_cast(int, now.ks), s1);
        const int vs0 = __builtin_amdgcn_readlane(__builtin_bit_cast(int, now.vs), s0), vs1 = __builtin_amdgcn_readlane(__builtin_bit_cast(int, now.vs), s1);
        const float ks = __builtin_bit_cast(float, half ? ks1 : ks0), vs = __builtin_bit_cast(float, half ? vs1 : vs0);
        if (at == 31) now = next;
        if (i + 1 < n_mine) load(now, (i + 1) & 31, kn, vn);

        floatx16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            s = mfma_bf16_32x32x16(codes_to_bf16<FMT>(kc[j][0], kc[j][1]), q[2 * j], s);
            s = mfma_bf16_32x32x16(codes_to_bf16<FMT>(kc[j][2], kc[j][3]), q[2 * j + 1], s);
        }
        const int key0 = (first + kWaves * i) * kCacheTile;
        float c = ks;
        int visible = 16;  // of this lane's block, for its row
        const bool edge = key0 + kCacheTile > all_see || (e0 | e1) < 0;
        if (edge) {
            const int e = half ? e1 : e0;
            visible = e < 0 ? 0 : min(max(seen - key0 - kCacheBlock * half, 0), 16);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = r < visible ? s[r] * c : -INFINITY;
            c = 1.f;
            const int there = e < 0 ? 0 : min(max(t.len - key0 - kCacheBlock * half, 0), 16);
#pragma unroll
            for (int j = 0; j < J; ++j) vc[j] = clear_behind(vc[j], there);
        }
        float top = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = __builtin_fmaxf(top, s[r]);
        top = halves_max(top * c);
        if (__any(top > m + kRescaleAbove)) {
            const float up = __builtin_fmaxf(m, top), sub = up == -INFINITY ? 0.f : up;
            const float f = __builtin_amdgcn_exp2f(msub - sub);
            const float by = m == -INFINITY ? 0.f : f;
            l *= by;
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[j][r] *= by;
            m = up;
            msub = sub;
        }
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -msub));
            l += p[r];
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] *= vs;
        if (edge) {  // a block whose scale is NaN is one only for the rows that see it
#pragma unroll
            for (int r = 0; r < 16; ++r) p[r] = r < visible ? p[r] : 0.f;
        }
        uint4v plo, phi;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            plo[r] = pack_bf16(p[2 * r], p[2 * r + 1]);
            phi[r] = pack_bf16(p[8 + 2 * r], p[9 + 2 * r]);
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            o[j] = mfma_bf16_32x32x16(codes_to_bf16<FMT>(vc[j][0], vc[j][1]), __builtin_bit_cast(bf16x8, plo), o[j]);
            o[j] = mfma_bf16_32x32x16(codes_to_bf16<FMT>(vc[j][2], vc[j][3]), __builtin_bit_cast(bf16x8, phi), o[j]);
        }
#pragma unroll
        for (int j = 0; j < J; ++j) kc[j] = kn[j], vc[j] = vn[j];
    }
    l = halves_sum(l);

    // the four wavefronts' parts: every one scales its own to the common maximum, then a quarter of the columns is added up by each
    float* stat = lds + kWaves * 32 * RS;  // [kWaves][2][32]
    if (half == 0) {
        stat[w * 64 + col] = m;
        stat[w * 64 + 32 + col] = l;
    }
    __syncthreads();
    float top = -INFINITY, L = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = __builtin_fmaxf(top, stat[i * 64 + col]);
    const float sub = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        const float mi = stat[i * 64 + col], li = stat[i * 64 + 32 + col];
        L += mi == -INFINITY ? li : li * __builtin_amdgcn_exp2f(mi - sub);  // a part that saw no key has l = 0
    }
    const float mine = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - sub);
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            floatx4 y;
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = o[j][4 * x + r] * mine;
            *(floatx4*)(lds + (w * 32 + col) * RS + 32 * j + 8 * x + 4 * half) = y;
        }
    __syncthreads();
    constexpr int Q4 = D / 4;  // 16-byte groups of columns per row
    const int rows = min(t.rows - t.row0, 32);
    if (unit.n == 1) {
        for (int x = tid; x < rows * Q4; x += 64 * kWaves) {
            const int r = x / Q4, c4 = x - r * Q4;
            floatx4 y = *(const floatx4*)(lds + r * RS + 4 * c4);
#pragma unroll
            for (int i = 1; i < kWaves; ++i) y += *(const floatx4*)(lds + (i * 32 + r) * RS + 4 * c4);
            float Lr = 0.f, tr = -INFINITY;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) tr = __builtin_fmaxf(tr, stat[i * 64 + r]);
            const float sr = tr == -INFINITY ? 0.f : tr;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                const float mi = stat[i * 64 + r], li = stat[i * 64 + 32 + r];
                Lr += mi == -INFINITY ? li : li * __builtin_amdgcn_exp2f(mi - sr);
            }
            const float inv = Lr == 0.f ? 0.f : 1.0f / Lr;
            const int rr = t.row0 + r, p = a.by_group.quotient(rr), gg = rr - p * a.group;
            floatx2 out;
            out[0] = __builtin_bit_cast(float, pack_bf16(y[0] * inv, y[1] * inv));
            out[1] = __builtin_bit_cast(float, pack_bf16(y[2] * inv, y[3] * inv));
            *(floatx2*)(a.O + ((size_t)(t.b * (size_t)a.H + kvh * a.group + gg) * a.Nq + p) * D + 4 * c4) = out;
        }
    } else {
        float* part_ws = a.ws + (size_t)(u * (size_t)a.heads + kvh) * (32 * (D + 2));
        for (int x = tid; x < rows * Q4; x += 64 * kWaves) {
            const int r = x / Q4, c4 = x - r * Q4;
            floatx4 y = *(const floatx4*)(lds + r * RS + 4 * c4);
#pragma unroll
            for (int i = 1; i < kWaves; ++i) y += *(const floatx4*)(lds + (i * 32 + r) * RS + 4 * c4);
            *(floatx4*)(part_ws + r * D + 4 * c4) = y;
        }
        if (w == 0 && half == 0 && col < rows) {
            part_ws[32 * D + col] = top;
            part_ws[32 * D + 32 + col] = L;
        }
    }
}

// Puts the parts of the rows together whose entry was divided: one workgroup per row of Q.
constexpr int kMergeThreads = 256;
template <int D>
__global__ __launch_bounds__(kMergeThreads) void cache8_merge_kernel(const Cache8Args a, const Divisor by_rows, int rows_per_b) {
    constexpr int Q4 = D / 4, LANES = kMergeThreads / Q4;
    __shared__ floatx4 red[kMergeThreads];
    __shared__ float wts[kMergeThreads], stat[2][kMergeThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63;
    // blockIdx = (b * heads + head of the cache) * rows_per_b + row
    const int bh = by_rows.quotient(blockIdx.x), row = blockIdx.x - bh * rows_per_b;
    const int b = a.by_heads.quotient(bh), kvh = bh - b * a.heads;
    const int rb = row / 32, e = b * a.row_blocks + rb, r = row - 32 * rb;
    const int chunk = cache_chunk(a, lane);
    const CacheEntry t = cache_entry(a, e);
    if (row >= t.rows) return;
    const CacheUnit unit = cache_units_of(a, e, chunk, lane);
    if (unit.n == 1) return;
    const size_t stride = (size_t)a.heads * (32 * (D + 2));
    const float* base = a.ws + ((size_t)unit.before * a.heads + kvh) * (32 * (D + 2));
    const int c4 = tid % Q4, first = tid / Q4;

    float top = -INFINITY;
    for (int s = tid; s < unit.n; s += kMergeThreads) top = __builtin_fmaxf(top, base[s * stride + 32 * D + r]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) stat[0][tid >> 6] = top;
    __syncthreads();
    top = __builtin_fmaxf(__builtin_fmaxf(stat[0][0], stat[0][1]), __builtin_fmaxf(stat[0][2], stat[0][3]));
    const float sub = top == -INFINITY ? 0.f : top;

    floatx4 acc{0.f, 0.f, 0.f, 0.f};
    float L = 0.f;
    for (int s0 = 0; s0 < unit.n; s0 += kMergeThreads) {
        if (s0 + tid < unit.n) {
            const float* p = base + (s0 + tid) * stride;
            const float ms = p[32 * D + r], ls = p[32 * D + 32 + r];
            const float wt = ms == -INFINITY ? (ls == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(ms - sub);  // no key seen: nothing; a NaN stays one
            wts[tid] = wt;
            L += wt * ls;
        }
        __syncthreads();
        const int n = min(unit.n - s0, kMergeThreads);
        if (first < LANES) {
#pragma unroll 4
            for (int s = first; s < n; s += LANES) {
                const floatx4 y = *(const floatx4*)(base + (s0 + s) * stride + r * D + 4 * c4);
                const float wt = wts[s];
                if (wt != 0.f) acc += y * wt;
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) L += __shfl_xor(L, o);
    if (lane == 0) stat[1][tid >> 6] = L;
    red[tid] = acc;
    __syncthreads();
    if (tid >= Q4) return;
    L = (stat[1][0] + stat[1][1]) + (stat[1][2] + stat[1][3]);
    for (int k = 1; k < LANES; ++k) acc += red[k * Q4 + c4];
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    const int p = a.by_group.quotient(row), g = row - p * a.group;
    floatx2 out;
    out[0] = __builtin_bit_cast(float, pack_bf16(acc[0] * inv, acc[1] * inv));
    out[1] = __builtin_bit_cast(float, pack_bf16(acc[2] * inv, acc[3] * inv));
    *(floatx2*)(a.O + ((size_t)(b * (size_t)a.H + kvh * a.group + g) * a.Nq + p) * D + 4 * c4) = out;
}

template <int D, int FMT>
hipError_t launch(const Cache8Args& args, const Cache8Plan& plan, hipStream_t stream) {
    static std::atomic<uint64_t> lds_allowed{0};
    constexpr int lds = (kWaves * 32 * (D + 4) + kWaves * 64) * (int)sizeof(float);
    hipError_t e = allow_dynamic_lds((const void*)cache8_few_rows_kernel<D, FMT>, lds, &lds_allowed);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((cache8_few_rows_kernel<D, FMT>), dim3((unsigned)plan.max_units * (unsigned)args.heads), dim3(64 * kWaves), lds, stream, args);
    e = hipGetLastError();
    if (e != hipSuccess || plan.target == 0) return e;
    const int rows = args.Nq * args.group;
    hipLaunchKernelGGL((cache8_merge_kernel<D>), dim3((unsigned)(args.B * args.heads) * (unsigned)rows), dim3(kMergeThreads), 0, stream, args, Divisor(rows), rows);
    return hipGetLastError();
}

template <int D>
hipError_t launch(const Cache8Args& args, int format, const Cache8Plan& plan, hipStream_t stream) {
    return format == FLAT_CACHE8_E4M3 ? launch<D, FLAT_CACHE8_E4M3>(args, plan, stream) : launch<D, FLAT_CACHE8_INT8>(args, plan, stream);
}

}  // namespace

hipError_t launch_cache8_fwd(const flat_cache8& c, const Cache8Attend& a, const Cache8Plan& plan, hipStream_t stream) {
    Cache8Args args{(const uint8_t*)c.k, (const uint8_t*)c.v, c.k_scale, c.v_scale, (const bf16*)a.Q, (bf16*)a.O, a.page_table, a.lens, a.q_lens,
                    a.workspace, c.n_pages, c.n_heads, a.max_pages, a.max_pages * c.page_tokens, a.B, a.H, a.Nq, a.H / c.n_heads, a.scale * kLog2e, a.causal,
                    plan.rows_per_block, plan.row_blocks, plan.entries, plan.target, plan.least_tiles, Divisor(c.n_heads), Divisor(a.H / c.n_heads),
                    Divisor(plan.row_blocks), Divisor(c.page_tokens / kCacheBlock), c.page_tokens / kCacheBlock};
    switch (c.d) {
        case 32: return launch<32>(args, c.format, plan, stream);
        case 64: return launch<64>(args, c.format, plan, stream);
        case 96: return launch<96>(args, c.format, plan, stream);
        case 128: return launch<128>(args, c.format, plan, stream);
        case 256: return launch<256>(args, c.format, plan, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace flat
