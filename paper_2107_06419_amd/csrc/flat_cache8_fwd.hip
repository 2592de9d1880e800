// Attention over the paged 8-bit cache.  See flat_cache8.hpp for the layout that this rests on.
//
// A tile of 32 keys is S^T = K Q^T and O^T += V^T P^T on the 32 x 32 x 16 bf16 MFMAs.  Row m of the K operand is block (m / 4) % 2, token 4 (m / 8) + m % 4, so
// that the accumulator of a lane in wave half h holds the 16 tokens of block h in order: exactly the contraction order in which the same half
// holds V's bytes.  The probabilities go from one MFMA to the other without leaving their lane, and a lane needs the scales of one block only.
#include <type_traits>

#include "flat_cache8_fwd.hpp"

namespace flat {

namespace {

// Where a row of a batch entry and head of the cache lies in Q and O: row = position * group + query head of the group.
template <int D>
__device__ __forceinline__ size_t row_at(const Cache8Args& a, int b, int kvh, int row) {
    const int pos = a.by_group.quotient(row), g = row - pos * a.group;
    return ((size_t)(b * (size_t)a.H + kvh * a.group + g) * a.Nq + pos) * D;
}
// Partial results of a unit: rows_per_block rows of D, then their reference maxima, then their sums.
template <int D, int ROWS>
__device__ __forceinline__ float* part_of(const Cache8Args& a, int u, int kvh) {
    return a.parts + (size_t)(u * (size_t)a.heads + kvh) * (ROWS * (D + 2));
}
__device__ __forceinline__ floatx2 four_bf16(const floatx4& y, float by) {
    floatx2 out;
    out[0] = __builtin_bit_cast(float, pack_bf16(y[0] * by, y[1] * by));
    out[1] = __builtin_bit_cast(float, pack_bf16(y[2] * by, y[3] * by));
    return out;
}

// ---- Few rows: up to ROWS = 16 or 32 of the Nq * group rows that share a head of the cache.  The four wavefronts of a workgroup take the unit's steps
// of TPS tiles in turn, with K and V widened from their codes in registers: no LDS and no barrier before the end.  What bounds it is the reading of the
// codes, and where few workgroups run the instructions of a wavefront: a wavefront asks for the next codes as soon as it has widened these.
//
// A tile is 64 / ROWS blocks: 32 keys on the 32 x 32 x 16 MFMA, 64 keys on the 16 x 16 x 32 one, four products of 16 keys each.  With 16 rows the tokens of
// K's operand are dealt out likewise, row m of product t is block m / 4, token 4 t + m % 4, and a lane again ends up with the 16 tokens of one block.  The lanes'
// work per key is half that of 32 rows: 16 workgroups over 4096 keys, 32 rows -> 16, d = 64 18.9 -> 14.8 us, d = 128 26.8 -> 20.1.
constexpr int NW = 4;  // wavefronts of a workgroup, here and in the kernel of many rows at d = 256

// DIVIDED: the entries' keys are divided over units; else a unit is an entry, and its page ids are fetched along with its lengths.
template <int D, int ROWS, int FMT, bool DIVIDED>
__global__ __launch_bounds__(64 * NW, D == 256 ? 1 : 2) void cache8_few_rows_kernel(const Cache8Args a, int lds_rows) {
    constexpr int LG = 64 / ROWS;                                 // lane groups: each has one block of a tile
    constexpr int NQ = D / (16 * LG);                             // contraction pieces of a row, 16 channels per lane group
    constexpr int KL = ROWS == 32 ? NQ : 4 * NQ, VL = D / ROWS;   // 16-byte loads of K and V per lane and tile
    constexpr int TPS = cache8_step_keys(ROWS, D) / (16 * LG), BPS = LG * TPS, GROUP = 64 / BPS;  // tiles and blocks of a step; steps whose blocks 64 lanes know
    constexpr int RS = D + 4;                                     // row stride of the merge buffer, floats: spreads the rows over the banks
    typedef std::conditional_t<ROWS == 32, floatx16, floatx4> acc_t;
    constexpr int AR = ROWS == 32 ? 16 : 4;                       // its registers
    extern __shared__ __align__(16) float lds[];  // [NW][lds_rows][RS], then statistics
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = lane / ROWS, col = lane % ROWS;
    const int id = blockIdx.x, u = a.by_heads.quotient(id), kvh = id - u * a.heads;

    CacheUnit unit;
    int step0 = 0, page0 = -1;
    if (DIVIDED) {
        unit = cache_find_unit(a, u, lane);
        if (unit.e < 0) return;
    } else {
        const int at = a.by_page_blocks.quotient(BPS * (w + NW * (lane / BPS)) + lane % BPS);
        if (at < a.max_pages) page0 = a.page_table[(size_t)a.by_row_blocks.quotient(u) * a.max_pages + at];
        unit.entry = cache_entry(a, u);
        unit.e = unit.before = u;
        unit.n = 1;
    }
    const CacheEntry& t = unit.entry;
    if (t.row0 >= t.rows) return;
    int step1 = t.tiles;
    if (DIVIDED) cache_part(t.tiles, u - unit.before, unit.n, &step0, &step1);

    // blocks of the wavefront's steps first, first + NW, ...
    const int* table = a.page_table + (size_t)t.b * a.max_pages;
    const int first = step0 + w, n_mine = first < step1 ? (step1 - first + NW - 1) / NW : 0;
    const int my_block = BPS * (first + NW * (lane / BPS)) + lane % BPS;  // of this lane in the first group
    auto page_of = [&](int group) __attribute__((always_inline)) {
        const int blk = my_block + group * (BPS * NW * GROUP);
        return kCacheBlock * blk < t.len ? table[a.by_page_blocks.quotient(blk)] : -1;
    };
    auto block_of = [&](int group, int page) __attribute__((always_inline)) {
        return cache_block(a, kvh, t.len, my_block + group * (BPS * NW * GROUP), page);
    };
    if (DIVIDED && n_mine) page0 = page_of(0);

    const int row = t.row0 + col, pos = a.by_group.quotient(row);
    const bool has_row = row < t.rows;
    bf16x8 q[2 * NQ];
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            q[2 * j + i] = bf16x8{};
            if (has_row) q[2 * j + i] = *(const bf16x8*)(a.Q + row_at<D>(a, t.b, kvh, row) + 16 * (LG * j + grp) + 8 * i);
        }
    }
    const int seen = !has_row ? t.len : a.causal ? min(max(pos + 1 + t.len - t.q_len, 0), t.len) : t.len;  // keys that this row sees
    const int all_see = __builtin_amdgcn_readfirstlane(a.causal ? min(max(a.by_group.quotient(t.row0) + 1 + t.len - t.q_len, 0), t.len) : t.len);

    CacheBlock now = block_of(0, page0), next = now;
    int next_page = -1;
    int now_at = max(now.e, 0);  // of the group that the next loads are for; holes read block 0, and what they read counts for nothing
    uint64_t lacking = __ballot(now.there < 16);  // blocks of the group of which a token or more is not there
    // the lane's place in a block, and which block of the tile: K as the A operand's rows, V by lane group
    const int k_block = ROWS == 32 ? (col >> 2) & 1 : col >> 2;
    const uint8_t *k_lane = a.k + (ROWS == 32 ? 4 * (col >> 3) + (col & 3) : col & 3) * 16 + grp * 256, *v_lane = a.v + col * 16;
    uint4v kc[TPS][KL], vc[TPS][VL];
    auto block_at = [&](int i, int t2, int block) __attribute__((always_inline)) {
        return (uint64_t)(uint32_t)__builtin_amdgcn_ds_bpermute(4 * (BPS * (i % GROUP) + LG * t2 + block), now_at) * (16 * D);
    };
    auto load_k = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int t2 = 0; t2 < TPS; ++t2) {
            const uint8_t* p = k_lane + block_at(i, t2, k_block);
#pragma unroll
            for (int x = 0; x < KL; ++x) kc[t2][x] = *(const uint4v*)(p + (ROWS == 32 ? 512 * x : 1024 * (x / 4) + 64 * (x % 4)));
        }
    };
    auto load_v = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int t2 = 0; t2 < TPS; ++t2) {
            const uint8_t* p = v_lane + block_at(i, t2, grp);
#pragma unroll
            for (int x = 0; x < VL; ++x) vc[t2][x] = *(const uint4v*)(p + 16 * ROWS * x);
        }
    };

    acc_t o[VL];
#pragma unroll
    for (int j = 0; j < VL; ++j)
#pragma unroll
        for (int r = 0; r < AR; ++r) o[j][r] = 0.f;
    RowState st{-INFINITY, 0.f, 0.f};

    if (n_mine > 0) {
        load_k(0);
        load_v(0);
    }
    auto step = [&](int i) __attribute__((always_inline)) {  // (as the loop's own body it came out a tenth slower, by the order the compiler gives it)
        const int at = i % GROUP;
        // pages and scales of the next GROUP steps: fetched over these, so that their two round trips are not waited for
        if (at == 0 && i + GROUP < n_mine) next_page = page_of(i / GROUP + 1);
        if (at == GROUP / 2 && i + GROUP - GROUP / 2 < n_mine) next = block_of(i / GROUP + 1, next_page);
        float c[TPS], vs_log2[TPS], vs_inv[TPS];
#pragma unroll
        for (int t2 = 0; t2 < TPS; ++t2) {
            const int from = 4 * (BPS * at + LG * t2 + grp);
            c[t2] = value_of_lane(from, now.ks);
            vs_log2[t2] = value_of_lane(from, now.vs_log2);
            vs_inv[t2] = value_of_lane(from, now.vs_inv);
        }
        const int key0 = (first + NW * i) * (16 * BPS);
        const bool edge = key0 + 16 * BPS > all_see || ((lacking >> (BPS * at)) & ((1ull << BPS) - 1)) != 0;
        int there[TPS], hole[TPS];
        if (edge) {
#pragma unroll
            for (int t2 = 0; t2 < TPS; ++t2) {
                const int from = 4 * (BPS * at + LG * t2 + grp);
                there[t2] = __builtin_amdgcn_ds_bpermute(from, now.there);
                hole[t2] = __builtin_amdgcn_ds_bpermute(from, now.e);
            }
        }
        if (at == GROUP - 1) {
            now = next;
            lacking = __ballot(now.there < 16);
        }
        now_at = at == GROUP - 1 ? max(next.e, 0) : now_at;

        float s[TPS][16];  // logits of the lane's row and block, token by token
        int visible[TPS];
        float top = -INFINITY;
#pragma unroll
        for (int t2 = 0; t2 < TPS; ++t2) {
#pragma unroll
            for (int y = 0; y < KL / NQ; ++y) {
                acc_t z;
#pragma unroll
                for (int r = 0; r < AR; ++r) z[r] = 0.f;
#pragma unroll
                for (int j = 0; j < NQ; ++j) {
                    const uint4v k = kc[t2][KL / NQ * j + y];
                    if constexpr (ROWS == 32) {
                        z = mfma_bf16_32x32x16(codes_to_bf16<FMT>(k[0], k[1]), q[2 * j], z);
                        z = mfma_bf16_32x32x16(codes_to_bf16<FMT>(k[2], k[3]), q[2 * j + 1], z);
                    } else {
                        z = mfma_bf16_16x16x32(codes_to_bf16<FMT>(k[0], k[1]), q[2 * j], z);
                        z = mfma_bf16_16x16x32(codes_to_bf16<FMT>(k[2], k[3]), q[2 * j + 1], z);
                    }
                    if (FMT == FLAT_CACHE8_INT8) __builtin_amdgcn_sched_barrier(0);  // the widening takes registers: not all of it at once
                }
#pragma unroll
                for (int r = 0; r < AR; ++r) s[t2][AR * y + r] = z[r];
            }
        }
        // K's registers are free: the next step's codes into them, and V's below.  Never skipped (behind the last step, the last one's once more): if they
        // could be, the compiler would not count on them being on their way, and wait for more than it needs.  (Two steps ahead instead of one: no faster at
        // 16 workgroups, slower at 1024 by what short walks fetch in vain, 128 keys, d = 64, 5.7 -> 7.5 us.)
        load_k(min(i + 1, n_mine - 1));
#pragma unroll
        for (int t2 = 0; t2 < TPS; ++t2) {
            visible[t2] = 16;
            float most;
            if (edge) {
                visible[t2] = hole[t2] < 0 ? 0 : min(max(seen - key0 - kCacheBlock * (LG * t2 + grp), 0), 16);
#pragma unroll
                for (int j = 0; j < VL; ++j) vc[t2][j] = clear_behind(vc[t2][j], there[t2]);
                most = -INFINITY;
#pragma unroll
                for (int r = 0; r < 16; ++r) most = __builtin_fmaxf(most, r < visible[t2] ? s[t2][r] : -INFINITY);
                most = most == -INFINITY ? most : most * c[t2];  // a scale of 0 leaves nothing unseen a maximum
            } else {
                most = s[t2][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) most = __builtin_fmaxf(most, s[t2][r]);
                most *= c[t2];
            }
            top = __builtin_fmaxf(top, most);
        }
        top = row_max<ROWS>(top);
        if (__any(top > st.m + kRescaleAbove)) {
            const float up = __builtin_fmaxf(st.m, top), sub = up == -INFINITY ? 0.f : up;
            const float by = st.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.sub - sub);
            st.l *= by;
#pragma unroll
            for (int j = 0; j < VL; ++j)
#pragma unroll
                for (int r = 0; r < AR; ++r) o[j][r] *= by;
            st.m = up;
            st.sub = sub;
        }
#pragma unroll
        for (int t2 = 0; t2 < TPS; ++t2) {
            bf16x8 lo, hi;
            if (edge) tile_probabilities<true>(s[t2], c[t2], vs_log2[t2], vs_inv[t2], st.sub, visible[t2], &lo, &hi, &st.l);
            else tile_probabilities<false>(s[t2], c[t2], vs_log2[t2], vs_inv[t2], st.sub, 16, &lo, &hi, &st.l);
#pragma unroll
            for (int j = 0; j < VL; ++j) {
                const uint4v v = vc[t2][j];
                if constexpr (ROWS == 32) {
                    o[j] = mfma_bf16_32x32x16(codes_to_bf16<FMT>(v[0], v[1]), lo, o[j]);
                    o[j] = mfma_bf16_32x32x16(codes_to_bf16<FMT>(v[2], v[3]), hi, o[j]);
                } else {
                    o[j] = mfma_bf16_16x16x32(codes_to_bf16<FMT>(v[0], v[1]), lo, o[j]);
                    o[j] = mfma_bf16_16x16x32(codes_to_bf16<FMT>(v[2], v[3]), hi, o[j]);
                }
                if (FMT == FLAT_CACHE8_INT8) __builtin_amdgcn_sched_barrier(0);
            }
        }
        load_v(min(i + 1, n_mine - 1));
    };
    for (int i = 0; i < n_mine; ++i) step(i);
    st.l = row_sum<ROWS>(st.l);

    // the wavefronts' parts: every one scales its own to the common maximum, then all add up
    float* stat = lds + NW * lds_rows * RS;  // [NW][2][ROWS]
    if (grp == 0) {
        stat[w * 2 * ROWS + col] = st.m;
        stat[w * 2 * ROWS + ROWS + col] = st.l;
    }
    __syncthreads();
    auto joined = [&](int r, float* top, float* sum) __attribute__((always_inline)) {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < NW; ++i) m = __builtin_fmaxf(m, stat[i * 2 * ROWS + r]);
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const float mi = stat[i * 2 * ROWS + r], li = stat[i * 2 * ROWS + ROWS + r];
            l += mi == -INFINITY ? li : li * __builtin_amdgcn_exp2f(mi - m);  // without a maximum the sum is 0, or not a number
        }
        *top = m;
        *sum = l;
    };
    float top, sum;
    joined(col, &top, &sum);
    const float mine = st.m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m - top);
    const int rows = min(t.rows - t.row0, ROWS);
    if (col < rows) {
#pragma unroll
        for (int j = 0; j < VL; ++j)
#pragma unroll
            for (int x = 0; x < AR / 4; ++x) {
                floatx4 y;
#pragma unroll
                for (int r = 0; r < 4; ++r) y[r] = o[j][4 * x + r] * mine;
                *(floatx4*)(lds + (w * lds_rows + col) * RS + ROWS * j + 8 * x + 4 * grp) = y;
            }
    }
    __syncthreads();
    constexpr int Q4 = D / 4;  // 16-byte groups of columns per row
    float* part = part_of<D, ROWS>(a, u, kvh);
    for (int x = tid; x < rows * Q4; x += 64 * NW) {
        const int r = x / Q4, c4 = x - r * Q4;
        floatx4 y = *(const floatx4*)(lds + r * RS + 4 * c4);
#pragma unroll
        for (int i = 1; i < NW; ++i) y += *(const floatx4*)(lds + (i * lds_rows + r) * RS + 4 * c4);
        if (DIVIDED && unit.n > 1) {
            *(floatx4*)(part + r * D + 4 * c4) = y;
            continue;
        }
        float m, l;
        joined(r, &m, &l);
        *(floatx2*)(a.O + row_at<D>(a, t.b, kvh, t.row0 + r) + 4 * c4) = four_bf16(y, l == 0.f ? 0.f : 1.0f / l);
    }
    if (DIVIDED && unit.n > 1 && tid < rows) {
        part[ROWS * D + tid] = top;
        part[ROWS * D + ROWS + tid] = sum;
    }
    if (DIVIDED && u == unit.before && kvh == 0 && tid == 0) a.units[unit.e] = make_int2(unit.before, unit.n);
}

// ---- Many rows: every wavefront has 32 rows of its own and takes all keys of the entry; d up to 128.  The eight wavefronts of a workgroup, two per SIMD, widen
// each tile of 64 keys once, in LDS, as the MFMA operands in the order of their lanes (1 KiB each), so that reading and writing them meets no bank twice.
//
// A step multiplies the last tile's V by its probabilities and this tile's K by Q, 4 D / 16 MFMAs in a row; while they run, the wavefront widens its share of the tile
// after the next one and asks for its share of the one behind that.  Then come the probabilities.  There are four tiles in LDS: the last one, this one, the next,
// whose first operands may be asked for, and the one being written; so one barrier per step is enough, and a wavefront's products run beside the vector work of the
// other one of its SIMD.  What bounds it is power: at d = 128 the clock falls to 1.83 GHz of 2.4 (a large matrix product of the library reaches 53 % of the peak too).
//
// The row's largest logit is not looked for in every tile: the probabilities are taken against the reference there is, and their sum, which is needed anyway, shows whether
// one of them may be above 2^8.  Only then the tile is taken again, with the maximum.  2 x 2048 queries of 16 heads over 16384 keys, d = 128: 566 us with the maximum, a
// barrier and two tiles in LDS, workgroups of 128 rows; 488 so; two groups of wavefronts in opposite phases 505, d = 64 348 against 319.
template <int D, int FMT>
__global__ __launch_bounds__(512, 2) void cache8_rows_kernel(const Cache8Args a, int blocks_per_xcd) {
    constexpr int RW = 8;                               // wavefronts
    constexpr int J = D / 32, PAIRS = 4 * J;            // pairs of operands of a tile: K of (sub-tile, j), then V
    constexpr int MINE = (PAIRS + RW - 1) / RW;         // of a wavefront: pairs w, w + RW
    constexpr int BUF = PAIRS * 2 * 1024, SLOTS = 4;    // bytes of a tile; tiles in LDS
    constexpr int GROUP = 16;                           // tiles whose blocks 64 lanes know
    constexpr int AHEAD = D == 128 ? 3 : 4;             // operands asked for ahead of their MFMA: d = 128 507 us (3) against 533 (4), d = 64 340 against 327
    extern __shared__ __align__(16) uint8_t smem[];
    float* scales = (float*)(smem + SLOTS * BUF);       // [2][64 blocks][4]: ks, vs_log2, vs_inv, tokens there as int (-1: a hole)
    int* numbers = (int*)(scales + 2 * 64 * 4);         // [2][64 blocks]: their numbers in the pool; holes read block 0, and what they read counts for nothing
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, col = lane & 31;
    // blocks of one batch entry and head follow each other on one XCD: they read the same codes.  Later rows see more keys: they go first
    const int id = xcd_logical_block(blockIdx.x, blocks_per_xcd), bh = a.by_row_blocks.quotient(id), b = a.by_heads.quotient(bh), kvh = bh - b * a.heads;
    if (b >= a.B) return;
    const CacheEntry t = cache_entry(a, b * a.row_blocks + a.row_blocks - 1 - (id - bh * a.row_blocks));
    if (t.row0 >= t.rows) return;
    const int n = t.tiles;

    const int* table = a.page_table + (size_t)t.b * a.max_pages;
    auto page_of = [&](int group) __attribute__((always_inline)) {
        const int blk = 4 * GROUP * group + lane;
        return kCacheBlock * blk < t.len ? table[a.by_page_blocks.quotient(blk)] : -1;
    };
    // tells the workgroup of a group's blocks; the result: those of which a token or more is not there
    auto blocks_of = [&](int group, int page) __attribute__((always_inline)) {
        const CacheBlock x = cache_block(a, kvh, t.len, 4 * GROUP * group + lane, page);
        if (w == 0) {
            *(floatx4*)(scales + 4 * (64 * (group & 1) + lane)) = floatx4{x.ks, x.vs_log2, x.vs_inv, __builtin_bit_cast(float, x.e < 0 ? -1 : x.there)};
            numbers[64 * (group & 1) + lane] = max(x.e, 0);
        }
        return __ballot(x.there < 16);
    };
    uint64_t lacking = blocks_of(0, page_of(0)), lacking_next = 0;  // of the group that is worked on, and of the next one
    int next_page = -1;

    const int row = t.row0 + 32 * w + col;
    const bool has_row = row < t.rows;
    bf16x8 q[2 * J];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            q[2 * j + i] = bf16x8{};
            if (has_row) q[2 * j + i] = *(const bf16x8*)(a.Q + row_at<D>(a, t.b, kvh, row) + 32 * j + 16 * half + 8 * i);
        }
    auto seen_by = [&](int r) __attribute__((always_inline)) { return a.causal ? min(max(a.by_group.quotient(r) + 1 + t.len - t.q_len, 0), t.len) : t.len; };
    const int seen = has_row ? seen_by(row) : t.len;
    const int all_see = __builtin_amdgcn_readfirstlane(seen_by(t.row0 + 32 * w));  // keys that every row of this wavefront sees

    // this wavefront's operand pairs: p = w, w + RW of [K, V][sub-tile][j]; of each the lane's place in a block, and its block of the tile
    const uint8_t* base[MINE];
    int block[MINE];
#pragma unroll
    for (int x = 0; x < MINE; ++x) {
        const int p = min(w + RW * x, PAIRS - 1), is_v = p >= 2 * J, q2 = p - (is_v ? 2 * J : 0), sub = q2 / J;
        block[x] = 2 * sub + (is_v ? half : (col >> 2) & 1);
        base[x] = (is_v ? a.v + col * 16 : a.k + (4 * (col >> 3) + (col & 3)) * 16 + half * 256) + 512 * (q2 - sub * J);
    }
    uint4v codes[MINE];
    uint32_t number[MINE];
    auto in_two_groups = [](int i) __attribute__((always_inline)) { return 4 * (i & (2 * GROUP - 1)); };  // first block of tile i
    auto find = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < MINE; ++x) number[x] = numbers[in_two_groups(i) + block[x]];
    };
    auto load = [&](int x) __attribute__((always_inline)) { codes[x] = *(const uint4v*)(base[x] + (uint64_t)number[x] * (16 * D)); };
    auto clear = [&](int i) __attribute__((always_inline)) {  // what lies behind the entry's last token, of V
#pragma unroll
        for (int x = 0; x < MINE; ++x)
            if (w + RW * x >= 2 * J) codes[x] = clear_behind(codes[x], __builtin_bit_cast(int, scales[4 * (in_two_groups(i) + block[x]) + 3]));
    };
    auto widen = [&](int i, int x, int part) __attribute__((always_inline)) {
        const int p = w + RW * x;
        if (PAIRS % RW && p >= PAIRS) return;
        *(bf16x8*)(smem + (i % SLOTS) * BUF + p * 2048 + part * 1024 + lane * 16) = codes_to_bf16<FMT>(codes[x][2 * part], codes[x][2 * part + 1]);
    };

    floatx16 o[J];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[j][r] = 0.f;
    RowState st{-INFINITY, 0.f, 0.f};
    auto raise = [&](float top) __attribute__((always_inline)) {
        const float up = __builtin_fmaxf(st.m, top), to = up == -INFINITY ? 0.f : up;
        const float by = st.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.sub - to);
        st.l *= by;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[j][r] *= by;
        st.m = up;
        st.sub = to;
    };

    // the first two tiles; the third is asked for, and the fourth known.  V of the slot before the first meets probabilities of 0: it has to be numbers
    for (int x = tid; x < BUF / 2 / 16; x += 64 * RW) *(uint4v*)(smem + (SLOTS - 1) * BUF + BUF / 2 + 16 * x) = uint4v{0, 0, 0, 0};
    __syncthreads();
    if (n > 0) {
        for (int i = 0; i < 3; ++i) {
            find(min(i, n - 1));
#pragma unroll
            for (int x = 0; x < MINE; ++x) load(x);
            if (i == 2) break;
            clear(min(i, n - 1));
#pragma unroll
            for (int x = 0; x < 2 * MINE; ++x) widen(i, x / 2, x % 2);
        }
        find(min(3, n - 1));
    }
    __syncthreads();

    // What the next group's blocks are: pages at the start of a group, the rest in its middle.  Tiles behind the last one stand for the last, or for whatever their slot
    // holds: nobody reads them.
    auto look_ahead = [&](int i) __attribute__((always_inline)) {
        const int at = i % GROUP;
        if (at == 0 && i + GROUP < n) next_page = page_of(i / GROUP + 1);
        if (at == GROUP / 2 && i + GROUP - GROUP / 2 < n) lacking_next = blocks_of(i / GROUP + 1, next_page);
    };
    auto done = [&](int i) __attribute__((always_inline)) {
        if (i % GROUP == GROUP - 1) lacking = lacking_next;
        look_ahead(i + 1);
    };
    auto lacks_after_next = [&](int i) __attribute__((always_inline)) {
        const int at = i % GROUP + 2;
        return ((at < GROUP ? lacking >> (4 * at) : lacking_next >> (4 * (at - GROUP))) & 15) != 0;
    };
    bf16x8 f[AHEAD];
    // operand x of step i: V of tile i - 1, then K of tile i
    auto fetch = [&](int i, int x) __attribute__((always_inline)) {
        const int k = x - 4 * J;
        const int at = x < 4 * J ? (2 + x / (2 * J)) * J * 2 + 2 * (x % J) + x / J % 2 : (k & 1) * 2 * J + k / 2;
        if (x < 8 * J) f[x % AHEAD] = *(const bf16x8*)(smem + ((x < 4 * J ? i + SLOTS - 1 : i) % SLOTS) * BUF + at * 1024 + lane * 16);
        __builtin_amdgcn_sched_barrier(0x616);  // MFMAs and LDS reads stay in this order: the compiler would ask for an operand just before its use
    };
    bf16x8 p[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) p[x] = bf16x8{};
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) fetch(0, x);
    if (n > 0) look_ahead(0);
    for (int i = 0; i < n;) {
        floatx16 s[2];
        floatx4 c[2];
        for (;;) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[x][r] = 0.f;
            if (lacks_after_next(i)) clear(i + 2);
            constexpr int STEP = (8 * J - 2) / (2 * MINE);
#pragma unroll
            for (int x = 0; x < 8 * J; ++x) {
                if (x < 4 * J) o[x % J] = mfma_bf16_32x32x16(f[x % AHEAD], p[x / J], o[x % J]);
                else s[x & 1] = mfma_bf16_32x32x16(f[x % AHEAD], q[(x - 4 * J) / 2], s[x & 1]);
                fetch(i, x + AHEAD);
                if (x % STEP == 1 && x / STEP < 2 * MINE) {
                    widen(i + 2, x / STEP / 2, x / STEP % 2);
                    if (x / STEP % 2) load(x / STEP / 2);
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) c[x] = *(const floatx4*)(scales + 4 * (in_two_groups(i) + 2 * x + half));
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) fetch(i + 1, x);
            find(min(i + 4, n - 1));
            // a tile that a row does not see whole, or that is not all there, and a reference that has to rise are the other path's: with the rescaling in here, the
            // compiler moves the accumulators to other registers and back in every tile
            if (64 * i + 64 > all_see || ((lacking >> (4 * (i % GROUP))) & 15) != 0) break;
            bf16x8 y[4];
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int x = 0; x < 2; ++x) tile_probabilities<false>(s[x], c[x][0], c[x][1], c[x][2], st.sub, 16, &y[2 * x], &y[2 * x + 1], &sum[x]);
            if (__any(__builtin_fmaxf(sum[0], sum[1]) > (float)(1 << kRescaleAbove) || st.m == -INFINITY)) break;
            st.l += sum[0] + sum[1];
#pragma unroll
            for (int x = 0; x < 4; ++x) p[x] = y[x];
            done(i);
            ++i;
            __builtin_amdgcn_sched_barrier(0);
            __syncthreads();
            __builtin_amdgcn_sched_barrier(0);
            if (i >= n) break;
        }
        if (i >= n) break;
        int visible[2];
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const float last = c[x][3];  // (the bits of a vector's element taken directly would be those of its first)
            visible[x] = __builtin_bit_cast(int, last) < 0 ? 0 : min(max(seen - 64 * i - 32 * x - kCacheBlock * half, 0), 16);
            float m = -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) m = __builtin_fmaxf(m, r < visible[x] ? s[x][r] : -INFINITY);
            top = __builtin_fmaxf(top, m == -INFINITY ? m : m * c[x][0]);
        }
        top = halves_max(top);
        if (__any(top > st.m + (kRescaleAbove - 4))) raise(top);  // sixteen probabilities up to 2^4 are no more than 2^8: such logits do not come here again
#pragma unroll
        for (int x = 0; x < 2; ++x) tile_probabilities<true>(s[x], c[x][0], c[x][1], c[x][2], st.sub, visible[x], &p[2 * x], &p[2 * x + 1], &st.l);
        done(i);
        ++i;
        __syncthreads();
    }
#pragma unroll
    for (int x = 0; x < 4 * J; ++x) {  // V of the last tile
        o[x % J] = mfma_bf16_32x32x16(f[x % AHEAD], p[x / J], o[x % J]);
        if (x + AHEAD < 4 * J) fetch(n, x + AHEAD);
    }
    st.l = halves_sum(st.l);
    if (!has_row) return;
    const float by = st.l == 0.f ? 0.f : 1.0f / st.l;
    bf16* to = a.O + row_at<D>(a, t.b, kvh, row) + 4 * half;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) *(floatx2*)(to + 32 * j + 8 * x) = four_bf16(floatx4{o[j][4 * x], o[j][4 * x + 1], o[j][4 * x + 2], o[j][4 * x + 3]}, by);
}

// ---- Many rows at d = 256: a wavefront's 32 rows take more than 256 registers, so four of them share a tile of 64 keys and one is on each SIMD.  Of two tiles in LDS
// one is worked on while the next one's codes are widened into the other, and the loads of the one after it are in flight.  One barrier per tile.
template <int FMT>
__global__ __launch_bounds__(64 * NW, 1) void cache8_wide_rows_kernel(const Cache8Args a, int blocks_per_xcd) {
    constexpr int D = 256, J = D / 32, PAIRS = 4 * J;            // pairs of operands of a tile: K of (sub-tile, j), then V
    constexpr int MINE = PAIRS / NW;                    // of a wavefront: pairs w, w + NW, ...
    constexpr int BUF = PAIRS * 2 * 1024;               // bytes of a tile
    constexpr int GROUP = 16;                           // tiles whose blocks 64 lanes know
    extern __shared__ __align__(16) uint8_t smem[];
    float* scales = (float*)(smem + 2 * BUF);           // [2][64 blocks][4]: ks, vs_log2, vs_inv, tokens there as int (-1: a hole)
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, col = lane & 31;
    // blocks of one batch entry and head follow each other on one XCD: they read the same codes.  Later rows see more keys: they go first
    const int id = xcd_logical_block(blockIdx.x, blocks_per_xcd), bh = a.by_row_blocks.quotient(id), b = a.by_heads.quotient(bh), kvh = bh - b * a.heads;
    if (b >= a.B) return;
    const CacheEntry t = cache_entry(a, b * a.row_blocks + a.row_blocks - 1 - (id - bh * a.row_blocks));
    if (t.row0 >= t.rows) return;
    const int n = t.tiles;

    const int* table = a.page_table + (size_t)t.b * a.max_pages;
    auto page_of = [&](int group) __attribute__((always_inline)) {
        const int blk = 4 * GROUP * group + lane;
        return kCacheBlock * blk < t.len ? table[a.by_page_blocks.quotient(blk)] : -1;
    };
    auto block_of = [&](int group, int page) __attribute__((always_inline)) {
        const CacheBlock x = cache_block(a, kvh, t.len, 4 * GROUP * group + lane, page);
        if (w == 0) *(floatx4*)(scales + 4 * (64 * (group & 1) + lane)) = floatx4{x.ks, x.vs_log2, x.vs_inv, __builtin_bit_cast(float, x.e < 0 ? -1 : x.there)};
        return x;
    };
    CacheBlock now = block_of(0, page_of(0)), next = now;
    int next_page = -1;

    const int row = t.row0 + 32 * w + col;
    const bool has_row = row < t.rows;
    bf16x8 q[2 * J];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            q[2 * j + i] = bf16x8{};
            if (has_row) q[2 * j + i] = *(const bf16x8*)(a.Q + row_at<D>(a, t.b, kvh, row) + 32 * j + 16 * half + 8 * i);
        }
    auto seen_by = [&](int r) __attribute__((always_inline)) { return a.causal ? min(max(a.by_group.quotient(r) + 1 + t.len - t.q_len, 0), t.len) : t.len; };
    const int seen = has_row ? seen_by(row) : t.len;
    const int first_row = t.row0 + 32 * w, last_row = min(first_row + 31, t.rows - 1);
    const int all_see = __builtin_amdgcn_readfirstlane(seen_by(first_row));                           // keys that every row of this wavefront sees
    const int any_sees = __builtin_amdgcn_readfirstlane(first_row < t.rows ? seen_by(last_row) : 0);  // and that some row sees: 0 without rows

    // this wavefront's operand pairs: p = w, w + NW, ... of [K, V][sub-tile][j]; of each the lane's place in a block, and which block it is of the sub-tile
    const uint8_t* base[MINE];
    int sub[MINE];
    bool second[MINE];
#pragma unroll
    for (int x = 0; x < MINE; ++x) {
        const int p = w + NW * x, is_v = p >= 2 * J, q2 = p - (is_v ? 2 * J : 0);
        sub[x] = q2 / J;
        second[x] = is_v ? half : (col >> 2) & 1;
        base[x] = (is_v ? a.v + col * 16 : a.k + (4 * (col >> 3) + (col & 3)) * 16 + half * 256) + 512 * (q2 - sub[x] * J);
    }
    uint4v codes[MINE];
    int now_at = 0;  // max(now.e, 0): holes read block 0, and what they read counts for nothing
    auto load = [&](int i) __attribute__((always_inline)) {  // the share of tile i of the unit; `now` is the group it lies in
#pragma unroll
        for (int x = 0; x < MINE; ++x) {
            const int at = 4 * (i % GROUP) + 2 * sub[x];
            const int e0 = __builtin_amdgcn_readlane(now_at, at), e1 = __builtin_amdgcn_readlane(now_at, at + 1);
            codes[x] = *(const uint4v*)(base[x] + (uint64_t)(uint32_t)(second[x] ? e1 : e0) * (16 * D));
        }
    };
    auto widen = [&](int i, int buf, bool whole) __attribute__((always_inline)) {  // the loaded share into LDS; whole: all tokens are there
#pragma unroll
        for (int x = 0; x < MINE; ++x) {
            const int p = w + NW * x;
            uint4v c = codes[x];
            if (!whole && p >= 2 * J) c = clear_behind(c, __builtin_bit_cast(int, scales[4 * (64 * ((i / GROUP) & 1) + 4 * (i % GROUP) + 2 * sub[x] + half) + 3]));
            uint8_t* to = smem + buf * BUF + p * 2048 + lane * 16;
            *(bf16x8*)to = codes_to_bf16<FMT>(c[0], c[1]);
            *(bf16x8*)(to + 1024) = codes_to_bf16<FMT>(c[2], c[3]);
        }
    };

    floatx16 o[J];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[j][r] = 0.f;
    RowState st{-INFINITY, 0.f, 0.f};

    // S^T of both sub-tiles, and the largest scaled logit of the row
    auto logits = [&](const uint8_t* frag, floatx16 (&s)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = 0.f;
#pragma unroll
            for (int j = 0; j < 2 * J; ++j) s[b] = mfma_bf16_32x32x16(*(const bf16x8*)(frag + (b * J * 2 + j) * 1024), q[j], s[b]);
        }
    };
    auto raise = [&](float top) __attribute__((always_inline)) {
        const float up = __builtin_fmaxf(st.m, top), to = up == -INFINITY ? 0.f : up;
        const float by = st.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.sub - to);
        st.l *= by;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[j][r] *= by;
        st.m = up;
        st.sub = to;
    };
    auto attend = [&](const uint8_t* frag, int b, const bf16x8 (&p)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2 * J; ++j) o[j / 2] = mfma_bf16_32x32x16(*(const bf16x8*)(frag + ((2 + b) * J * 2 + j) * 1024), p[j & 1], o[j / 2]);
    };

    now_at = max(now.e, 0);
    uint64_t lacking = __ballot(now.there < 16), lacking_next = 0;  // blocks of the group that `now` is, and of the one before while it is worked on
    if (n > 0) load(0);
    __syncthreads();  // the scales of the first group
    if (n > 0) {
        widen(0, 0, false);
        if (n > 1) load(1);
    }
    __syncthreads();
    // what the next group's blocks are: pages at the start of a group, scales in its middle; its first tile is loaded two tiles ahead
    auto look_ahead = [&](int i) __attribute__((always_inline)) {
        const int at = i % GROUP;
        if (at == 0 && i + GROUP < n) next_page = page_of(i / GROUP + 1);
        if (at == GROUP / 2 && i + GROUP - GROUP / 2 < n) {
            next = block_of(i / GROUP + 1, next_page);
            lacking_next = __ballot(next.there < 16);
        }
        if (at == GROUP - 2) now_at = max(next.e, 0);
    };
    auto done = [&](int i) __attribute__((always_inline)) {
        if (i % GROUP == GROUP - 1) lacking = lacking_next;
        __syncthreads();
    };
    // a tile that every row sees whole, followed by one whose tokens are all there: no masks to apply
    auto plain = [&](int i) __attribute__((always_inline)) {
        const int at = i % GROUP;
        const uint64_t here = (lacking >> (4 * at)) & 15, after = at == GROUP - 1 ? lacking_next & 15 : (lacking >> (4 * at + 4)) & 15;
        return i + 2 < n && 64 * i + 64 <= all_see && (here | after) == 0;
    };
    bool ahead = false;  // whether the next tile is widened and the one after it asked for
    for (int i = 0; i < n;) {
        look_ahead(i);
        while (plain(i)) {
            const int buf = i & 1;
            const uint8_t* frag = smem + buf * BUF + lane * 16;
            const float* sc = scales + 4 * (64 * ((i / GROUP) & 1) + 4 * (i % GROUP) + half);
            const floatx4 x0 = *(const floatx4*)sc, x1 = *(const floatx4*)(sc + 8);
            floatx16 s[2];
            widen(i + 1, buf ^ 1, true);
            load(i + 2);
            ahead = true;
            logits(frag, s);
            float top[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                top[b] = s[b][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) top[b] = __builtin_fmaxf(top[b], s[b][r]);
            }
            const float most = halves_max(__builtin_fmaxf(top[0] * x0[0], top[1] * x1[0]));
            // A maximum that has to rise is the other path's: with the rescaling in here, the compiler moves the accumulators to other registers and
            // back in every tile.
            if (__any(most > st.m + kRescaleAbove)) break;
            bf16x8 p[2];
            tile_probabilities<false>(s[0], x0[0], x0[1], x0[2], st.sub, 16, &p[0], &p[1], &st.l);
            attend(frag, 0, p);
            tile_probabilities<false>(s[1], x1[0], x1[1], x1[2], st.sub, 16, &p[0], &p[1], &st.l);
            attend(frag, 1, p);
            ahead = false;
            done(i);
            look_ahead(++i);
        }
        if (i >= n) break;
        const int buf = i & 1, key0 = 64 * i;
        if (!ahead) {
            if (i + 1 < n) widen(i + 1, buf ^ 1, false);
            if (i + 2 < n) load(i + 2);
        }
        ahead = false;
        if (key0 < any_sees) {
            const uint8_t* frag = smem + buf * BUF + lane * 16;
            const float* sc = scales + 4 * (64 * ((i / GROUP) & 1) + 4 * (i % GROUP) + half);
            floatx16 s[2];
            logits(frag, s);
            float most = -INFINITY;
            int visible[2];
            floatx4 x[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                x[b] = *(const floatx4*)(sc + 8 * b);
                const float last = x[b][3];  // (the bits of a vector's element taken directly would be those of its first)
                visible[b] = __builtin_bit_cast(int, last) < 0 ? 0 : min(max(seen - key0 - 32 * b - kCacheBlock * half, 0), 16);
                float top = -INFINITY;
#pragma unroll
                for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, r < visible[b] ? s[b][r] : -INFINITY);
                most = __builtin_fmaxf(most, top == -INFINITY ? top : top * x[b][0]);
            }
            most = halves_max(most);
            if (__any(most > st.m + kRescaleAbove)) raise(most);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                bf16x8 p[2];
                tile_probabilities<true>(s[b], x[b][0], x[b][1], x[b][2], st.sub, visible[b], &p[0], &p[1], &st.l);
                attend(frag, b, p);
            }
        }
        done(i);
        ++i;
    }
    st.l = halves_sum(st.l);
    if (!has_row) return;
    const float by = st.l == 0.f ? 0.f : 1.0f / st.l;
    bf16* to = a.O + row_at<D>(a, t.b, kvh, row) + 4 * half;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) *(floatx2*)(to + 32 * j + 8 * x) = four_bf16(floatx4{o[j][4 * x], o[j][4 * x + 1], o[j][4 * x + 2], o[j][4 * x + 3]}, by);
}

// ---- Puts the parts of a row together whose entry was divided.  M = max m_s, O = sum 2^(m_s - M) O_s / sum 2^(m_s - M) l_s.  Both kernels are chains of
// round trips (the entry's units, then statistics and results together), so the first results are asked for before their weights are known.
__device__ __forceinline__ float part_weight(float m, float l, float top) {
    return m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - top);  // no key seen: nothing; what is no number stays so
}
__device__ __forceinline__ void add_part(floatx4& acc, float wt, const floatx4& y) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = wt == 0.f ? acc[i] : acc[i] + wt * y[i];
}

// Few parts per entry: a wavefront per row.  Workgroups whose entry was not divided end at once.
template <int D>
__global__ __launch_bounds__(256) void cache8_merge_kernel(const Cache8Args a) {
    constexpr int Q4 = D / 4, LANES = 64 / Q4, AHEAD = 8;
    const int lane = threadIdx.x & 63;
    const int e = a.by_heads.quotient(blockIdx.x), kvh = blockIdx.x - e * a.heads;
    const int2 unit = a.units[e];  // unset where the entry has no rows
    const CacheEntry t = cache_entry(a, e);
    const int r = 4 * blockIdx.y + (threadIdx.x >> 6), row = t.row0 + r;
    if (row >= t.rows || unit.y == 1) return;
    const int n = unit.y, c4 = lane % Q4, first = lane / Q4 < LANES ? lane / Q4 : n;  // d = 96: some lanes have no column
    const size_t size = (size_t)a.rows_per_block * (D + 2), stride = size * a.heads;
    const float* base = a.parts + ((size_t)unit.x * a.heads + kvh) * size;
    const float *m_of = base + a.rows_per_block * D + r, *o_of = base + (size_t)r * D + 4 * c4;
    floatx4 ahead[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        ahead[i] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (first + i * LANES < n) ahead[i] = *(const floatx4*)(o_of + (size_t)(first + i * LANES) * stride);
    }
    float top = -INFINITY;
    for (int s = lane; s < n; s += 64) top = __builtin_fmaxf(top, m_of[s * stride]);
    top = wave_max(top);
    floatx4 acc{0.f, 0.f, 0.f, 0.f};
    float L = 0.f;
    for (int s0 = 0; s0 < n; s0 += 64) {
        float wt = 0.f;
        if (s0 + lane < n) {
            const float m = m_of[(s0 + lane) * stride], l = m_of[(s0 + lane) * stride + a.rows_per_block];
            wt = part_weight(m, l, top);
            L += wt * l;
        }
        const int end = min(n - s0, 64);
        if (s0 == 0) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) add_part(acc, __shfl(wt, min(first + i * LANES, 63)), ahead[i]);  // those behind n have weight 0, or fetched nothing
        }
        for (int i = s0 ? 0 : AHEAD * LANES; i < end; i += LANES) {
            const float x = __shfl(wt, min(first + i, 63));
            if (first + i < end) add_part(acc, x, *(const floatx4*)(o_of + (size_t)(s0 + first + i) * stride));
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) L += __shfl_xor(L, o);
    floatx4 all = acc;
#pragma unroll
    for (int k = 1; k < LANES; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) all[i] += __shfl(acc[i], min(k * Q4 + c4, 63));
    if (lane < Q4) *(floatx2*)(a.O + row_at<D>(a, t.b, kvh, row) + 4 * c4) = four_bf16(all, L == 0.f ? 0.f : 1.0f / L);
}

// Many parts per entry: a workgroup per row and 32 columns.
template <int D>
__global__ __launch_bounds__(256) void cache8_merge_many_kernel(const Cache8Args a) {
    constexpr int THREADS = 256, COLS = 32, Q4 = COLS / 4, LANES = THREADS / Q4, WAVES = THREADS / 64, AHEAD = 4;
    __shared__ floatx4 red[THREADS];
    __shared__ float wts[THREADS], stat[2][WAVES];
    const int tid = threadIdx.x, lane = tid & 63;
    const int e = a.by_heads.quotient(blockIdx.x), kvh = blockIdx.x - e * a.heads;
    const int2 unit = a.units[e];
    const CacheEntry t = cache_entry(a, e);
    const int r = blockIdx.y, row = t.row0 + r;
    if (row >= t.rows || unit.y == 1) return;
    const int n = unit.y;
    const size_t size = (size_t)a.rows_per_block * (D + 2), stride = size * a.heads;
    const float* base = a.parts + ((size_t)unit.x * a.heads + kvh) * size;
    const float* m_of = base + a.rows_per_block * D + r;
    const int c4 = tid % Q4, first = tid / Q4;
    const float* o_of = base + (size_t)r * D + COLS * blockIdx.z + 4 * c4;

    floatx4 ahead[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        ahead[i] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (first + i * LANES < n) ahead[i] = *(const floatx4*)(o_of + (size_t)(first + i * LANES) * stride);
    }
    float top = -INFINITY, m0 = -INFINITY, l0 = 0.f;
    if (tid < n) {
        m0 = m_of[tid * stride];
        l0 = m_of[tid * stride + a.rows_per_block];
    }
    top = m0;
    for (int s = tid + THREADS; s < n; s += THREADS) top = __builtin_fmaxf(top, m_of[s * stride]);
    top = wave_max(top);
    if (lane == 0) stat[0][tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) top = __builtin_fmaxf(top, stat[0][i]);
    floatx4 acc{0.f, 0.f, 0.f, 0.f};
    float L = 0.f;
    for (int s0 = 0; s0 < n; s0 += THREADS) {
        if (s0 + tid < n) {
            if (s0) {
                m0 = m_of[(s0 + tid) * stride];
                l0 = m_of[(s0 + tid) * stride + a.rows_per_block];
            }
            const float wt = part_weight(m0, l0, top);
            wts[tid] = wt;
            L += wt * l0;
        }
        __syncthreads();
        const int end = min(n - s0, THREADS);
        int s = first;
        if (s0 == 0) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (first + i * LANES < end) add_part(acc, wts[first + i * LANES], ahead[i]);
            s = first + AHEAD * LANES;
        }
#pragma unroll 4
        for (; s < end; s += LANES) add_part(acc, wts[s], *(const floatx4*)(o_of + (size_t)(s0 + s) * stride));
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
    *(floatx2*)(a.O + row_at<D>(a, t.b, kvh, row) + COLS * blockIdx.z + 4 * c4) = four_bf16(acc, L == 0.f ? 0.f : 1.0f / L);
}

template <int D, int ROWS, int FMT, bool DIVIDED>
hipError_t launch_few(const Cache8Args& args, hipStream_t stream) {
    static std::atomic<uint64_t> lds_allowed{0};
    constexpr auto lds_bytes = [](int rows) { return (NW * rows * (D + 4) + NW * 2 * ROWS) * (int)sizeof(float); };
    static_assert(lds_bytes(ROWS) <= 160 * 1024, "the wavefronts' results must fit the LDS");
    const hipError_t e = allow_dynamic_lds((const void*)cache8_few_rows_kernel<D, ROWS, FMT, DIVIDED>, lds_bytes(ROWS), &lds_allowed);
    if (e != hipSuccess) return e;
    const int rows = args.Nq * args.group < ROWS ? args.Nq * args.group : ROWS;
    const unsigned units = (unsigned)(DIVIDED ? args.limit : args.entries);
    hipLaunchKernelGGL((cache8_few_rows_kernel<D, ROWS, FMT, DIVIDED>), dim3(units * (unsigned)args.heads), dim3(64 * NW), lds_bytes(rows), stream, args, rows);
    return hipGetLastError();
}
template <int D, int ROWS, int FMT>
hipError_t launch_few(const Cache8Args& args, hipStream_t stream) {
    return args.limit ? launch_few<D, ROWS, FMT, true>(args, stream) : launch_few<D, ROWS, FMT, false>(args, stream);
}

template <int D, int FMT>
hipError_t launch_rows(const Cache8Args& args, hipStream_t stream) {
    static std::atomic<uint64_t> lds_allowed{0};
    constexpr int tile = (D / 32) * 4 * 2048, lds = D == 256 ? 2 * tile + 2 * 64 * 16 : 4 * tile + 2 * 64 * 20;
    static_assert(lds <= 160 * 1024, "the tiles must fit the LDS");
    const auto kernel = [] {
        if constexpr (D == 256) return cache8_wide_rows_kernel<FMT>;
        else return cache8_rows_kernel<D, FMT>;
    }();
    const hipError_t e = allow_dynamic_lds((const void*)kernel, lds, &lds_allowed);
    if (e != hipSuccess) return e;
    const int per_xcd = (int)(((long long)args.entries * args.heads + 7) / 8);
    hipLaunchKernelGGL(kernel, dim3((unsigned)per_xcd * 8u), dim3(D == 256 ? 64 * NW : 512), lds, stream, args, per_xcd);
    return hipGetLastError();
}

template <int D>
hipError_t launch_merge(const Cache8Args& args, hipStream_t stream) {
    const int rows = args.Nq * args.group < args.rows_per_block ? args.Nq * args.group : args.rows_per_block;  // that a block has at most
    const unsigned grid = (unsigned)args.entries * (unsigned)args.heads;
    if (args.limit <= 16 * args.entries) hipLaunchKernelGGL((cache8_merge_kernel<D>), dim3(grid, (unsigned)(rows + 3) / 4), dim3(256), 0, stream, args);
    else hipLaunchKernelGGL((cache8_merge_many_kernel<D>), dim3(grid, (unsigned)rows, D / 32), dim3(256), 0, stream, args);
    return hipGetLastError();
}

template <int D, int FMT>
hipError_t launch(const Cache8Args& args, hipStream_t stream) {
    hipError_t e = hipErrorInvalidValue;
    if (args.rows_per_block > 32) e = launch_rows<D, FMT>(args, stream);
    else if (args.rows_per_block == 32) e = launch_few<D, 32, FMT>(args, stream);
    else if constexpr (D % 64 == 0) e = launch_few<D, 16, FMT>(args, stream);
    return e != hipSuccess || args.limit == 0 ? e : launch_merge<D>(args, stream);
}

template <int D>
hipError_t launch(const Cache8Args& args, int format, hipStream_t stream) {
    return format == FLAT_CACHE8_E4M3 ? launch<D, FLAT_CACHE8_E4M3>(args, stream) : launch<D, FLAT_CACHE8_INT8>(args, stream);
}

}  // namespace

hipError_t launch_cache8_fwd(const flat_cache8& c, const Cache8Attend& a, const Cache8Plan& plan, hipStream_t stream) {
    int shift = 0;
    while (1 << shift < plan.tile_keys) ++shift;
    const Cache8Args args{(const uint8_t*)c.k, (const uint8_t*)c.v, c.k_scale, c.v_scale, (const bf16*)a.Q, (bf16*)a.O, a.page_table, a.lens, a.q_lens,
                          (int2*)a.workspace, (float*)((char*)a.workspace + plan.parts_at), c.n_pages, c.n_heads, a.max_pages, a.max_pages * c.page_tokens,
                          a.B, a.H, a.Nq, a.H / c.n_heads, a.scale * kLog2e, a.causal, plan.rows_per_block, plan.row_blocks, plan.entries, shift, plan.aim,
                          plan.limit, plan.least_tiles, Divisor(c.n_heads), Divisor(a.H / c.n_heads), Divisor(plan.row_blocks),
                          Divisor(c.page_tokens / kCacheBlock), c.page_tokens / kCacheBlock};
    switch (c.d) {
        case 32: return launch<32>(args, c.format, stream);
        case 64: return launch<64>(args, c.format, stream);
        case 96: return launch<96>(args, c.format, stream);
        case 128: return launch<128>(args, c.format, stream);
        case 256: return launch<256>(args, c.format, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace flat
