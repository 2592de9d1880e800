// Pages of the 8-bit cache: copying, forking, freeing, compacting.  What moves is moved in pieces of 16 KiB of a page, one workgroup each, with
// every load of a piece issued before its stores: 16 bytes a lane, read once and written once, HBM's rate.  What is listed goes
// through a bitmap of held pages in the LDS of one workgroup: the table is read once, and no global atomics and nothing to clear beforehand are needed.
#include "flat_cache8.hpp"
#include "flat_common.hpp"
#include "flat_launch.hpp"

namespace flat {

namespace {

constexpr int kThreads = 256;
constexpr int kPerThread = 4;
constexpr int kPiece = kThreads * kPerThread * 16;

struct PageArgs {
    uint8_t *k, *v;
    float *ks, *vs;
    int n_pages, page_scales;  // scales of a page, K or V
    size_t page_bytes;         // codes of a page, K or V
    int pieces;                // of the codes of K, or of V
};
PageArgs page_args(const flat_cache8& c) {
    const size_t bytes = (size_t)c.n_heads * c.page_tokens * c.d;
    return PageArgs{(uint8_t*)c.k, (uint8_t*)c.v, c.k_scale, c.v_scale, c.n_pages, c.n_heads * (c.page_tokens / kCacheBlock), bytes,
                    (int)((bytes + kPiece - 1) / kPiece)};
}

// Piece `piece` of page src to page dst: 0 .. pieces - 1 are K's codes, then V's, then the scales.
__device__ __forceinline__ void copy_piece(const PageArgs& a, int src, int dst, int piece) {
    const int tid = threadIdx.x;
    if (piece == 2 * a.pieces) {
        for (int i = tid; i < a.page_scales; i += kThreads) {
            a.ks[(size_t)dst * a.page_scales + i] = a.ks[(size_t)src * a.page_scales + i];
            a.vs[(size_t)dst * a.page_scales + i] = a.vs[(size_t)src * a.page_scales + i];
        }
        return;
    }
    uint8_t* pool = piece < a.pieces ? a.k : a.v;
    const size_t at = (size_t)(piece < a.pieces ? piece : piece - a.pieces) * kPiece + 16 * tid;
    const uint8_t* s = pool + src * a.page_bytes + at;
    uint8_t* t = pool + dst * a.page_bytes + at;
    uint4v x[kPerThread];
#pragma unroll
    for (int i = 0; i < kPerThread; ++i)
        if (at + i * (16 * kThreads) < a.page_bytes) x[i] = *(const uint4v*)(s + i * (16 * kThreads));
#pragma unroll
    for (int i = 0; i < kPerThread; ++i)
        if (at + i * (16 * kThreads) < a.page_bytes) *(uint4v*)(t + i * (16 * kThreads)) = x[i];
}

// Pair blockIdx.y.  Every workgroup looks through the whole list for what would make two copies meet, so that what it reads is written by nobody.
__global__ __launch_bounds__(kThreads) void cache8_copy_kernel(const PageArgs a, const int* src, const int* dst, int n, int pair0) {
    const int i = pair0 + blockIdx.y, s = src[i], d = dst[i];
    if ((unsigned)s >= (unsigned)a.n_pages || (unsigned)d >= (unsigned)a.n_pages || s == d) return;
    int out = 0;
    for (int j = threadIdx.x; j < n; j += kThreads) {
        const int sj = src[j], dj = dst[j];
        const bool counts = (unsigned)sj < (unsigned)a.n_pages && sj != dj;
        out |= counts && (dj == s || (dj == d && j > i));
    }
    if (__syncthreads_or(out)) return;
    copy_piece(a, s, d, blockIdx.x);
}

struct ForkArgs {
    int* page_table;
    int max_pages, n_seqs, page_tokens;
    int* lens;
    const int *parents, *children, *spares;
    int n;
};
__global__ __launch_bounds__(kThreads) void cache8_fork_kernel(const PageArgs a, const ForkArgs f, int fork0) {
    const int i = fork0 + blockIdx.y, p = f.parents[i], c = f.children[i];
    if ((unsigned)p >= (unsigned)f.n_seqs || (unsigned)c >= (unsigned)f.n_seqs || p == c) return;
    int out = 0;
    for (int j = threadIdx.x; j < f.n; j += kThreads) out |= f.children[j] == p || (j > i && f.children[j] == c);
    if (__syncthreads_or(out)) return;
    // from here on the parent's row and length are nobody's to write
    const int len = min(max(f.lens[p], 0), f.max_pages * f.page_tokens);
    const int full = len / f.page_tokens;
    const int* from = f.page_table + (size_t)p * f.max_pages;
    const int begun = len - full * f.page_tokens > 0 ? from[full] : -1;  // the page that is copied, if there is one
    const bool copies = (unsigned)begun < (unsigned)a.n_pages;
    const int spare = f.spares[i];
    if (copies && ((unsigned)spare >= (unsigned)a.n_pages || spare == begun)) return;
    out = 0;
    for (int j = i + 1 + threadIdx.x; j < f.n; j += kThreads) out |= copies && f.spares[j] == spare;
    if (__syncthreads_or(out)) return;
    if (blockIdx.x <= 2 * (unsigned)a.pieces) {
        if (copies) copy_piece(a, begun, spare, blockIdx.x);
        return;
    }
    int* to = f.page_table + (size_t)c * f.max_pages;
    for (int x = threadIdx.x; x < f.max_pages; x += kThreads) to[x] = x < full ? from[x] : x == full && copies ? spare : -1;
    if (threadIdx.x == 0) f.lens[c] = f.lens[p];
}

// ---- lists of held and unused pages: one workgroup, a bitmap in LDS ------------------------------------------------------------------
constexpr int kListThreads = 1024;
constexpr int kListWaves = kListThreads / 64;

// One compute unit reads the whole table, so what bounds it is how much is on its way: 16 bytes a load, eight loads a thread, 128 KiB at once.
__device__ __forceinline__ void mark_held(uint32_t* bits, int n_pages, const int* table, int n) {
    const int tid = threadIdx.x;
    auto mark = [&](int id) __attribute__((always_inline)) {
        if ((unsigned)id < (unsigned)n_pages) atomicOr(&bits[id >> 5], 1u << (id & 31));
    };
    for (int i = tid; i < (n_pages + 63) / 64 * 2; i += kListThreads) bits[i] = 0;
    __syncthreads();
    const int head = min((int)((0 - (reinterpret_cast<uintptr_t>(table) >> 2)) & 3), n);  // ids before the first 16-byte boundary
    const int quads = (n - head) / 4, tail = n - head - 4 * quads;
    if (tid < head) mark(table[tid]);
    if (tid < tail) mark(table[head + 4 * quads + tid]);
    const uint4v* body = (const uint4v*)(table + head);
    constexpr int U = 8;
    for (int i0 = tid; i0 < quads; i0 += U * kListThreads) {
        uint4v id[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            id[u] = uint4v{~0u, ~0u, ~0u, ~0u};
            if (quads - i0 > u * kListThreads) id[u] = body[i0 + u * kListThreads];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int x = 0; x < 4; ++x) mark((int)id[u][x]);
    }
    __syncthreads();
}

// Wavefront w has the groups of 64 pages [first, last): counts pages for which keep(group, bits of it) has a bit, and returns in *before the
// number in the wavefronts before it and in *total that of all.
template <typename F>
__device__ __forceinline__ void count_kept(const uint64_t* groups, int first, int last, int* sums, const F& keep, int* before, int* total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int mine = 0;
    for (int g = first + lane; g < last; g += 64) mine += __popcll(keep(g, groups[g]));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o);
    __syncthreads();  // sums may still be read
    if (lane == 0) sums[w] = mine;
    __syncthreads();
    *before = *total = 0;
    for (int i = 0; i < kListWaves; ++i) {
        *before += i < w ? sums[i] : 0;
        *total += sums[i];
    }
}

// Their ids, ascending, from list[at] on.  64 groups at a time, a lane has the bits of one.  Where all have few, every lane writes its own, bit by bit; else
// the wavefront takes the groups in turn, a lane for a bit.
template <typename F>
__device__ __forceinline__ void list_kept(const uint64_t* groups, int first, int last, const F& keep, int* list, int at) {
    constexpr int kFew = 16;
    const int lane = threadIdx.x & 63;
    for (int g0 = first; g0 < last; g0 += 64) {
        uint64_t mine = g0 + lane < last ? keep(g0 + lane, groups[g0 + lane]) : 0;
        const int count = __popcll(mine), upto = wave_prefix(count);
        if (!__any(count > kFew)) {
            for (int to = at + upto - count; __any(mine != 0); ++to) {
                if (mine) list[to] = 64 * (g0 + lane) + __builtin_ctzll(mine);
                mine &= mine - 1;
            }
        } else {
            int to = at;
            const int end = min(last - g0, 64);
            for (int i = 0; i < end; ++i) {
                const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, i), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(mine >> 32), i);
                const uint64_t bits = ((uint64_t)hi << 32) | lo;
                if ((bits >> lane) & 1) list[to + (int)__builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0))] = 64 * (g0 + i) + lane;
                to += __popcll(bits);
            }
        }
        at += __builtin_amdgcn_readlane(upto, 63);
    }
}

__device__ __forceinline__ void fill_unused(int* list, int n) {
    const int tid = threadIdx.x, head = min((int)((0 - (reinterpret_cast<uintptr_t>(list) >> 2)) & 3), n);
    const int quads = (n - head) / 4, tail = n - head - 4 * quads;
    if (tid < head) list[tid] = -1;
    if (tid < tail) list[head + 4 * quads + tid] = -1;
    uint4v* body = (uint4v*)(list + head);
    for (int i = tid; i < quads; i += kListThreads) body[i] = uint4v{~0u, ~0u, ~0u, ~0u};
}

// Bits of group g that are pages below `end`.
__device__ __forceinline__ uint64_t below(int g, int end) {
    const int n = end - 64 * g;
    return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
}

__global__ __launch_bounds__(kListThreads) void cache8_free_kernel(int* page_table, int max_pages, int n_seqs, int* lens, const int* seqs, int n,
                                                                   int n_pages, int* unused, int* n_unused) {
    extern __shared__ __align__(16) uint64_t bitmap[];
    __shared__ int sums[kListWaves];
    const int tid = threadIdx.x, w = tid >> 6;
    for (int i = w; i < n; i += kListWaves) {
        const int s = seqs[i];
        if ((unsigned)s >= (unsigned)n_seqs) continue;
        for (int x = tid & 63; x < max_pages; x += 64) page_table[(size_t)s * max_pages + x] = -1;
        if ((tid & 63) == 0) lens[s] = 0;
    }
    fill_unused(unused, n_pages);  // all of it, while the table is on its way; the list overwrites its beginning
    __syncthreads();  // the rows are read below
    mark_held((uint32_t*)bitmap, n_pages, page_table, n_seqs * max_pages);
    const int groups = (n_pages + 63) / 64, share = (groups + kListWaves - 1) / kListWaves;
    const int first = min(w * share, groups), last = min(first + share, groups);
    auto keep = [&](int g, uint64_t held) { return ~held & below(g, n_pages); };
    int before, total;
    count_kept(bitmap, first, last, sums, keep, &before, &total);
    list_kept(bitmap, first, last, keep, unused, before);
    if (tid == 0) *n_unused = total;
}

// Workspace of a compaction, ints: [0] the number of moves, then src, dst and the new id of a page that moves, n_pages each.
__global__ __launch_bounds__(kListThreads) void cache8_compact_plan_kernel(const int* page_table, int entries, int n_pages, int* n_used, int* ws) {
    extern __shared__ __align__(16) uint64_t bitmap[];
    __shared__ int sums[kListWaves];
    const int tid = threadIdx.x, w = tid >> 6;
    mark_held((uint32_t*)bitmap, n_pages, page_table, entries);
    const int groups = (n_pages + 63) / 64, share = (groups + kListWaves - 1) / kListWaves;
    const int first = min(w * share, groups), last = min(first + share, groups);
    int before, used, moves;
    count_kept(bitmap, first, last, sums, [&](int, uint64_t held) { return held; }, &before, &used);
    int *src = ws + 1, *dst = src + n_pages, *now = dst + n_pages;
    auto moving = [&](int g, uint64_t held) { return held & ~below(g, used); };
    auto hole = [&](int g, uint64_t held) { return ~held & below(g, used); };
    count_kept(bitmap, first, last, sums, moving, &before, &moves);
    list_kept(bitmap, first, last, moving, src, before);
    count_kept(bitmap, first, last, sums, hole, &before, &moves);
    list_kept(bitmap, first, last, hole, dst, before);
    __syncthreads();
    for (int i = tid; i < moves; i += kListThreads) now[src[i]] = dst[i];
    if (tid == 0) {
        *n_used = used;
        ws[0] = moves;
    }
}

// Moves the pages and renames them in the table; workgroups share both, whose extent only the device knows.
__global__ __launch_bounds__(kThreads) void cache8_compact_move_kernel(const PageArgs a, const int* page_table, int* new_table, int entries,
                                                                       const int* n_used, const int* ws) {
    const int moves = ws[0], used = *n_used, pieces = 2 * a.pieces + 1;
    const int *src = ws + 1, *dst = src + a.n_pages, *now = dst + a.n_pages;
    for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < entries; i += (long long)gridDim.x * kThreads) {
        const int id = page_table[i];
        new_table[i] = id >= used && id < a.n_pages ? now[id] : id;
    }
    const long long items = (long long)moves * pieces;
    for (long long i = blockIdx.x; i < items; i += gridDim.x) {
        const int m = (int)(i / pieces);
        copy_piece(a, src[m], dst[m], (int)(i - (long long)m * pieces));
    }
}

std::atomic<uint64_t> g_free_lds{0}, g_plan_lds{0};
int bitmap_bytes(int n_pages) { return (n_pages + 63) / 64 * 8; }
constexpr int kMaxBitmap = FLAT_CACHE8_MAX_LISTED_PAGES / 8;

}  // namespace

hipError_t launch_cache8_copy(const flat_cache8& c, const int* src, const int* dst, int n, hipStream_t stream) {
    const PageArgs a = page_args(c);
    for (int i = 0; i < n; i += 65535) {
        hipLaunchKernelGGL(cache8_copy_kernel, dim3(2 * (unsigned)a.pieces + 1, (unsigned)(n - i < 65535 ? n - i : 65535)), dim3(kThreads), 0, stream, a, src, dst, n, i);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_cache8_fork(const flat_cache8& c, int* page_table, int max_pages, int n_seqs, int* lens, const int* parents,
                              const int* children, const int* spares, int n, hipStream_t stream) {
    const PageArgs a = page_args(c);
    const ForkArgs f{page_table, max_pages, n_seqs, c.page_tokens, lens, parents, children, spares, n};
    for (int i = 0; i < n; i += 65535) {
        hipLaunchKernelGGL(cache8_fork_kernel, dim3(2 * (unsigned)a.pieces + 2, (unsigned)(n - i < 65535 ? n - i : 65535)), dim3(kThreads), 0, stream, a, f, i);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_cache8_free(int* page_table, int max_pages, int n_seqs, int* lens, const int* seqs, int n, int n_pages, int* unused,
                              int* n_unused, hipStream_t stream) {
    const hipError_t e = allow_dynamic_lds((const void*)cache8_free_kernel, kMaxBitmap, &g_free_lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(cache8_free_kernel, dim3(1), dim3(kListThreads), bitmap_bytes(n_pages), stream, page_table, max_pages, n_seqs, lens, seqs, n, n_pages, unused,
                       n_unused);
    return hipGetLastError();
}

hipError_t launch_cache8_compact(const flat_cache8& c, const int* page_table, int* new_table, int max_pages, int n_seqs, int* n_used,
                                 int* workspace, hipStream_t stream) {
    hipError_t e = allow_dynamic_lds((const void*)cache8_compact_plan_kernel, kMaxBitmap, &g_plan_lds);
    if (e != hipSuccess) return e;
    const int entries = n_seqs * max_pages;  // fits: the C ABI checks
    hipLaunchKernelGGL(cache8_compact_plan_kernel, dim3(1), dim3(kListThreads), bitmap_bytes(c.n_pages), stream, page_table, entries, c.n_pages, n_used, workspace);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(cache8_compact_move_kernel, dim3(2048), dim3(kThreads), 0, stream, page_args(c), page_table, new_table, entries, n_used, workspace);
    return hipGetLastError();
}

}  // namespace flat
