// The paged key/value cache of 8-bit codes: its layout, and the host-side launchers behind flat_cache8_api.hip.
//
// A block is kCacheBlock = 16 tokens of one head of one page, with one scale for K and one for V; a value is code * scale.  Block number
// e = (page * heads + head) * blocks_per_page + block of the page; its 16 d codes are contiguous, and ordered so that the 16 bytes a lane
// loads are a matrix operand as they lie:
//   K: [d / 16][16 tokens][16 channels]   a lane's 16 bytes are 16 channels (contraction of Q K^T) of one token
//   V: [d channels][16 tokens]            a lane's 16 bytes are the 16 tokens (contraction of P V) of one channel
// A wavefront's load of 64 x 16 bytes is then 1 KiB in one or two contiguous pieces, and nothing is ever transposed on the way to the MFMAs.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/flat_attn.h"

namespace flat {

constexpr int kCacheBlock = FLAT_CACHE8_BLOCK;

// A row of Q (q = 0) and K heads that are rotated together (flat_rope.hip)
struct RopeProblem {
    const void* in[2];
    void* out[2];
    int heads[2];  // 0: not there
    int B, N, d, rot;
    const double* freqs;
    const int* positions;  // [B, N] or null
    float magnitude;
    int interleaved, transpose, f32;
};
hipError_t launch_rope(const RopeProblem& p, hipStream_t stream);

// Blocks that N tokens touch at most, wherever they start.
inline int cache8_write_blocks(int N) { return (int)(((long long)N + 2 * kCacheBlock - 2) / kCacheBlock); }
struct CacheWrite {
    const void *K, *V;
    int B, N;
    const int* page_table;
    int max_pages;
    const int* lens;
    const int* n_new;
};
hipError_t launch_cache8_write(const flat_cache8& c, const CacheWrite& w, hipStream_t stream);

hipError_t launch_cache8_copy(const flat_cache8& c, const int* src, const int* dst, int n, hipStream_t stream);
hipError_t launch_cache8_fork(const flat_cache8& c, int* page_table, int max_pages, int n_seqs, int* lens, const int* parents,
                              const int* children, const int* spares, int n, hipStream_t stream);
hipError_t launch_cache8_free(int* page_table, int max_pages, int n_seqs, int* lens, const int* seqs, int n, int n_pages, int* unused,
                              int* n_unused, hipStream_t stream);
hipError_t launch_cache8_compact(const flat_cache8& c, const int* page_table, int* new_table, int max_pages, int n_seqs, int* n_used,
                                 int* workspace, hipStream_t stream);

// Attention over the cache (flat_cache8_fwd.hip).  A row block is rows_per_block of the Nq * (H / heads) rows that share a head of the cache;
// an entry is a row block of a batch entry, and its keys are divided over one or more units, a workgroup per unit and head.
struct Cache8Plan {
    int rows_per_block;  // 16, 32: the wavefronts of a workgroup share the keys of a block's rows; 256 (d = 256: 128): each has 32 rows of its own
    int row_blocks;      // per batch entry, for Nq queries
    int entries;         // B * row_blocks
    int tile_keys;       // what a kernel takes of the keys at a time: a power of two
    int aim, limit;      // blocks of 16 and 32 rows: units aimed at over all entries, and the most there are (per head of the cache); 0: every entry is one unit
    int least_tiles;     // that a unit has, unless its entry has fewer
    size_t parts_at;     // bytes of the workspace before the units' partial results
    size_t workspace_bytes;
};
// Keys of a step of one wavefront, blocks of 16 and 32 rows.
constexpr int cache8_step_keys(int rows, int d) { return rows == 16 || d == 64 ? 64 : d == 32 ? 128 : 32; }
void cache8_plan(int B, int H, int heads, int Nq, int max_tokens, int d, Cache8Plan* out);  // host arithmetic only
struct Cache8Attend {
    const void* Q;
    void* O;
    int B, H, Nq;
    const int* page_table;
    int max_pages;
    const int* lens;
    const int* q_lens;
    float scale;
    int causal;
    float* workspace;
};
hipError_t launch_cache8_fwd(const flat_cache8& c, const Cache8Attend& a, const Cache8Plan& plan, hipStream_t stream);

}  // namespace flat
