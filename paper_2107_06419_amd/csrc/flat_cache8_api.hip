// C ABI of rotary positions and of the paged 8-bit cache (see include/flat_attn.h for the contract).  Every argument check runs before
// the first HIP call.
#include <math.h>
#include <stdint.h>

#include "flat_cache8.hpp"

namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// A buffer of a call, for the overlap checks.
struct Span {
    const void* at;
    size_t bytes;
};
bool overlaps(const Span& a, const Span& b) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.at), b0 = reinterpret_cast<uintptr_t>(b.at);
    return a.at && b.at && a.bytes && b.bytes && a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}
template <size_t N>
bool overlaps_any(const Span& a, const Span (&others)[N]) {
    for (const Span& o : others)
        if (overlaps(a, o)) return true;
    return false;
}

bool head_dim(int d) { return d == 32 || d == 64 || d == 96 || d == 128 || d == 256; }
constexpr long long kMaxInt = 0x7fffffffLL;
size_t ints(long long n) { return (size_t)n * sizeof(int); }

// The cache itself; on success its four buffers.
int check_cache(const flat_cache8* c, Span (&buf)[4]) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return FLAT_ERR_NULL;
    if (c->n_pages <= 0 || c->n_heads <= 0 || c->page_tokens <= 0 || c->page_tokens % FLAT_CACHE8_BLOCK || c->page_tokens > 65536) return FLAT_ERR_SHAPE;
    if (!head_dim(c->d)) return FLAT_ERR_UNSUPPORTED;
    if (c->format != FLAT_CACHE8_E4M3 && c->format != FLAT_CACHE8_INT8) return FLAT_ERR_UNSUPPORTED;
    const long long per_page = (long long)c->n_heads * (c->page_tokens / FLAT_CACHE8_BLOCK);
    if (per_page > kMaxInt || per_page > kMaxInt / c->n_pages) return FLAT_ERR_SHAPE;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return FLAT_ERR_ALIGN;
    const size_t blocks = (size_t)per_page * c->n_pages, codes = blocks * FLAT_CACHE8_BLOCK * c->d, scales = blocks * sizeof(float);
    buf[0] = {c->k, codes};
    buf[1] = {c->v, codes};
    buf[2] = {c->k_scale, scales};
    buf[3] = {c->v_scale, scales};
    for (int i = 0; i < 4; ++i)
        for (int j = i + 1; j < 4; ++j)
            if (overlaps(buf[i], buf[j])) return FLAT_ERR_ALIAS;
    return FLAT_OK;
}

// A page table of `rows` rows over pages of page_tokens tokens: its entries fit 31 bits, and so do its token numbers and those some thousands behind its end, which wavefronts
// that know their blocks in groups look at.
constexpr long long kMaxTokens = kMaxInt - 65536;
bool table_fits(int rows, int max_pages, int page_tokens) {
    return rows > 0 && max_pages > 0 && max_pages <= kMaxTokens / page_tokens && (long long)rows * max_pages <= kMaxInt;
}

int from_hip(hipError_t e) { return e == hipSuccess ? FLAT_OK : FLAT_ERR_HIP; }

}  // namespace

extern "C" {

int flat_attn_rope(const void* Q, void* Q_out, int Hq, const void* K, void* K_out, int Hk, int B, int N, int d, int dtype, int rot_d, int layout,
                   const double* freqs, const int* positions, float magnitude, int transpose, void* stream) {
    if (!Q || !Q_out || !freqs || !K != !K_out) return FLAT_ERR_NULL;
    if (!K) Hk = 0;
    if (Hq <= 0 || (K && Hk <= 0) || B <= 0 || N <= 0) return FLAT_ERR_SHAPE;
    if (!head_dim(d) || rot_d < 2 || rot_d > d || rot_d % 2) return FLAT_ERR_UNSUPPORTED;
    if (dtype != FLAT_DTYPE_BF16 && dtype != FLAT_DTYPE_F32) return FLAT_ERR_UNSUPPORTED;
    if (layout != FLAT_ROPE_HALF && layout != FLAT_ROPE_INTERLEAVED) return FLAT_ERR_UNSUPPORTED;
    if (!isfinite(magnitude)) return FLAT_ERR_UNSUPPORTED;
    if ((long long)B * N > kMaxInt / d || (long long)Hq + Hk > kMaxInt) return FLAT_ERR_SHAPE;
    const unsigned __int128 row = (unsigned __int128)B * (unsigned)N * (unsigned)d * (dtype == FLAT_DTYPE_F32 ? 4 : 2);
    if (row * (unsigned)(Hq > Hk ? Hq : Hk) >= ((unsigned __int128)1 << 62)) return FLAT_ERR_SHAPE;
    if (!aligned(Q, 16) || !aligned(Q_out, 16) || !aligned(K, 16) || !aligned(K_out, 16) || !aligned(freqs, 8) || !aligned(positions, 4)) return FLAT_ERR_ALIGN;
    const Span q{Q, (size_t)row * Hq}, qo{Q_out, q.bytes}, k{K, (size_t)row * Hk}, ko{K_out, k.bytes};
    const Span f{freqs, (size_t)rot_d / 2 * sizeof(double)}, p{positions, ints((long long)B * N)};
    if ((Q != Q_out && overlaps(qo, q)) || (K != K_out && overlaps(ko, k)) || overlaps(qo, k) || overlaps(ko, q) || overlaps(qo, ko)) return FLAT_ERR_ALIAS;
    if (overlaps(qo, f) || overlaps(ko, f) || overlaps(qo, p) || overlaps(ko, p)) return FLAT_ERR_ALIAS;
    const flat::RopeProblem prob{{Q, K}, {Q_out, K_out}, {Hq, Hk}, B, N, d, rot_d, freqs, positions, magnitude, layout == FLAT_ROPE_INTERLEAVED, transpose != 0,
                                 dtype == FLAT_DTYPE_F32};
    return from_hip(flat::launch_rope(prob, static_cast<hipStream_t>(stream)));
}

int flat_attn_cache8_write(const flat_cache8* cache, const void* K, const void* V, int B, int N, const int* page_table, int max_pages, const int* lens,
                           const int* n_new, void* stream) {
    Span buf[4];
    const int rc = check_cache(cache, buf);
    if (rc != FLAT_OK) return rc;
    if (!K || !V || !page_table || !lens) return FLAT_ERR_NULL;
    if (N <= 0 || !table_fits(B, max_pages, cache->page_tokens)) return FLAT_ERR_SHAPE;
    const long long per = (long long)flat::cache8_write_blocks(N) * 2;
    if ((long long)B * cache->n_heads > kMaxInt / per) return FLAT_ERR_SHAPE;  // one wavefront per block, K and V
    if (!aligned(K, 16) || !aligned(V, 16) || !aligned(page_table, 4) || !aligned(lens, 4) || !aligned(n_new, 4)) return FLAT_ERR_ALIGN;
    const size_t bytes = (size_t)B * cache->n_heads * N * cache->d * 2;
    const Span in[5] = {{K, bytes}, {V, bytes}, {page_table, ints((long long)B * max_pages)}, {lens, ints(B)}, {n_new, ints(B)}};
    for (const Span& b : buf)
        if (overlaps_any(b, in)) return FLAT_ERR_ALIAS;
    const flat::CacheWrite w{K, V, B, N, page_table, max_pages, lens, n_new};
    return from_hip(flat::launch_cache8_write(*cache, w, static_cast<hipStream_t>(stream)));
}

// What the attention call can number; its plan on success.
static bool attend_plan(int B, int H, int heads, int Nq, long long max_tokens, int d, flat::Cache8Plan* plan) {
    if (B <= 0 || H <= 0 || heads <= 0 || Nq <= 0 || H % heads || max_tokens <= 0 || max_tokens > kMaxTokens || !head_dim(d)) return false;
    const long long rows = (long long)Nq * (H / heads);
    if (rows > kMaxInt / 2 || (long long)B * heads > kMaxInt / 2 / rows) return false;  // the grids: one workgroup per row in the merge
    if ((unsigned long long)Nq * (unsigned)d * 2u > 0xffffffffULL) return false;
    flat::cache8_plan(B, H, heads, Nq, (int)max_tokens, d, plan);
    const long long grid = plan->limit ? plan->limit : plan->entries;
    return grid * heads <= kMaxInt - 7;
}

size_t flat_attn_fwd_cache8_workspace_bytes(int B, int H, int n_heads, int Nq, int max_tokens, int d) {
    flat::Cache8Plan plan;
    return attend_plan(B, H, n_heads, Nq, max_tokens, d, &plan) ? plan.workspace_bytes : 0;
}

int flat_attn_fwd_cache8(const flat_cache8* cache, const void* Q, void* O, int B, int H, int Nq, const int* page_table, int max_pages, const int* lens,
                         const int* q_lens, float scale, int mask_kind, void* workspace, size_t workspace_bytes, void* stream) {
    Span buf[4];
    const int rc = check_cache(cache, buf);
    if (rc != FLAT_OK) return rc;
    if (!Q || !O || !page_table || !lens) return FLAT_ERR_NULL;
    if (mask_kind != FLAT_MASK_NONE && mask_kind != FLAT_MASK_CAUSAL) return FLAT_ERR_UNSUPPORTED;
    if (!(scale >= 0.0f) || isinf(scale)) return FLAT_ERR_UNSUPPORTED;
    flat::Cache8Plan plan;
    if (!table_fits(B, max_pages, cache->page_tokens)) return FLAT_ERR_SHAPE;
    if (!attend_plan(B, H, cache->n_heads, Nq, (long long)max_pages * cache->page_tokens, cache->d, &plan)) return FLAT_ERR_SHAPE;
    if (!aligned(Q, 16) || !aligned(O, 16) || !aligned(page_table, 4) || !aligned(lens, 4) || !aligned(q_lens, 4)) return FLAT_ERR_ALIGN;
    const size_t bytes = (size_t)B * H * Nq * cache->d * 2;
    const Span in[8] = {buf[0], buf[1], buf[2], buf[3], {Q, bytes}, {page_table, ints((long long)B * max_pages)}, {lens, ints(B)}, {q_lens, ints(B)}};
    const Span out{O, bytes}, ws{workspace, plan.workspace_bytes};
    if (overlaps_any(out, in)) return FLAT_ERR_ALIAS;
    if (plan.workspace_bytes) {
        if (!workspace) return FLAT_ERR_NULL;
        if (!aligned(workspace, 16)) return FLAT_ERR_ALIGN;
        if (workspace_bytes < plan.workspace_bytes) return FLAT_ERR_WORKSPACE;
        if (overlaps(ws, out) || overlaps_any(ws, in)) return FLAT_ERR_ALIAS;
    }
    const flat::Cache8Attend a{Q, O, B, H, Nq, page_table, max_pages, lens, q_lens, scale, mask_kind == FLAT_MASK_CAUSAL, static_cast<float*>(workspace)};
    return from_hip(flat::launch_cache8_fwd(*cache, a, plan, static_cast<hipStream_t>(stream)));
}

int flat_attn_cache8_copy_pages(const flat_cache8* cache, const int* src, const int* dst, int n, void* stream) {
    Span buf[4];
    const int rc = check_cache(cache, buf);
    if (rc != FLAT_OK) return rc;
    if (n < 0) return FLAT_ERR_SHAPE;
    if (n == 0) return FLAT_OK;
    if (!src || !dst) return FLAT_ERR_NULL;
    if (!aligned(src, 4) || !aligned(dst, 4)) return FLAT_ERR_ALIGN;
    for (const Span& b : buf)
        if (overlaps(b, {src, ints(n)}) || overlaps(b, {dst, ints(n)})) return FLAT_ERR_ALIAS;
    return from_hip(flat::launch_cache8_copy(*cache, src, dst, n, static_cast<hipStream_t>(stream)));
}

int flat_attn_cache8_fork(const flat_cache8* cache, int* page_table, int max_pages, int n_seqs, int* lens, const int* parents, const int* children,
                          const int* spares, int n, void* stream) {
    Span buf[4];
    const int rc = check_cache(cache, buf);
    if (rc != FLAT_OK) return rc;
    if (n < 0 || !table_fits(n_seqs, max_pages, cache->page_tokens)) return FLAT_ERR_SHAPE;
    if (!page_table || !lens) return FLAT_ERR_NULL;
    if (n == 0) return FLAT_OK;
    if (!parents || !children || !spares) return FLAT_ERR_NULL;
    if (!aligned(page_table, 4) || !aligned(lens, 4) || !aligned(parents, 4) || !aligned(children, 4) || !aligned(spares, 4)) return FLAT_ERR_ALIGN;
    const Span table{page_table, ints((long long)n_seqs * max_pages)}, len{lens, ints(n_seqs)};
    const Span lists[3] = {{parents, ints(n)}, {children, ints(n)}, {spares, ints(n)}};
    if (overlaps(table, len) || overlaps_any(table, lists) || overlaps_any(len, lists) || overlaps_any(table, buf) || overlaps_any(len, buf)) return FLAT_ERR_ALIAS;
    for (const Span& b : buf)
        if (overlaps_any(b, lists)) return FLAT_ERR_ALIAS;
    return from_hip(flat::launch_cache8_fork(*cache, page_table, max_pages, n_seqs, lens, parents, children, spares, n, static_cast<hipStream_t>(stream)));
}

int flat_attn_cache8_free(int* page_table, int max_pages, int n_seqs, int* lens, const int* seqs, int n, int n_pages, int* unused, int* n_unused, void* stream) {
    if (!page_table || !lens || !unused || !n_unused || (n > 0 && !seqs)) return FLAT_ERR_NULL;
    if (n < 0 || n_pages <= 0 || n_pages > FLAT_CACHE8_MAX_LISTED_PAGES || !table_fits(n_seqs, max_pages, 1)) return FLAT_ERR_SHAPE;
    if (!aligned(page_table, 4) || !aligned(lens, 4) || !aligned(seqs, 4) || !aligned(unused, 4) || !aligned(n_unused, 4)) return FLAT_ERR_ALIGN;
    const Span all[5] = {{page_table, ints((long long)n_seqs * max_pages)}, {lens, ints(n_seqs)}, {unused, ints(n_pages)}, {n_unused, ints(1)}, {seqs, ints(n)}};
    for (int i = 0; i < 5; ++i)
        for (int j = i + 1; j < 5; ++j)
            if (overlaps(all[i], all[j])) return FLAT_ERR_ALIAS;
    return from_hip(flat::launch_cache8_free(page_table, max_pages, n_seqs, lens, seqs, n, n_pages, unused, n_unused, static_cast<hipStream_t>(stream)));
}

size_t flat_attn_cache8_compact_workspace_bytes(int n_pages) {
    if (n_pages <= 0 || n_pages > FLAT_CACHE8_MAX_LISTED_PAGES) return 0;
    return ints(3LL * n_pages + 1);
}

int flat_attn_cache8_compact(const flat_cache8* cache, const int* page_table, int* new_table, int max_pages, int n_seqs, int* n_used, void* workspace,
                             size_t workspace_bytes, void* stream) {
    Span buf[4];
    const int rc = check_cache(cache, buf);
    if (rc != FLAT_OK) return rc;
    if (!page_table || !new_table || !n_used || !workspace) return FLAT_ERR_NULL;
    if (cache->n_pages > FLAT_CACHE8_MAX_LISTED_PAGES || !table_fits(n_seqs, max_pages, cache->page_tokens)) return FLAT_ERR_SHAPE;
    if (!aligned(page_table, 4) || !aligned(new_table, 4) || !aligned(n_used, 4) || !aligned(workspace, 4)) return FLAT_ERR_ALIGN;
    const size_t need = flat_attn_cache8_compact_workspace_bytes(cache->n_pages);
    if (workspace_bytes < need) return FLAT_ERR_WORKSPACE;
    const size_t table_bytes = ints((long long)n_seqs * max_pages);
    const Span in{page_table, table_bytes}, out{new_table, table_bytes}, used{n_used, ints(1)}, ws{workspace, need};
    if (page_table != new_table && overlaps(in, out)) return FLAT_ERR_ALIAS;
    if (overlaps(used, in) || overlaps(used, out) || overlaps(used, ws) || overlaps(ws, in) || overlaps(ws, out)) return FLAT_ERR_ALIAS;
    if (overlaps_any(in, buf) || overlaps_any(out, buf) || overlaps_any(used, buf) || overlaps_any(ws, buf)) return FLAT_ERR_ALIAS;
    return from_hip(flat::launch_cache8_compact(*cache, page_table, new_table, max_pages, n_seqs, n_used, static_cast<int*>(workspace), static_cast<hipStream_t>(stream)));
}

}  // extern "C"
