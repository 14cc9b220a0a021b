// What the cache operators share: the checked arguments of a call, a request's chunk, the paged cache's
// addresses, a tree node's ancestors.
#pragma once

#include "hvd_internal.cuh"

namespace hvd {

constexpr int kTileRows = 128;   // query rows of one tensor-core tile (a row = one token's query head of a group)
constexpr int kTileKeys = 64;    // keys of one tile
constexpr int kTreeRows = 65;    // rows of the largest token tree (k_cap <= 64 nodes and the root)

// One call's chunks and cache, as checked on the host.
struct ChunkArgs {
    int32_t B;
    int32_t k_cap;
    const int32_t* cache_len;
    const int64_t* row_off;  // NULL: k_uniform + 1 rows each
    int32_t k_uniform;
    int64_t total_rows;
    const int32_t* sel_len;  // NULL: every row is a new token
    const int32_t* parent;   // NULL: chains
    // the cache
    char* k;
    char* v;
    int64_t n_pages;
    int32_t page_size;
    int32_t table_stride;
    const int32_t* page_table;
    int64_t page_stride, slot_stride, head_stride;  // in elements (16 bits each)
    int* dev_error;
};

struct Chunk {
    int64_t r0;  // first row
    int rows;    // rows of the request
    int n_new;   // ... that are new tokens (0: the request is skipped, or empty)
    int base;    // tokens cached before the chunk
    bool bad;    // HVD_REQ_BAD_LEN
};

#ifdef __CUDACC__

__device__ __forceinline__ Chunk load_chunk(const ChunkArgs& a, int b) {
    Chunk c;
    int64_t r1;
    if (a.row_off) { c.r0 = a.row_off[b]; r1 = a.row_off[b + 1]; }
    else { c.r0 = (int64_t)b * (a.k_uniform + 1); r1 = c.r0 + a.k_uniform + 1; }
    const int n = a.cache_len[b];
    const int sl = a.sel_len ? a.sel_len[b] : 0;
    c.base = n;
    c.bad = c.r0 < 0 || r1 > a.total_rows || r1 < c.r0;
    if (c.bad) { c.r0 = 0; r1 = 0; }
    c.rows = (int)(r1 - c.r0);
    int m = c.rows;
    if (a.sel_len) {
        m = min(max(0, min(sl, a.k_cap)) + 1, c.rows);
        c.bad = c.bad || c.rows == 0;
    }
    c.bad = c.bad || n < 0 || (int64_t)n + m > (int64_t)a.table_stride * a.page_size;
    c.n_new = c.bad ? 0 : m;
    if (c.bad) c.base = 0;
    return c;
}

// The line from row i of a tree chunk up to the root: the nodes on it as bits (node j = row j + 1) and its length.
// false: the line leaves {-1, 0 .. i-1} and the row is unreachable.
__device__ __forceinline__ bool tree_line(const ChunkArgs& a, int b, int i, unsigned long long& nodes, int& depth) {
    nodes = 0ull;
    depth = 0;
    int cur = i - 1;
    const int32_t* par = a.parent + (int64_t)b * a.k_cap;
    while (cur >= 0) {  // strictly decreasing: at most k_cap steps
        nodes |= 1ull << cur;
        ++depth;
        const int p = HVD_IN_BOUNDS(a.dev_error, cur, 0, a.k_cap) ? par[cur] : -1;
        if (p < -1 || p >= cur) { nodes = 0ull; depth = 0; return false; }
        cur = p;
    }
    return true;
}

// The page of token t of request b, -1 if the entry lies outside the pool.
__device__ __forceinline__ int64_t page_of(const ChunkArgs& a, int b, int t) {
    const int j = t / a.page_size;
    if (!HVD_IN_BOUNDS(a.dev_error, j, 0, a.table_stride)) return -1;
    const int64_t p = a.page_table[(int64_t)b * a.table_stride + j];
    return p >= 0 && p < a.n_pages ? p : -1;
}

__device__ __forceinline__ int64_t slot_offset(const ChunkArgs& a, int64_t page, int t) {
    return page * a.page_stride + (int64_t)(t % a.page_size) * a.slot_stride;
}

#endif

struct HeadsArgs {
    char* p;
    int64_t row_stride, head_stride;
};

struct RopeArgs {
    ChunkArgs c;
    HeadsArgs q, k, v, q_out;
    int32_t n_q_heads, n_kv_heads, head_dim, rot_dim;
    const unsigned long long* turns;  // [rot_dim / 2] angular frequency in 2^-64 turns per position
    float magnitude;
    int32_t* status;
};

struct AttnArgs {
    ChunkArgs c;
    HeadsArgs q, out;
    float* lse;
    int32_t* status;
    int32_t n_q_heads, n_kv_heads, group, head_dim;
    float scale_log2;  // softmax_scale * log2(e)
};

struct KvCommitArgs {
    ChunkArgs c;  // cache, cache_len, parent, sel_len, k_cap, B
    int32_t n_layers, n_kv_heads, head_dim;
    int64_t layer_stride;
    const int32_t* sel_draft;
    const int32_t* accepted;
    const int32_t* committed;
    const int32_t* n_commit;
    int32_t* new_len;
    int32_t* status;    // may be NULL
    bool in_place;      // new_len is cache_len
    uint32_t* arrived;  // [max_batch], zero at rest
};

hvd_status launch_rope_append(hvd_ctx* ctx, const RopeArgs& a, bool f16, int layout, cudaStream_t stream);
size_t attn_workspace_bytes(int num_sms, int head_dim);
hvd_status attn_setup(hvd_ctx* ctx);  // per-device opt-ins of the attention kernels
hvd_status launch_attn(hvd_ctx* ctx, const AttnArgs& a, bool f16, cudaStream_t stream);
hvd_status launch_kv_commit(hvd_ctx* ctx, const KvCommitArgs& a, cudaStream_t stream);

}  // namespace hvd
