// C ABI of the cache operators: attention set-up, rotary frequencies, argument checks.
#include <math.h>

#include "hvd_attn.cuh"

using namespace hvd;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// NULL if the configuration can be used, else what is wrong with it
const char* config_fault(const hvd_attn_config& c) {
    if (c.n_kv_heads < 1 || c.n_q_heads < 1 || c.n_q_heads % c.n_kv_heads != 0) return "n_q_heads must be a multiple of n_kv_heads >= 1";
    if (c.n_q_heads / c.n_kv_heads > HVD_MAX_HEAD_GROUP) return "more than HVD_MAX_HEAD_GROUP query heads per key/value head";
    if (c.n_kv_heads > 4096) return "n_kv_heads above 4096";
    if (c.head_dim < 8 || c.head_dim > HVD_MAX_HEAD_DIM || c.head_dim % 8 != 0) return "head_dim must be a multiple of 8 in [8, HVD_MAX_HEAD_DIM]";
    if (c.dtype != HVD_BF16 && c.dtype != HVD_F16) return "dtype must be HVD_BF16 or HVD_F16";
    if (!(c.softmax_scale >= 0.0f) || isinf(c.softmax_scale)) return "softmax_scale must be finite and >= 0";
    if (c.rot_dim < 0 || c.rot_dim > c.head_dim || c.rot_dim % 2 != 0) return "rot_dim must be even, in [0, head_dim]";
    if (c.rot_layout != HVD_ROPE_HALVES && c.rot_layout != HVD_ROPE_PAIRS) return "unknown rot_layout";
    if (c.rope_scaling < HVD_ROPE_PLAIN || c.rope_scaling > HVD_ROPE_BANDS) return "unknown rope_scaling";
    if (!(c.rope_magnitude >= 0.0) || isinf(c.rope_magnitude)) return "rope_magnitude must be finite and >= 0";
    if (c.rot_dim == 0) return nullptr;
    if (!(c.rope_base > 1.0) || isinf(c.rope_base)) return "rope_base must be finite and above 1";
    if (c.rope_scaling != HVD_ROPE_PLAIN && (!(c.rope_factor >= 1.0) || isinf(c.rope_factor))) return "rope_factor must be finite and >= 1";
    if (c.rope_scaling == HVD_ROPE_BASE && c.rot_dim < 4) return "HVD_ROPE_BASE needs rot_dim above 2";
    if (c.rope_scaling >= HVD_ROPE_PARTS) {
        if (!(c.rope_original_len > 0.0) || isinf(c.rope_original_len)) return "rope_original_len must be finite and above 0";
        if (!(c.rope_low > 0.0) || !(c.rope_high > c.rope_low) || isinf(c.rope_high)) return "0 < rope_low < rope_high is needed";
    }
    return nullptr;
}

constexpr double kTwoPi = 6.283185307179586476925286766559;

void frequencies(const hvd_attn_config& c, double* freq) {
    const double rot = c.rot_dim, L = c.rope_original_len;
    const double base = c.rope_scaling == HVD_ROPE_BASE ? c.rope_base * pow(c.rope_factor, rot / (rot - 2.0)) : c.rope_base;
    double lo = 0.0, hi = 0.0;
    if (c.rope_scaling == HVD_ROPE_PARTS) {
        // pair i makes L * base^(-2i/rot) / 2pi turns within L positions: solved for i
        lo = fmax(floor(rot * log(L / (c.rope_high * kTwoPi)) / (2.0 * log(base))), 0.0);
        hi = fmin(ceil(rot * log(L / (c.rope_low * kTwoPi)) / (2.0 * log(base))), rot - 1.0);
    }
    for (int i = 0; i < c.rot_dim / 2; ++i) {
        const double w = pow(base, -2.0 * i / rot);
        double keep = 1.0;  // the share of the unscaled frequency
        if (c.rope_scaling == HVD_ROPE_LINEAR) keep = 0.0;
        if (c.rope_scaling == HVD_ROPE_PARTS) keep = 1.0 - fmin(fmax((i - lo) / fmax(hi - lo, 1e-3), 0.0), 1.0);
        if (c.rope_scaling == HVD_ROPE_BANDS) keep = fmin(fmax((L * w / kTwoPi - c.rope_low) / (c.rope_high - c.rope_low), 0.0), 1.0);
        freq[i] = keep == 1.0 ? w : w * keep + (w / c.rope_factor) * (1.0 - keep);
    }
}

const char* heads_fault(const hvd_heads& h, int64_t total_rows) {
    if (!h.p && total_rows > 0) return "NULL pointer";
    if (!aligned16(h.p)) return "the rows of heads must be 16-byte aligned";
    if (h.row_stride <= 0 || h.head_stride <= 0 || h.row_stride % 8 != 0 || h.head_stride % 8 != 0)
        return "row and head strides must be positive multiples of 8";
    return nullptr;
}

HeadsArgs heads(const hvd_heads& h) { return HeadsArgs{static_cast<char*>(h.p), h.row_stride, h.head_stride}; }

hvd_status fail_at(hvd_ctx* ctx, hvd_status s, const char* where, const char* what) {
    snprintf(ctx->last_error, sizeof(ctx->last_error), "%s: %s", where, what);
    return s;
}

// what the three operators check alike
const char* cache_fault(hvd_ctx* ctx, int32_t B, const hvd_kv_cache* c, const int32_t* cache_len) {
    if (!ctx->has_attention) return "call hvd_set_attention first";
    if (B < 1 || B > ctx->cfg.max_batch) return "B outside [1, max_batch]";
    if (!c || !c->k || !c->v || !c->page_table || !cache_len) return "NULL pointer";
    if (!aligned16(c->k) || !aligned16(c->v)) return "the cache must be 16-byte aligned";
    if (c->n_pages < 1 || c->n_pages > 0x7fffffffLL) return "n_pages outside [1, 2^31 - 1]";
    if (c->page_size < 8 || c->page_size > 65536 || c->page_size % 8 != 0) return "page_size must be a multiple of 8 in [8, 65536]";
    if (c->table_stride < 1 || (int64_t)c->table_stride * c->page_size > 0x7fffffffLL) return "table_stride * page_size outside [1, 2^31 - 1]";
    for (int64_t s : {c->page_stride, c->slot_stride, c->head_stride})
        if (s <= 0 || s % 8 != 0) return "cache strides must be positive multiples of 8";
    return nullptr;
}

const char* chunk_fault(hvd_ctx* ctx, const int64_t* row_off, int32_t k_uniform, int64_t total_rows, int32_t B,
                        const int32_t* sel_len, const int32_t* parent) {
    if (total_rows < 0 || total_rows > ctx->cfg.max_rows) return "total_rows outside [0, max_rows]";
    if (!row_off && (k_uniform < 0 || (int64_t)B * ((int64_t)k_uniform + 1) > total_rows)) return "k_uniform and total_rows do not fit";
    if (parent && !sel_len) return "parent needs sel_len";
    return nullptr;
}

ChunkArgs chunk_args(hvd_ctx* ctx, int32_t B, const hvd_kv_cache& c, const int32_t* cache_len, const int64_t* row_off,
                     int32_t k_uniform, int64_t total_rows, const int32_t* sel_len, const int32_t* parent) {
    ChunkArgs a = {};
    a.B = B; a.k_cap = ctx->cfg.k_cap; a.cache_len = cache_len;
    a.row_off = row_off; a.k_uniform = k_uniform; a.total_rows = total_rows;
    a.sel_len = sel_len; a.parent = parent;
    a.k = static_cast<char*>(c.k); a.v = static_cast<char*>(c.v);
    a.n_pages = c.n_pages; a.page_size = c.page_size; a.table_stride = c.table_stride; a.page_table = c.page_table;
    a.page_stride = c.page_stride; a.slot_stride = c.slot_stride; a.head_stride = c.head_stride;
    a.dev_error = ctx->dev_error;
    return a;
}

}  // namespace

extern "C" {

hvd_status hvd_rope_frequencies(const hvd_attn_config* cfg, double* freq, double* magnitude) {
    if (!cfg || !freq || !magnitude || config_fault(*cfg)) return HVD_ERR_INVALID_ARG;
    frequencies(*cfg, freq);
    *magnitude = cfg->rope_magnitude > 0.0 ? cfg->rope_magnitude : 1.0;
    return HVD_OK;
}

hvd_status hvd_set_attention(hvd_ctx* ctx, const hvd_attn_config* cfg) {
    if (!ctx) return HVD_ERR_INVALID_ARG;
    if (!cfg) return fail(ctx, HVD_ERR_INVALID_ARG, "hvd_set_attention: NULL pointer");
    if (const char* w = config_fault(*cfg)) return fail_at(ctx, HVD_ERR_INVALID_ARG, "hvd_set_attention", w);
    double freq[HVD_MAX_HEAD_DIM / 2];
    unsigned long long turns[HVD_MAX_HEAD_DIM / 2] = {};
    frequencies(*cfg, freq);
    for (int i = 0; i < cfg->rot_dim / 2; ++i) {
        // radians per position to 2^-64 turns per position; frequencies are at most 1, a turn is 2 pi
        const double t = freq[i] / kTwoPi;
        turns[i] = (unsigned long long)(t * 18446744073709551616.0);
    }
    ctx->has_attention = false;
    HVD_CUDA_TRY(ctx, cudaDeviceSynchronize());
    const hvd_status st = attn_setup(ctx);
    if (st != HVD_OK) return st;
    // once, for the widest heads: graphs that were captured under an earlier geometry hold its address
    if (!ctx->at_ws && cudaMalloc(&ctx->at_ws, attn_workspace_bytes(ctx->num_sms, HVD_MAX_HEAD_DIM)) != cudaSuccess) {
        ctx->at_ws = nullptr;
        (void)cudaGetLastError();
        return fail(ctx, HVD_ERR_ALLOC, "hvd_set_attention: out of device memory for the scratch");
    }
    if (!ctx->at_turns) HVD_CUDA_TRY(ctx, cudaMalloc(&ctx->at_turns, sizeof(turns)));
    HVD_CUDA_TRY(ctx, cudaMemcpy(ctx->at_turns, turns, sizeof(turns), cudaMemcpyHostToDevice));
    if (!ctx->at_arrived) {
        HVD_CUDA_TRY(ctx, cudaMalloc(&ctx->at_arrived, (size_t)ctx->cfg.max_batch * sizeof(uint32_t)));
        HVD_CUDA_TRY(ctx, cudaMemset(ctx->at_arrived, 0, (size_t)ctx->cfg.max_batch * sizeof(uint32_t)));
        HVD_CUDA_TRY(ctx, cudaDeviceSynchronize());
    }
    ctx->attn = *cfg;
    if (ctx->attn.softmax_scale == 0.0f) ctx->attn.softmax_scale = (float)(1.0 / sqrt((double)cfg->head_dim));
    if (ctx->attn.rope_magnitude == 0.0) ctx->attn.rope_magnitude = 1.0;
    ctx->has_attention = true;
    return HVD_OK;
}

hvd_status hvd_rope_append(hvd_ctx* ctx, int32_t B, const hvd_kv_cache* cache, const int32_t* cache_len,
                           const int64_t* row_off, int32_t k_uniform, int64_t total_rows, const int32_t* sel_len,
                           const int32_t* parent, const hvd_heads* q, const hvd_heads* k, const hvd_heads* v,
                           const hvd_heads* q_out, int32_t* status, void* stream) {
    static const char* who = "hvd_rope_append";
    if (!ctx) return HVD_ERR_INVALID_ARG;
    if (const char* w = cache_fault(ctx, B, cache, cache_len)) return fail_at(ctx, HVD_ERR_INVALID_ARG, who, w);
    if (const char* w = chunk_fault(ctx, row_off, k_uniform, total_rows, B, sel_len, parent))
        return fail_at(ctx, HVD_ERR_INVALID_ARG, who, w);
    if (!q || !k || !v || !q_out || !status) return fail_at(ctx, HVD_ERR_INVALID_ARG, who, "NULL pointer");
    for (const hvd_heads* h : {q, k, v, q_out})
        if (const char* w = heads_fault(*h, total_rows)) return fail_at(ctx, HVD_ERR_INVALID_ARG, who, w);
    if (q_out->p == q->p && (q_out->row_stride != q->row_stride || q_out->head_stride != q->head_stride))
        return fail_at(ctx, HVD_ERR_INVALID_ARG, who, "q_out in the place of q needs the same strides");
    RopeArgs a = {};
    a.c = chunk_args(ctx, B, *cache, cache_len, row_off, k_uniform, total_rows, sel_len, parent);
    a.q = heads(*q); a.k = heads(*k); a.v = heads(*v); a.q_out = heads(*q_out);
    a.n_q_heads = ctx->attn.n_q_heads; a.n_kv_heads = ctx->attn.n_kv_heads;
    a.head_dim = ctx->attn.head_dim; a.rot_dim = ctx->attn.rot_dim;
    a.turns = ctx->at_turns; a.magnitude = (float)ctx->attn.rope_magnitude; a.status = status;
    return launch_rope_append(ctx, a, ctx->attn.dtype == HVD_F16, ctx->attn.rot_layout, static_cast<cudaStream_t>(stream));
}

hvd_status hvd_attn_paged(hvd_ctx* ctx, int32_t B, const hvd_kv_cache* cache, const int32_t* cache_len,
                          const int64_t* row_off, int32_t k_uniform, int64_t total_rows, const int32_t* sel_len,
                          const int32_t* parent, const hvd_heads* q, const hvd_heads* out, float* lse, int32_t* status,
                          void* stream) {
    static const char* who = "hvd_attn_paged";
    if (!ctx) return HVD_ERR_INVALID_ARG;
    if (const char* w = cache_fault(ctx, B, cache, cache_len)) return fail_at(ctx, HVD_ERR_INVALID_ARG, who, w);
    if (const char* w = chunk_fault(ctx, row_off, k_uniform, total_rows, B, sel_len, parent))
        return fail_at(ctx, HVD_ERR_INVALID_ARG, who, w);
    if (!q || !out) return fail_at(ctx, HVD_ERR_INVALID_ARG, who, "NULL pointer");
    for (const hvd_heads* h : {q, out})
        if (const char* w = heads_fault(*h, total_rows)) return fail_at(ctx, HVD_ERR_INVALID_ARG, who, w);
    if (q->p == out->p && total_rows > 0) return fail_at(ctx, HVD_ERR_INVALID_ARG, who, "out must be another array than q");
    AttnArgs a = {};
    a.c = chunk_args(ctx, B, *cache, cache_len, row_off, k_uniform, total_rows, sel_len, parent);
    a.q = heads(*q); a.out = heads(*out); a.lse = lse; a.status = status;
    a.n_q_heads = ctx->attn.n_q_heads; a.n_kv_heads = ctx->attn.n_kv_heads;
    a.group = a.n_q_heads / a.n_kv_heads; a.head_dim = ctx->attn.head_dim;
    a.scale_log2 = (float)(ctx->attn.softmax_scale * 1.4426950408889634);
    if (total_rows == 0 && !status) return HVD_OK;
    return launch_attn(ctx, a, ctx->attn.dtype == HVD_F16, static_cast<cudaStream_t>(stream));
}

hvd_status hvd_kv_commit(hvd_ctx* ctx, int32_t B, const hvd_kv_cache* cache, int32_t n_layers, int64_t layer_stride,
                         const int32_t* cache_len, const int32_t* parent, const int32_t* sel_draft,
                         const int32_t* sel_len, const int32_t* accepted, const int32_t* committed,
                         const int32_t* n_commit, int32_t* new_len, void* stream) {
    return hvd_kv_commit_checked(ctx, B, cache, n_layers, layer_stride, cache_len, parent, sel_draft, sel_len, accepted, committed,
                                 n_commit, new_len, nullptr, stream);
}

hvd_status hvd_kv_commit_checked(hvd_ctx* ctx, int32_t B, const hvd_kv_cache* cache, int32_t n_layers, int64_t layer_stride,
                                 const int32_t* cache_len, const int32_t* parent, const int32_t* sel_draft,
                                 const int32_t* sel_len, const int32_t* accepted, const int32_t* committed,
                                 const int32_t* n_commit, int32_t* new_len, int32_t* status, void* stream) {
    static const char* who = "hvd_kv_commit";
    if (!ctx) return HVD_ERR_INVALID_ARG;
    if (const char* w = cache_fault(ctx, B, cache, cache_len)) return fail_at(ctx, HVD_ERR_INVALID_ARG, who, w);
    if (!n_commit || !new_len || (parent && (!sel_draft || !sel_len || !accepted || !committed)))
        return fail_at(ctx, HVD_ERR_INVALID_ARG, who, "NULL pointer");
    if (n_layers < 1 || n_layers > 4096) return fail_at(ctx, HVD_ERR_INVALID_ARG, who, "n_layers outside [1, 4096]");
    if (layer_stride % 8 != 0 || (n_layers > 1 && layer_stride <= 0))
        return fail_at(ctx, HVD_ERR_INVALID_ARG, who, "layer_stride must be a positive multiple of 8");
    KvCommitArgs a = {};
    a.c = chunk_args(ctx, B, *cache, cache_len, nullptr, 0, 0, sel_len, parent);
    a.n_layers = n_layers; a.n_kv_heads = ctx->attn.n_kv_heads; a.head_dim = ctx->attn.head_dim;
    a.layer_stride = layer_stride;
    a.sel_draft = sel_draft; a.accepted = accepted; a.committed = committed; a.n_commit = n_commit; a.new_len = new_len; a.status = status; a.in_place = new_len == cache_len;
    a.arrived = ctx->at_arrived;
    return launch_kv_commit(ctx, a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
