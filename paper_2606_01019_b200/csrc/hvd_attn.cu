// hvd_attn_paged: attention of a chunk's rows over the paged cache.
//
// One warp per (row, query head) walks the keys that the row sees with the running maximum and sum of a softmax;
// lanes split the head.
#include "hvd_attn.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace hvd {

namespace {

template <typename E>
__global__ void __launch_bounds__(256) attn_rows_kernel(const AttnArgs a) {
    const ChunkArgs& c = a.c;
    const int b = blockIdx.x, lane = threadIdx.x & 31;
    pdl_trigger();
    pdl_wait();
    const Chunk ch = load_chunk(c, b);
    if (a.status && blockIdx.y == 0 && threadIdx.x == 0) a.status[b] = ch.bad ? HVD_REQ_BAD_LEN : HVD_REQ_OK;
    const int64_t items = (int64_t)ch.rows * a.n_q_heads;
    for (int64_t w = (int64_t)blockIdx.y * 8 + (threadIdx.x >> 5); w < items; w += (int64_t)gridDim.y * 8) {
        const int i = (int)(w / a.n_q_heads), h = (int)(w % a.n_q_heads), hk = h / a.group;
        const int64_t row = ch.r0 + i;
        unsigned long long nodes = 0ull;
        int depth = 0;
        bool sees = i < ch.n_new;
        if (sees && c.parent) sees = tree_line(c, b, i, nodes, depth);
        const E* q = reinterpret_cast<const E*>(a.q.p) + row * a.q.row_stride + (int64_t)h * a.q.head_stride;
        float qf[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) qf[k] = lane + 32 * k < a.head_dim ? (float)q[lane + 32 * k] * a.scale_log2 : 0.f;
        const int end = sees ? ch.base + i + 1 : 0;
        for (int t = 0; t < end; ++t) {
            const int node = t - ch.base - 1;  // >= 0: a node of the chunk
            if (c.parent && node >= 0 && !((nodes >> node) & 1ull)) continue;
            const int64_t page = page_of(c, b, t);
            const int64_t off = page < 0 ? 0 : slot_offset(c, page, t) + (int64_t)hk * c.head_stride;
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (page >= 0 && lane + 32 * k < a.head_dim) s += qf[k] * (float)(reinterpret_cast<const E*>(c.k) + off)[lane + 32 * k];
#pragma unroll
            for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
            const float top = fmaxf(m, s), f = exp2f(m - top), p = exp2f(s - top);
            m = top;
            l = l * f + p;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (lane + 32 * k < a.head_dim)
                    o[k] = o[k] * f + (page >= 0 ? p * (float)(reinterpret_cast<const E*>(c.v) + off)[lane + 32 * k] : 0.f);
        }
        E* out = reinterpret_cast<E*>(a.out.p) + row * a.out.row_stride + (int64_t)h * a.out.head_stride;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (lane + 32 * k < a.head_dim) out[lane + 32 * k] = (E)(l > 0.f ? o[k] / l : 0.f);
        if (a.lse && lane == 0) a.lse[row * a.n_q_heads + h] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    }
}

}  // namespace

hvd_status launch_attn(hvd_ctx* ctx, const AttnArgs& a, bool f16, cudaStream_t stream) {
    const bool pdl = (ctx->pdl_mask & 16) != 0;
    const dim3 grid((unsigned)a.c.B, 256);
    const cudaError_t e = f16 ? launch_kernel(pdl, attn_rows_kernel<__half>, grid, dim3(256), 0, stream, a)
                              : launch_kernel(pdl, attn_rows_kernel<__nv_bfloat16>, grid, dim3(256), 0, stream, a);
    return e == cudaSuccess ? HVD_OK : cuda_fail(ctx, e, "attn_rows_kernel");
}

}  // namespace hvd
