// hvd_rope_append: rotary positions on the new tokens' queries and keys, keys and values into the paged cache.
//
// A pair (x, y) of a head turns by the angle a = t * w at position t.  The frequency is held in units of 2^-64
// turns, so that t * w modulo one turn is an integer product that wraps: exact at every position, where a
// 32-bit float product is off by thousandths of a radian from position 10^5 on.  The upper 32 bits go to sincospi.
//
// Bandwidth: every element is read once and written once.  A CTA takes a few tokens: their sines and cosines (the same
// for all heads) are computed once into shared memory, then 16-byte vectors stream through, a thread keeping its
// place inside the head and stepping over the heads, so that no index is divided in the loop.
#include "hvd_attn.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace hvd {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 4;   // tokens of a CTA, large calls

template <typename E> __device__ __forceinline__ float2 widen2(uint32_t w);
template <> __device__ __forceinline__ float2 widen2<__nv_bfloat16>(uint32_t w) {
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w));
}
template <> __device__ __forceinline__ float2 widen2<__half>(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <typename E> __device__ __forceinline__ uint32_t narrow2(float x, float y);
template <> __device__ __forceinline__ uint32_t narrow2<__nv_bfloat16>(float x, float y) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t narrow2<__half>(float x, float y) {
    const __half2 v = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename E> __device__ __forceinline__ float widen(E x) { return (float)x; }

struct Token {
    int64_t row;
    int64_t kv;   // element offset of its cache slot, -1: not cached
    int b;        // -1: not a new token
};

// The request of a row: the last one whose rows start at or before it.  All threads of the CTA count starts.
__device__ __forceinline__ int request_of(const ChunkArgs& c, int64_t row) {
    if (!c.row_off) return (int)min(row / (c.k_uniform + 1), (int64_t)c.B);
    int lo = 0, hi = c.B;  // row_off[lo] <= row < row_off[hi], as far as the offsets ascend
    while (hi - lo > 1) {
        const int step = (hi - lo + (int)blockDim.x) / (int)blockDim.x;
        const int at = lo + ((int)threadIdx.x + 1) * step;
        const int n = __syncthreads_count(at < hi && c.row_off[at] <= row);
        lo += n * step;
        hi = min(hi, lo + step);
        if (step == 1) break;
    }
    return lo;
}

// One vector of 8 elements, both layouts: `w` turns with `other` (HALVES) or within itself (PAIRS).
template <typename E>
__device__ __forceinline__ void turn_halves(uint4& x, uint4& y, const float2* cs) {
    uint32_t* xa = &x.x;
    uint32_t* ya = &y.x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 a = widen2<E>(xa[j]), b = widen2<E>(ya[j]);
        const float2 c0 = cs[2 * j], c1 = cs[2 * j + 1];
        xa[j] = narrow2<E>(a.x * c0.x - b.x * c0.y, a.y * c1.x - b.y * c1.y);
        ya[j] = narrow2<E>(a.x * c0.y + b.x * c0.x, a.y * c1.y + b.y * c1.x);
    }
}

template <typename E>
__device__ __forceinline__ void turn_pairs(uint4& x, const float2* cs, int n) {
    uint32_t* xa = &x.x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (j < n) {
            const float2 a = widen2<E>(xa[j]);
            const float2 c = cs[j];
            xa[j] = narrow2<E>(a.x * c.x - a.y * c.y, a.x * c.y + a.y * c.x);
        }
    }
}

template <typename E, int LAYOUT>
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const RopeArgs a, const int tokens_per_cta) {
    __shared__ Token tok[kRopeTokens];
    __shared__ __align__(16) float2 cs[kRopeTokens][HVD_MAX_HEAD_DIM / 2];
    __shared__ int pos[kRopeTokens];
    const ChunkArgs& c = a.c;
    pdl_trigger();
    pdl_wait();
    const int n_token_ctas = (int)((c.total_rows + tokens_per_cta - 1) / tokens_per_cta);
    if ((int)blockIdx.x >= n_token_ctas) {  // the requests' verdicts, a warp each
        const int b = ((int)blockIdx.x - n_token_ctas) * (kRopeThreads / 32) + ((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
        if (b >= c.B) return;
        const Chunk ch = load_chunk(c, b);
        bool outside = false;
        if (ch.n_new > 0)
            for (int j = ch.base / c.page_size + lane; j <= (ch.base + ch.n_new - 1) / c.page_size; j += 32)
                outside = outside || page_of(c, b, j * c.page_size) < 0;
        outside = __any_sync(0xffffffffu, outside);
        if (lane == 0) a.status[b] = ch.bad ? HVD_REQ_BAD_LEN : (outside ? HVD_REQ_BAD_PAGE : HVD_REQ_OK);
        return;
    }
    const int64_t first = (int64_t)blockIdx.x * tokens_per_cta;
    const int b0 = request_of(c, first);
    if ((int)threadIdx.x < tokens_per_cta) {
        const int i = threadIdx.x;
        Token t = {first + i, -1, -1};
        if (t.row < c.total_rows) {
            int b = b0;
            if (c.row_off) while (b + 1 < c.B && c.row_off[b + 1] <= t.row) ++b;
            else b = (int)min(t.row / (c.k_uniform + 1), (int64_t)c.B);
            if (b < c.B) {
                const Chunk ch = load_chunk(c, b);
                const int64_t at = t.row - ch.r0;
                if (!ch.bad && at >= 0 && at < ch.n_new) {
                    t.b = b;
                    const int p = ch.base + (int)at;
                    const int64_t page = page_of(c, b, p);
                    if (page >= 0) t.kv = slot_offset(c, page, p);
                    int depth = (int)at;
                    unsigned long long nodes;
                    if (c.parent) tree_line(c, b, (int)at, nodes, depth);
                    pos[i] = ch.base + depth;
                }
            }
        }
        tok[i] = t;
    }
    __syncthreads();
    const int half = a.rot_dim / 2;
    for (int i = threadIdx.x; i < tokens_per_cta * half; i += blockDim.x) {
        const int t = i / half, j = i - t * half;
        if (tok[t].b >= 0) {
            const unsigned long long turn = (unsigned long long)pos[t] * a.turns[j];  // modulo one turn
            float s, co;
            sincospif((float)(int32_t)(turn >> 32) * 4.656612873077393e-10f, &s, &co);  // 2^-31: turns to half turns
            cs[t][j] = make_float2(co * a.magnitude, s * a.magnitude);
        }
    }
    __syncthreads();

    const int D = a.head_dim, nvec = D / 8;
    const bool whole = LAYOUT == HVD_ROPE_PAIRS || half % 8 == 0;  // pairs lie in whole 16-byte vectors
    const int n_turned = a.n_q_heads + a.n_kv_heads;
    for (int t = 0; t < tokens_per_cta; ++t) {
        const Token tk = tok[t];
        if (tk.b < 0) continue;
        // queries and keys: `units` pieces per head
        const int units = LAYOUT == HVD_ROPE_PAIRS ? nvec : (whole ? half / 8 + (D - a.rot_dim) / 8 : half + (D - a.rot_dim));
        const int per = (int)blockDim.x / units;  // heads side by side
        const int u = (int)threadIdx.x % units, h0 = (int)threadIdx.x / units;
        for (int h = h0; h < n_turned && h0 < per; h += per) {
            const bool isq = h < a.n_q_heads;
            const int hk = h - a.n_q_heads;
            if (!isq && tk.kv < 0) continue;
            const E* src = isq ? reinterpret_cast<const E*>(a.q.p) + tk.row * a.q.row_stride + (int64_t)h * a.q.head_stride
                               : reinterpret_cast<const E*>(a.k.p) + tk.row * a.k.row_stride + (int64_t)hk * a.k.head_stride;
            E* dst = isq ? reinterpret_cast<E*>(a.q_out.p) + tk.row * a.q_out.row_stride + (int64_t)h * a.q_out.head_stride
                         : reinterpret_cast<E*>(c.k) + tk.kv + (int64_t)hk * c.head_stride;
            if (LAYOUT == HVD_ROPE_PAIRS) {
                uint4 x = *reinterpret_cast<const uint4*>(src + 8 * u);
                turn_pairs<E>(x, &cs[t][min(4 * u, HVD_MAX_HEAD_DIM / 2 - 4)], half - 4 * u);
                *reinterpret_cast<uint4*>(dst + 8 * u) = x;
            } else if (whole) {
                if (u < half / 8) {
                    uint4 x = *reinterpret_cast<const uint4*>(src + 8 * u);
                    uint4 y = *reinterpret_cast<const uint4*>(src + half + 8 * u);
                    turn_halves<E>(x, y, &cs[t][8 * u]);
                    *reinterpret_cast<uint4*>(dst + 8 * u) = x;
                    *reinterpret_cast<uint4*>(dst + half + 8 * u) = y;
                } else {
                    const int e = a.rot_dim + 8 * (u - half / 8);
                    *reinterpret_cast<uint4*>(dst + e) = *reinterpret_cast<const uint4*>(src + e);
                }
            } else if (u < half) {
                const float x = widen(src[u]), y = widen(src[u + half]);
                dst[u] = (E)(x * cs[t][u].x - y * cs[t][u].y);
                dst[u + half] = (E)(x * cs[t][u].y + y * cs[t][u].x);
            } else {
                const int e = a.rot_dim + u - half;
                dst[e] = src[e];
            }
        }
        if (tk.kv >= 0) {  // values
            const int perv = (int)blockDim.x / nvec, uv = (int)threadIdx.x % nvec, hv = (int)threadIdx.x / nvec;
            for (int h = hv; h < a.n_kv_heads && hv < perv; h += perv) {
                const E* src = reinterpret_cast<const E*>(a.v.p) + tk.row * a.v.row_stride + (int64_t)h * a.v.head_stride;
                E* dst = reinterpret_cast<E*>(c.v) + tk.kv + (int64_t)h * c.head_stride;
                *reinterpret_cast<uint4*>(dst + 8 * uv) = *reinterpret_cast<const uint4*>(src + 8 * uv);
            }
        }
    }
}

}  // namespace

hvd_status launch_rope_append(hvd_ctx* ctx, const RopeArgs& a, bool f16, int layout, cudaStream_t stream) {
    const int tpc = a.c.total_rows > 4LL * ctx->num_sms ? kRopeTokens : 1;
    const int64_t grid = (a.c.total_rows + tpc - 1) / tpc + (a.c.B + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
    const bool pdl = (ctx->pdl_mask & 16) != 0;
    auto run = [&](auto kernel) { return launch_kernel(pdl, kernel, dim3((unsigned)grid), dim3(kRopeThreads), 0, stream, a, tpc); };
    cudaError_t e;
    if (f16) e = layout == HVD_ROPE_PAIRS ? run(rope_append_kernel<__half, HVD_ROPE_PAIRS>) : run(rope_append_kernel<__half, HVD_ROPE_HALVES>);
    else e = layout == HVD_ROPE_PAIRS ? run(rope_append_kernel<__nv_bfloat16, HVD_ROPE_PAIRS>) : run(rope_append_kernel<__nv_bfloat16, HVD_ROPE_HALVES>);
    return e == cudaSuccess ? HVD_OK : cuda_fail(ctx, e, "rope_append_kernel");
}

}  // namespace hvd
