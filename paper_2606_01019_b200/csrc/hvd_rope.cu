// hvd_rope_append: rotary positions on the new tokens' queries and keys, keys and values into the paged cache.
//
// A pair (x, y) of a head turns by the angle a = t * w at position t.  The frequency is held in units of 2^-64
// turns, so that t * w modulo one turn is an integer product that wraps, exact for the frequency as held, where a
// 32-bit float product is off by thousandths of a radian from position 10^5 on.  The upper 32 bits go to sincospi.  (The frequency
// comes through 64-bit floats, good to 2^-52 of itself, and the angle is rounded to 24 bits of half a turn: together 2^-25 of a
// turn at positions up to 2^27, 2^-23 at 2^31.)
//
// Bandwidth: every element is read once and written once.  A CTA takes a few tokens.  Where a token goes hangs on four or five global
// round trips (request, lengths, page), so the rows themselves, which hang on none, are asked for first and wait in registers;
// the sines and cosines, the same for all heads, are computed once into shared memory.  A thread keeps its piece of a head through
// all the CTA's tokens and then goes on to its next head: with a place worked out anew for every vector the kernel ran 153
// instructions for each and was bound by them (8188 tokens of 48 heads: 53.5 us; now 37.0 us, 5.4 TB/s of what is read and written,
// 0.83 of the copy bandwidth).  Four tokens a CTA from four per SM on, below that one: 36 tokens 4.5 us, 1040 tokens of trees 6.2 us.
#include "hvd_attn.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

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

// The request of a row where the offsets ascend: the last one whose rows start at or before it.  All threads of the CTA count starts.
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

// A head of the CTA's tokens: where its first token's row is, where it goes.
template <typename E>
struct Lane {
    const E* src;
    E* dst;
    int64_t src_row, dst_row;  // from one token to the next; dst_row = 0: the token's cache slot counts
    bool turns, any;
    __device__ __forceinline__ Lane(const RopeArgs& a, int64_t row, int h) {
        any = h < a.n_q_heads + 2 * a.n_kv_heads;
        turns = h < a.n_q_heads + a.n_kv_heads;
        if (h < a.n_q_heads) {
            src = reinterpret_cast<const E*>(a.q.p) + row * a.q.row_stride + (int64_t)h * a.q.head_stride;
            dst = reinterpret_cast<E*>(a.q_out.p) + row * a.q_out.row_stride + (int64_t)h * a.q_out.head_stride;
            src_row = a.q.row_stride;
            dst_row = a.q_out.row_stride;
        } else {
            h -= a.n_q_heads;
            if (!turns) h -= a.n_kv_heads;
            const HeadsArgs& from = turns ? a.k : a.v;
            src = reinterpret_cast<const E*>(from.p) + row * from.row_stride + (int64_t)h * from.head_stride;
            dst = reinterpret_cast<E*>(turns ? a.c.k : a.c.v) + (int64_t)h * a.c.head_stride;
            src_row = from.row_stride;
            dst_row = 0;
        }
    }
    // NULL: the token is not written here
    __device__ __forceinline__ E* at(const Token& tk, int t) const {
        if (dst_row) return tk.b >= 0 ? dst + t * dst_row : nullptr;
        return tk.kv >= 0 ? dst + tk.kv : nullptr;
    }
};

// WHOLE: rotated elements come in whole 16-byte vectors with their partners (always so for PAIRS; HALVES need rot_dim / 2 to be a
// multiple of 8).
template <typename E, int LAYOUT, bool WHOLE, int T>
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const RopeArgs a) {
    __shared__ Token tok[T];
    __shared__ __align__(16) float2 cs[T][HVD_MAX_HEAD_DIM / 2];
    __shared__ unsigned long long turns[HVD_MAX_HEAD_DIM / 2];
    __shared__ int pos[T], owner[T];
    const ChunkArgs& c = a.c;
    pdl_trigger();
    pdl_wait();
    const int n_token_ctas = (int)((c.total_rows + T - 1) / T);
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
    const int64_t first = (int64_t)blockIdx.x * T;
    const int n_tok = (int)min((int64_t)T, c.total_rows - first);

    // ---- a unit is a piece of a head: HALVES turn vector u with its partner half a rotation on, the rest are single vectors
    const int D = a.head_dim, nvec = D / 8, half = a.rot_dim / 2, heads = a.n_q_heads + 2 * a.n_kv_heads;
    const int n_turn = LAYOUT == HVD_ROPE_HALVES && WHOLE ? half / 8 : 0;
    const int units = !WHOLE ? D - half : (LAYOUT == HVD_ROPE_PAIRS ? nvec : n_turn + (D - a.rot_dim) / 8);
    const int per = (int)blockDim.x / units;  // heads side by side
    const int u = (int)threadIdx.x % units, h0 = (int)threadIdx.x / units;
    const bool mine = h0 < per, turned = u < n_turn;
    const int e0 = turned || LAYOUT == HVD_ROPE_PAIRS ? 8 * u : a.rot_dim + 8 * (u - n_turn);  // first element of the (first) vector
    constexpr bool kPartner = LAYOUT == HVD_ROPE_HALVES;
    uint4 x[T], y[kPartner ? T : 1];
    int h = mine ? h0 : heads;
    Lane<E> lane(a, first, h);
    auto fetch = [&](const Lane<E>& l, uint4 (&vx)[T], uint4 (&vy)[kPartner ? T : 1]) {
#pragma unroll
        for (int i = 0; i < T; ++i)
            if (l.any && i < n_tok) {
                const E* src = l.src + i * l.src_row + e0;
                vx[i] = *reinterpret_cast<const uint4*>(src);
                if (kPartner && turned) vy[kPartner ? i : 0] = *reinterpret_cast<const uint4*>(src + half);
            }
    };
    if (WHOLE) fetch(lane, x, y);

    for (int j = threadIdx.x; j < half; j += blockDim.x) turns[j] = a.turns[j];
    const int b0 = request_of(c, first);
    const int64_t row = first + (int)threadIdx.x;  // this thread's token, the first n_tok threads
    int b = b0;
    if (c.row_off) {
        if ((int)threadIdx.x < n_tok) while (b + 1 < c.B && c.row_off[b + 1] <= row) ++b;
    } else {
        b = (int)min(row / (c.k_uniform + 1), (int64_t)c.B);
    }
    for (bool again = false;; again = true) {
        bool astray = false;
        if ((int)threadIdx.x < n_tok) {
            const int i = threadIdx.x;
            Token t = {row, -1, -1};
            astray = true;
            if (b < c.B) {
                const Chunk ch = load_chunk(c, b);
                const int64_t at = row - ch.r0;
                astray = at < 0 || at >= ch.rows;
                if (!ch.bad && at >= 0 && at < ch.n_new) {
                    t.b = b;
                    const int p = ch.base + (int)at;
                    const int64_t page = page_of(c, b, p);
                    int depth = (int)at;
                    unsigned long long nodes;
                    if (c.parent) tree_line(c, b, (int)at, nodes, depth);
                    pos[i] = ch.base + depth;
                    if (page >= 0 && HVD_IN_BOUNDS(c.dev_error, t.row, 0, c.total_rows)) t.kv = slot_offset(c, page, p);
                }
            }
            tok[i] = t;
        }
        if (!__syncthreads_or(astray && c.row_off && !again)) break;
        // Offsets that do not ascend led past a token's request: every request is asked, the first that has the row takes it.
        if ((int)threadIdx.x < T) owner[threadIdx.x] = c.B;
        __syncthreads();
        for (int i = threadIdx.x; i < c.B; i += blockDim.x) {
            const int64_t r0 = c.row_off[i], r1 = c.row_off[i + 1];
            if (r0 >= 0 && r1 <= c.total_rows)
                for (int t = 0; t < n_tok; ++t)
                    if (first + t >= r0 && first + t < r1) atomicMin(&owner[t], i);
        }
        __syncthreads();
        b = owner[min((int)threadIdx.x, T - 1)];
    }
    for (int i = threadIdx.x; i < n_tok * half; i += blockDim.x) {
        const int t = i / half, j = i - t * half;
        if (tok[t].b >= 0) {
            const unsigned long long turn = (unsigned long long)pos[t] * turns[j];  // modulo one turn
            float s, co;
            sincospif((float)(int32_t)(turn >> 32) * 4.656612873077393e-10f, &s, &co);  // 2^-31: turns to half turns
            cs[t][j] = make_float2(co * a.magnitude, s * a.magnitude);
        }
    }
    __syncthreads();

    if (WHOLE) {
        while (lane.any) {
            h += per;
            const Lane<E> next(a, first, h);
            uint4 nx[T], ny[kPartner ? T : 1];
            fetch(next, nx, ny);  // on its way while this head goes out
#pragma unroll
            for (int i = 0; i < T; ++i) {
                if (i >= n_tok) break;
                E* dst = lane.at(tok[i], i);
                if (!dst) continue;
                if (lane.turns) {
                    if (LAYOUT == HVD_ROPE_PAIRS) turn_pairs<E>(x[i], &cs[i][min(4 * u, HVD_MAX_HEAD_DIM / 2 - 4)], half - 4 * u);
                    else if (turned) turn_halves<E>(x[i], y[kPartner ? i : 0], &cs[i][8 * u]);
                }
                *reinterpret_cast<uint4*>(dst + e0) = x[i];
                if (kPartner && turned) *reinterpret_cast<uint4*>(dst + e0 + half) = y[kPartner ? i : 0];
            }
            lane = next;
#pragma unroll
            for (int i = 0; i < T; ++i) {
                x[i] = nx[i];
                if (kPartner) y[kPartner ? i : 0] = ny[kPartner ? i : 0];
            }
        }
    } else {  // element by element: u < half an element and its partner, then single ones
        for (; lane.any; h += per, lane = Lane<E>(a, first, h))
            for (int i = 0; i < n_tok; ++i) {
                E* dst = lane.at(tok[i], i);
                if (!dst) continue;
                const E* src = lane.src + i * lane.src_row;
                if (u < half) {
                    const E x0 = src[u], y0 = src[u + half];
                    const float2 f = cs[i][u];
                    dst[u] = lane.turns ? (E)(widen(x0) * f.x - widen(y0) * f.y) : x0;
                    dst[u + half] = lane.turns ? (E)(widen(x0) * f.y + widen(y0) * f.x) : y0;
                } else {
                    dst[u + half] = src[u + half];  // rot_dim + (u - half)
                }
            }
    }
}

}  // namespace

hvd_status launch_rope_append(hvd_ctx* ctx, const RopeArgs& a, bool f16, int layout, cudaStream_t stream) {
    const int tpc = a.c.total_rows > 4LL * ctx->num_sms ? kRopeTokens : 1;
    const int64_t grid = (a.c.total_rows + tpc - 1) / tpc + (a.c.B + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
    const bool pdl = (ctx->pdl_mask & 16) != 0;
    const bool whole = a.rot_dim % 16 == 0;
    auto run = [&](auto kernel) { return launch_kernel(pdl, kernel, dim3((unsigned)grid), dim3(kRopeThreads), 0, stream, a); };
    auto form = [&](auto e, auto tokens) {
        using E = decltype(e);
        constexpr int T = decltype(tokens)::value;
        if (layout == HVD_ROPE_PAIRS) return run(rope_append_kernel<E, HVD_ROPE_PAIRS, true, T>);
        return whole ? run(rope_append_kernel<E, HVD_ROPE_HALVES, true, T>) : run(rope_append_kernel<E, HVD_ROPE_HALVES, false, T>);
    };
    auto pick = [&](auto e) {
        return tpc == 1 ? form(e, std::integral_constant<int, 1>()) : form(e, std::integral_constant<int, kRopeTokens>());
    };
    const cudaError_t e = f16 ? pick(__half()) : pick(__nv_bfloat16());
    return e == cudaSuccess ? HVD_OK : cuda_fail(ctx, e, "rope_append_kernel");
}

}  // namespace hvd
