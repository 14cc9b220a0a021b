// hvd_attn_paged: attention of a chunk's rows over the paged cache, on the 5th-generation tensor cores.
//
// The rows of a key/value head are the chunk's tokens times the query heads of its group, packed into tiles of
// 128 rows; keys come in tiles of 64.  Per pair of tiles, S = Q K^T lands in tensor memory, a warpgroup turns it into
// weights P = exp2(S - m) with the running maximum m and sum of a softmax (one thread per row: no shuffles), and
// O += P V takes P from tensor memory.
//
// Two STREAMS of such steps run against each other, each with two score buffers, so that products run ahead of the
// softmax:
//   wide items (more than 128 rows)   the streams are two row tiles that share every key tile
//   narrow items                      the streams are the even and the odd key tiles of one row tile, joined at the end
// Tensor memory, 512 columns: scores [stream][buffer][64] (the weights overwrite the scores they come from), sums [stream][128].
// Roles of the 12 warps: 0-3 and 4-7 softmax, rescaling and output of stream 0 and 1; 8 and 9 issue the products of
// stream 0 and 1 (one issuing thread for both was measured to be the bound: 2400 cycles a tile pair, where the products take
// 1285); 10 deals out the work and loads queries and keys, 11 the values, box by box through the page table, by TMA into a
// ring of slots each.
//
// Work is counted in steps (a row tile with a key tile) over all (request, head, group of rows) items and dealt to the SMs in
// equal consecutive shares, whatever the lengths; every CTA finds its share from the lengths itself.  An item that
// several CTAs share leaves partial sums, which attn_finish_kernel joins in the order of the CTAs: no result depends on
// timing.
//
// Measured on one B200, in graphs of a few milliseconds / in long runs, which the power limit slows down: 64 requests of 16 K tokens with 17
// rows, 32/8 heads of 128: 666 / 797 us for 4.3 GB of keys and values (6.5 / 5.4 TB/s, bound by HBM, then by power); 96 ragged requests, one
// row: 484 / 541 us (6.3 / 5.6 TB/s); 4 x 2047 rows behind 1.5 to 9 K tokens: 681 / 790 us (1019 / 879 TFLOP/s; bound by the alternation
// of products and softmax: 1860 cycles a pair of steps, the products alone 1285); one token behind 1037: 13.6 / 13.9 us (two launches
// and their round trips).  Key tiles of 64 instead of 128: with 128 a stream's scores, weights and sums
// leave no room for a second buffer, and six tiles in flight hide HBM better than two and a half (one-token decode 104 -> 93 us).
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "hvd_attn.cuh"
#include "hvd_sm100.cuh"

namespace hvd {

using namespace sm100;

namespace {

constexpr int kSoftmaxWarps = 8, kMmaWarp = 8, kLoadWarp = 10, kLoadVWarp = 11;  // kMmaWarp + 1: stream 1
constexpr int kThreads = 384;
// registers: 384 threads start with 168 each; the softmax warpgroups take 208, the third keeps 88 (208 + 208 + 88 = 3 * 168)
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;
constexpr int kFinishThreads = 256;
constexpr int kJoin = 4;  // pieces whose sums are fetched together (6 and 8: 17 pieces of 4 rows 0.3 us faster, many items with few pieces 1 to 2 us slower)
constexpr int kShortPiece = 32;         // key tiles; below, only the query boxes that hold tokens are loaded
constexpr float kRescaleAbove = 8.0f;  // log2: a maximum that grew by less keeps its old value
// log2 of the weight of a row's maximum: 1, or 2^7 for f16, whose numbers end at 2^-24 below and 2^16 above.  A long context behind one
// large weight adds up from small ones, which would be rounded to zero from 2^-25 on (131071 keys of 2^-25.2 each: 0.33 % of the
// output); the sum has them all.  With kRescaleAbove weights reach 2^15.
template <typename E> constexpr float kTopWeight = std::is_same<E, __half>::value ? 7.0f : 0.0f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kPieces = 4;             // pieces of work announced ahead
// Flags of items, of which the loading warp is at most kPieces ahead of a softmax warp: that one's flag is its own until it is through.
constexpr int kFlags = 8;
static_assert(kFlags > kPieces, "see above");

template <int DP> struct Shape {
    static constexpr int kHalves = DP / 64;                         // 128-byte columns of a tile row
    static constexpr int kQHalf = kTileRows * 128, kQBytes = kHalves * kQHalf;
    static constexpr int kKvHalf = kTileKeys * 128, kKvBytes = kHalves * kKvHalf;
    // The rings, 160 or 144 KB.  Even, so that a narrow piece's streams, which take every second tile, never share a slot: a stream
    // waits for a slot's fill by its parity and must have seen the fill before it.
    static constexpr int kKSlots = DP == 128 ? 4 : 8, kVSlots = DP == 128 ? 6 : 10;
    static_assert(kKSlots % 2 == 0 && kVSlots % 2 == 0, "see above");
    static constexpr int kSlots = kKSlots + kVSlots;
};
constexpr int kMaxSlots = 20;

struct Piece {  // what a CTA does of one item
    int b, h, qt;
    int r0, base;       // the request's first row, tokens cached before the chunk
    int tok0, n_tok;    // tokens of the item; n_tok = 0: no more work
    int kv0, kv1, nkv;  // key tiles of the piece, of the item
    int pad[2];
};

struct Shared {  // behind the tiles
    uint64_t full[kMaxSlots], empty[kMaxSlots];  // slots of the K ring, then of the V ring
    uint64_t q_full, q_empty;                    // the item's query tiles
    uint64_t s_full[2][2], p_full[2][2];         // [stream][buffer] scores written, weights written
    uint64_t o_full[2][2];                       // [stream][buffer] a step's product with V is done
    uint64_t stats, o_free;                      // maxima and sums of both streams exchanged; the item's sums are read
    uint64_t piece_full[kPieces], piece_empty[kPieces];
    uint64_t landed;                             // a V tile that is cleaned before it is full
    uint64_t drain;
    Piece piece[kPieces];
    int not_finite[kFlags];  // [item % kFlags] some value of the chunk's own tokens was infinite or NaN
    uint32_t tmem;
    int gave_up;
    struct { int b, h, qt, kv, r0, n_new, base; } start;  // where the CTA's share begins
    long long start_left;
    long long open_unit;  // of the item that the share leaves unfinished: its last tile's first unit
    long long warp_sum[kThreads / 32];
    float m[2][128], l[2][128];  // [stream][row]
};
template <int DP> constexpr int kTilesBytes = 2 * Shape<DP>::kQBytes + Shape<DP>::kSlots * Shape<DP>::kKvBytes;
template <int DP> constexpr int kSmemBytes = kTilesBytes<DP> + (int)sizeof(Shared);
static_assert(kSmemBytes<128> <= 227 * 1024 && kSmemBytes<64> <= 227 * 1024, "shared memory of a CTA");

// One CTA's partial sums: slot 0 an item that an earlier CTA began, slot 1 an item that a later CTA goes on with.
struct SplitDesc {
    int valid, h, r0, tok0, n_tok, c_last, pad[2];
};

struct Work {
    SplitDesc* desc;   // [CTAs]
    float* o;          // [CTAs][2][DP / 4][256 rows][4]: a warp's rows side by side, for writing and for reading
    float2* ml;        // [CTAs][2][256] maximum (log2 units), sum
    int* spare;        // some row is no new token
};

// ---------------------------------------------------------------- items

struct Geometry {
    int tile_tok;  // tokens of a row tile
    int item_tok;  // tokens of an item: two row tiles
};

__device__ __forceinline__ int key_tiles(const Chunk& c, const Geometry& g, int qt) {
    return (c.base + min(c.n_new, (qt + 1) * g.item_tok) - 1) / kTileKeys + 1;
}

// row tiles of an item: 1 (narrow) or 2 (wide)
__device__ __forceinline__ int row_tiles(const Chunk& c, const Geometry& g, int qt) { return c.n_new - qt * g.item_tok > g.tile_tok ? 2 : 1; }

// steps of one head of a request
__device__ __forceinline__ long long head_units(const Chunk& c, const Geometry& g) {
    long long u = 0;
    for (int qt = 0; qt * g.item_tok < c.n_new; ++qt) u += (long long)key_tiles(c, g, qt) * row_tiles(c, g, qt);
    return u;
}

// 32 bits nearly always do; the 64-bit division is a long way round at the start of a short kernel
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}

// Consecutive shares of `total` units: CTA c begins at unit share_start(c).  A wide item is cut between key tiles
// (two units each), so that where there are wide items a share has two units at least.
struct Shares {
    long long total, q;
    int n, r;
};
__device__ __forceinline__ long long share_start(const Shares& s, int c) { return c * s.q + min(c, s.r); }
__device__ __forceinline__ int share_owner(const Shares& s, long long unit) {
    const long long longer = s.r * (s.q + 1);  // units of the first r shares, which hold one more
    return unit < longer ? (int)quotient(unit, s.q + 1) : s.r + (int)quotient(unit - longer, s.q);
}

// a wait of a whole warp: all lanes go on, or none
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* gave_up) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, gave_up));
}

// The pages of a piece's boxes, 32 at a time in the lanes of a loading warp, and the 32 after them on their way.
struct PageWindow {
    int page, in, page_next, in_next;
    __device__ __forceinline__ static void fetch(const ChunkArgs& c, int b, int box, int box_keys, int kv_end, int& page, int& in) {
        const int64_t key = (int64_t)(box + (int)(threadIdx.x & 31)) * box_keys;
        page = -1;
        in = 0;
        if (key < kv_end) {
            const int j = (int)key / c.page_size;
            in = (int)key - j * c.page_size;
            if (HVD_IN_BOUNDS(c.dev_error, j, 0, c.table_stride)) page = c.page_table[(int64_t)b * c.table_stride + j];
        }
    }
};

// ---------------------------------------------------------------- the kernel

template <typename E> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// visible columns of a key tile, one bit each: those below n, and the nodes, node j at column at + j (at may be negative)
__device__ __forceinline__ unsigned long long seen_columns(int n, unsigned long long nodes, int at) {
    unsigned long long s = n >= 64 ? ~0ull : (n <= 0 ? 0ull : (1ull << n) - 1ull);
    if (at >= 0 && at < 64) s |= nodes << at;
    else if (at < 0 && at > -64) s |= nodes >> -at;
    return s;
}

// 2^x of two finite numbers on the multiply-add pipe: x = n + f with n the nearest whole number, 2^f as the minimax polynomial of
// degree 4 on [-1/2, 1/2] (Remez exchange; relative error 2.6e-6), n added to the exponent.  x is held above -126.
__device__ __forceinline__ float2 exp2_poly(float2 x) {
    const float2 magic = make_float2(12582912.0f, 12582912.0f), unmagic = make_float2(-12582912.0f, -12582912.0f);  // 1.5 * 2^23
    x = make_float2(fmaxf(x.x, -126.0f), fmaxf(x.y, -126.0f));
    const float2 t = add2(x, magic);
    const float2 f = fma2(add2(t, unmagic), make_float2(-1.0f, -1.0f), x);
    float2 p = make_float2(0.009570102014629326f, 0.009570102014629326f);
    p = fma2(p, f, make_float2(0.05591786030632565f, 0.05591786030632565f));
    p = fma2(p, f, make_float2(0.24024744824991692f, 0.24024744824991692f));
    p = fma2(p, f, make_float2(0.6931218147429867f, 0.6931218147429867f));
    p = fma2(p, f, make_float2(0.9999992614469312f, 0.9999992614469312f));
    return make_float2(__uint_as_float(__float_as_uint(p.x) + (__float_as_uint(t.x) << 23)), __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(t.y) << 23)));
}

// w = exp2(x * scale - m) (m: the maximum less kTopWeight) of a row's 64 scores, rounded to the cache's type and packed, into tensor memory over the scores; returns
// their sums before rounding.  Every eighth pair goes through exp2_poly, which relieves the special function unit but takes more power,
// by which long runs are bound (2047 rows behind 1.5 to 9 K tokens, long runs, us: none 823, every 8th pair 791, 5th 811, 3rd 837,
// 2nd 862; short runs are fastest with every 3rd).  That makes 2^-126 of a score of -infinity: where there are some (`edge`) those
// weights are cleared by `seen`.
template <typename E>
__device__ __forceinline__ float2 weights(const uint32_t (&x)[2][32], uint32_t dst, float2 scale2, float m, bool edge, unsigned long long seen) {
    const float shift = m == -INFINITY ? 0.0f : -m;
    const float2 shift2 = make_float2(shift, shift);
    float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t w[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            float2 e = fma2(make_float2(__uint_as_float(x[i][2 * k]), __uint_as_float(x[i][2 * k + 1])), scale2, shift2);
            if (k % 8 == 7) e = exp2_poly(e);
            else e = make_float2(exp2_approx(e.x), exp2_approx(e.y));
            sum[k & 1] = add2(sum[k & 1], e);
            w[k] = pack2<E>(e.x, e.y);
        }
        if (edge) {
            const uint32_t bits = (uint32_t)(seen >> (32 * i));
#pragma unroll
            for (int k = 7; k < 16; k += 8) w[k] &= (((bits >> (2 * k)) & 1u) ? 0xffffu : 0u) | (((bits >> (2 * k + 1)) & 1u) ? 0xffff0000u : 0u);
        }
        tmem_st16(dst + 16 * i, w);
    }
    return add2(sum[0], sum[1]);
}

// Row statistics (m, l) with l = 0: m = -infinity of a row that sees nothing, kLowest of one whose scores are all -infinity (0 / 0).
constexpr float kLowest = -3.402823466e38f;
__device__ __forceinline__ float inverse_sum(float m, float l) { return l == 0.0f ? (m == -INFINITY ? 0.0f : NAN) : 1.0f / l; }
__device__ __forceinline__ float log_sum(float m, float l) { return l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2; }

// Infinities and NaN that were cleared from the values of tokens [lo, hi), back into a row that sees them: columns [c0, c1) of its
// output, or of its partial sums.  (Any positive weight times such a value is that value.)
template <typename E>
__device__ __noinline__ void restore_cleared(const AttnArgs& a, int b, int h, int lo, int hi, int upto, unsigned long long nodes, int node0, int c0, int c1,
                                             E* out, float* part) {
    for (int t = lo; t < hi; ++t) {
        if (!(t < upto || (a.c.parent && ((nodes >> (t - node0)) & 1ull)))) continue;
        const int64_t page = page_of(a.c, b, t);
        if (page < 0) continue;
        const E* val = reinterpret_cast<const E*>(a.c.v) + slot_offset(a.c, page, t) + (int64_t)h * a.c.head_stride;
        for (int c = c0; c < c1; ++c) {
            const float e = (float)val[c];
            if (isfinite(e)) continue;
            if (out) out[c] = (E)((float)out[c] + e);
            else part[(c >> 2) * 1024 + (c & 3)] += e;
        }
    }
}

template <typename E, int DP>
__global__ void __launch_bounds__(kThreads, 1)
attn_tile_kernel(const AttnArgs a, const Work ws, const Geometry g, const int box_keys, const int box_tok, const __grid_constant__ CUtensorMap map_q,
                 const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    using S = Shape<DP>;
    extern __shared__ __align__(1024) unsigned char dyn[];
    Shared& sh = *reinterpret_cast<Shared*>(dyn + kTilesBytes<DP>);
    const uint32_t tiles = smem_addr(dyn);  // 1024-byte aligned: the kernel has no other shared memory
    const uint32_t ring = tiles + 2 * S::kQBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* gave_up = &sh.gave_up;

    pdl_trigger();
    if (warp == kMmaWarp) tmem_alloc(smem_addr(&sh.tmem), 512);
    if (warp == kLoadWarp) {
        if (lane < 3) tma_prefetch_map(lane == 0 ? &map_q : (lane == 1 ? &map_k : &map_v));
        if (lane < S::kSlots) { mbar_init(smem_addr(&sh.full[lane]), 1); mbar_init(smem_addr(&sh.empty[lane]), 2); }
        if (lane < 4) { mbar_init(smem_addr(&sh.s_full[0][lane]), 1); mbar_init(smem_addr(&sh.p_full[0][lane]), 4); mbar_init(smem_addr(&sh.o_full[0][lane]), 1); }
        if (lane < kPieces) { mbar_init(smem_addr(&sh.piece_full[lane]), 1); mbar_init(smem_addr(&sh.piece_empty[lane]), kSoftmaxWarps + 3); }
        if (lane == 0) {
            mbar_init(smem_addr(&sh.q_full), 1);
            mbar_init(smem_addr(&sh.q_empty), 2);
            mbar_init(smem_addr(&sh.stats), kSoftmaxWarps);
            mbar_init(smem_addr(&sh.o_free), kSoftmaxWarps);
            mbar_init(smem_addr(&sh.landed), 1);
            mbar_init(smem_addr(&sh.drain), 2);
            sh.gave_up = 0;
        }
        mbar_init_fence();
    }
    pdl_wait();

    // ---- this CTA's share: units of all requests before each thread's, then the request that holds the share's first unit
    const int per = (a.c.B + kThreads - 1) / kThreads;
    const int b0 = min(a.c.B, (int)threadIdx.x * per), b1 = min(a.c.B, b0 + per);
    long long mine = 0;
    Chunk c0 = {};
    bool any_wide = false, spare = false;
    for (int b = b0; b < b1; ++b) {
        const Chunk c = load_chunk(a.c, b);
        if (b == b0) c0 = c;
        any_wide = any_wide || c.n_new > g.tile_tok;
        spare = spare || c.rows > c.n_new;
        mine += head_units(c, g) * a.n_kv_heads;
    }
    long long upto_b = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, upto_b, d);
        if (lane >= d) upto_b += t;
    }
    if (lane == 31) sh.warp_sum[warp] = upto_b;
    any_wide = __syncthreads_or(any_wide);
    Shares shares;
    shares.total = 0;
    long long before = upto_b - mine;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) {
        const long long w = sh.warp_sum[i];
        if (i < warp) before += w;
        shares.total += w;
    }
    shares.n = (int)min((long long)gridDim.x, any_wide ? (shares.total + 1) / 2 : shares.total);
    const int cta = blockIdx.x;
    long long first = 0, last = 0;
    if (cta < shares.n) {
        shares.q = quotient(shares.total, shares.n);
        shares.r = (int)(shares.total - shares.q * shares.n);
        first = share_start(shares, cta);
        last = share_start(shares, cta + 1);
        if (first >= before && first < before + mine) {
            long long off = first - before, left = last - first, hu = head_units(c0, g);
            Chunk c = c0;
            int b = b0;
            while (off >= hu * a.n_kv_heads) {
                off -= hu * a.n_kv_heads;
                c = load_chunk(a.c, ++b);
                hu = head_units(c, g);
            }
            const int h = (int)quotient(off, hu);
            off -= h * hu;
            int qt = 0, w = row_tiles(c, g, 0);
            for (long long u; off >= (u = (long long)key_tiles(c, g, qt) * w);) {
                off -= u;
                w = row_tiles(c, g, ++qt);
            }
            // a share that begins inside a wide item's step pair begins behind it
            int kv = (int)off;
            if (w == 2) {
                kv = (int)((off + 1) >> 1);
                left -= kv * 2 - off;
                if (kv == key_tiles(c, g, qt)) { kv = 0; ++qt; }
            }
            sh.start = {b, h, qt, kv, (int)c.r0, c.n_new, c.base};
            sh.start_left = left;
        }
    }
    if (threadIdx.x == 0) ws.desc[cta].valid = 0;
    fence_before_sync();
    spare = __syncthreads_or(spare);
    fence_after_sync();
    if (cta == 0 && threadIdx.x == 0) *ws.spare = spare;
    const uint32_t tmem = sh.tmem;
    const uint32_t full0 = smem_addr(&sh.full[0]), empty0 = smem_addr(&sh.empty[0]);

    if (warp >= kSoftmaxWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        const int n_box = kTileKeys / box_keys;
        // A piece's K or V tiles into their ring, from ring position `pos` on; around_first() runs ahead of and behind the first tile.
        // A weight of zero must keep out what it stands for, but 0 * NaN is NaN.  So in V tiles with keys that some row does not
        // see, slots at and behind the item's last key, which may hold anything, are cleared, and of the chunk's own tokens
        // infinities and NaN: rows that see those get them back at the end.
        int cleaned = 0;
        volatile int* not_finite = nullptr;  // the item's flag, in the warp that loads values
        auto load_tiles = [&](const Piece& p, const bool is_v, const CUtensorMap* map, uint32_t base, uint32_t full, uint32_t empty, int slots, int pos, auto around_first) {
            const int kv_end = p.base + p.tok0 + p.n_tok, n = p.kv1 - p.kv0, box0 = p.kv0 * n_box;
            const int item_sees = p.base + 1 + (a.c.parent ? 0 : p.tok0);  // every row of the item does, if it sees anything
            PageWindow w;
            PageWindow::fetch(a.c, p.b, box0, box_keys, kv_end, w.page, w.in);
            PageWindow::fetch(a.c, p.b, box0 + 32, box_keys, kv_end, w.page_next, w.in_next);
            int slot = pos % slots, round = pos / slots;
            if (!around_first(true)) return false;
            for (int i = 0; i < n; ++i) {
                const int at = i * n_box;  // box within the piece
                if (i > 0 && (at & 31) == 0) {
                    w.page = w.page_next;
                    w.in = w.in_next;
                    PageWindow::fetch(a.c, p.b, box0 + at + 32, box_keys, kv_end, w.page_next, w.in_next);
                }
                int page = __shfl_sync(0xffffffffu, w.page, (at + lane) & 31);
                const int in = __shfl_sync(0xffffffffu, w.in, (at + lane) & 31);
                if (page < 0 || page >= a.c.n_pages) page = -1;  // the box lies outside the tensor: zeros
                const int keys = kv_end - (p.kv0 + i) * kTileKeys;  // of the item, from this tile on
                const int boxes = keys >= kTileKeys ? n_box : (keys - 1) / box_keys + 1;
                if (!warp_wait(empty + 8 * slot, (round & 1) ^ 1, gave_up)) return false;
                const bool clean = is_v && (p.kv0 + i + 1) * (int64_t)kTileKeys > item_sees;
                const uint32_t bar = clean ? smem_addr(&sh.landed) : full + 8 * slot, tile = base + slot * S::kKvBytes;
                if (lane == 0) mbar_expect(bar, (uint32_t)(boxes * box_keys * 128 * S::kHalves));
                __syncwarp();
                if (lane < boxes) {
                    const uint32_t dst = tile + lane * box_keys * 128;
#pragma unroll
                    for (int hf = 0; hf < S::kHalves; ++hf) tma_load_4d(dst + hf * S::kKvHalf, map, bar, hf * 64, in, p.h, page);
                }
                __syncwarp();
                if (clean) {
                    if (!warp_wait(smem_addr(&sh.landed), cleaned & 1, gave_up)) return false;
                    ++cleaned;
                    const int end = min(kTileKeys, keys);
                    // 16-byte pieces, 8 lanes a row
                    for (int r = max(0, item_sees - (p.kv0 + i) * kTileKeys) + (lane >> 3); r < end; r += 4)
#pragma unroll
                        for (int hf = 0; hf < S::kHalves; ++hf) {
                            const uint32_t piece = tile + hf * S::kKvHalf + r * 128 + (lane & 7) * 16;
                            uint32_t x[4];
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(piece) : "memory");
                            constexpr uint32_t kExp = std::is_same<E, __half>::value ? 0x7c00u : 0x7f80u;
                            bool odd = false;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const bool lo = (x[k] & kExp) == kExp, hi = (x[k] & (kExp << 16)) == kExp << 16;
                                odd = odd || lo || hi;
                                x[k] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
                            }
                            if (odd) {
                                *not_finite = 1;
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(piece), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
                            }
                        }
                    for (int r = end + (lane >> 3); r < kTileKeys; r += 4)
#pragma unroll
                        for (int hf = 0; hf < S::kHalves; ++hf)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + hf * S::kKvHalf + r * 128 + (lane & 7) * 16), "r"(0) : "memory");
                    fence_async_proxy();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(full + 8 * slot);
                }
                if (i == 0 && !around_first(false)) return false;
                if (++slot == slots) { slot = 0; ++round; }
            }
            return true;
        };
        auto drain_loads = [&]() {  // gave up: time for the loads in flight to land before the shared memory is given back
            const unsigned long long t0 = now_ns();
            while (now_ns() - t0 < kWaitLimitNs / 100) {}
        };
        if (warp == kLoadWarp) {
            // -------------------------------------------------------- work and loads
            long long left = 0;
            int b = 0, h = 0, qt = 0, kv = 0, pos = 0, items = 0;  // pos: position in the K ring
            Chunk c = {};
            if (last > first) {
                left = sh.start_left;
                b = sh.start.b; h = sh.start.h; qt = sh.start.qt; kv = sh.start.kv;
                c.r0 = sh.start.r0; c.n_new = sh.start.n_new; c.base = sh.start.base;
            }
            bool ok = true;
            for (;; ++items) {
                // the next piece
                Piece p = {};
                if (left > 0) {
                    while (qt * g.item_tok >= c.n_new) {  // past the head's last item
                        qt = 0;
                        if (c.n_new == 0 || ++h == a.n_kv_heads) {
                            h = 0;
                            c = load_chunk(a.c, ++b);
                        }
                    }
                    p.b = b; p.h = h; p.qt = qt; p.r0 = (int)c.r0; p.base = c.base;
                    p.tok0 = qt * g.item_tok;
                    p.n_tok = min(g.item_tok, c.n_new - p.tok0);
                    p.nkv = key_tiles(c, g, qt);
                    p.kv0 = kv;
                    const int w = row_tiles(c, g, qt);
                    p.kv1 = (int)min((long long)p.nkv, kv + ((left + w - 1) >> (w - 1)));
                    left -= (long long)(p.kv1 - p.kv0) * w;
                    if (p.kv0 == 0 && p.kv1 < p.nkv && lane == 0) {
                        // What joins the pieces has to know the CTA with the item's last tile, by the tile's first unit.  (A share that
                        // begins with a tile's second unit begins behind it.)
                        sh.open_unit = last - left + (long long)(p.nkv - p.kv1 - 1) * w;
                    }
                    kv = 0;
                    ++qt;
                }
                const int ps = items % kPieces;
                ok = warp_wait(smem_addr(&sh.piece_empty[ps]), ((items / kPieces) & 1) ^ 1, gave_up);
                if (!ok) break;
                if (lane == 0) { sh.piece[ps] = p; mbar_arrive(smem_addr(&sh.piece_full[ps])); }
                if (p.n_tok == 0) break;
                // a first piece's queries go while its page entries are on their way; later ones go behind the first key tile, which
                // does not wait for the item before to be done with its own
                auto load_q = [&](bool ahead) {
                    if (ahead != (items == 0)) return true;
                    if (!warp_wait(smem_addr(&sh.q_empty), (items & 1) ^ 1, gave_up)) return false;
                    // Boxes behind the item's tokens lie outside the tensor and bring zeros: rows of zeros make scores and weights of
                    // zero, which cost the tensor cores less power than what the shared memory held (ragged decode, in a long run,
                    // 590 -> 549 us).  A short piece goes without them, its unused rows hold what was there and nothing reads what
                    // comes of them: power does not bound it, and issuing all boxes keeps its first keys waiting (one token 14.0 ->
                    // 13.6 us, 4 x 2 K 21.4 -> 21.0 us; from 8 to 32 tiles the border makes no difference).
                    const int nb = g.tile_tok / box_tok;  // boxes of a row tile
                    const int n_box_q = p.kv1 - p.kv0 < kShortPiece ? (p.n_tok + box_tok - 1) / box_tok : p.n_tok > g.tile_tok ? 2 * nb : nb;
                    if (lane == 0) mbar_expect(smem_addr(&sh.q_full), (uint32_t)(n_box_q * box_tok * a.group * 128 * S::kHalves));
                    __syncwarp();
                    for (int x = lane; x < n_box_q; x += 32) {
                        const int t = x >= nb, bx = x - (t ? nb : 0), tok = t * g.tile_tok + bx * box_tok;
                        const uint32_t dst = tiles + t * S::kQBytes + bx * box_tok * a.group * 128;
                        const int row = tok < p.n_tok ? p.r0 + p.tok0 + tok : (int)a.c.total_rows;
#pragma unroll
                        for (int hf = 0; hf < S::kHalves; ++hf)
                            tma_load_4d(dst + hf * S::kQHalf, &map_q, smem_addr(&sh.q_full), hf * 64, 0, row, p.h);
                    }
                    return true;
                };
                ok = load_tiles(p, false, &map_k, ring, full0, empty0, S::kKSlots, pos, load_q);
                if (!ok) break;
                pos += p.kv1 - p.kv0;
            }
            if (!ok) drain_loads();
        } else if (warp == kLoadVWarp) {
            int pos = 0;
            bool ok = true;
            for (int items = 0;; ++items) {
                const int ps = items % kPieces;
                ok = warp_wait(smem_addr(&sh.piece_full[ps]), (items / kPieces) & 1, gave_up);
                if (!ok) break;
                const Piece p = sh.piece[ps];
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.piece_empty[ps]));
                if (p.n_tok == 0) break;
                not_finite = &sh.not_finite[items % kFlags];
                if (lane == 0) *not_finite = 0;
                __syncwarp();
                ok = load_tiles(p, true, &map_v, ring + S::kKSlots * S::kKvBytes, full0 + 8 * S::kKSlots, empty0 + 8 * S::kKSlots, S::kVSlots, pos,
                                [](bool) { return true; });
                if (!ok) break;
                pos += p.kv1 - p.kv0;
            }
            if (!ok) drain_loads();
        } else {
            // -------------------------------------------------------- products of one stream
            const int s = warp - kMmaWarp;
            if (elect_one()) {
                const bool f16 = std::is_same<E, __half>::value;
                const int ksteps = (a.head_dim + 15) / 16;
                const uint32_t qk_desc = instr_desc(f16, 128, kTileKeys, false), pv_desc = instr_desc(f16, 128, ksteps * 16, true);
                const uint64_t k_base = operand_desc(ring, 16), v_base = operand_desc(ring + S::kKSlots * S::kKvBytes, S::kKvHalf);
                const uint32_t s_buf = tmem + s * 128, o_buf = tmem + 256 + s * 128;
                int pos = 0, items = 0;
                uint32_t done = 0;  // this stream's steps so far
                bool ok = true;
                for (;; ++items) {
                    const int ps = items % kPieces;
                    ok = mbar_wait(smem_addr(&sh.piece_full[ps]), (items / kPieces) & 1, gave_up);
                    if (!ok) break;
                    const int n_tok = sh.piece[ps].n_tok, n = sh.piece[ps].kv1 - sh.piece[ps].kv0;
                    mbar_arrive(smem_addr(&sh.piece_empty[ps]));
                    if (n_tok == 0) break;
                    const bool wide = n_tok > g.tile_tok;
                    // wide: this row tile with every key tile; narrow: the one row tile with every second key tile
                    const int steps = wide ? n : (n + 1 - s) / 2, stride = wide ? 1 : 2;
                    const uint64_t q_base = operand_desc(tiles + (wide ? s : 0) * S::kQBytes, 16);
                    int k_at = pos + (wide ? 0 : s), v_at = k_at;  // ring positions
                    // a slot is free when both streams are through with it; in a narrow piece one speaks for both
                    auto release = [&](int slot) {
                        mma_commit(empty0 + 8 * slot);
                        if (!wide) mma_commit(empty0 + 8 * slot);
                    };
                    ok = mbar_wait(smem_addr(&sh.q_full), items & 1, gave_up);
                    for (int i = 0; ok && i < steps + 2; ++i) {
                        const int ks = k_at % S::kKSlots, vs = v_at % S::kVSlots;
                        if (i < steps) ok = mbar_wait(full0 + 8 * ks, (k_at / S::kKSlots) & 1, gave_up);
                        if (ok && i >= 2) {  // O += P V of step i - 2
                            const uint32_t k = done + i - 2, buf = k & 1;
                            // the last item's sums are read, by which also all of its V tiles have been there
                            if (i == 2) ok = mbar_wait(smem_addr(&sh.o_free), (items & 1) ^ 1, gave_up);
                            ok = ok && mbar_wait(full0 + 8 * (S::kKSlots + vs), (v_at / S::kVSlots) & 1, gave_up) &&
                                 mbar_wait(smem_addr(&sh.p_full[s][buf]), (k >> 1) & 1, gave_up);
                            if (!ok) break;
                            fence_after_sync();
                            const uint64_t vd = v_base + ((vs * S::kKvBytes) >> 4);
#pragma unroll
                            for (int x = 0; x < kTileKeys / 16; ++x)
                                mma_ts(o_buf, s_buf + buf * 64 + 8 * x, vd + ((x * 2048) >> 4), pv_desc, i > 2 || x > 0);
                            mma_commit(smem_addr(&sh.o_full[s][buf]));
                            release(S::kKSlots + vs);
                            v_at += stride;
                        }
                        if (ok && i < steps) {  // S = Q K^T of step i
                            const uint32_t buf = (done + i) & 1;
                            fence_after_sync();
                            const uint64_t kd = k_base + ((ks * S::kKvBytes) >> 4);
#pragma unroll
                            for (int x = 0; x < DP / 16; ++x)
                                if (x < ksteps)
                                    mma_ss(s_buf + buf * 64, q_base + (((x >> 2) * S::kQHalf + (x & 3) * 32) >> 4),
                                           kd + (((x >> 2) * S::kKvHalf + (x & 3) * 32) >> 4), qk_desc, x > 0);
                            mma_commit(smem_addr(&sh.s_full[s][buf]));
                            release(ks);
                            if (i == steps - 1) mma_commit(smem_addr(&sh.q_empty));
                            k_at += stride;
                        }
                    }
                    if (!ok) break;
                    if (steps == 0) {  // every phase of o_free is waited for, so that none is mistaken for another
                        ok = mbar_wait(smem_addr(&sh.o_free), (items & 1) ^ 1, gave_up);
                        if (!ok) break;
                        mbar_arrive(smem_addr(&sh.q_empty));
                    }
                    done += steps;
                    pos += n;
                }
                mma_commit(smem_addr(&sh.drain));  // nothing is in flight when tensor memory is freed
                int never = 0;
                mbar_wait(smem_addr(&sh.drain), 0, &never);
                if (never) sh.gave_up = 1;
            }
            __syncwarp();
        }
    } else {
        // ------------------------------------------------------------ softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const int s = warp >> 2, row = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's quarter of the tensor memory's lanes (bits 16 up)
        const uint32_t s_col = tmem + lanes + s * 128, o_col = tmem + lanes + 256 + s * 128;
        const float2 scale2 = make_float2(a.scale_log2, a.scale_log2);
        int narrow_items = 0;
        uint32_t done = 0, done_other = 0;  // steps of this stream and of the other one so far
        // the last of a stream's steps so far is in its sums.  Up to two products with V are pending, which one barrier's parity
        // could not tell apart.
        auto sums_done = [&](int of, uint32_t steps_so_far) {
            const uint32_t k = steps_so_far - 1;
            return warp_wait(smem_addr(&sh.o_full[of][k & 1]), (k >> 1) & 1, gave_up);
        };
        bool ok = true;
        for (int items = 0;; ++items) {
            const int ps = items % kPieces;
            ok = warp_wait(smem_addr(&sh.piece_full[ps]), (items / kPieces) & 1, gave_up);
            if (!ok) break;
            const Piece p = sh.piece[ps];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sh.piece_empty[ps]));
            if (p.n_tok == 0) break;
            const bool wide = p.n_tok > g.tile_tok;
            const int n_tiles = p.kv1 - p.kv0, steps = wide ? 2 * n_tiles : n_tiles;
            const int tok0 = p.tok0 + (wide ? s * g.tile_tok : 0);
            const int kv_end = p.base + p.tok0 + p.n_tok;
            const int n_rows = min(g.tile_tok, p.tok0 + p.n_tok - tok0) * a.group;
            const int tok = tok0 + row / a.group, grp = row % a.group;
            const bool valid = row < n_rows && HVD_IN_BOUNDS(a.c.dev_error, (int64_t)p.r0 + tok, 0, a.c.total_rows), active = (row & ~31) < n_rows;
            // what the row sees: keys below `upto`, in a tree also the nodes on its line
            unsigned long long nodes = 0ull;
            int upto = p.base + tok + 1;
            if (a.c.parent) {
                int depth;
                const bool reach = !valid || tree_line(a.c, p.b, tok, nodes, depth);
                upto = reach ? p.base + 1 : 0;
            }
            const int item_sees = p.base + 1 + (a.c.parent ? 0 : p.tok0);
            // every row of the warp sees the whole of a tile that starts here or before (the first key behind a tile may be 2^31)
            const int whole_to = __reduce_min_sync(0xffffffffu, valid ? upto : 0x7fffffff) - kTileKeys;
            float m = -INFINITY, l = 0.0f, l_far = 0.0f;  // l: the sum of up to 32 steps, l_far: of those before
            for (int st = s; ok && st < steps; st += 2) {
                const int j = wide ? st >> 1 : st, key0 = (p.kv0 + j) * kTileKeys;
                const uint32_t buf = done & 1;
                ok = warp_wait(smem_addr(&sh.s_full[s][buf]), (done >> 1) & 1, gave_up);
                if (!ok) break;
                fence_after_sync();
                if (active) {
                    uint32_t x[2][32];
                    tmem_ld32(x[0], s_col + buf * 64);
                    tmem_ld32(x[1], s_col + buf * 64 + 32);
                    tmem_wait_ld(x[0]);
                    tmem_waited(x[1]);
                    const bool edge = key0 > whole_to;  // some row of the warp does not see the whole tile
                    unsigned long long seen = ~0ull;
                    if (edge) {
                        seen = seen_columns(upto - key0, nodes, p.base + 1 - key0);
                        const uint32_t w[2] = {(uint32_t)seen, (uint32_t)(seen >> 32)};
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (!((w[i] >> k) & 1u)) x[i][k] = 0xff800000u;
                    }
                    float top[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t* v = &x[i >> 1][(i & 1) * 16];
                        top[i] = __uint_as_float(v[0]);
#pragma unroll
                        for (int k = 1; k < 15; k += 2) top[i] = max_nan(top[i], __uint_as_float(v[k]), __uint_as_float(v[k + 1]));
                        top[i] = max_nan(top[i], __uint_as_float(v[15]));
                    }
                    // A NaN among the scores makes the maximum NaN from here on, and with it weights and sum (but for the columns of
                    // exp2_poly, which come out as some number).
                    const float mt = max_nan(max_nan(top[0], top[1]), max_nan(top[2], top[3])) * a.scale_log2 - kTopWeight<E>;
                    bool first = false;
                    if ((st & 62) == 0) {  // a tile behind thousands, or behind one large weight, is small against the whole sum
                        l_far += l;
                        l = 0.0f;
                        first = st < 2;
                        if (first) m = mt;
                    }
                    if (!first) {
                        const bool grown = valid && !(mt <= m + kRescaleAbove);  // or NaN
                        if (__any_sync(0xffffffffu, grown)) {
                            const float old = m;
                            m = max_nan(m, mt);
                            const float f = m == -INFINITY ? 1.0f : exp2_approx(old - m);
                            l *= f;
                            l_far *= f;
                            ok = sums_done(s, done);  // the step before
                            fence_after_sync();
                            if (ok) {
#pragma unroll 1
                                for (int i = 0; i < DP / 32; ++i) {
                                    uint32_t o[32];
                                    tmem_ld32(o, o_col + 32 * i);
                                    tmem_wait_ld(o);
#pragma unroll
                                    for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                                    tmem_st32(o_col + 32 * i, o);
                                }
                            }
                        }
                    }
                    const float2 sum = weights<E>(x, s_col + buf * 64, scale2, m, edge, seen);
                    l += sum.x + sum.y;
                    tmem_wait_st();
                }
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.p_full[s][buf]));
                ++done;
            }
            if (!ok) break;
            done_other += s ? (steps + 1) / 2 : steps / 2;
            const bool has_first = p.kv0 == 0, has_last = p.kv1 == p.nkv, whole = has_first && has_last;
            l += l_far;
            // exp2_poly leaves 2^-126 where a weight is zero, and where a score of +infinity stands against itself
            if (m == -INFINITY) l = 0.0f;
            else if (m == INFINITY) l = NAN;
            // every warp is through with the item before
            if (items > 0) ok = warp_wait(smem_addr(&sh.o_free), (items & 1) ^ 1, gave_up);
            if (!wide) {  // maxima and sums of both streams
                sh.m[s][row] = m;
                sh.l[s][row] = l;
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.stats));
                ok = ok && warp_wait(smem_addr(&sh.stats), narrow_items & 1, gave_up);
                ++narrow_items;
            }
            if (wide || s == 0 || steps > 1) ok = ok && sums_done(s, done);
            if (!wide && (s == 1 || steps > 1)) ok = ok && sums_done(s ^ 1, done_other);
            if (!ok) break;
            fence_after_sync();
            if (active) {
                float f0 = 1.0f, f1 = 0.0f;  // weights of the sums read below
                if (!wide) {
                    const float m0 = sh.m[0][row], m1 = sh.m[1][row];
                    m = max_nan(m0, m1);
                    f0 = m0 == -INFINITY ? 0.0f : exp2_approx(m0 - m);
                    f1 = m1 == -INFINITY ? 0.0f : exp2_approx(m1 - m);
                    l = sh.l[0][row] * f0 + sh.l[1][row] * f1;
                }
                if (has_first && m == -INFINITY && upto > 0) m = kLowest;  // a row that sees anything sees key 0
                const bool two = !wide && steps > 1;
                const int64_t out_row = p.r0 + tok;
                const int head = p.h * a.group + grp;
                const int64_t part_row = (int64_t)(2 * cta + (has_first ? 1 : 0)) * 256 + (wide ? s * 128 : 0) + row;
                if (whole) {
                    const float inv = inverse_sum(m, l);
                    f0 *= inv;
                    f1 *= inv;
                    if (valid && a.lse && (wide || s == 0)) a.lse[out_row * a.n_q_heads + head] = log_sum(m, l);
                } else if (valid && (wide || s == 0)) {
                    ws.ml[part_row] = make_float2(m, l);
                }
                E* const out = reinterpret_cast<E*>(a.out.p) + out_row * a.out.row_stride + (int64_t)head * a.out.head_stride;
                float* const po = ws.o + (part_row & ~255ll) * DP + (part_row & 255) * 4;  // column c: + (c / 4) * 1024 + c % 4
                const int c_lo = wide ? 0 : s * (DP / 2), c_hi = wide ? DP : c_lo + DP / 2;
                const uint32_t o0 = tmem + lanes + 256 + (wide ? s * 128 : 0);
#pragma unroll 1
                for (int c = c_lo; c < c_hi && c < a.head_dim; c += 32) {
                    uint32_t v[32], v1[32];
                    tmem_ld32(v, o0 + c);
                    if (two) tmem_ld32(v1, o0 + 128 + c);
                    tmem_wait_ld(v);
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * f0);
                    if (two) {
                        tmem_waited(v1);
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) + __uint_as_float(v1[k]) * f1);
                    }
                    if (!valid) continue;
                    if (whole ? m == -INFINITY : l == 0.0f) {  // nothing seen, or nothing of this piece, whatever values that was
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = 0u;
                    }
                    if (whole) {
#pragma unroll
                        for (int k = 0; k < 32; k += 8)
                            if (c + k < a.head_dim)
                                *reinterpret_cast<uint4*>(out + c + k) =
                                    make_uint4(pack2<E>(__uint_as_float(v[k]), __uint_as_float(v[k + 1])), pack2<E>(__uint_as_float(v[k + 2]), __uint_as_float(v[k + 3])),
                                               pack2<E>(__uint_as_float(v[k + 4]), __uint_as_float(v[k + 5])), pack2<E>(__uint_as_float(v[k + 6]), __uint_as_float(v[k + 7])));
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; k += 4)
                            if (c + k < a.head_dim) *reinterpret_cast<uint4*>(po + (c + k) * 256) = make_uint4(v[k], v[k + 1], v[k + 2], v[k + 3]);
                    }
                }
                if (valid && *static_cast<volatile int*>(&sh.not_finite[items % kFlags])) {
                    const int lo = max(item_sees, p.kv0 * kTileKeys), hi = p.kv1 == p.nkv ? kv_end : p.kv1 * kTileKeys;
                    restore_cleared<E>(a, p.b, p.h, lo, hi, upto, nodes, p.base + 1, c_lo, min(c_hi, a.head_dim), whole ? out : nullptr, po);
                }
            }
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sh.o_free));
            if (threadIdx.x == 0 && has_first && !has_last)
                ws.desc[cta] = SplitDesc{1, p.h, p.r0, p.tok0, p.n_tok, share_owner(shares, sh.open_unit), {0, 0}};

        }
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (warp == kMmaWarp) tmem_free(tmem, 512);
    if (threadIdx.x == 0 && sh.gave_up) atomicExch(a.c.dev_error, (int)HVD_DEV_WAIT_EXPIRED);
}

// Joins the pieces of the items that several CTAs shared (block x of the grid: the item that CTA x began and left
// unfinished), and gives the rows that see nothing for want of a token their zeros.  A warp takes 32 rows by 8 columns.
template <typename E, int DP>
__global__ void __launch_bounds__(kFinishThreads) attn_finish_kernel(const AttnArgs a, const Work ws, const int n_cta, const int tile_tok) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_trigger();
    pdl_wait();
    const int n_warp = gridDim.x * gridDim.y * (kFinishThreads / 32), me = (blockIdx.y * gridDim.x + blockIdx.x) * (kFinishThreads / 32) + warp;
    const bool spare = n_cta == 0 || *ws.spare != 0;
    const int chunks = a.head_dim / 8, at = blockIdx.x;
    SplitDesc d = {};
    if (at < n_cta) d = ws.desc[at];
    const int rows = d.valid ? d.n_tok * a.group : 0, n = d.c_last - at + 1;
    for (int u = blockIdx.y * (kFinishThreads / 32) + warp; u < (rows + 31) / 32 * chunks; u += gridDim.y * (kFinishThreads / 32)) {
        const int block = u / chunks, ch = u - block * chunks, row = block * 32 + lane;
        if (row >= rows) continue;
        // row of the item: token row / group; its place among the partial sums
        const int t = row / a.group, grp = row - t * a.group;
        const int place = t < tile_tok ? row : 128 + row - tile_tok * a.group;
        float acc[8] = {}, l = 0.0f, m = -INFINITY;
        for (int i0 = 0; i0 < n; i0 += kJoin) {  // rescaled to the largest maximum so far
            float2 ml[kJoin];
            float4 o[kJoin][2];
#pragma unroll
            for (int k = 0; k < kJoin; ++k) {
                ml[k] = make_float2(-INFINITY, 0.0f);
                o[k][0] = o[k][1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (i0 + k < n) {
                    const int64_t slot = 2 * (at + i0 + k) + (i0 + k == 0 ? 1 : 0);
                    ml[k] = ws.ml[slot * 256 + place];
                    const float* q = ws.o + (slot * (DP / 4) + 2 * ch) * 1024 + place * 4;
                    o[k][0] = *reinterpret_cast<const float4*>(q);
                    o[k][1] = *reinterpret_cast<const float4*>(q + 1024);
                }
            }
            const float old = m;
#pragma unroll
            for (int k = 0; k < kJoin; ++k) m = max_nan(m, ml[k].x);
            if (m == -INFINITY) continue;
            const float keep = exp2_approx(old - m);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] *= keep;
            l *= keep;
#pragma unroll
            for (int k = 0; k < kJoin; ++k) {
                const float f = exp2_approx(ml[k].x - m);
                l += ml[k].y * f;
                acc[0] += o[k][0].x * f; acc[1] += o[k][0].y * f; acc[2] += o[k][0].z * f; acc[3] += o[k][0].w * f;
                acc[4] += o[k][1].x * f; acc[5] += o[k][1].y * f; acc[6] += o[k][1].z * f; acc[7] += o[k][1].w * f;
            }
        }
        const int64_t out_row = d.r0 + d.tok0 + t;
        const int head = d.h * a.group + grp;
        if (!HVD_IN_BOUNDS(a.c.dev_error, out_row, 0, a.c.total_rows)) continue;
        const float inv = inverse_sum(m, l);
        *reinterpret_cast<uint4*>(reinterpret_cast<E*>(a.out.p) + out_row * a.out.row_stride + (int64_t)head * a.out.head_stride + 8 * ch) =
            make_uint4(pack2<E>(acc[0] * inv, acc[1] * inv), pack2<E>(acc[2] * inv, acc[3] * inv), pack2<E>(acc[4] * inv, acc[5] * inv),
                       pack2<E>(acc[6] * inv, acc[7] * inv));
        if (a.lse && ch == 0) a.lse[out_row * a.n_q_heads + head] = log_sum(m, l);
    }
    // Requests: status, rows that are no new token (with drafts shorter than their rows most of the batch), several warps a request.
    if (a.status && blockIdx.y == gridDim.y - 1)
        for (int b = blockIdx.x * kFinishThreads + threadIdx.x; b < a.c.B; b += gridDim.x * kFinishThreads)
            a.status[b] = load_chunk(a.c, b).bad ? HVD_REQ_BAD_LEN : HVD_REQ_OK;
    if (!spare) return;
    const int share = max(1, n_warp / a.c.B), nvec = a.head_dim / 8;
    for (uint32_t x = me; x < (uint32_t)(a.c.B * share); x += n_warp) {
        const int s = (int)(x / (uint32_t)a.c.B), b = (int)x - s * a.c.B;
        const Chunk c = load_chunk(a.c, b);
        for (int64_t i = (int64_t)c.n_new + s; i < c.rows; i += share) {
            const int64_t row = c.r0 + i;
            if (!HVD_IN_BOUNDS(a.c.dev_error, row, 0, a.c.total_rows)) continue;
            for (int v = lane; v < a.n_q_heads * nvec; v += 32) {
                const int h = v / nvec, e = v - h * nvec;
                *reinterpret_cast<uint4*>(reinterpret_cast<E*>(a.out.p) + row * a.out.row_stride + (int64_t)h * a.out.head_stride + 8 * e) = make_uint4(0u, 0u, 0u, 0u);
            }
            if (a.lse)
                for (int h = lane; h < a.n_q_heads; h += 32) a.lse[row * a.n_q_heads + h] = -INFINITY;
        }
    }
}

// ---------------------------------------------------------------- host

PFN_cuTensorMapEncodeTiled encode_fn() {
    static PFN_cuTensorMapEncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled>(p);
    }();
    return fn;
}

struct Dim {
    uint64_t size, stride;  // elements
    uint32_t box;
};

// a tensor of 16-bit elements, the head's elements innermost, in boxes of 64 of them (128 bytes, swizzled)
bool encode(CUtensorMap* map, bool f16, void* base, int head_dim, const Dim (&d)[3]) {
    const cuuint64_t size[4] = {(cuuint64_t)head_dim, d[0].size, d[1].size, d[2].size};
    const cuuint64_t stride[3] = {2 * d[0].stride, 2 * d[1].stride, 2 * d[2].stride};
    const cuuint32_t box[4] = {64, d[0].box, d[1].box, d[2].box}, one[4] = {1, 1, 1, 1};
    return encode_fn()(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, size, stride, box, one,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int gcd(int x, int y) { return y == 0 ? x : gcd(y, x % y); }

template <typename E, int DP>
hvd_status run(hvd_ctx* ctx, const AttnArgs& a, bool f16, cudaStream_t stream) {
    const ChunkArgs& c = a.c;
    const bool pdl = (ctx->pdl_mask & 16) != 0;
    const int n_cta = ctx->num_sms;
    Work ws;
    char* p = static_cast<char*>(ctx->at_ws);
    ws.o = reinterpret_cast<float*>(p);
    ws.ml = reinterpret_cast<float2*>(p + (size_t)n_cta * 2 * 256 * DP * sizeof(float));
    ws.desc = reinterpret_cast<SplitDesc*>(ws.ml + (size_t)n_cta * 2 * 256);
    ws.spare = reinterpret_cast<int*>(ws.desc + n_cta);
    // query boxes: as few tokens as fill whole groups of 8 rows, so that every box starts on a 1024-byte boundary
    int box_tok = 8 / gcd(a.group, 8);
    if (box_tok * a.group > kTileRows) box_tok = kTileRows / a.group;
    int tile_tok = kTileRows / a.group;
    if (tile_tok > box_tok) tile_tok -= tile_tok % box_tok;
    const int box_keys = gcd(c.page_size, kTileKeys);
    cudaError_t e;
    if (c.total_rows > 0) {
        CUtensorMap mq, mk, mv;
        const Dim dq[3] = {{(uint64_t)a.group, (uint64_t)a.q.head_stride, (uint32_t)a.group},
                           {(uint64_t)c.total_rows, (uint64_t)a.q.row_stride, (uint32_t)box_tok},
                           {(uint64_t)a.n_kv_heads, (uint64_t)a.q.head_stride * a.group, 1}};
        const Dim dk[3] = {{(uint64_t)c.page_size, (uint64_t)c.slot_stride, (uint32_t)box_keys},
                           {(uint64_t)a.n_kv_heads, (uint64_t)c.head_stride, 1},
                           {(uint64_t)c.n_pages, (uint64_t)c.page_stride, 1}};
        if (!encode(&mq, f16, a.q.p, a.head_dim, dq) || !encode(&mk, f16, c.k, a.head_dim, dk) || !encode(&mv, f16, c.v, a.head_dim, dk))
            return fail(ctx, HVD_ERR_INVALID_ARG, "hvd_attn_paged: q or the cache has strides that TMA does not take");
        e = launch_kernel(pdl, attn_tile_kernel<E, DP>, dim3(n_cta), dim3(kThreads), kSmemBytes<DP>, stream, a, ws, Geometry{tile_tok, 2 * tile_tok}, box_keys, box_tok, mq, mk, mv);
        if (e != cudaSuccess) return cuda_fail(ctx, e, "attn_tile_kernel");
    }
    // blocks for as many units as an item can have here, eight at most: the SMs hold so many at once
    const int64_t units = ((c.total_rows * a.group < 256 ? c.total_rows * a.group : 256) + 31) / 32 * (a.head_dim / 8);
    const int by = units > 56 ? 8 : units > 8 ? (int)((units + 7) / 8) : 1;
    e = launch_kernel(pdl, attn_finish_kernel<E, DP>, dim3(n_cta, by), dim3(kFinishThreads), 0, stream, a, ws, c.total_rows > 0 ? n_cta : 0, tile_tok);
    return e == cudaSuccess ? HVD_OK : cuda_fail(ctx, e, "attn_finish_kernel");
}

}  // namespace

size_t attn_workspace_bytes(int num_sms, int head_dim) {
    const int dp = head_dim > 64 ? 128 : 64;
    return (size_t)num_sms * (2 * 256 * (dp * sizeof(float) + sizeof(float2)) + sizeof(SplitDesc)) + 16;
}

hvd_status attn_setup(hvd_ctx* ctx) {
    if (!encode_fn()) return fail(ctx, HVD_ERR_UNSUPPORTED, "hvd_set_attention: the driver does not encode tensor maps");
    auto opt_in = [](auto kernel, int bytes) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); };
    HVD_CUDA_TRY(ctx, opt_in(attn_tile_kernel<__nv_bfloat16, 64>, kSmemBytes<64>));
    HVD_CUDA_TRY(ctx, opt_in(attn_tile_kernel<__nv_bfloat16, 128>, kSmemBytes<128>));
    HVD_CUDA_TRY(ctx, opt_in(attn_tile_kernel<__half, 64>, kSmemBytes<64>));
    HVD_CUDA_TRY(ctx, opt_in(attn_tile_kernel<__half, 128>, kSmemBytes<128>));
    return HVD_OK;
}

hvd_status launch_attn(hvd_ctx* ctx, const AttnArgs& a, bool f16, cudaStream_t stream) {
    if (a.head_dim > 64) return f16 ? run<__half, 128>(ctx, a, true, stream) : run<__nv_bfloat16, 128>(ctx, a, false, stream);
    return f16 ? run<__half, 64>(ctx, a, true, stream) : run<__nv_bfloat16, 64>(ctx, a, false, stream);
}

}  // namespace hvd
