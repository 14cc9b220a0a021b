// hvd_attn_paged: attention of a chunk's rows over the paged cache, on the 5th-generation tensor cores.
//
// The rows of a key/value head are the chunk's tokens times the query heads of its group, packed into tiles of
// 128 rows; keys come in tiles of 128.  Per pair of tiles, S = Q K^T lands in tensor memory, a warpgroup turns it into
// weights P = exp2(S - m) with the running maximum m and sum of a softmax (one thread per row: no shuffles), and
// O += P V takes P from tensor memory.
//
// Two STREAMS of such products run against each other, so that one's softmax hides behind the other's products:
//   wide items (more than 128 rows)   the streams are two row tiles that share every key tile
//   narrow items                      the streams are the even and the odd key tiles of one row tile, joined at the end
// Roles of the 12 warps: 0-3 and 4-7 softmax, rescaling and output of stream 0 and 1; 8 issues the products; 9 the
// TMA loads, box by box through the page table; 10 and 11 only lend their registers.  K and V tiles share one ring of slots in the order of their use.
//
// Work is counted in key tiles over all (request, head, group of rows) items and dealt to the SMs in equal
// consecutive shares, whatever the lengths; every CTA finds its share from the lengths itself.  An item that
// several CTAs share leaves partial sums, which attn_finish_kernel joins in the order of the CTAs: no result depends on
// timing.
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hvd_attn.cuh"
#include "hvd_sm100.cuh"

namespace hvd {

using namespace sm100;

namespace {

constexpr int kSoftmaxWarps = 8, kMmaWarp = 8, kLoadWarp = 9;
constexpr int kThreads = 384;
// registers: 384 threads start with 168 each; the softmax warpgroups take 208, the third keeps 88 (208 + 208 + 88 = 3 * 168)
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;
constexpr int kFinishThreads = 256;
constexpr float kRescaleAbove = 8.0f;  // log2: a maximum that grew by less keeps its old value (weights up to 2^8 are exact in either type)
constexpr float kLn2 = 0.6931471805599453f;

template <int DP> struct Shape {
    static constexpr int kHalves = DP / 64;                     // 128-byte columns of a tile row
    static constexpr int kHalfBytes = 128 * 128;
    static constexpr int kTileBytes = kHalves * kHalfBytes;     // one tile of Q, K or V
    static constexpr int kSlots = DP == 128 ? 5 : 8;            // K / V ring: 160 or 128 KB
};

struct Shared {  // behind the tiles
    uint64_t full[8], empty[8];      // ring slots
    uint64_t q_full, q_empty;        // the item's query tiles
    uint64_t s_full[2], p_full[2];   // scores written, weights written
    uint64_t o_full[2];              // a step's product with V is done
    uint64_t stats, o_free;          // maxima and sums of both streams exchanged; the item's sums are read
    uint64_t drain;
    uint32_t tmem;
    int gave_up;
    int start_b;
    long long start_off;
    long long warp_sum[kThreads / 32];
    float m[2][128], l[2][128];  // [stream][row]
};
template <int DP> constexpr int kSmemBytes = (2 + Shape<DP>::kSlots) * Shape<DP>::kTileBytes + (int)sizeof(Shared);
static_assert(kSmemBytes<128> <= 227 * 1024 && kSmemBytes<64> <= 227 * 1024, "shared memory of a CTA");

// One CTA's partial sums: slot 0 an item that an earlier CTA began, slot 1 an item that a later CTA goes on with.
struct SplitDesc {
    int valid, b, h, qt, tok0, n_tok, c_last, wide;
};

struct Work {
    SplitDesc* desc;   // [CTAs]
    float* o;          // [CTAs][2][256][DP]
    float2* ml;        // [CTAs][2][256] maximum (log2 units), sum
};

// ---------------------------------------------------------------- items

struct Geometry {
    int tile_tok;  // tokens of a row tile
    int item_tok;  // tokens of an item: two row tiles
};

__device__ __forceinline__ int key_tiles(const Chunk& c, const Geometry& g, int qt) {
    return (c.base + min(c.n_new, (qt + 1) * g.item_tok) - 1) / kTileKeys + 1;
}

// key tiles of one head of a request
__device__ __forceinline__ long long head_units(const Chunk& c, const Geometry& g) {
    long long u = 0;
    for (int qt = 0; qt * g.item_tok < c.n_new; ++qt) u += key_tiles(c, g, qt);
    return u;
}

struct Piece {
    Chunk c;
    int b, h, qt;
    int tok0, n_tok;    // tokens of the item
    int kv0, kv1, nkv;  // key tiles of this CTA's piece, of the whole item
    int kv_end;         // tokens that any row of the item may see
    bool wide;
};

// A CTA's share as a sequence of pieces; every role walks it for itself.
struct Walk {
    long long left;  // units still to do
    int b, h, qt, kv;
    Chunk c;
};

__device__ __forceinline__ bool next_piece(const AttnArgs& a, const Geometry& g, Walk& w, Piece& p) {
    if (w.left <= 0) return false;
    while (w.qt * g.item_tok >= w.c.n_new) {  // past the head's last item
        w.qt = 0;
        if (w.c.n_new == 0 || ++w.h == a.n_kv_heads) {
            w.h = 0;
            if (++w.b >= a.c.B) return false;
            w.c = load_chunk(a.c, w.b);
        }
    }
    p.c = w.c; p.b = w.b; p.h = w.h; p.qt = w.qt;
    p.tok0 = w.qt * g.item_tok;
    p.n_tok = min(g.item_tok, w.c.n_new - p.tok0);
    p.wide = p.n_tok > g.tile_tok;
    p.nkv = key_tiles(w.c, g, w.qt);
    p.kv_end = w.c.base + p.tok0 + p.n_tok;
    p.kv0 = w.kv;
    p.kv1 = (int)min((long long)p.nkv, p.kv0 + w.left);
    w.left -= p.kv1 - p.kv0;
    w.kv = 0;
    ++w.qt;
    return true;
}

// a wait of a whole warp: all lanes go on, or none
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* gave_up) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, gave_up));
}

// position of a step's K and V tile in the order of loads (and of use) of a piece
__device__ __forceinline__ int k_pos(bool wide, int n) { return wide ? (n & ~1) : (n == 0 ? 0 : 2 * n - 1); }
__device__ __forceinline__ int v_pos(bool wide, int n, int steps) { return wide ? (n | 1) : (n < steps - 1 ? 2 * n + 2 : 2 * steps - 1); }

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

// visible columns of a key tile, one bit each
struct Seen {
    uint32_t w[4];
};

__device__ __forceinline__ Seen first_columns(int n) {
    Seen s;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = n - 32 * i;
        s.w[i] = k >= 32 ? 0xffffffffu : (k <= 0 ? 0u : (1u << k) - 1u);
    }
    return s;
}

// bits of `nodes` shifted so that node j is column at + j (at may be negative)
__device__ __forceinline__ void add_nodes(Seen& s, unsigned long long nodes, int at) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int sh = 32 * i - at;  // first node of word i
        unsigned long long v = 0ull;
        if (sh >= 0 && sh < 64) v = nodes >> sh;
        else if (sh < 0 && sh > -32) v = nodes << (-sh);
        s.w[i] |= (uint32_t)v;
    }
}

template <typename E, int DP>
__global__ void __launch_bounds__(kThreads, 1)
attn_tile_kernel(const AttnArgs a, const Work ws, const int box_keys, const int box_tok, const __grid_constant__ CUtensorMap map_q,
                 const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    using S = Shape<DP>;
    extern __shared__ __align__(1024) unsigned char dyn[];
    Shared& sh = *reinterpret_cast<Shared*>(dyn + (2 + S::kSlots) * S::kTileBytes);
    const uint32_t tiles = smem_addr(dyn);  // 1024-byte aligned: the kernel has no other shared memory
    const uint32_t ring = tiles + 2 * S::kTileBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* gave_up = &sh.gave_up;

    pdl_trigger();
    if (warp == kMmaWarp) tmem_alloc(smem_addr(&sh.tmem), 512);
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kSlots; ++i) { mbar_init(smem_addr(&sh.full[i]), 1); mbar_init(smem_addr(&sh.empty[i]), 1); }
        mbar_init(smem_addr(&sh.q_full), 1);
        mbar_init(smem_addr(&sh.q_empty), 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&sh.s_full[i]), 1);
            mbar_init(smem_addr(&sh.p_full[i]), 4);
            mbar_init(smem_addr(&sh.o_full[i]), 1);
        }
        mbar_init(smem_addr(&sh.stats), kSoftmaxWarps);
        mbar_init(smem_addr(&sh.o_free), kSoftmaxWarps);
        mbar_init(smem_addr(&sh.drain), 1);
        mbar_init_fence();
        sh.gave_up = 0;
    }
    if (warp == kLoadWarp && lane < 3) tma_prefetch_map(lane == 0 ? &map_q : (lane == 1 ? &map_k : &map_v));
    pdl_wait();

    // ---- this CTA's share: units of all requests before each thread's, then the request that holds the share's first unit
    Geometry g;
    g.tile_tok = kTileRows / a.group;
    if (g.tile_tok > box_tok) g.tile_tok -= g.tile_tok % box_tok;
    g.item_tok = 2 * g.tile_tok;
    const int per = (a.c.B + kThreads - 1) / kThreads;
    const int b0 = min(a.c.B, (int)threadIdx.x * per), b1 = min(a.c.B, b0 + per);
    long long mine = 0;
    for (int b = b0; b < b1; ++b) mine += head_units(load_chunk(a.c, b), g) * a.n_kv_heads;
    long long upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += t;
    }
    if (lane == 31) sh.warp_sum[warp] = upto;
    __syncthreads();
    long long total = 0, before = upto - mine;
    for (int i = 0; i < kThreads / 32; ++i) {
        if (i < warp) before += sh.warp_sum[i];
        total += sh.warp_sum[i];
    }
    const int n_cta = (int)min((long long)gridDim.x, total);
    const int cta = blockIdx.x;
    const long long first = cta < n_cta ? cta * total / n_cta : 0;
    const long long last = cta < n_cta ? (cta + 1) * total / n_cta : 0;
    if (cta < n_cta && first >= before && first < before + mine) {
        long long off = first - before;
        int b = b0;
        for (; b < b1 - 1; ++b) {
            const long long u = head_units(load_chunk(a.c, b), g) * a.n_kv_heads;
            if (off < u) break;
            off -= u;
        }
        sh.start_b = b;
        sh.start_off = off;
    }
    if (threadIdx.x == 0) ws.desc[cta].valid = 0;
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = sh.tmem;

    Walk walk = {};
    walk.left = last - first;
    if (walk.left > 0) {
        walk.b = sh.start_b;
        walk.c = load_chunk(a.c, walk.b);
        long long off = sh.start_off;
        const long long hu = head_units(walk.c, g);
        walk.h = (int)(off / hu);
        off -= walk.h * hu;
        for (;; ++walk.qt) {
            const int u = key_tiles(walk.c, g, walk.qt);
            if (off < u) break;
            off -= u;
        }
        walk.kv = (int)off;
    }
    const uint32_t full0 = smem_addr(&sh.full[0]), empty0 = smem_addr(&sh.empty[0]);
    Piece p;

    if (warp >= kSoftmaxWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == kLoadWarp) {
        // ------------------------------------------------------------ loads
        int pos = 0, items = 0;  // ring position of the piece's first tile; pieces done
        const int n_box = kTileKeys / box_keys;
        bool ok = true;
        while (ok && next_piece(a, g, walk, p)) {
            const int tiles_n = p.kv1 - p.kv0;
            const int* table = a.c.page_table + (int64_t)p.b * a.c.table_stride;
            auto load = [&](const CUtensorMap* map, int at, int tile) {  // one K or V tile into ring position `at`
                const int slot = at % S::kSlots, round = at / S::kSlots;
                const uint32_t bar = full0 + 8 * slot;
                const int key = tile * kTileKeys + lane * box_keys;
                const bool need = lane < n_box && key < p.kv_end;
                int page = -1, in = 0;
                if (need) {
                    const int j = key / a.c.page_size;
                    in = key - j * a.c.page_size;
                    if (HVD_IN_BOUNDS(a.c.dev_error, j, 0, a.c.table_stride)) page = table[j];
                    if (page < 0 || page >= a.c.n_pages) page = -1;  // the box lies outside the tensor: zeros
                }
                if (!warp_wait(empty0 + 8 * slot, (round & 1) ^ 1, gave_up)) return false;
                const int boxes = __popc(__ballot_sync(0xffffffffu, need));
                if (lane == 0) mbar_expect(bar, (uint32_t)(boxes * box_keys * 128 * S::kHalves));
                __syncwarp();
                if (need) {
#pragma unroll
                    for (int hf = 0; hf < S::kHalves; ++hf)
                        tma_load_4d(ring + slot * S::kTileBytes + hf * S::kHalfBytes + lane * box_keys * 128, map, bar, hf * 64, in, p.h, page);
                }
                return true;
            };
            // the first keys do not wait for the previous item's queries to be done with
            ok = load(&map_k, pos, p.kv0);
            ok = ok && warp_wait(smem_addr(&sh.q_empty), (items & 1) ^ 1, gave_up);
            if (!ok) break;
            const int per_tile = g.tile_tok, n_tiles = p.wide ? 2 : 1;
            int q_boxes = 0;
            for (int t = 0; t < n_tiles; ++t) q_boxes += (min(per_tile, p.n_tok - t * per_tile) + box_tok - 1) / box_tok;
            if (lane == 0) mbar_expect(smem_addr(&sh.q_full), (uint32_t)(q_boxes * box_tok * a.group * 128 * S::kHalves));
            __syncwarp();
            for (int t = 0; t < n_tiles; ++t) {
                const int nb = (min(per_tile, p.n_tok - t * per_tile) + box_tok - 1) / box_tok;
                for (int i = lane; i < nb * S::kHalves; i += 32) {
                    const int bx = i / S::kHalves, hf = i % S::kHalves;
                    tma_load_4d(tiles + t * S::kTileBytes + hf * S::kHalfBytes + bx * box_tok * a.group * 128, &map_q, smem_addr(&sh.q_full), hf * 64,
                                0, (int)(p.c.r0 + p.tok0 + t * per_tile + bx * box_tok), p.h);
                }
            }
            if (p.wide) {
                ok = load(&map_v, pos + 1, p.kv0);
                for (int j = 1; ok && j < tiles_n; ++j)
                    ok = load(&map_k, pos + 2 * j, p.kv0 + j) && load(&map_v, pos + 2 * j + 1, p.kv0 + j);
            } else {
                if (tiles_n > 1) ok = load(&map_k, pos + 1, p.kv0 + 1);
                for (int j = 0; ok && j < tiles_n; ++j) {
                    ok = load(&map_v, pos + v_pos(false, j, tiles_n), p.kv0 + j);
                    if (ok && j + 2 < tiles_n) ok = load(&map_k, pos + k_pos(false, j + 2), p.kv0 + j + 2);
                }
            }
            pos += 2 * tiles_n;
            ++items;
        }
        if (!ok) {  // gave up: a bounded wait for every slot's last load before the shared memory is given back
            const unsigned long long t0 = now_ns();
            while (now_ns() - t0 < kWaitLimitNs / 100) {}
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------ products
        if (elect_one()) {
            const bool f16 = sizeof(E) == 2 && std::is_same<E, __half>::value;
            const int ksteps = (a.head_dim + 15) / 16;
            const uint32_t qk_desc = instr_desc(f16, 128, kTileKeys, false), pv_desc = instr_desc(f16, 128, ksteps * 16, true);
            int pos = 0, items = 0, steps_done[2] = {0, 0};
            bool ok = true;
            while (ok && next_piece(a, g, walk, p)) {
                const int tiles_n = p.kv1 - p.kv0, steps = p.wide ? 2 * tiles_n : tiles_n;
                auto scores = [&](int n) {  // S = Q K^T of step n
                    const int s = n & 1, at = pos + k_pos(p.wide, n), slot = at % S::kSlots;
                    if (!mbar_wait(full0 + 8 * slot, (at / S::kSlots) & 1, gave_up)) return false;
                    fence_after_sync();
                    const uint32_t qa = tiles + (p.wide ? s : 0) * S::kTileBytes, kb = ring + slot * S::kTileBytes;
                    for (int k = 0; k < ksteps; ++k) {
                        const uint32_t off = (k >> 2) * S::kHalfBytes + (k & 3) * 32;
                        mma_ss(tmem + s * 128, operand_desc(qa + off, 16), operand_desc(kb + off, 16), qk_desc, k > 0);
                    }
                    mma_commit(smem_addr(&sh.s_full[s]));
                    if (!p.wide || s == 1) mma_commit(empty0 + 8 * slot);
                    if (n == steps - 1) mma_commit(smem_addr(&sh.q_empty));
                    return true;
                };
                ok = mbar_wait(smem_addr(&sh.q_full), items & 1, gave_up) && scores(0) && (steps == 1 || scores(1));
                for (int n = 0; ok && n < steps; ++n) {
                    const int s = n & 1, at = pos + v_pos(p.wide, n, steps), slot = at % S::kSlots;
                    ok = mbar_wait(smem_addr(&sh.p_full[s]), steps_done[s] & 1, gave_up) && mbar_wait(full0 + 8 * slot, (at / S::kSlots) & 1, gave_up);
                    if (ok && n == 0) ok = mbar_wait(smem_addr(&sh.o_free), (items & 1) ^ 1, gave_up);  // the last item's sums are read
                    if (!ok) break;
                    fence_after_sync();
                    const uint32_t vb = ring + slot * S::kTileBytes;
#pragma unroll
                    for (int k = 0; k < kTileKeys / 16; ++k)
                        mma_ts(tmem + 256 + s * 128, tmem + s * 128 + 8 * k, operand_desc(vb + k * 2048, S::kHalfBytes), pv_desc, n >= 2 || k > 0);
                    mma_commit(smem_addr(&sh.o_full[s]));
                    if (!p.wide || s == 1) mma_commit(empty0 + 8 * slot);
                    ++steps_done[s];
                    if (n + 2 < steps) ok = scores(n + 2);
                }
                pos += 2 * tiles_n;
                ++items;
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
        int pos = 0, items = 0, narrow_items = 0, done[2] = {0, 0};
        bool ok = true;
        while (ok && next_piece(a, g, walk, p)) {
            const int tiles_n = p.kv1 - p.kv0, steps = p.wide ? 2 * tiles_n : tiles_n;
            const int tok0 = p.tok0 + (p.wide ? s * g.tile_tok : 0);
            const int n_rows = min(g.tile_tok, p.tok0 + p.n_tok - tok0) * a.group;
            const int tok = tok0 + row / a.group, grp = row % a.group;
            const bool valid = row < n_rows, active = (row & ~31) < n_rows;
            // what the row sees: keys below `upto`, in a tree also the nodes on its line
            unsigned long long nodes = 0ull;
            int upto = p.c.base + tok + 1;
            if (a.c.parent) {
                int depth;
                const bool reach = !valid || tree_line(a.c, p.b, tok, nodes, depth);
                upto = reach ? p.c.base + 1 : 0;
            }
            const int all_see = __reduce_min_sync(0xffffffffu, valid ? upto : 0x7fffffff);
            float m = -INFINITY, l = 0.0f;
            for (int n = s; ok && n < steps; n += 2) {
                const int tile = p.kv0 + (p.wide ? n >> 1 : n), key0 = tile * kTileKeys;
                ok = warp_wait(smem_addr(&sh.s_full[s]), done[s] & 1, gave_up);
                if (!ok) break;
                fence_after_sync();
                if (active) {
                    uint32_t x[4][32];
#pragma unroll
                    for (int i = 0; i < 4; ++i) tmem_ld32(x[i], s_col + 32 * i);
                    tmem_wait_ld(x[0]);
#pragma unroll
                    for (int i = 1; i < 4; ++i) tmem_waited(x[i]);
                    if (key0 + kTileKeys > all_see) {  // some row of the warp does not see the whole tile
                        Seen seen = first_columns(upto - key0);
                        if (a.c.parent) add_nodes(seen, nodes, p.c.base + 1 - key0);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (!((seen.w[i] >> j) & 1u)) x[i][j] = 0xff800000u;
                    }
                    float top[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        top[i] = __uint_as_float(x[i][0]);
#pragma unroll
                        for (int j = 1; j < 32; ++j) top[i] = fmaxf(top[i], __uint_as_float(x[i][j]));
                    }
                    const float mt = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.scale_log2;
                    if (n < 2) {
                        m = mt;
                    } else {
                        const bool grown = valid && mt > m + kRescaleAbove;
                        if (__any_sync(0xffffffffu, grown)) {
                            const float old = m;
                            m = fmaxf(m, mt);
                            const float f = m == -INFINITY ? 1.0f : exp2_approx(old - m);
                            l *= f;
                            ok = warp_wait(smem_addr(&sh.o_full[s]), (done[s] & 1) ^ 1, gave_up);  // the step before
                            fence_after_sync();
                            if (ok) {
#pragma unroll
                                for (int i = 0; i < DP / 32; ++i) {
                                    uint32_t o[32];
                                    tmem_ld32(o, o_col + 32 * i);
                                    tmem_wait_ld(o);
#pragma unroll
                                    for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                                    tmem_st32(o_col + 32 * i, o);
                                }
                            }
                        }
                    }
                    const float shift = m == -INFINITY ? 0.0f : m;
                    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t w[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const float p0 = exp2_approx(fmaf(__uint_as_float(x[i][2 * j]), a.scale_log2, -shift));
                            const float p1 = exp2_approx(fmaf(__uint_as_float(x[i][2 * j + 1]), a.scale_log2, -shift));
                            sum[j & 3] += p0 + p1;
                            w[j] = pack2<E>(p0, p1);
                        }
                        tmem_st16(s_col + 16 * i, w);
                    }
                    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    tmem_wait_st();
                }
                // slots at and behind the item's last key may hold anything: 0 * NaN must not reach the sums
                if (key0 + kTileKeys > p.kv_end && (!p.wide || s == 0)) {
                    const int at = pos + v_pos(p.wide, n, steps), slot = at % S::kSlots;
                    ok = ok && warp_wait(full0 + 8 * slot, (at / S::kSlots) & 1, gave_up);
                    const int keep = p.kv_end - key0;  // rows that stay
                    for (int i = row; i < (kTileKeys - keep) * 8 * S::kHalves; i += 128) {
                        const int hf = i / ((kTileKeys - keep) * 8), r = i - hf * (kTileKeys - keep) * 8;
                        const uint32_t at_b = ring + slot * S::kTileBytes + hf * S::kHalfBytes + keep * 128 + r * 16;
                        if (ok) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at_b), "r"(0) : "memory");
                    }
                    fence_async_proxy();
                }
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.p_full[s]));
                ++done[s];
            }
            // the other stream's steps, for its barrier's parity
            const int steps_of[2] = {(steps + 1) / 2, steps / 2};
            done[s ^ 1] += steps_of[s ^ 1];
            const bool has_first = p.kv0 == 0, has_last = p.kv1 == p.nkv, whole = has_first && has_last;
            float* const part_o = ws.o + ((int64_t)(2 * cta + (has_first ? 1 : 0)) * 256) * DP;
            float2* const part_ml = ws.ml + (int64_t)(2 * cta + (has_first ? 1 : 0)) * 256;
            if (!p.wide) {  // maxima and sums of both streams, once every warp is through with the item before
                if (items > 0) ok = ok && warp_wait(smem_addr(&sh.o_free), (items & 1) ^ 1, gave_up);
                sh.m[s][row] = m;
                sh.l[s][row] = l;
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.stats));
                ok = ok && warp_wait(smem_addr(&sh.stats), narrow_items & 1, gave_up);
                ++narrow_items;
            }
            if (steps_of[0] && (!p.wide || s == 0)) ok = ok && warp_wait(smem_addr(&sh.o_full[0]), (done[0] & 1) ^ 1, gave_up);
            if (steps_of[1] && (!p.wide || s == 1)) ok = ok && warp_wait(smem_addr(&sh.o_full[1]), (done[1] & 1) ^ 1, gave_up);
            fence_after_sync();
            if (ok && active) {
                float f0 = 1.0f, f1 = 0.0f;  // weights of the sums read below
                if (!p.wide) {
                    const float m0 = sh.m[0][row], m1 = sh.m[1][row];
                    m = fmaxf(m0, m1);
                    f0 = m0 == -INFINITY ? 0.0f : exp2_approx(m0 - m);
                    f1 = m1 == -INFINITY ? 0.0f : exp2_approx(m1 - m);
                    l = sh.l[0][row] * f0 + (f1 > 0.0f ? sh.l[1][row] * f1 : 0.0f);
                }
                const bool two = !p.wide && steps > 1;
                const int64_t out_row = p.c.r0 + tok;
                const int head = p.h * a.group + grp;
                if (whole) {
                    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                    f0 *= inv;
                    f1 *= inv;
                    if (valid && a.lse && (p.wide || s == 0)) a.lse[out_row * a.n_q_heads + head] = l > 0.0f ? (m + log2f(l)) * kLn2 : -INFINITY;
                } else if (valid && (p.wide || s == 0)) {
                    part_ml[(p.wide ? s * 128 : 0) + row] = make_float2(m, l);
                }
                E* const out = reinterpret_cast<E*>(a.out.p) + out_row * a.out.row_stride + (int64_t)head * a.out.head_stride;
                float* const po = part_o + (int64_t)((p.wide ? s * 128 : 0) + row) * DP;
                const int c_lo = p.wide ? 0 : s * (DP / 2), c_hi = p.wide ? DP : c_lo + DP / 2;
                const uint32_t o0 = tmem + lanes + 256 + (p.wide ? s * 128 : 0);
#pragma unroll 1
                for (int c = c_lo; c < c_hi && c < a.head_dim; c += 32) {
                    uint32_t v[32];
                    tmem_ld32(v, o0 + c);
                    tmem_wait_ld(v);
                    if (two) {
                        uint32_t v1[32];
                        tmem_ld32(v1, o0 + 128 + c);
                        tmem_wait_ld(v1);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * f0 + __uint_as_float(v1[j]) * f1);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * f0);
                    }
                    if (!valid) continue;
                    if (whole) {
#pragma unroll
                        for (int j = 0; j < 32; j += 8)
                            if (c + j < a.head_dim)
                                *reinterpret_cast<uint4*>(out + c + j) =
                                    make_uint4(pack2<E>(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), pack2<E>(__uint_as_float(v[j + 2]), __uint_as_float(v[j + 3])),
                                               pack2<E>(__uint_as_float(v[j + 4]), __uint_as_float(v[j + 5])), pack2<E>(__uint_as_float(v[j + 6]), __uint_as_float(v[j + 7])));
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; j += 4)
                            if (c + j < a.head_dim) *reinterpret_cast<uint4*>(po + c + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                    }
                }
            }
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sh.o_free));
            if (threadIdx.x == 0 && has_first && !has_last) {
                // the CTA that holds the item's last unit; this piece is the share's last
                const long long last_unit = last + (p.nkv - p.kv1) - 1;
                ws.desc[cta] = SplitDesc{1, p.b, p.h, p.qt, p.tok0, p.n_tok, (int)(((last_unit + 1) * n_cta - 1) / total), p.wide};
            }
            pos += 2 * tiles_n;
            ++items;
        }
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (warp == kMmaWarp) tmem_free(tmem, 512);
    if (threadIdx.x == 0 && sh.gave_up) atomicExch(a.c.dev_error, (int)HVD_DEV_WAIT_EXPIRED);
}

// Joins the pieces of the items that several CTAs shared (CTA x of the grid: the item that CTA x began and left
// unfinished), and gives the rows that see nothing for want of a token their zeros.
template <typename E, int DP>
__global__ void __launch_bounds__(kFinishThreads) attn_finish_kernel(const AttnArgs a, const Work ws, const int n_cta, const int tile_tok) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_trigger();
    pdl_wait();
    constexpr int kPerLane = DP / 32;
    const int part = blockIdx.y * (kFinishThreads / 32) + warp, n_part = gridDim.y * (kFinishThreads / 32);
    if (blockIdx.x < (unsigned)n_cta) {
        const SplitDesc d = ws.desc[blockIdx.x];
        if (d.valid) {
            const Chunk c = load_chunk(a.c, d.b);
            const int rows = d.n_tok * a.group, n = d.c_last - (int)blockIdx.x + 1;
            for (int r = part; r < rows; r += n_part) {
                // row r of the item: token r / group; its place among the partial sums
                const int t = r / a.group, grp = r - t * a.group;
                const int place = t < tile_tok ? r : 128 + r - tile_tok * a.group;
                auto slot = [&](int i) { return (int64_t)(2 * ((int)blockIdx.x + i) + (i == 0 ? 1 : 0)) * 256 + place; };
                float m = -INFINITY;
                for (int i = lane; i < n; i += 32) m = fmaxf(m, ws.ml[slot(i)].x);
#pragma unroll
                for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
                float acc[kPerLane] = {}, l = 0.0f;
                for (int i0 = 0; i0 < n; i0 += 32) {
                    float f = 0.0f, li = 0.0f;
                    if (i0 + lane < n) {
                        const float2 ml = ws.ml[slot(i0 + lane)];
                        f = ml.x == -INFINITY ? 0.0f : exp2f(ml.x - m);
                        li = ml.y * f;
                    }
                    const int e = min(32, n - i0);
                    for (int i = 0; i < e; ++i) {
                        const float fi = __shfl_sync(0xffffffffu, f, i);
                        l += __shfl_sync(0xffffffffu, li, i);
                        const float* o = ws.o + slot(i0 + i) * DP + lane * kPerLane;
                        if (lane * kPerLane < a.head_dim) {
                            if (kPerLane == 4) {
                                const float4 v = *reinterpret_cast<const float4*>(o);
                                acc[0] += v.x * fi; acc[1] += v.y * fi; acc[2 % kPerLane] += v.z * fi; acc[3 % kPerLane] += v.w * fi;
                            } else {
                                const float2 v = *reinterpret_cast<const float2*>(o);
                                acc[0] += v.x * fi; acc[1] += v.y * fi;
                            }
                        }
                    }
                }
                const int64_t row = c.r0 + d.tok0 + t;
                const int head = d.h * a.group + grp;
                const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                if (lane * kPerLane < a.head_dim) {
                    uint32_t* out = reinterpret_cast<uint32_t*>(reinterpret_cast<E*>(a.out.p) + row * a.out.row_stride + (int64_t)head * a.out.head_stride + lane * kPerLane);
#pragma unroll
                    for (int k = 0; k < kPerLane / 2; ++k) out[k] = pack2<E>(acc[2 * k] * inv, acc[2 * k + 1] * inv);
                }
                if (a.lse && lane == 0) a.lse[row * a.n_q_heads + head] = l > 0.0f ? (m + log2f(l)) * kLn2 : -INFINITY;
            }
        }
    }
    // requests: status, rows that are no new token
    const int who = blockIdx.y * gridDim.x + blockIdx.x, n_who = gridDim.x * gridDim.y;
    for (int b = who * (kFinishThreads / 32) + warp; b < a.c.B; b += n_who * (kFinishThreads / 32)) {
        const Chunk c = load_chunk(a.c, b);
        if (a.status && lane == 0) a.status[b] = c.bad ? HVD_REQ_BAD_LEN : HVD_REQ_OK;
        for (int i = c.n_new; i < c.rows; ++i)
            for (int h = 0; h < a.n_q_heads; ++h) {
                E* out = reinterpret_cast<E*>(a.out.p) + (c.r0 + i) * a.out.row_stride + (int64_t)h * a.out.head_stride;
                if (8 * lane < a.head_dim) *reinterpret_cast<uint4*>(out + 8 * lane) = make_uint4(0u, 0u, 0u, 0u);
                if (a.lse && lane == 0) a.lse[(c.r0 + i) * a.n_q_heads + h] = -INFINITY;
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
        e = launch_kernel(pdl, attn_tile_kernel<E, DP>, dim3(n_cta), dim3(kThreads), kSmemBytes<DP>, stream, a, ws, box_keys, box_tok, mq, mk, mv);
        if (e != cudaSuccess) return cuda_fail(ctx, e, "attn_tile_kernel");
    }
    e = launch_kernel(pdl, attn_finish_kernel<E, DP>, dim3(n_cta, 8), dim3(kFinishThreads), 0, stream, a, ws, c.total_rows > 0 ? n_cta : 0, tile_tok);
    return e == cudaSuccess ? HVD_OK : cuda_fail(ctx, e, "attn_finish_kernel");
}

}  // namespace

size_t attn_workspace_bytes(int num_sms, int head_dim) {
    const int dp = head_dim > 64 ? 128 : 64;
    return (size_t)num_sms * (2 * 256 * (dp * sizeof(float) + sizeof(float2)) + sizeof(SplitDesc));
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
