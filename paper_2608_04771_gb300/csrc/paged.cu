// paged.cu -- decode attention of one new token over a paged cache (the per-token attention of
// Sec. 1, 2.2 and 4.2, rows in pages), and the accumulation of the rows' attention weights (Eq. 2's
// sums, taken token by token as the tokens are decoded).
//
// x_gj = scale q_g . k_j over the rows j in sight, an online softmax (running max and sum in float32, to base 2),
// out_g = sum_j p_gj v_j.  A row's 4 d bytes (bf16) serve 4 G d operations, G at most 16: the bytes of K and V are the
// bound, and everything here is there to keep them coming.
//
// paged_decode: persistent, one CTA per SM of eight computing warps (float32: twelve), one that copies and, for
// calls with weights, three more.  The blocks of 16 rows (bf16: 8 KB of K and V at d = 128) of all units are shared out
// to the CTAs:
//   units that fit the grid are cut into equal pieces, one piece per CTA, so that every CTA joins and publishes once;
//   more units: the blocks are laid end to end and every CTA takes an equal range, cut across units;
//   many short units would spend their time joining: each goes whole to one stream of its CTA.
// Inside a CTA's range the blocks go round the streams.  A stream is a ring of stages, filled by TMA copies (bf16) or
// bulk copies (float32), and the warps that read it: one, or several that take a part of the query heads each (float32
// of more than two heads: F32Wide).  Lane s of the copying warp feeds stream s: it walks the same units, looks the pages
// up (a block never straddles two; the next block's entry loads while this one's copies go out) and waits for free
// stages, so that the computing warps spend nothing on either: with the copies and the look-ups in the computing warps,
// as the contiguous decode has its copies, the 7B-class stack of 16K rows took 1308 us, so 1020 (7.05 TB/s, 1.04 of the
// copy rate).  What a warp does with a block is decode_block.cuh's.  At the end of a piece the streams join their (max,
// sum, output) through shared memory; a unit cut between CTAs leaves one partial per CTA, which the last CTA to
// finish (atomic ticket, no waiting) joins in the order of the pieces: the same inputs give the same bits.
//
// A window leaves the blocks that hold rows in sight: the first `head` ones and those `gap` further on
// are the unit's list, in which everything above counts; a block that a border crosses masks its rows.
//
// A call with weights has the kernel leave its logits (4 G bytes a row, against 4 d bytes of K and V in
// bf16) in the workspace: a second product with K would read half of the cache again.  The three warps turn those of a
// unit that the CTA sees through into weights while they are still in L2 and the next unit streams; with few rows in
// sight the CTA that joins a unit's pieces does it; paged_weights does the rest.  (7B-class stack of 4K rows: 287 us
// without weights; 370 with all of them in paged_weights, 342 so, of which some 40 go with the logits' stores.)
#include <algorithm>

#include "decode_block.cuh"
#include "internal.h"

namespace reco {

constexpr int kRingBytes = 24 * 8192;  // ring of a CTA, all streams
constexpr int kWeightWarps = 3;        // they cost no registers: 9 warps or 12, an SM's quarter holds three of 168
// Blocks per working CTA at least (fewer CTAs rather than less): two units of 512 rows 10.9 us, with 16 12.1, with 2
// 10.9; 8 units of 1000 rows 11.5, 13.1 and 11.9 (with the plan of before kWarpUnits: now 10.1 and 11.1).
constexpr int kMinBlocks = 8;
// Up to this many units, if they fit the grid, every warp plans by itself, without barriers (a Tiny layer 10.7 -> 10.1).
constexpr int kWarpUnits = 128;
// A cut this near to a unit's end moves there.  From an eighth of a CTA's range: window of 4000 over 32K rows 185 ->
// 165 us; 4, 16 and 32 blocks within 1% but for 448 units of 300 to 2000 rows (32: 47 -> 50).
constexpr int kSnapBlocks = 8;
// More units than CTAs, none longer than this, go whole to a stream: 1792 units of 60 to 200 rows 33.8 us, cut 51; the
// same of 200 to 400 rows 73.7 whole, 64.7 cut.
constexpr int kWholeBlocks = 16;
// Calls with no more rows in sight than this, whose units fit the grid, make their weights where pieces join: 32 units
// of 2000 rows 16.9 us, with a launch for them 19.1; 4 units of 4000 rows 19.3 and 18.5.
constexpr int kInlineRows = 2560;

PagedDecodeWs paged_decode_ws_layout(const reco_paged_kv &kv, bool weights, void *base)
{
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char *r = base ? (char *)base + off : nullptr;
        off += align256(bytes);
        return r;
    };
    const size_t heads = (size_t)kv.n_layers * kv.B * kv.H_q;
    const size_t G = kv.H_q / kv.H_kv;
    PagedDecodeWs ws;
    // what has to be zero on entry, in a place that no descriptor moves: whatever call used the workspace last left it zero
    ws.counters = (int32_t *)take((2 + kPagedMaxGrid) * 4);
    ws.cuts = (int32_t *)take((2 + kPagedMaxGrid) * 4);
    static_assert(2 * align256((2 + kPagedMaxGrid) * 4) <= kPagedZeroBytes, "counters and cuts");
    off = kPagedZeroBytes;
    ws.part_ml = (float *)take(2 * kPagedMaxGrid * G * 2 * 4);
    ws.part_o = (float *)take(2 * kPagedMaxGrid * G * kv.d * 4);
    ws.lse2 = weights ? (float *)take(heads * 4) : nullptr;
    ws.logits = weights ? (float *)take(heads * paged_cap(kv) * 4) : nullptr;
    ws.bytes = off;
    return ws;
}

struct PagedArgs {
    void *K, *V;
    const int32_t *table;
    const void *q, *k_new, *v_new;
    int32_t *lens;
    void *out;
    float *lse;      // or nullptr
    float *lse2;     // with logits: log2 of the softmax sums of the units that are cut between CTAs
    float *logits;   // or nullptr: [unit][cap / 16][G][16] base-2 logits of the rows seen (logit_place)
    float *weights;  // with logits: the running sums; an appended row's starts at zero
    int32_t *counters;  // [0] warps that stopped and units in error, [1] CTAs done, [2 + c] ticket of the unit that CTA c starts
    float *part_ml, *part_o;
    int32_t *cuts;  // units cut between CTAs: [0] counted, [1] their number once the launch is done, [2 ...] the units
    int units, B, Hq, Hkv, G, cap, n_pages, max_pages, shift, append, out_bf16, window, sinks;
    int inline_weights;  // no paged_weights follows: pieces become weights where they join
    float c2;  // scale * log2(e)
    unsigned *err;
};

// Rows [h0, h1) of a unit are out of sight.  Its list of blocks: the first `head` ones, then those `gap`
// further on.
struct Sight {
    int head, gap, h0, h1;
};
template <int KB> __device__ __forceinline__ Sight sight_of(const PagedArgs &a, int le)
{
    if (a.window == 0 || le <= a.window) return Sight{0, 0, 0, 0};
    const int h1 = le - a.window, h0 = min(a.sinks, h1);
    const int head = (h0 + KB - 1) / KB;
    return Sight{head, max(0, h1 / KB - head), h0, h1};
}

// Rows of a unit with the appended one, 0 for a unit in error.
__device__ __forceinline__ int rows_of(const PagedArgs &a, int L) { return unit_ok(L, a.cap, a.append) ? L + a.append : 0; }
template <int KB> __device__ __forceinline__ int blocks_of(const PagedArgs &a, int le)
{
    return (le + KB - 1) / KB - sight_of<KB>(a, le).gap;
}

// A unit's table, and its row in page 0 of its layer.
struct Pages {
    const int32_t *table;
    int base;
};
__device__ __forceinline__ Pages pages_of(const PagedArgs &a, int u)
{
    const int lb = u / a.Hkv, layer = lb / a.B;
    return Pages{a.table + (long)(lb - layer * a.B) * a.max_pages, (layer * a.n_pages * a.Hkv + (u - lb * a.Hkv)) << a.shift};
}
__device__ __forceinline__ int page_entry(const PagedArgs &a, const Pages &p, int k) { return __ldg(p.table + (k >> a.shift)); }
// Pool row of row k, -1 where its table entry e names no page of the pool.
__device__ __forceinline__ int paged_row(const PagedArgs &a, const Pages &p, int k, int e)
{
    if ((unsigned)e >= (unsigned)a.n_pages) return -1;
    return p.base + ((e * a.Hkv) << a.shift) + (k & ((1 << a.shift) - 1));
}

// The walk of a CTA over its range of blocks, a piece (its part of one unit) at a time.
struct Piece {
    int u, le, nb, lo, hi;  // unit, its rows, its blocks, and those of this piece: [lo, hi)
    int at;                 // lo counted from the start of the CTA's range
    Sight sg;
};
struct Walk {
    int u, b, ub, nb, le, begin, end;
};
template <int KB> __device__ __forceinline__ bool next_piece(const PagedArgs &a, Walk &w, Piece &p)
{
    while (w.b < w.end) {
        if (w.b >= w.ub + w.nb) {
            w.ub += w.nb;
            ++w.u;
            w.le = rows_of(a, a.lens[w.u]);
            w.nb = blocks_of<KB>(a, w.le);
            continue;
        }
        p.u = w.u;
        p.le = w.le;
        p.nb = w.nb;
        p.lo = w.b - w.ub;
        p.hi = min(w.end - w.ub, w.nb);
        p.at = w.b - w.begin;
        p.sg = sight_of<KB>(a, w.le);
        w.b = w.ub + p.hi;
        return true;
    }
    return false;
}

// Whole units: those of a CTA's units [w.u, w.end) that fall to stream s, every NS-th one (w.u is moved there
// before the first call).
template <int KB, int NS> __device__ __forceinline__ bool next_whole(const PagedArgs &a, Walk &w, Piece &p)
{
    while (w.u < w.end) {
        p.u = w.u;
        w.u += NS;
        p.le = rows_of(a, a.lens[p.u]);
        if (p.le == 0) continue;
        p.nb = p.hi = blocks_of<KB>(a, p.le);
        p.lo = p.at = 0;
        p.sg = sight_of<KB>(a, p.le);
        return true;
    }
    return false;
}

// Barrier of the warps of a stream (one barrier per stream).
template <int THREADS> __device__ __forceinline__ void bar_stream(int id) { asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(THREADS) : "memory"); }
// Barrier of the computing warps.
template <int THREADS> __device__ __forceinline__ void bar_compute() { asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory"); }

__device__ __forceinline__ void put_lse(const PagedArgs &a, size_t row, float l2)
{
    if (a.lse) a.lse[row] = l2 * kLn2;
}

__device__ __forceinline__ void store_out4(const PagedArgs &a, size_t i, float4 v)
{
    if (a.out_bf16) {
        uint2 w;
        w.x = pack_bf16(v.x, v.y);
        w.y = pack_bf16(v.z, v.w);
        *reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(a.out) + i) = w;
    } else {
        *reinterpret_cast<float4 *>(reinterpret_cast<float *>(a.out) + i) = v;
    }
}

// weights[j] += (1/G) sum_g 2^(logit_g[j] - z_g) for the rows in sight of a unit of n rows, by `step` threads of
// which this is number `from`, the loads of GB heads in flight.  A thread takes four rows of a block at a time, as
// they lie among the logits: rows 2 c, 2 c + 1, 2 c + 8 and 2 c + 9 (logit_place).
template <int GB>
__device__ __forceinline__ void add_weights(const float *logits, const float *z, float *weights, int G, int n, int window,
                                            int sinks, int from, int step)
{
    const int start = window > 0 && n > window ? n - window : 0, head = min(sinks, start);
    const float inv = 1.f / (float)G;
    auto seen = [&](int j) { return j < n && (j < head || j >= start); };
    for (int i = from; 16 * (i >> 2) < n; i += step) {
        const int k = 16 * (i >> 2), j0 = k + 2 * (i & 3), j1 = j0 + 8;
        if (k >= head && k + 16 <= start) continue;  // a block out of sight
        const float *src = logits + (size_t)k * G + 4 * (i & 3);
        float2 *w0 = reinterpret_cast<float2 *>(weights + j0), *w1 = reinterpret_cast<float2 *>(weights + j1);
        const float2 a = *w0, b = *w1;
        float4 p = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int g0 = 0; g0 < G; g0 += GB) {
            float4 x[GB];
#pragma unroll
            for (int h = 0; h < GB; ++h)
                x[h] = g0 + h < G ? __ldcg(reinterpret_cast<const float4 *>(src + 16 * (g0 + h))) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int h = 0; h < GB; ++h) {
                const float zh = g0 + h < G ? z[g0 + h] : INFINITY;  // (2^-inf is 0)
                if (zh == -INFINITY) continue;
                p.x += fast_exp2(x[h].x - zh);
                p.y += fast_exp2(x[h].y - zh);
                p.z += fast_exp2(x[h].z - zh);
                p.w += fast_exp2(x[h].w - zh);
            }
        }
        const float2 s0 = make_float2(fmaf(p.x, inv, a.x), fmaf(p.y, inv, a.y));
        const float2 s1 = make_float2(fmaf(p.z, inv, b.x), fmaf(p.w, inv, b.y));
        if (k + 16 <= n && (k + 16 <= head || k >= start)) {
            *w0 = s0;
            *w1 = s1;
        } else {
            if (seen(j0)) w0->x = s0.x;
            if (seen(j0 + 1)) w0->y = s0.y;
            if (seen(j1)) w1->x = s1.x;
            if (seen(j1 + 1)) w1->y = s1.y;
        }
    }
}

// Ring, then [warp][head][D] floats: the warps' outputs as they join (and, until then, each warp's scratch).
template <class Block, int NW> constexpr int paged_smem()
{
    return 1024 + kRingBytes + NW * (Block::GM < 8 ? Block::GM : 8) * Block::D * 4;
}

// NW computing warps in NS = NW / HS streams of HS warps: each takes a part of a unit's query heads.
template <class Block, int HS, int NW>
__global__ void __launch_bounds__(32 * (NW + 1 + kWeightWarps), 1)
    paged_decode(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, PagedArgs a)
{
    constexpr int D = Block::D, KB = Block::KB, GM = Block::GM;
    constexpr int STAGE = 2 * KB * Block::ROW, STAGES = kRingBytes / STAGE;  // a stage holds a block of K and V rows
    constexpr int NS = NW / HS, S = STAGES / NS;
    constexpr int JH = GM < 8 ? GM : 8;  // heads that join at a time
    constexpr int NC = 32 * NW, NT = NC + 32 * (1 + kWeightWarps), CPR = Block::ROW / 16;
    static_assert(NS * HS == NW && S * NS == STAGES, "equal streams");
    static_assert(GM % JH == 0 && (GM == JH || HS == 1), "heads join in whole tiles");
    static_assert(Block::SCRATCH <= JH * D - 16, "a warp's scratch lies in its part of the join buffer");
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[STAGES], empty[STAGES];
    __shared__ int sm_row[STAGES];  // pool row of a stage's block, -1: none
    // calls with weights: units that are done, for the weight warps (log2 of the sums; unit and rows, -1: no more)
    __shared__ __align__(8) uint64_t job_full[2], job_empty[2];
    __shared__ float sm_lse[2][16];
    __shared__ int2 sm_job[2];
    __shared__ float2 sm_ml[NW][GM];      // joins: the warps' (max, sum), a sum of -1 for a piece in error
    __shared__ int sm_scan[4][NT / 32];
    __shared__ int sm_cut[2][4];  // unit, its first block (or CTA), blocks and rows, at the start and the end of the range
    __shared__ int sm_flags, sm_old;
    const uint32_t raw0 = smem_addr(smem_raw), ring0 = (raw0 + 1023u) & ~1023u;
    float *join = reinterpret_cast<float *>(smem_raw + (ring0 - raw0) + kRingBytes);
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int P = a.units, G = a.G, GS = (G + HS - 1) / HS;
    if (Block::TENSOR_MAPS && tid == 0) {
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
    }
    if (tid < STAGES) {
        mbar_init(smem_addr(&full[tid]), 1);
        mbar_init(smem_addr(&empty[tid]), HS);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 0) {
        sm_flags = 0;
        for (int k = 0; k < 2; ++k) {
            mbar_init(smem_addr(&job_full[k]), 1);
            mbar_init(smem_addr(&job_empty[k]), kWeightWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    wait_prior_grid();  // lens, the table, q and the new rows may come from the previous kernels
    auto look = [&](int L) {
        if (blockIdx.x == 0 && !unit_ok(L, a.cap, a.append))
            raise_error(a.err, (a.append && L == a.cap) ? ERR_ROOM : ERR_LEN);
        return rows_of(a, L);
    };
    // Few units: every warp plans by itself, up to kWarpUnits / 32 of them in a row per lane
    const bool by_warp = P <= kWarpUnits && P <= (int)gridDim.x;
    constexpr int UL = kWarpUnits / 32;
    const int per_lane = (P + 31) / 32;
    int le_w[UL];
    if (by_warp) {
#pragma unroll
        for (int i = 0; i < UL; ++i) {
            const int u = lane * per_lane + i;
            le_w[i] = i < per_lane && u < P ? __ldcg(a.lens + u) : 0;
        }
    }
    __syncthreads();  // the barriers are ready

    // ---- plan, the same in every CTA
    const int c = blockIdx.x, grid = gridDim.x;
    int NB = 0, max_nb = 0, n_ne = 0, c1 = 0, pieces = 1;  // c1, pieces: split: the CTA after the first piece's, the pieces
    bool split = true, whole = false;
    int quot = 0, rest = 0, T = 0;
    Walk start;
    start.begin = start.end = start.u = 0;
    // Units that fit the grid are cut into equal pieces of at most `per` blocks, a CTA each, so that a CTA joins
    // and publishes once.  `per` is the longest unit's share when it is cut as often as its part of all blocks allows,
    // or once, twice or three times less, whichever leaves no more pieces than CTAs, and failing those one that
    // cannot leave more.
    auto share = [&](int j) {
        const int target = max(n_ne, min(grid, NB / kMinBlocks));
        const int j0 = max(1, (int)((float)max_nb * (float)target / (float)NB));
        const int div = max(1, j0 - j), room = max(1, grid - n_ne);
        return j < 4 ? (max_nb + div - 1) / div : (NB + room - 1) / room;
    };
    auto take = [&](int u, int nb, int le, int first, int per) {  // this CTA's piece of unit u, whose first CTA is `first`
        start.u = u;
        start.ub = 0;
        start.nb = nb;
        start.le = le;
        c1 = first + 1;
        pieces = (nb + per - 1) / per;
        const int s = c - first, pq = nb / pieces, pr = nb - pq * pieces;
        start.begin = pq * s + min(s, pr);
        start.end = pq * (s + 1) + min(s + 1, pr);
    };
    if (by_warp) {
        int my_b = 0, my_max = 0, my_ne = 0, nb[UL];
#pragma unroll
        for (int i = 0; i < UL; ++i) {
            const bool mine = i < per_lane && lane * per_lane + i < P;
            le_w[i] = mine ? (wid == 0 ? look(le_w[i]) : rows_of(a, le_w[i])) : 0;
            nb[i] = blocks_of<KB>(a, le_w[i]);
            my_b += nb[i];
            my_max = max(my_max, nb[i]);
            my_ne += nb[i] > 0;
        }
        NB = __reduce_add_sync(0xffffffffu, (unsigned)my_b);
        max_nb = __reduce_max_sync(0xffffffffu, (unsigned)my_max);
        n_ne = __reduce_add_sync(0xffffffffu, (unsigned)my_ne);
        for (int j = 0; NB > 0 && j < 5; ++j) {
            const int per = share(j);
            int my_k = 0;
#pragma unroll
            for (int i = 0; i < UL; ++i) my_k += (nb[i] + per - 1) / per;
            int at = my_k;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, at, o);
                if (lane >= o) at += v;
            }
            const int total = __shfl_sync(0xffffffffu, at, 31);
            at -= my_k;
            if (total > grid) continue;
            int u = 0, unb = 0, le = 0;
            const bool mine = c >= at && c < at + my_k;
            if (mine) {
                bool found = false;
#pragma unroll
                for (int i = 0; i < UL; ++i) {
                    const int k = (nb[i] + per - 1) / per;
                    if (!found && c < at + k) {
                        found = true;
                        u = lane * per_lane + i;
                        unb = nb[i];
                        le = le_w[i];
                    }
                    at += found ? 0 : k;
                }
            }
            const unsigned who = __ballot_sync(0xffffffffu, mine);
            if (who != 0u) {
                const int src = __ffs(who) - 1;
                u = __shfl_sync(0xffffffffu, u, src);
                unb = __shfl_sync(0xffffffffu, unb, src);
                le = __shfl_sync(0xffffffffu, le, src);
                at = __shfl_sync(0xffffffffu, at, src);
                take(u, unb, le, at, per);
            }
            break;
        }
    } else {
        const int seg = (P + NT - 1) / NT, u_lo = min(P, tid * seg), u_hi = min(P, u_lo + seg);
        int le0 = 0;  // with a unit per thread at most: its rows; with more, the rows of all lie in the (still idle) ring
        int *sm_le = reinterpret_cast<int *>(smem_raw + (ring0 - raw0));
        const bool staged = seg > 1 && P <= kRingBytes / 4;
        if (seg == 1) {
            if (tid < P) le0 = look(__ldcg(a.lens + tid));
        } else {
            for (int u0 = tid; u0 < P; u0 += 8 * NT) {  // eight loads in flight
                int L[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) L[k] = u0 + k * NT < P ? __ldcg(a.lens + u0 + k * NT) : 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int u = u0 + k * NT;
                    if (u < P) {
                        const int le = look(L[k]);
                        if (staged) sm_le[u] = le;
                    }
                }
            }
            __syncthreads();
        }
        // rows of a unit of this thread's share
        auto le_of = [&](int u) { return seg == 1 ? le0 : (staged ? sm_le[u] : rows_of(a, __ldcg(a.lens + u))); };
        int my_b = 0, my_max = 0, my_ne = 0;
        for (int u = u_lo; u < u_hi; ++u) {
            const int nb = blocks_of<KB>(a, le_of(u));
            my_b += nb;
            my_max = max(my_max, nb);
            my_ne += nb > 0;
        }
        my_max = __reduce_max_sync(0xffffffffu, (unsigned)my_max);
        my_ne = __reduce_add_sync(0xffffffffu, (unsigned)my_ne);
        const int warp_b = __reduce_add_sync(0xffffffffu, (unsigned)my_b);
        if (lane == 0) {
            sm_scan[0][wid] = warp_b;
            sm_scan[1][wid] = my_max;
            sm_scan[2][wid] = my_ne;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NT / 32; ++w) {
            NB += sm_scan[0][w];
            max_nb = max(max_nb, sm_scan[1][w]);
            n_ne += sm_scan[2][w];
        }
        // exclusive prefix of x over the CTA's threads, and its sum
        auto scan = [&](int x, int &total) {
            int incl = x;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            if (lane == 31) sm_scan[3][wid] = incl;
            __syncthreads();
            int before = incl - x;
            total = 0;
#pragma unroll
            for (int w = 0; w < NT / 32; ++w) {
                const int v = sm_scan[3][w];
                before += w < wid ? v : 0;
                total += v;
            }
            return before;
        };
        // (64-bit products and divisions here cost a short call 0.5 us: equal parts are cut as quotient and rest)
        split = n_ne <= grid;
        whole = !split && max_nb <= kWholeBlocks;
        quot = NB / grid;  // (more units than CTAs: at least 1)
        rest = NB - quot * grid;
        T = whole ? 1 << 30 : min(kSnapBlocks, max(1, quot / 4));
        if (split && NB > 0) {
            int per = 0, total = 0, at = 0;
            for (int j = 0; j < 5; ++j) {
                per = share(j);
                int my_k = 0;
                for (int u = u_lo; u < u_hi; ++u) my_k += (blocks_of<KB>(a, le_of(u)) + per - 1) / per;
                if (j > 0) __syncthreads();  // the last scan has been read
                at = scan(my_k, total);
                if (total <= grid) {
                    if (c >= at && c < at + my_k) {
                        for (int u = u_lo; u < u_hi; ++u) {
                            const int le = le_of(u), nb = blocks_of<KB>(a, le), k = (nb + per - 1) / per;
                            if (c < at + k) {
                                sm_cut[0][0] = u;
                                sm_cut[0][1] = at;
                                sm_cut[0][2] = nb;
                                sm_cut[0][3] = le;
                                break;
                            }
                            at += k;
                        }
                    }
                    break;
                }
            }
            __syncthreads();
            if (c < total) take(sm_cut[0][0], sm_cut[0][2], sm_cut[0][3], sm_cut[0][1], per);
        } else if (NB > 0) {
            // More units than CTAs: equal ranges of the blocks laid end to end
            int total;
            const int before = scan(my_b, total);
            auto ideal = [&](int k) { return quot * k + min(k, rest); };
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int t = ideal(c + k);
                if (t >= before && t < before + my_b) {  // in one of this thread's units
                    int ub = before, u = u_lo, nb = 0, le = 0;
                    for (; u < u_hi; ++u) {
                        le = le_of(u);
                        nb = blocks_of<KB>(a, le);
                        if (t < ub + nb) break;
                        ub += nb;
                    }
                    sm_cut[k][0] = u;
                    sm_cut[k][1] = ub;
                    sm_cut[k][2] = nb;
                    sm_cut[k][3] = le;
                }
            }
            __syncthreads();
            auto cut = [&](int k) {
                const int t = ideal(c + k), ub = sm_cut[k][1], ue = ub + sm_cut[k][2];
                if (t >= NB) return NB;
                if (min(t - ub, ue - t) >= T) return t;
                return t - ub <= ue - t ? ub : ue;
            };
            start.begin = cut(0);
            start.end = cut(1);
            start.u = sm_cut[0][0];
            if (whole) {  // the units [start.u, start.end)
                start.u += start.begin == sm_cut[0][1] ? 0 : 1;
                start.end = ideal(c + 1) >= NB ? P : sm_cut[1][0] + (start.end == sm_cut[1][1] ? 0 : 1);
            }
            start.ub = sm_cut[0][1];
            start.nb = sm_cut[0][2];
            start.le = sm_cut[0][3];
        }
    }
    start.b = start.begin;

    // the first block of a piece that falls to stream s (block x of the CTA's range falls to stream x % NS)
    auto first_of = [](int s, int at) { return (int)((unsigned)(s + NS - at % NS) % (unsigned)NS); };

    if (wid == NW) {
        // ---- copies: lane s feeds stream s
        if (lane < NS) {
            constexpr unsigned MASK = (1u << NS) - 1u;
            const uint64_t policy = l2_evict_first_policy();  // K and V rows are read once
            Walk w = start;
            Piece p = {};
            Pages pg = {};
            int i = 0, e = 0;  // next block of the piece, and its table entry
            if (whole) w.u += lane;
            auto first_row = [&]() { return KB * (i + (i >= p.sg.head ? p.sg.gap : 0)); };
            auto begin_piece = [&]() {
                while (whole ? next_whole<KB, NS>(a, w, p) : next_piece<KB>(a, w, p)) {
                    i = whole ? 0 : p.lo + first_of(lane, p.at);
                    if (i >= p.hi) continue;
                    pg = pages_of(a, p.u);
                    e = page_entry(a, pg, first_row());
                    return true;
                }
                return false;
            };
            bool have = begin_piece();
            uint32_t issued = 0, slot = 0, par = 1;
            long long idle = 0;
            while (__any_sync(MASK, have)) {
                const int st = lane * S + (int)slot;
                const bool go = have && mbar_test(smem_addr(&empty[st]), par);
                if (go) {
                    const int k = first_row(), row = paged_row(a, pg, k, e);
                    const uint32_t bar = smem_addr(&full[st]), dst = ring0 + (uint32_t)st * STAGE;
                    sm_row[st] = row;
                    fence_async_shared();
                    if (row >= 0)
                        Block::load(dst, bar, &tmK, &tmV, a.K, a.V, (typename Block::RowIndex)row,
                                    min(KB, p.le - a.append - k), policy);
                    else
                        mbar_expect_tx(bar, 0);  // what the stage holds counts for nothing
                    ++issued;
                    if (++slot == (uint32_t)S) {
                        slot = 0;
                        par ^= 1u;
                    }
                    i += whole ? 1 : NS;
                    if (i >= p.hi)
                        have = begin_piece();
                    else
                        e = page_entry(a, pg, first_row());
                }
                if (__any_sync(MASK, go)) {
                    idle = 0;
                } else {
                    if (++idle > kSpinLimit / 4) {  // a warp stopped taking its blocks
                        raise_error(a.err, ERR_INTERNAL);
                        break;
                    }
                    __nanosleep(20);
                }
            }
            // no copy is left in flight when the CTA ends
            for (uint32_t j = issued > (uint32_t)S ? issued - S : 0; j < issued; ++j)
                mbar_wait_bounded(smem_addr(&full[lane * S + j % S]), (j / S) & 1u, kSpinLimit);
        }
        return;
    }

    if (wid > NW) {
        // ---- weights of units that the CTA sees through, while the computing warps go on with the next
        if (a.logits == nullptr || split || whole) return;
        for (int k = 0;; ++k) {
            const int slot = k & 1;
            if (!mbar_wait_bounded(smem_addr(&job_full[slot]), (k >> 1) & 1, kSpinLimit)) {
                if (lane == 0) raise_error(a.err, ERR_INTERNAL);
                return;
            }
            const int2 job = sm_job[slot];
            if (job.x < 0) return;
            const size_t at = (size_t)job.x * a.cap;
            add_weights<8>(a.logits + at * G, sm_lse[slot], a.weights + at, G, job.y, a.window, a.sinks,
                           tid - NC - 32, 32 * kWeightWarps);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&job_empty[slot]));
        }
    }

    // ---- computing warps: stream `st`, heads [hp * GS, hp * GS + nh)
    const int st = wid % NS, hp = wid / NS;
    const int nh = max(0, min(GS, G - hp * GS));
    Block blk(lane, join + wid * JH * D);
    auto head_row = [&](int u) { return (size_t)(u / a.Hkv) * a.Hq + (size_t)(u % a.Hkv) * G; };
    // units without rows: zeros, lse = -inf
    for (int u = n_ne < P ? c * NW + wid : P; u < P; u += grid * NW) {
        if (rows_of(a, a.lens[u]) > 0) continue;
        const size_t q0 = head_row(u);
        for (int x = lane; x < G * D / 4; x += 32) store_out4(a, q0 * D + 4 * x, make_float4(0.f, 0.f, 0.f, 0.f));
        if (lane < G) put_lse(a, q0 + lane, -INFINITY);
    }
    bool dead = false;
    uint32_t slot = 0, par = 0;
    Walk w = start;
    Piece p = {};
    if (whole) w.u += st;
    int q_of = -1;  // whole: the unit whose queries were loaded ahead
    auto load_q = [&](int u) { blk.load_q(a.q, (long)head_row(u) + hp * GS, nh); };
    auto begin_piece = [&]() {
        if (whole) {
            if (!next_whole<KB, NS>(a, w, p)) return false;
            if (q_of != p.u) load_q(p.u);
            blk.start();
            q_of = w.u < w.end ? w.u : -1;
            if (q_of >= 0) load_q(q_of);
            return true;
        }
        if (!next_piece<KB>(a, w, p)) return false;
        load_q(p.u);
        blk.start();
        return true;
    };
    bool have = begin_piece();
    // jobs given to the weight warps: the next one's place is free once the one before the last is done
    int jobs = 0;
    auto give = [&](int2 job) {
        sm_job[jobs & 1] = job;
        mbar_arrive(smem_addr(&job_full[jobs & 1]));
    };
    auto place_free = [&]() {
        if (!mbar_wait_bounded(smem_addr(&job_empty[jobs & 1]), ((jobs >> 1) & 1) ^ 1, kSpinLimit)) {
            raise_error(a.err, ERR_INTERNAL);
            atomicOr(&sm_flags, 1);
        }
    };
    auto list_cut = [&](int u) {  // for paged_weights
        const int at = atomicAdd(&a.cuts[0], 1);
        if ((unsigned)at < (unsigned)kPagedMaxGrid) a.cuts[2 + at] = u;
    };
    const bool hand_on = a.logits != nullptr && !split && !whole;
    while (have) {
        bool bad = false;
        const size_t q0 = head_row(p.u);
        const int Lapp = a.append && p.hi == p.nb ? p.le - 1 : -1;  // the new row, in its unit's last block
        float *lg = a.logits ? a.logits + (size_t)p.u * G * a.cap + 16 * hp * GS : nullptr;  // of the unit's row 0
        for (int i = whole ? 0 : p.lo + first_of(st, p.at); i < p.hi; i += whole ? 1 : NS) {
            const int at = st * S + (int)slot;
            const bool app = Lapp >= 0 && i == p.nb - 1;
            uint4 rows[Block::APP];  // this lane's chunks of the new rows, K's then V's
            if (app) {
#pragma unroll
                for (int x = 0; x < Block::APP; ++x) {
                    const int t = lane + 32 * x;
                    rows[x] = make_uint4(0, 0, 0, 0);
                    if (t < 2 * CPR)
                        rows[x] = reinterpret_cast<const uint4 *>(t < CPR ? a.k_new : a.v_new)[(long)p.u * CPR + t % CPR];
                }
            }
            if (!dead && !mbar_wait_bounded(smem_addr(&full[at]), par, kSpinLimit)) {  // a copy never landed
                dead = true;
                if (lane == 0) {
                    raise_error(a.err, ERR_INTERNAL);
                    atomicOr(&sm_flags, 1);
                }
            }
            if (!dead) {
                const int row = sm_row[at];
                const int kb = KB * (i + (i >= p.sg.head ? p.sg.gap : 0));
                const uint32_t Ks = ring0 + (uint32_t)at * STAGE, Vs = Ks + STAGE / 2;
                bad |= row < 0;
                // zero the V rows that are not seen (their weights are zero, but NaN times zero is not) and put
                // the new row, which is not in the cache yet, in place
                const bool border = kb < p.sg.h1 && kb + KB > p.sg.h0;
                if (border || kb + KB > p.le || app) {
                    for (int t = lane; t < KB * CPR; t += 32) {
                        const int k = kb + t / CPR;
                        if (k >= p.le || (k >= p.sg.h0 && k < p.sg.h1))
                            sts_u4(Vs + Block::chunk(t / CPR, t % CPR), make_uint4(0, 0, 0, 0));
                    }
                    if (app) {
#pragma unroll
                        for (int x = 0; x < Block::APP; ++x) {
                            const int t = lane + 32 * x;
                            if (t < 2 * CPR) sts_u4((t < CPR ? Ks : Vs) + Block::chunk(Lapp - kb, t % CPR), rows[x]);
                        }
                    }
                    fence_async_shared();  // these writes come before the copy that fills the stage next
                    __syncwarp();
                }
                blk.consume(Ks, Vs, kb, p.le, a.c2, p.sg.h0, p.sg.h1, lg ? lg + (size_t)kb * G : nullptr, nh);
                if (app && row >= 0 && hp == 0) {  // and into the cache
                    const long r = (long)row + (Lapp - kb);
#pragma unroll
                    for (int x = 0; x < Block::APP; ++x) {
                        const int t = lane + 32 * x;
                        if (t < 2 * CPR) reinterpret_cast<uint4 *>(t < CPR ? a.K : a.V)[r * CPR + t % CPR] = rows[x];
                    }
                    if (lane == 0 && a.weights) a.weights[(size_t)p.u * a.cap + Lapp] = 0.f;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&empty[at]));
            }
            if (++slot == (uint32_t)S) {
                slot = 0;
                par ^= 1u;
            }
        }
        blk.finish();
        if (bad && lane == 0) {
            raise_error(a.err, ERR_PAGE);
            atomicOr(&sm_flags, 2);
        }
        if (whole) {
            float *z = join + (st + 1) * JH * D - 16;  // log2 of the sums (the join buffer is not used otherwise)
            if (bad) {
                for (int x = lane; x < nh * D / 4; x += 32)
                    store_out4(a, (q0 + hp * GS) * D + 4 * x, make_float4(0.f, 0.f, 0.f, 0.f));
                if (lane < nh) put_lse(a, q0 + hp * GS + lane, -INFINITY);
            } else {
                blk.store(a.out, a.out_bf16 != 0, (long)q0 + hp * GS, nh);
                blk.each_lse(nh, [&](int q, float m, float l) {
                    const float l2 = sum_log2(m, l);
                    put_lse(a, q0 + hp * GS + q, l2);
                    if (a.logits) z[hp * GS + q] = l2;
                });
            }
            if (a.logits) {
                if constexpr (HS > 1) bar_stream<32 * HS>(2 + st);  // the warps of this stream have all their heads' sums
                else __syncwarp();
                const size_t at = (size_t)p.u * a.cap;
                if (!bad) add_weights<4>(a.logits + at * G, z, a.weights + at, G, p.le, a.window, a.sinks,
                                      hp * 32 + lane, 32 * HS);
                if constexpr (HS > 1) bar_stream<32 * HS>(2 + st);
                else __syncwarp();
            }
            have = begin_piece();
            continue;
        }

        // ---- join, eight heads at a time: one barrier after the warps' results are in shared memory, one after
        // they have been read
        const Piece d = p;  // done
        const bool all = d.lo == 0 && d.hi == d.nb;
        const int out_slot = 2 * c + (d.lo == 0 ? 1 : 0);
        blk.each_lse(nh, [&](int q, float m, float l) { sm_ml[wid][q] = make_float2(m, bad ? -1.f : l); });
#pragma unroll
        for (int tile = 0; tile < GM / JH; ++tile) {
            blk.store_tile(tile, join + wid * JH * D, nh - tile * JH);
            if (tile == GM / JH - 1) have = begin_piece();  // the next piece's queries load meanwhile
            if (tile == 0 && tid == 0 && hand_on && all) place_free();
            bar_compute<NC>();
            const int tile0 = tile * JH, heads = HS == 1 ? min(JH, G - tile0) : G;
            for (int x = tid; x < heads * D / 4; x += NC) {
                const int q = x / (D / 4), d4 = x % (D / 4), part = HS == 1 ? 0 : q / GS, ql = q - part * GS;
                float M = -INFINITY, Ls = 0.f;
                bool err = false;
                float2 ml[NS];
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    ml[s] = sm_ml[part * NS + s][tile0 + ql];
                    M = fmaxf(M, ml[s].x);
                    err |= ml[s].y < 0.f;
                }
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
                if (!err) {
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        const float f = part_factor(ml[s].x, M);
                        const float4 v = *reinterpret_cast<const float4 *>(join + ((part * NS + s) * JH + ql) * D + 4 * d4);
                        Ls += ml[s].y * f;
                        o.x += v.x * f;
                        o.y += v.y * f;
                        o.z += v.z * f;
                        o.w += v.w * f;
                    }
                }
                const int head = tile0 + q;
                if (all) {
                    const float inv = sum_inverse(Ls);
                    store_out4(a, (q0 + head) * D + 4 * d4, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
                    if (d4 == 0) {
                        const float l2 = sum_log2(M, Ls);
                        put_lse(a, q0 + head, l2);
                        sm_lse[jobs & 1][head] = l2;
                        if (a.lse2) a.lse2[q0 + head] = l2;
                    }
                } else {
                    *reinterpret_cast<float4 *>(a.part_o + ((size_t)out_slot * G + head) * D + 4 * d4) = o;
                    if (d4 == 0)
                        reinterpret_cast<float2 *>(a.part_ml)[(size_t)out_slot * G + head] = make_float2(M, err ? -1.f : Ls);
                }
            }
            bar_compute<NC>();
        }
        if (all) {
            if (a.logits && split && !a.inline_weights) {  // (nothing to hide it behind: the next launch has all CTAs)
                if (tid == 0) list_cut(d.u);
            } else if (a.logits && have) {
                if (tid == 0) give(make_int2(d.u, d.le));
                ++jobs;
            } else if (a.logits) {  // the CTA's last unit (in error: sums of -inf, nothing is added)
                const size_t at = (size_t)d.u * a.cap;
                add_weights<4>(a.logits + at * G, sm_lse[jobs & 1], a.weights + at, G, d.le, a.window, a.sinks, tid, NC);
            }
            continue;
        }

        // ---- a unit cut between CTAs: publish; the last one joins the pieces
        if (!split) {  // cuts inside [ub, ue) stay where they fall from ub + T to ue - T; piece 0 is the CTA's before the first
            const int ub = start.begin + d.at - d.lo, ue = ub + d.nb;
            auto first_at = [&](int b) {  // first CTA whose ideal start is >= b
                const int big = rest * (quot + 1);
                return b <= big ? (b + quot) / (quot + 1) : rest + (b - big + quot - 1) / quot;
            };
            c1 = first_at(ub + T);
            pieces = 1 + max(0, first_at(ue - T + 1) - c1);
        }
        // the unit's ticket is that of the CTA with its first piece, which starts no other unit that is cut
        int32_t *ticket = &a.counters[2 + c1 - 1];
        if (tid == 0) sm_old = atom_add_acq_rel(ticket, 1);
        bar_compute<NC>();
        if (sm_old == pieces - 1) {
            if (tid == 0) {
                *ticket = 0;  // every piece has counted: clear for the next launch
                if (a.logits && !a.inline_weights) list_cut(d.u);
            }
            for (int x = tid; x < G * D / 4; x += NC) {
                const int q = x / (D / 4), d4 = x % (D / 4);
                auto slot_of = [&](int s) { return (size_t)(2 * (c1 - 1 + s) + (s == 0 ? 1 : 0)) * G + q; };
                // four pieces at a time, their loads in flight together, with a running maximum
                float M = -INFINITY, Ls = 0.f;
                bool err = false;
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int s0 = 0; s0 < pieces; s0 += 4) {
                    float2 ml[4];
                    float4 v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const bool in = s0 + k < pieces;
                        const size_t at = slot_of(in ? s0 + k : s0);
                        ml[k] = __ldcg(reinterpret_cast<const float2 *>(a.part_ml) + at);
                        v[k] = __ldcg(reinterpret_cast<const float4 *>(a.part_o + at * D + 4 * d4));
                        if (!in) {
                            ml[k] = make_float2(-INFINITY, 0.f);
                            v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                        }
                    }
                    float Mn = M;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        Mn = fmaxf(Mn, ml[k].x);
                        err |= ml[k].y < 0.f;
                    }
                    const float base = Mn == -INFINITY ? 0.f : Mn, f0 = fast_exp2(M - base);
                    Ls *= f0;
                    o.x *= f0;
                    o.y *= f0;
                    o.z *= f0;
                    o.w *= f0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float f = fast_exp2(ml[k].x - base);
                        Ls += ml[k].y * f;
                        o.x += v[k].x * f;
                        o.y += v[k].y * f;
                        o.z += v[k].z * f;
                        o.w += v[k].w * f;
                    }
                    M = Mn;
                }
                if (err) {
                    Ls = 0.f;
                    o = make_float4(0.f, 0.f, 0.f, 0.f);
                }
                const float inv = sum_inverse(Ls);
                store_out4(a, (q0 + q) * D + 4 * d4, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
                if (d4 == 0) {
                    const float l2 = sum_log2(M, Ls);
                    put_lse(a, q0 + q, l2);
                    if (a.lse2) a.lse2[q0 + q] = l2;
                    if (a.inline_weights) sm_lse[0][q] = l2;
                }
            }
            if (a.inline_weights) {
                bar_compute<NC>();
                const size_t at = (size_t)d.u * a.cap;
                add_weights<4>(a.logits + at * G, sm_lse[0], a.weights + at, G, d.le, a.window, a.sinks, tid, NC);
            }
        }
    }

    if (tid == 0 && hand_on) {
        place_free();
        give(make_int2(-1, 0));
    }

    // ---- the last CTA to finish advances the lengths (every plan has been read by then) and leaves the
    // counters zero, as it found them
    bar_compute<NC>();
    if (tid == 0) {
        const unsigned f = (unsigned)sm_flags;
        const unsigned long long add = (1ull << 32) | (f & 1u ? 1ull : 0ull) | (f & 2u ? 1ull << 16 : 0ull);
        const unsigned long long old = atom_add_acq_rel_u64(reinterpret_cast<unsigned long long *>(a.counters), add);
        const unsigned seen = (unsigned)(old + add);
        sm_old = (int)(old >> 32) == (int)gridDim.x - 1 ? 1 | (seen & 0xffffu ? 2 : 0) | (seen >> 16 ? 4 : 0) : 0;
    }
    bar_compute<NC>();
    const int last = sm_old;
    if (last == 0) return;
    if (last & 2) {  // tickets of units whose pieces stopped early may still count
        for (int k = tid; k < kPagedMaxGrid; k += NC) a.counters[2 + k] = 0;
    } else if (a.append) {
#pragma unroll 4
        for (int u = tid; u < P; u += NC) {
            const int L = __ldcg(a.lens + u);
            bool ok = unit_ok(L, a.cap, a.append);
            if (ok && (last & 4)) {  // units whose table names no page for a row in sight keep their length
                const Sight sg = sight_of<KB>(a, L + 1);
                const Pages pg = pages_of(a, u);
                const int page = 1 << a.shift;
                for (int k = 0; k <= L; k += page)
                    if (k < KB * sg.head || k + page > KB * (sg.head + sg.gap)) ok &= paged_row(a, pg, k, page_entry(a, pg, k)) >= 0;
            }
            if (ok) a.lens[u] = L + 1;
        }
    }
    if (tid == 0) {
        *reinterpret_cast<unsigned long long *>(a.counters) = 0ull;
        if (a.logits) {
            a.cuts[1] = min(__ldcg(a.cuts), kPagedMaxGrid);
            a.cuts[0] = 0;
        }
    }
}

// The weights of the units that were cut between CTAs: their sums are known once all their pieces are.  The CTAs
// share the units out evenly, an equal part of each unit's rows per CTA.
constexpr int kWeightThreads = 256;

__global__ void __launch_bounds__(kWeightThreads) paged_weights(const float *__restrict__ logits,
                                                                const float *__restrict__ lse2,
                                                                const int32_t *__restrict__ lens,
                                                                const int32_t *__restrict__ cuts, int units, int G, int cap,
                                                                int window, int sinks, float *weights)
{
    __shared__ float sm_lse[16];
    wait_prior_grid();
    const int n_cut = cuts[1];
    if (n_cut <= 0) return;
    const int parts = max(1, (int)gridDim.x / n_cut);  // CTAs per unit
    for (int i = blockIdx.x; i < n_cut * parts; i += gridDim.x) {
        const int u = cuts[2 + i / parts];
        if ((unsigned)u >= (unsigned)units) continue;
        const int n = lens[u];
        __syncthreads();
        if (threadIdx.x < G) sm_lse[threadIdx.x] = lse2[(size_t)u * G + threadIdx.x];
        __syncthreads();
        bool any = false;
        for (int g = 0; g < G; ++g) any |= sm_lse[g] != -INFINITY;
        if (!any || n < 0 || n > cap) continue;  // in error
        const size_t at = (size_t)u * cap;
        add_weights<8>(logits + at * G, sm_lse, weights + at, G, n, window, sinks,
                    (i % parts) * kWeightThreads + threadIdx.x, parts * kWeightThreads);
    }
}

// ---------------------------------------------------------------- host side
typedef void (*PagedKernel)(CUtensorMap, CUtensorMap, PagedArgs);
struct PagedLaunch {
    PagedKernel fn;
    int smem, threads;
};
template <class Block, int HS, int NW> static PagedLaunch with()
{
    static_assert(paged_smem<Block, NW>() + 2048 <= 227 * 1024, "shared memory of a CTA (2 KB of it static)");
    return PagedLaunch{paged_decode<Block, HS, NW>, paged_smem<Block, NW>(), 32 * (NW + 1 + kWeightWarps)};
}
template <int D> static PagedLaunch paged_kernel(bool f32, int G)
{
    if (!f32) return G > 8 ? with<Bf16Block<D, 2>, 1, 8>() : with<Bf16Block<D, 1>, 1, 8>();
    // float32: two heads per warp, whose queries and sums leave registers for twelve warps (plain FMAs wait for each
    // other and for shared memory: 224 units of 1150 rows, 6 heads, eight warps of four heads 82 us, so 68, in blocks
    // of 16 rows 58; pairs of FMAs in one instruction 61)
    if (G > 12) return with<F32Wide<D, 4>, 4, 8>();
    if (G > 8) return with<F32Wide<D, 2>, 6, 12>();
    if (G > 6) return with<F32Wide<D, 2>, 4, 12>();
    if (G > 4) return with<F32Wide<D, 2>, 3, 12>();
    return G > 2 ? with<F32Wide<D, 2>, 2, 12>() : with<F32Wide<D, 2>, 1, 12>();
}

cudaError_t launch_paged_decode(const reco_paged_kv &kv, const void *q, const void *k_new, const void *v_new,
                                int32_t *lens, float scale, int window, int sinks, void *out, reco_dtype out_dtype,
                                float *lse, float *weights, const PagedDecodeWs &ws, unsigned *err, cudaStream_t s)
{
    const bool f32 = kv.dtype == RECO_F32;
    const int cap = paged_cap(kv), units = kv.n_layers * kv.B * kv.H_kv, G = kv.H_q / kv.H_kv;
    PagedArgs a = {};
    a.K = kv.k;
    a.V = kv.v;
    a.table = kv.table;
    a.q = q;
    a.k_new = k_new;
    a.v_new = v_new;
    a.lens = lens;
    a.out = out;
    a.lse = lse;
    a.lse2 = ws.lse2;
    a.logits = ws.logits;
    a.weights = weights;
    a.counters = ws.counters;
    a.part_ml = ws.part_ml;
    a.cuts = ws.cuts;
    a.part_o = ws.part_o;
    a.units = units;
    a.B = kv.B;
    a.Hq = kv.H_q;
    a.Hkv = kv.H_kv;
    a.G = G;
    a.cap = cap;
    a.n_pages = kv.n_pages;
    a.max_pages = kv.max_pages;
    a.shift = __builtin_ctz((unsigned)kv.page);
    a.append = k_new ? 1 : 0;
    a.out_bf16 = out_dtype == RECO_BF16 ? 1 : 0;
    a.window = window;
    a.sinks = sinks;
    a.c2 = scale * kLog2e;
    a.err = err;
    CUtensorMap mk = {}, mv = {};
    const unsigned long long rows = (unsigned long long)kv.n_layers * kv.n_pages * kv.H_kv * kv.page;
    if (!f32 && (!encode_bf16_2d(&mk, kv.k, rows, kv.d, 64, 16) || !encode_bf16_2d(&mv, kv.v, rows, kv.d, 64, 16)))
        return cudaErrorInvalidValue;
    // (units that fit the grid are cut one piece per CTA: no unit is left for the weight warps)
    const int most_seen = window > 0 ? (int)std::min<long long>(cap, (long long)window + sinks) : cap;
    a.inline_weights = weights && units <= std::min(device_sm_count(), kPagedMaxGrid) && most_seen <= kInlineRows ? 1 : 0;
    const PagedLaunch k = kv.d == 64 ? paged_kernel<64>(f32, G) : paged_kernel<128>(f32, G);
    cudaError_t e = allow_smem((const void *)k.fn, k.smem);
    if (e != cudaSuccess) return e;
    // no more CTAs than the cache can hold work for
    const long long most = (long long)units * ((cap + 15) / 16);
    const int grid = (int)std::min<long long>(std::min(device_sm_count(), kPagedMaxGrid), std::max<long long>(units, most / kMinBlocks));
    e = launch_pdl(k.fn, dim3(grid), dim3(k.threads), k.smem, s, mk, mv, a);
    if (e != cudaSuccess || (e = cudaGetLastError()) != cudaSuccess || !weights || a.inline_weights) return e;
    e = launch_pdl(paged_weights, dim3(4 * device_sm_count()), dim3(kWeightThreads), 0, s, (const float *)ws.logits,
                   (const float *)ws.lse2, (const int32_t *)lens, (const int32_t *)ws.cuts, units, G, cap, window, sinks,
                   weights);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace reco
