// prefix_tc.cu -- the prefix part of decode attention over shared prefixes (prefix.cu) for bf16 caches, on the tensor
// cores (tcgen05, TMEM): S = Q K^T and O += P V over tiles of 128 query rows and 128 keys, with an online softmax
// between them (running maximum and sum in float32, to base 2).
//
// R query rows of a group serve 4 R d operations per 4 d bytes of K and V: below some 285 rows the bytes are the bound,
// above it the tensor cores.  A product's 128 rows cost the same however many are there, so that few rows cost
// nothing more while the bytes are.
//
// One CTA per SM, persistent over its share of the key tiles (PrefixArgs::next), of warps
//   0      finds the pieces, a few ahead of the others, and copies, all by TMA: queries (a box of a group's sequences, or
//          one sequence's, into one of two places) and K tiles (a box per page and 64 columns, a lane each, into a ring);
//   2      copies V tiles the same way, into a ring of their own (a copy takes some 75 cycles to issue: pages of 16 rows are
//          32 copies a tile, as long as a tile's bytes take);
//   1, 3   issue the products of a stream each;
//   4..11  two softmax groups of four warps, one per stream, a query row per thread.
// The two streams: a row tile of more than 128 rows has a half in each, otherwise each takes half of the keys of every tile
// and they join at the end of the piece.  A stream goes by blocks of 64 keys, two of which have a place for their S in
// TMEM, so that the group works on one while the other's product runs.  S is overwritten by P in bf16, which the second
// product takes from there; O stays in TMEM, and is rescaled only when a row's probabilities against
// the maximum so far sum to more than 2^12 in a block.
//
// Measured, GB300, the whole call with its plan and its join.  28 layers, 8 sequences of 28 query and 4 key heads of 128 over
// 16001 shared rows and 1000 to 4000 of their own (1.9 GB of K and V): 313 us, 0.90 of the copy rate.  64 sequences of 40 and
// 8 heads over 100001 shared rows: 204 us, where the bytes once and the products (P in one part) are 67 us each; two row tiles
// read every K and V tile, one of 250 rows in some 2.4 us of a CTA and one of 70 in 1.2.  Memory is not what bounds them (46%
// of its rate): the tensor cores are active 49% of the time, a product of Q with 64 keys reads 6 KB of shared memory, 48
// cycles, for 32 cycles of theirs, and a block's softmax and two hand-overs are as long as the other stream's products.  One
// layer, 16 sequences of 28 and 4 heads, 4001 shared rows and 200 to 2000 of their own, 34 MB: 31.6 us, a chain of launches
// and look-ups more than of bytes.  (With one warp copying K and V in turn and another clearing V rows, 301, 169 and 28.4 us
// when they took 293, 170 and 27.4.)
//
// P enters its product in parts of bf16: with bf16 output in two, as the decode's (2^-17 of each probability; one part, 2^-8, added
// half as much again to the error of the output's own rounding: 2.3e-3 of the result against 1.7e-3), with float32 output
// in three (2^-26; two would lose 2^-17).  Sums take the probabilities as they were before.  Two parts are made
// once a block's sum has been looked at: as every pair of probabilities came, they cost 100 bytes of spills, or stores to
// TMEM in between (100001 rows below: 219 us either way, 209 so).
// The tensor cores cut sums off rather than round them: some 2^-26 of the output is lost with every addition to it, always
// towards zero (11 tiles cost 2.2e-6, 46 tiles 1.1e-5 of the result, against 64 bits).  With bf16 output that is nothing.
// With float32 output every block's product starts from zero, and four warps add the blocks up in registers: one stream
// with two places for its products, the other stream's softmax warps are those that add, and a row tile has 128 rows.  The
// 28 layers above take 525 us so, 2500 cycles a block: 1600 for the softmax of the one warp that a scheduler has, the rest
// waits and hand-overs (a third place for S: no gain; parts by cutting bits off instead of conversions: spills, 706 us).
//
// A barrier's phases alternate in one bit: a wait for phase k must not begin before phase k - 1 is over, nor be still
// to come when phase k + 1 is.  So every place is waited for by both issuing warps, every time; what a group waits for
// only now and then (pv_done) has a barrier for even and for odd blocks, which it cannot fall behind.
// Every wait is bounded; one that runs out raises the error word and the CTA's abort flag, which ends the others, and the
// join then takes no partial of the call (PrefixTotal::stopped).
#include <algorithm>

#include "decode_block.cuh"
#include "prefix.cuh"
#include "tc.cuh"

namespace reco {

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// (a, b) as two parts of bf16 and what is left, which a third holds but for 2^-26.
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t &hi, uint32_t &lo, float &ra, float &rb)
{
    hi = pack_bf16(a, b);
    ra = a - __uint_as_float(hi << 16);
    rb = b - __uint_as_float(hi & 0xffff0000u);
    lo = pack_bf16(ra, rb);
    ra -= __uint_as_float(lo << 16);
    rb -= __uint_as_float(lo & 0xffff0000u);
}

__device__ __forceinline__ void st_global_v8(float *p, const float *x)  // a whole sector
{
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]),
                 "f"(x[5]), "f"(x[6]), "f"(x[7])
                 : "memory");
}

constexpr long long kPolls = 1LL << 19;  // of a wait, each suspended for up to two microseconds

// The blocks of 64 keys of a piece that fall to stream s: block j begins `first` + `step` j columns from the start of the
// piece, of whose columns [lo, hi) count.
struct PrefixBlocks {
    int n, first, step, lo, hi;
    __device__ __forceinline__ PrefixBlocks(const PrefixPiece &x, bool pair, int s)
    {
        const int k0 = x.k0 + x.t0 * kPrefixTile, nt = x.t1 - x.t0;
        lo = max(0, x.lo - k0);
        hi = min(x.end - k0, nt * kPrefixTile);
        n = pair ? 2 * nt : nt;
        first = pair ? 0 : 64 * s;
        step = pair ? 64 : 128;
    }
};

template <int D, int PARTS> struct PrefixTc {
    static constexpr int HALVES = D / 64;
    static constexpr int BOX = 128 * 128;  // 128 rows of 64 bf16
    static constexpr int TILE = HALVES * BOX;
    static constexpr int Q_BYTES = 2 * TILE;
    static constexpr int STREAMS = PARTS == 3 ? 1 : 2;
    static constexpr int TILES = 5 * 128 / D, NK = (TILES + 1) / 2, NV = TILES - NK, NS = TILES;  // places for K tiles, then V tiles
    static constexpr int NP = 4;                  // pieces found ahead
    static constexpr int THREADS = 32 * 12;
    struct Small {  // behind the tiles
        uint64_t full[NS], empty[NS], q_full[2], q_empty[2], s_full[2][2], p_full[2][2], pv_done[2][2];
        uint64_t o_free, met[2], o_read[2];
        uint64_t piece_full[NP], piece_empty[NP];
        float2 ml[2][STREAMS == 1 ? 1 : 128];
        float al[2][STREAMS == 1 ? 128 : 1];
        PrefixPiece piece[NP];
        int bad[NP];  // a page that is none was met
        uint32_t tmem;
        int abort;
    };
    // (all of it dynamic: the tiles begin where the CTA's shared memory does, at a multiple of 1024)
    static constexpr int SMEM = Q_BYTES + NS * TILE + (int)sizeof(Small);
    static_assert(SMEM <= 227 * 1024, "shared memory of a CTA");
};

template <int D, int PARTS>
__global__ void __launch_bounds__(PrefixTc<D, PARTS>::THREADS, 1)
    prefix_tc(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
              const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmQ1, const __grid_constant__ PrefixArgs a)
{
    using C = PrefixTc<D, PARTS>;
    constexpr int NS = C::NS, NK = C::NK, NV = C::NV, NP = C::NP, BOX = C::BOX, TILE = C::TILE, HALVES = C::HALVES;
    constexpr bool ALONE = C::STREAMS == 1;
    constexpr uint32_t S_COL = 0, O_COL = 256;  // TMEM: S (then P) of the streams, 128 columns each, then their O;
    constexpr uint32_t P3_COL = 128, ML_COL = 192;  // one stream: third parts of P, 32 columns a place; maxima and sums of two pieces
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = smem_addr(smem_raw), Qs = base, ring = base + C::Q_BYTES;
    typename C::Small &sm = *reinterpret_cast<typename C::Small *>(smem_raw + C::Q_BYTES + NS * TILE);
    if (base & 1023u) {  // swizzled tiles need it
        wait_prior_grid();
        if (tid == 0) {
            raise_error(a.err, ERR_INTERNAL);
            a.total->stopped = 1;
        }
        return;
    }
    if (tid == 0) {
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
        prefetch_tensormap(&tmQ);
        prefetch_tensormap(&tmQ1);
        for (int i = 0; i < NS; ++i) {
            mbar_init(smem_addr(&sm.full[i]), 1);
            mbar_init(smem_addr(&sm.empty[i]), ALONE ? 1 : 2);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_addr(&sm.q_full[s]), 1);
            mbar_init(smem_addr(&sm.q_empty[s]), ALONE ? 1 : 2);
            mbar_init(smem_addr(&sm.met[s]), ALONE ? 4 : 8);
            mbar_init(smem_addr(&sm.o_read[s]), 4);
            for (int b = 0; b < 2; ++b) {
                mbar_init(smem_addr(&sm.s_full[s][b]), 1);
                mbar_init(smem_addr(&sm.p_full[s][b]), 4);
                mbar_init(smem_addr(&sm.pv_done[s][b]), 1);
            }
        }
        mbar_init(smem_addr(&sm.o_free), 8);
        for (int i = 0; i < C::NP; ++i) {
            mbar_init(smem_addr(&sm.piece_full[i]), 1);
            mbar_init(smem_addr(&sm.piece_empty[i]), ALONE ? 10 : 11);  // warps 1, 2 and 3, and from 4 on eight
        }
        sm.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_shared();
    }
    if (warp == 1) {
        tmem_alloc(smem_addr(&sm.tmem), 512);
        tmem_relinquish();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;
    wait_prior_grid();
    release_next_grid();  // (the join's CTAs start as this grid's end, and wait for all of it)
    // A wait for phase k of a barrier, by every lane for itself; `ok` says whether it came (the same in all lanes but
    // where a wait runs out: the roles look at all lanes' once per step).
    bool ok = true;
    auto await = [&](uint32_t bar, int k) {
        if (!mbar_try_wait(bar, k & 1)) ok &= thread_wait(bar, k & 1, &sm.abort, a.err, kPolls);
    };
    auto fine = [&]() { return __all_sync(0xffffffffu, ok) != 0; };

    // A box takes 64 columns of a page, or of half a page of 256: lane (box, half) of a tile looks its row up and copies it.
    const int box_rows = min(128, 1 << a.shift), box = lane / HALVES, half = lane % HALVES;
    auto box_needed = [&](const PrefixPiece &x, int t) {
        return box < 128 / box_rows && x.k0 + t * kPrefixTile + box * box_rows < x.end;
    };
    auto box_row = [&](const PrefixPiece &x, int t) {
        return box_needed(x, t) ? (int)a.pool_row(x, x.k0 + t * kPrefixTile + box * box_rows) : -1;
    };
    auto copy_tile = [&](int i, int phase, int row, const CUtensorMap *map) {  // into place i, for its phase
        const int n = __popc(__ballot_sync(0xffffffffu, row >= 0));
        await(smem_addr(&sm.empty[i]), phase + 1);
        if (!fine()) return;
        const uint32_t bar = smem_addr(&sm.full[i]);
        if (lane == 0) mbar_expect_tx(bar, (uint32_t)(n * box_rows * 128));
        __syncwarp();
        if (row >= 0) tma_load_2d(ring + i * TILE + half * BOX + box * box_rows * 128, map, 64 * half, row, bar);
        __syncwarp();
    };
    // registers of the launch, 168 a thread: 88 for warps 0 to 3, 208 for the softmax, which holds a row of a block
    static_assert(128 * 88 + 256 * 208 <= C::THREADS * 168, "no more than the launch has");
    if (warp == 0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        PrefixWalk w = a.range();
        PrefixPiece pc;
        // ---- pieces, queries, K tiles
        int slot = 0, nq = 0;
        for (int np = 0; fine(); ++np) {
            const bool more = a.next(w, pc);
            await(smem_addr(&sm.piece_empty[np % NP]), np / NP + 1);
            if (!fine()) break;
            if (lane == 0) {
                if (!more) pc.t1 = pc.t0 = 0;
                sm.piece[np % NP] = pc;
                sm.bad[np % NP] = 0;
                mbar_arrive(smem_addr(&sm.piece_full[np % NP]));
            }
            __syncwarp();
            if (!more) break;
            int row = box_row(pc, pc.t0);
            for (int s = 0; s < (pc.nseq > a.rows.half ? 2 : 1); ++s, ++nq) {
                const int i = nq & 1;
                await(smem_addr(&sm.q_empty[i]), (nq >> 1) + 1);
                if (!fine()) break;
                if (lane == 0) {
                    const uint32_t bar = smem_addr(&sm.q_full[i]);
                    mbar_expect_tx(bar, (uint32_t)((pc.own ? 1 : a.rows.half) * a.G * HALVES * 128));
                    for (int hh = 0; hh < HALVES; ++hh)
                        tma_load_3d(Qs + i * TILE + hh * BOX, pc.own ? &tmQ1 : &tmQ, 64 * hh, pc.h * a.G,
                                    pc.layer * a.B + pc.b0 + pc.s0 + s * a.rows.half, bar);
                }
                __syncwarp();
            }
            for (int t = pc.t0; fine() && t < pc.t1; ++t, ++slot) {
                if (__any_sync(0xffffffffu, box_needed(pc, t) && row < 0) && lane == 0) {
                    *(volatile int *)&sm.bad[np % NP] = 1;
                    raise_error(a.err, ERR_PAGE);
                }
                const int next = t + 1 < pc.t1 ? box_row(pc, t + 1) : -1;
                copy_tile(slot % NK, slot / NK, row, &tmK);
                row = next;
            }
        }
        // no copy is left in flight when the CTA ends
        for (int j = max(0, slot - NK); j < slot; ++j) mbar_wait_bounded(smem_addr(&sm.full[j % NK]), (j / NK) & 1, kPolls);
        for (int j = max(0, nq - 2); j < nq; ++j) mbar_wait_bounded(smem_addr(&sm.q_full[j & 1]), (j >> 1) & 1, kPolls);
    } else if (warp == 2) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        // ---- V tiles
        int slot = 0;
        for (int np = 0; fine(); ++np) {
            await(smem_addr(&sm.piece_full[np % NP]), np / NP);
            if (!fine()) break;
            const PrefixPiece x = sm.piece[np % NP];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sm.piece_empty[np % NP]));
            if (x.t1 == x.t0) break;
            int row = box_row(x, x.t0);
            for (int t = x.t0; fine() && t < x.t1; ++t, ++slot) {
                const int next = t + 1 < x.t1 ? box_row(x, t + 1) : -1;
                copy_tile(NK + slot % NV, slot / NV, row, &tmV);
                row = next;
            }
        }
        for (int j = max(0, slot - NV); j < slot; ++j) mbar_wait_bounded(smem_addr(&sm.full[NK + j % NV]), (j / NV) & 1, kPolls);
    } else if (ALONE && warp == 3) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    } else if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        // ---- products of stream s
        constexpr uint32_t ID_S = idesc_bf16(128, 64), ID_O = idesc_bf16(128, D) | kIdescMnB;
        const int s = warp >> 1;
        // (the whole warp goes through the loops, so that what it computes is known to be uniform: operands of the products
        // come from uniform registers, and one thread alone issued a product every 70 to 125 cycles)
        const uint64_t qd = sw128_desc(Qs), kd = sw128_desc(ring), vd = sw128_desc_mn(ring, BOX);
        const uint32_t st = tmem + S_COL + 128 * s, o0 = tmem + O_COL + D * s;
        const uint32_t full0 = smem_addr(&sm.full[0]), empty0 = smem_addr(&sm.empty[0]), s_full0 = smem_addr(&sm.s_full[s][0]),
                       p_full0 = smem_addr(&sm.p_full[s][0]), pv_done0 = smem_addr(&sm.pv_done[s][0]);
        // places of the next K and V tile, and the parity of their phase; query tiles, blocks so far
        int ki = 0, vi = NK, kp = 0, vp = 0, nq = 0, n = 0;
        auto step_k = [&]() {
            if (++ki == NK) {
                ki = 0;
                kp ^= 1;
            }
        };
        auto step_v = [&]() {
            if (++vi == NS) {
                vi = NK;
                vp ^= 1;
            }
        };
        for (int np = 0; fine(); ++np) {
            await(smem_addr(&sm.piece_full[np % NP]), np / NP);
            if (!fine()) break;
            const PrefixPiece x = sm.piece[np % NP];
            const bool pair = x.nseq > a.rows.half;
            const bool both = pair || ALONE;  // the stream takes all keys
            const PrefixBlocks bl(x, both, s);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sm.piece_empty[np % NP]));
            if (bl.n == 0) break;
            const int q = nq + (pair ? s : 0);
            for (int i = 0; i < (pair ? 2 : 1); ++i, ++nq) await(smem_addr(&sm.q_full[nq & 1]), nq >> 1);
            if (!fine()) break;
            const uint64_t ad = qd + (uint64_t)((q & 1) * TILE >> 4);
            uint32_t more = 0;
#pragma unroll 1
            for (int j = 0; j < bl.n + 2; ++j) {
                const int odd = j & 1;
                if (j >= 2) {  // O += P V of block j - 2
                    const int c = bl.first + bl.step * (j - 2), nv = n + j - 2;
                    if (!both || !odd) await(full0 + 8 * vi, vp);
                    // rows that no query sees, within the product's steps of 16: zero, as their probabilities are (NaN times zero is
                    // not).  (With a pair, both warps may do it: zeros over zeros.)
                    const int r0 = c < bl.lo ? min(64, bl.lo - c) : 0, r1 = max(0, min(64, bl.hi - c));  // rows that count: [r0, r1)
                    if (((r0 | r1) & 15) != 0 && fine()) {
                        const uint32_t rows = ring + vi * TILE + (c & 64) * 128;
                        auto clear = [&](int r, int k) {
                            for (int i = lane; i < k * 8 * HALVES; i += 32)
                                sts_u4(rows + (i / (8 * k)) * BOX + (r + (i >> 3) % k) * 128 + (i & 7) * 16, make_uint4(0, 0, 0, 0));
                        };
                        if (r0 & 15) clear(r0 & ~15, r0 & 15);
                        if (r1 & 15) clear(r1, 16 - (r1 & 15));
                        fence_async_shared();
                        __syncwarp();
                    }
                    await(p_full0 + 8 * (nv & 1), nv >> 1);
                    // (every piece waits for the outputs of the one before to have been read, for the barrier's phases)
                    if (ALONE)
                        await(smem_addr(&sm.o_read[nv & 1]), (nv >> 1) + 1);
                    else if (j == 2 && np > 0)
                        await(smem_addr(&sm.o_free), np - 1);
                    if (!fine()) break;  // (a place whose copy has not come is not let go: it would be filled again with one under way)
                    tc_fence_after();
                    const uint64_t bd = vd + (uint32_t)((vi * TILE + (c & 64) * 128) >> 4);
                    const uint32_t p = st + 64 * (nv & 1), o = o0 + (ALONE ? D * (nv & 1) : 0);
                    const int k0 = r0 >> 4, k1 = (r1 + 15) >> 4;
                    if (elect_one()) {
                        if (k0 == 0 && k1 == 4) {
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                tc_mma_ts(o, p + 8 * k, bd + (uint32_t)(k * 2048 >> 4), ID_O, k > 0 ? 1u : more);
                                tc_mma_ts(o, p + 32 + 8 * k, bd + (uint32_t)(k * 2048 >> 4), ID_O, 1);
                                if (PARTS == 3) tc_mma_ts(o, tmem + P3_COL + 32 * (nv & 1) + 8 * k, bd + (uint32_t)(k * 2048 >> 4), ID_O, 1);
                            }
                        } else {
#pragma unroll 1
                            for (int k = k0; k < k1; ++k) {
                                tc_mma_ts(o, p + 8 * k, bd + (uint32_t)(k * 2048 >> 4), ID_O, k > k0 ? 1u : more);
                                tc_mma_ts(o, p + 32 + 8 * k, bd + (uint32_t)(k * 2048 >> 4), ID_O, 1);
                                if (PARTS == 3) tc_mma_ts(o, tmem + P3_COL + 32 * (nv & 1) + 8 * k, bd + (uint32_t)(k * 2048 >> 4), ID_O, 1);
                            }
                        }
                        tc_commit(pv_done0 + 8 * (nv & 1));
                        if (!both || odd) tc_commit(empty0 + 8 * vi);
                    }
                    __syncwarp();
                    if (!ALONE) more |= k0 < k1 ? 1u : 0u;
                    if (!both || odd) step_v();
                }
                if (j < bl.n) {  // S = Q K^T of block j
                    if (!both || !odd) await(full0 + 8 * ki, kp);
                    if (!fine()) break;
                    tc_fence_after();
                    const uint64_t bd = kd + (uint32_t)((ki * TILE + ((bl.first + bl.step * j) & 64) * 128) >> 4);
                    const uint32_t d = st + 64 * ((n + j) & 1);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint32_t off = ((k >> 2) * BOX + (k & 3) * 32) >> 4;
                            tc_mma(d, ad + off, bd + off, ID_S, k > 0);
                        }
                        tc_commit(s_full0 + 8 * ((n + j) & 1));
                        if (!both || odd) tc_commit(empty0 + 8 * ki);
                        if (j == bl.n - 1) {
                            tc_commit(smem_addr(&sm.q_empty[q & 1]));
                            if (pair) mbar_arrive(smem_addr(&sm.q_empty[(q & 1) ^ 1]));
                        }
                    }
                    __syncwarp();
                    if (!both || odd) step_k();
                }
            }
            n += bl.n;
        }
    } else if (ALONE && warp >= 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        // ---- outputs: the blocks' products add up in registers, query row r
        const int quarter = warp & 3, r = quarter * 32 + lane, seq_r = r / a.G, g = r - seq_r * a.G;
        const uint32_t oa = tmem + ((uint32_t)(quarter * 32) << 16) + O_COL;
        int n = 0;
        for (int np = 0; fine(); ++np) {
            await(smem_addr(&sm.piece_full[np % NP]), np / NP);
            if (!fine()) break;
            const PrefixPiece pc = sm.piece[np % NP];
            if (pc.t1 == pc.t0) break;
            const PrefixBlocks bl(pc, true, 0);
            const bool any_row = quarter * 32 < pc.nseq * a.G;
            float o[D];
#pragma unroll
            for (int i = 0; i < D; ++i) o[i] = 0.f;
#pragma unroll 1
            for (int j = 0; j < bl.n && fine(); ++j, ++n) {
                await(smem_addr(&sm.pv_done[0][n & 1]), n >> 1);
                __syncwarp();
                tc_fence_after();
                if (any_row) {
                    await(smem_addr(&sm.p_full[0][n & 1]), n >> 1);  // (long over: what the softmax wrote is seen)
                    const float al = sm.al[n & 1][ALONE ? r : 0];
                    if (__any_sync(0xffffffffu, al != 1.f)) {
#pragma unroll
                        for (int i = 0; i < D; ++i) o[i] *= al;
                    }
                    const int c = bl.step * j;
                    if (c < bl.hi && c + 64 > bl.lo) {  // (otherwise nothing was multiplied)
#pragma unroll
                        for (int x = 0; x < D; x += 32) {
                            float y[32];
                            tmem_ld32_nowait(oa + D * (n & 1) + x, y);
                            tmem_ld_wait_regs<32>(y);
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[x + i] += y[i];
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sm.o_read[n & 1]));
            }
            if (!fine()) break;
            await(smem_addr(&sm.met[np & 1]), np >> 1);
            __syncwarp();
            tc_fence_after();
            float ml[16];
            tmem_ld16_nowait(oa - O_COL + ML_COL + 16 * (np & 1), ml);
            tmem_ld_wait_regs<16>(ml);
            tc_fence_before();
            if (seq_r < pc.nseq) {
                float *po;
                float2 *pm;
                a.partial<D>(pc, seq_r, g, po, pm);
                *pm = make_float2(ml[0], *(volatile int *)&sm.bad[np % NP] ? -1.f : ml[1]);
#pragma unroll
                for (int y = 0; y < D; y += 8) st_global_v8(po + y, o + y);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sm.piece_empty[np % NP]));
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        // ---- softmax: stream s, query row r of its tile
        const int s = (warp - 4) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
        // (In place of zero the smallest scale there is, 2^-149: it leaves every finite logit below 2^-21 and hides what is masked.  Only
        // a logit of -inf then weighs nothing, where times zero it would be NaN; a factor ahead of the mask, which tells them
        // apart, cost float32 output 38 us of 525.)
        const float c2 = a.c2 == 0.f ? 0x1p-149f : a.c2, hide = c2 < 0.f ? INFINITY : -INFINITY;
        const int seq_r = r / a.G, g = r - seq_r * a.G;
        const uint32_t s_full0 = smem_addr(&sm.s_full[s][0]), p_full0 = smem_addr(&sm.p_full[s][0]);
        int n = 0, met_n = 0;  // blocks of this stream; meetings of the groups
        for (int np = 0; fine(); ++np) {
            await(smem_addr(&sm.piece_full[np % NP]), np / NP);
            if (!fine()) break;
            const PrefixPiece pc = sm.piece[np % NP];
            const int nt = pc.t1 - pc.t0;
            if (nt == 0) break;
            const bool pair = pc.nseq > a.rows.half;
            const int seq0 = pair && s ? a.rows.half : 0, nseq = pair ? (s ? pc.nseq - seq0 : a.rows.half) : pc.nseq;
            const bool any_row = quarter * 32 < nseq * a.G;
            const PrefixBlocks bl(pc, pair || ALONE, s);
            const bool there = seq_r < nseq;
            float m = -INFINITY, l = 0.f;
            const int first = n;
#pragma unroll 1
            for (int j = 0, c = bl.first; j < bl.n && fine(); ++j, c += bl.step) {
                await(s_full0 + 8 * (n & 1), n >> 1);
                __syncwarp();
                tc_fence_after();
                if (any_row) {
                    const uint32_t sa = lane_base + S_COL + 128 * s + 64 * (n & 1);
                    float v[64];
                    auto logits = [&]() {
                        tmem_ld32_nowait(sa, v);
                        tmem_ld32_nowait(sa + 32, v + 32);
                        tmem_ld_wait_regs<64>(v);
                        if (c < bl.lo || c + 64 > bl.hi) {
                            const int low = max(0, bl.lo - c), live = max(0, bl.hi - c - low);  // columns that count, from the first on
#pragma unroll
                            for (int x = 0; x < 64; ++x) v[x] = (unsigned)(x - low) < (unsigned)live ? v[x] : hide;
                        }
                    };
                    logits();
                    // Probabilities against the maximum so far.  No maximum of the block is looked for while their sum stays below
                    // 2^12 (each of them is below it, which float32 sums and bf16's range do not mind).  Two parts are made once that
                    // is known, from the probabilities in place of the logits; three as the probabilities come, which leaves the one
                    // group of warps that makes them least to wait for (28 layers below 524 us, made later 689).
                    float sum, factor = 1.f;
                    uint32_t hi[32], lo[32], rest[PARTS == 3 ? 32 : 1];
                    auto parts = [&](int y, float p0, float p1) {
                        float r0, r1;
                        split_bf16(p0, p1, hi[y], lo[y], r0, r1);
                        if (PARTS == 3) rest[y] = pack_bf16(r0, r1);
                    };
                    auto rise = [&](bool grow) {  // the maximum, for those whose probabilities it must lower
                        float mx = -INFINITY;
#pragma unroll
                        for (int x = 0; x < 64; x += 2) mx = max3(mx, v[x] * c2, v[x + 1] * c2);
                        const float mn = grow ? fmaxf(m, mx) : m;
                        factor = grow ? part_factor(m, mn) : 1.f;
                        l *= factor;
                        m = mn;
                    };
                    bool again = PARTS == 2 && n == first;
                    if (again) rise(there);
                    for (;;) {
                        const float nb = again && m == -INFINITY ? 0.f : -m;
                        const unsigned long long cc = pair_of(c2, c2), nn = pair_of(nb, nb);
                        unsigned long long s4[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
                        for (int y = 0; y < 32; ++y) {
                            float p0, p1;
                            unpair(fma_pair(pair_of(v[2 * y], v[2 * y + 1]), cc, nn), p0, p1);
                            p0 = fast_exp2(p0);
                            p1 = fast_exp2(p1);
                            s4[y & 3] = add_pair(s4[y & 3], pair_of(p0, p1));
                            if (PARTS == 3) {
                                parts(y, p0, p1);
                            } else {
                                v[2 * y] = p0;
                                v[2 * y + 1] = p1;
                            }
                        }
                        float s0, s1;
                        unpair(add_pair(add_pair(s4[0], s4[1]), add_pair(s4[2], s4[3])), s0, s1);
                        sum = s0 + s1;
                        const bool grow = there && !again && !(sum <= 0x1p12f);  // (while the maximum is -inf: infinities and NaN)
                        if (!__any_sync(0xffffffffu, grow)) break;
                        again = true;
                        if (PARTS == 2) logits();
                        rise(grow);
                        if (!ALONE && n > first) {  // the output so far
                            await(smem_addr(&sm.pv_done[s][(n - 1) & 1]), (n - 1) >> 1);
                            __syncwarp();
                            tc_fence_after();
#pragma unroll 1
                            for (int x = 0; x < D / 16; ++x) {
                                float o[16];
                                tmem_ld16_nowait(lane_base + O_COL + D * s + 16 * x, o);
                                tmem_ld_wait_regs<16>(o);
                                uint32_t ob[16];
#pragma unroll
                                for (int y = 0; y < 16; ++y) ob[y] = __float_as_uint(o[y] * factor);
                                tmem_st16(lane_base + O_COL + D * s + 16 * x, ob);
                            }
                        }
                    }
                    l += sum;
                    if (PARTS == 2) {
#pragma unroll
                        for (int y = 0; y < 32; ++y) parts(y, v[2 * y], v[2 * y + 1]);
                    }
                    tmem_st16(sa, hi);
                    tmem_st16(sa + 16, hi + 16);
                    tmem_st16(sa + 32, lo);
                    tmem_st16(sa + 48, lo + 16);
                    if (PARTS == 3) {
                        tmem_st16(lane_base + P3_COL + 32 * (n & 1), rest);
                        tmem_st16(lane_base + P3_COL + 32 * (n & 1) + 16, rest + 16);
                        await(smem_addr(&sm.o_read[n & 1]), (n >> 1) + 1);  // (the factor of two blocks before, too)
                        sm.al[n & 1][ALONE ? r : 0] = factor;
                        __syncwarp();
                    }
                    tmem_st_wait();
                } else if (ALONE) {
                    await(smem_addr(&sm.o_read[n & 1]), (n >> 1) + 1);  // (warps without rows go no further ahead than the others)
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full0 + 8 * (n & 1));
                ++n;
            }
            if (!fine()) break;
            if (ALONE) {
                uint32_t ml[16] = {__float_as_uint(m), __float_as_uint(l)};  // (in TMEM, as S was: 16 columns are the least that a store takes here)
                tmem_st16(lane_base + ML_COL + 16 * (np & 1), ml);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_addr(&sm.met[np & 1]));
                    mbar_arrive(smem_addr(&sm.piece_empty[np % NP]));
                }
                continue;
            }
            // ---- the piece's partial
            await(smem_addr(&sm.pv_done[s][(n - 1) & 1]), (n - 1) >> 1);
            __syncwarp();
            tc_fence_after();
            float f0 = 1.f, f1 = 0.f;
            if (!pair) {  // the streams join: each group takes half of the columns
                sm.ml[s][ALONE ? 0 : r] = make_float2(m, l);
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sm.met[0]));
                await(smem_addr(&sm.met[0]), met_n++);
                __syncwarp();
                tc_fence_after();
                const float2 x = sm.ml[0][ALONE ? 0 : r], y = sm.ml[1][ALONE ? 0 : r];
                m = fmaxf(x.x, y.x);
                f0 = part_factor(x.x, m);
                f1 = part_factor(y.x, m);
                l = x.y * f0 + y.y * f1;
            }
            if (any_row) {
                float *po = nullptr;
                float2 *pm = nullptr;
                if (there) {
                    a.partial<D>(pc, seq0 + seq_r, g, po, pm);
                    if (pair || s == 0) *pm = make_float2(m, *(volatile int *)&sm.bad[np % NP] ? -1.f : l);
                }
                auto store = [&](int c, const float (&o)[32]) {
                    if (po != nullptr)
#pragma unroll
                        for (int y = 0; y < 32; y += 8) st_global_v8(po + c + y, o + y);
                };
                if (pair) {
#pragma unroll 1
                    for (int x = 0; x < D; x += 64) {
                        float o[2][32];
                        __syncwarp();  // (lanes without a row stored nothing)
                        tmem_ld32_nowait(lane_base + O_COL + D * s + x, o[0]);
                        tmem_ld32_nowait(lane_base + O_COL + D * s + x + 32, o[1]);
                        tmem_ld_wait_regs<32>(o[0]);
                        tmem_ld_wait_regs<32>(o[1]);
                        store(x, o[0]);
                        store(x + 32, o[1]);
                    }
                } else {
                    // (a stream that saw nothing has a factor of zero, and maybe no output)
                    constexpr int H = D / 2;
                    const uint32_t oa = lane_base + O_COL + H * s;
#pragma unroll 1
                    for (int x = 0; x < H; x += 32) {
                        float o[2][32];
                        __syncwarp();
                        tmem_ld32_nowait(oa + x, o[0]);
                        tmem_ld32_nowait(oa + D + x, o[1]);
                        tmem_ld_wait_regs<32>(o[0]);
                        tmem_ld_wait_regs<32>(o[1]);
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[0][i] = (f0 != 0.f ? o[0][i] * f0 : 0.f) + (f1 != 0.f ? o[1][i] * f1 : 0.f);
                        store(H * s + x, o[0]);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_addr(&sm.o_free));
                mbar_arrive(smem_addr(&sm.piece_empty[np % NP]));
            }
        }
    }
    __syncthreads();
    if (tid == 0 && *(volatile int *)&sm.abort != 0) a.total->stopped = 1;
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

cudaError_t launch_prefix_tc(const reco_paged_kv &kv, const PrefixArgs &a, int grid, reco_dtype out_dtype, cudaStream_t s)
{
    CUtensorMap mk = {}, mv = {}, mq = {}, mq1 = {};
    const unsigned long long rows = (unsigned long long)kv.n_layers * kv.n_pages * kv.H_kv * kv.page;
    const unsigned long long tokens = (unsigned long long)kv.n_layers * kv.B;
    const int box = std::min(128, kv.page);
    if (!encode_bf16_2d(&mk, kv.k, rows, kv.d, 64, box) || !encode_bf16_2d(&mv, kv.v, rows, kv.d, 64, box) ||
        !encode_bf16_heads(&mq, a.q, tokens, kv.H_q, kv.d, a.G, a.rows.half) ||
        !encode_bf16_heads(&mq1, a.q, tokens, kv.H_q, kv.d, a.G, 1))
        return cudaErrorInvalidValue;
    typedef void (*Kernel)(CUtensorMap, CUtensorMap, CUtensorMap, CUtensorMap, PrefixArgs);
    const bool two = out_dtype == RECO_BF16;
    const Kernel fn = kv.d == 64 ? (two ? prefix_tc<64, 2> : prefix_tc<64, 3>) : (two ? prefix_tc<128, 2> : prefix_tc<128, 3>);
    const int smem = kv.d == 64 ? (two ? PrefixTc<64, 2>::SMEM : PrefixTc<64, 3>::SMEM) : (two ? PrefixTc<128, 2>::SMEM : PrefixTc<128, 3>::SMEM);
    cudaError_t e = allow_smem((const void *)fn, smem);
    if (e != cudaSuccess) return e;
    e = launch_pdl(fn, dim3(grid), dim3(PrefixTc<64, 2>::THREADS), smem, s, mk, mv, mq, mq1, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace reco
