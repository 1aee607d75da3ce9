// prefix_tc.cu -- the prefix part of decode attention over shared prefixes (prefix.cu) for bf16 caches, on the tensor
// cores (tcgen05, TMEM): S = Q K^T and O += P V over tiles of 128 query rows and 128 keys, with an online softmax
// between them (running maximum and sum in float32, to base 2).
//
// R query rows of a group serve 4 R d operations per 4 d bytes of K and V: below some 285 rows the bytes are the bound,
// above it the tensor cores.  A product's 128 rows cost the same however many are there, so that few rows cost
// nothing more while the bytes are.
//
// One CTA per SM, persistent over its share of the key tiles (PrefixArgs::next), of warps
//   0      copies, all by TMA: queries (a box of a group's sequences, or one sequence's, into one of two tiles), K and V
//          (a box per page and 64 columns, one lane each, into a ring of tiles);
//   1      issues the products;
//   4..11  two softmax groups of four warps, a query row per thread.
// Two streams of products alternate, so that one's softmax runs beside the other's products: a row tile of more than
// 128 rows has a half in each stream, which share every K and V tile; otherwise the streams are the even and the
// odd key tiles, and join at the end of the piece.  A stream's S (128 columns of TMEM) is overwritten by its P in bf16, which
// the second product takes from there; O stays in TMEM, and is rescaled only when a row's maximum has grown by
// more than 2^8 (kLazyLog2: probabilities against the older maximum stay exact in float32).
// The copies and the score products run ahead into the next piece while the groups finish one.
//
// P enters its product in bf16: with float32 output in two parts (2^-17 of each probability is lost), with bf16
// output in one (2^-8 of each, on average over the rows the size of the output's own rounding).  Sums take the
// probabilities as they were before.
//
// Every wait is bounded; one that runs out raises the error word and the CTA's abort flag, which ends the others.
#include <algorithm>

#include "decode_block.cuh"
#include "prefix.cuh"
#include "tc.cuh"

namespace reco {

// Two float32 in a register pair, and arithmetic on both at once.
__device__ __forceinline__ unsigned long long pair_of(float a, float b)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(unsigned long long x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ unsigned long long fma_pair(unsigned long long a, unsigned long long b, unsigned long long c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long add_pair(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

template <int D> struct PrefixTc {
    static constexpr int HALVES = D / 64;
    static constexpr int BOX = 128 * 128;  // 128 rows of 64 bf16
    static constexpr int TILE = HALVES * BOX;
    static constexpr int Q_BYTES = 2 * TILE;
    static constexpr int NS = D == 128 ? 5 : 10;  // K and V tiles in the ring
    static constexpr int THREADS = 32 * 12;
    struct Small {  // behind the tiles
        uint64_t full[NS], empty[NS], q_full[2], q_empty[2], s_full[2], p_full[2], pv_done[2], o_free, met;
        float2 ml[2][128];
        uint32_t tmem;
        int abort;
    };
    // (all of it dynamic: the tiles begin where the CTA's shared memory does, at a multiple of 1024)
    static constexpr int SMEM = Q_BYTES + NS * TILE + (int)sizeof(Small);
    static_assert(SMEM <= 227 * 1024, "shared memory of a CTA");
};

template <int D, int PARTS>
__global__ void __launch_bounds__(PrefixTc<D>::THREADS, 1)
    prefix_tc(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
              const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmQ1, const __grid_constant__ PrefixArgs a)
{
    using C = PrefixTc<D>;
    constexpr int NS = C::NS, BOX = C::BOX, TILE = C::TILE, HALVES = C::HALVES;
    constexpr uint32_t S_COL = 0, O_COL = 256;  // TMEM: S (then P) of the streams, 128 columns each, then their O
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = smem_addr(smem_raw), Qs = base, ring = base + C::Q_BYTES;
    typename C::Small &sm = *reinterpret_cast<typename C::Small *>(smem_raw + C::Q_BYTES + NS * TILE);
    if (base & 1023u) {  // swizzled tiles need it
        if (tid == 0) raise_error(a.err, ERR_INTERNAL);
        return;
    }
    if (tid == 0) {
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
        prefetch_tensormap(&tmQ);
        prefetch_tensormap(&tmQ1);
        for (int i = 0; i < NS; ++i) {
            mbar_init(smem_addr(&sm.full[i]), 1);
            mbar_init(smem_addr(&sm.empty[i]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_addr(&sm.q_full[s]), 1);
            mbar_init(smem_addr(&sm.q_empty[s]), 1);
            mbar_init(smem_addr(&sm.s_full[s]), 1);
            mbar_init(smem_addr(&sm.p_full[s]), 4);
            mbar_init(smem_addr(&sm.pv_done[s]), 1);
        }
        mbar_init(smem_addr(&sm.o_free), 8);
        mbar_init(smem_addr(&sm.met), 8);
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
    volatile int *abort_flag = &sm.abort;
    wait_prior_grid();
    release_next_grid();  // the join looks up its places meanwhile
    // registers of the launch, 168 a thread: 88 for warps 0 to 3, 208 for the softmax, which holds a row of S
    static_assert(128 * 88 + 256 * 208 <= C::THREADS * 168, "no more than the launch has");
    auto wait = [&](uint64_t &bar, int k) { return warp_wait(smem_addr(&bar), k & 1, abort_flag, a.err); };  // its phase k

    if (warp == 0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        PrefixWalk w = a.range();
        PrefixPiece pc;
        // ---- copies.  Lane (box, half) of a tile copies 64 columns of the box's rows: a page, or half a page of 256
        const int rows = min(128, 1 << a.shift), boxes = 128 / rows;
        const int box = lane / HALVES, half = lane % HALVES;
        int slot = 0, nq = 0;
        bool ok = true;
        while (ok && a.next(w, pc)) {
            auto row_of = [&](int t) {
                const int k = pc.k0 + t * kPrefixTile + box * rows;
                return box < boxes && k < pc.end ? a.pool_row(pc, k) : -1ll;
            };
            long long row = row_of(pc.t0);
            for (int s = 0; s < (pc.nseq > a.rows.half ? 2 : 1); ++s, ++nq) {
                const int i = nq & 1;
                if (!(ok = wait(sm.q_empty[i], (nq >> 1) + 1))) break;
                if (lane == 0) {
                    const uint32_t bar = smem_addr(&sm.q_full[i]);
                    mbar_expect_tx(bar, (uint32_t)((pc.own ? 1 : a.rows.half) * a.G * HALVES * 128));
                    for (int hh = 0; hh < HALVES; ++hh)
                        tma_load_3d(Qs + i * TILE + hh * BOX, pc.own ? &tmQ1 : &tmQ, 64 * hh, pc.h * a.G,
                                    pc.layer * a.B + pc.b0 + pc.s0 + s * a.rows.half, bar);
                }
                __syncwarp();
            }
            for (int t = pc.t0; ok && t < pc.t1; ++t) {
                const int n = __popc(__ballot_sync(0xffffffffu, row >= 0));
                const long long next = t + 1 < pc.t1 ? row_of(t + 1) : -1ll;
                for (int kv = 0; kv < 2; ++kv, ++slot) {
                    const int i = slot % NS;
                    if (!(ok = wait(sm.empty[i], slot / NS + 1))) break;
                    const uint32_t bar = smem_addr(&sm.full[i]);
                    if (lane == 0) mbar_expect_tx(bar, (uint32_t)(n * rows * 128));
                    __syncwarp();
                    if (row >= 0)
                        tma_load_2d(ring + i * TILE + half * BOX + box * rows * 128, kv ? &tmV : &tmK, 64 * half, (int)row, bar);
                    __syncwarp();
                }
                row = next;
            }
        }
        // no copy is left in flight when the CTA ends
        for (int j = max(0, slot - NS); j < slot; ++j) mbar_wait_bounded(smem_addr(&sm.full[j % NS]), (j / NS) & 1, kTcSpin);
        for (int j = max(0, nq - 2); j < nq; ++j) mbar_wait_bounded(smem_addr(&sm.q_full[j & 1]), (j >> 1) & 1, kTcSpin);
    } else if (warp == 1) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        PrefixWalk w = a.range();
        PrefixPiece pc;
        // ---- products
        constexpr uint32_t ID_S = idesc_bf16(128, 128), ID_O = idesc_bf16(128, D) | kIdescMnB;
        int slot0 = 0, nq = 0, ns[2] = {0, 0}, pieces = 0;  // ring slots, query tiles, products of each stream so far
        bool ok = true;
        while (ok && a.next(w, pc)) {
            const int nt = pc.t1 - pc.t0;
            const bool pair = pc.nseq > a.rows.half;
            const int jobs = pair ? 2 * nt : nt;
            auto scores = [&](int j) {
                const int s = j & 1, t = pair ? j >> 1 : j, slot = slot0 + 2 * t, i = slot % NS;
                const int q = nq + (pair ? s : 0);  // the tile of queries
                if ((pair ? j < 2 : j == 0) && !wait(sm.q_full[q & 1], q >> 1)) return false;
                if ((!pair || s == 0) && !wait(sm.full[i], slot / NS)) return false;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t ad = sw128_desc(Qs + (q & 1) * TILE), bd = sw128_desc(ring + i * TILE);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint64_t off = (uint64_t)(((k >> 2) * BOX + (k & 3) * 32) >> 4);
                        tc_mma(tmem + S_COL + 128 * s, ad + off, bd + off, ID_S, k > 0);
                    }
                    tc_commit(smem_addr(&sm.s_full[s]));
                    if (!pair || s == 1) tc_commit(smem_addr(&sm.empty[i]));
                    if (pair ? t == nt - 1 : j == jobs - 1) tc_commit(smem_addr(&sm.q_empty[q & 1]));
                }
                __syncwarp();
                return true;
            };
            auto values = [&](int j) {
                const int s = j & 1, t = pair ? j >> 1 : j, slot = slot0 + 2 * t + 1, i = slot % NS;
                // rows of the tile that count: [low, live); the product takes them in steps of 16
                const int k0 = pc.k0 + (pc.t0 + t) * kPrefixTile, low = max(0, pc.lo - k0), live = min(kPrefixTile, pc.end - k0);
                const int step0 = low >> 4, step1 = (live + 15) / 16;
                if (!pair || s == 0) {
                    if (!wait(sm.full[i], slot / NS)) return false;
                    // other rows of those steps: zero, as their probabilities are (NaN times zero is not)
                    auto clear = [&](int r0, int n) {
                        for (int x = lane; x < n * 8 * HALVES; x += 32)
                            sts_u4(ring + i * TILE + (x / (8 * n)) * BOX + (r0 + (x >> 3) % n) * 128 + (x & 7) * 16, make_uint4(0, 0, 0, 0));
                    };
                    if ((low | live) & 15) {
                        if (low & 15) clear(low & ~15, low & 15);
                        if (live & 15) clear(live, 16 * step1 - live);
                        fence_async_shared();
                        __syncwarp();
                    }
                }
                if (!wait(sm.p_full[s], ns[s]++)) return false;
                if (j == 0 && pieces > 0 && !wait(sm.o_free, pieces - 1)) return false;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t bd = sw128_desc_mn(ring + i * TILE, BOX);
                    const uint32_t p = tmem + S_COL + 128 * s, o = tmem + O_COL + D * s;
                    for (int k = step0; k < step1; ++k) {
                        tc_mma_ts(o, p + 8 * k, bd + (uint64_t)(k * 2048 >> 4), ID_O, k > step0 || j > 1);
                        if (PARTS == 2) tc_mma_ts(o, p + 64 + 8 * k, bd + (uint64_t)(k * 2048 >> 4), ID_O, 1);
                    }
                    tc_commit(smem_addr(&sm.pv_done[s]));
                    if (!pair || s == 1) tc_commit(smem_addr(&sm.empty[i]));
                }
                __syncwarp();
                return true;
            };
            for (int j = 0; ok && j < jobs + 2; ++j) {
                if (j >= 2 && j - 2 < jobs) ok = values(j - 2);
                if (ok && j < jobs) ok = scores(j);
            }
            slot0 += 2 * nt;
            nq += pair ? 2 : 1;
            ++pieces;
        }
    } else if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        PrefixWalk w = a.range();
        PrefixPiece pc;
        // ---- softmax: stream s, query row r of its tile
        const int s = (warp - 4) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t sa = lane_base + S_COL + 128 * s;
        // (a scale of zero: one that leaves every finite logit next to zero, and hides what is masked with -inf)
        const float c2 = fmaxf(fabsf(a.c2), 1e-30f);
        const bool minus = a.c2 < 0.f;
        const int seq_r = r / a.G, g = r - seq_r * a.G;
        int n = 0, met_n = 0, pieces = 0;  // products of this stream; meetings of the groups
        bool ok = true;
        while (ok && a.next(w, pc)) {
            const int nt = pc.t1 - pc.t0;
            const bool pair = pc.nseq > a.rows.half;
            const int seq0 = pair && s ? a.rows.half : 0, nseq = pair ? (s ? pc.nseq - seq0 : a.rows.half) : pc.nseq;
            const bool any_row = quarter * 32 < nseq * a.G;
            bool bad = false;  // a page that is none among the piece's
            {
                const int e0 = max(pc.lo, pc.k0 + pc.t0 * kPrefixTile) >> a.shift;
                const int e1 = (min(pc.end, pc.k0 + pc.t1 * kPrefixTile) - 1) >> a.shift;
                for (int e = e0 + lane; e <= e1; e += 32)
                    bad |= (unsigned)__ldg(a.table + (long long)pc.b0 * a.max_pages + e) >= (unsigned)a.n_pages;
                bad = __any_sync(0xffffffffu, bad);
            }
            float m = -INFINITY, l = 0.f;
            const int first = n;
            for (int t = pc.t0 + (pair ? 0 : s); ok && t < pc.t1; t += pair ? 1 : 2, ++n) {
                if (!(ok = wait(sm.s_full[s], n))) break;
                tc_fence_after();
                const int k0 = pc.k0 + t * kPrefixTile, live = min(kPrefixTile, pc.end - k0), low = pc.lo - k0;
                const bool whole = live == kPrefixTile && low <= 0;
                if (any_row) {
                    float v[128];
#pragma unroll
                    for (int x = 0; x < 4; ++x) tmem_ld32_nowait(sa + 32 * x, v + 32 * x);
                    tmem_ld_wait_regs<128>(v);
                    if (minus || !whole) {
#pragma unroll
                        for (int x = 0; x < 128; ++x) v[x] = x < live && x >= low ? (minus ? -v[x] : v[x]) : -INFINITY;
                    }
                    float mx[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
                    for (int x = 4; x + 8 <= 128; x += 8)
#pragma unroll
                        for (int y = 0; y < 4; ++y) mx[y] = max3(mx[y], v[x + y], v[x + 4 + y]);
#pragma unroll
                    for (int y = 0; y < 4; ++y) mx[y] = fmaxf(mx[y], v[124 + y]);
                    const float mb = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * c2;
                    const bool grow = mb > m + kLazyLog2;
                    if (__any_sync(0xffffffffu, grow)) {
                        const float mn = grow ? mb : m, al = grow ? fast_exp2(m - mn) : 1.f;
                        l *= al;
                        m = mn;
                        if (n > first) {  // the output so far
                            if (!(ok = wait(sm.pv_done[s], n - 1))) break;
                            tc_fence_after();
#pragma unroll 1
                            for (int x = 0; x < D / 16; ++x) {
                                float o[16];
                                tmem_ld16_nowait(lane_base + O_COL + D * s + 16 * x, o);
                                tmem_ld_wait_regs<16>(o);
                                uint32_t ob[16];
#pragma unroll
                                for (int y = 0; y < 16; ++y) ob[y] = __float_as_uint(o[y] * al);
                                tmem_st16(lane_base + O_COL + D * s + 16 * x, ob);
                            }
                        }
                    }
                    const float nb = m == -INFINITY ? 0.f : -m;
                    const unsigned long long cc = pair_of(c2, c2), nn = pair_of(nb, nb);
                    unsigned long long sum[2] = {0ull, 0ull};
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        uint32_t hi[16], lo[16];
#pragma unroll
                        for (int y = 0; y < 16; ++y) {
                            const int i = 32 * x + 2 * y;
                            float p0, p1;
                            unpair(fma_pair(pair_of(v[i], v[i + 1]), cc, nn), p0, p1);
                            p0 = fast_exp2(p0);
                            p1 = fast_exp2(p1);
                            sum[y & 1] = add_pair(sum[y & 1], pair_of(p0, p1));
                            if (PARTS == 2)
                                split_bf16(p0, p1, hi[y], lo[y]);
                            else
                                hi[y] = pack_bf16(p0, p1);
                        }
                        tmem_st16(sa + 16 * x, hi);
                        if (PARTS == 2) tmem_st16(sa + 64 + 16 * x, lo);
                    }
                    float s0, s1;
                    unpair(add_pair(sum[0], sum[1]), s0, s1);
                    l += s0 + s1;
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sm.p_full[s]));
            }
            if (!ok) break;
            // ---- the piece's partial
            if (n > first && !(ok = wait(sm.pv_done[s], n - 1))) break;
            tc_fence_after();
            int cols = D, col0 = 0;
            float f0 = 1.f, f1 = 0.f;
            if (!pair) {  // the streams join: each group takes half of the columns
                // (a group without a product in this piece has not waited for the other to be done with the one before)
                if (n == first && pieces > 0 && !(ok = wait(sm.o_free, pieces - 1))) break;
                sm.ml[s][r] = make_float2(m, l);
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sm.met));
                if (!(ok = wait(sm.met, met_n++))) break;
                const float2 x = sm.ml[0][r], y = sm.ml[1][r];
                m = fmaxf(x.x, y.x);
                f0 = part_factor(x.x, m);
                f1 = part_factor(y.x, m);
                l = x.y * f0 + (nt > 1 ? y.y * f1 : 0.f);
                cols = D / 2;
                col0 = s * cols;
            }
            if (any_row) {
                float *po = nullptr;
                float2 *pm = nullptr;
                if (seq_r < nseq) {
                    a.partial<D>(pc, seq0 + seq_r, g, po, pm);
                    if (pair || s == 0) *pm = make_float2(m, bad ? -1.f : l);
                }
#pragma unroll 1
                for (int x = 0; x < cols; x += 16) {
                    float o[16];
                    const uint32_t oa = lane_base + O_COL + col0 + x;
                    tmem_ld16_nowait(oa + (pair ? D * s : 0), o);
                    tmem_ld_wait_regs<16>(o);
                    if (!pair) {
                        float o1[16];
                        if (nt > 1) {
                            tmem_ld16_nowait(oa + D, o1);
                            tmem_ld_wait_regs<16>(o1);
                        }
#pragma unroll
                        for (int y = 0; y < 16; ++y) o[y] = o[y] * f0 + (nt > 1 ? o1[y] * f1 : 0.f);
                    }
                    if (po != nullptr)
#pragma unroll
                        for (int y = 0; y < 16; y += 4)
                            *reinterpret_cast<float4 *>(po + col0 + x + y) = make_float4(o[y], o[y + 1], o[y + 2], o[y + 3]);
                }
            }
            if (bad && tid == 128) raise_error(a.err, ERR_PAGE);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sm.o_free));
            ++pieces;
        }
    }
    __syncthreads();
    if (warp == 1) {
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
    const bool one = out_dtype == RECO_BF16;
    const Kernel fn = kv.d == 64 ? (one ? prefix_tc<64, 1> : prefix_tc<64, 2>) : (one ? prefix_tc<128, 1> : prefix_tc<128, 2>);
    const int smem = kv.d == 64 ? PrefixTc<64>::SMEM : PrefixTc<128>::SMEM;
    cudaError_t e = allow_smem((const void *)fn, smem);
    if (e != cudaSuccess) return e;
    e = launch_pdl(fn, dim3(grid), dim3(PrefixTc<64>::THREADS), smem, s, mk, mv, mq, mq1, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace reco
