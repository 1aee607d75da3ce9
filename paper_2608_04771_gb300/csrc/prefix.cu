// prefix.cu -- decode attention of a batch whose sequences share the rows of a prefix: several answers to one question
// (the paper samples several reasoning paths per question), whose rows lie once in the pool, in pages that the group's
// first sequence names.
//
// For a query head with logits x_j over the prefix (j < P) and over its sequence's own rows (j >= P), the softmax over
// both is that of the parts joined: with M the largest of the parts' maxima m_i (to base 2),
//   l = sum_i 2^(m_i - M) l_i,   out = sum_i 2^(m_i - M) o_i / l.
// Three launches: prefix_plan appends the new rows, lists the groups and counts the work; the attention (float32 here, bf16
// in prefix_tc.cu) reads a prefix's rows once for all query heads of its group, and each unit's own rows;
// prefix_join joins the parts and advances the lengths.
//
// The work: the n sequences of a group are cut into row tiles, rows into tiles of 128; the (row tile, key tile) pairs of
// all layers, heads and groups, then the key tiles of the units' own rows, laid end to end, are shared out evenly to
// one CTA per SM.  An item (a row tile against its prefix, a unit against its own rows) that is cut between CTAs leaves
// several partials (max, sum, output), joined in the order of the CTAs: the same inputs give the same bits.
#include <algorithm>

#include "decode_block.cuh"
#include "prefix.cuh"
#include "tc.cuh"

namespace reco {

// ---------------------------------------------------------------- plan
// Inclusive scan over the CTA's threads: of maxima or sums.
template <bool MAX, typename V> __device__ __forceinline__ V scan_block(V x, V *sm)
{
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x = MAX ? max(x, y) : x + y;
    }
    __syncthreads();
    if (lane == 31) sm[wid] = x;
    __syncthreads();
    for (int w = 0; w < wid; ++w) x = MAX ? max(x, sm[w]) : x + sm[w];
    return x;
}

struct PlanArgs {
    void *K, *V;
    const void *k_new, *v_new;  // or nullptr
    const int32_t *table, *lens, *group, *shared;
    int units, B, Hkv, cap, n_pages, max_pages, shift, row_bytes;
    PrefixRows rows;
    PrefixWs ws;
    unsigned *err;
};

__device__ __forceinline__ bool has_company(const int32_t *group, int B, int b)
{
    const int g = __ldg(group + b);
    const int prev = b > 0 ? __ldg(group + b - 1) : ~g, next = b + 1 < B ? __ldg(group + b + 1) : ~g;
    return prev == g || next == g;
}

// The groups of at least two sequences that share rows, in order, and each sequence's.
__device__ void plan_groups(const PlanArgs &a)
{
    __shared__ long long sm[kPrefixBlock / 32], sm_work;
    __shared__ int sm_start, sm_runs;
    __shared__ int sm_most;
    if (threadIdx.x == 0) sm_most = a.rows.own();
    if (threadIdx.x == 0) {
        sm_work = 0;
        sm_start = -1;
        sm_runs = 0;
    }
    bool off = false;
    for (int b0 = 0; b0 < a.B; b0 += kPrefixBlock) {
        const int b = b0 + threadIdx.x;
        const bool in = b < a.B;
        const int g = in ? __ldg(a.group + b) : 0;
        const bool first = in && (b == 0 || __ldg(a.group + b - 1) != g), last = in && (b == a.B - 1 || __ldg(a.group + b + 1) != g);
        __syncthreads();
        const int c_start = sm_start, c_runs = sm_runs;
        const long long c_work = sm_work;
        const int start = max(c_start, scan_block<true>(first ? b : -1, reinterpret_cast<int *>(sm)));
        const int p = in ? __ldg(a.shared + start) : 0;
        const bool valid = p >= 0 && p <= a.cap, kept = in && valid && p > 0 && !(first && last);
        const int run = c_runs + scan_block<false>(first && kept ? 1 : 0, reinterpret_cast<int *>(sm)) - 1;
        const long long mine = last && kept ? a.rows.work(b - start + 1, p) : 0;
        const long long work = c_work + scan_block<false>(mine, sm);
        if (last && kept) atomicMax(&sm_most, a.rows.unit(b - start + 1, 0));
        if (last && kept) a.ws.runs[run] = PrefixRun{start, b - start + 1, p, 0, work - mine};
        if (in) {
            const bool wrong = !valid || __ldg(a.shared + b) != p;
            off |= wrong;
            a.ws.run_of[b] = wrong ? -2 : (kept ? run : -1);
        }
        __syncthreads();
        if (threadIdx.x == kPrefixBlock - 1) {
            sm_start = start;
            sm_runs = run + 1;
            sm_work = work;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) *a.ws.total = PrefixTotal{sm_work, sm_runs, sm_most, 0};
    if (off) raise_error(a.err, ERR_LEN);
}

// Whether a unit's length and prefix are in order, and the pool row of its new row (-1: its table names no page for it).
__device__ __forceinline__ bool unit_fine(const PlanArgs &a, int L, int p) { return unit_ok(L, a.cap, a.k_new != nullptr) && p >= 0 && p <= L; }
__device__ __forceinline__ long long new_row(const PlanArgs &a, int u, int L)
{
    const int lb = u / a.Hkv, layer = lb / a.B, b = lb - layer * a.B;
    const int e = __ldg(a.table + (long long)b * a.max_pages + (L >> a.shift));
    if ((unsigned)e >= (unsigned)a.n_pages) return -1;
    return ((((long long)layer * a.n_pages + e) * a.Hkv + (u - lb * a.Hkv)) << a.shift) + (L & ((1 << a.shift) - 1));
}

// A block of units: their own rows and the work of those.
__device__ void plan_units(const PlanArgs &a, int block)
{
    __shared__ int sm[kPrefixBlock / 32];
    const int u = block * kPrefixBlock + threadIdx.x, append = a.k_new ? 1 : 0;
    PrefixUnit x = {0, 0, 0, -1};
    int work = 0;
    if (u < a.units) {
        const int L = __ldcg(a.lens + u), b = u / a.Hkv % a.B, p = __ldg(a.shared + b);
        const bool company = has_company(a.group, a.B, b);
        if (!unit_fine(a, L, p)) {
            raise_error(a.err, append && L == a.cap ? ERR_ROOM : ERR_LEN);
        } else if (append && new_row(a, u, L) < 0) {
            raise_error(a.err, ERR_PAGE);
        } else {
            x.n = L + append;
            x.lo = company ? p : 0;
            x.k0 = x.lo & -min(kPrefixTile, 1 << a.shift);  // the tensor cores' kernel copies whole boxes
            work = x.n - x.lo > a.rows.few ? a.rows.own() * ((x.n - x.k0 + kPrefixTile - 1) / kPrefixTile) + a.rows.extra() : 0;
        }
    }
    const int before = scan_block<false>(work, sm) - work;
    if (u < a.units) {
        x.work = before;
        a.ws.units[u] = x;
    }
    if (threadIdx.x == kPrefixBlock - 1) a.ws.block_work[block] = before + work;
}

// New rows into the pool, 16 bytes a thread.
__device__ void plan_rows(const PlanArgs &a, int block)
{
    const int chunks = a.row_bytes / 16;
    const long long i = (long long)block * kPrefixBlock + threadIdx.x;
    const int u = (int)(i / (2 * chunks)), c = (int)(i - (long long)u * 2 * chunks), at = c < chunks ? c : c - chunks;
    if (u >= a.units) return;
    const uint4 x = __ldg(reinterpret_cast<const uint4 *>(c < chunks ? a.k_new : a.v_new) + (long long)u * chunks + at);
    const int L = __ldcg(a.lens + u);
    if (!unit_fine(a, L, __ldg(a.shared + u / a.Hkv % a.B))) return;
    const long long r = new_row(a, u, L);
    if (r >= 0) reinterpret_cast<uint4 *>(c < chunks ? a.K : a.V)[r * chunks + at] = x;
}

__global__ void __launch_bounds__(kPrefixBlock) prefix_plan(const __grid_constant__ PlanArgs a)
{
    release_next_grid();  // (the attention's CTAs set themselves up meanwhile)
    wait_prior_grid();
    const int blocks = (a.units + kPrefixBlock - 1) / kPrefixBlock;
    if (blockIdx.x == 0)
        plan_groups(a);
    else if ((int)blockIdx.x <= blocks)
        plan_units(a, blockIdx.x - 1);
    else
        plan_rows(a, blockIdx.x - 1 - blocks);
}

// ---------------------------------------------------------------- attention, float32
// Plain FMAs (two to an instruction), every sum float32.  A warp finds the pieces and copies; eight compute: one takes RW of
// the tile's query rows (32 at most) and a share of its 128 keys (WR row groups, 8 / WR key groups).  K and V tiles come
// by TMA, a box per page and 32 columns, into a ring of three; swizzled, so that lanes that read the same columns of
// different rows meet different banks.  A warp waits for a tile, and lets it go, for itself.
// QK^T: eight lanes share a row group's keys, four the rows: RW / 4 rows and KEYS / 8 keys to a lane, so that six to eight
// 16-byte reads feed up to 64 FMAs.  PV: a lane has D / 32 columns of all RW rows, and takes the probabilities from shared
// memory.  28 layers of 8 sequences in two groups (12 and 2 heads of 128, 1500 to 2000 shared rows, 315 MB): 125 us, where
// the bytes are 46 and the FMAs 40.  A tile of 32 rows takes 14300 cycles, of which the FMAs could issue in 8200: no tile
// is waited for, two warps a scheduler hide too little of what shared memory takes.  Halving its reads (8 keys and 8
// rows to a lane, d split four ways and joined by shuffles) gained nothing; one FMA to an instruction: 131 us; row
// groups of 8 with 16 lanes a row, at 168 registers: 146 us.
constexpr int kPlainRows = 32;
constexpr long long kPlainPolls = 1LL << 19;  // of a wait, each suspended for up to two microseconds
constexpr int kPlainWarps = 8, kPlainThreads = 32 * (kPlainWarps + 4);  // (registers are split by groups of four warps)

template <int D> struct PlainSmem {
    float ring[3][kPrefixTile * D];       // [D / 32][128][32], swizzled
    float q[kPlainRows * D];              // queries, then probabilities by warp; at a piece's end the warps' outputs as they
    float p[D == 128 ? 32 * D : 64 * D];  // join: 8 warps of 8 rows
    float2 ml[128];
    uint64_t full[3], empty[3], piece_full[4], piece_empty[4];
    PrefixPiece piece[4];                 // found ahead by the copying warp
    int bad[4];                           // a page that is none was met, by piece
    int abort;
};
static_assert(sizeof(PlainSmem<128>) <= 227 * 1024, "shared memory of a CTA");

__device__ __forceinline__ ulonglong2 ld2x2(const float *p) { return *reinterpret_cast<const ulonglong2 *>(p); }
__device__ __forceinline__ float4 ld4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
// Float offset of 16-byte chunk c of row r of a tile, of the queries.
__device__ __forceinline__ int tile_at(int r, int c) { return (c >> 3) * (kPrefixTile * 32) + r * 32 + (((c ^ r) & 7) << 2); }
template <int D> __device__ __forceinline__ int query_at(int r, int c) { return r * D + ((c ^ (r & 7)) << 2); }
__device__ __forceinline__ void bar_plain() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kPlainWarps) : "memory"); }

// Whether x holds in all threads that compute; also their barrier.
__device__ __forceinline__ bool all_plain(bool x)
{
    int r;
    asm volatile("{.reg .pred p, q; setp.ne.b32 p, %1, 0; barrier.cta.red.and.pred q, 1, %2, p; selp.b32 %0, 1, 0, q;}"
                 : "=r"(r)
                 : "r"((int)x), "n"(32 * kPlainWarps)
                 : "memory");
    return r != 0;
}

template <int D, int WR, int RW>
__device__ __forceinline__ void plain_piece(const PrefixArgs &a, const PrefixPiece &pc, int piece, PlainSmem<D> &sm, int &slot, bool &ok)
{
    constexpr int WK = 8 / WR, E = D / 32, KEYS = kPrefixTile / WK;  // keys of a tile that a warp takes
    constexpr int RPL = RW / 4, KPL = KEYS / 8;                      // rows and keys of a lane
    constexpr int PASSES = RW > 8 ? 2 : 1, RH = RW / PASSES;         // the warps' outputs meet in 64 rows of shared memory
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, rw = wid % WR, kg = wid / WR, kl = (lane >> 1 & 3) | (lane >> 4 & 1) << 2, rl = (lane & 1) | (lane >> 3 & 1) << 1;
    const int nrows = pc.nseq * a.G;
    float *ps = sm.p + wid * RW * KEYS;  // [KEYS][RW]
    for (int i = tid; i < RW * WR * (D / 4); i += 32 * kPlainWarps) {
        const int r = i / (D / 4), c = i % (D / 4);
        *reinterpret_cast<float4 *>(sm.q + query_at<D>(r, c)) =
            r < nrows ? ld4((const float *)a.q + a.q_row(pc, r / a.G, r % a.G) * D + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    bar_plain();
    float o[RW][E], m[RPL], l[RPL];
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
        for (int e = 0; e < E; ++e) o[r][e] = 0.f;
#pragma unroll
    for (int r = 0; r < RPL; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
    }
    // (a tile that has not come is not let go either: its place would be filled again with a copy under way)
    auto landed = [&]() {
        const uint32_t bar = smem_addr(&sm.full[slot % 3]);
        if (!mbar_try_wait(bar, slot / 3 & 1)) ok &= thread_wait(bar, slot / 3 & 1, &sm.abort, a.err, kPlainPolls);
        return __all_sync(0xffffffffu, ok) != 0;
    };
    auto done = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&sm.empty[slot % 3]));
        ++slot;
    };
#pragma unroll 1
    for (int t = pc.t0; t < pc.t1; ++t) {
        const int k0 = pc.k0 + t * kPrefixTile, live = pc.end - k0, low = pc.lo - k0;  // rows of the tile that count: [low, live)
        if (!landed()) break;
        unsigned long long s2[RPL][KPL];  // (sums over even and over odd columns)
#pragma unroll
        for (int r = 0; r < RPL; ++r)
#pragma unroll
            for (int j = 0; j < KPL; ++j) s2[r][j] = 0ull;
        const int kb = kg * KEYS + kl;
        {
            const float *K = sm.ring[slot % 3] + kb * 32, *Q = sm.q + (rw * RW + rl) * D;
            const int kx = kb & 7, qx = rw * RW + rl;
#pragma unroll 1
            for (int cc = 0; cc < D / 4; cc += 8, K += kPrefixTile * 32)
#pragma unroll 4
                for (int c = 0; c < 8; ++c) {
                    ulonglong2 qv[RPL];
#pragma unroll
                    for (int r = 0; r < RPL; ++r) qv[r] = ld2x2(Q + 4 * r * D + (((cc + c) ^ ((qx + 4 * r) & 7)) << 2));
#pragma unroll
                    for (int j = 0; j < KPL; ++j) {
                        const ulonglong2 kv = ld2x2(K + 8 * j * 32 + ((c ^ kx) << 2));
#pragma unroll
                        for (int r = 0; r < RPL; ++r)
                            s2[r][j] = fma_pair(qv[r].y, kv.y, fma_pair(qv[r].x, kv.x, s2[r][j]));
                    }
                }
        }
        done();
        float s[RPL][KPL];
#pragma unroll
        for (int r = 0; r < RPL; ++r)
#pragma unroll
            for (int j = 0; j < KPL; ++j) {
                float x, y;
                unpair(s2[r][j], x, y);
                s[r][j] = x + y;
            }
        float al[RPL];
        bool any = false;
#pragma unroll
        for (int r = 0; r < RPL; ++r) {
            float mb = -INFINITY;
#pragma unroll
            for (int j = 0; j < KPL; ++j) {
                s[r][j] = kb + 8 * j < live && kb + 8 * j >= low ? s[r][j] * a.c2 : -INFINITY;
                mb = fmaxf(mb, s[r][j]);
            }
#pragma unroll
            for (int x = 0; x < 3; ++x) mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, x < 2 ? 2 << x : 16));
            const bool grow = mb > m[r] + kLazyLog2;  // lazy rescale, as in the decode's consumers
            const float mn = grow ? mb : m[r];
            al[r] = grow ? fast_exp2(m[r] - mn) : 1.f;
            l[r] *= al[r];
            m[r] = mn;
            any |= grow;
            const float base = mn == -INFINITY ? 0.f : mn;
#pragma unroll
            for (int j = 0; j < KPL; ++j) {
                s[r][j] = fast_exp2(s[r][j] - base);
                l[r] += s[r][j];
            }
        }
#pragma unroll
        for (int j = 0; j < KPL; ++j)
#pragma unroll
            for (int r = 0; r < RPL; ++r) ps[(kl + 8 * j) * RW + 4 * r + rl] = s[r][j];
        if (__any_sync(0xffffffffu, any)) {
#pragma unroll
            for (int r = 0; r < RW; ++r) {
                const float f = __shfl_sync(0xffffffffu, al[r / 4], (r & 1) | (r & 2) << 2);
#pragma unroll
                for (int e = 0; e < E; ++e) o[r][e] *= f;
            }
        }
        __syncwarp();
        if (!landed()) break;
        // a tile's products are summed before they join the output: the chain of additions into it is as long as the tiles
        unsigned long long acc[RW / 2][E];  // (of two rows)
#pragma unroll
        for (int r = 0; r < RW / 2; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) acc[r][e] = 0ull;
        const float *V = sm.ring[slot % 3] + (D == 128 ? (lane >> 3) * (kPrefixTile * 32) : (lane >> 4) * (kPrefixTile * 32));
        const int vc = D == 128 ? lane & 7 : (lane & 15) >> 1, vo = D == 128 ? 0 : 2 * (lane & 1);
        // (rows that do not count are not touched: whatever they hold, NaN times a probability of zero is not zero)
        const int ka = max(0, low - kg * KEYS), ke = min(KEYS, live - kg * KEYS);
#pragma unroll 4
        for (int k = ka; k < ke; ++k) {
            float v[E];
            const float *vr = V + (kg * KEYS + k) * 32 + (((vc ^ k) & 7) << 2) + vo;
            if constexpr (E == 4) {
                const float4 f = ld4(vr);
                v[0] = f.x;
                v[1] = f.y;
                v[2] = f.z;
                v[3] = f.w;
            } else {
                const float2 f = *reinterpret_cast<const float2 *>(vr);
                v[0] = f.x;
                v[1] = f.y;
            }
#pragma unroll
            for (int r = 0; r < RW; r += 4) {
                const ulonglong2 p = ld2x2(ps + RW * k + r);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const unsigned long long vv = pair_of(v[e], v[e]);
                    acc[r / 2][e] = fma_pair(p.x, vv, acc[r / 2][e]);
                    acc[r / 2 + 1][e] = fma_pair(p.y, vv, acc[r / 2 + 1][e]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < RW / 2; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float x, y;
                unpair(acc[r][e], x, y);
                o[2 * r][e] += x;
                o[2 * r + 1][e] += y;
            }
        done();
    }
#pragma unroll
    for (int r = 0; r < RPL; ++r)
#pragma unroll
        for (int x = 0; x < 3; ++x) l[r] += __shfl_xor_sync(0xffffffffu, l[r], x < 2 ? 2 << x : 16);
    // the key groups join through shared memory
    const bool bad = *(volatile int *)&sm.bad[piece & 3] != 0;
    if (kl == 0)
#pragma unroll
        for (int r = 0; r < RPL; ++r) sm.ml[wid * RW + 4 * r + rl] = make_float2(m[r], l[r]);
    float *os = sm.q + wid * RH * D;
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        bar_plain();  // queries and probabilities, or the outputs of the pass before, have been read
#pragma unroll
        for (int r = 0; r < RH; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) os[r * D + lane * E + e] = o[pass * RH + r][e];
        bar_plain();
        for (int i = tid; i < RH * WR * (D / 4); i += 32 * kPlainWarps) {
            const int at = i / (D / 4), c = i % (D / 4), w0 = at / RH, rh = at - w0 * RH, rr = pass * RH + rh, r = w0 * RW + rr;
            if (r >= nrows) continue;
            float M = -INFINITY, L = 0.f;
#pragma unroll
            for (int x = 0; x < WK; ++x) M = fmaxf(M, sm.ml[(w0 + x * WR) * RW + rr].x);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int x = 0; x < WK; ++x) {
                const int w = w0 + x * WR;
                const float2 y = sm.ml[w * RW + rr];
                const float f = part_factor(y.x, M);
                const float4 v = ld4(sm.q + (w * RH + rh) * D + 4 * c);
                L += y.y * f;
                acc.x += v.x * f;
                acc.y += v.y * f;
                acc.z += v.z * f;
                acc.w += v.w * f;
            }
            float *po;
            float2 *pm;
            a.partial<D>(pc, r / a.G, r % a.G, po, pm);
            *reinterpret_cast<float4 *>(po + 4 * c) = acc;
            if (c == 0) *pm = make_float2(M, bad ? -1.f : L);
        }
    }
    bar_plain();
}

template <int D>
__global__ void __launch_bounds__(kPlainThreads, 1)
    prefix_plain(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PrefixArgs a)
{
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    PlainSmem<D> &sm = *reinterpret_cast<PlainSmem<D> *>(smem_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (smem_addr(smem_raw) & 1023u) {  // swizzled tiles need it
        wait_prior_grid();
        if (threadIdx.x == 0) {
            raise_error(a.err, ERR_INTERNAL);
            a.total->stopped = 1;
        }
        return;
    }
    if (threadIdx.x == 0) {
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
        for (int i = 0; i < 3; ++i) {
            mbar_init(smem_addr(&sm.full[i]), 1);
            mbar_init(smem_addr(&sm.empty[i]), kPlainWarps);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(smem_addr(&sm.piece_full[i]), 1);
            mbar_init(smem_addr(&sm.piece_empty[i]), kPlainWarps);
        }
        sm.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_shared();
    }
    __syncthreads();
    wait_prior_grid();
    release_next_grid();  // (the join's CTAs start as this grid's end, and wait for all of it)
    bool ok = true;
    int slot = 0;
    auto await = [&](uint64_t *bar, int k) {
        if (!mbar_try_wait(smem_addr(bar), k & 1)) ok &= thread_wait(smem_addr(bar), k & 1, &sm.abort, a.err, kPlainPolls);
    };
    auto fine = [&]() { return __all_sync(0xffffffffu, ok) != 0; };
    // registers of the launch, 168 a thread, as the roles need them: 128 (56) + 256 (224)
    if (warp >= kPlainWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // ---- pieces and copies.  Lane (box, part) of a tile copies 32 columns of the box's rows: a page, or half a page of 256
        constexpr int PARTS = D / 32;
        const int rows = min(kPrefixTile, 1 << a.shift), boxes = kPrefixTile / rows;
        const int box = lane / PARTS, part = lane % PARTS;
        PrefixWalk w = a.range();
        PrefixPiece pc;
        for (int piece = 0; warp == kPlainWarps && fine(); ++piece) {
            const bool more = a.next(w, pc);
            await(&sm.piece_empty[piece & 3], piece / 4 + 1);
            if (!fine()) break;
            if (lane == 0) {
                if (!more) pc.t1 = pc.t0 = 0;
                sm.piece[piece & 3] = pc;
                sm.bad[piece & 3] = 0;
                mbar_arrive(smem_addr(&sm.piece_full[piece & 3]));
            }
            __syncwarp();
            if (!more) break;
            for (int t = pc.t0; t < pc.t1 && fine(); ++t) {
                const int k = pc.k0 + t * kPrefixTile + box * rows;
                const bool needed = box < boxes && k < pc.end;
                const long long row = needed ? a.pool_row(pc, k) : -1;
                const int n = __popc(__ballot_sync(0xffffffffu, row >= 0));
                if (__any_sync(0xffffffffu, needed && row < 0) && lane == 0) {
                    *(volatile int *)&sm.bad[piece & 3] = 1;
                    raise_error(a.err, ERR_PAGE);
                }
                for (int kv = 0; kv < 2; ++kv, ++slot) {
                    await(&sm.empty[slot % 3], slot / 3 + 1);
                    if (!fine()) break;
                    const uint32_t full = smem_addr(&sm.full[slot % 3]);
                    if (lane == 0) mbar_expect_tx(full, (uint32_t)(n * rows * 128));
                    __syncwarp();
                    if (row >= 0)
                        tma_load_2d(smem_addr(sm.ring[slot % 3]) + part * (kPrefixTile * 128) + box * rows * 128, kv ? &tmV : &tmK, 32 * part,
                                    (int)row, full);
                    __syncwarp();
                }
            }
        }
        // no copy is left in flight when the CTA ends
        for (int j = max(0, slot - 3); j < slot; ++j) mbar_wait_bounded(smem_addr(&sm.full[j % 3]), j / 3 & 1, kPlainPolls);
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        // ---- attention
        for (int piece = 0;; ++piece) {
            await(&sm.piece_full[piece & 3], piece / 4);
            __syncwarp();
            const PrefixPiece pc = sm.piece[piece & 3];
            if (!all_plain(ok) || pc.t0 == pc.t1) break;
            const int nrows = pc.nseq * a.G;
            if (nrows <= 8)
                plain_piece<D, 1, 8>(a, pc, piece, sm, slot, ok);
            else if (nrows <= 16)
                plain_piece<D, 2, 8>(a, pc, piece, sm, slot, ok);
            else if (nrows <= 24)
                plain_piece<D, 2, 12>(a, pc, piece, sm, slot, ok);
            else
                plain_piece<D, 2, 16>(a, pc, piece, sm, slot, ok);
            if (lane == 0) mbar_arrive(smem_addr(&sm.piece_empty[piece & 3]));
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && *(volatile int *)&sm.abort != 0) a.total->stopped = 1;
}

// ---------------------------------------------------------------- join
// One CTA per unit.  The partials of a query head: the own rows' first one, their others by CTA, and the same of the
// prefix.  A warp finds a head's factors; then a thread adds up four columns of a head over an equal part of the partials.
// Where units are many, own rows that are few (at the start of an answer) are one more part, taken here with plain FMAs: as
// an item of the attention they cost 2 us and more of a CTA that holds an SM, here several units share one.  Few units
// would rather have the attention take them beside the prefixes than the join behind it.  (28 query and 4 key heads, up to
// 32 own rows behind 1000: 128 units 28 us without, 34 with, 320 units 32 and 35, 640 units 47 and 40, 896 units 61 and 49,
// 2560 units 144 and 96, 4992 units 245 and 172; where half of the units have 300 own rows, 36 and 38 with 320 units, 55
// either way with 640, 78 and 73 with 896.)
struct JoinArgs {
    PrefixArgs p;
    int32_t *lens;
    void *out;
    float *lse;  // or nullptr
    int grid, append, out_bf16;
};
constexpr int kJoinThreads = 256;

template <int D, bool FEW> __global__ void __launch_bounds__(kJoinThreads) prefix_join(const __grid_constant__ JoinArgs a)
{
    constexpr int Q = D / 4;
    extern __shared__ float sm_f[];  // [G][np] factors
    __shared__ float2 sm_ML[16];
    __shared__ float sm_p[16][kPrefixJoinRows], sm_fo[16];
    __shared__ int sm_row[kPrefixJoinRows];
    __shared__ __align__(16) float4 sm_o[kJoinThreads];
    wait_prior_grid();  // (the plan's lists too: what earlier grids wrote is sure to be seen only behind this grid's own wait)
    const int u = blockIdx.x, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int h = u % a.p.Hkv, lb = u / a.p.Hkv, layer = lb / a.p.B, b = lb - layer * a.p.B, G = a.p.G;
    const int run = a.p.run_of[b];
    const PrefixUnit x = a.p.units[u];
    const PrefixTotal total = *a.p.total;
    const size_t q0 = (size_t)lb * a.p.Hq + (size_t)h * G;
    const bool ok = x.lo >= 0 && run != -2 && total.stopped == 0;
    // partials: [0, n_own) of the own rows, then n_pre of the prefix; CTAs of the first ones
    int n_own = 0, n_pre = 0, own_c = 0, pre_c = 0, pre_row = 0;
    if (ok) {
        const long long pre = total.work * a.p.layers * a.p.Hkv;
        const long long all = pre + a.p.own_total();
        const PrefixShare share(all, a.grid, total.most);
        auto ctas = [&](long long w0, int tiles, int unit, int &c) {
            c = share.cta(w0);
            return 1 + share.cta(w0 + (long long)(tiles - 1) * unit) - c;
        };
        if (x.n - x.lo > a.p.rows.few) {
            long long w0 = pre + x.work + a.p.rows.extra();
            for (int i = 0; i < u / kPrefixBlock; ++i) w0 += __ldg(a.p.block_work + i);
            n_own = ctas(w0, (x.n - x.k0 + kPrefixTile - 1) / kPrefixTile, a.p.rows.own(), own_c);
        }
        if (run >= 0) {
            const PrefixRun rn = a.p.runs[run];
            const PrefixRows rows = a.p.rows;
            const int i = b - rn.b0, rt = i / rows.per, kt = (rn.p + kPrefixTile - 1) / kPrefixTile;
            n_pre = ctas(((long long)layer * a.p.Hkv + h) * total.work + rn.work + (long long)rt * kt * rows.unit(rn.n, 0), kt,
                         rows.unit(rn.n, rt), pre_c);
            pre_row = (i - rt * rows.per) * G;
        }
    }
    // ---- few own rows: logits, then probabilities in sm_p (a warp's heads are those that it joins below)
    const int few = FEW && ok && x.n > x.lo && x.n - x.lo <= a.p.rows.few ? x.n - x.lo : 0;
    bool err = !ok;
    auto four = [&](const void *base, size_t at, int n, float (&v)[4]) {  // n = 2 or 4 elements
        if (a.p.rows.f32) {
            const float *f = (const float *)base + at;
            if (n == 4) {
                const float4 y = *reinterpret_cast<const float4 *>(f);
                v[0] = y.x, v[1] = y.y, v[2] = y.z, v[3] = y.w;
            } else {
                const float2 y = *reinterpret_cast<const float2 *>(f);
                v[0] = y.x, v[1] = y.y;
            }
        } else {
            const uint32_t *f = reinterpret_cast<const uint32_t *>((const __nv_bfloat16 *)base + at);
#pragma unroll
            for (int i = 0; i < 4; i += 2)
                if (i < n) {
                    const uint32_t y = f[i / 2];
                    v[i] = __uint_as_float(y << 16);
                    v[i + 1] = __uint_as_float(y & 0xffff0000u);
                }
        }
    };
    float2 own_ml[2];  // of heads wid and wid + 8
    if (few > 0) {
        constexpr int E = D / 32, R = kPrefixJoinRows * 32 / kJoinThreads;  // elements of a lane, rows of a warp
        PrefixPiece pc = {};
        pc.layer = layer;
        pc.h = h;
        pc.b0 = b;
        float k[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int j = wid + kJoinThreads / 32 * i;
            const long long row = j < few ? a.p.pool_row(pc, x.lo + j) : 0;
            if (row < 0 && lane == 0) raise_error(a.p.err, ERR_PAGE);
            err |= row < 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) k[i][e] = 0.f;
            if (j < few && row >= 0) four(a.p.K, (size_t)row * D + lane * E, E, k[i]);
            if (j < few && lane == 0) sm_row[j] = row < 0 ? 0 : (int)row;
        }
        for (int g = 0; g < G; ++g) {
            float q[4];
            four(a.p.q, (q0 + g) * D + lane * E, E, q);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                float dot = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) dot = fmaf(q[e], k[i][e], dot);
                dot = warp_sum(dot);
                if (lane == 0) sm_p[g][wid + kJoinThreads / 32 * i] = dot * a.p.c2;
            }
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int g = wid + t * (kJoinThreads / 32);
            if (g >= G) break;
            const float s = lane < few ? sm_p[g][lane] : -INFINITY, M = warp_max(s);
            const float p = fast_exp2(s - (M == -INFINITY ? 0.f : M));
            sm_p[g][lane] = p;
            own_ml[t] = make_float2(M, warp_sum(p));
        }
    }
    const int np = n_own + n_pre;
    auto place = [&](int i, int g, const float *&o, const float2 *&ml) {
        const bool own = i < n_own;
        const int k = own ? i : i - n_own;
        const size_t at = k == 0 ? q0 + g : (size_t)((own ? own_c : pre_c) + k) * a.p.cont_rows + (own ? 0 : pre_row) + g;
        o = (k > 0 ? a.p.cont_o : (own ? a.p.own_o : a.p.part_o)) + at * D;
        ml = (k > 0 ? a.p.cont_ml : (own ? a.p.own_ml : a.p.part_ml)) + at;
    };
    const float *po;
    const float2 *pm;
    for (int g = wid; g < G; g += kJoinThreads / 32) {
        const float2 own = g < kJoinThreads / 32 ? own_ml[0] : own_ml[1];
        float M = few > 0 ? own.x : -INFINITY, L = 0.f;
        for (int i = lane; i < np; i += 32) {
            place(i, g, po, pm);
            M = fmaxf(M, pm->x);
        }
        M = warp_max(M);
        for (int i = lane; i < np; i += 32) {
            place(i, g, po, pm);
            const float2 y = *pm;
            const float f = part_factor(y.x, M);
            err |= y.y < 0.f;
            L += y.y * f;
            sm_f[g * np + i] = f;
        }
        L = warp_sum(L);
        const float fo = few > 0 ? part_factor(own.x, M) : 0.f;
        if (few > 0) L += own.y * fo;
        if (lane == 0) {
            sm_ML[g] = make_float2(M, L);
            sm_fo[g] = fo;
        }
    }
    err = __syncthreads_or(err);
    // threads: (part, head, four columns)
    const int slots = G * Q, parts = max(1, kJoinThreads / slots), part = tid / slots;
    auto sum = [&](int s) {  // of head and columns s, over the rows and partials of this thread's part
        const int g = s / Q, c = s - g * Q;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int j = part; j < few; j += parts) {
            float v[4];
            four(a.p.V, (size_t)sm_row[j] * D + 4 * c, 4, v);
            const float p = sm_p[g][j];
            o.x = fmaf(p, v[0], o.x);
            o.y = fmaf(p, v[1], o.y);
            o.z = fmaf(p, v[2], o.z);
            o.w = fmaf(p, v[3], o.w);
        }
        if (few > 0) {
            const float f = sm_fo[g];
            o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
        }
#pragma unroll 4
        for (int i = part; i < np; i += parts) {
            place(i, g, po, pm);
            const float4 v = *reinterpret_cast<const float4 *>(po + 4 * c);
            const float f = sm_f[g * np + i];
            o.x += v.x * f;
            o.y += v.y * f;
            o.z += v.z * f;
            o.w += v.w * f;
        }
        return o;
    };
    auto store = [&](int s, float4 o) {
        const int g = s / Q, c = s - g * Q;
        const float2 ML = sm_ML[g];
        const float L = err ? 0.f : ML.y, inv = sum_inverse(L);
        if (err) o = make_float4(0.f, 0.f, 0.f, 0.f);
        const float4 v = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        if (a.out_bf16)
            *reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(a.out) + (q0 + g) * D + 4 * c) =
                make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
        else
            *reinterpret_cast<float4 *>(reinterpret_cast<float *>(a.out) + (q0 + g) * D + 4 * c) = v;
        if (c == 0 && a.lse) a.lse[q0 + g] = sum_log2(ML.x, L) * kLn2;
    };
    if (parts > 1) {  // one turn; threads behind the last part (16, with d 64 and 3 or 5 heads) meet the barrier with the others
        if (part < parts) sm_o[tid] = sum(tid - part * slots);
        __syncthreads();
        if (part == 0) {
            float4 o = sm_o[tid];
            for (int k = 1; k < parts; ++k) {
                const float4 v = sm_o[k * slots + tid];
                o.x += v.x;
                o.y += v.y;
                o.z += v.z;
                o.w += v.w;
            }
            store(tid, o);
        }
    } else {
        for (int s = tid; s < slots; s += kJoinThreads) store(s, sum(s));
    }
    if (tid == 0 && a.append && !err) a.lens[u] = x.n;
}

// ---------------------------------------------------------------- host side
static int prefix_cont_rows(const reco_paged_kv &kv)
{
    return (int)std::min<long long>(kPrefixMaxRows, (long long)kv.B * (kv.H_q / kv.H_kv));
}

static PrefixRows prefix_rows(const reco_paged_kv &kv)
{
    const int G = kv.H_q / kv.H_kv, few = (long long)kv.n_layers * kv.B * kv.H_kv > 600 ? kPrefixJoinRows : 0;
    return kv.dtype == RECO_F32 ? PrefixRows{kPlainRows / G, kPlainRows / G, G, 1, few} : PrefixRows{2 * (128 / G), 128 / G, G, 0, few};
}

long long prefix_own_most(const reco_paged_kv &kv)
{
    const long long tiles = ((long long)paged_cap(kv) + kPrefixTile - 1) / kPrefixTile + 1;  // (the first may begin before the own rows)
    return (long long)kv.n_layers * kv.B * kv.H_kv * (tiles * prefix_rows(kv).own() + prefix_rows(kv).extra());
}

PrefixWs prefix_ws_layout(const reco_paged_kv &kv, void *base)
{
    size_t off = kPagedZeroBytes;
    auto take = [&](size_t bytes) {
        char *r = base ? (char *)base + off : nullptr;
        off += align256(bytes);
        return r;
    };
    const size_t heads = (size_t)kv.n_layers * kv.B * kv.H_q, units = (size_t)kv.n_layers * kv.B * kv.H_kv;
    const size_t rows = (size_t)prefix_cont_rows(kv) * kPagedMaxGrid;
    PrefixWs ws;
    ws.run_of = (int32_t *)take((size_t)kv.B * 4);
    ws.runs = (PrefixRun *)take(((size_t)kv.B / 2 + 1) * sizeof(PrefixRun));
    ws.total = (PrefixTotal *)take(sizeof(PrefixTotal));
    ws.units = (PrefixUnit *)take(units * sizeof(PrefixUnit));
    ws.block_work = (int32_t *)take((units + kPrefixBlock - 1) / kPrefixBlock * 4);
    ws.own_o = (float *)take(heads * kv.d * 4);
    ws.own_ml = (float2 *)take(heads * 8);
    ws.part_o = (float *)take(heads * kv.d * 4);
    ws.part_ml = (float2 *)take(heads * 8);
    ws.cont_o = (float *)take(rows * kv.d * 4);
    ws.cont_ml = (float2 *)take(rows * 8);
    ws.bytes = off;
    return ws;
}

cudaError_t launch_paged_prefix(const reco_paged_kv &kv, const void *q, const void *k_new, const void *v_new, int32_t *lens,
                                const int32_t *group, const int32_t *shared, float scale, void *out, reco_dtype out_dtype,
                                float *lse, const PrefixWs &ws, unsigned *err, cudaStream_t s)
{
    const bool f32 = kv.dtype == RECO_F32;
    const int units = kv.n_layers * kv.B * kv.H_kv, G = kv.H_q / kv.H_kv, blocks = (units + kPrefixBlock - 1) / kPrefixBlock;
    PrefixRows rows = prefix_rows(kv);
    if (!f32 && out_dtype == RECO_F32) rows.per = rows.half;  // (one stream of products)
    PlanArgs p = {};
    p.K = kv.k;
    p.V = kv.v;
    p.k_new = k_new;
    p.v_new = v_new;
    p.table = kv.table;
    p.lens = lens;
    p.group = group;
    p.shared = shared;
    p.units = units;
    p.B = kv.B;
    p.Hkv = kv.H_kv;
    p.cap = paged_cap(kv);
    p.n_pages = kv.n_pages;
    p.max_pages = kv.max_pages;
    p.shift = __builtin_ctz((unsigned)kv.page);
    p.row_bytes = kv.d * (f32 ? 4 : 2);
    p.rows = rows;
    p.ws = ws;
    p.err = err;
    const long long copies = k_new ? ((long long)units * 2 * (p.row_bytes / 16) + kPrefixBlock - 1) / kPrefixBlock : 0;
    cudaError_t e = launch_pdl(prefix_plan, dim3((unsigned)(1 + blocks + copies)), dim3(kPrefixBlock), 0, s, p);
    if (e != cudaSuccess) return e;
    PrefixArgs a = {};
    a.K = kv.k;
    a.V = kv.v;
    a.q = q;
    a.table = kv.table;
    a.runs = ws.runs;
    a.run_of = ws.run_of;
    a.total = ws.total;
    a.units = ws.units;
    a.block_work = ws.block_work;
    a.part_o = ws.part_o;
    a.part_ml = ws.part_ml;
    a.own_o = ws.own_o;
    a.own_ml = ws.own_ml;
    a.cont_o = ws.cont_o;
    a.cont_ml = ws.cont_ml;
    a.layers = kv.n_layers;
    a.B = kv.B;
    a.Hq = kv.H_q;
    a.Hkv = kv.H_kv;
    a.G = G;
    a.n_pages = kv.n_pages;
    a.max_pages = kv.max_pages;
    a.shift = p.shift;
    a.n_units = units;
    a.n_blocks = blocks;
    a.rows = rows;
    a.cont_rows = prefix_cont_rows(kv);
    a.c2 = scale * kLog2e;
    a.err = err;
    const int grid = std::min(device_sm_count(), kPagedMaxGrid);
    if (f32) {
        CUtensorMap mk = {}, mv = {};
        const unsigned long long pool = (unsigned long long)kv.n_layers * kv.n_pages * kv.H_kv * kv.page;
        const int box = std::min(kPrefixTile, kv.page);
        if (!encode_f32_2d(&mk, kv.k, pool, kv.d, 32, box) || !encode_f32_2d(&mv, kv.v, pool, kv.d, 32, box)) return cudaErrorInvalidValue;
        void (*fn)(CUtensorMap, CUtensorMap, PrefixArgs) = kv.d == 64 ? prefix_plain<64> : prefix_plain<128>;
        const int smem = kv.d == 64 ? (int)sizeof(PlainSmem<64>) : (int)sizeof(PlainSmem<128>);
        if ((e = allow_smem((const void *)fn, smem)) != cudaSuccess) return e;
        if ((e = launch_pdl(fn, dim3(grid), dim3(kPlainThreads), smem, s, mk, mv, a)) != cudaSuccess) return e;
    } else {
        if ((e = launch_prefix_tc(kv, a, grid, out_dtype, s)) != cudaSuccess) return e;
    }
    JoinArgs j = {};
    j.p = a;
    j.lens = lens;
    j.out = out;
    j.lse = lse;
    j.grid = grid;
    j.append = k_new ? 1 : 0;
    j.out_bf16 = out_dtype == RECO_BF16 ? 1 : 0;
    void (*join)(JoinArgs) = rows.few ? (kv.d == 64 ? prefix_join<64, true> : prefix_join<128, true>)
                                      : (kv.d == 64 ? prefix_join<64, false> : prefix_join<128, false>);
    e = launch_pdl(join, dim3(units), dim3(kJoinThreads), (size_t)G * (2 * grid + 2) * 4, s, j);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace reco
