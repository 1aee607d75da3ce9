// evict.cu -- eviction of a paged cache down to a budget by accumulated attention weight (the selection
// and in-place compaction of Sec. 3.2 with running sums in place of Eq. 2's scores).
//
// The selection (select.cu) writes every cut unit's kept rows in ascending order, compacts the weights and
// lists the units and their chunks.  kept[r] >= r, so a destination row is the source of rows at or below it
// only, and the rows can move in place.  With many cut units a CTA walks a column of a unit in order
// (compact_columns).  With few, their chunks of 16 KB of K and 16 KB of V move in parallel (compact_chunks: 32
// units of 3900 rows 69 -> 32 us): a CTA reads its chunk's rows into registers, says so in the chunk's flag, and
// writes them once the chunks have been read whose sources lie in its destination rows.  Those are known from the
// kept rows counted before the chunk's first row and its end (`rank`): no more than a chunk has, so two chunks at
// most.  CTAs claim chunks in the order of the list, a unit's own in ascending order, each the next one before the
// present one is done.  Every wait ends: the first unread chunk of the list is some CTA's present one, which it reads at
// once, or the next one of a CTA whose present chunk lies further up the list, has been read, and waits only for chunks
// above itself, all read.  (A wait that runs out all the same reports it, and the chunk's rows are not written: they
// could lie over rows that nobody has read.)  The chunks would do for many units too, but slower: 896 units cut to
// 3900 rows 881 us (each chunk's chain of index, table, row and flag), by columns 581, 0.91 of the copy rate.
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace reco {

EvictWs evict_ws_layout(const reco_paged_kv &kv, void *base)
{
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char *r = base ? (char *)base + off : nullptr;
        off += align256(bytes);
        return r;
    };
    const size_t units = (size_t)kv.n_layers * kv.B * kv.H_kv, chunks = evict_chunks(kv);
    EvictWs ws;
    ws.counters = (int32_t *)take(kPagedZeroBytes);  // (16 bytes of them)
    ws.idx = (int32_t *)take(units * paged_cap(kv) * 4);
    ws.rank = (int32_t *)take(units * (chunks + 1) * 4);
    ws.flags = (int32_t *)take(units * chunks * 4);
    ws.list = (int4 *)take(units * chunks * 16);
    ws.ulist = (int32_t *)take(units * 4);
    ws.bytes = off;
    return ws;
}

struct CompactArgs {
    char *K, *V;
    const int32_t *table, *idx, *lens;
    EvictWs ws;
    int units, B, Hkv, n_pages, max_pages, page_shift, page_mask, pitch, cap, chunks;  // pitch: pool rows from page to page
    int column_ctas;  // CTAs of compact_columns, 0: not launched
    unsigned *err;
};

constexpr int kCompactThreads = 256;
constexpr long long kFlagSpin = 1LL << 22;  // polls of a chunk's flag (about a second)

__device__ __forceinline__ int ld_acquire(const int *p)
{
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void st_release(int *p, int v)
{
    asm volatile("st.release.gpu.global.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}

// 16 bytes that are read once (streamed past what L2 holds), before the barrier behind which they may be written over.
__device__ __forceinline__ uint4 ld_once(const char *p)
{
    uint4 v;
    asm volatile("ld.global.cs.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// Where the rows of a unit lie.  The selection has checked the table entries of all its rows; an entry is
// held inside the pool all the same, and a kept row inside the cache, so that a workspace or an index array that
// something else has written to costs no access out of bounds.
struct UnitRows {
    const int32_t *table;
    int base;  // pool row of the unit's row 0 in page 0
    __device__ __forceinline__ UnitRows(const CompactArgs &a, int u)
    {
        const int lb = u / a.Hkv, layer = lb / a.B;
        table = a.table + (long)(lb - layer * a.B) * a.max_pages;
        base = layer * a.n_pages * a.pitch + ((u - lb * a.Hkv) << a.page_shift);
    }
    template <int ROW> __device__ __forceinline__ size_t at(const CompactArgs &a, int r) const  // byte of row r in the pool
    {
        const int e = (int)min((unsigned)__ldg(table + (r >> a.page_shift)), (unsigned)a.n_pages - 1u);
        return (size_t)(unsigned)(base + e * a.pitch + (r & a.page_mask)) * ROW;
    }
};

// Many cut units: a CTA moves a unit's 128-byte column slice of K or of V, its destinations in order in steps of
// 32 U rows, U rows per thread: a step's reads, a barrier, its writes, with the next step's reads issued before this
// one's writes (two steps in registers).  kept[r] >= r, so no source is a row that an earlier step has written.
template <int ROW> __device__ __forceinline__ void compact_column(const CompactArgs &a, int u, bool is_v, int slice)
{
    constexpr int U = 2, RPP = kCompactThreads / 8, STEP = U * RPP;
    const UnitRows rows(a, u);
    const int m = min(a.lens[u], a.cap), sub = threadIdx.x / 8;
    const int32_t *idx = a.idx + (size_t)u * a.cap;
    char *pool = (is_v ? a.V : a.K) + slice * 128 + (threadIdx.x % 8) * 16;
    auto load = [&](int r0, uint4 (&v)[U]) {  // which of the thread's rows move, a bit each
        unsigned moves = 0;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int r = r0 + i * RPP + sub;
            if (r < m) {
                const int src = __ldg(idx + r);
                if (src > r && src < a.cap) {  // else already in place
                    v[i] = *reinterpret_cast<const uint4 *>(pool + rows.at<ROW>(a, src));
                    moves |= 1u << i;
                }
            }
        }
        return moves;
    };
    auto store = [&](int r0, const uint4 (&v)[U], unsigned moves) {
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (moves & (1u << i)) *reinterpret_cast<uint4 *>(pool + rows.at<ROW>(a, r0 + i * RPP + sub)) = v[i];
    };
    uint4 va[U], vb[U];
    unsigned ma = load(0, va);
    for (int r0 = 0; r0 < m; r0 += 2 * STEP) {
        const unsigned mb = load(r0 + STEP, vb);
        __syncthreads();
        store(r0, va, ma);
        if (r0 + STEP >= m) break;
        ma = load(r0 + 2 * STEP, va);
        __syncthreads();
        store(r0 + STEP, vb, mb);
    }
}

// Few cut units: a chunk of a unit, 16 KB of K and 16 KB of V, four pieces of 16 bytes of each per thread.
template <int ROW> struct Chunk {
    static constexpr int PIECES = ROW / 16, RPP = kCompactThreads / PIECES, U = 4, R = RPP * U;
    int u, c;     // unit and chunk
    int src[U];   // the rows that move to this thread's rows (those rows themselves: nothing moves)

    __device__ __forceinline__ int row(int i) const { return c * R + i * RPP + (int)threadIdx.x / PIECES; }

    // entry t of the list
    __device__ __forceinline__ void find(const CompactArgs &a, int t)
    {
        const int4 it = __ldg(a.ws.list + t);  // (unit, chunk, kept rows)
        const bool ok = (unsigned)it.x < (unsigned)a.units && (unsigned)it.y < (unsigned)a.chunks;
        if (!ok && threadIdx.x == 0) raise_error(a.err, ERR_INTERNAL);
        u = ok ? it.x : 0;
        c = ok ? it.y : 0;
        const int m = ok ? min(it.z, a.cap) : 0;
        const int32_t *idx = a.idx + (size_t)u * a.cap;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int r = row(i), s = r < m ? __ldg(idx + r) : r;
            src[i] = s < r || s >= a.cap ? r : s;
        }
    }
};

// Whether the columns of the cut units keep most of the `ctas` of compact_columns busy: then they move, and
// else the chunks.
__device__ __forceinline__ bool by_columns(const CompactArgs &a, int columns)
{
    return a.column_ctas > 0 && 4LL * columns >= 3LL * a.column_ctas;
}

template <int ROW> __global__ void __launch_bounds__(kCompactThreads, 8) compact_columns(CompactArgs a)
{
    wait_prior_grid();  // the selection's results
    const int cut = min(a.ws.counters[3], a.units);
    if (!by_columns(a, cut * 2 * (ROW / 128))) return;
    for (int i = blockIdx.x; i < cut; i += gridDim.x) {
        const int u = a.ws.ulist[i];
        if ((unsigned)u >= (unsigned)a.units) continue;
        compact_column<ROW>(a, u, blockIdx.y != 0, blockIdx.z);
        __syncthreads();
    }
}

template <int ROW> __global__ void __launch_bounds__(kCompactThreads, 4) compact_chunks(CompactArgs a)
{
    constexpr int U = Chunk<ROW>::U, R = Chunk<ROW>::R;
    __shared__ int sm_next;
    wait_prior_grid();  // the selection's results
    const int columns = min(a.ws.counters[3], a.units) * 2 * (ROW / 128);
    const int chunks = min(a.ws.counters[1], a.units * a.chunks);
    const int total = by_columns(a, columns) ? 0 : chunks;
    const int off = (threadIdx.x % Chunk<ROW>::PIECES) * 16;
    if (threadIdx.x == 0) sm_next = total > 0 ? atomicAdd(&a.ws.counters[0], 1) : 0;
    __syncthreads();
    int t = sm_next;
    Chunk<ROW> cur, nxt;
    if (t < total) cur.find(a, t);
    while (t < total) {
        int claimed = 0;
        if (threadIdx.x == 0) claimed = atomicAdd(&a.ws.counters[0], 1);  // the next chunk, while this one moves
        const UnitRows rows(a, cur.u);
        uint4 k[U], v[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (cur.src[i] == cur.row(i)) continue;  // already in place, or behind the last row
            const size_t p = rows.at<ROW>(a, cur.src[i]) + off;
            k[i] = ld_once(a.K + p);
            v[i] = ld_once(a.V + p);
        }
        if (threadIdx.x == 0) sm_next = claimed;
        __syncthreads();  // the chunk has been read
        t = sm_next;
        if (t < total) nxt.find(a, t);  // its rows are looked up while this chunk waits for its turn
        bool late = false;
        if (threadIdx.x == 0) {
            int *flags = a.ws.flags + (size_t)cur.u * a.chunks;
            st_release(flags + cur.c, 1);
            // kept rows in this chunk's destination rows: their destinations' chunks have to have been read
            const int32_t *rank = a.ws.rank + (size_t)cur.u * (a.chunks + 1);
            const int lo = max(0, __ldg(rank + cur.c)), hi = __ldg(rank + cur.c + 1);
            for (int b = lo / R; b < cur.c && b * R < hi && !late; ++b) {
                long long spin = 0;
                while (ld_acquire(flags + b) == 0 && spin < kFlagSpin) ++spin;
                late = spin >= kFlagSpin;
            }
            if (late) raise_error(a.err, ERR_INTERNAL);
        }
        late = __syncthreads_or(late);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int r = cur.row(i);
            if (late || cur.src[i] == r) continue;
            const size_t p = rows.at<ROW>(a, r) + off;
            *reinterpret_cast<uint4 *>(a.K + p) = k[i];
            *reinterpret_cast<uint4 *>(a.V + p) = v[i];
        }
        cur = nxt;
    }
    // the last CTA to finish leaves the counters zero, as the call found them
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(&a.ws.counters[2], 1) == (int)gridDim.x - 1)
            *reinterpret_cast<int4 *>(a.ws.counters) = make_int4(0, 0, 0, 0);
    }
}

cudaError_t launch_paged_evict(const reco_paged_kv &kv, float *weights, int32_t *lens, const int32_t *budget, int w,
                               int sinks, int32_t *kept_idx, const EvictWs &ws, unsigned *err, cudaStream_t s)
{
    int32_t *idx = kept_idx ? kept_idx : ws.idx;
    cudaError_t e = launch_select_budget(kv, weights, lens, budget, w, sinks, idx, ws, err, s);
    if (e != cudaSuccess) return e;
    const int units = kv.n_layers * kv.B * kv.H_kv;
    const int row = kv.d * (kv.dtype == RECO_F32 ? 4 : 2), sms = device_sm_count();
    const long long columns = (long long)units * 2 * (row / 128);
    CompactArgs a{(char *)kv.k, (char *)kv.v, kv.table, idx, lens, ws, units, kv.B, kv.H_kv, kv.n_pages, kv.max_pages,
                  __builtin_ctz((unsigned)kv.page), kv.page - 1, kv.H_kv * kv.page, paged_cap(kv), evict_chunks(kv), 0, err};
    if (4 * columns >= 3LL * 8 * sms) {  // (else not even all units' columns would do)
        a.column_ctas = 8 * sms;
        e = launch_pdl(row == 128 ? compact_columns<128> : (row == 256 ? compact_columns<256> : compact_columns<512>),
                       dim3(a.column_ctas / (2 * (row / 128)), 2, row / 128), dim3(kCompactThreads), 0, s, a);
        if (e != cudaSuccess) return e;
    }
    const dim3 grid((unsigned)std::min<long long>((long long)units * a.chunks, 4LL * sms));
    e = launch_pdl(row == 128 ? compact_chunks<128> : (row == 256 ? compact_chunks<256> : compact_chunks<512>), grid,
                   dim3(kCompactThreads), 0, s, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace reco
