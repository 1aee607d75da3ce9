// prefix.cuh -- what the kernels of decode attention over shared prefixes (prefix.cu) have in common: the work, a
// CTA's walk over its share of it, and where partials go.
#pragma once
#include "common.cuh"
#include "internal.h"

namespace reco {

// A row tile takes the query heads of up to `per` sequences of a group, of which `half` make what the tensor cores take
// at once (128 rows).  Work is counted in units of about 0.2 us of a CTA, measured with all of them busy.  bf16: a key tile
// takes 8 where its bytes come from HBM (1.45 us) and a stream has half of its keys, 12 where the row tile has more than `half`
// sequences (each stream all keys: products and softmax are the bound), 6 for a last row tile of no more, whose bytes the
// others have brought (64 sequences of 5 heads over 100001 rows, two row tiles: 199 us with 12 and 6, 204 with 9 and 5, 209 with
// 9 and 6, 221 with 9 and 7, 217 with 13 and 7).  With float32 output (one stream) row tiles of a group cost the same.  float32 (twice the bytes, plain FMAs): 15 with 8 rows (5300 cycles), 24 with 16 (8300), 33 with
// 24, 40 with 32 (14300).  The start and the end of a unit's own rows take extra() more.
struct PrefixRows {
    int per, half, G, f32;
    int few;  // so many own rows at most are left to the join
    __host__ __device__ int plain(int n) const { return n * G <= 8 ? 15 : (n * G <= 16 ? 24 : (n * G <= 24 ? 33 : 40)); }
    // a key tile's of row tile rt of n sequences (all but the last row tile have the first one's), of a unit's own rows
    __host__ __device__ int unit(int n, int rt) const
    {
        if (f32) return plain(n - rt * per < per ? n - rt * per : per);
        if (per == half) return n <= per ? 8 : 9;
        return n - rt * per > half ? 12 : (n <= per ? 8 : 6);
    }
    __host__ __device__ int extra() const { return f32 ? 5 : 11; }
    __host__ __device__ int own() const { return f32 ? plain(1) : 8; }
    // a group's of n sequences with p rows, per layer and KV head
    __host__ __device__ long long work(int n, int p) const
    {
        const int last = (n - 1) / per, kt = (p + kPrefixTile - 1) / kPrefixTile;
        return (long long)kt * ((long long)last * unit(n, 0) + unit(n, last));
    }
};

#ifdef __CUDACC__
// (64-bit divisions take some hundred instructions: most are of 32-bit numbers)
__device__ __noinline__ static long long quotient(long long a, long long b)
{
    return ((unsigned long long)a | (unsigned long long)b) >> 32 ? a / b : (long long)((unsigned)a / (unsigned)b);
}
// How the work is shared out to the CTAs: evenly, or, where that left less than a key tile's to each, a tile's (`most`).
// A key tile whose work is cut goes to the CTA that its first unit falls to: tile t of an item whose tiles begin at w0,
// `unit` to each, to that of w0 + t * unit.  (Every CTA between an item's first and last then has one of its tiles.)
struct PrefixShare {
    long long total;
    int n, most;  // CTAs with work; 0: evenly
    __device__ __forceinline__ PrefixShare(long long all, int grid, int most_unit) : total(all)
    {
        const bool few = all <= (long long)grid * most_unit;
        most = few ? most_unit : 0;
        n = few ? ((int)all + most_unit - 1) / most_unit : grid;
    }
    __device__ __forceinline__ long long begin(int c) const { return most ? min(total, (long long)c * most) : quotient(total * c, n); }
    __device__ __forceinline__ int cta(long long w) const { return most ? (int)w / most : (int)quotient((w + 1) * n - 1, total); }
};

// The last i of [0, n) with key(i) <= x, by a warp (key does not decrease, key(0) <= x).
template <typename F> __device__ __forceinline__ int warp_last(int n, long long x, F key)
{
    const int lane = threadIdx.x & 31;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 31) / 32, at = lane * step;
        const bool le = at < n && (lane == 0 || key(lo + at) <= x);
        const int k = 31 - __clz(__ballot_sync(0xffffffffu, le));
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

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

// A CTA's part of an item: a row tile (nseq sequences from s0 on of the group that begins at sequence b0) against key
// tiles [t0, t1) of the rows [lo, end), looked up in b0's table; tile t begins at row k0 + 128 t.
struct PrefixPiece {
    int layer, h, b0, s0, nseq, k0, lo, end, t0, t1;
    bool own;
};
// The work of the prefixes of all layers and heads lies before that of the units' own rows.
struct PrefixWalk {
    long long w, end, prefix;  // next unit of the work, the last, and where the own rows' begins
    int u, base;               // next unit (-1: not looked for), and the work before its block
};

struct PrefixArgs {
    const void *K, *V, *q;
    const int32_t *table;
    const PrefixRun *runs;
    const int32_t *run_of;
    PrefixTotal *total;  // (the attention sets `stopped`)
    const PrefixUnit *units;
    const int32_t *block_work;
    float *part_o, *own_o, *cont_o;
    float2 *part_ml, *own_ml, *cont_ml;  // (max to base 2, sum; -1: in error)
    int layers, B, Hq, Hkv, G, n_pages, max_pages, shift, n_units, n_blocks;
    PrefixRows rows;
    int cont_rows;  // rows a CTA has in cont_o: those of the largest row tile
    float c2;       // scale * log2(e)
    unsigned *err;

    __device__ __forceinline__ long long prefix_total() const { return total->work * layers * Hkv; }
    __device__ __forceinline__ int own_total() const
    {
        int sum = 0;
#pragma unroll 8
        for (int i = 0; i < n_blocks; ++i) sum += __ldg(block_work + i);
        return sum;
    }
    __device__ __forceinline__ PrefixWalk range() const
    {
        PrefixWalk w;
        w.prefix = prefix_total();
        w.u = -1;
        w.base = 0;
        const PrefixShare share(w.prefix + own_total(), (int)gridDim.x, total->most);
        const int c = blockIdx.x;
        w.w = c < share.n ? share.begin(c) : 0;
        w.end = c < share.n ? share.begin(c + 1) : 0;
        return w;
    }
    // (whole warps)
    __device__ __forceinline__ bool next(PrefixWalk &w, PrefixPiece &pc) const
    {
        while (w.w < w.end) {
            if (w.w < w.prefix) {
                const long long per = total->work, lh = quotient(w.w, per), rem = w.w - lh * per;
                const PrefixRun r = runs[warp_last(total->n, rem, [&](int i) { return runs[i].work; })];
                const int kt = (r.p + kPrefixTile - 1) / kPrefixTile;
                const long long in = rem - r.work, full = (long long)kt * rows.unit(r.n, 0);
                const int rt = (int)quotient(in, full), unit = rows.unit(r.n, rt), u = (int)(in - rt * full);
                const int e = (int)min((long long)kt * unit, u + (w.end - w.w));
                pc.layer = (int)lh / Hkv;
                pc.h = (int)lh - pc.layer * Hkv;
                pc.b0 = r.b0;
                pc.s0 = rt * rows.per;
                pc.nseq = min(rows.per, r.n - pc.s0);
                pc.k0 = pc.lo = 0;
                pc.end = r.p;
                pc.t0 = (u + unit - 1) / unit;
                pc.t1 = (e + unit - 1) / unit;
                pc.own = false;
                w.w += e - u;
                if (pc.t0 < pc.t1) return true;
                continue;
            }
            const int at = (int)(w.w - w.prefix);
            if (w.u < 0) {  // the unit that this falls to
                int blk = 0;
                while (blk + 1 < n_blocks && w.base + __ldg(block_work + blk) <= at) w.base += __ldg(block_work + blk++);
                const int u0 = blk * kPrefixBlock;
                w.u = u0 + warp_last(min(kPrefixBlock, n_units - u0), at - w.base, [&](int i) { return units[u0 + i].work; });
            }
            if (w.u >= n_units) return false;
            const PrefixUnit x = units[w.u];
            const int kt = x.lo >= 0 && x.n - x.lo > rows.few ? (x.n - x.k0 + kPrefixTile - 1) / kPrefixTile : 0;
            const int lb = w.u / Hkv;
            pc.layer = lb / B;
            pc.h = w.u - lb * Hkv;
            pc.b0 = lb - pc.layer * B;
            pc.s0 = 0;
            pc.nseq = 1;
            pc.k0 = x.k0;
            pc.lo = x.lo;
            pc.end = x.n;
            const int in = at - w.base - x.work, unit = rows.own(), size = kt > 0 ? unit * kt + rows.extra() : 0;
            if (size == 0) {  // (and maybe many like it: the next one with work is looked for)
                w.u = -1;
                w.base = 0;
                continue;
            }
            const int e = (int)min((long long)size, in + (w.end - w.w));
            pc.t0 = max(0, in - rows.extra() + unit - 1) / unit;
            pc.t1 = max(0, e - rows.extra() + unit - 1) / unit;
            pc.own = true;
            if (e == size) {  // the next unit, maybe of the next block
                ++w.u;
                if (w.u % kPrefixBlock == 0 && w.u < n_units) w.base += __ldg(block_work + w.u / kPrefixBlock - 1);
            }
            w.w += e - in;
            if (pc.t0 < pc.t1) return true;
        }
        return false;
    }
    // Query head g of a tile's sequence s, as a row of q.
    __device__ __forceinline__ long long q_row(const PrefixPiece &pc, int s, int g) const
    {
        return ((long long)pc.layer * B + pc.b0 + pc.s0 + s) * Hq + pc.h * G + g;
    }
    // Pool row of row j, -1 where its table entry names no page.
    __device__ __forceinline__ long long pool_row(const PrefixPiece &pc, int j) const
    {
        const int e = __ldg(table + (long long)pc.b0 * max_pages + (j >> shift));
        if ((unsigned)e >= (unsigned)n_pages) return -1;
        return ((((long long)pc.layer * n_pages + e) * Hkv + pc.h) << shift) + (j & ((1 << shift) - 1));
    }
    // Where the partial of head g of the tile's sequence s goes: an item's first by query head, the others by CTA.
    template <int D> __device__ __forceinline__ void partial(const PrefixPiece &pc, int s, int g, float *&o, float2 *&ml) const
    {
        const long long at = pc.t0 == 0 ? q_row(pc, s, g) : (long long)blockIdx.x * cont_rows + s * G + g;
        o = (pc.t0 != 0 ? cont_o : (pc.own ? own_o : part_o)) + at * D;
        ml = (pc.t0 != 0 ? cont_ml : (pc.own ? own_ml : part_ml)) + at;
    }
};

// The attention of all pieces over bf16 caches (prefix_tc.cu).
cudaError_t launch_prefix_tc(const reco_paged_kv &kv, const PrefixArgs &a, int grid, reco_dtype out_dtype, cudaStream_t s);
#endif

}  // namespace reco
