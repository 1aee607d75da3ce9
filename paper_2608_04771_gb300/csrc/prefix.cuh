// prefix.cuh -- what the kernels of decode attention over shared prefixes (prefix.cu) have in common: the list of groups,
// a CTA's walk over its share of the work, and where partials go.
#pragma once
#include "common.cuh"
#include "internal.h"

namespace reco {

// The work of a row tile (rt of a group of R query rows, `rows` to a tile) against one key tile: 1 for every 128 query
// rows begun, what the tensor cores take at once.
__host__ __device__ inline int prefix_unit(int R, int rt, int rows)
{
    const int left = R - rt * rows;
    return ((left < rows ? left : rows) + 127) / 128;
}
// Work of a group per layer and KV head.
__host__ __device__ inline long long prefix_work(int n, int G, int p, int rows)
{
    const int R = n * G, last = (R - 1) / rows, kt = (p + kPrefixTile - 1) / kPrefixTile;
    return (long long)kt * ((long long)last * ((rows + 127) / 128) + prefix_unit(R, last, rows));
}
// The work is shared out to n CTAs, each with some key tile of every row tile that it gets (so that the joining kernel
// finds a partial from every CTA between an item's first and last).  CTA c's begins at total * c / n; the CTA that unit w
// of the work falls to.  A key tile whose work is cut goes to the CTA that its first unit falls to.
__device__ __forceinline__ long long prefix_ctas(long long total, int grid, int rows)
{
    const long long most = total / ((rows + 127) / 128);
    return most < 1 ? 1 : (most < grid ? most : grid);
}
__device__ __forceinline__ long long prefix_begin(long long c, long long total, long long n) { return total * c / n; }
__device__ __forceinline__ int prefix_cta(long long w, long long total, long long n) { return (int)(((w + 1) * n - 1) / total); }

// A CTA's part of an item: key tiles [t0, t1) of the prefix (p rows, first sequence b0) against row tile rt of nrows rows.
struct PrefixPiece {
    int layer, h, b0, p, rt, nrows, t0, t1;
};
struct PrefixWalk {
    long long w, end;
};

struct PrefixArgs {
    const void *K, *V, *q;
    const int32_t *table;
    const PrefixRun *runs;
    const int32_t *run_of;
    const PrefixTotal *total;
    float *part_o, *cont_o;      // by query head; by CTA and row of the tile
    float2 *part_ml, *cont_ml;   // (max to base 2, sum; -1: in error)
    int layers, B, Hq, Hkv, G, n_pages, max_pages, shift;
    int rows;       // query rows of a row tile
    int cont_rows;  // rows a CTA has in cont_o: those of the largest row tile
    float c2;  // scale * log2(e)
    unsigned *err;

#ifdef __CUDACC__
    __device__ __forceinline__ PrefixWalk range() const
    {
        const long long all = total->work * layers * Hkv;
        const long long n = prefix_ctas(all, (int)gridDim.x, rows);
        if (all == 0 || blockIdx.x >= n) return PrefixWalk{0, 0};
        return PrefixWalk{prefix_begin(blockIdx.x, all, n), prefix_begin(blockIdx.x + 1, all, n)};
    }
    __device__ __forceinline__ bool next(PrefixWalk &w, PrefixPiece &pc) const
    {
        while (w.w < w.end) {
            const long long per = total->work, lh = w.w / per, rem = w.w - lh * per;
            int lo = 0, n = total->n;
            while (n > 1) {  // the last group that begins at or before rem
                const int half = n >> 1;
                if (runs[lo + half].work <= rem) {
                    lo += half;
                    n -= half;
                } else {
                    n = half;
                }
            }
            const PrefixRun r = runs[lo];
            const int kt = (r.p + kPrefixTile - 1) / kPrefixTile;
            const long long in = rem - r.work, full = (long long)kt * ((rows + 127) / 128);
            pc.layer = (int)(lh / Hkv);
            pc.h = (int)(lh - (long long)pc.layer * Hkv);
            pc.b0 = r.b0;
            pc.p = r.p;
            pc.rt = (int)(in / full);
            pc.nrows = min(rows, r.n * G - pc.rt * rows);
            const int unit = prefix_unit(r.n * G, pc.rt, rows), u = (int)(in - pc.rt * full);
            const int e = (int)min((long long)kt * unit, u + (w.end - w.w));
            pc.t0 = (u + unit - 1) / unit;
            pc.t1 = (e + unit - 1) / unit;
            w.w += e - u;
            if (pc.t0 < pc.t1) return true;
        }
        return false;
    }
    // Query head of row r of the group's rows (sequence by sequence), as a row of q.
    __device__ __forceinline__ long long q_row(const PrefixPiece &pc, int r) const
    {
        const int s = r / G;
        return ((long long)pc.layer * B + pc.b0 + s) * Hq + pc.h * G + (r - s * G);
    }
    // Pool row of row j of the prefix, -1 where its table entry names no page.
    __device__ __forceinline__ long long pool_row(const PrefixPiece &pc, int j) const
    {
        const int e = __ldg(table + (long long)pc.b0 * max_pages + (j >> shift));
        if ((unsigned)e >= (unsigned)n_pages) return -1;
        return ((((long long)pc.layer * n_pages + e) * Hkv + pc.h) << shift) + (j & ((1 << shift) - 1));
    }
    template <int D> __device__ __forceinline__ void partial(const PrefixPiece &pc, int r, float *&o, float2 *&ml) const
    {
        if (pc.t0 == 0) {
            const long long at = q_row(pc, pc.rt * rows + r);
            o = part_o + at * D;
            ml = part_ml + at;
        } else {
            const long long at = (long long)blockIdx.x * cont_rows + r;
            o = cont_o + at * D;
            ml = cont_ml + at;
        }
    }
#endif
};

// The prefix part over bf16 caches (prefix_tc.cu).
cudaError_t launch_prefix_tc(const reco_paged_kv &kv, const PrefixArgs &a, int grid, reco_dtype out_dtype, cudaStream_t s);

struct PrefixJoin {
    PrefixArgs p;
    const float *own_out, *own_l2;
    int32_t *lens;
    void *out;
    float *lse;  // or nullptr
    int grid, cap, append, out_bf16;
};

}  // namespace reco
