// paged.cu -- decode attention of one new token over a paged cache: the host side of paged_kernel.cuh's kernel, and
// the weights of the units that it cuts between CTAs.
#include "paged_kernel.cuh"

namespace reco {

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

cudaError_t launch_paged_decode(const reco_paged_kv &kv, const void *q, const void *k_new, const void *v_new,
                                int32_t *lens, float scale, int window, int sinks, void *out, reco_dtype out_dtype,
                                float *lse, float *weights, const PagedDecodeWs &ws, unsigned *err, cudaStream_t s)
{
    PagedArgs a = paged_args(kv, q, k_new, v_new, lens, scale, out, out_dtype, lse, ws, err);
    a.lse2 = ws.lse2;
    a.logits = ws.logits;
    a.weights = weights;
    a.cuts = ws.cuts;
    a.window = window;
    a.sinks = sinks;
    // (units that fit the grid are cut one piece per CTA: no unit is left for the weight warps)
    const int most_seen = window > 0 ? (int)std::min<long long>(a.cap, (long long)window + sinks) : a.cap;
    a.inline_weights = weights && a.units <= std::min(device_sm_count(), kPagedMaxGrid) && most_seen <= kInlineRows ? 1 : 0;
    const bool f32 = kv.dtype == RECO_F32;
    cudaError_t e = launch_paged_kernel(kv, kv.d == 64 ? paged_kernel<64, false>(f32, a.G) : paged_kernel<128, false>(f32, a.G), a, s);
    if (e != cudaSuccess || !weights || a.inline_weights) return e;
    e = launch_pdl(paged_weights, dim3(4 * device_sm_count()), dim3(kWeightThreads), 0, s, (const float *)ws.logits,
                   (const float *)ws.lse2, (const int32_t *)lens, (const int32_t *)ws.cuts, a.units, a.G, a.cap, window, sinks,
                   weights);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace reco
