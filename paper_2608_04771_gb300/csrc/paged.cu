// paged.cu -- decode attention of one new token over a paged cache, and the accumulation of the
// rows' attention weights (Eq. 2's sums, taken token by token as the tokens are decoded).
//
// The attention is the streamed kernel of decode_stream.cuh over pages.  A call with weights has it
// leave its logits (4 G bytes a row, against 4 d bytes of K and V in bf16) in the workspace; they
// become weights once a unit's log-sum-exps are known, in paged_weights, mostly from L2, where a
// second product with K would read half of the cache again.
#include "decode_stream.cuh"

namespace reco {

PagedDecodeWs paged_decode_ws_layout(const reco_paged_kv &kv, bool weights, void *base)
{
    const reco_kv units{kv.k, kv.v, kv.n_layers, kv.B, kv.H_q, kv.H_kv, paged_cap(kv), kv.d, kv.dtype};
    PagedDecodeWs ws;
    ws.dec = decode_ws_layout(units, base);
    size_t off = ws.dec.bytes;
    auto take = [&](size_t bytes) {
        char *r = base ? (char *)base + off : nullptr;
        off += align256(bytes);
        return r;
    };
    const size_t heads = (size_t)kv.n_layers * kv.B * kv.H_q;
    ws.lse2 = weights ? (float *)take(heads * 4) : nullptr;
    ws.logits = weights ? (float *)take(heads * paged_cap(kv) * 4) : nullptr;
    ws.bytes = off;
    return ws;
}

// weights[u, j] += (1/G) sum_g 2^(logit - lse2) for the rows in sight.  Threads take four rows at a time
// (a block of the decode holds all four or none).
constexpr int kWeightThreads = 256, kWeightRows = 4 * kWeightThreads;

__global__ void __launch_bounds__(kWeightThreads) paged_weights(const float *__restrict__ logits,
                                                                const float *__restrict__ lse2,
                                                                const int32_t *__restrict__ lens, int G, int cap,
                                                                int window, int sinks, float *weights)
{
    wait_prior_grid();
    const long u = blockIdx.y;
    const int n = lens[u];
    if (n < 0 || n > cap) return;  // reported by the decode
    __shared__ float sm_lse[16];
    if (threadIdx.x < G) sm_lse[threadIdx.x] = lse2[u * G + threadIdx.x];
    __syncthreads();
    bool any = false;
    for (int g = 0; g < G; ++g) any |= sm_lse[g] != -INFINITY;
    if (!any) return;  // no rows, or in error
    const int start = window > 0 && n > window ? n - window : 0, head = min(sinks, start);
    const float inv = 1.f / (float)G;
    for (int j0 = (blockIdx.x * kWeightThreads + threadIdx.x) * 4; j0 < n; j0 += gridDim.x * kWeightRows) {
        if (j0 >= head && j0 + 4 <= start) continue;
        float4 *dst = reinterpret_cast<float4 *>(weights + u * cap + j0);
        const float *src = logits + u * G * cap + j0;
        const float4 old = *dst;
        float4 p = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int g = 0; g < G; ++g) {
            const float4 x = __ldcs(reinterpret_cast<const float4 *>(src + (long)g * cap));
            const float z = sm_lse[g];
            if (z == -INFINITY) continue;
            p.x += fast_exp2(x.x - z);
            p.y += fast_exp2(x.y - z);
            p.z += fast_exp2(x.z - z);
            p.w += fast_exp2(x.w - z);
        }
        const float4 sum = make_float4(fmaf(p.x, inv, old.x), fmaf(p.y, inv, old.y), fmaf(p.z, inv, old.z),
                                       fmaf(p.w, inv, old.w));
        if (j0 + 4 <= n && (j0 + 4 <= head || j0 >= start)) {
            *dst = sum;
        } else {
            auto seen = [&](int j) { return j < n && (j < head || j >= start); };
            if (seen(j0)) dst->x = sum.x;
            if (seen(j0 + 1)) dst->y = sum.y;
            if (seen(j0 + 2)) dst->z = sum.z;
            if (seen(j0 + 3)) dst->w = sum.w;
        }
    }
}

cudaError_t launch_paged_decode(const reco_paged_kv &kv, const void *q, const void *k_new, const void *v_new,
                                int32_t *lens, float scale, int window, int sinks, void *out, reco_dtype out_dtype,
                                float *lse, float *weights, const PagedDecodeWs &ws, unsigned *err, cudaStream_t s)
{
    const bool f32 = kv.dtype == RECO_F32;
    const int cap = paged_cap(kv);
    DecodeArgs a = {};
    a.K = kv.k;
    a.V = kv.v;
    a.counters = ws.dec.counters;
    a.part_ml = ws.dec.part_ml;
    a.part_o = ws.dec.part_o;
    a.Hq = kv.H_q;
    a.Hkv = kv.H_kv;
    a.G = kv.H_q / kv.H_kv;
    a.L_cap = cap;
    a.append = k_new ? 1 : 0;
    a.out_bf16 = out_dtype == RECO_BF16 ? 1 : 0;
    a.c2 = scale * kLog2e;
    a.err = err;
    a.table = kv.table;
    a.B = kv.B;
    a.n_pages = kv.n_pages;
    a.max_pages = kv.max_pages;
    a.page_shift = __builtin_ctz((unsigned)kv.page);
    a.window = window;
    a.sinks = sinks;
    const int units = kv.n_layers * kv.B * kv.H_kv;
    const StreamKernel k = stream_kernel<true>(kv.d, f32, units, a.G, cap);
    a.hs_min = k.hs;
    CUtensorMap mk = {}, mv = {};
    const unsigned long long rows = (unsigned long long)kv.n_layers * kv.n_pages * kv.H_kv * kv.page;
    if (!f32 && (!encode_cache_map(&mk, kv.k, rows, kv.d) || !encode_cache_map(&mv, kv.v, rows, kv.d)))
        return cudaErrorInvalidValue;
    const size_t row_b = (size_t)kv.d * (f32 ? 4 : 2), out_b = (size_t)kv.d * (a.out_bf16 ? 2 : 4);
    for (long long u0 = 0; u0 < units; u0 += k.part_units) {  // as many units as one plan holds
        const int cu = (int)std::min(k.part_units, units - u0);
        const size_t q0 = (size_t)u0 * a.G;
        DecodeArgs at = a;
        at.u0 = (int)u0;
        at.units = cu;
        at.hs_max = k.most_halves(cu, a.G);
        at.q = static_cast<const char *>(q) + q0 * row_b;
        at.k_new = k_new ? static_cast<const char *>(k_new) + (size_t)u0 * row_b : nullptr;
        at.v_new = v_new ? static_cast<const char *>(v_new) + (size_t)u0 * row_b : nullptr;
        at.lens = lens + u0;
        at.out = static_cast<char *>(out) + q0 * out_b;
        at.lse = lse ? lse + q0 : nullptr;
        if (weights) {
            at.lse2 = ws.lse2 + q0;
            at.logits = ws.logits + q0 * cap;
            at.weights = weights + (size_t)u0 * cap;
        }
        const cudaError_t e = launch_stream(k.fn, kv.d, mk, mv, at, ws.dec.part_slots, s);
        if (e != cudaSuccess) return e;
    }
    if (!weights) return cudaSuccess;
    // CTAs over a unit's rows: enough that all units together fill the GPU four times over, never more than
    // the rows of a unit need (lengths are not known here, and CTAs without rows cost time too)
    const int need = (cap + kWeightRows - 1) / kWeightRows, fill = 4 * 8 * device_sm_count() / units;
    const cudaError_t e = launch_pdl(paged_weights, dim3(std::max(1, std::min(need, fill)), units), dim3(kWeightThreads),
                                     0, s, (const float *)ws.logits, (const float *)ws.lse2, (const int32_t *)lens, a.G,
                                     cap, window, sinks, weights);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace reco
