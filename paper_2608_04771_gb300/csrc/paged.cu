// paged.cu -- decode attention of one new token over a paged cache, and the accumulation of the
// rows' attention weights.
//
// paged_decode: one CTA per unit; its warps take the visible rows in turn, each with an online
// softmax over all query heads, and join at the end.  paged_weights: the second pass of a call
// with weights, one warp per row, from the log-sum-exps of the first.
#include "common.cuh"
#include "internal.h"

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

struct PagedArgs {
    void *K, *V;
    const int32_t *table;
    const void *q, *k_new, *v_new;
    int32_t *lens;
    void *out;
    float *lse, *lse2, *weights;
    int B, Hq, Hkv, G, cap, n_pages, max_pages, shift, append, out_bf16, window, sinks;
    float c2;  // scale * log2(e)
    unsigned *err;
};

// Row j of the unit, or -1 where the table names no page of the pool.
__device__ __forceinline__ long paged_row(const PagedArgs &a, long u, int j)
{
    const long lb = u / a.Hkv;
    const int e = a.table[(lb % a.B) * a.max_pages + (j >> a.shift)];
    if ((unsigned)e >= (unsigned)a.n_pages) return -1;
    return ((((lb / a.B) * a.n_pages + e) * a.Hkv + u % a.Hkv) << a.shift) + (j & ((1 << a.shift) - 1));
}

template <typename T, int D>
__global__ void __launch_bounds__(128) paged_decode(PagedArgs a)
{
    constexpr int NW = 4, PER = D / 32, GM = 16;
    __shared__ float sm_m[NW][GM], sm_l[NW][GM];
    __shared__ float sm_o[NW][GM][D];
    const long u = blockIdx.x;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int L = a.lens[u];
    bool ok = L >= 0 && L <= a.cap && (!a.append || L < a.cap);
    if (!ok && threadIdx.x == 0) raise_error(a.err, (a.append && L == a.cap) ? ERR_ROOM : ERR_LEN);
    const int n = ok ? L + a.append : 0;
    const int start = a.window > 0 && n > a.window ? n - a.window : 0;  // rows from here on are seen
    const int head = min(a.sinks, start);                               // and the rows before this
    // all needed table entries first
    bool bad = false;
    for (int p = threadIdx.x; p << a.shift < n; p += blockDim.x)
        if (((p + 1) << a.shift) > start || p << a.shift < head) bad |= paged_row(a, u, p << a.shift) < 0;
    if (__syncthreads_or(bad)) {
        if (threadIdx.x == 0) raise_error(a.err, ERR_PAGE);
        ok = false;
    }
    const int Le = ok ? n : 0;
    const long lb = u / a.Hkv;
    const int h = (int)(u % a.Hkv), G = a.G;
    T *K = reinterpret_cast<T *>(a.K), *V = reinterpret_cast<T *>(a.V);
    const T *kn = reinterpret_cast<const T *>(a.k_new) + u * D, *vn = reinterpret_cast<const T *>(a.v_new) + u * D;
    const T *qp = reinterpret_cast<const T *>(a.q) + (lb * a.Hq + (long)h * G) * D;
    float q[GM][PER], o[GM][PER], m[GM], l[GM];
#pragma unroll
    for (int g = 0; g < GM; ++g) {
        m[g] = -INFINITY;
        l[g] = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            q[g][i] = g < G ? to_float(qp[(long)g * D + lane * PER + i]) : 0.f;
            o[g][i] = 0.f;
        }
    }
    for (int v = wid; v < head + Le - start; v += NW) {
        const int j = v < head ? v : v - head + start;
        const bool app = a.append && j == L;
        const long r = paged_row(a, u, j);
        const T *kr = app ? kn : K + r * D, *vr = app ? vn : V + r * D;
        float kk[PER], vv[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            kk[i] = to_float(kr[lane * PER + i]);
            vv[i] = to_float(vr[lane * PER + i]);
        }
#pragma unroll
        for (int g = 0; g < GM; ++g) {
            if (g < G) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < PER; ++i) s = fmaf(q[g][i], kk[i], s);
                s = warp_sum(s) * a.c2;
                const float mn = fmaxf(m[g], s);
                const float base = mn == -INFINITY ? 0.f : mn;
                const float al = fast_exp2(m[g] - base), p = fast_exp2(s - base);
                l[g] = l[g] * al + p;
#pragma unroll
                for (int i = 0; i < PER; ++i) o[g][i] = fmaf(o[g][i], al, p * vv[i]);
                m[g] = mn;
            }
        }
    }
#pragma unroll
    for (int g = 0; g < GM; ++g) {
        if (g < G) {
            if (lane == 0) {
                sm_m[wid][g] = m[g];
                sm_l[wid][g] = l[g];
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) sm_o[wid][g][lane * PER + i] = o[g][i];
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < G * D; e += blockDim.x) {
        const int g = e / D, dd = e % D;
        float M = -INFINITY;
        for (int w = 0; w < NW; ++w) M = fmaxf(M, sm_m[w][g]);
        float Ls = 0.f, O = 0.f;
        if (M != -INFINITY) {
            for (int w = 0; w < NW; ++w) {
                const float wt = fast_exp2(sm_m[w][g] - M);
                Ls += sm_l[w][g] * wt;
                O += sm_o[w][g][dd] * wt;
            }
        }
        const size_t row = (size_t)(lb * a.Hq + (long)h * G + g);
        const float res = Ls > 0.f ? O / Ls : 0.f;
        if (a.out_bf16)
            reinterpret_cast<__nv_bfloat16 *>(a.out)[row * D + dd] = __float2bfloat16_rn(res);
        else
            reinterpret_cast<float *>(a.out)[row * D + dd] = res;
        if (dd == 0) {
            const float l2 = Ls > 0.f ? M + log2f(Ls) : -INFINITY;
            if (a.lse) a.lse[row] = l2 * kLn2;
            if (a.lse2) a.lse2[row] = l2;
        }
    }
    if (ok && a.append) {
        const long r = paged_row(a, u, L);
        for (int e = threadIdx.x; e < D; e += blockDim.x) {
            K[r * D + e] = kn[e];
            V[r * D + e] = vn[e];
        }
        if (threadIdx.x == 0) {
            a.lens[u] = L + 1;
            if (a.weights) a.weights[u * a.cap + L] = 0.f;
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(256) paged_weights(PagedArgs a)
{
    constexpr int PER = D / 32;
    const long u = blockIdx.x;
    const int lane = threadIdx.x & 31;
    const int n = a.lens[u];
    if (n < 0 || n > a.cap) return;
    const long lb = u / a.Hkv;
    const size_t q0 = lb * a.Hq + (u % a.Hkv) * a.G;
    bool any = false;
    for (int g = 0; g < a.G; ++g) any |= a.lse2[q0 + g] != -INFINITY;
    if (!any) return;
    const int start = a.window > 0 && n > a.window ? n - a.window : 0, head = min(a.sinks, start);
    for (int v = blockIdx.y * 8 + (threadIdx.x >> 5); v < head + n - start; v += gridDim.y * 8) {
        const int j = v < head ? v : v - head + start;
        const T *kr = reinterpret_cast<const T *>(a.K) + paged_row(a, u, j) * D;
        float w = 0.f;
        for (int g = 0; g < a.G; ++g) {
            const T *qp = reinterpret_cast<const T *>(a.q) + (q0 + g) * D;
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) s = fmaf(to_float(qp[lane * PER + i]), to_float(kr[lane * PER + i]), s);
            s = warp_sum(s) * a.c2;
            if (a.lse2[q0 + g] != -INFINITY) w += fast_exp2(s - a.lse2[q0 + g]);
        }
        if (lane == 0) a.weights[u * a.cap + j] += w / (float)a.G;
    }
}

template <typename T, int D> static cudaError_t launch(const PagedArgs &a, unsigned units, cudaStream_t s)
{
    paged_decode<T, D><<<units, 128, 0, s>>>(a);
    if (a.weights) paged_weights<T, D><<<dim3(units, 8), 256, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_paged_decode(const reco_paged_kv &kv, const void *q, const void *k_new, const void *v_new,
                                int32_t *lens, float scale, int window, int sinks, void *out, reco_dtype out_dtype,
                                float *lse, float *weights, const PagedDecodeWs &ws, unsigned *err, cudaStream_t s)
{
    const PagedArgs a{kv.k, kv.v, kv.table, q, k_new, v_new, lens, out, lse, ws.lse2, weights, kv.B, kv.H_q, kv.H_kv,
                      kv.H_q / kv.H_kv, paged_cap(kv), kv.n_pages, kv.max_pages, __builtin_ctz((unsigned)kv.page),
                      k_new ? 1 : 0, out_dtype == RECO_BF16 ? 1 : 0, window, sinks, scale * kLog2e, err};
    const unsigned units = (unsigned)(kv.n_layers * kv.B * kv.H_kv);
    if (kv.dtype == RECO_F32) return kv.d == 64 ? launch<float, 64>(a, units, s) : launch<float, 128>(a, units, s);
    return kv.d == 64 ? launch<__nv_bfloat16, 64>(a, units, s) : launch<__nv_bfloat16, 128>(a, units, s);
}

}  // namespace reco
