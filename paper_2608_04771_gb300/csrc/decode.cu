// decode.cu -- decode attention over the ragged compacted cache, the per-token attention
// whose cost the compression lowers (Sec. 1; Sec. 2.2; Sec. 4.2): the streamed kernel of
// decode_stream.cuh, and decode_simt for bf16 calls for which no tensor map can be made.
#include "decode_stream.cuh"

namespace reco {

DecodeWs decode_ws_layout(const reco_kv &kv, void *base)
{
    size_t units = (size_t)kv.n_layers * kv.B * kv.H_kv;
    size_t G = kv.H_q / kv.H_kv;
    char *p = (char *)base;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char *r = p ? p + off : nullptr;
        off += align256(bytes);
        return r;
    };
    DecodeWs ws;
    ws.part_slots = kDecodePartSlots;
    // merge tickets per unit; a unit of G > 8 heads may run as two
    ws.counters = (int32_t *)take((2 + units * (G > 8 ? 2 : 1)) * 4);
    ws.part_ml = (float *)take((size_t)ws.part_slots * G * 2 * 4);
    ws.part_o = (float *)take((size_t)ws.part_slots * G * kv.d * 4);
    ws.bytes = off;
    return ws;
}

// ---------------------------------------------------------------- SIMT path
template <typename T, int D>
__global__ void __launch_bounds__(128) decode_simt(DecodeArgs a)
{
    constexpr int NW = 4, PER = D / 32, GM = 16;
    __shared__ float sm_m[NW][GM], sm_l[NW][GM];
    __shared__ float sm_o[NW][GM][D];
    const long u = blockIdx.x;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int L = a.lens[u];
    const long long rs = ring_row(a);
    const bool ok = unit_ok(L, a.L_cap, a.append);
    if (!ok && threadIdx.x == 0) raise_error(a.err, (a.append && L == a.L_cap) ? ERR_ROOM : ERR_LEN);
    const int Le = ok ? L + a.append : 0;
    const long lb = u / a.Hkv;
    const int h = (int)(u % a.Hkv);
    const int G = a.G;
    T *Kp = reinterpret_cast<T *>(a.K) + u * (long)a.L_cap * D;
    T *Vp = reinterpret_cast<T *>(a.V) + u * (long)a.L_cap * D;
    const T *kn = a.append ? reinterpret_cast<const T *>(a.k_new) + u * D : nullptr;
    const T *vn = a.append ? reinterpret_cast<const T *>(a.v_new) + u * D : nullptr;
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
    for (int j = wid; j < Le; j += NW) {
        const T *kr = (a.append && j == L) ? kn : Kp + (long)j * D;
        const T *vr = (a.append && j == L) ? vn : Vp + (long)j * D;
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
                const float al = fast_exp2(m[g] - mn);
                const float p = fast_exp2(s - mn);
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
        store_out(a.out, a.out_bf16, row * D + dd, Ls > 0.f ? O / Ls : 0.f);
        if (dd == 0) put_lse(a, rs, row, Ls > 0.f ? M + log2f(Ls) : -INFINITY);
    }
    if (ok && a.append) {
        for (int e = threadIdx.x; e < D; e += blockDim.x) {
            Kp[(long)L * D + e] = kn[e];
            Vp[(long)L * D + e] = vn[e];
        }
        if (threadIdx.x == 0) a.lens[u] = L + 1;
    }
}

// The launch's queries into the window ring after the SIMT decode: chunk c (16 bytes)
// of query row c / ch goes to row *slot of that head's `slots` rows.
__global__ void qring_copy(const uint4 *__restrict__ q, uint4 *__restrict__ qring, long long n16, int ch, int slots,
                           const long long *slot)
{
    const long long s = *slot;
    if (s < 0 || s >= slots) return;  // the decode has reported the slot
    for (long long c = (long long)blockIdx.x * blockDim.x + threadIdx.x; c < n16; c += (long long)gridDim.x * blockDim.x)
        qring[(c / ch * slots + s) * ch + c % ch] = q[c];
}

// The ring slot's advance after the SIMT decode (its CTAs have no last-warp step).
__global__ void ring_advance(long long *slot, int slots)
{
    const long long s = *slot;
    if (s >= 0 && s < slots) *slot = (s + 1) % slots;
}

// ---------------------------------------------------------------- host side
cudaError_t launch_decode(const reco_kv &kv, const void *q, const void *k_new, const void *v_new,
                          int32_t *lens, float scale, void *out, reco_dtype out_dtype, float *lse,
                          const DecodeWs &ws, unsigned *err, cudaStream_t s, float *ring, int slots,
                          long long *slot, void *qring)
{
    DecodeArgs a = {};
    a.K = kv.k;
    a.V = kv.v;
    a.q = q;
    a.k_new = k_new;
    a.v_new = v_new;
    a.lens = lens;
    a.out = out;
    a.lse = lse;
    a.counters = ws.counters;
    a.part_ml = ws.part_ml;
    a.part_o = ws.part_o;
    a.units = kv.n_layers * kv.B * kv.H_kv;
    a.Hq = kv.H_q;
    a.Hkv = kv.H_kv;
    a.G = kv.H_q / kv.H_kv;
    a.L_cap = kv.L_cap;
    a.append = (k_new && v_new) ? 1 : 0;
    a.out_bf16 = out_dtype == RECO_BF16 ? 1 : 0;
    a.c2 = scale * kLog2e;
    a.err = err;
    a.ring = ring;
    a.slot = slot;
    a.slots = slots;
    a.nq = (long long)kv.n_layers * kv.B * kv.H_q;
    a.qring = ring ? qring : nullptr;
    a.nq_rows = a.nq;
    a.advance = 1;
    const bool f32 = kv.dtype == RECO_F32;
    const StreamKernel k = stream_kernel<false>(kv.d, f32, a.units, a.G, kv.L_cap);
    const int hs = k.hs;
    a.hs_min = hs;
    const DecodeKernel fn = k.fn;
    // More units than one plan holds in shared memory run as consecutive launches over
    // contiguous unit ranges (every unit is independent): each part gets its own K/V, q,
    // output, lens and ring pointers, and only the last part advances the ring slot.
    const long long part_units = k.part_units;  // cache units per launch
    // bf16 rows are addressed by tensor-map coordinates
    if (f32 || (unsigned long long)std::min<long long>(a.units, part_units) * kv.L_cap < (1ull << 31)) {
        const size_t row_b = (size_t)kv.d * (f32 ? 4 : 2);  // cache and query rows
        const size_t out_b = (size_t)kv.d * (out_dtype == RECO_BF16 ? 2 : 4);
        for (long long u0 = 0; u0 < a.units; u0 += part_units) {
            const long long cu = std::min(part_units, (long long)a.units - u0);
            const long long q0 = u0 * a.G;  // first query head of the part
            const unsigned long long rows = (unsigned long long)cu * kv.L_cap;
            CUtensorMap mk = {}, mv = {};
            const char *kb = static_cast<const char *>(kv.k) + (size_t)u0 * kv.L_cap * row_b;
            const char *vb = static_cast<const char *>(kv.v) + (size_t)u0 * kv.L_cap * row_b;
            if (!f32 && (!encode_cache_map(&mk, kb, rows, kv.d) || !encode_cache_map(&mv, vb, rows, kv.d))) {
                if (u0 == 0) break;  // the SIMT path below takes the whole call
                return cudaErrorInvalidValue;
            }
            DecodeArgs at = a;  // this part
            at.units = (int)cu;
            at.hs_max = k.most_halves((int)cu, a.G);
            at.K = const_cast<char *>(kb);
            at.V = const_cast<char *>(vb);
            at.q = static_cast<const char *>(q) + (size_t)q0 * row_b;
            at.k_new = k_new ? static_cast<const char *>(k_new) + (size_t)u0 * row_b : nullptr;
            at.v_new = v_new ? static_cast<const char *>(v_new) + (size_t)u0 * row_b : nullptr;
            at.lens = lens + u0;
            at.out = static_cast<char *>(out) + (size_t)q0 * out_b;
            at.lse = lse ? lse + q0 : nullptr;
            at.ring = ring ? ring + q0 : nullptr;  // ring rows keep their full stride nq
            at.qring = a.qring ? static_cast<char *>(a.qring) + (size_t)q0 * slots * row_b : nullptr;
            at.nq_rows = cu * a.G;
            at.advance = u0 + cu >= a.units ? 1 : 0;
            const cudaError_t e = launch_stream(fn, kv.d, mk, mv, at, ws.part_slots, s);
            if (e != cudaSuccess) return e;
            if (u0 + cu >= a.units) return cudaSuccess;
        }
    }
    // bf16 caches that no tensor map covers
    const unsigned grid = (unsigned)a.units;
    if (kv.d == 64) decode_simt<__nv_bfloat16, 64><<<grid, 128, 0, s>>>(a);
    else decode_simt<__nv_bfloat16, 128><<<grid, 128, 0, s>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !ring) return e;
    if (a.qring) {
        const int ch = kv.d * 2 / 16;
        const long long n16 = a.nq * ch;
        const unsigned blocks = (unsigned)std::min<long long>((n16 + 255) / 256, 4LL * device_sm_count());
        qring_copy<<<blocks, 256, 0, s>>>(reinterpret_cast<const uint4 *>(q), reinterpret_cast<uint4 *>(a.qring), n16,
                                          ch, slots, slot);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    ring_advance<<<1, 1, 0, s>>>(slot, slots);
    return cudaGetLastError();
}

}  // namespace reco
