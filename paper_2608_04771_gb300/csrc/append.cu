// append.cu -- appends new tokens' keys and values to a paged cache, keys (and queries) rotated by the tokens'
// positions on the way.
//
// A pair (x, y) of a row turns by the angle pos * f:  x cos - y sin, y cos + x sin.  The angle is kept in turns, as a
// 64-bit fraction: f / (2 pi), multiplied out in whole numbers with those digits of 1 / (2 pi) that make fractions of a turn (Payne
// and Hanek's reduction, 1983), is rounded to a multiple of 2^-64, and times pos it wraps around at whole turns by itself.  What is
// left is off by 2^-34 turns at most, however far the position (a float32 product pos * f is off by 2^-24 of itself: 0.06
// rad at a position of a million).  Then the nearest quarter of a turn is taken off, exactly, and the rest, an eighth of a turn
// at most either way, is rounded to float32 (2^-28 turns, 0.4 of 2^-24 in rad; half a turn would lose four times that) and goes
// to sincospif.
//
// Every row is read once and written once (bf16, d 128: 256 bytes each way), some ten operations an element: the copy
// rate is the bound, and for a token per sequence the latency of a launch and of the chain starts -> lens -> table.
// A warp takes a token (or, where tokens are few, a slice of its heads): a thread holds the two 16-byte chunks of a row
// that turn together, the same two for every head, so that the sines are computed once for all heads of the token; the
// lanes share them out (a warp of bf16 rows computes 64 pairs of sine and cosine, two a lane).
//
// The lengths are read by every warp and advanced by the last CTA of a layer to finish (atomic count, no waiting).
#include <algorithm>

#include "decode_block.cuh"
#include "internal.h"

namespace reco {

struct AppendArgs {
    char *K, *V;
    const int32_t *table;
    const char *k, *v, *q;
    char *qo;
    long long k_layer, k_token, k_head, v_layer, v_token, v_head, q_layer, q_token, q_head, qo_layer, qo_token, qo_head;  // bytes
    const int32_t *starts, *pos;
    const float *inv_freq;
    int32_t *lens;
    unsigned long long *counters;  // per group of layers: CTAs done << 32 | CTAs that met a page out of range
    int T, B, Hq, Hkv, layers, cap, n_pages, max_pages, shift, rot, slices, iters, n_counters;
    unsigned *err;
};

// Small CTAs, 40 warps of them on an SM (28 layers of 4096 tokens, 7B-class heads: 330 us; with eight warps a CTA 357; two or
// three rows of a lane in flight take registers that cost warps: 368 and 371).
constexpr int kAppendWarps = 4;

// f / (2 pi) in 2^-64 turns, modulo whole turns, rounded (off by 0.51 of them).  f is m 2^e with a whole m below 2^24: the digits
// of 1 / (2 pi) from the e-th behind the point on, 96 of them, times m.  (The same with doubles, in two parts, took 2.5 us of 640
// tokens' 11: an SM has room for few of them at a time.)
__constant__ uint32_t kPerRadian[12] = {0, 0, 0, 0, 0, 0x28be60dbu, 0x9391054au, 0x7f09d5f4u, 0x7d4d3770u, 0x36d8a566u, 0x4f10e410u, 0x7f9458eau};
__device__ __forceinline__ unsigned long long turn_step(float f)
{
    const uint32_t bits = __float_as_uint(f) & 0x7fffffffu, ex = min(bits >> 23, 254u);
    const uint32_t m = ex ? (bits & 0x7fffffu) | 0x800000u : bits;
    const int at = (int)max(ex, 1u) - 150 + 160, shift = at & 31;  // e + 160: 160 zeros stand before the point's digits
    const uint32_t *w = kPerRadian + (at >> 5);
    const uint32_t a = w[0], b = w[1], c = w[2], d = w[3];
    unsigned long long t = (unsigned long long)m * __funnelshift_l(d, c, shift);
    const uint32_t round = (uint32_t)t >> 31;
    t = (unsigned long long)m * __funnelshift_l(c, b, shift) + (t >> 32);
    const uint32_t lo = (uint32_t)t, hi = m * __funnelshift_l(b, a, shift) + (uint32_t)(t >> 32);
    t = ((unsigned long long)hi << 32 | lo) + round;
    return (int)__float_as_uint(f) < 0 ? 0ull - t : t;
}

// Sine and cosine of a phase in 2^-64 turns.
__device__ __forceinline__ void turn_sincos(unsigned long long ph, float &s, float &c)
{
    const unsigned quarter = (unsigned)((ph + (1ull << 61)) >> 62);
    float s0, c0;
    sincospif(__ll2float_rn((long long)(ph - ((unsigned long long)quarter << 62))) * 0x1p-63f, &s0, &c0);
    s = quarter & 1 ? c0 : s0;
    c = quarter & 1 ? -s0 : c0;
    if (quarter & 2) {
        s = -s;
        c = -c;
    }
}

template <typename T> struct Chunk;  // 16 bytes as floats
template <> struct Chunk<__nv_bfloat16> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void unpack(const uint4 &w, float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = i == 0 ? w.x : (i == 1 ? w.y : (i == 2 ? w.z : w.w));
            x[2 * i] = __uint_as_float(u << 16);
            x[2 * i + 1] = __uint_as_float(u & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8])
    {
        return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
};
template <> struct Chunk<float> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void unpack(const uint4 &w, float (&x)[4])
    {
        x[0] = __uint_as_float(w.x);
        x[1] = __uint_as_float(w.y);
        x[2] = __uint_as_float(w.z);
        x[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[4])
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};

// The sequence of token t: the last b with starts[b] <= t, by all lanes of a warp, 32 candidates a turn.
__device__ __forceinline__ int sequence_of(const int32_t *starts, int B, int t, int lane)
{
    int lo = 0, n = B;  // starts[lo] <= t (or lo is 0); candidates lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 31) / 32;
        const int at = lo + lane * step;
        const bool le = lane * step < n && (lane == 0 || __ldg(starts + at) <= t);
        const int k = 31 - __clz(__ballot_sync(0xffffffffu, le));
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

template <typename T, int D, bool PAIRS>
__global__ void __launch_bounds__(32 * kAppendWarps, 10) paged_append(const __grid_constant__ AppendArgs a)
{
    constexpr int E = Chunk<T>::E, PL = D / (2 * E), HP = 32 / PL, A = E / HP;  // chunks of E elements; PL lanes a row
    constexpr int ROW = D * (int)sizeof(T);
    static_assert(A * HP == E, "the lanes that hold the same chunks share their angles");
    __shared__ int sm_bad, sm_last;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, p = lane % PL, hg = lane / PL;
    const int layer = blockIdx.y;
    if (threadIdx.x == 0) sm_bad = 0;
    __syncthreads();
    wait_prior_grid();

    const long long item = (long long)blockIdx.x * kAppendWarps + wid;
    const int t = (int)(item / a.slices), slice = (int)(item - (long long)t * a.slices);
    if (t < a.T) {
        const int b = sequence_of(a.starts, a.B, t, lane);
        const int s0 = __ldg(a.starts + b), s1 = __ldg(a.starts + b + 1);
        if (s0 >= 0 && s0 <= t && t < s1 && s1 <= a.T) {
            const int rp = a.rot / (2 * E);  // lanes of a row whose chunks turn
            // chunks of this lane: those that turn together, behind them the rest in order
            const int c0 = PAIRS ? 2 * p : (p < rp ? p : 2 * p), c1 = PAIRS ? c0 + 1 : (p < rp ? p + rp : c0 + 1);
            float cs[E], sn[E];
            if (a.rot > 0) {
                float mc[A], ms[A];
#pragma unroll
                for (int i = 0; i < A; ++i) {
                    mc[i] = 1.f;
                    ms[i] = 0.f;
                    if (p < rp) {
                        const float f = __ldg(a.inv_freq + p * E + hg * A + i);
                        const unsigned long long ph = turn_step(f) * (unsigned long long)(long long)__ldg(a.pos + t);
                        turn_sincos(ph, ms[i], mc[i]);
                        if (!isfinite(f)) ms[i] = mc[i] = NAN;
                    }
                }
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    cs[e] = __shfl_sync(0xffffffffu, mc[e % A], (e / A) * PL + p);
                    sn[e] = __shfl_sync(0xffffffffu, ms[e % A], (e / A) * PL + p);
                }
            }
            const int heads = 2 * a.Hkv + (a.q ? a.Hq : 0);
            const int it1 = min(a.iters * (slice + 1), (heads + HP - 1) / HP);
            for (int it = a.iters * slice; it < it1; ++it) {
                const int j = it * HP + hg;  // keys, values, then queries
                if (j >= heads) continue;
                const bool is_k = j < a.Hkv, is_v = !is_k && j < 2 * a.Hkv;
                const int h = is_k ? j : (is_v ? j - a.Hkv : j - 2 * a.Hkv);
                const char *src = is_k ? a.k + layer * a.k_layer + t * a.k_token + h * a.k_head
                                       : (is_v ? a.v + layer * a.v_layer + t * a.v_token + h * a.v_head
                                               : a.q + layer * a.q_layer + t * a.q_token + h * a.q_head);
                uint4 x = reinterpret_cast<const uint4 *>(src)[c0], y = reinterpret_cast<const uint4 *>(src)[c1];
                char *dst;
                if (is_k || is_v) {
                    const int L = a.lens[((long long)layer * a.B + b) * a.Hkv + h];
                    if (L < 0 || L > a.cap || s1 - s0 > a.cap - L) continue;  // (the error is the last CTA's to raise)
                    const int row = L + (t - s0), e = __ldg(a.table + (long long)b * a.max_pages + (row >> a.shift));
                    if ((unsigned)e >= (unsigned)a.n_pages) {
                        sm_bad = 1;
                        continue;
                    }
                    const long long r = ((((long long)layer * a.n_pages + e) * a.Hkv + h) << a.shift) + (row & ((1 << a.shift) - 1));
                    dst = (is_k ? a.K : a.V) + r * ROW;
                } else {
                    dst = a.qo + layer * a.qo_layer + t * a.qo_token + h * a.qo_head;
                }
                if (!is_v && p < rp) {
                    float u[E], w[E];
                    Chunk<T>::unpack(x, u);
                    Chunk<T>::unpack(y, w);
                    if constexpr (PAIRS) {
#pragma unroll
                        for (int e = 0; e < E; e += 2) {
                            const float u0 = u[e], w0 = w[e];
                            u[e] = u0 * cs[e / 2] - u[e + 1] * sn[e / 2];
                            u[e + 1] = u[e + 1] * cs[e / 2] + u0 * sn[e / 2];
                            w[e] = w0 * cs[(E + e) / 2] - w[e + 1] * sn[(E + e) / 2];
                            w[e + 1] = w[e + 1] * cs[(E + e) / 2] + w0 * sn[(E + e) / 2];
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            const float u0 = u[e];
                            u[e] = u0 * cs[e] - w[e] * sn[e];
                            w[e] = w[e] * cs[e] + u0 * sn[e];
                        }
                    }
                    x = Chunk<T>::pack(u);
                    y = Chunk<T>::pack(w);
                }
                reinterpret_cast<uint4 *>(dst)[c0] = x;
                reinterpret_cast<uint4 *>(dst)[c1] = y;
            }
        }
    }

    // ---- the last CTA of a group of layers advances their lengths: every other has read them
    __syncthreads();
    const int group = layer % a.n_counters;
    if (threadIdx.x == 0) {
        const unsigned long long add = (1ull << 32) | (sm_bad ? 1ull : 0ull);
        const unsigned long long now = atom_add_acq_rel_u64(a.counters + group, add) + add;
        const unsigned of = gridDim.x * (unsigned)((a.layers - group + a.n_counters - 1) / a.n_counters);
        const bool last = (unsigned)(now >> 32) == of;
        if (last) a.counters[group] = 0ull;
        sm_last = last ? 1 | ((unsigned)now ? 2 : 0) : 0;
    }
    __syncthreads();
    const int last = sm_last;
    if (last == 0) return;
    unsigned bits = 0;
    bool fine = true;  // starts must not decrease, within [0, T]
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
        const int s0 = __ldg(a.starts + b), s1 = __ldg(a.starts + b + 1);
        fine &= s0 >= 0 && s0 <= s1 && s1 <= a.T;
    }
    if (!__syncthreads_and(fine)) {
        if (threadIdx.x == 0) raise_error(a.err, ERR_LEN);
        return;
    }
    const int per = a.B * a.Hkv;
    for (int ly = group; ly < a.layers; ly += a.n_counters)
        for (int x = threadIdx.x; x < per; x += blockDim.x) {
            const int b = x / a.Hkv, n = __ldg(a.starts + b + 1) - __ldg(a.starts + b);
            int32_t *at = a.lens + (long long)ly * per + x;
            const int L = __ldcg(at);
            if (n == 0) continue;
            if (L < 0 || L > a.cap) {
                bits |= ERR_LEN;
                continue;
            }
            if (n > a.cap - L) {
                bits |= ERR_ROOM;
                continue;
            }
            bool ok = true;
            if (last & 2)  // a page out of range was met: which units' it was
                for (int g = L >> a.shift; g <= (L + n - 1) >> a.shift; ++g)
                    ok &= (unsigned)__ldg(a.table + (long long)b * a.max_pages + g) < (unsigned)a.n_pages;
            if (ok) *at = L + n;
            else bits |= ERR_PAGE;
        }
    if (bits) raise_error(a.err, bits);
}

typedef void (*AppendKernel)(AppendArgs);
template <typename T> static AppendKernel append_kernel(int d, bool pairs)
{
    if (d == 64) return pairs ? paged_append<T, 64, true> : paged_append<T, 64, false>;
    return pairs ? paged_append<T, 128, true> : paged_append<T, 128, false>;
}

cudaError_t launch_paged_append(const reco_paged_kv &kv, const reco_rows &k, const reco_rows &v, const reco_rows *q,
                                const reco_rows *q_out, int T, const int32_t *starts, const int32_t *pos,
                                const float *inv_freq, int rot, int interleaved, int32_t *lens, void *ws, unsigned *err,
                                cudaStream_t s)
{
    const bool f32 = kv.dtype == RECO_F32;
    const long long es = f32 ? 4 : 2;
    AppendArgs a = {};
    a.K = (char *)kv.k;
    a.V = (char *)kv.v;
    a.table = kv.table;
    auto set = [&](const reco_rows &r, long long &layer, long long &token, long long &head) {
        layer = r.layer * es;
        token = r.token * es;
        head = r.head * es;
        return (char *)r.p;
    };
    a.k = set(k, a.k_layer, a.k_token, a.k_head);
    a.v = set(v, a.v_layer, a.v_token, a.v_head);
    if (q) {
        a.q = set(*q, a.q_layer, a.q_token, a.q_head);
        a.qo = set(*q_out, a.qo_layer, a.qo_token, a.qo_head);
    }
    a.starts = starts;
    a.pos = pos;
    a.inv_freq = inv_freq;
    a.lens = lens;
    a.counters = (unsigned long long *)((char *)ws + kAppendCounters);
    a.T = T;
    a.B = kv.B;
    a.Hq = kv.H_q;
    a.Hkv = kv.H_kv;
    a.layers = kv.n_layers;
    a.cap = paged_cap(kv);
    a.n_pages = kv.n_pages;
    a.max_pages = kv.max_pages;
    a.shift = __builtin_ctz((unsigned)kv.page);
    a.rot = rot;
    a.n_counters = std::min(kv.n_layers, kAppendGroups);
    a.err = err;
    const int chunk = f32 ? 4 : 8, per_warp = 32 / (kv.d / (2 * chunk));  // rows a warp takes at once
    const int all = (2 * kv.H_kv + (q ? kv.H_q : 0) + per_warp - 1) / per_warp;
    // a warp per token once that fills the GPU (32 warps an SM), a slice of its heads before
    const long long warps = 32ll * device_sm_count(), tokens = (long long)T * kv.n_layers;
    const int want = (int)std::min<long long>(all, std::max<long long>(1, warps / tokens));
    a.iters = (all + want - 1) / want;
    a.slices = (all + a.iters - 1) / a.iters;
    const long long blocks = ((long long)T * a.slices + kAppendWarps - 1) / kAppendWarps;
    const AppendKernel fn = f32 ? append_kernel<float>(kv.d, interleaved != 0) : append_kernel<__nv_bfloat16>(kv.d, interleaved != 0);
    const cudaError_t e = launch_pdl(fn, dim3((unsigned)blocks, (unsigned)kv.n_layers), dim3(32 * kAppendWarps), 0, s, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace reco
