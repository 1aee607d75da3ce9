// decode_block.cuh -- what a warp does with a block of cached rows in decode attention: the block
// consumers of decode.cu (contiguous units) and paged.cu (pages), and the helpers they share.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "common.cuh"
#include "tma.cuh"

namespace reco {

constexpr long long kSpinLimit = 1LL << 24;  // bounded mbarrier waits (about a second)
constexpr float kLazyLog2 = 8.f;             // output rescale threshold (log2 units)

// atomicAdd with acquire-release semantics at GPU scope.
__device__ __forceinline__ int atom_add_acq_rel(int *p, int v)
{
    int old;
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], %2;" : "=r"(old) : "l"(p), "r"(v) : "memory");
    return old;
}

__device__ __forceinline__ unsigned long long atom_add_acq_rel_u64(unsigned long long *p, unsigned long long v)
{
    unsigned long long old;
    asm volatile("atom.acq_rel.gpu.global.add.u64 %0, [%1], %2;" : "=l"(old) : "l"(p), "l"(v) : "memory");
    return old;
}

__device__ __forceinline__ bool unit_ok(int L, int L_cap, int append)
{
    return L >= 0 && L <= L_cap && (!append || L < L_cap);
}

// What the sum of a softmax (l, of maximum m, to base 2) leaves: the factor of the output, and the sum's logarithm.  A
// sum of zero is that of no rows, or of logits that are all -inf: zeros and -inf.  Anything else goes by its value,
// so that a NaN among the logits (of a query, of a row in sight; an infinite logit is one of them when its maximum is
// taken away) comes out as NaN.  m may still be -inf then: NaN raises no maximum.
__device__ __forceinline__ float sum_inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float sum_log2(float m, float l) { return l == 0.f ? -INFINITY : m + log2f(l); }
// What a part's sum and output, of maximum m, are multiplied by where parts of maximum M, the largest, join.
__device__ __forceinline__ float part_factor(float m, float M) { return fast_exp2(m - (M == -INFINITY ? 0.f : M)); }

__device__ __forceinline__ void store_out(void *out, bool bf16, size_t i, float v)
{
    if (bf16)
        reinterpret_cast<__nv_bfloat16 *>(out)[i] = __float2bfloat16_rn(v);
    else
        reinterpret_cast<float *>(out)[i] = v;
}

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&v);
}

// (a, b) -> bf16x2 hi = round(a, b) and lo = round((a, b) - hi).
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t &hi, uint32_t &lo)
{
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    const float2 f = __bfloat1622float2(h);
    hi = *reinterpret_cast<uint32_t *>(&h);
    lo = pack_bf16(a - f.x, b - f.y);
}

__device__ __forceinline__ uint32_t word(const uint4 &v, int x)
{
    return x == 0 ? v.x : (x == 1 ? v.y : (x == 2 ? v.z : v.w));
}

// Byte offset of 16-byte chunk ch (0..7) of row rr inside a 128B-swizzled 16-row box.
__device__ __forceinline__ uint32_t swz(int rr, int ch) { return rr * 128 + ((ch ^ (rr & 7)) << 4); }

// Where row k of a block of 16 lies among a head's 16 logits: as the bf16 product leaves them, four to a lane (rows
// 2 c, 2 c + 1, 2 c + 8, 2 c + 9), so that a warp stores a block of all its heads in whole lines (the 7B-class stack
// of 4K rows, calls with weights, from 8-byte stores a head apart: 345 -> 342 us).
__host__ __device__ constexpr int logit_place(int k) { return 4 * ((k & 7) >> 1) + 2 * (k >> 3) + (k & 1); }

// A block consumer holds one item's queries, running (max, sum) and output in a warp's registers
// and takes the item's keys in blocks of KB rows from the warp's ring.  It says how a block is
// copied (load), where a 16-byte chunk of a row lies in a stage (chunk), and how results leave.

// bf16: QK^T and PV run on mma.sync m16n8k16 with NT * 8 query heads per unit.  The QK tile has
// 16 query rows: heads 0-7 fill its first eight, heads 8-15 (NT = 2) the others, which cost the
// product nothing more; PV takes one 8-head column tile per NT.
template <class T> struct Tag {
    using type = T;
};

template <int D_, int NT_, int HALVES_ = 1> struct Bf16Block {
    static constexpr int D = D_, NT = NT_, KB = 16, GM = 8 * NT;
    // units run as two halves of their heads (HALVES = 2), or may (NT = 2): then by consumer Half
    static constexpr bool SPLIT = NT == 2 || HALVES_ == 2, ALWAYS = HALVES_ == 2;
    using Half = Bf16Block<D_, 1, HALVES_>;
    static constexpr int ROW = 2 * D, HALVES = D / 64, TILE = 16 * 128, MT = D / 16;
    static constexpr int APP = (2 * ROW / 16 + 31) / 32, SCRATCH = 0;
    static constexpr bool TENSOR_MAPS = true, PREFETCH_Q = NT == 1;
    using RowIndex = int;  // tensor-map coordinates
    // half the warps with deeper rings for long work: with up to eight heads a block leaves a warp
    // waiting for data
    static constexpr bool DEEP = true;

    uint32_t qa[D / 16][2 * NT], qn[PREFETCH_Q ? D / 16 : 1][2 * NT];
    float o[NT][MT][4], m[NT], l[NT];
    const __nv_bfloat16 *q_src = nullptr;
    int nh_src = 0;
    const int g, c;

    static_assert(NT_ == 1 || HALVES_ == 1, "sixteen heads need no halves");
    __device__ __forceinline__ Bf16Block(int lane, float *) : g(lane >> 2), c(lane & 3) {}

    __device__ static __forceinline__ uint32_t chunk(int row, int ch) { return (ch >> 3) * TILE + swz(row, ch & 7); }

    // 128-byte swizzled 16 x 64 boxes of K, then of V, from row y of the tensor maps (whole boxes: rows past
    // the item are masked)
    __device__ static __forceinline__ void load(uint32_t dst, uint32_t bar, const CUtensorMap *tmK,
                                                const CUtensorMap *tmV, const void *, const void *, int y, int,
                                                uint64_t policy)
    {
        mbar_expect_tx(bar, 2 * HALVES * TILE);
#pragma unroll
        for (int hh = 0; hh < HALVES; ++hh) {
            tma_load_2d_hint(dst + hh * TILE, tmK, 64 * hh, y, bar, policy);
            tma_load_2d_hint(dst + (HALVES + hh) * TILE, tmV, 64 * hh, y, bar, policy);
        }
    }

    // Q fragments, the head dim permuted to match the K chunks: k-step j = 4*hh + 2*e + half takes
    // elements 64*hh + 16c + 8e + 4*half + {0,1} and + {2,3} (of rows g, then g + 8)
    __device__ __forceinline__ void fragments(const __nv_bfloat16 *q, int nh, uint32_t (&f)[D / 16][2 * NT]) const
    {
#pragma unroll
        for (int hh = 0; hh < HALVES; ++hh)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint4 wv = make_uint4(0, 0, 0, 0);
                    if (g + 8 * n < nh) wv = *reinterpret_cast<const uint4 *>(q + (g + 8 * n) * D + 64 * hh + 16 * c + 8 * e);
                    const int j = 4 * hh + 2 * e;
                    f[j][n] = wv.x;
                    f[j][NT + n] = wv.y;
                    f[j + 1][n] = wv.z;
                    f[j + 1][NT + n] = wv.w;
                }
    }

    // the queries of the item that start() will begin
    __device__ __forceinline__ void load_q(const void *q, long qrow, int nh)
    {
        q_src = reinterpret_cast<const __nv_bfloat16 *>(q) + qrow * D;
        nh_src = nh;
        if constexpr (PREFETCH_Q) fragments(q_src, nh, qn);
    }

    __device__ __forceinline__ void start()
    {
        if constexpr (PREFETCH_Q) {
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
                for (int n = 0; n < 2 * NT; ++n) qa[j][n] = qn[j][n];
        } else {
            fragments(q_src, nh_src, qa);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = -INFINITY;
            l[n] = 0.f;
#pragma unroll
            for (int t = 0; t < MT; ++t) o[n][t][0] = o[n][t][1] = o[n][t][2] = o[n][t][3] = 0.f;
        }
    }

    // The block of rows kb, kb + 1, ... below k1, rows [h0, h1) out of sight.  `lg`: or nullptr, where the block's
    // base-2 logits go: 16 floats per head, of nh, in the order of logit_place.
    __device__ __forceinline__ void consume(uint32_t Ks, uint32_t Vs, int kb, int k1, float c2, int h0 = 0, int h1 = 0,
                                            float *lg = nullptr, int nh = 0)
    {
        // four accumulators (keys 0-7 / 8-15, even / odd k-steps): dependent MMA chains
        // of D/32 instead of D/16
        float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
        float t0[4] = {0.f, 0.f, 0.f, 0.f}, t1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int hh = 0; hh < HALVES; ++hh)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint4 ka = lds_u4(Ks + hh * TILE + swz(g, 2 * c + e));
                const uint4 kc = lds_u4(Ks + hh * TILE + swz(8 + g, 2 * c + e));
                const int j = 4 * hh + 2 * e;
                const uint32_t a1 = NT == 2 ? qa[j][1 % (2 * NT)] : 0u, a3 = NT == 2 ? qa[j][3 % (2 * NT)] : 0u;
                const uint32_t b1 = NT == 2 ? qa[j + 1][1 % (2 * NT)] : 0u, b3 = NT == 2 ? qa[j + 1][3 % (2 * NT)] : 0u;
                mma_bf16(s0, qa[j][0], a1, qa[j][NT], a3, ka.x, ka.y);
                mma_bf16(s1, qa[j][0], a1, qa[j][NT], a3, kc.x, kc.y);
                mma_bf16(t0, qa[j + 1][0], b1, qa[j + 1][NT], b3, ka.z, ka.w);
                mma_bf16(t1, qa[j + 1][0], b1, qa[j + 1][NT], b3, kc.z, kc.w);
            }
        uint32_t ph[NT][2], pl[NT][2];
        const int kA = kb + 2 * c, kB = kb + 8 + 2 * c;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            // scores of query g + 8n for keys kb+2c, kb+2c+1, kb+8+2c, kb+9+2c
            auto seen = [&](int k) { return k < k1 && (k < h0 || k >= h1); };
            const float x0 = seen(kA) ? (s0[2 * n] + t0[2 * n]) * c2 : -INFINITY;
            const float x1 = seen(kA + 1) ? (s0[2 * n + 1] + t0[2 * n + 1]) * c2 : -INFINITY;
            const float x2 = seen(kB) ? (s1[2 * n] + t1[2 * n]) * c2 : -INFINITY;
            const float x3 = seen(kB + 1) ? (s1[2 * n + 1] + t1[2 * n + 1]) * c2 : -INFINITY;
            if (lg != nullptr && g + 8 * n < nh)
                *reinterpret_cast<float4 *>(lg + 16 * (g + 8 * n) + 4 * c) = make_float4(x0, x1, x2, x3);
            float mb = fmaxf(fmaxf(x0, x1), fmaxf(x2, x3));
            mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, 1));
            mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, 2));
            // Lazy rescale: a row's reference max m moves only when a block max exceeds it
            // by more than 2^kLazyLog2, so probabilities against a stale m stay <= 2^8
            // (exact in fp32, and the bf16 hi + lo split keeps 16 bits of them); the
            // output rescale below then runs on few blocks.  m, l and o stay consistent, so
            // o / l and lse = m + log2 l are the same quantities as with an exact max.
            const bool grow = mb > m[n] + kLazyLog2;
            if (__any_sync(0xffffffffu, grow)) {
                const float mn = grow ? mb : m[n];
                const float alpha = grow ? fast_exp2(m[n] - mn) : 1.f;  // m = -inf gives 0
                l[n] *= alpha;
                m[n] = mn;
                const float al0 = __shfl_sync(0xffffffffu, alpha, (2 * c) * 4);
                const float al1 = __shfl_sync(0xffffffffu, alpha, (2 * c + 1) * 4);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    o[n][t][0] *= al0;
                    o[n][t][1] *= al1;
                    o[n][t][2] *= al0;
                    o[n][t][3] *= al1;
                }
            }
            const float base = (m[n] == -INFINITY) ? 0.f : m[n];
            const float p0 = fast_exp2(x0 - base), p1 = fast_exp2(x1 - base);
            const float p2 = fast_exp2(x2 - base), p3 = fast_exp2(x3 - base);
            l[n] += (p0 + p1) + (p2 + p3);
            // P enters the PV product as bf16 hi + lo parts (two MMAs), which keeps about
            // 16 significant bits of each probability instead of 8.
            split_bf16(p0, p1, ph[n][0], pl[n][0]);
            split_bf16(p2, p3, ph[n][1], pl[n][1]);
        }
#pragma unroll
        for (int hh = 0; hh < HALVES; ++hh) {
            const uint4 v0 = lds_u4(Vs + hh * TILE + swz(2 * c, g));
            const uint4 v1 = lds_u4(Vs + hh * TILE + swz(2 * c + 1, g));
            const uint4 v2 = lds_u4(Vs + hh * TILE + swz(2 * c + 8, g));
            const uint4 v3 = lds_u4(Vs + hh * TILE + swz(2 * c + 9, g));
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t W0 = word(v0, x), W1 = word(v1, x), W2 = word(v2, x), W3 = word(v3, x);
                const uint32_t A0 = __byte_perm(W0, W1, 0x5410), A1 = __byte_perm(W0, W1, 0x7632);
                const uint32_t A2 = __byte_perm(W2, W3, 0x5410), A3 = __byte_perm(W2, W3, 0x7632);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    mma_bf16(o[n][4 * hh + x], A0, A1, A2, A3, ph[n][0], ph[n][1]);
                    mma_bf16(o[n][4 * hh + x], A0, A1, A2, A3, pl[n][0], pl[n][1]);
                }
            }
        }
    }

    __device__ __forceinline__ void finish()
    {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            l[n] += __shfl_xor_sync(0xffffffffu, l[n], 1);
            l[n] += __shfl_xor_sync(0xffffffffu, l[n], 2);
        }
    }

    template <typename F> __device__ __forceinline__ void each_lse(int G, F f) const
    {
#pragma unroll
        for (int n = 0; n < NT; ++n)
            if (c == 0 && g + 8 * n < G) f(g + 8 * n, m[n], l[n]);
    }

    __device__ __forceinline__ void store(void *out, bool bf16, long qrow0, int G) const
    {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int q0 = 8 * n + 2 * c, q1 = q0 + 1;
            const float l0 = __shfl_sync(0xffffffffu, l[n], 8 * c), l1 = __shfl_sync(0xffffffffu, l[n], 8 * c + 4);
            const float inv0 = sum_inverse(l0), inv1 = sum_inverse(l1);
#pragma unroll
            for (int hh = 0; hh < HALVES; ++hh) {
                const long d0 = 64 * hh + 8 * g;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float *v = o[n][4 * hh + x];
                    if (q0 < G) {
                        store_out(out, bf16, (qrow0 + q0) * D + d0 + 2 * x, v[0] * inv0);
                        store_out(out, bf16, (qrow0 + q0) * D + d0 + 2 * x + 1, v[2] * inv0);
                    }
                    if (q1 < G) {
                        store_out(out, bf16, (qrow0 + q1) * D + d0 + 2 * x, v[1] * inv1);
                        store_out(out, bf16, (qrow0 + q1) * D + d0 + 2 * x + 1, v[3] * inv1);
                    }
                }
            }
        }
    }

    __device__ __forceinline__ void store_partial(float *po, int G) const
    {
#pragma unroll
        for (int n = 0; n < NT; ++n) store_tile(n, po + (size_t)8 * n * D, G - 8 * n);
    }

    // heads 8 n .. 8 n + 7, of which the first G are there
    __device__ __forceinline__ void store_tile(int n, float *po, int G) const
    {
        const int q0 = 2 * c, q1 = q0 + 1;
#pragma unroll
        for (int hh = 0; hh < HALVES; ++hh) {
            const int d0 = 64 * hh + 8 * g;
            const float(*v)[4] = &o[n][4 * hh];
            if (q0 < G) {
                float4 *dst = reinterpret_cast<float4 *>(po + (size_t)q0 * D + d0);
                dst[0] = make_float4(v[0][0], v[0][2], v[1][0], v[1][2]);
                dst[1] = make_float4(v[2][0], v[2][2], v[3][0], v[3][2]);
            }
            if (q1 < G) {
                float4 *dst = reinterpret_cast<float4 *>(po + (size_t)q1 * D + d0);
                dst[0] = make_float4(v[0][1], v[0][3], v[1][1], v[1][3]);
                dst[1] = make_float4(v[2][1], v[2][3], v[3][1], v[3][3]);
            }
        }
    }
};

// float32: plain FMAs in float32 throughout, GT >= G (or half of G) query heads.  In QK^T
// lane (kq = lane / 8, part = lane % 8) holds D / 8 elements of every head's query (32-element
// groups, four at part * 4) and multiplies them with keys kq and kq + 4 of the block; the eight
// parts are then added by halving exchanges that leave each (key, head) sum in one lane.  In PV a
// lane owns D / 32 columns of every head's output and takes the probabilities from shared memory.
template <int D_, int GT_> struct F32Block {
    static constexpr int D = D_, KB = 8, GM = GT_, GT = GT_, E = D / 32, QE = D / 8;
    static constexpr int ROW = 4 * D;
    static constexpr bool SPLIT = GT == 8, ALWAYS = false;  // units of more than 8 heads run as two halves
    using Half = F32Block;
    static constexpr int APP = (2 * ROW / 16 + 31) / 32, SCRATCH = KB * GT;
    static constexpr bool TENSOR_MAPS = false;
    using RowIndex = size_t;
    static constexpr bool DEEP = false;  // bound by its arithmetic: all the warps (93 against 70 us)
    static constexpr int GP = GT == 8 ? 4 : GT;  // heads per turn of the PV product
    static constexpr int VPL = GT == 8 ? 2 : (GT == 6 ? 3 : 1);  // (key, head) sums per lane

    float q[GT][QE], o[GT][E], m[VPL], l[VPL];
    const float *q_src = nullptr;
    int nh_src = 0;
    float *const p_sm;  // [KB][GT] probabilities of the block
    const int lane;

    __device__ __forceinline__ F32Block(int lane_, float *scratch) : p_sm(scratch), lane(lane_) {}

    __device__ static __forceinline__ uint32_t chunk(int row, int ch) { return row * ROW + ch * 16; }

    // `rows` rows of K, then of V, each one contiguous copy (none when only the appended row is left)
    __device__ static __forceinline__ void load(uint32_t dst, uint32_t bar, const CUtensorMap *, const CUtensorMap *,
                                                const void *K, const void *V, size_t row, int rows, uint64_t policy)
    {
        const uint32_t bytes = (uint32_t)max(rows, 0) * ROW;
        mbar_expect_tx(bar, 2 * bytes);
        if (bytes == 0) return;
        const size_t off = row * ROW;
        bulk_load_hint(dst, static_cast<const char *>(K) + off, bytes, bar, policy);
        bulk_load_hint(dst + KB * ROW, static_cast<const char *>(V) + off, bytes, bar, policy);
    }

    __device__ __forceinline__ void load_q(const void *qp, long qrow, int nh)
    {
        q_src = reinterpret_cast<const float *>(qp) + qrow * D;
        nh_src = nh;
    }

    __device__ __forceinline__ void start()
    {
#pragma unroll
        for (int g = 0; g < GT; ++g) {
#pragma unroll
            for (int i = 0; i < QE / 4; ++i) {
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                if (g < nh_src) x = *reinterpret_cast<const float4 *>(q_src + (long)g * D + 32 * i + 4 * (lane & 7));
                q[g][4 * i] = x.x;
                q[g][4 * i + 1] = x.y;
                q[g][4 * i + 2] = x.z;
                q[g][4 * i + 3] = x.w;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) o[g][e] = 0.f;
        }
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            m[v] = -INFINITY;
            l[v] = 0.f;
        }
    }

    // the lane (of kq = 0, first key) and its value that hold head g after the exchanges
    __device__ static __forceinline__ constexpr int lane_of(int g)
    {
        return GT == 8 ? g >> 1 : (GT == 6 ? 2 * (g / 3) : (GT == 4 ? g : 2 * g));
    }
    __device__ static __forceinline__ constexpr int value_of(int g) { return GT == 8 ? g & 1 : (GT == 6 ? g % 3 : 0); }
    __device__ __forceinline__ int head_of(int v) const
    {
        return GT == 8 ? 2 * (lane & 3) + v : (GT == 4 ? lane & 3 : ((lane >> 1) & 1) * VPL + v);
    }

    // Halving exchange over lane bit `bit`: of 2N partial sums this lane keeps the lower N (bit
    // clear) or the upper N, each with its partner's added.
    template <int N> __device__ __forceinline__ void halve(float *s, int bit) const
    {
        const bool up = lane & bit;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float send = up ? s[i] : s[i + N];
            const float keep = up ? s[i + N] : s[i];
            s[i] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
        }
    }

    __device__ __forceinline__ void consume(uint32_t Ks, uint32_t Vs, int kb, int k1, float c2)
    {
        float s[2 * GT];  // keys kq, then kq + 4
#pragma unroll
        for (int i = 0; i < 2 * GT; ++i) s[i] = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t row = Ks + ((lane >> 3) + 4 * k) * ROW + (lane & 7) * 16;
#pragma unroll
            for (int i = 0; i < QE / 4; ++i) {
                const float4 x = lds_f4(row + 128 * i);
#pragma unroll
                for (int g = 0; g < GT; ++g) {
                    float t = s[k * GT + g];
                    t = fmaf(q[g][4 * i], x.x, t);
                    t = fmaf(q[g][4 * i + 1], x.y, t);
                    t = fmaf(q[g][4 * i + 2], x.z, t);
                    s[k * GT + g] = fmaf(q[g][4 * i + 3], x.w, t);
                }
            }
        }
        halve<GT>(s, 4);      // lane bit 2: the key
        halve<GT / 2>(s, 2);  // bit 1: the head's high bit
        if constexpr (GT % 4 == 0) {
            halve<GT / 4>(s, 1);
        } else {  // both lanes keep the sums
#pragma unroll
            for (int v = 0; v < VPL; ++v) s[v] += __shfl_xor_sync(0xffffffffu, s[v], 1);
        }
        const int kk = (lane >> 3) + (lane & 4);  // this lane's key of the block
        float x[VPL], mb[VPL];
        bool any = false;
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            x[v] = kb + kk < k1 ? s[v] * c2 : -INFINITY;
            mb[v] = x[v];
#pragma unroll
            for (int o2 = 4; o2 <= 16; o2 <<= 1) mb[v] = fmaxf(mb[v], __shfl_xor_sync(0xffffffffu, mb[v], o2));
            any |= mb[v] > m[v] + kLazyLog2;
        }
        if (__any_sync(0xffffffffu, any)) {  // lazy rescale, as in the bf16 consumer
            float al[VPL];
#pragma unroll
            for (int v = 0; v < VPL; ++v) {
                const float mn = mb[v] > m[v] + kLazyLog2 ? mb[v] : m[v];
                al[v] = mn == m[v] ? 1.f : fast_exp2(m[v] - mn);  // m = -inf gives 0
                l[v] *= al[v];
                m[v] = mn;
            }
#pragma unroll
            for (int g = 0; g < GT; ++g) {
                const float f = __shfl_sync(0xffffffffu, al[value_of(g)], lane_of(g));
#pragma unroll
                for (int e = 0; e < E; ++e) o[g][e] *= f;
            }
        }
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const float p = fast_exp2(x[v] - (m[v] == -INFINITY ? 0.f : m[v]));
            l[v] += p;
            p_sm[kk * GT + head_of(v)] = p;
        }
        __syncwarp();
        // A block's products are summed before they are added to the output: the chain of additions into it
        // is as long as the item's blocks, not its keys.  Eight heads take the block in two turns
        // (registers).
#pragma unroll
        for (int g0 = 0; g0 < GT; g0 += GP) {
            if (g0 > 0) __syncwarp();
            float acc[GP][E];
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                float p[GP], x[E];
                if constexpr (GP % 4 == 0) {
#pragma unroll
                    for (int g = 0; g < GP; g += 4) {
                        const float4 f = *reinterpret_cast<const float4 *>(p_sm + k * GT + g0 + g);
                        p[g] = f.x;
                        p[g + 1] = f.y;
                        p[g + 2] = f.z;
                        p[g + 3] = f.w;
                    }
                } else {
#pragma unroll
                    for (int g = 0; g < GP; g += 2) {
                        const float2 f = *reinterpret_cast<const float2 *>(p_sm + k * GT + g0 + g);
                        p[g] = f.x;
                        p[g + 1] = f.y;
                    }
                }
                if constexpr (E == 4) {
                    const float4 f = lds_f4(Vs + k * ROW + lane * 16);
                    x[0] = f.x;
                    x[1] = f.y;
                    x[2] = f.z;
                    x[3] = f.w;
                } else {
                    const float2 f = lds_f2(Vs + k * ROW + lane * 8);
                    x[0] = f.x;
                    x[1] = f.y;
                }
#pragma unroll
                for (int g = 0; g < GP; ++g)
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[g][e] = k ? fmaf(p[g], x[e], acc[g][e]) : p[g] * x[e];
            }
#pragma unroll
            for (int g = 0; g < GP; ++g)
#pragma unroll
                for (int e = 0; e < E; ++e) o[g0 + g][e] += acc[g][e];
        }
    }

    __device__ __forceinline__ void finish()
    {
#pragma unroll
        for (int v = 0; v < VPL; ++v)
#pragma unroll
            for (int o2 = 4; o2 <= 16; o2 <<= 1) l[v] += __shfl_xor_sync(0xffffffffu, l[v], o2);
        __syncwarp();  // the probabilities have been read
    }

    template <typename F> __device__ __forceinline__ void each_lse(int G, F f) const
    {
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const int g = head_of(v);
            if (lane == lane_of(g) && g < G) f(g, m[v], l[v]);
        }
    }

    __device__ __forceinline__ void store(void *out, bool bf16, long qrow0, int G) const
    {
#pragma unroll
        for (int g = 0; g < GT; ++g) {
            const float lg = __shfl_sync(0xffffffffu, l[value_of(g)], lane_of(g));
            if (g < G) {
                const float inv = sum_inverse(lg);
#pragma unroll
                for (int e = 0; e < E; ++e) store_out(out, bf16, (qrow0 + g) * D + lane * E + e, o[g][e] * inv);
            }
        }
    }

    __device__ __forceinline__ void store_partial(float *po, int G) const
    {
#pragma unroll
        for (int g = 0; g < GT; ++g)
            if (g < G) {
                float *dst = po + (size_t)g * D + lane * E;
                if constexpr (E == 4) *reinterpret_cast<float4 *>(dst) = make_float4(o[g][0], o[g][1], o[g][2], o[g][3]);
                else *reinterpret_cast<float2 *>(dst) = make_float2(o[g][0], o[g][1]);
            }
    }
};


// float32 in blocks of 16 rows, two or four heads a warp: what a warp spends on a block besides its products (the
// exchanges, the maximum, the vote, the barrier around the probabilities) is latency, and costs the same for
// 16 rows as F32Block's for eight.  Lane (kq = lane / 8, part = lane % 8) multiplies rows kq, kq + 4, kq + 8 and
// kq + 12; halving exchanges over the parts leave each (row, head) sum in one lane.
template <int D_, int GT_> struct F32Wide {
    static constexpr int D = D_, KB = 16, GM = GT_, GT = GT_, E = D / 32, QE = D / 8;
    static constexpr int ROW = 4 * D, APP = (2 * ROW / 16 + 31) / 32, SCRATCH = KB * GT;
    static constexpr bool TENSOR_MAPS = false;
    using RowIndex = size_t;
    static constexpr int VPL = GT / 2;  // heads per lane after the exchanges
    static_assert(GT == 2 || GT == 4, "two or four heads");

    float q[GT][QE], o[GT][E], m[VPL], l[VPL];
    const float *q_src = nullptr;
    int nh_src = 0;
    float *const p_sm;  // [KB][GT] probabilities of the block
    const int lane;

    __device__ __forceinline__ F32Wide(int lane_, float *scratch) : p_sm(scratch), lane(lane_) {}

    __device__ static __forceinline__ uint32_t chunk(int row, int ch) { return row * ROW + ch * 16; }

    // `rows` rows of K, then of V, each one contiguous copy (none when only the appended row is left)
    __device__ static __forceinline__ void load(uint32_t dst, uint32_t bar, const CUtensorMap *, const CUtensorMap *,
                                                const void *K, const void *V, size_t row, int rows, uint64_t policy)
    {
        const uint32_t bytes = (uint32_t)max(rows, 0) * ROW;
        mbar_expect_tx(bar, 2 * bytes);
        if (bytes == 0) return;
        bulk_load_hint(dst, static_cast<const char *>(K) + row * ROW, bytes, bar, policy);
        bulk_load_hint(dst + KB * ROW, static_cast<const char *>(V) + row * ROW, bytes, bar, policy);
    }

    __device__ __forceinline__ void load_q(const void *qp, long qrow, int nh)
    {
        q_src = reinterpret_cast<const float *>(qp) + qrow * D;
        nh_src = nh;
    }

    __device__ __forceinline__ void start()
    {
#pragma unroll
        for (int g = 0; g < GT; ++g) {
#pragma unroll
            for (int i = 0; i < QE / 4; ++i) {
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                if (g < nh_src) x = *reinterpret_cast<const float4 *>(q_src + (long)g * D + 32 * i + 4 * (lane & 7));
                q[g][4 * i] = x.x;
                q[g][4 * i + 1] = x.y;
                q[g][4 * i + 2] = x.z;
                q[g][4 * i + 3] = x.w;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) o[g][e] = 0.f;
        }
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            m[v] = -INFINITY;
            l[v] = 0.f;
        }
    }

    // head v of this lane; the lane (of row 0) and the value that hold head g
    __device__ __forceinline__ int head_of(int v) const { return (lane & 1) * VPL + v; }
    __device__ static __forceinline__ constexpr int lane_of(int g) { return g / VPL; }
    __device__ static __forceinline__ constexpr int value_of(int g) { return g % VPL; }

    template <int N> __device__ __forceinline__ void halve(float *s, int bit) const
    {
        const bool up = lane & bit;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float send = up ? s[i] : s[i + N];
            const float keep = up ? s[i + N] : s[i];
            s[i] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
        }
    }

    __device__ __forceinline__ void consume(uint32_t Ks, uint32_t Vs, int kb, int k1, float c2, int h0, int h1, float *lg,
                                            int nh)
    {
        float s[4 * GT];  // rows kq, kq + 4, kq + 8, kq + 12
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t row = Ks + ((lane >> 3) + 4 * k) * ROW + (lane & 7) * 16;
#pragma unroll
            for (int g = 0; g < GT; ++g) s[k * GT + g] = 0.f;
#pragma unroll
            for (int i = 0; i < QE / 4; ++i) {
                const float4 x = lds_f4(row + 128 * i);
#pragma unroll
                for (int g = 0; g < GT; ++g) {
                    float t = s[k * GT + g];
                    t = fmaf(q[g][4 * i], x.x, t);
                    t = fmaf(q[g][4 * i + 1], x.y, t);
                    t = fmaf(q[g][4 * i + 2], x.z, t);
                    s[k * GT + g] = fmaf(q[g][4 * i + 3], x.w, t);
                }
            }
        }
        halve<2 * GT>(s, 4);   // lane bit 2: rows + 8
        halve<GT>(s, 2);       // bit 1: rows + 4
        halve<GT / 2>(s, 1);   // bit 0: the upper heads
        const int kk = (lane >> 3) + 2 * (lane & 6);  // this lane's row of the block
        const int k = kb + kk;
        const bool seen = k < k1 && (k < h0 || k >= h1);
        float x[VPL], mb[VPL];
        bool any = false;
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            x[v] = seen ? s[v] * c2 : -INFINITY;
            if (lg != nullptr && head_of(v) < nh) lg[16 * head_of(v) + logit_place(kk)] = x[v];
            mb[v] = x[v];
#pragma unroll
            for (int o2 = 2; o2 <= 16; o2 <<= 1) mb[v] = fmaxf(mb[v], __shfl_xor_sync(0xffffffffu, mb[v], o2));
            any |= mb[v] > m[v] + kLazyLog2;
        }
        if (__any_sync(0xffffffffu, any)) {  // lazy rescale, as in the bf16 consumer
            float al[VPL];
#pragma unroll
            for (int v = 0; v < VPL; ++v) {
                const float mn = mb[v] > m[v] + kLazyLog2 ? mb[v] : m[v];
                al[v] = mn == m[v] ? 1.f : fast_exp2(m[v] - mn);  // m = -inf gives 0
                l[v] *= al[v];
                m[v] = mn;
            }
#pragma unroll
            for (int g = 0; g < GT; ++g) {
                const float f = __shfl_sync(0xffffffffu, al[value_of(g)], lane_of(g));
#pragma unroll
                for (int e = 0; e < E; ++e) o[g][e] *= f;
            }
        }
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const float p = fast_exp2(x[v] - (m[v] == -INFINITY ? 0.f : m[v]));
            l[v] += p;
            p_sm[kk * GT + head_of(v)] = p;
        }
        __syncwarp();
        // a block's products are summed before they join the output (F32Block)
        float acc[GT][E];
#pragma unroll
        for (int r = 0; r < KB; ++r) {
            float p[GT], y[E];
            if constexpr (GT == 4) {
                const float4 f = *reinterpret_cast<const float4 *>(p_sm + r * GT);
                p[0] = f.x;
                p[1] = f.y;
                p[2] = f.z;
                p[3] = f.w;
            } else {
                const float2 f = *reinterpret_cast<const float2 *>(p_sm + r * GT);
                p[0] = f.x;
                p[1] = f.y;
            }
            if constexpr (E == 4) {
                const float4 f = lds_f4(Vs + r * ROW + lane * 16);
                y[0] = f.x;
                y[1] = f.y;
                y[2] = f.z;
                y[3] = f.w;
            } else {
                const float2 f = lds_f2(Vs + r * ROW + lane * 8);
                y[0] = f.x;
                y[1] = f.y;
            }
#pragma unroll
            for (int g = 0; g < GT; ++g)
#pragma unroll
                for (int e = 0; e < E; ++e) acc[g][e] = r ? fmaf(p[g], y[e], acc[g][e]) : p[g] * y[e];
        }
#pragma unroll
        for (int g = 0; g < GT; ++g)
#pragma unroll
            for (int e = 0; e < E; ++e) o[g][e] += acc[g][e];
        __syncwarp();  // the probabilities have been read
    }

    __device__ __forceinline__ void finish()
    {
#pragma unroll
        for (int v = 0; v < VPL; ++v)
#pragma unroll
            for (int o2 = 2; o2 <= 16; o2 <<= 1) l[v] += __shfl_xor_sync(0xffffffffu, l[v], o2);
    }

    template <typename F> __device__ __forceinline__ void each_lse(int G, F f) const
    {
#pragma unroll
        for (int v = 0; v < VPL; ++v)
            if (lane < 2 && head_of(v) < G) f(head_of(v), m[v], l[v]);
    }

    __device__ __forceinline__ void store(void *out, bool bf16, long qrow0, int G) const
    {
#pragma unroll
        for (int g = 0; g < GT; ++g) {
            const float lg = __shfl_sync(0xffffffffu, l[value_of(g)], lane_of(g));
            if (g < G) {
                const float inv = sum_inverse(lg);
#pragma unroll
                for (int e = 0; e < E; ++e) store_out(out, bf16, (qrow0 + g) * D + lane * E + e, o[g][e] * inv);
            }
        }
    }

    __device__ __forceinline__ void store_tile(int, float *po, int G) const
    {
#pragma unroll
        for (int g = 0; g < GT; ++g)
            if (g < G) {
                float *dst = po + (size_t)g * D + lane * E;
                if constexpr (E == 4) *reinterpret_cast<float4 *>(dst) = make_float4(o[g][0], o[g][1], o[g][2], o[g][3]);
                else *reinterpret_cast<float2 *>(dst) = make_float2(o[g][0], o[g][1]);
            }
    }
};

}  // namespace reco
