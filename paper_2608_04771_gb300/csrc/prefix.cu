// prefix.cu -- decode attention of a batch whose sequences share the rows of a prefix: several answers to one question
// (the paper samples several reasoning paths per question), whose rows lie once in the pool, in pages that the group's
// first sequence names.
//
// For a query head with logits x_j over the prefix (j < P) and over its sequence's own rows (j >= P), the softmax over
// both is that of the two parts joined: with M = max(m_p, m_o) to base 2,
//   l = 2^(m_p - M) l_p + 2^(m_o - M) l_o,   out = (2^(m_p - M) o_p + 2^(m_o - M) o_o) / l.
// Four launches: prefix_plan lists the groups; the own part is paged_kernel.cuh's decode kernel, with the prefix out of
// sight; the prefix part reads the prefix's rows once for all query heads of a group; prefix_join joins the parts and
// advances the lengths.
//
// The prefix part: of a layer, KV head and group of n sequences, R = n G query rows are cut into tiles, the P rows of
// the prefix into tiles of 128; the (row tile, key tile) pairs of all layers, heads and groups laid end to end
// (key tiles innermost) are shared out evenly to one CTA per SM.  An item (a row tile against its prefix) that is cut
// between CTAs leaves several partials (max, sum, output); its first one lies by query head, the others by CTA.
#include <algorithm>

#include "decode_block.cuh"
#include "prefix.cuh"

namespace reco {

// ---------------------------------------------------------------- plan
constexpr int kPlanThreads = 1024;

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

__global__ void __launch_bounds__(kPlanThreads) prefix_plan(const int32_t *__restrict__ group, const int32_t *__restrict__ shared,
                                                            int B, int G, int cap, int rows, PrefixRun *runs,
                                                            int32_t *run_of, PrefixTotal *total, unsigned *err)
{
    __shared__ long long sm[kPlanThreads / 32], sm_work;
    __shared__ int sm_start, sm_runs;
    if (threadIdx.x == 0) {
        sm_work = 0;
        sm_start = -1;
        sm_runs = 0;
    }
    wait_prior_grid();
    bool off = false;
    for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
        const int b = b0 + threadIdx.x;
        const bool in = b < B;
        const int g = in ? __ldg(group + b) : 0;
        const bool first = in && (b == 0 || __ldg(group + b - 1) != g), last = in && (b == B - 1 || __ldg(group + b + 1) != g);
        __syncthreads();
        const int c_start = sm_start, c_runs = sm_runs;
        const long long c_work = sm_work;
        const int start = max(c_start, scan_block<true>(first ? b : -1, reinterpret_cast<int *>(sm)));
        const int p = in ? __ldg(shared + start) : 0;
        const bool valid = p >= 0 && p <= cap, kept = in && valid && p > 0 && !(first && last);
        const int run = c_runs + scan_block<false>(first && kept ? 1 : 0, reinterpret_cast<int *>(sm)) - 1;
        const long long mine = last && kept ? prefix_work(b - start + 1, G, p, rows) : 0;
        const long long work = c_work + scan_block<false>(mine, sm);
        if (last && kept) runs[run] = PrefixRun{start, b - start + 1, p, 0, work - mine};
        if (in) {
            const bool wrong = !valid || __ldg(shared + b) != p;
            off |= wrong;
            run_of[b] = wrong ? -2 : (kept ? run : -1);
        }
        __syncthreads();
        if (threadIdx.x == kPlanThreads - 1) {
            sm_start = start;
            sm_runs = run + 1;
            sm_work = work;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) *total = PrefixTotal{sm_work, sm_runs};
    if (off) raise_error(err, ERR_LEN);
}

// ---------------------------------------------------------------- prefix part, float32
// Eight warps.  A warp takes 8 of the tile's query rows and, where the tile has fewer than 64, a share of the keys of
// each tile (WR row groups, 8 / WR key groups).  QK^T: a half-warp has four rows, a lane of it WR keys; PV: a lane has D / 32
// columns of all eight rows and takes the probabilities from shared memory.  Every sum is float32.
constexpr int kPlainRows = 64;

template <int D> constexpr int plain_smem() { return (kPlainRows * D + 2 * kPrefixTile * D + 8 * 8 * kPrefixTile) * 4 + 8 * 8 * 8; }

// Float offset of 16-byte chunk c of row r: rows that lie a multiple of 8 chunks apart spread over the banks.
template <int D> __device__ __forceinline__ int chunk_at(int r, int c) { return r * D + ((c ^ (r & 7)) << 2); }

__device__ __forceinline__ float4 ld4(const float *p) { return *reinterpret_cast<const float4 *>(p); }

template <int D, int WR>
__device__ __forceinline__ void plain_piece(const PrefixArgs &a, const PrefixPiece &pc, float *sm, int *sm_bad)
{
    constexpr int WK = 8 / WR, E = D / 32, KEYS = kPrefixTile / WK;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, rw = wid % WR, kg = wid / WR, half = lane >> 4, l16 = lane & 15;
    float *Q = sm, *K = Q + kPlainRows * D, *V = K + kPrefixTile * D, *ps = V + kPrefixTile * D + wid * 8 * kPrefixTile;
    float2 *ml = reinterpret_cast<float2 *>(V + kPrefixTile * D + 8 * 8 * kPrefixTile);
    const int nrows = pc.nrows;
    __syncthreads();
    if (tid == 0) *sm_bad = 0;
    for (int i = tid; i < 8 * WR * (D / 4); i += 256) {
        const int r = i / (D / 4), c = i % (D / 4);
        *reinterpret_cast<float4 *>(Q + r * D + 4 * c) =
            r < nrows ? ld4((const float *)a.q + a.q_row(pc, pc.rt * kPlainRows + r) * D + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    float o[8][E], m[4], l[4];
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int e = 0; e < E; ++e) o[r][e] = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
    }
    for (int t = pc.t0; t < pc.t1; ++t) {
        const int k0 = t * kPrefixTile, live = min(kPrefixTile, pc.p - k0);
        __syncthreads();  // the last tile has been read
        for (int i = tid; i < kPrefixTile * (D / 4); i += 256) {
            const int r = i / (D / 4), c = i % (D / 4);
            float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
            if (r < live) {
                const long long row = a.pool_row(pc, k0 + r);
                if (row >= 0) {
                    k = ld4((const float *)a.K + row * D + 4 * c);
                    v = ld4((const float *)a.V + row * D + 4 * c);
                } else {
                    *sm_bad = 1;
                }
            }
            *reinterpret_cast<float4 *>(K + chunk_at<D>(r, c)) = k;
            *reinterpret_cast<float4 *>(V + chunk_at<D>(r, c)) = v;
        }
        __syncthreads();
        float s[4][WR];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < WR; ++j) s[r][j] = 0.f;
        const int kb = kg * KEYS + l16;
#pragma unroll 4
        for (int c = 0; c < D / 4; ++c) {
            float4 qv[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) qv[r] = ld4(Q + (rw * 8 + half * 4 + r) * D + 4 * c);
#pragma unroll
            for (int j = 0; j < WR; ++j) {
                const float4 kv = ld4(K + chunk_at<D>(kb + 16 * j, c));
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    s[r][j] = fmaf(qv[r].w, kv.w, fmaf(qv[r].z, kv.z, fmaf(qv[r].y, kv.y, fmaf(qv[r].x, kv.x, s[r][j]))));
            }
        }
        float al[4];
        bool any = false;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float mb = -INFINITY;
#pragma unroll
            for (int j = 0; j < WR; ++j) {
                s[r][j] = kb + 16 * j < live ? s[r][j] * a.c2 : -INFINITY;
                mb = fmaxf(mb, s[r][j]);
            }
#pragma unroll
            for (int x = 1; x < 16; x <<= 1) mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, x));
            const bool grow = mb > m[r] + kLazyLog2;  // lazy rescale, as in the decode's consumers
            const float mn = grow ? mb : m[r];
            al[r] = grow ? fast_exp2(m[r] - mn) : 1.f;
            l[r] *= al[r];
            m[r] = mn;
            any |= grow;
            const float base = mn == -INFINITY ? 0.f : mn;
#pragma unroll
            for (int j = 0; j < WR; ++j) {
                s[r][j] = fast_exp2(s[r][j] - base);
                l[r] += s[r][j];
            }
        }
#pragma unroll
        for (int j = 0; j < WR; ++j)
            *reinterpret_cast<float4 *>(ps + (l16 + 16 * j) * 8 + 4 * half) = make_float4(s[0][j], s[1][j], s[2][j], s[3][j]);
        if (__any_sync(0xffffffffu, any)) {
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const float f = __shfl_sync(0xffffffffu, al[r & 3], (r >> 2) * 16);
#pragma unroll
                for (int e = 0; e < E; ++e) o[r][e] *= f;
            }
        }
        __syncwarp();
// a tile's products are summed before they join the output: the chain of additions into it is as long as the tiles
        float acc[8][E];
#pragma unroll
        for (int r = 0; r < 8; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) acc[r][e] = 0.f;
#pragma unroll 4
        for (int k = 0; k < KEYS; ++k) {
            float v[E];
            const float *vr = V + chunk_at<D>(kg * KEYS + k, lane * E / 4) + (lane * E & 3);
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
            const float4 p0 = ld4(ps + 8 * k), p1 = ld4(ps + 8 * k + 4);
            const float p[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
#pragma unroll
            for (int r = 0; r < 8; ++r)
#pragma unroll
                for (int e = 0; e < E; ++e) acc[r][e] = fmaf(p[r], v[e], acc[r][e]);
        }
#pragma unroll
        for (int r = 0; r < 8; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) o[r][e] += acc[r][e];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], x);
    // the key groups join through shared memory (the tile's place)
    __syncthreads();
    float *os = K + wid * 8 * D;
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int e = 0; e < E; ++e) os[r * D + lane * E + e] = o[r][e];
    if (l16 == 0)
#pragma unroll
        for (int r = 0; r < 4; ++r) ml[wid * 8 + half * 4 + r] = make_float2(m[r], l[r]);
    __syncthreads();
    const bool bad = *sm_bad != 0;
    for (int i = tid; i < nrows * (D / 4); i += 256) {
        const int r = i / (D / 4), c = i % (D / 4), w0 = r >> 3;
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int x = 0; x < WK; ++x) M = fmaxf(M, ml[(w0 + x * WR) * 8 + (r & 7)].x);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int x = 0; x < WK; ++x) {
            const int w = w0 + x * WR;
            const float2 y = ml[w * 8 + (r & 7)];
            const float f = part_factor(y.x, M);
            const float4 v = ld4(K + (w * 8 + (r & 7)) * D + 4 * c);
            L += y.y * f;
            acc.x += v.x * f;
            acc.y += v.y * f;
            acc.z += v.z * f;
            acc.w += v.w * f;
        }
        float *po;
        float2 *pm;
        a.partial<D>(pc, r, po, pm);
        *reinterpret_cast<float4 *>(po + 4 * c) = acc;
        if (c == 0) *pm = make_float2(M, bad ? -1.f : L);
    }
    if (bad && tid == 0) raise_error(a.err, ERR_PAGE);
}

template <int D> __global__ void __launch_bounds__(256, 1) prefix_plain(const __grid_constant__ PrefixArgs a)
{
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ int sm_bad;
    float *sm = reinterpret_cast<float *>(smem_raw);
    wait_prior_grid();
    PrefixWalk w = a.range();
    PrefixPiece pc;
    while (a.next(w, pc)) {
        if (pc.nrows <= 8)
            plain_piece<D, 1>(a, pc, sm, &sm_bad);
        else if (pc.nrows <= 16)
            plain_piece<D, 2>(a, pc, sm, &sm_bad);
        else if (pc.nrows <= 32)
            plain_piece<D, 4>(a, pc, sm, &sm_bad);
        else
            plain_piece<D, 8>(a, pc, sm, &sm_bad);
    }
}

// ---------------------------------------------------------------- join
// One CTA per unit: a query head's own part and the partials of its prefix, in the order of the CTAs.
template <int D> __global__ void __launch_bounds__(128) prefix_join(const __grid_constant__ PrefixJoin a)
{
    wait_prior_grid();
    const int u = blockIdx.x, h = u % a.p.Hkv, lb = u / a.p.Hkv, b = lb % a.p.B, layer = lb / a.p.B, G = a.p.G;
    const int run = a.p.run_of[b], L = a.lens[u];
    PrefixRun rn = {};
    long long total = 0, lh0 = 0, ctas = 1;
    if (run >= 0) {
        rn = a.p.runs[run];
        total = a.p.total->work * a.p.layers * a.p.Hkv;
        ctas = prefix_ctas(total, a.grid, a.p.rows);
        lh0 = ((long long)layer * a.p.Hkv + h) * a.p.total->work;
    }
    const size_t q0 = (size_t)lb * a.p.Hq + (size_t)h * G;
    bool ok = unit_ok(L, a.cap, a.append) && run != -2;
    for (int x = threadIdx.x; x < G * (D / 4); x += blockDim.x) {
        const int g = x / (D / 4), c = x % (D / 4);
        float M = a.own_l2[q0 + g], Ls = M == -INFINITY ? 0.f : 1.f;
        bool err = M == INFINITY || !ok;
        float4 o = ld4(a.own_out + (q0 + g) * D + 4 * c);
        auto add = [&](float2 ml, float4 v) {
            const float Mn = fmaxf(M, ml.x), f = part_factor(M, Mn), k = part_factor(ml.x, Mn);
            err |= ml.y < 0.f;
            Ls = Ls * f + ml.y * k;
            o.x = o.x * f + v.x * k;
            o.y = o.y * f + v.y * k;
            o.z = o.z * f + v.z * k;
            o.w = o.w * f + v.w * k;
            M = Mn;
        };
        if (run >= 0 && !err) {
            const int rows = a.p.rows, r = (b - rn.b0) * G + g, rt = r / rows, kt = (rn.p + kPrefixTile - 1) / kPrefixTile;
            const int unit = prefix_unit(rn.n * G, rt, rows);
            const long long w0 = lh0 + rn.work + (long long)rt * kt * ((rows + 127) / 128);
            const int c0 = prefix_cta(w0, total, ctas);
            int c1 = prefix_cta(w0 + (long long)kt * unit - 1, total, ctas);
            // (the last one may have no more than the end of a key tile, which is the one's before)
            if (c1 > c0 && prefix_begin(c1, total, ctas) - w0 > (long long)(kt - 1) * unit) --c1;
            add(a.p.part_ml[q0 + g], ld4(a.p.part_o + (q0 + g) * D + 4 * c));
            for (int s = c0 + 1; s <= c1; ++s) {
                const size_t at = (size_t)s * a.p.cont_rows + r % rows;
                add(a.p.cont_ml[at], ld4(a.p.cont_o + at * D + 4 * c));
            }
        }
        if (err) {
            Ls = 0.f;
            o = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        const float inv = sum_inverse(Ls);
        const float4 v = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        if (a.out_bf16)
            *reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(a.out) + (q0 + g) * D + 4 * c) =
                make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
        else
            *reinterpret_cast<float4 *>(reinterpret_cast<float *>(a.out) + (q0 + g) * D + 4 * c) = v;
        if (c == 0 && a.lse) a.lse[q0 + g] = sum_log2(M, Ls) * kLn2;
        ok &= !err;
    }
    if (__syncthreads_and(ok) && a.append && threadIdx.x == 0) a.lens[u] = L + 1;
}

// ---------------------------------------------------------------- host side
static int prefix_cont_rows(const reco_paged_kv &kv)
{
    return (int)std::min<long long>(kPrefixMaxRows, (long long)kv.B * (kv.H_q / kv.H_kv));
}

PrefixWs prefix_ws_layout(const reco_paged_kv &kv, void *base)
{
    PrefixWs ws;
    ws.own = paged_decode_ws_layout(kv, false, base);
    size_t off = align256(ws.own.bytes);
    auto take = [&](size_t bytes) {
        char *r = base ? (char *)base + off : nullptr;
        off += align256(bytes);
        return r;
    };
    const size_t heads = (size_t)kv.n_layers * kv.B * kv.H_q;
    const size_t rows = (size_t)prefix_cont_rows(kv) * kPagedMaxGrid;
    ws.run_of = (int32_t *)take((size_t)kv.B * 4);
    ws.runs = (PrefixRun *)take(((size_t)kv.B / 2 + 1) * sizeof(PrefixRun));
    ws.total = (PrefixTotal *)take(sizeof(PrefixTotal));
    ws.own_out = (float *)take(heads * kv.d * 4);
    ws.own_l2 = (float *)take(heads * 4);
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
    const int cap = paged_cap(kv), units = kv.n_layers * kv.B * kv.H_kv, G = kv.H_q / kv.H_kv;
    const int rows = f32 ? kPlainRows : kPrefixMaxRows;
    cudaError_t e = launch_pdl(prefix_plan, dim3(1), dim3(kPlanThreads), 0, s, group, shared, kv.B, G, cap, rows, ws.runs,
                               ws.run_of, ws.total, err);
    if (e != cudaSuccess) return e;
    e = launch_paged_own(kv, q, k_new, v_new, lens, group, shared, scale, ws.own_out, ws.own_l2, ws.own, err, s);
    if (e != cudaSuccess) return e;
    const int grid = std::min(device_sm_count(), kPagedMaxGrid);
    PrefixArgs a = {};
    a.K = kv.k;
    a.V = kv.v;
    a.q = q;
    a.table = kv.table;
    a.runs = ws.runs;
    a.run_of = ws.run_of;
    a.total = ws.total;
    a.part_o = ws.part_o;
    a.part_ml = ws.part_ml;
    a.cont_o = ws.cont_o;
    a.cont_ml = ws.cont_ml;
    a.layers = kv.n_layers;
    a.B = kv.B;
    a.Hq = kv.H_q;
    a.Hkv = kv.H_kv;
    a.G = G;
    a.n_pages = kv.n_pages;
    a.max_pages = kv.max_pages;
    a.shift = __builtin_ctz((unsigned)kv.page);
    a.rows = rows;
    a.cont_rows = prefix_cont_rows(kv);
    a.c2 = scale * kLog2e;
    a.err = err;
    if (f32) {
        void (*fn)(PrefixArgs) = kv.d == 64 ? prefix_plain<64> : prefix_plain<128>;
        const int smem = kv.d == 64 ? plain_smem<64>() : plain_smem<128>();
        if ((e = allow_smem((const void *)fn, smem)) != cudaSuccess) return e;
        if ((e = launch_pdl(fn, dim3(grid), dim3(256), smem, s, a)) != cudaSuccess) return e;
    } else {
        if ((e = launch_prefix_tc(kv, a, grid, out_dtype, s)) != cudaSuccess) return e;
    }
    PrefixJoin j = {};
    j.p = a;
    j.own_out = ws.own_out;
    j.own_l2 = ws.own_l2;
    j.lens = lens;
    j.out = out;
    j.lse = lse;
    j.grid = grid;
    j.cap = cap;
    j.append = k_new ? 1 : 0;
    j.out_bf16 = out_dtype == RECO_BF16 ? 1 : 0;
    e = launch_pdl(kv.d == 64 ? prefix_join<64> : prefix_join<128>, dim3(units), dim3(128), 0, s, j);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace reco
