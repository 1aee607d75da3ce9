// own.cu -- paged_kernel.cuh's decode kernel over the rows that are a sequence's own, behind a prefix that it shares
// (prefix.cu): its instances and their launch.
#include "paged_kernel.cuh"

namespace reco {

cudaError_t launch_paged_own(const reco_paged_kv &kv, const void *q, const void *k_new, const void *v_new, int32_t *lens,
                             const int32_t *group, const int32_t *shared, float scale, float *out, float *l2,
                             const PagedDecodeWs &ws, unsigned *err, cudaStream_t s)
{
    const PagedArgs a = [&] {
        PagedArgs x = paged_args(kv, q, k_new, v_new, lens, scale, out, RECO_F32, l2, ws, err);
        x.group = group;
        x.shared = shared;
        return x;
    }();
    const bool f32 = kv.dtype == RECO_F32;
    return launch_paged_kernel(kv, kv.d == 64 ? paged_kernel<64, true>(f32, a.G) : paged_kernel<128, true>(f32, a.G), a, s);
}

}  // namespace reco
