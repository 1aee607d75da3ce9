// internal.h -- launcher interface between the C ABI layer (api.cu) and the kernels.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/reco.h"

namespace reco {

// Keys per chunk of a unit: a tensor-core scoring pass's work item, and a row partial's keys.
constexpr int kScoreChunk = 2048;
// Decode (m, l, O) partial slots in the workspace: two per warp of a grid of up to
// 256 SMs x 8 warps (the workspace size may not depend on the device; the grid is
// clipped to them).
constexpr int kDecodePartSlots = 4096;
// Sampling: logits per pass-1 segment, and the most segments a row may have.
constexpr int kSampleSeg = 4096;
constexpr int kSampleMaxSeg = 1024;

constexpr size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// First bytes of a paged call's workspace, zero between calls where the call counts in them: nothing else lies
// there, whatever the call and its descriptor, so that one workspace serves them all.  (2560 would do.  What follows
// is read across the GPU, and where it falls in L2 is felt: the eviction of one unit of 131072 rows takes 37.4 us with
// 256, 1024 or 8192 bytes here, 39 to 40.4 with 2048, 4352, 12288 or 16384; other evictions stay within 3%.)
constexpr size_t kPagedZeroBytes = 8192;

struct ScoreWs {  // regions carved from the caller's workspace
    float *part_m, *part_z;  // [units][parts][R]     a part's row reference (log2) / row sum: up to two parts per 2048
                             // keys on the tensor cores, one per 128 keys otherwise
    float *rowb;             // [units][R]            log2 of the row normaliser
    float *raw;              // [units][L_cap]        unpooled scores
    int32_t *ulist;          // [units]               units scored by a planned masked call, ascending
    int32_t *ucount;         // [1]                   entries of ulist
    size_t bytes;
};

// Which units a scoring call covers.  With keep == nullptr every unit; otherwise a
// unit whose sequence keeps its whole cache this time (keep[b] >= lens[unit], the
// selection's no-op) is skipped: none of its keys are read and its scores are not
// written.  A unit with an out-of-range length is never skipped, so it still raises
// the length error.
struct ScoreMask {
    const int32_t *keep;  // [B] or nullptr
    int B, Hkv;
#ifdef __CUDACC__
    __device__ __forceinline__ bool skip(long u, int L, int w, int L_cap) const
    {
        return keep != nullptr && L >= w && L <= L_cap && keep[((int)u / Hkv) % B] >= L;
    }
#endif
};

struct SelectWs {
    int32_t *idx;    // [units][L_cap] kept indices (when the caller passes none)
    int32_t *count;  // [units] rows to compact (0 = skip unit)
    size_t bytes;
};

struct DecodeWs {
    int32_t *counters;  // [0] warps stopped early, [1] finished warps, [2 + w] merge ticket of the unit (or half of one)
                        // that warp w of the grid starts
    float *part_ml;     // [part_slots][G][2]  (m log2, l)
    float *part_o;      // [part_slots][G][d]  unnormalised output
    int part_slots;
    size_t bytes;
};

// Regions of the paged decode's workspace; the last two for calls with weights: the token's
// normalisers and logits.
struct PagedDecodeWs {
    int32_t *counters;  // [2 + CTAs]: [0] stops and errors, [1] CTAs done, [2 + c] ticket of the unit that CTA c starts
    int32_t *cuts;      // [2 + CTAs]: calls with weights: the units cut between CTAs
    float *part_ml;     // [2 * CTAs][G][2]   (m log2, l)
    float *part_o;      // [2 * CTAs][G][d]   unnormalised output
    float *lse2;    // [n_layers * B * H_q]         log2 of the softmax sums
    float *logits;  // [units][cap / 16][G][16]     scale * log2(e) * q . k of a block of 16 rows
    size_t bytes;
};

// Regions of the paged eviction's workspace.  The compaction moves chunks of 2^evict_shift rows.
struct EvictWs {
    int32_t *counters;  // [0] items claimed, [1] chunks and [3] units listed, [2] CTAs done: zero between calls
    int32_t *idx;       // [units][cap] kept rows (when the caller passes none)
    int32_t *rank;      // [units][chunks + 1] kept rows before row i << shift
    int32_t *flags;     // [units][chunks] the chunk's rows have been read
    int4 *list;         // [units * chunks] (unit, chunk, kept rows) to move, a unit's chunks in order
    int32_t *ulist;     // [units] units that are cut
    size_t bytes;
};

ScoreWs score_ws_layout(const reco_kv &kv, int w, void *base);
SelectWs select_ws_layout(const reco_kv &kv, void *base);
DecodeWs decode_ws_layout(const reco_kv &kv, void *base);
PagedDecodeWs paged_decode_ws_layout(const reco_paged_kv &kv, bool weights, void *base);
EvictWs evict_ws_layout(const reco_paged_kv &kv, void *base);

// Rows a unit of the paged cache may hold.
inline int paged_cap(const reco_paged_kv &kv) { return kv.max_pages * kv.page; }
// Chunks of the eviction's compaction: 16 KB of K and 16 KB of V, 128 to 32 rows.
inline int evict_shift(const reco_paged_kv &kv)
{
    const int row = kv.d * (kv.dtype == RECO_F32 ? 4 : 2);
    return row == 128 ? 7 : (row == 256 ? 6 : 5);
}
inline int evict_chunks(const reco_paged_kv &kv) { return (paged_cap(kv) + (1 << evict_shift(kv)) - 1) >> evict_shift(kv); }

// Launchers return cudaSuccess or the launch error.  All arguments validated by the caller.
cudaError_t launch_score(const reco_kv &kv, const void *q_win, const int32_t *lens, const int32_t *keep, int w,
                         int pool, float scale, float *scores, const ScoreWs &ws, unsigned *err, cudaStream_t s);
cudaError_t launch_score_lse(const reco_kv &kv, const void *q_win, const int32_t *lens, const int32_t *keep,
                             const float *row_lse, int w, int pool, float scale, float *scores, const ScoreWs &ws,
                             unsigned *err, cudaStream_t s);
cudaError_t launch_copy_row(const void *src, long long rows, long long row_bytes, const long long *index, void *dst,
                            unsigned *err, cudaStream_t s);
cudaError_t launch_lse_push(const float *lse, long n, float *ring, int slots, long long *slot, unsigned *err,
                            cudaStream_t s);
cudaError_t launch_select_compact(const reco_kv &kv, const float *scores, int32_t *lens,
                                  const int32_t *keep, int w, int32_t *kept_idx, const SelectWs &ws,
                                  unsigned *err, cudaStream_t s);
cudaError_t launch_select_only(const reco_kv &kv, const float *scores, const int32_t *lens, const int32_t *keep,
                               int w, int32_t *kept_idx, const SelectWs &ws, unsigned *err, cudaStream_t s);
cudaError_t launch_compact(const reco_kv &kv, const int32_t *kept_idx, int32_t *lens, const int32_t *keep, int w,
                           unsigned *err, cudaStream_t s);
// ring: optional [2 * slots][layers * B * H_q] lse ring; the launch writes rows *slot and
// *slot + slots and advances *slot.
cudaError_t launch_decode(const reco_kv &kv, const void *q, const void *k_new, const void *v_new,
                          int32_t *lens, float scale, void *out, reco_dtype out_dtype, float *lse,
                          const DecodeWs &ws, unsigned *err, cudaStream_t s, float *ring = nullptr,
                          int slots = 0, long long *slot = nullptr, void *qring = nullptr);
// weights: nullptr, or the running sums that the rows' attention weights are added to.
cudaError_t launch_paged_decode(const reco_paged_kv &kv, const void *q, const void *k_new, const void *v_new,
                                int32_t *lens, float scale, int window, int sinks, void *out, reco_dtype out_dtype,
                                float *lse, float *weights, const PagedDecodeWs &ws, unsigned *err, cudaStream_t s);
cudaError_t launch_paged_evict(const reco_paged_kv &kv, float *weights, int32_t *lens, const int32_t *budget, int w,
                               int sinks, int32_t *kept_idx, const EvictWs &ws, unsigned *err, cudaStream_t s);
// The eviction's selection: kept rows into idx, weights compacted, lens cut, the compaction's list.
cudaError_t launch_select_budget(const reco_paged_kv &kv, float *weights, int32_t *lens, const int32_t *budget, int w,
                                 int sinks, int32_t *idx, const EvictWs &ws, unsigned *err, cudaStream_t s);
cudaError_t launch_penalty(float *logits, int B, int V, const int32_t *ids, int n_ids,
                           const float *rewards, float tau_l, float tau_h, float beta, float *beta_out,
                           unsigned *err, cudaStream_t s);
cudaError_t launch_penalty_sample(float *logits, int B, int V, const int32_t *ids, int n_ids, const float *rewards,
                                  float tau_l, float tau_h, float beta, const float *uniforms, int32_t *tokens,
                                  float *beta_out, float2 *part, unsigned *err, cudaStream_t s);
cudaError_t launch_ppl(const float *logits, const int32_t *tokens, const int32_t *n_valid, int B, int n,
                       int V, float tau_p, float *ppl, uint8_t *stop, float *lp_ws, unsigned *err,
                       cudaStream_t s);

// Device properties cached per device.
int device_sm_count();

// Encode a 2-D tensor map over a row-major bf16 matrix [rows, cols] with boxes of
// box_rows x box_cols elements and 128-byte swizzle (box_cols * 2 <= 128).
// Returns false if the driver entry point is unavailable or the encode fails.
bool encode_bf16_2d(void *map /* CUtensorMap */, const void *base, unsigned long long rows, int cols,
                    int box_cols, int box_rows);

}  // namespace reco
