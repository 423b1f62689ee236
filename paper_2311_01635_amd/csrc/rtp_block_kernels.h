// Launch interface between rtp_block.cpp (the entry points around a unit: router, combination, norms, AdamW) and their
// kernels.  Arguments have been checked and leading dimensions filled in; nothing here is zero that the kernels divide by.
#pragma once
#include "../../include/rtp.h"
#include <hip/hip_runtime.h>

namespace rtp {

hipError_t launch_route_fwd(const rtp_route_desc &d, const void *logits, const float *bias, int32_t *ids, float *weights, hipStream_t s);
hipError_t launch_route_bwd(const rtp_route_desc &d, const void *logits, const int32_t *ids, const float *dweights, void *dlogits, hipStream_t s);

struct CombineArgs {
    int64_t T, D;
    int k;
    rtp_dtype dtype;
    const void *dY, *Yk; // backward's inputs; forward: Yk
    int64_t ld_y, ld_yk, ld_dyk;
    const float *weights;
    void *Y;             // forward
    void *dYk;           // backward, may be null
    float *dweights;     // backward, may be null
};
hipError_t launch_combine_fwd(const CombineArgs &a, hipStream_t s);
hipError_t launch_combine_bwd(const CombineArgs &a, hipStream_t s);

hipError_t launch_norm_fwd(const rtp_norm_desc &d, const rtp_norm_io &io, hipStream_t s);
// column sums of the backward pass: which of them a description asks for, one bit each
enum : unsigned { SUM_PRE_W = 1, SUM_PRE_B = 2, SUM_POST_W = 4, SUM_POST_B = 8 };
int norm_bwd_parts(const rtp_norm_desc &d); // rows of partial sums the backward pass leaves at most
hipError_t launch_norm_bwd(const rtp_norm_desc &d, const rtp_norm_grads &g, unsigned sums, hipStream_t s);

// ---- AdamW ---------------------------------------------------------------------------------
// The table in device memory: `count` entries, then for each chunk of ADAMW_CHUNK moments the tensor it belongs to
// (a chunk is within one tensor).
constexpr int ADAMW_CHUNK_BLOCKS = 16, ADAMW_CHUNK = ADAMW_CHUNK_BLOCKS * RTP_ADAMW_BLOCK;
struct AdamwEntry {
    void *param;
    const float *grad;
    float *master;
    int64_t numel;
    int64_t block;   // its first block among all
    int64_t chunk;   // its first chunk among all
    int dtype;
    float weight_decay;
};
struct AdamwArgs {
    const AdamwEntry *entries;
    const int32_t *owner;  // chunk -> entry
    int64_t chunks;
    void *m, *v;
    uint8_t *exps;
    rtp_adamw_scalars sc;
    const rtp_adamw_scalars *sc_dev; // instead of sc where it is not null
    const float *scale;
};
hipError_t launch_adamw(rtp_moments moments, const AdamwArgs &a, hipStream_t s);
hipError_t launch_adamw_moments(rtp_moments moments, rtp_dtype out, const void *m, const void *v, const uint8_t *exps, int64_t blocks,
                                void *m_out, void *v_out, hipStream_t s);

} // namespace rtp
