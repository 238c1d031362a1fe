// Host-side launchers of the client's other steps (internal to the library).
#pragma once

#include "launch.h"

namespace pv {

constexpr int kMostLimit = 1 << 22;  // of integers to write

struct NormJob {
    int T, D;
    bool has_y, has_gate, has_residual;
    pvmvmd_rows y, gate, residual;
    pvmvmd_rows_out residual_out, out;  // data_dev null: not written
    pvmvmd_norm post, pre;              // kind 0: none
    float residual_scale, branch_scale;
};
cudaError_t launch_block_norm(const NormJob &j, cudaStream_t s);

struct GluJob {
    int T, D, act;
    bool has_up;
    pvmvmd_rows gate, up;
    pvmvmd_rows_out out;
};
cudaError_t launch_glu(const GluJob &j, cudaStream_t s);

struct SampleJob {
    int T, V;
    pvmvmd_rows logits;
    pvmvmd_sampling how;
    const uint32_t *allowed, *random;
    int64_t allowed_row;
    int32_t *token;
    float *logprob;
};
cudaError_t launch_sample(const SampleJob &j, cudaStream_t s);

}  // namespace pv
