// Launch interface of the head norm with position rotation (internal to the library).
#pragma once

#include "common.cuh"

namespace mdraft {

constexpr int kQkNormMaxRows = 0x7fffffff - 4096;   // the last pass may count this far past the end

struct QkNormArgs {
    const void *q, *k;
    void *q_out, *k_out;
    int64_t ldq, ldk, ldqo, ldko;
    const int32_t* positions;
    const float *q_w, *k_w, *freqs;
    int rows, d_head, n_q_heads, n_k_heads, norm, rot_dim, rot_layout;
    float eps, rot_scale;
};

cudaError_t launch_qk_norm(const QkNormArgs& p, int act, cudaStream_t st);

}  // namespace mdraft
