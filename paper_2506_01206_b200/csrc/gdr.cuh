// Launch interface of the gated-delta-rule kernels (internal to the library).
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace mdraft {

constexpr int kGdrQ = 64;   // tokens per chunk of the chunked context encode

// Per-layer constants as the kernels take them.
struct GdrLayerDev {
    const float* A;        // (Hv)
    const float* dt_bias;  // (Hv) or NULL
    const float* norm_w;   // (d_v) or NULL: no output norm
    int n_k_heads, n_v_heads;
    uint32_t flags;
    float scale, eps;
};

// Activations of a call; rows are tokens or nodes.
struct GdrIo {
    const void *q, *k, *v, *z, *dt, *beta;   // z may be NULL: no gate
    void* out;
    int64_t ldq, ldk, ldv, ldz, lddt, ldb, ldo;
};

struct GdrPrefillArgs {
    GdrLayerDev L;
    PoolDev pool;              // slot = (Hv * d_v, d_k) fp32
    GdrIo io;
    int T, n_seq, n_chunks_bound;
    const int32_t *cu, *init_slot, *final_slot;
    int32_t* dev_status;
};

// Token by token: one kernel, no workspace.  Blocks hold 16 rows of a state where the call has few of them, else 32: 16 rows are one warp to a scheduler, whose tokens take
// 0.12 us instead of 0.16, but the same work is more blocks and more copies of a head's keys.  Measured (16 against 32 rows; 128 x 128): 12 heads x 32 tokens 8.3
// against 10.4 us, fp32 512 tokens 72 against 109, four such 160 against 202; six sequences of 512 in fp32 (3.9 blocks of 16 to an SM) 305 against 305. Beyond, 16 rows lose: eight
// sequences of 32 tokens (5.2 blocks to an SM) 23.6 against 21.1, eight of 512 in fp32 325 against 305.
inline bool gdr_few_rows(int n_v_heads, int d_v, int n_seq) { return (int64_t)n_v_heads * (d_v / 16) * n_seq <= 4 * sm_count(); }
cudaError_t launch_gdr_sequential(const GdrPrefillArgs& p, int d_k, int d_v, int act, cudaStream_t st);

// Scratch of the chunked encode, per (chunk, value head).
constexpr uint32_t kGdrTBytes = 15360, kGdrMBytes = 10240;  // lower triangles in 16 x 16 blocks, as the chain's lanes hold them (T in three parts, M in two)
constexpr uint32_t kGdrWideTBytes = 24576, kGdrWideMBytes = 16384;   // the wide chain's: 64 rows of 128 bytes, 128-byte swizzle, for each part
struct GdrChunkWs {
    unsigned char* T;   // (1 + A)^-1 diag(beta), split into three bf16 values
    unsigned char* M;   // masked products of queries and keys, split into two bf16 values; for the wide chain times T
    float2* ef;         // decays of 64 rows: from the chunk's start, to its end
    float* o;           // (T, Hv * d_v) fp32 outputs before the norm; NULL: there is no norm, or the chain does it
};

// TMA descriptors of one call: boxes of 64 values x 64 rows of q and k, of a slice x 64 rows of v and (for the wide chain, where there is a gate) of z.
struct GdrMaps {
    CUtensorMap q, k, v, z;
};

// Chunks side by side, then a chain over the chunks of each sequence; `slice` = values of a head per block of the chain: 16, or d_v for the wide
// chain.
cudaError_t launch_gdr_chunked(const GdrPrefillArgs& p, const GdrChunkWs& ws, const GdrMaps& maps, int d_k, int d_v, int slice, cudaStream_t st);
cudaError_t launch_gdr_chain_wide(const GdrPrefillArgs& p, const GdrChunkWs& ws, const GdrMaps& maps, int d_k, int d_v, cudaStream_t st);

struct GdrStepArgs {
    GdrLayerDev L;
    PoolDev pool;
    GdrIo io;
    const int32_t *parent_slot, *node_slot;
    int level_in_call;   // kernels this call has launched before this level
    int lvl_begin, lvl_end;
    int32_t* dev_status;
};

cudaError_t launch_gdr_step(const GdrStepArgs& p, int d_k, int d_v, int act, cudaStream_t st);

// ---------------------------------------------------------------- device helpers shared by the kernels
// 2^(hi + lo) to about one unit of the last place (the hardware's 2^x is off by up to four): a decay is multiplied into the state token after token or chunk after
// chunk, so what it is off by adds up over as many as a head remembers (state of 400 fp32 tokens off by 1.4e-6 with the hardware's functions, 2.8e-7 with these).  hi = n + f, and e^y, y = (f + lo) ln 2, by its Taylor series (|y| <= 0.347: what follows y^7 / 7! is
// below 6e-9).  2^n comes in two factors, as n may go past the exponent's range either way.
__device__ __forceinline__ float exp2_f32(float hi, float lo) {
    hi = hi < -252.f ? -252.f : (hi > 252.f ? 252.f : hi);   // (a NaN stays one)
    const float n = rintf(hi), y = ((hi - n) + lo) * kLn2;
    float e = fmaf(y, 1.0f / 5040, 1.0f / 720);
    e = fmaf(y, e, 1.0f / 120);
    e = fmaf(y, e, 1.0f / 24);
    e = fmaf(y, e, 1.0f / 6);
    e = fmaf(y, e, 0.5f);
    e = fmaf(y * y, e, y) + 1.0f;
    const int half = (int)n >> 1, rest = (int)n - half;
    return e * __int_as_float((half + 127) << 23) * __int_as_float((rest + 127) << 23);
}
__device__ __forceinline__ float exp_f32(float x) {
    x = x < -174.f ? -174.f : (x > 174.f ? 174.f : x);
    const float hi = x * kLog2e;
    return exp2_f32(hi, fmaf(x, 1.92596299e-8f, fmaf(x, kLog2e, -hi)));   // log2 e = kLog2e + 1.926e-8
}
// Step size of a token and head times A: the log of its decay.
template <typename T>
__device__ __forceinline__ float gdr_log_decay(const GdrLayerDev& L, const T* dt, int head) {
    const float v = Act<T>::to_f32(*dt) + (L.dt_bias ? __ldg(L.dt_bias + head) : 0.f);
    return ((L.flags & MDRAFT_DT_SOFTPLUS) ? (v > 20.f ? v : log1pf(exp_f32(v))) : v) * __ldg(L.A + head);
}
// Write strength beta (MDRAFT_BETA_SIGMOID: of its pre-activation).
template <typename T>
__device__ __forceinline__ float gdr_beta(const GdrLayerDev& L, const T* b) {
    const float v = Act<T>::to_f32(*b);
    return (L.flags & MDRAFT_BETA_SIGMOID) ? __frcp_rn(1.0f + exp_f32(-v)) : v;
}

}  // namespace mdraft
