// One-token forms of the gated delta rule: the draft-tree step and the token-by-token context encode.
//
// Per value head (key head = head / group), with the state S of d_v rows of d_k values:
//
//     alpha = exp(Delta A),   r = beta (v - alpha S k),   S <- alpha S + r k^T,   o = scale S q
//     out = [o rsqrt(mean o^2 + eps) w] [SiLU(z)]
//
// so a row of S needs two dot products of d_k values and one multiply-add per entry, and rows meet only in the output norm.  Eight
// lanes share a row (d_k / 8 values each in registers, two at a time in packed arithmetic); three shuffles finish a dot product.
//
// The tree step is memory traffic: 64 KB read and 64 KB written per node and head of 128 x 128.  A block takes one head of one
// node, 256 threads with four rows per lane group, all of whose loads are in flight before the first is used.  The fork is the gather itself
// (read slot parent_slot[i], write slot node_slot[i]).  Levels of a call are chained by programmatic dependent launch: slots, constants and
// input rows are fetched while the level ahead still runs.
//
// The token-by-token encode keeps the state in registers for the whole sequence; 32 rows to a block, so that a head of 128 rows is
// a cluster of four blocks, which exchange their sums of squares for the output norm through distributed shared memory.  It is
// bound by the latency of one token's chain (dot product, three shuffles, update).
#include "chunk_map.cuh"
#include "common.cuh"
#include "gdr.cuh"

namespace mdraft {

namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerPass = kThreads / 8;   // rows of a state that a block holds at eight lanes a row

// Four consecutive activations as two packed pairs of fp32.
__device__ __forceinline__ ulonglong2 load4(const float* p) { return *reinterpret_cast<const ulonglong2*>(p); }
__device__ __forceinline__ ulonglong2 load4(const __nv_bfloat16* p) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    return make_ulonglong2(pk(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u)),
                           pk(__uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)));
}
__device__ __forceinline__ float sum2(u64 a, u64 b) {
    float x, y, z, w;
    unpk(a, x, y);
    unpk(b, z, w);
    return (x + y) + (z + w);
}
// Sum over the eight lanes of a row; every lane gets it.
__device__ __forceinline__ float row_sum(float v) {
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    v += __shfl_xor_sync(0xffffffffu, v, 2);
    return v + __shfl_xor_sync(0xffffffffu, v, 4);
}

template <typename T, int DK, int DV>
__global__ void __launch_bounds__(kThreads, 2) gdr_step_kernel(const GdrStepArgs p) {
    constexpr int NP = DV / kRowsPerPass, KI = DK / 32;   // rows per lane group; words of four values per lane and row
    __shared__ float so[DV];
    __shared__ float ssum[kThreads / 32];
    grid_release_dependents();   // the next level may begin its own look-ups
    const int node = p.lvl_begin + blockIdx.x, head = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, j = lane & 7, row0 = tid >> 3;
    const int pslot = __ldg(p.parent_slot + node), nslot = __ldg(p.node_slot + node);
    if (pslot < -1 || pslot >= p.pool.n_slots || nslot < 0 || nslot >= p.pool.n_slots) {   // a no-op; every block passes the wait on every path
        if (tid == 0 && head == 0) flag(p.dev_status, MDRAFT_DEV_BAD_SLOT);
        grid_wait();
        return;
    }
    const int khead = head / (p.L.n_v_heads / p.L.n_k_heads);
    const T* kr = static_cast<const T*>(p.io.k) + (size_t)node * p.io.ldk + (size_t)khead * DK + 4 * j;
    const T* qr = static_cast<const T*>(p.io.q) + (size_t)node * p.io.ldq + (size_t)khead * DK + 4 * j;
    const T* vr = static_cast<const T*>(p.io.v) + (size_t)node * p.io.ldv + (size_t)head * DV;
    ulonglong2 k[KI], q[KI];
    float v[NP];
#pragma unroll
    for (int i = 0; i < KI; ++i) { k[i] = load4(kr + 32 * i); q[i] = load4(qr + 32 * i); }
#pragma unroll
    for (int r = 0; r < NP; ++r) v[r] = Act<T>::to_f32(vr[row0 + r * kRowsPerPass]);
    const float alpha = ex2(gdr_log2_decay(p.L, static_cast<const T*>(p.io.dt) + (size_t)node * p.io.lddt + head, head));
    const float beta = gdr_beta(p.L, static_cast<const T*>(p.io.beta) + (size_t)node * p.io.ldb + head);
    float z = 0.f, w = 1.f;
    if (tid < DV) {
        if (p.io.z) z = Act<T>::to_f32(static_cast<const T*>(p.io.z)[(size_t)node * p.io.ldz + (size_t)head * DV + tid]);
        if (p.L.norm_w) w = __ldg(p.L.norm_w + tid);
    }
    const size_t at = ((size_t)head * DV + row0) * DK + 4 * j;
    const float* hp = p.pool.ssm + (size_t)(pslot < 0 ? 0 : pslot) * p.pool.ssm_slot_stride + at;
    float* hc = p.pool.ssm + (size_t)nslot * p.pool.ssm_slot_stride + at;

    grid_wait();   // the parent's state may be the work of the level ahead
    ulonglong2 S[NP][KI];
#pragma unroll
    for (int r = 0; r < NP; ++r)
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            S[r][i] = make_ulonglong2(0ull, 0ull);
            if (pslot >= 0) S[r][i] = *reinterpret_cast<const ulonglong2*>(hp + (size_t)r * kRowsPerPass * DK + 32 * i);
        }
    const u64 al = pk(alpha, alpha);
    float o[NP], sq = 0.f;
#pragma unroll
    for (int r = 0; r < NP; ++r) {
        u64 a = 0ull, b = 0ull;
#pragma unroll
        for (int i = 0; i < KI; ++i) { a = fma2(S[r][i].x, k[i].x, a); b = fma2(S[r][i].y, k[i].y, b); }
        const float held = row_sum(sum2(a, b));
        const float nv = beta * (v[r] - alpha * held);
        const u64 n2 = pk(nv, nv);
        u64 c = 0ull, d = 0ull;
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            S[r][i].x = fma2(n2, k[i].x, mul2(al, S[r][i].x));
            S[r][i].y = fma2(n2, k[i].y, mul2(al, S[r][i].y));
            *reinterpret_cast<ulonglong2*>(hc + (size_t)r * kRowsPerPass * DK + 32 * i) = S[r][i];
            c = fma2(S[r][i].x, q[i].x, c);
            d = fma2(S[r][i].y, q[i].y, d);
        }
        o[r] = row_sum(sum2(c, d)) * p.L.scale;
        sq = fmaf(o[r], o[r], sq);
        if (j == 0) so[row0 + r * kRowsPerPass] = o[r];
    }
    // sum of squares over the head: the four lane groups of a warp, then the warps
    sq += __shfl_xor_sync(0xffffffffu, sq, 8);
    sq += __shfl_xor_sync(0xffffffffu, sq, 16);
    if (lane == 0) ssum[warp] = sq;
    __syncthreads();
    if (tid < DV) {
        float y = so[tid];
        if (p.L.norm_w) {
            float all = 0.f;
#pragma unroll
            for (int i = 0; i < kThreads / 32; ++i) all += ssum[i];
            y *= rsqrtf(all * (1.0f / DV) + p.L.eps) * w;
        }
        if (p.io.z) y *= silu(z);
        static_cast<T*>(p.io.out)[(size_t)node * p.io.ldo + (size_t)head * DV + tid] = Act<T>::from_f32(y);
    }
}

// ---------------------------------------------------------------- token by token
constexpr int kTile = 16;   // tokens staged in shared memory at a time

__device__ __forceinline__ void cp_async16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(__cvta_generic_to_global(src)) : "memory");
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <typename T, int DK>
struct SeqTile {
    T k[kTile][DK], q[kTile][DK], v[kTile][kRowsPerPass], z[kTile][kRowsPerPass];
    float alpha[kTile], beta[kTile];
};

template <typename T, int DK, int DV>
__global__ void __launch_bounds__(kThreads) gdr_sequential_kernel(const GdrPrefillArgs p) {
    constexpr int KI = DK / 32, kSlices = DV / kRowsPerPass, kVec = 16 / sizeof(T);
    __shared__ __align__(16) SeqTile<T, DK> tile[2];
    __shared__ float so[kTile][kRowsPerPass + 1];
    __shared__ float sums[2][kSlices][kTile];   // of squares, by parity of the tile and rank of the block
    const int slice = blockIdx.x % kSlices, head = blockIdx.x / kSlices, seq = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 31, j = lane & 7, row = tid >> 3;
    int t0, len;
    bool bad;
    seq_span(p.cu, p.n_seq, p.T, seq, t0, len, bad);
    if (bad) {   // the whole cluster leaves
        if (tid == 0 && blockIdx.x == 0) flag(p.dev_status, MDRAFT_DEV_BAD_SEQLENS);
        return;
    }
    const int islot = load_slot(p.init_slot, seq), fslot = load_slot(p.final_slot, seq);
    if (islot >= p.pool.n_slots || fslot >= p.pool.n_slots) {
        if (tid == 0 && blockIdx.x == 0) flag(p.dev_status, MDRAFT_DEV_BAD_SLOT);
        return;
    }
    const int khead = head / (p.L.n_v_heads / p.L.n_k_heads);
    const int col = head * DV + slice * kRowsPerPass;   // first channel of the block
    const T* kp = static_cast<const T*>(p.io.k) + (size_t)t0 * p.io.ldk + (size_t)khead * DK;
    const T* qp = static_cast<const T*>(p.io.q) + (size_t)t0 * p.io.ldq + (size_t)khead * DK;
    const T* vp = static_cast<const T*>(p.io.v) + (size_t)t0 * p.io.ldv + col;
    const T* zp = p.io.z ? static_cast<const T*>(p.io.z) + (size_t)t0 * p.io.ldz + col : nullptr;

    auto fetch = [&](int first, SeqTile<T, DK>& s) {   // tokens first .. of the sequence, as far as there are any
        const int n = min(kTile, len - first);
        for (int i = tid; i < n * (DK / kVec); i += kThreads) {
            const int t = i / (DK / kVec), c = i % (DK / kVec) * kVec;
            cp_async16(&s.k[t][c], kp + (size_t)(first + t) * p.io.ldk + c);
            cp_async16(&s.q[t][c], qp + (size_t)(first + t) * p.io.ldq + c);
        }
        for (int i = tid; i < n * (kRowsPerPass / kVec); i += kThreads) {
            const int t = i / (kRowsPerPass / kVec), c = i % (kRowsPerPass / kVec) * kVec;
            cp_async16(&s.v[t][c], vp + (size_t)(first + t) * p.io.ldv + c);
            if (zp) cp_async16(&s.z[t][c], zp + (size_t)(first + t) * p.io.ldz + c);
        }
        if (tid < n) {
            const size_t t = (size_t)(t0 + first + tid);
            s.alpha[tid] = ex2(gdr_log2_decay(p.L, static_cast<const T*>(p.io.dt) + t * p.io.lddt + head, head));
            s.beta[tid] = gdr_beta(p.L, static_cast<const T*>(p.io.beta) + t * p.io.ldb + head);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (len > 0) fetch(0, tile[0]);
    ulonglong2 S[KI];
    const size_t at = (size_t)(col + row) * DK + 4 * j;
#pragma unroll
    for (int i = 0; i < KI; ++i) {
        S[i] = make_ulonglong2(0ull, 0ull);
        if (islot >= 0) S[i] = *reinterpret_cast<const ulonglong2*>(p.pool.ssm + (size_t)islot * p.pool.ssm_slot_stride + at + 32 * i);
    }
    uint32_t rank;   // of the block in its cluster
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    cluster_arrive();
    cluster_wait();   // the head's other blocks have begun: their shared memory may be written
    for (int first = 0, n_tile = 0; first < len; first += kTile, ++n_tile) {
        const int n = min(kTile, len - first);
        SeqTile<T, DK>& s = tile[n_tile & 1];
        if (first + kTile < len) {
            fetch(first + kTile, tile[(n_tile + 1) & 1]);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        __syncthreads();
        // The output of a token is summed over its lanes together with the next token's first product, and a token's operands are fetched one token ahead.
        ulonglong2 k[KI], q[KI], k_next[KI], q_next[KI];
        float v, alpha, beta, v_next, alpha_next, beta_next, pending = 0.f;
        auto fetch_next = [&](int t) {
#pragma unroll
            for (int i = 0; i < KI; ++i) { k_next[i] = load4(&s.k[t][4 * j + 32 * i]); q_next[i] = load4(&s.q[t][4 * j + 32 * i]); }
            v_next = Act<T>::to_f32(s.v[t][row]);
            alpha_next = s.alpha[t];
            beta_next = s.beta[t];
        };
        fetch_next(0);
#pragma unroll 2
        for (int t = 0; t < n; ++t) {
#pragma unroll
            for (int i = 0; i < KI; ++i) { k[i] = k_next[i]; q[i] = q_next[i]; }
            v = v_next; alpha = alpha_next; beta = beta_next;
            fetch_next(min(t + 1, n - 1));
            const u64 al = pk(alpha, alpha);
            u64 a = 0ull, b = 0ull;
#pragma unroll
            for (int i = 0; i < KI; ++i) {
                a = fma2(S[i].x, k[i].x, a);
                b = fma2(S[i].y, k[i].y, b);
                S[i].x = mul2(al, S[i].x);
                S[i].y = mul2(al, S[i].y);
            }
            float held = sum2(a, b);
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) {
                held += __shfl_xor_sync(0xffffffffu, held, d);
                pending += __shfl_xor_sync(0xffffffffu, pending, d);
            }
            if (j == 0 && t > 0) so[t - 1][row] = pending * p.L.scale;
            const float nv = beta * (v - alpha * held);
            const u64 n2 = pk(nv, nv);
            u64 c = 0ull, d = 0ull;
#pragma unroll
            for (int i = 0; i < KI; ++i) {
                S[i].x = fma2(n2, k[i].x, S[i].x);
                S[i].y = fma2(n2, k[i].y, S[i].y);
                c = fma2(S[i].x, q[i].x, c);
                d = fma2(S[i].y, q[i].y, d);
            }
            pending = sum2(c, d);
        }
        pending = row_sum(pending);
        if (j == 0) so[n - 1][row] = pending * p.L.scale;
        __syncthreads();
        if (p.L.norm_w) {
            // sum of squares of the block's rows of each token, handed to every block of the head
            const int t = tid >> 4, l = tid & 15;
            float sq = 0.f;
            if (t < n) sq = so[t][l] * so[t][l] + so[t][l + 16] * so[t][l + 16];
            sq += __shfl_xor_sync(0xffffffffu, sq, 1);
            sq += __shfl_xor_sync(0xffffffffu, sq, 2);
            sq += __shfl_xor_sync(0xffffffffu, sq, 4);
            sq += __shfl_xor_sync(0xffffffffu, sq, 8);
            if (l < kSlices) {
                uint32_t to;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_u32(&sums[n_tile & 1][rank][t])), "r"(l));
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(sq) : "memory");
            }
            cluster_arrive();
            cluster_wait();
        }
        for (int i = tid; i < n * kRowsPerPass; i += kThreads) {
            const int t = i / kRowsPerPass, r = i % kRowsPerPass;
            float y = so[t][r];
            if (p.L.norm_w) {
                float all = 0.f;
#pragma unroll
                for (int l = 0; l < kSlices; ++l) all += sums[n_tile & 1][l][t];
                y *= rsqrtf(all * (1.0f / DV) + p.L.eps) * __ldg(p.L.norm_w + slice * kRowsPerPass + r);
            }
            if (zp) y *= silu(Act<T>::to_f32(s.z[t][r]));
            static_cast<T*>(p.io.out)[(size_t)(t0 + first + t) * p.io.ldo + col + r] = Act<T>::from_f32(y);
        }
        __syncthreads();   // the tile and the outputs are free
    }
    if (fslot >= 0 && (len > 0 || fslot != islot)) {
#pragma unroll
        for (int i = 0; i < KI; ++i) *reinterpret_cast<ulonglong2*>(p.pool.ssm + (size_t)fslot * p.pool.ssm_slot_stride + at + 32 * i) = S[i];
    }
}

template <typename T, int DK, int DV>
cudaError_t step(const GdrStepArgs& p, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.lvl_end - p.lvl_begin, p.L.n_v_heads);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.level_in_call > 0 ? 1 : 0;   // what runs ahead of the first level is usually not this library's
    return cudaLaunchKernelEx(&cfg, gdr_step_kernel<T, DK, DV>, p);
}

template <typename T, int DK, int DV>
cudaError_t sequential(const GdrPrefillArgs& p, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.L.n_v_heads * (DV / kRowsPerPass), p.n_seq);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)(DV / kRowsPerPass), 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, gdr_sequential_kernel<T, DK, DV>, p);
}

// f<T, DK, DV> for the sizes of a call, which the argument checks have narrowed to these.
#define MDRAFT_GDR_SIZES(f, ...)                                                                          \
    do {                                                                                                  \
        if (act == MDRAFT_BF16) {                                                                         \
            if (d_k == 128) return d_v == 128 ? f<__nv_bfloat16, 128, 128>(__VA_ARGS__) : f<__nv_bfloat16, 128, 64>(__VA_ARGS__); \
            return d_v == 128 ? f<__nv_bfloat16, 64, 128>(__VA_ARGS__) : f<__nv_bfloat16, 64, 64>(__VA_ARGS__);                   \
        }                                                                                                 \
        if (d_k == 128) return d_v == 128 ? f<float, 128, 128>(__VA_ARGS__) : f<float, 128, 64>(__VA_ARGS__);                     \
        return d_v == 128 ? f<float, 64, 128>(__VA_ARGS__) : f<float, 64, 64>(__VA_ARGS__);               \
    } while (0)

}  // namespace

cudaError_t launch_gdr_step(const GdrStepArgs& p, int d_k, int d_v, int act, cudaStream_t st) {
    if (p.lvl_end <= p.lvl_begin) return cudaSuccess;
    MDRAFT_GDR_SIZES(step, p, st);
}

cudaError_t launch_gdr_sequential(const GdrPrefillArgs& p, int d_k, int d_v, int act, cudaStream_t st) { MDRAFT_GDR_SIZES(sequential, p, st); }

}  // namespace mdraft
