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
// input rows are fetched while the level ahead still runs; decay and write strength are formed while the states are on their way (ahead of their loads: 10 % more time; by one warp
// for the block: 20 %).  Measured (12 heads of 128 x 128, bf16): 32 sequences x 32 nodes in 5 levels 214 us, 5.4 TB/s of the
// states that have to move; a round of 150 nodes in 6 levels 43 us, bound by the latency of its small levels.
//
// The token-by-token encode keeps the state in registers for the whole sequence; 16 or 32 rows to a block, so that a head of 128 rows is
// a cluster of eight or four blocks, which exchange their sums of squares for the output norm through distributed shared memory.  It is
// bound by the latency of one token's chain (dot product, three shuffles, update): 0.11 to 0.14 us a token where a scheduler has one warp of rows.  So the warps that hold
// the state do nothing else; four helper warps bring the tiles of 16 tokens, and sum, norm, gate and store a tile's outputs while the next is at work
// (fp32, 12 heads of 128 x 128, 512 tokens: 164 us where all warps did both, 72 with the helpers and 16 rows).  Taking the product with the next key ahead of the
// update (by the recurrence of the products, through k_{t-1} . k_t) shortens the chain on paper and won nothing: what it saves it adds in instructions.
#include "chunk_map.cuh"
#include "common.cuh"
#include "gdr.cuh"

namespace mdraft {

namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerPass = kThreads / 8;   // rows of a state that a block holds at eight lanes a row

// Four consecutive activations, as they lie in memory and as two packed pairs of fp32.
__device__ __forceinline__ ulonglong2 load_raw4(const float* p) { return *reinterpret_cast<const ulonglong2*>(p); }
__device__ __forceinline__ uint2 load_raw4(const __nv_bfloat16* p) { return *reinterpret_cast<const uint2*>(p); }
__device__ __forceinline__ ulonglong2 widen(ulonglong2 v) { return v; }
__device__ __forceinline__ ulonglong2 widen(uint2 v) {
    return make_ulonglong2(pk(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u)),
                           pk(__uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)));
}
template <typename T>
__device__ __forceinline__ ulonglong2 load4(const T* p) { return widen(load_raw4(p)); }
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
    const T dt_raw = static_cast<const T*>(p.io.dt)[(size_t)node * p.io.lddt + head], beta_raw = static_cast<const T*>(p.io.beta)[(size_t)node * p.io.ldb + head];
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
    const float alpha = exp_f32(gdr_log_decay(p.L, &dt_raw, head)), beta = gdr_beta(p.L, &beta_raw);   // while the state is on its way
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
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

constexpr int kHelpers = 128, kStages = 3;   // threads beside those that hold the state; tiles in shared memory: at work, to come, and the one whose outputs are formed

template <typename T, int DK, int R>
struct SeqTile {
    T k[kTile][DK], q[kTile][DK], v[kTile][R], z[kTile][R];
    float alpha[kTile], beta[kTile];
};
template <typename T, int DK, int DV, int R>
struct SeqSmem {
    SeqTile<T, DK, R> tile[kStages];
    float so[2][kTile][8 * R];          // outputs, a share from each lane of a row
    float sums[2][DV / R][kTile];       // of squares, by parity of the tile and rank of the block
};

// Blocks to an SM: as many as the registers allow without spills (a token's operands wait as they lie in memory, which for bf16 halves them: eight sequences of up to 9
// tokens x 12 heads a fifth less time, 8.9 us, as three blocks of 384 threads fit instead of two).
template <typename T, int DK, int R>
constexpr int kSeqBlocks = R == 32 ? (DK == 64 || sizeof(T) == 2 ? 3 : 2) : (DK == 64 || sizeof(T) == 2 ? 4 : 3);

__device__ __forceinline__ void helpers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kHelpers) : "memory"); }

// R rows of a state to a block.  Eight lanes of a row do nothing but the recurrence; the helper threads bring the tiles, and form a tile's outputs from the lanes'
// shares while the next tile is at work.
template <typename T, int DK, int DV, int R>
__global__ void __launch_bounds__(8 * R + kHelpers, kSeqBlocks<T, DK, R>) gdr_sequential_kernel(const GdrPrefillArgs p) {
    constexpr int KI = DK / 32, kSlices = DV / R, kVec = 16 / sizeof(T), kRows = R / 8;
    static_assert(kHelpers == 8 * kTile && kSlices <= 8, "eight helpers to a token");
    using Smem = SeqSmem<T, DK, DV, R>;
    extern __shared__ __align__(16) unsigned char s_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(s_raw);
    const int slice = blockIdx.x % kSlices, head = blockIdx.x / kSlices, seq = blockIdx.y;
    const int tid = threadIdx.x, j = tid & 7, row = tid >> 3;
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
    const int col = head * DV + slice * R;   // first channel of the block
    const int n_tiles = (len + kTile - 1) / kTile;
    const bool norm = p.L.norm_w != nullptr;
    if (tid < 8 * R) {
        ulonglong2 S[KI];
        const size_t at = (size_t)(col + row) * DK + 4 * j;
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            S[i] = make_ulonglong2(0ull, 0ull);
            if (islot >= 0) S[i] = *reinterpret_cast<const ulonglong2*>(p.pool.ssm + (size_t)islot * p.pool.ssm_slot_stride + at + 32 * i);
        }
        cluster_arrive();
        cluster_wait();
        __syncthreads();   // the first tile is there
        for (int tile = 0; tile < n_tiles; ++tile) {
            const int n = min(kTile, len - tile * kTile);
            const SeqTile<T, DK, R>& s = sm.tile[tile % kStages];
            float* const so = &sm.so[tile & 1][0][tid];
            if (norm && tile > 0) cluster_arrive_relaxed();   // the helpers' exchange is none of these threads' business, but the barrier counts them
            ulonglong2 k[KI], q[KI];
            decltype(load_raw4(&s.k[0][0])) k_next[KI], q_next[KI];
            float v, alpha, beta, v_next, alpha_next, beta_next;
            auto fetch_next = [&](int t) {   // a token's operands are fetched one token ahead
#pragma unroll
                for (int i = 0; i < KI; ++i) { k_next[i] = load_raw4(&s.k[t][4 * j + 32 * i]); q_next[i] = load_raw4(&s.q[t][4 * j + 32 * i]); }
                v_next = Act<T>::to_f32(s.v[t][row]);
                alpha_next = s.alpha[t];
                beta_next = s.beta[t];
            };
            fetch_next(0);
#pragma unroll 8   // (against 2: a tenth less time for 480 tokens of 64 values, 52.6 us)
            for (int t = 0; t < n; ++t) {
#pragma unroll
                for (int i = 0; i < KI; ++i) { k[i] = widen(k_next[i]); q[i] = widen(q_next[i]); }
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
                const float held = row_sum(sum2(a, b));
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
                so[t * 8 * R] = sum2(c, d);
            }
            if (norm && tile > 0) cluster_wait();
            __syncthreads();   // this tile's outputs are there, and the next tile
        }
        if (norm && n_tiles > 0) cluster_arrive_relaxed();
        if (fslot >= 0 && (len > 0 || fslot != islot)) {
#pragma unroll
            for (int i = 0; i < KI; ++i) *reinterpret_cast<ulonglong2*>(p.pool.ssm + (size_t)fslot * p.pool.ssm_slot_stride + at + 32 * i) = S[i];
        }
        if (norm && n_tiles > 0) cluster_wait();
        return;
    }
    const int h = tid - 8 * R, khead = head / (p.L.n_v_heads / p.L.n_k_heads);
    const int token = h >> 3, l = h & 7;   // eight threads to a token, rows l, l + 8, ..
    const T* kp = static_cast<const T*>(p.io.k) + (size_t)t0 * p.io.ldk + (size_t)khead * DK;
    const T* qp = static_cast<const T*>(p.io.q) + (size_t)t0 * p.io.ldq + (size_t)khead * DK;
    const T* vp = static_cast<const T*>(p.io.v) + (size_t)t0 * p.io.ldv + col;
    const T* zp = p.io.z ? static_cast<const T*>(p.io.z) + (size_t)t0 * p.io.ldz + col : nullptr;
    T dt_raw = Act<T>::from_f32(0.f), beta_raw = dt_raw;   // of a tile to come, a token per thread
    auto fetch = [&](int tile) {   // as far as there are tokens
        const int first = tile * kTile, n = min(kTile, len - first);
        SeqTile<T, DK, R>& s = sm.tile[tile % kStages];
        for (int i = h; i < n * (DK / kVec); i += kHelpers) {
            const int t = i / (DK / kVec), c = i % (DK / kVec) * kVec;
            cp_async16(&s.k[t][c], kp + (size_t)(first + t) * p.io.ldk + c);
            cp_async16(&s.q[t][c], qp + (size_t)(first + t) * p.io.ldq + c);
        }
        for (int i = h; i < n * (R / kVec); i += kHelpers) {
            const int t = i / (R / kVec), c = i % (R / kVec) * kVec;
            cp_async16(&s.v[t][c], vp + (size_t)(first + t) * p.io.ldv + c);
            if (zp) cp_async16(&s.z[t][c], zp + (size_t)(first + t) * p.io.ldz + c);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (h < n) {
            const size_t t = (size_t)(t0 + first + h);
            dt_raw = static_cast<const T*>(p.io.dt)[t * p.io.lddt + head];
            beta_raw = static_cast<const T*>(p.io.beta)[t * p.io.ldb + head];
        }
    };
    auto put_gates = [&](int tile) {
        if (h < kTile) {
            sm.tile[tile % kStages].alpha[h] = exp_f32(gdr_log_decay(p.L, &dt_raw, head));
            sm.tile[tile % kStages].beta[h] = gdr_beta(p.L, &beta_raw);
        }
    };
    float w[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) w[i] = norm ? __ldg(p.L.norm_w + slice * R + 8 * i + l) : 1.f;
    uint32_t rank;   // of the block in its cluster
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    auto outputs = [&](int tile) {
        const int n = min(kTile, len - tile * kTile);
        const SeqTile<T, DK, R>& s = sm.tile[tile % kStages];
        float y[kRows], sq = 0.f;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const float4* part = reinterpret_cast<const float4*>(&sm.so[tile & 1][token][8 * (8 * i + l)]);
            const float4 a = part[0], b = part[1];
            y[i] = (((a.x + a.y) + (a.z + a.w)) + ((b.x + b.y) + (b.z + b.w))) * p.L.scale;
            sq = fmaf(y[i], y[i], sq);
        }
        if (norm) {   // sums of squares of the block's rows, handed to every block of the head
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) sq += __shfl_xor_sync(0xffffffffu, sq, d);
            if (l < kSlices) {
                uint32_t to;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_u32(&sm.sums[tile & 1][rank][token])), "r"(l));
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(sq) : "memory");
            }
            __syncwarp();
            cluster_arrive();
            cluster_wait();
            float all = 0.f;
#pragma unroll
            for (int r = 0; r < kSlices; ++r) all += sm.sums[tile & 1][r][token];
            const float f = rsqrtf(all * (1.0f / DV) + p.L.eps);
#pragma unroll
            for (int i = 0; i < kRows; ++i) y[i] *= f * w[i];
        }
        if (token < n) {
            T* op = static_cast<T*>(p.io.out) + (size_t)(t0 + tile * kTile + token) * p.io.ldo + col + l;
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                if (zp) y[i] *= silu(Act<T>::to_f32(s.z[token][8 * i + l]));
                op[8 * i] = Act<T>::from_f32(y[i]);
            }
        }
    };
    if (n_tiles > 0) {
        fetch(0);
        put_gates(0);
    }
    if (n_tiles > 1) fetch(1);
    __syncwarp();
    cluster_arrive();
    cluster_wait();   // the head's other blocks have begun: their shared memory may be written
    if (n_tiles > 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    for (int tile = 0; tile < n_tiles; ++tile) {
        if (tile > 0) outputs(tile - 1);
        if (tile + 1 < n_tiles) {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            put_gates(tile + 1);
        }
        __syncwarp();
        helpers_sync();   // the gate of the tile ahead has been read
        if (tile + 2 < n_tiles) fetch(tile + 2);
        __syncwarp();
        __syncthreads();
    }
    if (n_tiles > 0) outputs(n_tiles - 1);
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

template <typename T, int DK, int DV, int R>
cudaError_t sequential_rows(const GdrPrefillArgs& p, cudaStream_t st) {
    constexpr int smem = sizeof(SeqSmem<T, DK, DV, R>);
    static_assert(smem <= 113 * 1024, "two blocks to an SM");
    const cudaError_t e = allow_smem<gdr_sequential_kernel<T, DK, DV, R>>(smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.L.n_v_heads * (DV / R), p.n_seq);
    cfg.blockDim = dim3(8 * R + kHelpers);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)(DV / R), 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, gdr_sequential_kernel<T, DK, DV, R>, p);
}

template <typename T, int DK, int DV>
cudaError_t sequential(const GdrPrefillArgs& p, cudaStream_t st) {
    if (gdr_few_rows(p.L.n_v_heads, DV, p.n_seq)) return sequential_rows<T, DK, DV, 16>(p, st);
    return sequential_rows<T, DK, DV, 32>(p, st);
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
