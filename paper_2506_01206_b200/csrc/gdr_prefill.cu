// Chunked context encode of the gated delta rule (bf16 activations).
//
// Over a chunk of Q = 64 tokens, with G_i the running log decay, the recurrence is a triangular system: token i writes
//
//     x_i = beta_i (v_i - e^{G_i} S k_i - sum_{j<i} e^{G_i - G_j} (k_i . k_j) x_j)          S: the chunk's incoming state
//
// so with A_ij = beta_i e^{G_i - G_j} k_i . k_j (j < i) and T = (1 + A)^-1 diag(beta), per value head:
//
//     X  = T (V - e^G (K S^T))                                     what the chunk's tokens write
//     O  = scale (e^G (Q S^T) + (Q K^T o e^{G_i - G_j})_{j <= i} X)
//     S' = e^{G_end} S + (e^{G_end - G} X)^T K
//
// T and the masked products M = scale (Q K^T o e^{..}) need the chunk alone: kernel 1 forms them for all chunks side by side.  What is left is a
// chain over the chunks of a sequence, kernel 2, whose rows of S (values) are independent: a block takes a slice of them.
//
//   1. gdr_chunk_prepare, a block per (value head, chunk): [K; Q] K^T as one product of 128 rows on the tensor cores (tcgen05, operands by
//      TMA), then the triangle's inverse in fp32: its diagonal blocks of 16 by forward substitution, a column per lane, the blocks below by two rounds of
//      products (of the 16s, of the 32s).  Results go to the workspace in the order in which kernel 2's lanes hold them.  Bound by shared-memory
//      latency: 2048 tokens x 12 heads 13 us, 141000 x 12 0.69 ms (for the wide chain, with M T: 64^3 multiply-adds of a chunk and head out of shared memory, which is 84 % busy).
//   2. gdr_chain, a block per (slice of 16 values, value head, sequence): state in registers, three small products per chunk one after another
//      (K S^T; T times the difference; the update), beside them the two of the outputs.  2048 tokens: 66 us, 2 us a chunk whatever the width up to the SMs' number
//      of blocks.  Where there are many chains a block takes a whole head instead (gdr_wide.cu).
//   3. gdr_norm_gate where there is an output norm, which needs all slices of a row (the wide chain does it itself).  10 us for 2048 tokens x 12 heads.
//
// Precision.  States keep fp32 accuracy: q, k, v are bf16 as given; everything else that meets them in a product of the state's path (S, T, the
// differences, X) is split into three bf16 values (24 bits), which costs three products with an exact operand and six where both are
// split.  Two values (16 bits) left an error of 3e-6 in the states.  The outputs' products take S, M and X (the wide chain: S, M T
// and V - e^G (K S^T)) as two values each: what they lose is 2^-16 of the products' sizes, which shows in bf16 outputs only where the products cancel to a hundredth.  With one
// value the largest errors were ten steps of a result there.  Running log decays are summed in 64 bits and kept as two fp32 values, as differences of sums of 10^4 are wanted to 2^-24.
//
// Kernel 2 runs on the warp-level tensor instructions (mma.sync), not on tcgen05: its products are 64 x 16 x 128 and depend on
// one another, so what counts is the way from one to the next (registers to shared memory and back, a barrier) and not the rate.
#include "chunk_map.cuh"
#include "common.cuh"
#include "gdr.cuh"
#include "tensor_core.cuh"

namespace mdraft {

namespace {

constexpr int Q = kGdrQ;
constexpr int kBlocks = 10;                            // 16 x 16 blocks of a lower triangle of 64 x 64
constexpr uint32_t kTBytes = kGdrTBytes, kMBytes = kGdrMBytes, kMPart = kBlocks * 512;
static_assert(kTBytes == 3 * kMPart && kMBytes == 2 * kMPart, "workspace layout");

// ---------------------------------------------------------------- kernel 1
constexpr int kPrepThreads = 128;
constexpr int kPitch = 68;   // floats of a row of A and M

template <int DK>
struct PrepSmem {
    static constexpr int kOperands = DK / 64 * 128 * 128, kMatrices = 2 * Q * kPitch * 4;
    union {
        unsigned char kq[kOperands];   // [K; Q] rows in boxes of 64 values, 128-byte swizzle; free once the product is done, then
        struct {
            float A[Q][kPitch];        // blocks of A, each replaced by its block of the inverse
            float M[Q][kPitch];
        };
    };
    float Z[32][36];               // product on the way to a block of the inverse
    float2 csl[Q];                 // running log2 decay (value, remainder)
    float u[Q];                    // decay from the first row of a row's block to the row
    float v[4][Q];                 // decay from a row to the first row of a later block
    float beta[Q];
    double warp_sum;
    uint64_t bar_tma, bar_mma;
    uint32_t tmem_base;
};

// 16 bytes of a lane's share of a 16 x 16 block at (row0, col0) of a fp32 matrix as the A operand of a warp's product: pairs of neighbouring columns.
__device__ __forceinline__ void operand_pairs(const float (*m)[kPitch], int row0, int col0, int lane, float2 (&v)[4]) {
    const int g = lane >> 2, t = 2 * (lane & 3);
    v[0] = *reinterpret_cast<const float2*>(&m[row0 + g][col0 + t]);
    v[1] = *reinterpret_cast<const float2*>(&m[row0 + g + 8][col0 + t]);
    v[2] = *reinterpret_cast<const float2*>(&m[row0 + g][col0 + t + 8]);
    v[3] = *reinterpret_cast<const float2*>(&m[row0 + g + 8][col0 + t + 8]);
}

// What the state decays by from one token to another, log2.
__device__ __forceinline__ float log2_between(float2 from, float2 to) { return (to.x - from.x) + (to.y - from.y); }

// x as two or three bf16 values, two neighbours at a time.
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = pack_bf(a, b);
    lo = pack_bf(a - bf_lo(hi), b - bf_hi(hi));
}
__device__ __forceinline__ void split3(float a, float b, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
    hi = pack_bf(a, b);
    a -= bf_lo(hi); b -= bf_hi(hi);
    mid = pack_bf(a, b);
    lo = pack_bf(a - bf_lo(mid), b - bf_hi(mid));
}

// Four neighbouring columns of a row times a matrix: sum over k < K of a[k] b[k][0..3], b's rows `pitch` floats apart.
template <int K>
__device__ __forceinline__ float4 small_product(const float* a, const float* b, int pitch) {
    u64 lo = 0ull, hi = 0ull;
#pragma unroll
    for (int k = 0; k < K; k += 4) {
        const float4 x = *reinterpret_cast<const float4*>(a + k);
        const float e[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(b + (k + i) * pitch);
            lo = fma2(pk(e[i], e[i]), y.x, lo);
            hi = fma2(pk(e[i], e[i]), y.y, hi);
        }
    }
    float4 r;
    unpk(lo, r.x, r.y);
    unpk(hi, r.z, r.w);
    return r;
}

template <int DK, bool kWide>
__global__ void __launch_bounds__(kPrepThreads) gdr_chunk_prepare(const GdrPrefillArgs p, const GdrChunkWs ws, const __grid_constant__ GdrMaps maps) {
    extern __shared__ __align__(1024) unsigned char s_raw[];
    PrepSmem<DK>& sm = *reinterpret_cast<PrepSmem<DK>*>(s_raw + ((1024u - (smem_u32(s_raw) & 1023u)) & 1023u));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int head = blockIdx.x, cidx = blockIdx.y + blockIdx.z * gridDim.y;
    grid_wait();
    if (!kWide) grid_release_dependents();
    const ChunkInfo ci = find_chunk(p.cu, p.n_seq, p.T, Q, p.n_chunks_bound, cidx);
    if (ci.seq < 0) return;
    const int rows = ci.t1 - ci.t0;
    const int kcol = head / (p.L.n_v_heads / p.L.n_k_heads) * DK;
    if (tid == 0) {
        mbar_init(&sm.bar_tma, 1);
        mbar_init(&sm.bar_mma, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        mbar_expect_tx(&sm.bar_tma, DK / 64 * 128 * 128);
#pragma unroll
        for (int h = 0; h < DK / 64; ++h) {
            tma_box(sm.kq + h * 16384, &maps.k, kcol + 64 * h, ci.t0, &sm.bar_tma);
            tma_box(sm.kq + h * 16384 + 8192, &maps.q, kcol + 64 * h, ci.t0, &sm.bar_tma);
        }
    }
    if (warp == 3) { test_hold_up(); tmem_alloc(&sm.tmem_base, 64); tc_fence_before(); }
    float beta = 0.f;   // rows past the chunk's end: no decay, nothing written
    double sum = 0.0;
    if (tid < rows) {
        const size_t t = (size_t)(ci.t0 + tid);
        sum = 1.4426950408889634 * gdr_log_decay(p.L, static_cast<const __nv_bfloat16*>(p.io.dt) + t * p.io.lddt + head, head);
        if (sum < -256.0) sum = -256.0;   // no fp32 value survives that, and the running sums behind a step of 10^12 keep their last bits
        beta = gdr_beta(p.L, static_cast<const __nv_bfloat16*>(p.io.beta) + t * p.io.ldb + head);
    }
    // Running sums in 64 bits, kept as two fp32 values: what is wanted is their differences, and a head that forgets at once sums to 10^4.
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double up = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += up;
    }
    if (tid == 31) sm.warp_sum = sum;
    __syncthreads();
    // The wide chain takes all of an SM's tensor memory and then waits for this kernel's end: its blocks may start only once every block here has its own columns, or
    // one that shares an SM with them would wait for theirs for good.
    if (kWide) grid_release_dependents();
    tc_fence_after();
    if (tid < Q) {
        if (warp == 1) sum += sm.warp_sum;
        const float hi = (float)sum;
        sm.csl[tid] = make_float2(hi, (float)(sum - hi));
        sm.beta[tid] = beta;
    }
    __syncthreads();
    if (tid < Q) ws.ef[((size_t)cidx * p.L.n_v_heads + head) * Q + tid] = make_float2(exp2_f32(sm.csl[tid].x, sm.csl[tid].y), exp2_f32(log2_between(sm.csl[tid], sm.csl[Q - 1]), 0.f));
    const uint32_t tmem = sm.tmem_base;
    const bool in_ok = mbar_wait_bounded(&sm.bar_tma, 0u);
    if (in_ok && tid == 0) {
        tc_fence_after();
        const uint64_t d = operand_desc_sw128(smem_u32(sm.kq));
#pragma unroll
        for (int k = 0; k < DK / 16; ++k) {   // rows: keys and queries; columns: keys
            const uint64_t at = d + (uint64_t)(((k >> 2) * 16384 + (k & 3) * 32) >> 4);
            mma_bf16(tmem, at, at, instr_desc(Q, false, false), k > 0);
        }
        mma_commit(&sm.bar_mma);
    }
    // Decays between rows of different 16 x 16 blocks in two factors, both at most 1, by way of the first row of the later block.
    if (tid < Q) sm.u[tid] = ex2(log2_between(sm.csl[tid & ~15], sm.csl[tid]));
    for (int i = tid; i < 96; i += kPrepThreads) {
        const int blk = i < 16 ? 1 : (i < 48 ? 2 : 3), j = i - (blk == 1 ? 0 : (blk == 2 ? 16 : 48));
        sm.v[blk][j] = ex2(log2_between(sm.csl[j], sm.csl[16 * blk]));
    }
    bool ok = in_ok && mbar_wait_bounded(&sm.bar_mma, 0u);
    ok = !__syncthreads_or(!ok);   // the decays are visible, the operands are free
    if (ok) {
        tc_fence_after();
        const bool query = warp >= 2, upper = lane >= 16;   // rows of the odd 16 x 16 blocks
        const int i = tid & 63, rb = i >> 4, c0 = 32 * (warp & 1);
        float* row = query ? sm.M[i] : sm.A[i];
        const float2 mine = sm.csl[i];
        const float f = i < rows ? (query ? p.L.scale : sm.beta[i]) : 0.f, fu = f * sm.u[i];
        const uint32_t t = tmem + ((uint32_t)(warp * 32) << 16);
        auto off_diagonal = [&](const float (&v)[16], int c) {
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float4 d = *reinterpret_cast<const float4*>(&sm.v[rb][c + j]);
                float4 w = make_float4(v[j] * (fu * d.x), v[j + 1] * (fu * d.y), v[j + 2] * (fu * d.z), v[j + 3] * (fu * d.w));
                if (i >= rows) w = make_float4(0.f, 0.f, 0.f, 0.f);   // replaced, not scaled: what is masked may be anything
                *reinterpret_cast<float4*>(row + c + j) = w;
            }
        };
        float a[16], b[16];
        tmem_ld16(t + c0, a);
        tmem_ld16(t + c0 + 16, b);
        if (upper) off_diagonal(a, c0);
        else {
#pragma unroll
            for (int j = 0; j < 16; j += 4) *reinterpret_cast<float4*>(row + c0 + 16 + j) = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        __syncwarp();
        const int last = i < rows ? i - 16 * rb - (query ? 0 : 1) : -1;   // columns of the diagonal block up to here count
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
            float4 w;
            float* e = &w.x;
#pragma unroll
            for (int k = 0; k < 4; ++k) e[k] = j + k <= last ? (upper ? b[j + k] : a[j + k]) * f * ex2(log2_between(sm.csl[16 * rb + j + k], mine)) : 0.f;
            *reinterpret_cast<float4*>(row + 16 * rb + j) = w;
        }
        if (c0 > 0) {
            tmem_ld16(t, a);
            tmem_ld16(t + 16, b);
            off_diagonal(a, 0);
            off_diagonal(b, 16);
        }
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 3) tmem_free(tmem, 64);
    if (!ok) {
        if (tid == 0) {
            flag(p.dev_status, MDRAFT_DEV_WAIT_EXPIRED);
            if (!in_ok) mbar_wait_bounded(&sm.bar_tma, 0u);   // the copies target this block's shared memory: one more bounded chance
        }
        return;
    }
    // (1 + A)^-1 in place, by blocks.  Diagonal blocks of 16: a warp each, a column per lane, x_i = e_i - sum_{j<i} A_ij x_j.
    if (lane < 16) {
        const int o = 16 * warp;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float a = 0.f, b = 0.f;
#pragma unroll
            for (int j = 0; j < i; j += 4) {
                const float4 r = *reinterpret_cast<const float4*>(&sm.A[o + i][o + j]);   // zero from the diagonal on
                a = fmaf(r.x, x[j], a);
                if (j + 1 < i) b = fmaf(r.y, x[j + 1], b);
                if (j + 2 < i) a = fmaf(r.z, x[j + 2], a);
                if (j + 3 < i) b = fmaf(r.w, x[j + 3], b);
            }
            x[i] = (i == lane ? 1.f : 0.f) - (a + b);
        }
        __syncwarp(0xffffu);
#pragma unroll
        for (int i = 0; i < 16; ++i) sm.A[o + i][o + lane] = x[i];
    }
    __syncthreads();
    // Blocks (1, 0) and (3, 2): -T_11 (A_10 T_00); 64 threads each, four columns of a row per thread.
    {
        const int o = (tid >> 6) * 32, r = (tid & 63) >> 2, c = (tid & 3) * 4;
        float4 z = small_product<16>(&sm.A[o + 16 + r][o], &sm.A[o][o + c], kPitch);
        *reinterpret_cast<float4*>(&sm.Z[(tid >> 6) * 16 + r][c]) = z;
        __syncthreads();
        z = small_product<16>(&sm.A[o + 16 + r][o + 16], &sm.Z[(tid >> 6) * 16][c], 36);
        *reinterpret_cast<float4*>(&sm.A[o + 16 + r][o + c]) = make_float4(-z.x, -z.y, -z.z, -z.w);
    }
    __syncthreads();
    // The lower left 32 x 32 likewise, rows r and r + 16.
    {
        const int r = tid >> 3, c = (tid & 7) * 4;
        float4 z0 = small_product<32>(&sm.A[32 + r][0], &sm.A[0][c], kPitch), z1 = small_product<32>(&sm.A[48 + r][0], &sm.A[0][c], kPitch);
        *reinterpret_cast<float4*>(&sm.Z[r][c]) = z0;
        *reinterpret_cast<float4*>(&sm.Z[16 + r][c]) = z1;
        __syncthreads();
        z0 = small_product<16>(&sm.A[32 + r][32], &sm.Z[0][c], 36);   // the upper rows of T_11 end with its first block
        z1 = small_product<32>(&sm.A[48 + r][32], &sm.Z[0][c], 36);
        *reinterpret_cast<float4*>(&sm.A[32 + r][c]) = make_float4(-z0.x, -z0.y, -z0.z, -z0.w);
        *reinterpret_cast<float4*>(&sm.A[48 + r][c]) = make_float4(-z1.x, -z1.y, -z1.z, -z1.w);
    }
    __syncthreads();
    if (kWide) {
        // Rows of 64 values: T in three parts, M T diag(beta) in two.  A thread takes eight columns of rows lane and lane + 32; columns u and 7 - u, so that every warp has as
        // much of the triangle.
        unsigned char* to_T = ws.T + ((size_t)cidx * p.L.n_v_heads + head) * kGdrWideTBytes;
        unsigned char* to_M = ws.M + ((size_t)cidx * p.L.n_v_heads + head) * kGdrWideMBytes;
#pragma unroll 1
        for (int n = 0; n < 2; ++n) {
            const int u = n ? 7 - warp : warp, c = 8 * u;
            float b[8];
            *reinterpret_cast<float4*>(b) = *reinterpret_cast<const float4*>(&sm.beta[c]);
            *reinterpret_cast<float4*>(b + 4) = *reinterpret_cast<const float4*>(&sm.beta[c + 4]);
            u64 acc[2][4] = {};
            auto add = [&](int k, int rows_from) {   // M is zero behind the diagonal, T ahead of column c
                float x[2][4];
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    if (r >= rows_from) *reinterpret_cast<float4*>(x[r]) = *reinterpret_cast<const float4*>(&sm.M[lane + 32 * r][k]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const ulonglong2 y0 = *reinterpret_cast<const ulonglong2*>(&sm.A[k + j][c]), y1 = *reinterpret_cast<const ulonglong2*>(&sm.A[k + j][c + 4]);
#pragma unroll
                    for (int r = 0; r < 2; ++r)
                        if (r >= rows_from) {
                            const u64 d = pk(x[r][j], x[r][j]);
                            acc[r][0] = fma2(d, y0.x, acc[r][0]); acc[r][1] = fma2(d, y0.y, acc[r][1]);
                            acc[r][2] = fma2(d, y1.x, acc[r][2]); acc[r][3] = fma2(d, y1.y, acc[r][3]);
                        }
                }
            };
#pragma unroll 2
            for (int k = c; k < 32; k += 4) add(k, 0);
#pragma unroll 2
            for (int k = max(c, 32); k < 64; k += 4) add(k, 1);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int i = lane + 32 * r;
                const uint32_t to = (uint32_t)i * 128 + (uint32_t)((u ^ (i & 7)) * 16);
                uint4 t[3], m[2];
                uint32_t *th = &t[0].x, *tm = &t[1].x, *tl = &t[2].x, *mh = &m[0].x, *ml = &m[1].x;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 x = *reinterpret_cast<const float2*>(&sm.A[i][c + 2 * e]);
                    split3(c + 2 * e <= i ? x.x * b[2 * e] : 0.f, c + 2 * e + 1 <= i ? x.y * b[2 * e + 1] : 0.f, th[e], tm[e], tl[e]);
                    float p0, p1;
                    unpk(acc[r][e], p0, p1);
                    split2(p0 * b[2 * e], p1 * b[2 * e + 1], mh[e], ml[e]);
                }
#pragma unroll
                for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(to_T + k * 8192 + to) = t[k];
#pragma unroll
                for (int k = 0; k < 2; ++k) *reinterpret_cast<uint4*>(to_M + k * 8192 + to) = m[k];
            }
        }
        return;
    }
    unsigned char* to_T = ws.T + ((size_t)cidx * p.L.n_v_heads + head) * kTBytes + lane * 16;
    unsigned char* to_M = ws.M + ((size_t)cidx * p.L.n_v_heads + head) * kMBytes + lane * 16;
    for (int n = warp; n < kBlocks; n += kPrepThreads / 32) {
        const int mi = n < 1 ? 0 : (n < 3 ? 1 : (n < 6 ? 2 : 3)), ki = n - mi * (mi + 1) / 2;
        float2 v[4];
        operand_pairs(sm.A, mi * 16, ki * 16, lane, v);
        const float2 b0 = *reinterpret_cast<const float2*>(&sm.beta[ki * 16 + 2 * (lane & 3)]), b1 = *reinterpret_cast<const float2*>(&sm.beta[ki * 16 + 2 * (lane & 3) + 8]);
        uint32_t s[3][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) split3(v[e].x * (e < 2 ? b0.x : b1.x), v[e].y * (e < 2 ? b0.y : b1.y), s[0][e], s[1][e], s[2][e]);
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(to_T + (k * kBlocks + n) * 512) = make_uint4(s[k][0], s[k][1], s[k][2], s[k][3]);
        operand_pairs(sm.M, mi * 16, ki * 16, lane, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) split2(v[e].x, v[e].y, s[0][e], s[1][e]);
#pragma unroll
        for (int k = 0; k < 2; ++k) *reinterpret_cast<uint4*>(to_M + k * kMPart + n * 512) = make_uint4(s[k][0], s[k][1], s[k][2], s[k][3]);
    }
}

// ---------------------------------------------------------------- kernel 2
constexpr int kSlice = 16, kStages = 3;
constexpr int kChainThreads = 256;   // warps 0-3: the state's products; warps 4-7: the outputs'

template <int DK>
struct ChainStage {
    unsigned char k[Q * DK * 2], q[Q * DK * 2];   // boxes of 64 values x 64 rows, 128-byte swizzle
    unsigned char T[kTBytes], M[kMPart];   // M's leading part; the output warps fetch the other one themselves, there is no room for it
    __nv_bfloat16 v[Q][kSlice];
    float2 ef[Q];   // decay from the chunk's start to a row, from the row to the chunk's end
    unsigned char pad[1024 - (kTBytes + kMPart + Q * kSlice * 2 + Q * 8) % 1024];
};
template <int DK>
struct ChainSmem {
    static constexpr int kRow = kSlice + 8;                // values of a row of the operands below, padded against bank conflicts
    ChainStage<DK> stage[kStages];
    float4 part[4][3][kSlice / 8][32];                     // K S^T over a warp's share of d_k, for the warps of the other row tiles
    __nv_bfloat16 S[2][2][kSlice][DK];                     // leading two parts of the incoming state, by parity of the chunk; 16-byte units XOR-ed with the row index
    __nv_bfloat16 R[3][Q][kRow];                        // V - e^G (K S^T), split in three
    __nv_bfloat16 W[3][Q][kRow];                        // e^{G_end - G} X, split in three
    __nv_bfloat16 X[2][2][Q][kRow];                     // X, split in two, by parity
    uint64_t full[kStages];
};

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm2t(uint32_t (&r)[2], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void lds16(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// A state warp holds kSlice x DK / 4 of the state as accumulators of the update; split in three they are, as they lie, the operands of its share of K S^T
// (a quarter of d_k, all 64 tokens), so the state never passes through shared memory; the four partial sums do, to the warp of each row tile.
// What does not depend on the product ahead is loaded before the barrier in between.  The output warps trail by half a chunk.
template <int DK>
__global__ void __launch_bounds__(kChainThreads, 1) gdr_chain(const GdrPrefillArgs p, const GdrChunkWs ws, const __grid_constant__ GdrMaps maps, int d_v) {
    using Smem = ChainSmem<DK>;
    constexpr int kRow = Smem::kRow;
    constexpr int NT = kSlice / 8;         // 8-column tiles of a product of 64 x kSlice
    constexpr int NX = NT / 2;          // of which a state warp has these of each of two row tiles in T R
    constexpr int MS = kSlice / 16;        // 16-row tiles of the state slice
    constexpr int ND = DK / 32;         // 8-column tiles of a warp in the state slice
    constexpr int KS = DK / 16;         // steps over d_k
    extern __shared__ __align__(1024) unsigned char s_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(s_raw + ((1024u - (smem_u32(s_raw) & 1023u)) & 1023u));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool outputs = warp >= 4;
    const int slice = blockIdx.x, head = blockIdx.y, seq = blockIdx.z;
    grid_release_dependents();
    int first, nck, s0, len;
    bool bad;
    seq_chunks(p.cu, p.n_seq, p.T, Q, p.n_chunks_bound, seq, first, nck);
    seq_span(p.cu, p.n_seq, p.T, seq, s0, len, bad);
    const int islot = load_slot(p.init_slot, seq), fslot = load_slot(p.final_slot, seq);
    const bool bad_slot = islot >= p.pool.n_slots || fslot >= p.pool.n_slots;
    if (bad || bad_slot || (len > 0 && nck == 0)) {   // malformed offsets, chunks beyond the workspace, slots that are not there: left out
        if (tid == 0 && slice == 0 && head == 0) flag(p.dev_status, bad_slot ? MDRAFT_DEV_BAD_SLOT : MDRAFT_DEV_BAD_SEQLENS);
        grid_wait();
        return;
    }
    const int khead = head / (p.L.n_v_heads / p.L.n_k_heads), col = head * d_v + slice * kSlice;
    const size_t H = p.L.n_v_heads;
    if (tid == 0) {
#pragma unroll
        for (int i = 0; i < kStages; ++i) mbar_init(&sm.full[i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    grid_wait();   // T, M and the running decays are the work of the kernel just before
    __syncthreads();
    auto fetch = [&](int n) {   // one thread
        ChainStage<DK>& s = sm.stage[n % kStages];
        uint64_t* bar = &sm.full[n % kStages];
        const size_t ch = (size_t)(first + n) * H + head;
        mbar_expect_tx(bar, 2 * Q * DK * 2 + kTBytes + kMPart + Q * kSlice * 2 + Q * 8);
#pragma unroll
        for (int h = 0; h < DK / 64; ++h) {
            tma_box(s.k + h * 8192, &maps.k, khead * DK + 64 * h, s0 + n * Q, bar);
            tma_box(s.q + h * 8192, &maps.q, khead * DK + 64 * h, s0 + n * Q, bar);
        }
        tma_box(s.v, &maps.v, col, s0 + n * Q, bar);
        bulk_load(s.T, ws.T + ch * kTBytes, kTBytes, bar);
        bulk_load(s.M, ws.M + ch * kMBytes, kMPart, bar);
        bulk_load(s.ef, ws.ef + ch * Q, Q * 8, bar);
    };
    if (tid == kChainThreads - 32)
#pragma unroll 1
        for (int i = 0; i < kStages && i < nck; ++i) fetch(i);

    const int g = lane >> 2, t2 = 2 * (lane & 3);
    const uint32_t sR = smem_u32(sm.R), sW = smem_u32(sm.W);
    const int mt = warp & 3;   // row tile of the warp in products of 64 x kSlice
    const int r0 = mt * 16 + g, r1 = r0 + 8;
    // Operand of 16 rows of keys or queries, step ks of d_k.
    auto rows_operand = [&](uint32_t (&a)[4], const unsigned char* m, int tile, int ks) {
        const int row = tile * 16 + (lane & 15), unit = (ks & 3) * 2 + (lane >> 4);
        ldsm4(a, smem_u32(m) + (ks >> 2) * 8192 + row * 128 + ((unit ^ (row & 7)) * 16));
    };
    bool here = true, failed = false;
    int c = 0;
    auto arrive = [&](int n) { here = mbar_wait_bounded(&sm.full[n % kStages], (uint32_t)(n / kStages) & 1u) && here; };

    if (!outputs) {
        // State: rows (values) 16 ms + g and + 8, columns 8 (ND warp + nd) + t2 and + 1.
        float S[MS][ND][4];
        {
            const float* h0 = p.pool.ssm + (size_t)(islot < 0 ? 0 : islot) * p.pool.ssm_slot_stride + (size_t)col * DK;
#pragma unroll
            for (int ms = 0; ms < MS; ++ms)
#pragma unroll
                for (int nd = 0; nd < ND; ++nd) {
                    float2 a = make_float2(0.f, 0.f), b = a;
                    const int d = (warp * ND + nd) * 8 + t2;
                    if (islot >= 0) {
                        a = *reinterpret_cast<const float2*>(h0 + (size_t)(ms * 16 + g) * DK + d);
                        b = *reinterpret_cast<const float2*>(h0 + (size_t)(ms * 16 + g + 8) * DK + d);
                    }
                    S[ms][nd][0] = a.x; S[ms][nd][1] = a.y; S[ms][nd][2] = b.x; S[ms][nd][3] = b.y;
                }
        }
        // The state as operands: part, tile of 8 rows, tile of 8 columns; its leading parts go to the output warps too.
        uint32_t sp[3][NT][ND];
        auto split_state = [&](int parity) {
#pragma unroll
            for (int ms = 0; ms < MS; ++ms)
#pragma unroll
                for (int nd = 0; nd < ND; ++nd)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int n = 2 * ms + h, row = n * 8 + g, unit = warp * ND + nd;
                        split3(S[ms][nd][2 * h], S[ms][nd][2 * h + 1], sp[0][n][nd], sp[1][n][nd], sp[2][n][nd]);
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            *reinterpret_cast<uint32_t*>(reinterpret_cast<unsigned char*>(&sm.S[parity][k][row][0]) + ((unit ^ (row & 7)) * 16) + t2 * 2) = sp[k][n][nd];
                    }
        };
        split_state(0);
        constexpr int KW = KS / 4;   // the warp's steps over d_k
        uint32_t kr[4][KW][4];       // its keys: all rows of the chunk
        uint32_t vr[NT][2];          // values of row tile mt
        float e0 = 0.f, e1 = 0.f, ec = 0.f;
        // T R takes half the columns of row tile mt and the other half of row tile 3 - mt, five blocks of the triangle for every warp: first the
        // shorter row of blocks (one or two), then the longer.
        const int m_of[2] = {mt < 2 ? mt : 3 - mt, mt < 2 ? 3 - mt : mt}, n_of[2] = {mt < 2 ? 0 : NX, mt < 2 ? NX : 0};
        float fr[2][2] = {{0.f, 0.f}, {0.f, 0.f}};   // decay from their rows to the chunk's end
        auto preload = [&](int n) {
            const ChainStage<DK>& s = sm.stage[n % kStages];
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int j = 0; j < KW; ++j) rows_operand(kr[m][j], s.k, m, warp * KW + j);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                vr[i][0] = *reinterpret_cast<const uint32_t*>(&s.v[r0][i * 8 + t2]);
                vr[i][1] = *reinterpret_cast<const uint32_t*>(&s.v[r1][i * 8 + t2]);
            }
            e0 = s.ef[r0].x; e1 = s.ef[r1].x; ec = s.ef[Q - 1].x;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) fr[i][h] = s.ef[m_of[i] * 16 + g + 8 * h].y;
        };
        if (nck > 0) {
            arrive(0);
            preload(0);
        }
        for (; c < nck; ++c) {
            ChainStage<DK>& s = sm.stage[c % kStages];
            const int rows = len - c * Q;
            // K S^T over the warp's share of d_k
            float d[4][NT][4];
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[m][n][e] = 0.f;
#pragma unroll
            for (int k = 2; k >= 0; --k)
#pragma unroll
                for (int j = 0; j < KW; ++j)
#pragma unroll
                    for (int m = 0; m < 4; ++m)
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma16816(d[m][n], kr[m][j], sp[k][n][2 * j], sp[k][n][2 * j + 1]);
            float own[NT][4];
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (m == warp) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) own[n][e] = d[m][n][e];
                    } else {
                        sm.part[m][(warp - m - 1) & 3][n][lane] = make_float4(d[m][n][0], d[m][n][1], d[m][n][2], d[m][n][3]);
                    }
                }
            bar_sync(1, 128);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int cc = n * 8 + t2;
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    const float4 o = sm.part[mt][i][n][lane];
                    own[n][0] += o.x; own[n][1] += o.y; own[n][2] += o.z; own[n][3] += o.w;
                }
                own[n][0] = r0 < rows ? fmaf(-e0, own[n][0], bf_lo(vr[n][0])) : 0.f;
                own[n][1] = r0 < rows ? fmaf(-e0, own[n][1], bf_hi(vr[n][0])) : 0.f;
                own[n][2] = r1 < rows ? fmaf(-e1, own[n][2], bf_lo(vr[n][1])) : 0.f;
                own[n][3] = r1 < rows ? fmaf(-e1, own[n][3], bf_hi(vr[n][1])) : 0.f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t x[3];
                    split3(own[n][2 * h], own[n][2 * h + 1], x[0], x[1], x[2]);
#pragma unroll
                    for (int k = 0; k < 3; ++k) *reinterpret_cast<uint32_t*>(&sm.R[k][r0 + 8 * h][cc]) = x[k];
                }
            }
            bar_sync(1, 128);
            // X = T R, the six products that reach 24 bits
            float x[NX][3][4], xs[NX][4];
#pragma unroll
            for (int n = 0; n < NX; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) { x[n][0][e] = x[n][1][e] = x[n][2][e] = 0.f; xs[n][e] = 0.f; }
#pragma unroll
            for (int j = 0; j < 5; ++j) {
                const bool i = j > m_of[0];
                const int ki = i ? j - m_of[0] - 1 : j, mi = i ? m_of[1] : m_of[0], ni = i ? n_of[1] : n_of[0];
                uint32_t t[3][4], b[NX][3][2];
                const uint32_t sT = smem_u32(s.T) + (mi * (mi + 1) / 2 + ki) * 512 + lane * 16, sB = sR + ((ki * 16 + (lane & 15)) * kRow + ni * 8) * 2;
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    lds16(t[k], sT + k * kBlocks * 512);
#pragma unroll
                    for (int n = 0; n < NX; ++n) ldsm2t(b[n][k], sB + (k * Q * kRow + n * 8) * 2);
                }
#pragma unroll
                for (int n = 0; n < NX; ++n) {
                    mma16816(x[n][0], t[0], b[n][0][0], b[n][0][1]);
                    mma16816(x[n][1], t[0], b[n][1][0], b[n][1][1]);
                    mma16816(x[n][2], t[1], b[n][1][0], b[n][1][1]);
                    mma16816(x[n][1], t[1], b[n][0][0], b[n][0][1]);
                    mma16816(x[n][2], t[0], b[n][2][0], b[n][2][1]);
                    mma16816(x[n][0], t[2], b[n][0][0], b[n][0][1]);
                }
                if (j < 2 && j == m_of[0])   // the shorter row of blocks is complete
#pragma unroll
                    for (int n = 0; n < NX; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            xs[n][e] = (x[n][2][e] + x[n][1][e]) + x[n][0][e];
                            x[n][0][e] = x[n][1][e] = x[n][2][e] = 0.f;
                        }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int n = 0; n < NX; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int cc = (n_of[i] + n) * 8 + t2, row = m_of[i] * 16 + g + 8 * h;
                        const float v0 = i ? (x[n][2][2 * h] + x[n][1][2 * h]) + x[n][0][2 * h] : xs[n][2 * h];
                        const float v1 = i ? (x[n][2][2 * h + 1] + x[n][1][2 * h + 1]) + x[n][0][2 * h + 1] : xs[n][2 * h + 1];
                        uint32_t w[3];
                        split3(v0 * fr[i][h], v1 * fr[i][h], w[0], w[1], w[2]);
#pragma unroll
                        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint32_t*>(&sm.W[k][row][cc]) = w[k];
                        split2(v0, v1, w[0], w[1]);
#pragma unroll
                        for (int k = 0; k < 2; ++k) *reinterpret_cast<uint32_t*>(&sm.X[c & 1][k][row][cc]) = w[k];
                    }
            uint32_t kc[ND / 2][4];   // key columns of the warp's share of the state, 16 tokens at a time
            auto load_keys = [&](int ki) {
#pragma unroll
                for (int j = 0; j < ND / 2; ++j) {
                    const int row = ki * 16 + (lane & 15), u = warp * ND + 2 * j, unit = (u & 7) + (lane >> 4);
                    ldsm4t(kc[j], smem_u32(s.k) + (u >> 3) * 8192 + row * 128 + ((unit ^ (row & 7)) * 16));
                    if (rows < Q)   // keys of other sequences, which may be anything, would meet zeros
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int token = ki * 16 + t2 + 8 * (e & 1);
                            kc[j][e] &= (token < rows ? 0xffffu : 0u) | (token + 1 < rows ? 0xffff0000u : 0u);
                        }
                }
            };
            load_keys(0);
            failed = __syncthreads_or(!here);   // W, X and the state's leading parts are there; the output warps are done with the chunk before
            if (failed) break;                  // a copy did not arrive in time
            float m[MS][ND][4];
#pragma unroll
            for (int ms = 0; ms < MS; ++ms)
#pragma unroll
                for (int nd = 0; nd < ND; ++nd)
#pragma unroll
                    for (int e = 0; e < 4; ++e) { S[ms][nd][e] *= ec; m[ms][nd][e] = 0.f; }
#pragma unroll 1
            for (int ki = 0; ki < Q / 16; ++ki) {
#pragma unroll
                for (int ms = 0; ms < MS; ++ms)
#pragma unroll
                    for (int k = 0; k < 3; ++k) {
                        uint32_t a[4];
                        ldsm4t(a, sW + ((k * Q + ki * 16 + (lane & 7) + ((lane >> 4) & 1) * 8) * kRow + ms * 16 + ((lane >> 3) & 1) * 8) * 2);
#pragma unroll
                        for (int nd = 0; nd < ND; ++nd) mma16816(k == 0 ? S[ms][nd] : m[ms][nd], a, kc[nd / 2][2 * (nd & 1)], kc[nd / 2][2 * (nd & 1) + 1]);
                    }
                if (ki + 1 < Q / 16) load_keys(ki + 1);
            }
            if (c + 1 < nck) {
                arrive(c + 1);
                preload(c + 1);
            }
#pragma unroll
            for (int ms = 0; ms < MS; ++ms)
#pragma unroll
                for (int nd = 0; nd < ND; ++nd)
#pragma unroll
                    for (int e = 0; e < 4; ++e) S[ms][nd][e] += m[ms][nd][e];
            if (c + 1 < nck) split_state((c + 1) & 1);
        }
        if (!failed && fslot >= 0 && (nck > 0 || fslot != islot)) {
            float* h1 = p.pool.ssm + (size_t)fslot * p.pool.ssm_slot_stride + (size_t)col * DK;
#pragma unroll
            for (int ms = 0; ms < MS; ++ms)
#pragma unroll
                for (int nd = 0; nd < ND; ++nd) {
                    const int d = (warp * ND + nd) * 8 + t2;
                    *reinterpret_cast<float2*>(h1 + (size_t)(ms * 16 + g) * DK + d) = make_float2(S[ms][nd][0], S[ms][nd][1]);
                    *reinterpret_cast<float2*>(h1 + (size_t)(ms * 16 + g + 8) * DK + d) = make_float2(S[ms][nd][2], S[ms][nd][3]);
                }
        }
    } else {
        for (; c < nck; ++c) {
            const ChainStage<DK>& s = sm.stage[c % kStages];
            const int t0 = s0 + c * Q, rows = len - c * Q;
            uint32_t qr[KS][4], mr[4][4], ml[4][4], zr[NT][2];
            const unsigned char* M_low = ws.M + ((size_t)(first + c) * H + head) * kMBytes + kMPart + (mt * (mt + 1) / 2) * 512 + lane * 16;
#pragma unroll
            for (int ki = 0; ki < 4; ++ki)
                if (ki <= mt) *reinterpret_cast<uint4*>(ml[ki]) = *reinterpret_cast<const uint4*>(M_low + ki * 512);
            arrive(c);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) rows_operand(qr[ks], s.q, mt, ks);
            const uint32_t sM = smem_u32(s.M) + (mt * (mt + 1) / 2) * 512 + lane * 16;
#pragma unroll
            for (int ki = 0; ki < 4; ++ki)
                if (ki <= mt) lds16(mr[ki], sM + ki * 512);
            if (p.io.z && !ws.o) {
                const __nv_bfloat16* z = static_cast<const __nv_bfloat16*>(p.io.z) + (size_t)(t0 + r0) * p.io.ldz + col;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    zr[n][0] = zr[n][1] = 0u;
                    if (r0 < rows) zr[n][0] = *reinterpret_cast<const uint32_t*>(z + n * 8 + t2);
                    if (r1 < rows) zr[n][1] = *reinterpret_cast<const uint32_t*>(z + 8 * p.io.ldz + n * 8 + t2);
                }
            }
            const float e0 = s.ef[r0].x * p.L.scale, e1 = s.ef[r1].x * p.L.scale;
            failed = __syncthreads_or(!here);   // X and the state's leading parts are there
            if (failed) break;
            if (tid == kChainThreads - 32 && c > 0 && c - 1 + kStages < nck) fetch(c - 1 + kStages);   // all warps are done with the chunk before
            // O = scale e^G (Q S^T) + M X
            float o[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
            const uint32_t sS = smem_u32(sm.S[c & 1]), sX = smem_u32(sm.X[c & 1]);
#pragma unroll
            for (int k = 1; k >= 0; --k)
#pragma unroll
                for (int k2 = 0; k2 < KS / 2; ++k2)
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        uint32_t b[4];
                        const int row = n * 8 + (lane & 7), unit = 4 * k2 + (lane >> 3);
                        ldsm4(b, sS + (k * kSlice + row) * (DK * 2) + ((unit ^ (row & 7)) * 16));
                        mma16816(o[n], qr[2 * k2], b[0], b[1]);
                        mma16816(o[n], qr[2 * k2 + 1], b[2], b[3]);
                    }
#pragma unroll
            for (int n = 0; n < NT; ++n) { o[n][0] *= e0; o[n][1] *= e0; o[n][2] *= e1; o[n][3] *= e1; }
#pragma unroll
            for (int ki = 0; ki < 4; ++ki)
                if (ki <= mt) {
#pragma unroll
                    for (int k = 1; k >= 0; --k)
#pragma unroll
                        for (int n2 = 0; n2 < NT / 2; ++n2) {
                            uint32_t b[4];
                            ldsm4t(b, sX + ((k * Q + ki * 16 + (lane & 15)) * kRow + n2 * 16 + (lane >> 4) * 8) * 2);
                            mma16816(o[2 * n2], mr[ki], b[0], b[1]);
                            mma16816(o[2 * n2 + 1], mr[ki], b[2], b[3]);
                            if (k == 0) {
                                mma16816(o[2 * n2], ml[ki], b[0], b[1]);
                                mma16816(o[2 * n2 + 1], ml[ki], b[2], b[3]);
                            }
                        }
                }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = r0 + 8 * h;
                    if (r >= rows) continue;
                    const size_t t = (size_t)(t0 + r);
                    const int cc = col + n * 8 + t2;
                    float a = o[n][2 * h], b = o[n][2 * h + 1];
                    if (ws.o) {
                        *reinterpret_cast<float2*>(ws.o + t * (H * d_v) + cc) = make_float2(a, b);
                    } else {
                        if (p.io.z) { a *= silu(bf_lo(zr[n][h])); b *= silu(bf_hi(zr[n][h])); }
                        *reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(p.io.out) + t * p.io.ldo + cc) = pack_bf(a, b);
                    }
                }
        }
    }
    if (failed && tid == 0) {   // copies target this block's shared memory: one more bounded chance
        flag(p.dev_status, MDRAFT_DEV_WAIT_EXPIRED);
        for (int i = c > 0 ? c - 1 : 0; i < (c > 0 ? c - 1 : 0) + kStages && i < nck; ++i) mbar_wait_bounded(&sm.full[i % kStages], (uint32_t)(i / kStages) & 1u);
    }
}

// ---------------------------------------------------------------- kernel 3: output norm and gate, a warp per row and head
constexpr int kNormThreads = 256;

template <int DV>
__global__ void __launch_bounds__(kNormThreads) gdr_norm_gate(const GdrPrefillArgs p, const float* o) {
    constexpr int E = DV / 32;   // values of a lane
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, H = p.L.n_v_heads;
    grid_wait();
    grid_release_dependents();
    const ChunkInfo ci = find_chunk(p.cu, p.n_seq, p.T, Q, p.n_chunks_bound, blockIdx.y + blockIdx.z * gridDim.y);
    if (ci.seq < 0 || load_slot(p.init_slot, ci.seq) >= p.pool.n_slots || load_slot(p.final_slot, ci.seq) >= p.pool.n_slots) return;
    const int head = blockIdx.x;
    float w[E];
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = __ldg(p.L.norm_w + lane * E + e);
#pragma unroll 4
    for (int t = ci.t0 + warp; t < ci.t1; t += kNormThreads / 32) {
        const size_t c = (size_t)head * DV + lane * E;
        float v[E], z[E], sq = 0.f;
        uint32_t zr[E / 2];
        if (E == 4) *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(o + (size_t)t * H * DV + c);
        else *reinterpret_cast<float2*>(v) = *reinterpret_cast<const float2*>(o + (size_t)t * H * DV + c);
        if (p.io.z) {
            const __nv_bfloat16* zp = static_cast<const __nv_bfloat16*>(p.io.z) + (size_t)t * p.io.ldz + c;
            if (E == 4) *reinterpret_cast<uint2*>(zr) = *reinterpret_cast<const uint2*>(zp);
            else zr[0] = *reinterpret_cast<const uint32_t*>(zp);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) sq = fmaf(v[e], v[e], sq);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) sq += __shfl_xor_sync(0xffffffffu, sq, d);
        const float f = rsqrtf(sq * (1.0f / DV) + p.L.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            z[e] = p.io.z ? silu(e & 1 ? bf_hi(zr[e / 2]) : bf_lo(zr[e / 2])) : 1.f;
            v[e] *= f * w[e] * z[e];
        }
        __nv_bfloat16* op = static_cast<__nv_bfloat16*>(p.io.out) + (size_t)t * p.io.ldo + c;
        if (E == 4) *reinterpret_cast<uint2*>(op) = make_uint2(pack_bf(v[0], v[1]), pack_bf(v[2], v[3]));
        else *reinterpret_cast<uint32_t*>(op) = pack_bf(v[0], v[1]);
    }
}

// Blocks over (heads, chunks) where there may be more chunks than a grid's second index takes.
inline dim3 chunk_grid(int heads, int chunks) {
    const int z = (chunks + 65534) / 65535;
    return dim3(heads, (chunks + z - 1) / z, z);
}

template <int DK>
cudaError_t chain(const GdrPrefillArgs& p, const GdrChunkWs& ws, const GdrMaps& maps, int d_v, cudaStream_t st) {
    constexpr int smem = sizeof(ChainSmem<DK>) + 1024;
    static_assert(smem <= 227 * 1024, "one block per SM");
    const cudaError_t e = allow_smem<gdr_chain<DK>>(smem);
    if (e != cudaSuccess) return e;
    return launch_pdl(gdr_chain<DK>, dim3(d_v / kSlice, p.L.n_v_heads, p.n_seq), kChainThreads, smem, st, p, ws, maps, d_v);
}

template <int DK, bool kWide>
cudaError_t prepare(const GdrPrefillArgs& p, const GdrChunkWs& ws, const GdrMaps& maps, cudaStream_t st) {
    constexpr int smem = sizeof(PrepSmem<DK>) + 1024;
    const cudaError_t e = allow_smem<gdr_chunk_prepare<DK, kWide>>(smem);
    if (e != cudaSuccess) return e;
    return launch_pdl(gdr_chunk_prepare<DK, kWide>, chunk_grid(p.L.n_v_heads, p.n_chunks_bound), kPrepThreads, smem, st, p, ws, maps);
}

template <int DK>
cudaError_t chunked(const GdrPrefillArgs& p, const GdrChunkWs& ws, const GdrMaps& maps, int d_v, int slice, cudaStream_t st) {
    cudaError_t e = slice == d_v ? prepare<DK, true>(p, ws, maps, st) : prepare<DK, false>(p, ws, maps, st);
    if (e != cudaSuccess) return e;
    if (slice == d_v) return launch_gdr_chain_wide(p, ws, maps, DK, d_v, st);
    e = chain<DK>(p, ws, maps, d_v, st);
    if (e != cudaSuccess || !ws.o) return e;
    return launch_pdl(d_v == 128 ? gdr_norm_gate<128> : gdr_norm_gate<64>, chunk_grid(p.L.n_v_heads, p.n_chunks_bound), kNormThreads, 0, st, p, ws.o);
}

}  // namespace

cudaError_t launch_gdr_chunked(const GdrPrefillArgs& p, const GdrChunkWs& ws, const GdrMaps& maps, int d_k, int d_v, int slice, cudaStream_t st) {
    return d_k == 128 ? chunked<128>(p, ws, maps, d_v, slice, st) : chunked<64>(p, ws, maps, d_v, slice, st);
}

}  // namespace mdraft
