// The chain over the chunks of a sequence (gdr_prefill.cu) for calls with many chains: a block takes a whole head, on the tensor cores.
//
// Everything is laid out with the head's values as the 128 rows (lanes) of tensor memory, transposed against the formulas: per chunk
//
//     D1 = S K^T                      (values x tokens; S: the state, split into three bf16 parts, an operand in tensor memory)
//     R  = V^T - e^G D1               -> three parts in tensor memory
//     X  = R T^T                      W = e^{G_end - G} X -> three parts in tensor memory
//     S' = e^{G_end} S + W K
//     O  = scale e^G (S Q^T) + R (M T)^T
//
// S itself stays in registers (fp32), the operands of the other side (K, Q, T, M T) come by TMA as they are used.  M T instead of M makes the outputs
// wait for R, not for X.  Three products of a chunk depend on one another; in between 512 threads take accumulators to operands: tensor
// memory -> registers -> tensor memory.  A chunk of 128 x 128 costs 9500 cycles, 11000 with all SMs at work; the tensor pipe is busy for a third of that (ncu), the rest is the way between
// the products, on which the warps wait for tensor memory and for loads above all.  With as many chains of like length as SMs or more that beats the narrow chain, whose
// blocks share a head among eight SMs to be done with a chunk in 3900 (measured where the choice is made).  32 sequences of 1000 to 8000 tokens x 12 heads: 1.17 ms for
// the chain and 0.69 ms for the triangles ahead of it (cold, one behind the other), 2.0 ms in all, call after call, against 10.7 token by token.
//
// Warps 0-15: the state's, warps w, w + 4, .. share rows 32 (w % 4) .. and split the columns.  Four warps: outputs (norm and gate inside).  One warp issues the
// products, one the copies, one those of the gate.  All waits on mbarriers are bounded; a thread whose wait has run out goes on through the block's barriers without
// waiting again, so that all of them come to the end.
#include "chunk_map.cuh"
#include "common.cuh"
#include "gdr.cuh"
#include "tensor_core.cuh"

namespace mdraft {

namespace {

constexpr int Q = kGdrQ;
constexpr int kStateWarps = 16;                                     // four for each 32 lanes of tensor memory, which split the columns
constexpr int kOutWarp = kStateWarps, kMmaWarp = kOutWarp + 4, kCopyWarp = kMmaWarp + 1, kGateWarp = kMmaWarp + 2;
constexpr int kWideThreads = 32 * (kGateWarp + 1), kStages = 2;
constexpr int kMaxSorted = 512;   // sequences of a call that are taken in order of their length (a block ranks them all for itself)
constexpr int kBarLanes = 1, kBarRows = 5;   // named barriers: 1 to 4, the state warps of the same 32 lanes; 5, the output warps

template <int DK, int DV>
struct WideStage {
    unsigned char k[Q * DK * 2], q[Q * DK * 2];   // boxes of 64 values x 64 rows, 128-byte swizzle
    unsigned char T[kGdrWideTBytes], M[kGdrWideMBytes];   // 64 x 64 in rows of 128 bytes, 128-byte swizzle
    __nv_bfloat16 v[Q][DV];
};
template <int DK, int DV>
struct WideSmem {
    WideStage<DK, DV> stage[kStages];
    float2 ef[kStages][Q];       // of a stage too: decay from the chunk's start to a row, from the row to the chunk's end
    __nv_bfloat16 z[Q][DV];      // gate
    float eo[Q];                 // decay from the chunk's start times scale, for the output warps (which may fall behind the stages)
    float o[Q][DV];              // outputs on their way from a lane per value to a row per warp
    uint64_t full[kStages], done[kStages];                   // copies of a stage, all products that read it (and, through w, all that the state warps read of it)
    uint64_t state[2], r[2], w[2], free_o;                   // operands are in tensor memory (in two portions), output accumulators have been read
    uint64_t mma1, mma2, out, last;                          // products
    uint64_t z_full, z_free;
    uint32_t tmem_base;
    int picked;                                              // the block's sequence (a word that no copy targets: copies are not ordered behind ordinary accesses)
};

__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory"); }
// One lane of the warp, by an instruction that tells the compiler so (a branch on the lane index costs a tensor-core instruction 80 cycles of issue
// instead of 32).
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// Two neighbours as three bf16 values each.  The first is rounded, the others are truncated: the remainders are exact, and 8 + 8 + 8
// bits hold all 24 of a fp32 value.  The outputs take the first two, 2^-15 of a value.
__device__ __forceinline__ uint32_t leading_halves(u64 v) { return __byte_perm((uint32_t)v, (uint32_t)(v >> 32), 0x7632); }
__device__ __forceinline__ uint32_t split_first(u64& v) {   // leaves the remainder
    float a, b;
    unpk(v, a, b);
    const uint32_t hi = pack_bf(a, b);
    v = fma2(pk(bf_lo(hi), bf_hi(hi)), pk(-1.f, -1.f), v);
    return hi;
}
__device__ __forceinline__ uint32_t split_last(u64 v) { return leading_halves(fma2(v & 0xffff0000ffff0000ull, pk(-1.f, -1.f), v)); }

template <int DK, int DV>
__global__ void __launch_bounds__(kWideThreads, 1) gdr_chain_wide(const GdrPrefillArgs p, const GdrChunkWs ws, const __grid_constant__ GdrMaps maps) {
    using Smem = WideSmem<DK, DV>;
    constexpr uint32_t kS = 0, kR = 3 * DK / 2, kD1 = kR + 96, kDQ = kD1 + 64, kDO = kDQ + 64;   // columns of tensor memory
    constexpr uint32_t kD3 = kS;                        // the update, over the leading two parts of the state that it replaces
    constexpr uint32_t kW[3] = {DK == 128 ? kS + DK : kDO + 64, DK == 128 ? kS + DK + 32 : kDO + 96, kR + 64};   // over the state's last part where there is no room beside it
    static_assert(kDO + 64 + (DK == 128 ? 0 : 64) <= 512, "tensor memory");
    extern __shared__ __align__(1024) unsigned char s_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(s_raw + ((1024u - (smem_u32(s_raw) & 1023u)) & 1023u));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int head = blockIdx.x;
    grid_release_dependents();
    int seq = blockIdx.y;
    if (p.n_seq > 1 && p.n_seq <= kMaxSorted) {   // the longest sequences first: the blocks that start last are to be the short ones
        if (tid < p.n_seq) {
            int a, mine, b, other;
            bool bad_a, bad_b;
            seq_span(p.cu, p.n_seq, p.T, tid, a, mine, bad_a);
            int rank = 0;
            for (int i = 0; i < p.n_seq; ++i) {
                seq_span(p.cu, p.n_seq, p.T, i, b, other, bad_b);
                rank += other > mine || (other == mine && i < tid);
            }
            if (rank == (int)blockIdx.y) sm.picked = tid;
        }
        __syncthreads();
        seq = sm.picked;
    }
    int first, nck, s0, len;
    bool bad;
    seq_chunks(p.cu, p.n_seq, p.T, Q, p.n_chunks_bound, seq, first, nck);
    seq_span(p.cu, p.n_seq, p.T, seq, s0, len, bad);
    const int islot = load_slot(p.init_slot, seq), fslot = load_slot(p.final_slot, seq);
    const bool bad_slot = islot >= p.pool.n_slots || fslot >= p.pool.n_slots;
    if (bad || bad_slot || (len > 0 && nck == 0)) {   // malformed offsets, chunks beyond the workspace, slots that are not there: left out
        if (tid == 0 && head == 0) flag(p.dev_status, bad_slot ? MDRAFT_DEV_BAD_SLOT : MDRAFT_DEV_BAD_SEQLENS);
        grid_wait();
        return;
    }
    const size_t H = p.L.n_v_heads;
    if (tid == 0) {
#pragma unroll
        for (int i = 0; i < kStages; ++i) { mbar_init(&sm.full[i], 1); mbar_init(&sm.done[i], 1); }
#pragma unroll
        for (int i = 0; i < 2; ++i) { mbar_init(&sm.state[i], kStateWarps); mbar_init(&sm.r[i], kStateWarps); mbar_init(&sm.w[i], kStateWarps); }   // a lane of every warp
        mbar_init(&sm.free_o, 4);
        mbar_init(&sm.mma1, 1); mbar_init(&sm.mma2, 1); mbar_init(&sm.out, 1); mbar_init(&sm.last, 1);
        mbar_init(&sm.z_full, 1); mbar_init(&sm.z_free, 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) { tmem_alloc(&sm.tmem_base, 512); tc_fence_before(); }
    grid_wait();   // T, M T and the decays are the work of the kernel just before
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem_base;
    bool ok = true;
    auto wait = [&](uint64_t* bar, int phase) { ok = __all_sync(0xffffffffu, ok && mbar_wait_bounded(bar, (uint32_t)phase & 1u)); };
    auto arrive = [&](uint64_t* bar) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
    };

    if (warp < kStateWarps) {
        // ---------------------------------------------------------------- state
        const int part = warp >> 2, row = (warp & 3) * 32 + lane;   // rows past d_v idle along
        const bool rows_here = (warp & 3) * 32 < DV;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        constexpr int C = DK / 4;   // columns of the state that a thread holds
        u64 S[C / 2];               // two at a time
        const size_t at = ((size_t)head * DV + row) * DK + part * C;
#pragma unroll
        for (int i = 0; i < C; i += 4) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (islot >= 0 && rows_here) v = *reinterpret_cast<const float4*>(p.pool.ssm + (size_t)islot * p.pool.ssm_slot_stride + at + i);
            S[i / 2] = pk(v.x, v.y); S[i / 2 + 1] = pk(v.z, v.w);
        }
        auto put_state = [&] {   // every second step of d_k is handed over first
#pragma unroll
            for (int i = 0; i < C; i += 16) {
                if (rows_here) {
                    uint32_t a[3][8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        u64 v = S[i / 2 + j];
                        a[0][j] = split_first(v);
                        a[1][j] = leading_halves(v);
                        a[2][j] = split_last(v);
                    }
#pragma unroll
                    for (int k = 0; k < 3; ++k) tmem_st8(tmem + lanes + kS + k * (DK / 2) + part * (C / 2) + i / 2, a[k]);
                    tmem_wait_st();
                }
                arrive(&sm.state[i / 16]);
            }
        };
        if (nck > 0) put_state();
        for (int c = 0; c < nck; ++c) {
            WideStage<DK, DV>& s = sm.stage[c % kStages];
            // The thread takes eight tokens of the first half of the chunk and the eight that lie 32 further on, and hands them over in that order.
            const float2* ef = sm.ef[c % kStages] + 8 * part;
            const int rows = len - c * Q, mine = rows - 8 * part;
            wait(&sm.full[c % kStages], c / kStages);
            uint32_t vv[8];   // values of two tokens each
            {
                const unsigned short* vp = reinterpret_cast<const unsigned short*>(&s.v[8 * part][rows_here ? row : 0]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int t = 2 * j + (j < 4 ? 0 : 24);
                    vv[j] = (uint32_t)vp[t * DV] | (uint32_t)vp[(t + 1) * DV] << 16;
                }
            }
            wait(&sm.mma1, c);
            tc_fence_after();
            float v[2][8];
            auto load_d1 = [&] {
                if (rows_here && ok) {
                    tmem_ld8_begin(tmem + lanes + kD1 + 8 * part, v[0]);
                    tmem_ld8_begin(tmem + lanes + kD1 + 32 + 8 * part, v[1]);
                    tmem_ld_end(v[0], v[1]);
                }
            };
            auto hand_over = [&](const u64 (&x)[4], uint32_t hi, uint32_t mid, uint32_t lo, int hand, uint64_t* bar) {
                if (rows_here && ok) {
                    uint32_t a[3][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        u64 y = x[j];
                        a[0][j] = split_first(y);
                        a[1][j] = leading_halves(y);
                        a[2][j] = split_last(y);
                    }
                    const uint32_t to = tmem + lanes + 16 * hand + 4 * part;
                    tmem_st4(to + hi, a[0]);
                    tmem_st4(to + mid, a[1]);
                    tmem_st4(to + lo, a[2]);
                    tmem_wait_st();
                }
                arrive(bar);
            };
            load_d1();
            if (rows < Q && rows_here && ok) {   // tokens past the chunk's end may hold anything: replaced, not scaled
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[0][j] = j < mine ? v[0][j] : 0.f;
                    v[1][j] = 32 + j < mine ? v[1][j] : 0.f;
                    const int t = 2 * j + (j < 4 ? 0 : 24);
                    vv[j] &= (t < mine ? 0xffffu : 0u) | (t + 1 < mine ? 0xffff0000u : 0u);
                }
            }
#pragma unroll
            for (int hand = 0; hand < 2; ++hand) {
                u64 x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float4 e = *reinterpret_cast<const float4*>(&ef[32 * hand + 2 * j]);   // (e, f) of two tokens
                    const uint32_t w = vv[4 * hand + j];
                    x[j] = fma2(pk(-e.x, -e.z), pk(v[hand][2 * j], v[hand][2 * j + 1]), pk(bf_lo(w), bf_hi(w)));
                }
                hand_over(x, kR, kR + 32, kR + 64, hand, &sm.r[hand]);
            }
            if (rows < Q) {   // keys of other sequences, which may be anything, would meet zeros in the update
                for (int i = tid; i < (Q - rows) * (DK / 8); i += 32 * kStateWarps) {
                    const int r = rows + i / (DK / 8), u = i % (DK / 8);
                    *reinterpret_cast<uint4*>(s.k + (u >> 3) * 8192 + r * 128 + (u & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
                fence_async_smem();
            }
            wait(&sm.mma2, c);
            tc_fence_after();
            load_d1();
            const float all = sm.ef[c % kStages][Q - 1].x;
#pragma unroll
            for (int hand = 0; hand < 2; ++hand) {
                u64 x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float4 e = *reinterpret_cast<const float4*>(&ef[32 * hand + 2 * j]);
                    x[j] = mul2(pk(e.y, e.w), pk(v[hand][2 * j], v[hand][2 * j + 1]));
                }
                hand_over(x, kW[0], kW[1], kW[2], hand, &sm.w[hand]);
            }
            // From here on no state warp touches the stage: the arrivals on w[1] are all that `done` waits for, and behind `done` chunk c + 2 is copied into it.
            if (warp == 5) test_hold_up();
            wait(&sm.done[c % kStages], c / kStages);
            tc_fence_after();
            if (rows_here && ok) {
                float v[C];
                if constexpr (C == 32) tmem_ld32(tmem + lanes + kD3 + part * C, v);
                else tmem_ld16(tmem + lanes + kD3 + part * C, v);
#pragma unroll
                for (int j = 0; j < C / 2; ++j) S[j] = fma2(pk(all, all), S[j], pk(v[2 * j], v[2 * j + 1]));
            }
            if (c + 1 < nck) {
                tc_fence_before();
                bar_sync(kBarLanes + (warp & 3), 128);   // the other parts' columns have been read too: they are free
                tc_fence_after();
                put_state();
            }
        }
        if (fslot >= 0 && rows_here && ok && (nck > 0 || fslot != islot)) {
#pragma unroll
            for (int i = 0; i < C; i += 4)
                *reinterpret_cast<ulonglong2*>(p.pool.ssm + (size_t)fslot * p.pool.ssm_slot_stride + at + i) = make_ulonglong2(S[i / 2], S[i / 2 + 1]);
        }
    } else if (warp < kMmaWarp) {
        // ---------------------------------------------------------------- outputs
        const int w = warp - kOutWarp, row = w * 32 + lane;
        const uint32_t lanes = (uint32_t)(w * 32) << 16;
        constexpr int E = DV / 32;   // values of a lane in a row
        float nw[E];
#pragma unroll
        for (int e = 0; e < E; ++e) nw[e] = p.L.norm_w ? __ldg(p.L.norm_w + lane * E + e) : 1.f;
        const size_t col = (size_t)head * DV + lane * E;
        for (int c = 0; c < nck; ++c) {
            const int t0 = s0 + c * Q, rows = min(Q, len - c * Q);
            if (w < 2) sm.eo[row] = p.L.scale * ws.ef[((size_t)(first + c) * H + head) * Q + row].x;
            bar_sync(kBarRows, 128);   // and the rows' staging is free
            wait(&sm.out, c);
            tc_fence_after();
            if (w * 32 < DV && ok) {
#pragma unroll 1
                for (int h = 0; h < Q; h += 16) {
                    float a[16], b[16];
                    tmem_ld16(tmem + lanes + kDQ + h, a);
                    tmem_ld16(tmem + lanes + kDO + h, b);
#pragma unroll
                    for (int j = 0; j < 16; ++j) sm.o[h + j][row] = fmaf(sm.eo[h + j], a[j], b[j]);
                }
            }
            arrive(&sm.free_o);
            bar_sync(kBarRows, 128);
            if (p.io.z) wait(&sm.z_full, c);
            if (ok) {
#pragma unroll 1
                for (int t1 = w; t1 < rows; t1 += 16) {   // four rows side by side
                    float v[4][E], sq[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {   // (rows past the end are there to be read)
                        sq[i] = 0.f;
#pragma unroll
                        for (int e = 0; e < E; ++e) v[i][e] = sm.o[t1 + 4 * i][lane * E + e];
                    }
                    if (p.L.norm_w) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int e = 0; e < E; ++e) sq[i] = fmaf(v[i][e], v[i][e], sq[i]);
#pragma unroll
                        for (int d = 1; d < 32; d <<= 1)
#pragma unroll
                            for (int i = 0; i < 4; ++i) sq[i] += __shfl_xor_sync(0xffffffffu, sq[i], d);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float f = rsqrtf(sq[i] * (1.0f / DV) + p.L.eps);
#pragma unroll
                            for (int e = 0; e < E; ++e) v[i][e] *= f * nw[e];
                        }
                    }
                    if (p.io.z)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int e = 0; e < E; e += 2) {
                                const uint32_t z = *reinterpret_cast<const uint32_t*>(&sm.z[t1 + 4 * i][lane * E + e]);
                                v[i][e] *= silu(bf_lo(z));
                                v[i][e + 1] *= silu(bf_hi(z));
                            }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (t1 + 4 * i >= rows) break;
                        __nv_bfloat16* op = static_cast<__nv_bfloat16*>(p.io.out) + (size_t)(t0 + t1 + 4 * i) * p.io.ldo + col;
                        if (E == 4) *reinterpret_cast<uint2*>(op) = make_uint2(pack_bf(v[i][0], v[i][1]), pack_bf(v[i][2], v[i][3]));
                        else *reinterpret_cast<uint32_t*>(op) = pack_bf(v[i][0], v[i][1]);
                    }
                }
            }
            if (p.io.z && ok) arrive(&sm.z_free);   // not after a wait that ran out: the barrier of a copy that is still expected must not be armed again
        }
    } else if (warp == kMmaWarp) {
        // ---------------------------------------------------------------- products
        constexpr uint32_t idTok = instr_desc(Q, false, false), idUpd = instr_desc(DK, false, true);
        for (int c = 0; c < nck; ++c) {
            WideStage<DK, DV>& s = sm.stage[c % kStages];
            const uint64_t dK = operand_desc_sw128(smem_u32(s.k)), dQ = operand_desc_sw128(smem_u32(s.q)), dT = operand_desc_sw128(smem_u32(s.T)),
                           dM = operand_desc_sw128(smem_u32(s.M)), dKc = operand_desc_sw128_mn(smem_u32(s.k), 8192, 1024);
            wait(&sm.full[c % kStages], c / kStages);
            constexpr int kHands = DK / 64;   // portions in which the state comes
            auto keys = [&](int hand) {
#pragma unroll
                for (int part = 2; part >= 0; --part)
#pragma unroll
                    for (int k = hand; k < DK / 16; k += kHands)
                        mma_bf16_ts(tmem + kD1, tmem + kS + part * (DK / 2) + k * 8, dK + (uint64_t)(((k >> 2) * 8192 + (k & 3) * 32) >> 4), idTok, hand > 0 || part < 2 || k > 0);
            };
            auto tokens = [&](uint32_t to, int part, uint64_t d, int tile, int hand, bool more) {   // over half the tokens
#pragma unroll
                for (int k = 2 * hand; k < 2 * hand + 2; ++k)
                    mma_bf16_ts(tmem + to, tmem + kR + part * 32 + k * 8, d + (uint64_t)((tile * 8192 + k * 32) >> 4), idTok, more || k > 2 * hand);
            };
            // D1 = S K^T
#pragma unroll
            for (int hand = 0; hand < kHands; ++hand) {
                wait(&sm.state[hand], c);
                tc_fence_after();
                if (ok && elect_one()) {
                    keys(hand);
                    if (hand == kHands - 1) mma_commit(&sm.mma1);
                }
                __syncwarp();
            }
            if (c > 0) {
                wait(&sm.free_o, c - 1);   // the outputs ahead have left their accumulators
                tc_fence_after();
            }
            if (ok && elect_one()) {
#pragma unroll
                for (int part = 1; part >= 0; --part)
#pragma unroll
                    for (int k = 0; k < DK / 16; ++k)
                        mma_bf16_ts(tmem + kDQ, tmem + kS + part * (DK / 2) + k * 8, dQ + (uint64_t)(((k >> 2) * 8192 + (k & 3) * 32) >> 4), idTok, part < 1 || k > 0);
            }
            __syncwarp();
            // X = R T^T: the six products of parts that reach 24 bits, small ones first
#pragma unroll
            for (int hand = 0; hand < 2; ++hand) {
                wait(&sm.r[hand], c);
                tc_fence_after();
                if (ok && elect_one()) {
                    tokens(kD1, 2, dT, 0, hand, hand > 0);
                    tokens(kD1, 0, dT, 2, hand, true);
                    tokens(kD1, 1, dT, 1, hand, true);
                    tokens(kD1, 1, dT, 0, hand, true);
                    tokens(kD1, 0, dT, 1, hand, true);
                    tokens(kD1, 0, dT, 0, hand, true);
                    if (hand == 1) {
                        mma_commit(&sm.mma2);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {   // the three products of parts that reach 16 bits
                            tokens(kDO, 1, dM, 0, h, h > 0);
                            tokens(kDO, 0, dM, 1, h, true);
                            tokens(kDO, 0, dM, 0, h, true);
                        }
                        mma_commit(&sm.out);
                    }
                }
                __syncwarp();
            }
            // W K
#pragma unroll
            for (int hand = 0; hand < 2; ++hand) {
                wait(&sm.w[hand], c);
                tc_fence_after();
                if (ok && elect_one()) {
#pragma unroll
                    for (int part = 2; part >= 0; --part)
#pragma unroll
                        for (int k = 2 * hand; k < 2 * hand + 2; ++k)
                            mma_bf16_ts(tmem + kD3, tmem + kW[part] + k * 8, dKc + (uint64_t)(k * 2048 >> 4), idUpd, hand > 0 || part < 2 || k > 0);
                    if (hand == 1) mma_commit(&sm.done[c % kStages]);
                }
                __syncwarp();
            }
        }
    } else if (warp == kCopyWarp) {
        // ---------------------------------------------------------------- copies
        const int kcol = head / (p.L.n_v_heads / p.L.n_k_heads) * DK;
        for (int c = 0; c < nck; ++c) {
            if (c >= kStages) wait(&sm.done[c % kStages], c / kStages - 1);   // the chunk that had the stage is through
            if (!ok) break;
            if (lane == 0) {
                WideStage<DK, DV>& s = sm.stage[c % kStages];
                uint64_t* bar = &sm.full[c % kStages];
                const size_t ch = (size_t)(first + c) * H + head;
                mbar_expect_tx(bar, 2 * Q * DK * 2 + kGdrWideTBytes + kGdrWideMBytes + Q * DV * 2 + Q * 8);
#pragma unroll
                for (int h = 0; h < DK / 64; ++h) {
                    tma_box(s.k + h * 8192, &maps.k, kcol + 64 * h, s0 + c * Q, bar);
                    tma_box(s.q + h * 8192, &maps.q, kcol + 64 * h, s0 + c * Q, bar);
                }
                tma_box(s.v, &maps.v, head * DV, s0 + c * Q, bar);
                bulk_load(s.T, ws.T + ch * kGdrWideTBytes, kGdrWideTBytes, bar);
                bulk_load(s.M, ws.M + ch * kGdrWideMBytes, kGdrWideMBytes, bar);
                bulk_load(sm.ef[c % kStages], ws.ef + ch * Q, Q * 8, bar);
            }
            __syncwarp();
        }
    } else if (warp == kGateWarp && p.io.z) {
        for (int c = 0; c < nck; ++c) {
            // one buffer, asked for late: the rows are brought as far as L2 ahead of that
            if (lane == 0 && c + 1 < nck)
                asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(&maps.z)), "r"(head * DV), "r"(s0 + (c + 1) * Q) : "memory");
            if (c > 0) wait(&sm.z_free, c - 1);
            if (!ok) break;
            if (lane == 0) {
                mbar_expect_tx(&sm.z_full, Q * DV * 2);
                tma_box(sm.z, &maps.z, head * DV, s0 + c * Q, &sm.z_full);
            }
            __syncwarp();
        }
    }
    tc_fence_before();
    if (__syncthreads_or(!ok)) {   // copies target this block's shared memory, products its tensor memory: one more bounded chance
        if (warp == kMmaWarp) {
            if (elect_one()) mma_commit(&sm.last);
            __syncwarp();
            mbar_wait_bounded(&sm.last, 0u);
        }
        if (tid == 0) {
            flag(p.dev_status, MDRAFT_DEV_WAIT_EXPIRED);
            for (int i = 0; i < kStages && i < nck; ++i) {   // whatever the stage's last phase is, one of the two parities is behind it
                mbar_wait_bounded(&sm.full[i], 0u);
                mbar_wait_bounded(&sm.full[i], 1u);
            }
            if (p.io.z && nck > 0) {
                mbar_wait_bounded(&sm.z_full, 0u);
                mbar_wait_bounded(&sm.z_full, 1u);
            }
        }
        __syncthreads();
    }
    if (warp == kMmaWarp) tmem_free(tmem, 512);
}

template <int DK, int DV>
cudaError_t wide(const GdrPrefillArgs& p, const GdrChunkWs& ws, const GdrMaps& maps, cudaStream_t st) {
    constexpr int smem = sizeof(WideSmem<DK, DV>) + 1024;
    static_assert(smem <= 227 * 1024, "one block per SM");
    const cudaError_t e = allow_smem<gdr_chain_wide<DK, DV>>(smem);
    if (e != cudaSuccess) return e;
    return launch_pdl(gdr_chain_wide<DK, DV>, dim3(p.L.n_v_heads, p.n_seq), kWideThreads, smem, st, p, ws, maps);
}

}  // namespace

cudaError_t launch_gdr_chain_wide(const GdrPrefillArgs& p, const GdrChunkWs& ws, const GdrMaps& maps, int d_k, int d_v, cudaStream_t st) {
    if (d_k == 128) return d_v == 128 ? wide<128, 128>(p, ws, maps, st) : wide<128, 64>(p, ws, maps, st);
    return d_v == 128 ? wide<64, 128>(p, ws, maps, st) : wide<64, 64>(p, ws, maps, st);
}

}  // namespace mdraft
