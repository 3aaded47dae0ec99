// Norm of every query and key head and rotation of its first values by the row's position, one read and one write.
//
//     y = x / sqrt(mean x^2 + eps) w   or   x / sqrt(sum x^2 + eps) w   or   x
//     (y_a, y_b) <- rot_scale (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = position freqs[i],
//     (a, b) = (i, i + rot/2) or (2i, 2i + 1) for i < rot/2
//
// A head is 8 values per lane of a lane group (4 to 32 lanes), so the sum of squares takes two to five shuffles; a rotation by halves has four values of
// either half in a lane (two loads of 8 or 16 bytes), so that it takes none.  The turns of a row (position times frequency, reduced
// to [-1/2, 1/2] turns in 64 bits, as an fp32 product is off by whole radians at positions of a million) are formed once and shared by its heads
// through shared memory.  A block works through passes of rows and has the next one's loads in flight meanwhile.  Bound: memory.  Measured (bf16, 12 + 4 heads): heads of 64, 32
// values turned, 141000 rows 112 us on the device (119 a call), 5.2 TB/s (200 us with one head per thread and pass, without loads ahead; issue slots are nearly as full); heads of 128, all turned, 2048 rows 6.2
// us on the device (8.2 a call).
#include "common.cuh"
#include "qk_norm.cuh"

namespace mdraft {

namespace {

template <typename T> constexpr int kItemsOf = 8 / sizeof(T);   // heads a lane group has in flight: 64 bytes a lane
constexpr int kThreads = 256, kMaxThreads = 512;       // of a block as a rule, and where the heads of a row ask for more

constexpr size_t kMaxTurnBytes = 48 * 1024;             // of shared memory, what a block may have without asking

// Two times four values as they lie in memory, beside one another or not, and as packed pairs of fp32.
template <typename T> struct Raw;
template <> struct Raw<float> {
    float4 a, b;
    template <bool kBeside>
    __device__ __forceinline__ void load(const float* p, int to_b) {
        a = *reinterpret_cast<const float4*>(p);
        b = *reinterpret_cast<const float4*>(p + (kBeside ? 4 : to_b));
    }
    __device__ __forceinline__ void widen(u64 (&v)[4]) const { v[0] = pk(a.x, a.y); v[1] = pk(a.z, a.w); v[2] = pk(b.x, b.y); v[3] = pk(b.z, b.w); }
    template <bool kBeside>
    __device__ static __forceinline__ void store(float* p, int to_b, const float (&v)[8]) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(p + (kBeside ? 4 : to_b)) = make_float4(v[4], v[5], v[6], v[7]);
    }
};
template <> struct Raw<__nv_bfloat16> {
    uint4 w;
    template <bool kBeside>
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int to_b) {
        if (kBeside) { w = *reinterpret_cast<const uint4*>(p); return; }
        const uint2 a = *reinterpret_cast<const uint2*>(p), b = *reinterpret_cast<const uint2*>(p + to_b);
        w = make_uint4(a.x, a.y, b.x, b.y);
    }
    __device__ __forceinline__ void widen(u64 (&v)[4]) const {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pk(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
    }
    __device__ static __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&b);
    }
    template <bool kBeside>
    __device__ static __forceinline__ void store(__nv_bfloat16* p, int to_b, const float (&v)[8]) {
        const uint2 a = make_uint2(pack(v[0], v[1]), pack(v[2], v[3])), b = make_uint2(pack(v[4], v[5]), pack(v[6], v[7]));
        if (kBeside) { *reinterpret_cast<uint4*>(p) = make_uint4(a.x, a.y, b.x, b.y); return; }
        *reinterpret_cast<uint2*>(p) = a;
        *reinterpret_cast<uint2*>(p + to_b) = b;
    }
};

// How the work is cut.  A block takes `heads` heads (a part of a row's where there are more than fit) of `row_lanes` rows side by side, a lane group each: so a
// group has the same head throughout.  A pass is `items` such steps.
struct Cut {
    int heads, row_lanes, items, passes;
};

// G lanes per head.  A block loads its next pass before it works on the one at hand, and forms the next rows' turns behind it.
template <typename T, int G, bool kHalf>
__global__ void __launch_bounds__(kMaxThreads, 2) qk_norm_kernel(const QkNormArgs p, const Cut cut) {
    extern __shared__ __align__(16) float2 turns[];   // [2][row of the pass][rot_dim / 2, rounded up to 4] (cos, sin), times rot_scale
    constexpr int kItems = kItemsOf<T>;
    const int tid = threadIdx.x, l = tid % G, group = tid / G;
    const int lane_row = group / cut.heads, in_part = group - lane_row * cut.heads, half = p.rot_dim / 2, pitch = (half + 3) & ~3;
    const int h = blockIdx.y * cut.heads + in_part, per_pass = cut.row_lanes * cut.items;
    const bool key = h >= p.n_q_heads && p.n_k_heads > 0;   // (a group behind the last head reads along with its rows and strides, and writes nothing)
    const bool mine = lane_row < cut.row_lanes && h < p.n_q_heads + p.n_k_heads && 8 * l < p.d_head;
    // A rotation by halves takes four values of either half into a lane, so that every pair is in one lane.
    const bool turned = 8 * l < p.rot_dim;
    const int at = kHalf && turned ? 4 * l : 8 * l, to_b = kHalf && turned ? half : 4;
    const int64_t column = mine ? (int64_t)(key ? h - p.n_q_heads : h) * p.d_head + at : 0, ld = key ? p.ldk : p.ldq, ldo = key ? p.ldko : p.ldqo;
    const T* from = static_cast<const T*>(key ? p.k : p.q) + column;
    T* to = static_cast<T*>(key ? p.k_out : p.q_out) + column;
    const int reach = mine ? to_b : 4;
    const float per_value = p.norm == MDRAFT_NORM_RMS ? 1.0f / (float)p.d_head : 1.0f;
    u64 weight[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) weight[e] = pk(1.0f, 1.0f);
    if (const float* w = key ? p.k_w : p.q_w; w && mine && p.norm != MDRAFT_NORM_NONE)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float* pair = w + at + (e < 2 ? 2 * e : to_b + 2 * e - 4);
            weight[e] = pk(__ldg(pair), __ldg(pair + 1));
        }
    Raw<T> raw[kItems];
    auto load = [&](int pass) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int row = pass * per_pass + i * cut.row_lanes + lane_row;
            if (i < cut.items) raw[i].template load<!kHalf>(from + (row < p.rows ? row : p.rows - 1) * ld, reach);
        }
    };
    const int step_r = half > 0 ? blockDim.x / half : 0, step_c = half > 0 ? blockDim.x - step_r * half : 0;   // of the next value a thread turns
    auto turn = [&](int pass, float2* out) {
        const int row0 = pass * per_pass, n = min(per_pass, p.rows - row0) * half;
        int r = tid / half, c = tid - r * half;
        for (int i = tid; i < n; i += blockDim.x) {
            double t = (double)__ldg(p.positions + row0 + r) * (double)__ldg(p.freqs + c) * 0.15915494309189535;   // in turns
            t -= rint(t);
            float sn, cs;
            sincospif((float)(2.0 * t), &sn, &cs);
            out[r * pitch + c] = make_float2(cs * p.rot_scale, sn * p.rot_scale);
            r += step_r;
            c += step_c;
            if (c >= half) { c -= half; ++r; }
        }
    };
    const int pairs = kHalf ? 4 : (p.rot_dim - 8 * l) / 2;   // of the lane that are turned
    int pass = blockIdx.x, buffer = 0;
    load(pass);
    if (half > 0) {
        turn(pass, turns);
        __syncthreads();
    }
    for (; pass < cut.passes; pass += gridDim.x, buffer ^= 1) {
        Raw<T> now[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) now[i] = raw[i];
        const int next = pass + gridDim.x;
        if (next < cut.passes) load(next);
        const float2* tr = turns + (buffer * per_pass + (mine ? lane_row : 0)) * pitch;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {   // lanes without a head take part in the shuffles
            if (i >= cut.items) break;
            const int row = pass * per_pass + i * cut.row_lanes + lane_row;
            u64 v[4];
            now[i].widen(v);
            if (p.norm != MDRAFT_NORM_NONE) {
                u64 sum = 0ull;
#pragma unroll
                for (int e = 0; e < 4; ++e) sum = fma2(v[e], v[e], sum);
                float sq, odd;
                unpk(sum, sq, odd);
                sq = mine ? sq + odd : 0.f;
#pragma unroll
                for (int o = 1; o < G; o <<= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
                const float f = rsqrtf(fmaf(sq, per_value, p.eps));
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = mul2(v[e], mul2(pk(f, f), weight[e]));
            }
            float x[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) unpk(v[e], x[2 * e], x[2 * e + 1]);
            if (turned) {
                const float4* t = reinterpret_cast<const float4*>(tr + i * cut.row_lanes * pitch + 4 * l);
                const float4 t0 = t[0], t1 = t[1];
                const float c[4] = {t0.x, t0.z, t1.x, t1.z}, sn[4] = {t0.y, t0.w, t1.y, t1.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float& a = x[kHalf ? e : 2 * e];
                    float& b = x[kHalf ? e + 4 : 2 * e + 1];
                    if (e < pairs) {
                        const float was = a;
                        a = fmaf(-b, sn[e], was * c[e]);
                        b = fmaf(was, sn[e], b * c[e]);
                    }
                }
            }
            if (mine && row < p.rows) Raw<T>::template store<!kHalf>(to + row * ldo, to_b, x);
        }
        if (half > 0 && next < cut.passes) {
            turn(next, turns + (buffer ^ 1) * per_pass * pitch);
            __syncthreads();
        }
    }
}

template <typename T, int G>
cudaError_t launch(const QkNormArgs& p, cudaStream_t st) {
    const int heads = p.n_q_heads + p.n_k_heads;
    Cut cut;
    cut.heads = heads < kMaxThreads / G ? heads : kMaxThreads / G;
    cut.row_lanes = kThreads / (cut.heads * G) > 0 ? kThreads / (cut.heads * G) : 1;
    const int parts = (heads + cut.heads - 1) / cut.heads, threads = (cut.heads * cut.row_lanes * G + 31) / 32 * 32;
    // Few rows are spread over the SMs, many are taken by as many blocks as fit at once.
    cut.items = kItemsOf<T>;
    auto passes = [&] { return (p.rows + cut.row_lanes * cut.items - 1) / (cut.row_lanes * cut.items); };
    while (cut.items > 1 && passes() * (int64_t)parts < 2 * sm_count()) --cut.items;
    while (cut.row_lanes > 1 && passes() * (int64_t)parts < 2 * sm_count()) cut.row_lanes /= 2;
    auto smem_bytes = [&] { return 2 * (size_t)(cut.row_lanes * cut.items) * ((p.rot_dim / 2 + 3) & ~3) * sizeof(float2); };
    while (cut.items > 1 && smem_bytes() > kMaxTurnBytes) --cut.items;   // one or two heads to a row, most of their values turned
    cut.passes = passes();
    const int most = (2 * kMaxThreads / threads) * sm_count() / parts;   // resident at once
    const int blocks = cut.passes < most ? cut.passes : (most > 0 ? most : 1);
    const size_t smem = smem_bytes();
    if (p.rot_layout == MDRAFT_ROT_HALF) qk_norm_kernel<T, G, true><<<dim3(blocks, parts), threads, smem, st>>>(p, cut);
    else qk_norm_kernel<T, G, false><<<dim3(blocks, parts), threads, smem, st>>>(p, cut);
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch_width(const QkNormArgs& p, cudaStream_t st) {
    const int lanes = (p.d_head + 7) / 8;
    if (lanes <= 4) return launch<T, 4>(p, st);
    if (lanes <= 8) return launch<T, 8>(p, st);
    if (lanes <= 16) return launch<T, 16>(p, st);
    return launch<T, 32>(p, st);
}

}  // namespace

cudaError_t launch_qk_norm(const QkNormArgs& p, int act, cudaStream_t st) {
    return act == MDRAFT_BF16 ? launch_width<__nv_bfloat16>(p, st) : launch_width<float>(p, st);
}

}  // namespace mdraft
