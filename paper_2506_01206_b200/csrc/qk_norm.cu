// Norm of every query and key head and rotation of its first values by the row's position, one read and one write.
//
//     y = x / sqrt(mean x^2 + eps) w   or   x / sqrt(sum x^2 + eps) w   or   x
//     (y_a, y_b) <- rot_scale (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = position freqs[i],
//     (a, b) = (i, i + rot/2) or (2i, 2i + 1) for i < rot/2
//
// A head is 8 values (16 or 32 bytes) per lane of a lane group (2 to 32 lanes), so the sum of squares takes one to five shuffles and a
// rotation by halves finds its other half in another lane of the group.  The turns of a row (position times frequency, reduced
// to [-1/2, 1/2] turns in 64 bits, as an fp32 product is off by whole radians at positions of a million) are formed once and shared by its heads
// through shared memory.  A block takes as many rows as give each of its lane groups up to kItems heads, all loaded before the first is used.
#include "common.cuh"
#include "qk_norm.cuh"

namespace mdraft {

namespace {

constexpr int kThreads = 256, kItems = 4, kMaxRows = 16;

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// G lanes per head; `rows_per_block` rows, whose heads (row by row, queries first) the block's lane groups take in turn.
template <typename T, int G>
__global__ void __launch_bounds__(kThreads) qk_norm_kernel(const QkNormArgs p, int rows_per_block) {
    extern __shared__ float2 turns[];   // [row][rot_dim / 2] (cos, sin), times rot_scale
    constexpr int kGroups = kThreads / G;
    const int tid = threadIdx.x, l = tid % G, group = tid / G;
    const int row0 = blockIdx.x * rows_per_block, rows = min(rows_per_block, p.rows - row0);
    const int heads = p.n_q_heads + p.n_k_heads, items = rows * heads, half = p.rot_dim / 2;
    const bool mine = 8 * l < p.d_head;
    float x[kItems][8];
    auto source = [&](int item, bool& key, int64_t& row, int& h) {
        row = row0 + item / heads;
        h = item % heads;
        key = h >= p.n_q_heads;
        if (key) h -= p.n_q_heads;
    };
    for (int first = 0; first < items; first += kGroups * kItems) {   // the same trips for every thread
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int item = first + group + i * kGroups;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
            if (item < items && mine) {
                bool key; int64_t row; int h;
                source(item, key, row, h);
                const T* s = key ? static_cast<const T*>(p.k) + row * p.ldk : static_cast<const T*>(p.q) + row * p.ldq;
                load8(s + (size_t)h * p.d_head + 8 * l, x[i]);
            }
        }
        if (first == 0 && half > 0) {
            for (int i = tid; i < rows * half; i += kThreads) {
                const int r = i / half, c = i % half;
                double t = (double)__ldg(p.positions + row0 + r) * (double)__ldg(p.freqs + c) * 0.15915494309189535;   // in turns
                t -= rint(t);
                float sn, cs;
                sincospif((float)(2.0 * t), &sn, &cs);
                turns[i] = make_float2(cs * p.rot_scale, sn * p.rot_scale);
            }
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int item = first + group + i * kGroups;
            bool key; int64_t row; int h;
            source(min(item, items - 1), key, row, h);   // lanes without a head take part in the shuffles
            if (p.norm != MDRAFT_NORM_NONE) {
                float sq = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sq = fmaf(x[i][e], x[i][e], sq);
#pragma unroll
                for (int o = 1; o < G; o <<= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
                const float f = rsqrtf((p.norm == MDRAFT_NORM_RMS ? sq / (float)p.d_head : sq) + p.eps);
                const float* w = key ? p.k_w : p.q_w;
                float wv[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
                if (w && mine) load8(w + 8 * l, wv);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] *= f * wv[e];
            }
            const float2* tr = turns + (row - row0) * half;
            if (p.rot_layout == MDRAFT_ROT_PAIRS) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (8 * l + 2 * e < p.rot_dim) {
                        const float2 c = tr[4 * l + e];
                        const float a = x[i][2 * e], b = x[i][2 * e + 1];
                        x[i][2 * e] = a * c.x - b * c.y;
                        x[i][2 * e + 1] = b * c.x + a * c.y;
                    }
                }
            } else if (half > 0) {
                const int m = half / 8;   // lanes per half
                const bool low = l < m, turned = l < 2 * m;
                const int src = low ? l + m : (turned ? l - m : l);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float other = __shfl_sync(0xffffffffu, x[i][e], src, G);
                    if (turned) {
                        const float2 c = tr[8 * (low ? l : l - m) + e];
                        x[i][e] = low ? x[i][e] * c.x - other * c.y : x[i][e] * c.x + other * c.y;
                    }
                }
            }
            if (item < items && mine) {
                T* d = key ? static_cast<T*>(p.k_out) + row * p.ldko : static_cast<T*>(p.q_out) + row * p.ldqo;
                store8(d + (size_t)h * p.d_head + 8 * l, x[i]);
            }
        }
    }
}

template <typename T, int G>
cudaError_t launch(const QkNormArgs& p, cudaStream_t st) {
    // Enough rows that every lane group has kItems heads in flight, as long as that leaves two blocks per SM.
    const int heads = p.n_q_heads + p.n_k_heads;
    int rows = (kThreads / G * kItems) / heads;
    if (rows > kMaxRows) rows = kMaxRows;
    while (rows > 1 && (p.rows + rows - 1) / rows < 2 * sm_count()) --rows;
    if (rows < 1) rows = 1;
    qk_norm_kernel<T, G><<<(p.rows + rows - 1) / rows, kThreads, (size_t)rows * (p.rot_dim / 2) * sizeof(float2), st>>>(p, rows);
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
