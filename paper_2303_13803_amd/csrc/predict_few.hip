// Predictions of a few listed pairs (see fit.hip for what is computed), where nothing counts but the time until the answer is there: a workgroup a pair, in float32.
// Four lanes share a hidden unit.  Nothing is looked for or prepared before, and weights, which do not depend on the pair, are on their way to
// registers (those of layer 2, and of the first 128 columns of layer 1) before the pair's rows are known.  Bound by the latency of two loads that follow one another
// (indices, features) and four meetings; weights come from L2.  Measured: one pair of 32 features a workload through 128 units 3.5 us, 256 of them 4.2.
#include "fit_parts.h"

namespace {

typedef float float4v __attribute__((ext_vector_type(4), aligned(4)));

// max(v, 0) that keeps a NaN.
__device__ __forceinline__ float relu(float v) { return v < 0.0f ? 0.0f : v; }

template <int H>
__global__ __launch_bounds__(H * 4) void few_kernel(const FitArgs a)
{
    constexpr int WAVES = H / 16, EARLY = 8;
    __shared__ __align__(16) float x[512], h[H];
    __shared__ float sums[2][WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = tid >> 2, q = tid & 3, columns = 2 * a.F;
    const long long s = blockIdx.x;
    const int i = a.index[0][s], j = a.index[1][s];
    const float *row = a.W1 + (size_t)k * columns;
    float4v w1[EARLY];
#pragma unroll
    for (int t = 0; t < EARLY; ++t) w1[t] = 4 * q + 16 * t + 4 <= columns ? *(const float4v *)(row + 4 * q + 16 * t) : float4v{0.0f, 0.0f, 0.0f, 0.0f};
    float4 w2[H / 16];
#pragma unroll
    for (int t = 0; t < H / 16; ++t) w2[t] = *(const float4 *)(a.W2 + k * H + 4 * q + 16 * t);
    const float b1 = a.b1[k], b2 = a.b2[k], w3 = a.W3[0][k], w3s = a.W3[1] ? a.W3[1][k] : 0.0f, wsm = a.W1sm ? a.W1sm[k] : 0.0f;
    const float b3 = *a.b3[0], b3s = a.W3[1] ? *a.b3[1] : 0.0f;
    if ((unsigned)i >= (unsigned)a.rows[0] || (unsigned)j >= (unsigned)a.rows[1]) {         // (all of the workgroup agree)
        if (tid < 2 && (tid ? a.sigma[1] : a.sigma[0])) (tid ? a.sigma[1] : a.sigma[0])[s] = 0.0f;
        return;
    }
    if (wave < 2) {                                         // a side's features
        const float *from = wave ? a.X[1] + (size_t)j * a.F : a.X[0] + (size_t)i * a.F;
        float v[4], sum = 0.0f, squares = 0.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t) { v[t] = lane + 64 * t < a.F ? from[lane + 64 * t] : 0.0f; sum += v[t]; }
        if (a.norm) {
            const float mean = group_sum<64>(sum) / (float)a.F;
#pragma unroll
            for (int t = 0; t < 4; ++t) { v[t] -= mean; squares += lane + 64 * t < a.F ? v[t] * v[t] : 0.0f; }
            const float rstd = 1.0f / sqrtf(group_sum<64>(squares) / (float)a.F + a.eps);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int f = wave * a.F + lane + 64 * t;
                if (lane + 64 * t < a.F) v[t] = fmaf(v[t] * rstd, a.g[f], a.beta[f]);
            }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (lane + 64 * t < a.F) x[wave * a.F + lane + 64 * t] = v[t];
    }
    const float share = a.W1sm ? fminf(1.0f - a.X[0][(size_t)i * a.F + a.sm_feature[0]], a.X[1][(size_t)j * a.F + a.sm_feature[1]]) : 0.0f;
    __syncthreads();
    float z = 0.0f;
#pragma unroll
    for (int t = 0; t < EARLY; ++t) {
        const int c = 4 * q + 16 * t;
        if (c + 4 > columns) break;
        const float4 u = *(const float4 *)(x + c);
        z = fmaf(w1[t].w, u.w, fmaf(w1[t].z, u.z, fmaf(w1[t].y, u.y, fmaf(w1[t].x, u.x, z))));
    }
    for (int c = 4 * q + 16 * EARLY; c + 4 <= columns; c += 16) {
        const float4v w = *(const float4v *)(row + c);
        const float4 u = *(const float4 *)(x + c);
        z = fmaf(w.w, u.w, fmaf(w.z, u.z, fmaf(w.y, u.y, fmaf(w.x, u.x, z))));
    }
    if (q < columns % 4) z = fmaf(row[(columns & ~3) + q], x[(columns & ~3) + q], z);
    z = group_sum<4>(z) + b1;
    if (a.W1sm) z = fmaf(share, wsm, z);
    if (q == 0) h[k] = relu(z);
    __syncthreads();
    z = 0.0f;
#pragma unroll
    for (int t = 0; t < H / 16; ++t) {
        const float4 u = *(const float4 *)(h + 4 * q + 16 * t);
        z = fmaf(w2[t].w, u.w, fmaf(w2[t].z, u.z, fmaf(w2[t].y, u.y, fmaf(w2[t].x, u.x, z))));
    }
    z = group_sum<4>(z) + b2;                               // (by all four lanes)
    const float d2 = q == 0 ? relu(z) : 0.0f;
    const float p = group_sum<64>(d2 * w3), ps = group_sum<64>(d2 * w3s);
    if (lane == 0) { sums[0][wave] = p; sums[1][wave] = ps; }
    __syncthreads();
    float *const to = tid ? a.sigma[1] : a.sigma[0];
    if (tid > 1 || !to) return;
    z = tid ? b3s : b3;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) z += sums[tid][w];
    to[s] = 1.0f / (1.0f + expf(-z));
}

}  // namespace

int mf_launch_few(mf_ctx *ctx, const FitArgs &a, int H)
{
    if (H == 64) hipLaunchKernelGGL((few_kernel<64>), dim3((unsigned)a.count), dim3(256), 0, ctx->stream, a);
    else hipLaunchKernelGGL((few_kernel<128>), dim3((unsigned)a.count), dim3(512), 0, ctx->stream, a);
    MF_HIP(hipGetLastError());
    return MF_OK;
}
