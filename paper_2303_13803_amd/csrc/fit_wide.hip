// The pass over the samples in float32 products: of predictors of many features (65 to 256 a workload), and where a feature that no norm
// bounds is too large for pieces (FIT_LARGEST).  Features are staged 64 columns at a time, twice a sample, and gradients of layer 1 are kept for 256 columns at a
// time, which is as many as there are accumulators for: more take another pass over the samples each.  See fit.hip for what is computed.
// Measured with 128 units: 100,000 samples of 65 features 0.48 ms (35 TFLOP/s; float32's matrix instructions reach 152), 30,000 of 256 0.47, 200,003 predictions of 100
// 0.31; bound by waits between its stages, with one workgroup a compute unit (LDS lets no second one in), and with 91 vector registers in memory.
#include "fit_parts.h"

namespace {

constexpr int FIT_ROWS = 64, FIT_CHUNK = 64;                // samples a workgroup takes at a time; features staged at a time

// max(v, 0) that keeps a NaN: a fit that has diverged shows.
__device__ __forceinline__ float relu(float v) { return v < 0.0f ? 0.0f : v; }

template <int H>
constexpr size_t wide_lds_bytes(bool grad)
{
    return sizeof(float) * ((size_t)H * (H + 4) + FIT_ROWS * (FIT_CHUNK + 4) + (size_t)FIT_ROWS * (H + 4) * (grad ? 2 : 1) +
                            2 * (H / 32) * FIT_ROWS + FIT_ROWS * 6 + 4 * FIT_ROWS + 5 * H);
}

template <int H, int GT, bool GRAD>
__global__ __launch_bounds__(H * 4) void wide_kernel(const FitArgs a, const float *__restrict__ ranges, const int parts)
{
    if (parts > 0) {                                        // where nothing is too large fit_kernel's results stay, else all of them are written again
        float most = 0.0f;
        for (int k = threadIdx.x & 63; k < parts; k += 64) most = fmaxf(most, ranges[k]);
        if (!(wave_max(most) > FIT_LARGEST)) return;
    }
    constexpr int T = FIT_ROWS, PITCH = H + 4, XP = FIT_CHUNK + 4, UB = H / 32, THREADS = H * 4, QUADS = H / 8;
    using S = FitSums<H>;
    extern __shared__ __align__(16) float lds[];
    float *w2 = lds, *xs = w2 + H * PITCH, *act = xs + T * XP, *back = act + T * PITCH;
    float *part = back + (GRAD ? T * PITCH : 0), *target = part + 2 * UB * T, *target_slow = target + T, *share = target_slow + T;
    int *at_on = (int *)(share + T), *at_off = at_on + T;
    float2 *moments = (float2 *)(at_off + T);
    float *bad = (float *)(moments + 2 * T);                // with gradients: NaN where a sample's features are not finite, which are 0 then (see fit.hip)
    float *vec = bad + T;                                   // b1, b2, W3, W3 of the slowdown unit, W1sm
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nn = lane & 31, hh = lane >> 5;
    const int ub = wave % UB, sh = wave / UB;               // units 32 ub .. and samples 32 sh .. of the forward pass are this wavefront's
    const int unit = 32 * ub + tile_unit(nn), mine = 32 * sh + nn, u0 = 32 * ub + 8 * hh;
    DropRule rule = a.rule;
    if (a.step) { const unsigned long long s = *a.step; rule.s0 = (unsigned)s; rule.s1 = (unsigned)(s >> 32); }

    for (int e = tid; e < H * H / 4; e += THREADS) *(float4 *)(w2 + e / (H / 4) * PITCH + e % (H / 4) * 4) = ((const float4 *)a.W2)[e];
    for (int e = tid; e < H; e += THREADS) {
        vec[e] = a.b1[e];
        vec[H + e] = a.b2[e];
        vec[2 * H + e] = a.W3[0][e];
        vec[3 * H + e] = a.W3[1] ? a.W3[1][e] : 0.0f;
        vec[4 * H + e] = a.W1sm ? a.W1sm[e] : 0.0f;
    }
    const float b3 = *a.b3[0], b3s = a.W3[1] ? *a.b3[1] : 0.0f;
    const float factor = a.drop ? rule.factor : 1.0f;
    const int chunks = (a.padded + FIT_CHUNK - 1) / FIT_CHUNK;
    const int pass_chunk = blockIdx.y * GT;                 // this pass keeps gradients of layer 1 from this chunk on

    floatx16 gw2[UB / 2], gw1[GT];
    // gw3, gw3s: sums of the 16 units of a half over the wavefront's samples, lane nn of a half keeps that of unit nn; gb1, gb2, gsm: of unit
    // 32 ub + nn over all of the workgroup's that this half reads
    float gb1 = 0.0f, gb2 = 0.0f, gw3 = 0.0f, gw3s = 0.0f, gsm = 0.0f, gb3 = 0.0f, gb3s = 0.0f, loss = 0.0f;
    if (GRAD) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
#pragma unroll
            for (int t = 0; t < UB / 2; ++t) gw2[t][e] = 0.0f;
#pragma unroll
            for (int t = 0; t < GT; ++t) gw1[t][e] = 0.0f;
        }
    }
    // Features of columns 64 chunk .. 64 chunk + 63 are fetched a stage before they are laid into LDS (waited for one by one they took 12 us a
    // chunk, together 3).
    constexpr int EACH_FEATURE = T * FIT_CHUNK / THREADS;
    float feature[EACH_FEATURE];
    auto fetch = [&](const int chunk) {
        const int c = chunk * FIT_CHUNK + tid % FIT_CHUNK, side = c >= a.half, f = c - side * a.half;
        const float *X = (side ? a.X[1] : a.X[0]) + f;
#pragma unroll
        for (int k = 0; k < EACH_FEATURE; ++k) {
            const int s = tid / FIT_CHUNK + k * (THREADS / FIT_CHUNK), at = side ? at_off[s] : at_on[s];
            feature[k] = f < a.F && at >= 0 ? X[(size_t)at * a.F] : 0.0f;
        }
    };
    auto lay = [&](const int chunk) {
        unsigned not_finite = 0;
        const int c = chunk * FIT_CHUNK + tid % FIT_CHUNK, side = c >= a.half, f = c - side * a.half;
#pragma unroll
        for (int k = 0; k < EACH_FEATURE; ++k) {
            const int s = tid / FIT_CHUNK + k * (THREADS / FIT_CHUNK);
            const float2 m = moments[2 * s + side];
            const float v = f < a.F && at_on[s] >= 0 ? (feature[k] - m.x) * m.y : 0.0f;
            const bool finite = !GRAD || fabsf(v) < INFINITY;
            xs[s * XP + tid % FIT_CHUNK] = finite ? v : 0.0f;
            not_finite |= finite ? 0u : 1u << k;
        }
        if (GRAD && not_finite)
#pragma unroll 1
            for (int k = 0; k < EACH_FEATURE; ++k)
                if (not_finite >> k & 1u) bad[tid / FIT_CHUNK + k * (THREADS / FIT_CHUNK)] = __builtin_nanf("");
    };
    // bias, ReLU and dropout of this lane's 16 units of one layer
    auto activate = [&](const floatx16 &z, float (&h)[16], const float *bias, const float share_here, long long sample, unsigned layer) {
#pragma unroll
        for (int k = 0; k < 16; ++k) h[k] = z[k] + bias[u0 + 16 * (k >> 3) + (k & 7)];
        if (layer == 0 && a.W1sm)
#pragma unroll
            for (int k = 0; k < 16; ++k) h[k] = fmaf(share_here, vec[4 * H + u0 + 16 * (k >> 3) + (k & 7)], h[k]);
#pragma unroll
        for (int k = 0; k < 16; ++k) h[k] = relu(h[k]);
        if (a.drop)
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const Words4 bits = drop_bits(rule, (unsigned long long)sample * (H / 8) + (u0 + 16 * g) / 8, layer);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[8 * g + e] = drop_keeps(rule, bits, e) ? h[8 * g + e] * factor : 0.0f;
            }
    };
    auto add_lane = [&](float &sum, const int k, const float v) {
        const float all = group_sum<32>(v);
        sum += nn == k ? all : 0.0f;
    };
    auto put = [&](float *to, const float (&h)[16]) {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int q = 0; q < 2; ++q)
                *(float4 *)(to + mine * PITCH + u0 + 16 * g + 4 * q) = make_float4(h[8 * g + 4 * q], h[8 * g + 4 * q + 1], h[8 * g + 4 * q + 2], h[8 * g + 4 * q + 3]);
    };

    const long long tiles = (a.count + T - 1) / T;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        __syncthreads();                                    // everybody is done with the last samples
        if (tid < T) {
            const long long s = tile * T + tid;
            int i = -1, j = -1;
            if (s < a.count) { i = a.index[0][s]; j = a.index[1][s]; }
            // a sample that names no pair has no part in anything
            if (i < 0 || i >= a.rows[0] || j < 0 || j >= a.rows[1]) i = j = -1;
            at_on[tid] = i;
            at_off[tid] = j;
            const float none = __builtin_nanf("");
            target[tid] = i >= 0 && a.target[0] ? a.target[0][s] : none;
            target_slow[tid] = i >= 0 && a.target[1] ? a.target[1][s] : none;
            float at = i >= 0 && a.W1sm ? fminf(1.0f - a.X[0][(size_t)i * a.F + a.sm_feature[0]], a.X[1][(size_t)j * a.F + a.sm_feature[1]]) : 0.0f;
            bad[tid] = 0.0f;
            if (GRAD && !(at * 0.0f == 0.0f)) {
                at = 0.0f;
                bad[tid] = none;
            }
            share[tid] = at;
        }
        __syncthreads();
        fetch(0);
        {   // moments of the samples' feature rows, 2 T of them, by THREADS / (2 T) neighbouring lanes each
            constexpr int EACH = THREADS / (2 * T);
            const int r = tid / EACH, sub = tid % EACH, side = r & 1;
            const int at = side ? at_off[r >> 1] : at_on[r >> 1];
            float2 m = make_float2(0.0f, 1.0f);
            if (a.norm && at >= 0) {                        // (the lanes of a row agree)
                const float *x = (side ? a.X[1] : a.X[0]) + (size_t)at * a.F;
                float sum = 0.0f, squares = 0.0f;
#pragma unroll 8
                for (int f = sub; f < a.F; f += EACH) sum += x[f];
                m.x = group_sum<EACH>(sum) / (float)a.F;
#pragma unroll 8
                for (int f = sub; f < a.F; f += EACH) { const float d = x[f] - m.x; squares = fmaf(d, d, squares); }
                m.y = 1.0f / sqrtf(group_sum<EACH>(squares) / (float)a.F + a.eps);
            }
            if (sub == 0) moments[r] = m;
        }
        __syncthreads();
        floatx16 z;
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = 0.0f;
        for (int c = 0; c < chunks; ++c) {
            if (c > 0) __syncthreads();
            const int quads = (a.padded - c * FIT_CHUNK < FIT_CHUNK ? a.padded - c * FIT_CHUNK : FIT_CHUNK) / 8;
            float4 w1[FIT_CHUNK / 8];                       // (on their way while features are staged)
#pragma unroll
            for (int q = 0; q < FIT_CHUNK / 8; ++q)
                w1[q] = *(const float4 *)(a.W1 + (size_t)unit * a.padded + c * FIT_CHUNK + (q < quads ? 8 * q : 0) + 4 * hh);
            lay(c);
            __syncthreads();
            if (c + 1 < chunks) fetch(c + 1);
#pragma unroll
            for (int q = 0; q < FIT_CHUNK / 8; ++q) {
                if (q >= quads) break;
                const float4 w = w1[q];
                const float4 x = *(const float4 *)(xs + mine * XP + 8 * q + 4 * hh);
                z = __builtin_amdgcn_mfma_f32_32x32x2f32(w.x, x.x, z, 0, 0, 0);
                z = __builtin_amdgcn_mfma_f32_32x32x2f32(w.y, x.y, z, 0, 0, 0);
                z = __builtin_amdgcn_mfma_f32_32x32x2f32(w.z, x.z, z, 0, 0, 0);
                z = __builtin_amdgcn_mfma_f32_32x32x2f32(w.w, x.w, z, 0, 0, 0);
            }
        }
        const long long sample = tile * T + mine;
        const bool real = at_on[mine] >= 0;
        float h1[16], h2[16];
        activate(z, h1, vec, share[mine], sample, 0);
        put(act, h1);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = 0.0f;
#pragma unroll 2
        for (int q = 0; q < QUADS; ++q) {
            const float4 w = *(const float4 *)(w2 + unit * PITCH + 8 * q + 4 * hh);
            const float4 x = *(const float4 *)(act + mine * PITCH + 8 * q + 4 * hh);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w.x, x.x, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w.y, x.y, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w.z, x.z, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w.w, x.w, z, 0, 0, 0);
        }
        activate(z, h2, vec + H, 0.0f, sample, 1);
        float zp = 0.0f, zs = 0.0f;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                zp = fmaf(vec[2 * H + u0 + 16 * g + e], h2[8 * g + e], zp);
                if (a.W3[1]) zs = fmaf(vec[3 * H + u0 + 16 * g + e], h2[8 * g + e], zs);
            }
        zp = both_halves(zp);
        zs = both_halves(zs);
        if (hh == 0) { part[ub * T + mine] = zp; part[(UB + ub) * T + mine] = zs; }
        __syncthreads();
        zp = b3 + bad[mine]; zs = b3s + bad[mine];
#pragma unroll
        for (int k = 0; k < UB; ++k) { zp += part[k * T + mine]; zs += part[(UB + k) * T + mine]; }
        const float y = 1.0f / (1.0f + expf(-zp)), ys = 1.0f / (1.0f + expf(-zs));
        const bool speaks = ub == 0 && hh == 0 && blockIdx.y == 0;      // for its sample, among the wavefronts and passes that hold it
        if (speaks && sample < a.count) {
            if (a.sigma[0]) a.sigma[0][sample] = real ? y : 0.0f;
            if (a.sigma[1]) a.sigma[1][sample] = real ? ys : 0.0f;
        }
        // what nobody has measured (a NaN) has no part in the loss
        const float t0 = target[mine], t1 = target_slow[mine];
        const float miss = t0 == t0 ? y - t0 : 0.0f, miss_slow = t1 == t1 ? ys - t1 : 0.0f;
        if (speaks) loss += fmaf(miss, miss, miss_slow * miss_slow);
        if (!GRAD) continue;
        const float dz = t0 == t0 ? 2.0f * miss * y * (1.0f - y) : 0.0f;        // (the caller's scale comes last)
        const float dzs = t1 == t1 ? 2.0f * miss_slow * ys * (1.0f - ys) : 0.0f;
        if (speaks) { gb3 += dz; gb3s += dzs; }
        float d[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            d[k] = dz * vec[2 * H + u0 + 16 * (k >> 3) + (k & 7)];
            add_lane(gw3, k, dz * h2[k]);
        }
        if (a.W3[1])
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                d[k] = fmaf(dzs, vec[3 * H + u0 + 16 * (k >> 3) + (k & 7)], d[k]);
                add_lane(gw3s, k, dzs * h2[k]);
            }
#pragma unroll
        for (int k = 0; k < 16; ++k) d[k] = h2[k] > 0.0f ? d[k] * factor : 0.0f;
        put(back, d);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = 0.0f;
#pragma unroll 2
        for (int q = 0; q < QUADS; ++q) {                   // W2^T dz2
            const float *w = w2 + (8 * q + 4 * hh) * PITCH + unit;
            const float4 x = *(const float4 *)(back + mine * PITCH + 8 * q + 4 * hh);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w[0], x.x, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w[PITCH], x.y, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w[2 * PITCH], x.z, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w[3 * PITCH], x.w, z, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) d[k] = h1[k] > 0.0f ? z[k] * factor : 0.0f;
        if (chunks > 1) fetch(pass_chunk);
        // sums over samples: the lower half of a wavefront takes sample 16 b + i, the upper one 16 b + 8 + i
#pragma unroll 1
        for (int b = 0; b < T / 16; ++b)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int s = (16 * b + i + 8 * hh) * PITCH;
                const float v = back[s + 32 * ub + nn];
                gb2 += v;
#pragma unroll
                for (int t = 0; t < UB / 2; ++t)
                    gw2[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, act[s + 32 * (sh + 2 * t) + nn], gw2[t], 0, 0, 0);
            }
        __syncthreads();                                    // act has been read
        put(act, d);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < GT; ++t) {
            const int c = pass_chunk + t;
            if (c >= chunks) break;
            if (chunks > 1) {
                if (t > 0) __syncthreads();
                lay(c);
                __syncthreads();
                if (t + 1 < GT && c + 1 < chunks) fetch(c + 1);
            }
            if (c * FIT_CHUNK + 32 * sh >= a.padded) continue;      // (the last chunk may be half as wide)
#pragma unroll 1
            for (int b = 0; b < T / 16; ++b)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int s = 16 * b + i + 8 * hh;
                    if (t == 0) {
                        const float v = act[s * PITCH + 32 * ub + nn];
                        gb1 += v;
                        gsm = fmaf(share[s], v, gsm);
                    }
                    gw1[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(act[s * PITCH + 32 * ub + nn], xs[s * XP + 32 * sh + nn], gw1[t], 0, 0, 0);
                }
        }
    }

    // what this workgroup leaves
    if (!a.partial) return;
    float *out = a.partial + (size_t)blockIdx.x * a.partial_step;
    if (GRAD) {
        const int row = 4 * hh;                             // rows 8 g + 4 hh + e of a tile are this lane's
#pragma unroll
        for (int t = 0; t < GT; ++t) {
            const int c = (pass_chunk + t) * FIT_CHUNK + 32 * sh;
            if (c >= a.padded) continue;
#pragma unroll
            for (int e = 0; e < 16; ++e) out[S::G + (size_t)(32 * ub + 8 * (e >> 2) + row + (e & 3)) * a.padded + c + nn] = gw1[t][e];
        }
        if (blockIdx.y > 0) return;
#pragma unroll
        for (int t = 0; t < UB / 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) out[S::W2 + (32 * ub + 8 * (e >> 2) + row + (e & 3)) * H + 32 * (sh + 2 * t) + nn] = gw2[t][e];
        gb1 = both_halves(gb1);
        gb2 = both_halves(gb2);
        gsm = both_halves(gsm);
        if (sh == 0 && hh == 0) {
            out[S::B1 + 32 * ub + nn] = gb1;
            out[S::B2 + 32 * ub + nn] = gb2;
            out[S::SM + 32 * ub + nn] = gsm;
        }
        // the output weights': over the two wavefronts that hold a unit
        float *sums = act;                                  // [2][2][H]
        __syncthreads();
        if (nn < 16) {
            sums[sh * H + u0 + (nn >> 3) * 16 + (nn & 7)] = gw3;
            sums[(2 + sh) * H + u0 + (nn >> 3) * 16 + (nn & 7)] = gw3s;
        }
        __syncthreads();
        for (int e = tid; e < 2 * H; e += THREADS) out[S::W3 + e] = sums[2 * (e / H) * H + e % H] + sums[(2 * (e / H) + 1) * H + e % H];
    }
    const float v[3] = {group_sum<64>(gb3), group_sum<64>(gb3s), group_sum<64>(loss)};
    __syncthreads();
    if (lane == 0 && ub == 0)
#pragma unroll
        for (int q = 0; q < 3; ++q) part[3 * sh + q] = v[q];
    __syncthreads();
    if (tid < 3) out[S::REST + tid] = part[tid] + part[3 + tid];
}

template <int H, int GT, bool GRAD>
int launch_wide(mf_ctx *ctx, const FitArgs &a, const FitPlan &f, const float *ranges)
{
    constexpr unsigned long long flag = lds_bit_wide(H, GRAD);
    if (!(ctx->kernels_configured & flag)) {
        MF_HIP(hipFuncSetAttribute((const void *)wide_kernel<H, GT, GRAD>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)wide_lds_bytes<H>(GRAD)));
        ctx->kernels_configured |= flag;
    }
    hipLaunchKernelGGL((wide_kernel<H, GT, GRAD>), dim3(f.grid, GRAD ? f.passes : 1), dim3(H * 4), wide_lds_bytes<H>(GRAD), ctx->stream, a, ranges, f.parts);
    MF_HIP(hipGetLastError());
    return MF_OK;
}

}  // namespace

constexpr int FIT_WIDE_TILES = 4;

void mf_plan_wide(const mf_ctx *ctx, long long count, FitPlan *f)
{
    f->half = f->columns / 2;
    f->padded = (f->columns + 31) & ~31;
    const int chunks = (f->padded + FIT_CHUNK - 1) / FIT_CHUNK;
    f->passes = (chunks + FIT_WIDE_TILES - 1) / FIT_WIDE_TILES;
    const long long tiles = (count + FIT_ROWS - 1) / FIT_ROWS, units = (ctx->n_cus > 0 ? ctx->n_cus : 256) * (f->H == 64 ? 2 : 1);
    f->grid = (int)(tiles < units ? tiles : units);
}

int mf_launch_wide(mf_ctx *ctx, const FitArgs &a, const FitPlan &f, const float *ranges, bool grad)
{
    if (f.H == 64) return grad ? launch_wide<64, FIT_WIDE_TILES, true>(ctx, a, f, ranges) : launch_wide<64, 1, false>(ctx, a, f, ranges);
    return grad ? launch_wide<128, FIT_WIDE_TILES, true>(ctx, a, f, ranges) : launch_wide<128, 1, false>(ctx, a, f, ranges);
}

