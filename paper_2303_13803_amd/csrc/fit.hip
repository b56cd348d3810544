// Fitting a speed predictor: its loss over listed pairs with every gradient, and its predictions for listed pairs (paper:
// Section "Implementation", the predictor is trained on profiled pairs).
//
// For a sample s = (i, j, t), with u the features of both workloads, normalised where the predictor has a layer norm:
//     x = g u + beta,  z1 = W1 x + b1 (+ share W1sm),  d1 = drop(relu(z1)),  z2 = W2 d1 + b2,  d2 = drop(relu(z2)),
//     y = logistic(W3 d2 + b3),  loss = scale sum (y - t)^2  (and the same of the slowdown unit),
//     dz3 = 2 scale (y - t) y (1 - y),  dz2 = [d2 > 0] c W3 dz3,  dz1 = [d1 > 0] c W2^T dz2,
//     dW2 = sum dz2 d1^T,  G = sum dz1 u^T,  h = sum dz1.
// The norm's weight and bias fold into layer 1, and their gradients come out of sums that layer 1's needs anyway:
//     W1 x + b1 = (W1 diag g) u + (b1 + W1 beta),  dW1 = G diag g + h beta^T,  dg_f = sum_k W1[k,f] G[k,f],  dbeta = W1^T h,
// so a sample costs no more than without it.
//
// A workgroup takes FIT_ROWS samples at a time through all of that; activations pass from wavefront to wavefront through LDS and
// gradients of weights stay in the accumulators of its matrix instructions until it has no more samples.  Nothing of a
// sample goes to memory but what it predicts.  Workgroups' sums are added up by fit_sum_kernel, always in the same order.
#include "internal.h"
#include "philox.h"
#include "row_sums.h"
#include <math.h>

typedef float floatx16 __attribute__((ext_vector_type(16)));

namespace {

constexpr int FIT_ROWS = 64, FIT_CHUNK = 64;                // samples a workgroup takes at a time; features staged at a time
constexpr int FIT_COLUMNS_MAX = 512;                        // 2F, at most
constexpr int FIT_PASS_TILES = 8;                           // column tiles of G that one pass over the samples can keep

struct FitArgs {
    const float *X[2];
    int rows[2], F, columns, padded;                        // columns = 2F, padded to a multiple of 32
    const int32_t *index[2];
    const float *target[2];                                 // throughput, slowdown (null: not trained)
    float *sigma[2];                                        // (null: not wanted)
    long long count;
    const float *W1, *b1;                                   // folded, [H][padded] and [H]
    const float *W2, *b2, *W3[2], *b3[2], *W1sm;            // ([1] and W1sm may be null)
    int norm, sm_feature[2];
    float eps, scale;
    int drop;
    DropRule rule;
    const unsigned long long *step;
    float *partial;
    long long partial_step;
};

// What a workgroup leaves, one after the other.
template <int H>
struct FitSums {
    static constexpr int W2 = 0, B1 = H * H, B2 = B1 + H, W3 = B2 + H, W3S = W3 + H, SM = W3S + H, REST = SM + H, G = REST + 4;
};
enum { REST_B3 = 0, REST_B3S, REST_LOSS };

// Row r of a 32-row tile of matrix results lies in lane half (r >> 2) & 1; read as unit tile_unit(r), what a lane holds of
// a tile are the units 8 half .. 8 half + 7 and 16 + 8 half .. 16 + 8 half + 7: eight that share a counter.
__device__ __forceinline__ int tile_unit(int r) { return (r & 0x13) | (r & 4) << 1 | (r & 8) >> 1; }

__device__ __forceinline__ float other_half(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// max(v, 0) that keeps a NaN: a fit that has diverged shows.
__device__ __forceinline__ float relu(float v) { return v < 0.0f ? 0.0f : v; }

template <int H>
constexpr size_t fit_lds_bytes(bool grad)
{
    return sizeof(float) * ((size_t)H * (H + 4) + FIT_ROWS * (FIT_CHUNK + 4) + (size_t)FIT_ROWS * (H + 4) * (grad ? 2 : 1) +
                            2 * (H / 32) * FIT_ROWS + FIT_ROWS * 5 + 4 * FIT_ROWS + 5 * H);
}

template <int H, int GT, bool GRAD>
__global__ __launch_bounds__(H * 4) void fit_kernel(FitArgs a)
{
    constexpr int T = FIT_ROWS, PITCH = H + 4, XP = FIT_CHUNK + 4, UB = H / 32, THREADS = H * 4, QUADS = H / 8;
    using S = FitSums<H>;
    extern __shared__ __align__(16) float lds[];
    float *w2 = lds, *xs = w2 + H * PITCH, *act = xs + T * XP, *back = act + T * PITCH;
    float *part = back + (GRAD ? T * PITCH : 0), *target = part + 2 * UB * T, *target_slow = target + T, *share = target_slow + T;
    int *at_on = (int *)(share + T), *at_off = at_on + T;
    float2 *moments = (float2 *)(at_off + T);
    float *vec = (float *)(moments + 2 * T);                // b1, b2, W3, W3 of the slowdown unit, W1sm
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nn = lane & 31, hh = lane >> 5;
    const int ub = wave % UB, sh = wave / UB;               // units 32 ub .. and samples 32 sh .. of the forward pass are this wavefront's
    const int unit = 32 * ub + tile_unit(nn), mine = 32 * sh + nn, u0 = 32 * ub + 8 * hh;
    if (a.step) { const unsigned long long s = *a.step; a.rule.s0 = (unsigned)s; a.rule.s1 = (unsigned)(s >> 32); }

    for (int e = tid; e < H * H / 4; e += THREADS) *(float4 *)(w2 + e / (H / 4) * PITCH + e % (H / 4) * 4) = ((const float4 *)a.W2)[e];
    for (int e = tid; e < H; e += THREADS) {
        vec[e] = a.b1[e];
        vec[H + e] = a.b2[e];
        vec[2 * H + e] = a.W3[0][e];
        vec[3 * H + e] = a.W3[1] ? a.W3[1][e] : 0.0f;
        vec[4 * H + e] = a.W1sm ? a.W1sm[e] : 0.0f;
    }
    const float b3 = *a.b3[0], b3s = a.W3[1] ? *a.b3[1] : 0.0f;
    const float factor = a.drop ? a.rule.factor : 1.0f;
    const int chunks = (a.padded + FIT_CHUNK - 1) / FIT_CHUNK;
    const int pass_chunk = blockIdx.y * (FIT_PASS_TILES / 2);       // this pass keeps G from this chunk on

    floatx16 gw2[UB / 2], gw1[GT];
    float gb1[16], gb2[16], gw3[16], gw3s[16], gsm[16], gb3 = 0.0f, gb3s = 0.0f, loss = 0.0f;
    if (GRAD) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            gb1[e] = gb2[e] = gw3[e] = gw3s[e] = gsm[e] = 0.0f;
#pragma unroll
            for (int t = 0; t < UB / 2; ++t) gw2[t][e] = 0.0f;
#pragma unroll
            for (int t = 0; t < GT; ++t) gw1[t][e] = 0.0f;
        }
    }
    // features of columns 64 chunk .. 64 chunk + 63
    auto stage = [&](const int chunk) {
        for (int e = tid; e < T * FIT_CHUNK; e += THREADS) {
            const int s = e / FIT_CHUNK, c = chunk * FIT_CHUNK + e % FIT_CHUNK, side = c >= a.F;
            float v = 0.0f;
            if (c < a.columns && at_on[s] >= 0) {
                const float2 m = moments[2 * s + side];
                v = (a.X[side][(size_t)(side ? at_off[s] : at_on[s]) * a.F + c - (side ? a.F : 0)] - m.x) * m.y;
            }
            xs[s * XP + e % FIT_CHUNK] = v;
        }
    };
    // bias, ReLU and dropout of this lane's 16 units of one layer
    auto activate = [&](const floatx16 &z, float (&h)[16], const float *bias, const float share_here, long long sample, unsigned layer) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            Words4 bits;
            if (a.drop) bits = drop_bits(a.rule, (unsigned long long)sample * (H / 8) + (u0 + 16 * g) / 8, layer);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float v = z[8 * g + e] + bias[u0 + 16 * g + e];
                if (layer == 0 && a.W1sm) v = fmaf(share_here, vec[4 * H + u0 + 16 * g + e], v);
                v = relu(v);
                if (a.drop) v = drop_keeps(a.rule, bits, e) ? v * factor : 0.0f;
                h[8 * g + e] = v;
            }
        }
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
            share[tid] = i >= 0 && a.W1sm ? fminf(1.0f - a.X[0][(size_t)i * a.F + a.sm_feature[0]], a.X[1][(size_t)j * a.F + a.sm_feature[1]]) : 0.0f;
        }
        __syncthreads();
        {   // moments of the samples' feature rows, 2 T of them, by THREADS / (2 T) neighbouring lanes each
            constexpr int EACH = THREADS / (2 * T);
            const int r = tid / EACH, sub = tid % EACH, side = r & 1;
            const int at = side ? at_off[r >> 1] : at_on[r >> 1];
            float2 m = make_float2(0.0f, 1.0f);
            if (a.norm && at >= 0) {                        // (the lanes of a row agree)
                const float *x = a.X[side] + (size_t)at * a.F;
                float sum = 0.0f, squares = 0.0f;
                for (int f = sub; f < a.F; f += EACH) sum += x[f];
                m.x = group_sum<EACH>(sum) / (float)a.F;
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
            stage(c);
            __syncthreads();
            const int quads = (a.padded - c * FIT_CHUNK < FIT_CHUNK ? a.padded - c * FIT_CHUNK : FIT_CHUNK) / 8;
            for (int q = 0; q < quads; ++q) {
                const float4 w = *(const float4 *)(a.W1 + (size_t)unit * a.padded + c * FIT_CHUNK + 8 * q + 4 * hh);
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
        zp = other_half(zp);
        zs = other_half(zs);
        if (hh == 0) { part[ub * T + mine] = zp; part[(UB + ub) * T + mine] = zs; }
        __syncthreads();
        zp = b3; zs = b3s;
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
        const float dz = t0 == t0 ? 2.0f * a.scale * miss * y * (1.0f - y) : 0.0f;
        const float dzs = t1 == t1 ? 2.0f * a.scale * miss_slow * ys * (1.0f - ys) : 0.0f;
        if (speaks) { gb3 += dz; gb3s += dzs; }
        float d[16];
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = 8 * g + e;
                float v = dz * vec[2 * H + u0 + 16 * g + e];
                gw3[k] = fmaf(dz, h2[k], gw3[k]);
                if (a.W3[1]) {
                    v = fmaf(dzs, vec[3 * H + u0 + 16 * g + e], v);
                    gw3s[k] = fmaf(dzs, h2[k], gw3s[k]);
                }
                d[k] = h2[k] > 0.0f ? v * factor : 0.0f;
                gb2[k] += d[k];
            }
        put(back, d);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = 0.0f;
        for (int q = 0; q < QUADS; ++q) {                   // W2^T dz2
            const float *w = w2 + (8 * q + 4 * hh) * PITCH + unit;
            const float4 x = *(const float4 *)(back + mine * PITCH + 8 * q + 4 * hh);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w[0], x.x, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w[PITCH], x.y, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w[2 * PITCH], x.z, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(w[3 * PITCH], x.w, z, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            d[k] = h1[k] > 0.0f ? z[k] * factor : 0.0f;
            gb1[k] += d[k];
            if (a.W1sm) gsm[k] = fmaf(share[mine], d[k], gsm[k]);
        }
        // sums over samples: the lower half of a wavefront takes sample 16 b + i, the upper one 16 b + 8 + i
        for (int b = 0; b < T / 16; ++b)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int s = (16 * b + i + 8 * hh) * PITCH;
                const float v = back[s + 32 * ub + nn];
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
                stage(c);
                __syncthreads();
            }
            if (c * FIT_CHUNK + 32 * sh >= a.padded) continue;      // (the last chunk may be half as wide)
            for (int b = 0; b < T / 16; ++b)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int s = 16 * b + i + 8 * hh;
                    gw1[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(act[s * PITCH + 32 * ub + nn], xs[s * XP + 32 * sh + nn], gw1[t], 0, 0, 0);
                }
        }
    }

    // what this workgroup leaves
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
        // sums of a unit over the lanes that hold it, then over the two wavefronts that do
        float *sums = act;                                  // [5][2][H]
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const float v[5] = {group_sum<32>(gb1[k]), group_sum<32>(gb2[k]), group_sum<32>(gw3[k]), group_sum<32>(gw3s[k]), group_sum<32>(gsm[k])};
#pragma unroll
            for (int q = 0; q < 5; ++q)
                if (nn == 0) sums[(2 * q + sh) * H + u0 + (k >> 3) * 16 + (k & 7)] = v[q];
        }
        __syncthreads();
        for (int e = tid; e < 5 * H; e += THREADS) out[S::B1 + e] = sums[(2 * (e / H)) * H + e % H] + sums[(2 * (e / H) + 1) * H + e % H];
        __syncthreads();
    }
    if (a.partial) {
        const float v[3] = {group_sum<64>(gb3), group_sum<64>(gb3s), group_sum<64>(loss)};
        if (lane == 0 && ub == 0)
#pragma unroll
            for (int q = 0; q < 3; ++q) part[3 * sh + q] = v[q];
        __syncthreads();
        if (tid < 3) out[S::REST + tid] = part[tid] + part[3 + tid];
    }
}

// Layer 1 with the norm's weight and bias folded in, its rows padded with zeros: a wavefront for each hidden unit.
__global__ __launch_bounds__(64) void fold_kernel(const float *W1, const float *b1, const float *g, const float *beta, int columns, int padded, float *W, float *b)
{
    const int k = blockIdx.x;
    float sum = 0.0f;
    for (int c = threadIdx.x; c < padded; c += 64) {
        float v = 0.0f;
        if (c < columns) {
            v = W1[(size_t)k * columns + c];
            if (g) { sum = fmaf(v, beta[c], sum); v *= g[c]; }
        }
        W[(size_t)k * padded + c] = v;
    }
    sum = group_sum<64>(sum);
    if (threadIdx.x == 0) b[k] = b1[k] + sum;
}

// Sums of what the workgroups left: value v goes where it belongs.
struct FitOut {
    float *W1, *b1, *W2, *b2, *W3, *b3, *W3s, *b3s, *W1sm, *loss, *G;
    int H, columns, padded, norm, parts;
    float scale;
};
constexpr int FIT_SUM_VALUES = 64, FIT_SUM_SLICES = 16;

__global__ __launch_bounds__(FIT_SUM_VALUES * FIT_SUM_SLICES) void fit_sum_kernel(const float *__restrict__ partial, long long step, int first, int values, FitOut o)
{
    __shared__ float sums[FIT_SUM_SLICES][FIT_SUM_VALUES];
    const int place = threadIdx.x % FIT_SUM_VALUES, slice = threadIdx.x / FIT_SUM_VALUES;
    const int v = first + blockIdx.x * FIT_SUM_VALUES + place;
    float s = 0.0f;
    if (v < values)
        for (int p = slice; p < o.parts; p += FIT_SUM_SLICES) s += partial[p * step + v];
    sums[slice][place] = s;
    __syncthreads();
    if (slice > 0 || v >= values) return;
    for (int k = 1; k < FIT_SUM_SLICES; ++k) s += sums[k][place];
    const int H = o.H;
    int at = v;
    if (at < H * H) { o.W2[at] = s; return; }
    at -= H * H;
    if (at < 5 * H) {
        float *const to[5] = {o.b1, o.b2, o.W3, o.W3s, o.W1sm};
        if (to[at / H]) to[at / H][at % H] = s;
        return;
    }
    at -= 5 * H;
    if (at < 4) {
        if (at == REST_B3 && o.b3) *o.b3 = s;
        if (at == REST_B3S && o.b3s) *o.b3s = s;
        if (at == REST_LOSS && o.loss) *o.loss = s * o.scale;
        return;
    }
    at -= 4;
    const int k = at / o.padded, c = at % o.padded;
    if (o.norm) o.G[at] = s;
    else if (c < o.columns) o.W1[(size_t)k * o.columns + c] = s;
}

// dW1 = G diag g + h beta^T, dg_f = sum_k W1[k, f] G[k, f], dbeta = W1^T h.
constexpr int UNFOLD_SLICES = 16;

__global__ __launch_bounds__(64 * UNFOLD_SLICES) void unfold_kernel(const float *W1, const float *G, const float *h, const float *g, const float *beta, int H,
                                                                    int columns, int padded, float *dW1, float *dg, float *dbeta)
{
    __shared__ float sums[2][UNFOLD_SLICES][64];
    const int lane = threadIdx.x % 64, slice = threadIdx.x / 64, c = blockIdx.x * 64 + lane;
    float weight = 0.0f, bias = 0.0f;
    if (c < columns)
        for (int k = slice; k < H; k += UNFOLD_SLICES) {
            const float G1 = G[(size_t)k * padded + c], W = W1[(size_t)k * columns + c];
            dW1[(size_t)k * columns + c] = fmaf(G1, g[c], h[k] * beta[c]);
            weight = fmaf(W, G1, weight);
            bias = fmaf(W, h[k], bias);
        }
    sums[0][slice][lane] = weight;
    sums[1][slice][lane] = bias;
    __syncthreads();
    if (slice > 0 || c >= columns) return;
    for (int k = 1; k < UNFOLD_SLICES; ++k) { weight += sums[0][k][lane]; bias += sums[1][k][lane]; }
    dg[c] = weight;
    dbeta[c] = bias;
}

// Nothing to learn from: no samples.
__global__ void clear_kernel(float *p, int count)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < count) p[i] = 0.0f;
}

struct FitPlan {
    int H, columns, padded, passes, tiles_each, grid;
    int values(bool grad) const { return (H == 64 ? FitSums<64>::G : FitSums<128>::G) + (grad ? H * padded : 0); }
    long long step(bool grad) const { return (values(grad) + 15) & ~15; }
};

FitPlan fit_plan(const mf_ctx *ctx, const mf_predictor *p, long long count)
{
    FitPlan f{};
    f.H = p->H;
    f.columns = 2 * p->F;
    f.padded = (f.columns + 31) & ~31;
    const int chunks = (f.padded + FIT_CHUNK - 1) / FIT_CHUNK, most = FIT_PASS_TILES / 2;
    f.passes = (chunks + most - 1) / most;
    f.tiles_each = chunks == 1 ? 1 : chunks == 2 ? 2 : most;
    const long long tiles = (count + FIT_ROWS - 1) / FIT_ROWS;
    const long long units = (ctx->n_cus > 0 ? ctx->n_cus : 256) * (p->H == 64 ? 2 : 1);
    f.grid = (int)(tiles < units ? tiles : units);
    return f;
}

template <int H, int GT, bool GRAD>
int launch_fit(mf_ctx *ctx, const FitArgs &a, const FitPlan &f)
{
    const unsigned flag = 1u << (21 + (H == 128 ? 4 : 0) + (GRAD ? GT / 2 + 1 : 0));
    if (!(ctx->kernels_configured & flag)) {
        MF_HIP(hipFuncSetAttribute((const void *)fit_kernel<H, GT, GRAD>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)fit_lds_bytes<H>(GRAD)));
        ctx->kernels_configured |= flag;
    }
    hipLaunchKernelGGL((fit_kernel<H, GT, GRAD>), dim3(f.grid, GRAD ? f.passes : 1), dim3(H * 4), fit_lds_bytes<H>(GRAD), ctx->stream, a);
    MF_HIP(hipGetLastError());
    return MF_OK;
}

template <int H>
int launch_fit_for(mf_ctx *ctx, const FitArgs &a, const FitPlan &f, bool grad)
{
    if (!grad) return launch_fit<H, 1, false>(ctx, a, f);
    if (f.tiles_each == 1) return launch_fit<H, 1, true>(ctx, a, f);
    if (f.tiles_each == 2) return launch_fit<H, 2, true>(ctx, a, f);
    return launch_fit<H, 4, true>(ctx, a, f);
}

bool whole_floats(const void *p) { return ((uintptr_t)p & 3u) == 0; }

// Launches the forward pass over the samples, with gradients where there are any to be written.
int run_fit(mf_ctx *ctx, const mf_predictor *p, const float *d_on, int n, const float *d_off, int m, const mf_samples *s,
            const DropRule *rule, const uint64_t *d_step, float scale, const mf_gradients *g, float *d_loss, float *d_sigma, float *d_sigma_slow, void *d_work)
{
    const FitPlan f = fit_plan(ctx, p, s->count);
    FitArgs a{};
    a.X[0] = d_on; a.X[1] = d_off;
    a.rows[0] = n; a.rows[1] = m;
    a.F = p->F; a.columns = f.columns; a.padded = f.padded;
    a.index[0] = s->d_on; a.index[1] = s->d_off;
    a.target[0] = s->d_target; a.target[1] = s->d_target_slow;
    a.sigma[0] = d_sigma; a.sigma[1] = d_sigma_slow;
    a.count = s->count;
    a.W1 = ctx->fit_W1; a.b1 = ctx->fit_W1 + 128 * FIT_COLUMNS_MAX;
    a.W2 = p->d_W2; a.b2 = p->d_b2;
    a.W3[0] = p->d_W3; a.W3[1] = p->d_W3_slow;
    a.b3[0] = p->d_b3; a.b3[1] = p->d_b3_slow;
    a.W1sm = p->d_W1sm;
    a.norm = p->d_ln_w != nullptr; a.eps = p->ln_eps;
    a.sm_feature[0] = p->sm_on_feature; a.sm_feature[1] = p->sm_off_feature;
    a.scale = scale;
    a.drop = rule && rule->limit > 0;
    if (a.drop) { a.rule = *rule; a.step = (const unsigned long long *)d_step; }
    a.partial = (float *)d_work;
    a.partial_step = f.step(g != nullptr);
    hipLaunchKernelGGL(fold_kernel, dim3(f.H), dim3(64), 0, ctx->stream, p->d_W1, p->d_b1, p->d_ln_w, p->d_ln_b, f.columns, f.padded, ctx->fit_W1, ctx->fit_W1 + 128 * FIT_COLUMNS_MAX);
    MF_HIP(hipGetLastError());
    const int rc = f.H == 64 ? launch_fit_for<64>(ctx, a, f, g != nullptr) : launch_fit_for<128>(ctx, a, f, g != nullptr);
    if (rc != MF_OK || !a.partial) return rc;
    FitOut o{};
    if (g) {
        o.W1 = g->d_W1; o.b1 = g->d_b1; o.W2 = g->d_W2; o.b2 = g->d_b2; o.W3 = g->d_W3; o.b3 = g->d_b3;
        o.W3s = p->d_W3_slow ? g->d_W3_slow : nullptr; o.b3s = p->d_W3_slow ? g->d_b3_slow : nullptr;
        o.W1sm = p->d_W1sm ? g->d_W1sm : nullptr;
    }
    o.loss = d_loss;
    o.G = a.partial + (size_t)f.grid * a.partial_step;
    o.H = f.H; o.columns = f.columns; o.padded = f.padded; o.norm = a.norm; o.parts = f.grid; o.scale = scale;
    const int values = f.values(g != nullptr), first = g ? 0 : values - 4;
    hipLaunchKernelGGL(fit_sum_kernel, dim3((values - first + FIT_SUM_VALUES - 1) / FIT_SUM_VALUES), dim3(FIT_SUM_VALUES * FIT_SUM_SLICES), 0, ctx->stream,
                       a.partial, a.partial_step, first, values, o);
    if (g && a.norm)
        hipLaunchKernelGGL(unfold_kernel, dim3((f.columns + 63) / 64), dim3(64 * UNFOLD_SLICES), 0, ctx->stream, p->d_W1, o.G, g->d_b1, p->d_ln_w, p->d_ln_b,
                           f.H, f.columns, f.padded, g->d_W1, g->d_ln_w, g->d_ln_b);
    MF_HIP(hipGetLastError());
    return MF_OK;
}

int check_samples(const mf_ctx *ctx, const mf_predictor *p, const float *d_on, int n, const float *d_off, int m, const mf_samples *s)
{
    if (!ctx || !s || n < 0 || m < 0 || s->count < 0) return MF_ERR_ARG;
    const int rc = mf_check_predictor(p);
    if (rc != MF_OK) return rc;
    if (n > MF_MAX_DIM || m > MF_MAX_DIM || s->count > (1ll << 31) - 64) return MF_ERR_SHAPE;
    if ((n > 0 && !d_on) || (m > 0 && !d_off) || (s->count > 0 && (!s->d_on || !s->d_off))) return MF_ERR_ARG;
    for (const void *q : {(const void *)d_on, (const void *)d_off, (const void *)s->d_on, (const void *)s->d_off, (const void *)s->d_target, (const void *)s->d_target_slow})
        if (!whole_floats(q)) return MF_ERR_ARG;
    return MF_OK;
}

}  // namespace

extern "C" {

int64_t mf_predictor_loss_work(mf_ctx *ctx, const mf_predictor *pred, int64_t count)
{
    if (!ctx || count < 0) return MF_ERR_ARG;
    const int rc = mf_check_predictor(pred);
    if (rc != MF_OK) return rc;
    if (count > (1ll << 31) - 64) return MF_ERR_SHAPE;
    const FitPlan f = fit_plan(ctx, pred, count);
    return (int64_t)sizeof(float) * (f.grid * f.step(true) + f.H * f.padded);
}

int mf_predictor_loss(mf_ctx *ctx, const mf_predictor *pred, const float *d_on, int n, const float *d_off, int m,
                      const mf_samples *samples, const mf_dropout_rule *dropout, float scale,
                      const mf_gradients *grads, float *d_loss, float *d_sigma, float *d_sigma_slow,
                      void *d_work, int64_t work_bytes)
{
    const int rc = check_samples(ctx, pred, d_on, n, d_off, m, samples);
    if (rc != MF_OK) return rc;
    DropRule rule;
    if (!d_loss || !whole_floats(d_loss) || !whole_floats(d_sigma) || !whole_floats(d_sigma_slow)) return MF_ERR_ARG;
    if (!(scale > 0.0f) || isinf(scale) || (dropout && !mf_drop_rule(dropout, &rule))) return MF_ERR_ARG;
    if (samples->count > 0 && (!samples->d_target || (pred->d_W3_slow != nullptr) != (samples->d_target_slow != nullptr))) return MF_ERR_ARG;
    if (d_sigma_slow && !pred->d_W3_slow) return MF_ERR_ARG;
    if (grads) {
        const mf_gradients &g = *grads;
        if (!g.d_W1 || !g.d_b1 || !g.d_W2 || !g.d_b2 || !g.d_W3 || !g.d_b3 || (pred->d_W1sm && !g.d_W1sm) ||
            (pred->d_W3_slow && (!g.d_W3_slow || !g.d_b3_slow)) || (pred->d_ln_w && (!g.d_ln_w || !g.d_ln_b)))
            return MF_ERR_ARG;
        for (const float *q : {g.d_W1, g.d_b1, g.d_W2, g.d_b2, g.d_W3, g.d_b3, g.d_W1sm, g.d_W3_slow, g.d_b3_slow, g.d_ln_w, g.d_ln_b})
            if (!whole_floats(q)) return MF_ERR_ARG;
    }
    if (samples->count > 0 && (!d_work || ((uintptr_t)d_work & 15u) || work_bytes < mf_predictor_loss_work(ctx, pred, samples->count))) return MF_ERR_ARG;
    MF_HIP(hipSetDevice(ctx->device));
    if (samples->count == 0) {
        const auto clear = [&](float *p, int count) { if (p) hipLaunchKernelGGL(clear_kernel, dim3((count + 255) / 256), dim3(256), 0, ctx->stream, p, count); };
        const int H = pred->H, F = pred->F;
        clear(d_loss, 1);
        if (grads) {
            clear(grads->d_W1, 2 * F * H); clear(grads->d_b1, H); clear(grads->d_W2, H * H); clear(grads->d_b2, H); clear(grads->d_W3, H); clear(grads->d_b3, 1);
            if (pred->d_W1sm) clear(grads->d_W1sm, H);
            if (pred->d_W3_slow) { clear(grads->d_W3_slow, H); clear(grads->d_b3_slow, 1); }
            if (pred->d_ln_w) { clear(grads->d_ln_w, 2 * F); clear(grads->d_ln_b, 2 * F); }
        }
        MF_HIP(hipGetLastError());
        return MF_OK;
    }
    return run_fit(ctx, pred, d_on, n, d_off, m, samples, dropout ? &rule : nullptr, dropout ? dropout->d_step : nullptr, scale, grads, d_loss, d_sigma,
                   d_sigma_slow, d_work);
}

int mf_predict_pairs(mf_ctx *ctx, const mf_predictor *pred, const float *d_on, int n, const float *d_off, int m,
                     const int32_t *d_pair_on, const int32_t *d_pair_off, int64_t count, float *d_sigma, float *d_sigma_slow)
{
    const mf_samples s{d_pair_on, d_pair_off, nullptr, nullptr, count};
    const int rc = check_samples(ctx, pred, d_on, n, d_off, m, &s);
    if (rc != MF_OK) return rc;
    if (d_sigma_slow && (!pred->d_W3_slow || !whole_floats(d_sigma_slow))) return MF_ERR_ARG;
    if (count == 0) return MF_OK;
    if (!d_sigma || !whole_floats(d_sigma)) return MF_ERR_ARG;
    MF_HIP(hipSetDevice(ctx->device));
    return run_fit(ctx, pred, d_on, n, d_off, m, &s, nullptr, nullptr, 1.0f, nullptr, nullptr, d_sigma, d_sigma_slow, nullptr);
}

}  // extern "C"
