// Fitting a speed predictor: its loss over listed pairs with every gradient, and its predictions for listed pairs (paper:
// Section "Implementation", the predictor is trained on profiled pairs).
//
// For a sample s = (i, j, t), with u the features of both workloads, normalised where the predictor has a layer norm:
//     x = g u + beta,  z1 = W1 x + b1 (+ share W1sm),  d1 = drop(relu(z1)),  z2 = W2 d1 + b2,  d2 = drop(relu(z2)),
//     y = logistic(W3 d2 + b3),  loss = scale sum (y - t)^2  (and the same of the slowdown unit),
//     dz3 = 2 (y - t) y (1 - y),  dz2 = [d2 > 0] c W3 dz3,  dz1 = [d1 > 0] c W2^T dz2,
//     dW2 = sum dz2 d1^T,  G = sum dz1 u^T,  h = sum dz1, and all of that times scale at the end.
// The norm's weight and bias fold into layer 1, and their gradients come out of sums that layer 1's needs anyway:
//     W1 x + b1 = (W1 diag g) u + (b1 + W1 beta),  dW1 = G diag g + h beta^T,  dg_f = sum_k W1[k,f] G[k,f],  dbeta = W1^T h,
// so a sample costs no more than without it.  Nothing of a sample goes to memory but what it predicts.
//
// Matrix products.  A float32 operand goes to the fp16 matrix pipe as two fp16 pieces, v = hi + lo with either rounded to nearest
// (|v - hi - lo| <= 2^-22 |v|), and a product is hi hi + hi lo + lo hi, added up in float32: three fp16 products at sixteen times
// the rate of the float32 ones (2300 and 152 TFLOP/s measured).  fp16's range is seen to by scaling each operand with a power of two
// from a bound on it that is never exceeded, to below 2^14; what is within 2^-17 of the bound keeps all its 22 bits, smaller
// values lose absolute precision of 2^-39 of the bound.  The bounds: a normalised row has |u|_2 <= sqrt(F), so |z1_k| <= |W1_k|_2
// sqrt(2F) + |b1_k|; |dz3| <= (1 + max |t|) / 2; and through W3 and W2 by their largest values and columns' sums.  Rows of weights have a scale
// each, of their own largest value.
//
// A workgroup takes FIT_ROWS samples at a time.  Half of its wavefronts ("forward", 32 hidden units each) take them through the layers and back;
// activations pass between them through LDS.  The others ("sums") add up the gradients of weights, in accumulators that stay until there are no
// more samples, and get the next samples ready: features, their norm, random bits.  A SIMD has one wavefront of either kind, so that the matrix
// instructions of one run beside the arithmetic of the other:
//     forward   layer 1 -> d1      layer 2 -> output      loss, dz2           W2^T dz2 -> dz1
//     sums      G of the last      next features          next random bits    dW2
//
// NaN: a ReLU that is one instruction turns it into 0, so what is not finite among the weights, or a sample's features, is added to the output as a NaN.
#include "fit_parts.h"

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));

namespace {

constexpr int FIT_ROWS = 32;

// The largest power of two that takes a value of at most `bound` to below 2^14 (1 for bounds that are none).
__device__ __forceinline__ float scale_below(float bound)
{
    if (!(bound > 0.0f) || bound > 1e30f) return 1.0f;
    int e;
    (void)frexpf(bound, &e);                                // bound < 2^e
    e = e < -96 ? -96 : e > 96 ? 96 : e;
    return ldexpf(1.0f, 14 - e);
}

// v = hi + lo in fp16, to 22 bits.  The remainder is exact; written as a fused multiply-add by a -1 that the optimiser cannot see it is one
// instruction that reads the fp16 piece itself.
template <int N>
__device__ __forceinline__ void split(const float (&v)[N], _Float16 (&hi)[N], _Float16 (&lo)[N], const float minus_one)
{
#pragma unroll
    for (int t = 0; t < N; t += 2) {
        const float2v x = {v[t], v[t + 1]};
        const half2v h = __builtin_convertvector(x, half2v);
        const float2v r = {__builtin_fmaf((float)h[0], minus_one, v[t]), __builtin_fmaf((float)h[1], minus_one, v[t + 1])};
        const half2v l = __builtin_convertvector(r, half2v);
        hi[t] = h[0]; hi[t + 1] = h[1];
        lo[t] = l[0]; lo[t + 1] = l[1];
    }
}
__device__ __forceinline__ float hidden_minus_one()
{
    float v = -1.0f;
    asm volatile("" : "+s"(v));                             // no instruction
    return v;
}

struct Frag { half8v hi, lo; };

__device__ __forceinline__ floatx16 product(const Frag &a, const Frag &b, floatx16 c)
{
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.hi, b.hi, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.hi, b.lo, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a.lo, b.hi, c, 0, 0, 0);
}

// Eight values of a matrix kept in rows [sample][column], for sums over samples: lane l gets column `first` + l % 32 of samples
// 8 (l / 32) .. + 7.  The transposing read gives a group of sixteen lanes four rows of sixteen columns, a column to each lane.
__device__ __forceinline__ half8v read_columns(const _Float16 *m, int pitch, int first, int lane)
{
    const int group = lane >> 4, i = lane & 15;
    const _Float16 *p = m + (8 * (group >> 1) + (i >> 2)) * pitch + first + 16 * (group & 1) + 4 * (i & 3);
    const auto read = [](const _Float16 *q) {
        return __builtin_bit_cast(half4v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v *)q));
    };
    const half4v a = read(p), b = read(p + 4 * pitch);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}

// Waits for what this wavefront has put into or read from LDS, and for the other wavefronts to have come here, but not for loads and stores of
// global memory on their way: features are fetched a stage before they are looked at.
__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Everything of a workgroup's that wavefronts share.  Rows of pieces are 16 halves longer than what they hold: eight words, so that
// eight rows next to each other lie in different banks.
template <int H, int CT, bool GRAD>
struct FitShared {
    static constexpr int T = FIT_ROWS, UB = H / 32, KB = H / 16, HP = H + 16, XP = 32 * CT + 16;
    half8v w2t[GRAD ? UB : 1][GRAD ? KB : 1][2][64];        // W2^T as operands: [units of layer 1][of layer 2][piece][lane]
    _Float16 d1[2][T][HP];                                  // [piece]
    _Float16 xs[2][2][T][XP];                               // [of which samples][piece]
    _Float16 dz2[GRAD ? 2 : 1][GRAD ? T : 1][HP], dz1[GRAD ? 2 : 1][GRAD ? T : 1][HP];
    float part[2][UB][T];                                   // output units: partial sums over 32 hidden units
    float target[2][2][T], share[2][T], bad[2][2][T];       // bad: NaN where features are not finite
    int real[2][T];
    unsigned char keep[2][T][H / 8];                        // [layer]: which of eight units stay
    float b1[H], wsm[H], b2[H], w3[2][H];                   // by unit; b1, wsm and b2 with the scale and the dropout's factor of their layer
    float most[5][2 * UB];
};

// Layer 1 with the norm's weight and bias folded in, for the forward wavefronts' operands (or, wide, as rows of floats), with what its
// bounds are made of; the last FIT_RANGE_PARTS workgroups find the largest target and, where nothing else bounds them, feature.
struct FoldArgs {
    const float *W1, *b1, *g, *beta;
    int H, F, padded, half, wide;
    void *image;                                            // wide: [H][padded] floats; else fragments of pieces
    float *bias, *norm1, *norm2, *scale;                    // [H]; [1]
    float *ranges;                                          // [2][FIT_RANGE_PARTS]: targets, features
    const float *target[2], *X[2];
    const int32_t *index[2];
    int rows[2], features;                                  // features: 0 not wanted, 1 of all workloads, 2 of those the samples name
    long long count;
};

__global__ __launch_bounds__(256) void fold_kernel(FoldArgs a)
{
    const int lane = threadIdx.x & 63, rows = a.H / 4;
    if ((int)blockIdx.x >= rows) {
        __shared__ float most[2][4];
        const int part = blockIdx.x - rows;
        const long long first = (long long)part * 256 + threadIdx.x, step = FIT_RANGE_PARTS * 256;
        float t = 0.0f, x = 0.0f;
        for (int k = 0; k < 2; ++k)
            if (a.target[k])
                for (long long s = first; s < a.count; s += step) { const float v = fabsf(a.target[k][s]); if (v < INFINITY) t = fmaxf(t, v); }
        for (int k = 0; k < 2; ++k) {
            if (a.features == 1)
                for (long long e = first; e < (long long)a.rows[k] * a.F; e += step) { const float v = fabsf(a.X[k][e]); if (v < INFINITY) x = fmaxf(x, v); }
            if (a.features == 2)
                for (long long s = first; s < a.count; s += step) {
                    const int i = a.index[k][s];
                    if (i < 0 || i >= a.rows[k]) continue;
                    for (int f = 0; f < a.F; ++f) { const float v = fabsf(a.X[k][(size_t)i * a.F + f]); if (v < INFINITY) x = fmaxf(x, v); }
                }
        }
        t = wave_max(t);
        x = wave_max(x);
        if (lane == 0) { most[0][threadIdx.x >> 6] = t; most[1][threadIdx.x >> 6] = x; }
        __syncthreads();
        if (threadIdx.x < 2) a.ranges[threadIdx.x * FIT_RANGE_PARTS + part] = fmaxf(fmaxf(most[threadIdx.x][0], most[threadIdx.x][1]), fmaxf(most[threadIdx.x][2], most[threadIdx.x][3]));
        return;
    }
    const auto folded = [&](const int k, const int c, float *times_beta) {
        const int side = c >= a.half, f = c - side * a.half;
        if (f >= a.F) return 0.0f;
        const int at = side * a.F + f;
        const float w = a.W1[(size_t)k * 2 * a.F + at];
        if (times_beta) *times_beta = a.g ? w * a.beta[at] : 0.0f;
        return a.g ? w * a.g[at] : w;
    };
    const int k = blockIdx.x * 4 + (threadIdx.x >> 6);
    float sum = 0.0f, norm1 = 0.0f, norm2 = 0.0f;
    for (int c = lane; c < a.padded; c += 64) {
        float more = 0.0f;
        const float v = folded(k, c, &more);
        sum += more;
        norm1 += fabsf(v);
        norm2 = fmaf(v, v, norm2);
        if (a.wide) ((float *)a.image)[(size_t)k * a.padded + c] = v;
    }
    sum = group_sum<64>(sum);
    norm1 = group_sum<64>(norm1);
    norm2 = group_sum<64>(norm2);
    if (lane == 0) {
        a.bias[k] = a.b1[k] + sum;
        a.norm1[k] = norm1;
        a.norm2[k] = sqrtf(norm2);
    }
    if (a.wide) return;
    // (every workgroup looks for the largest weight itself: no more than 48 KB, and no launch between)
    __shared__ float most[4];
    float largest = 0.0f;
#pragma unroll 8
    for (int e = threadIdx.x; e < a.H * 2 * a.F; e += 256) largest = fmaxf(largest, fabsf(a.g ? a.W1[e] * a.g[e % (2 * a.F)] : a.W1[e]));
    largest = wave_max(largest);
    if (lane == 0) most[threadIdx.x >> 6] = largest;
    __syncthreads();
    const float scale = scale_below(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])));
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.scale = scale;
    const int blocks = a.padded / 16, m = tile_unit(k & 31);
    for (int c = lane; c < a.padded; c += 64) {
        const float v[2] = {folded(k, c, nullptr) * scale, 0.0f};
        _Float16 hi[2], lo[2];
        split(v, hi, lo, -1.0f);
        _Float16 *to = (_Float16 *)a.image + ((size_t)((k >> 5) * blocks + (c >> 4)) * 2 * 64 + ((c >> 3) & 1) * 32 + m) * 8 + (c & 7);
        to[0] = hi[0];
        to[64 * 8] = lo[0];
    }
}

// EXTRA: the predictor has the slowdown unit or the SM share (or both).
template <int H, int CT, bool GRAD, bool EXTRA>
__global__ __launch_bounds__(H * 4, 2) void fit_kernel(FitArgs a, const float *__restrict__ scale1, const float *__restrict__ norm1, const float *__restrict__ norm2,
                                                       const float *__restrict__ ranges)
{
    using L = FitShared<H, CT, GRAD>;
    using S = FitSums<H>;
    constexpr int T = FIT_ROWS, UB = H / 32, KB = H / 16, XB = 2 * CT, HALF = 16 * CT, HP = L::HP, XP = L::XP;
    extern __shared__ __align__(16) char lds[];
    L &sh = *(L *)lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), nn = lane & 31, hh = lane >> 5;
    const float minus_one = hidden_minus_one();
    if (a.step) { const unsigned long long s = *a.step; a.rule.s0 = (unsigned)s; a.rule.s1 = (unsigned)(s >> 32); }
    const bool slow = EXTRA && a.W3[1], with_share = EXTRA && a.W1sm;
    const float factor = a.drop ? a.rule.factor : 1.0f;
    const long long tiles = (a.count + T - 1) / T;
    const int mine = (int)((tiles - blockIdx.x + gridDim.x - 1) / gridDim.x);
    const auto tile_of = [&](const int it) { return (long long)blockIdx.x + (long long)it * gridDim.x; };
    const bool forward = wave < UB;
    const int ub = forward ? wave : wave - UB, unit = 32 * ub + tile_unit(nn), u0 = 32 * ub + 8 * hh;

    // ---- bounds, and the scales that follow.  W2 and its transpose are read as the operands that the forward wavefronts make of them.
    float w[KB][8], largest = 0.0f, column = 0.0f, poison = 0.0f;
    if (forward) {
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[b][e] = a.W2[(16 * b + 8 * hh + e) * H + unit];
                largest = fmaxf(largest, fabsf(w[b][e]));
                column += fabsf(w[b][e]);
            }
        column = both_halves(column);
        poison = column * 0.0f;                             // NaN if one of them is not finite
    }
    // largest of: targets, features, output weights of either unit, W2 and its columns' sums, z1
    float v[6] = {0.0f, 0.0f, 0.0f, 0.0f, largest, column};
    if (tid < FIT_RANGE_PARTS) { v[0] = ranges[tid]; v[1] = ranges[FIT_RANGE_PARTS + tid]; }
    if (tid < H) {
        v[2] = fabsf(a.W3[0][tid]);
        v[3] = slow ? fabsf(a.W3[1][tid]) : 0.0f;
        poison += (norm1[tid] + a.b1[tid] + a.b2[tid] + (with_share ? a.W1sm[tid] : 0.0f)) * 0.0f;
    }
    const auto most_of = [&](float (&v)[6]) {
#pragma unroll
        for (int q = 0; q < 6; ++q) v[q] = wave_max(v[q]);
        for (int q = 0; q < 6; q += 5) {                    // five at a time
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 5; ++k) if (q + k < 6 && lane == 0) sh.most[k][wave] = v[q + k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 5; ++k)
                if (q + k < 6)
                    for (int x = 0; x < 2 * UB; ++x) v[q + k] = fmaxf(v[q + k], sh.most[k][x]);
        }
    };
    most_of(v);
    const float most_x = v[1], length = sqrtf((float)a.F);
    const float s_x = scale_below(a.norm ? length * 1.001f : most_x), s_w2 = scale_below(v[4]);
    const float bound2 = 0.5f * (1.0f + v[0]) * (v[2] + v[3]) * factor * 1.001f;
    const float s_dz2 = scale_below(bound2), s_dz1 = scale_below(bound2 * factor * v[5] * 1.001f);
    float z1 = 0.0f;
    if (tid < H) {
        z1 = fabsf(a.b1[tid]) + (a.norm ? norm2[tid] * length * 1.42f : norm1[tid] * most_x);
        if (with_share) z1 += fabsf(a.W1sm[tid]) * (1.0f + most_x);
    }
    z1 = wave_max(z1);
    poison = group_sum<64>(poison);
    __syncthreads();
    if (lane == 0) { sh.most[0][wave] = z1; sh.most[1][wave] = poison; }
    __syncthreads();
    poison = 0.0f;
    for (int x = 0; x < 2 * UB; ++x) { z1 = fmaxf(z1, sh.most[0][x]); poison += sh.most[1][x]; }
    const float s_d1 = scale_below(z1 * factor * 1.001f);
    // what accumulators of the three products are multiplied with
    const float by_z1 = factor * s_d1 / (s_x * *scale1), by_z2 = factor / (s_d1 * s_w2), by_d1 = factor * s_dz1 / (s_dz2 * s_w2), by_dz = factor * s_dz2;
    if (tid < H) {
        sh.b1[tid] = a.b1[tid] * (factor * s_d1);
        sh.wsm[tid] = with_share ? a.W1sm[tid] * (factor * s_d1) : 0.0f;
        sh.b2[tid] = a.b2[tid] * factor;
        sh.w3[0][tid] = a.W3[0][tid];
        sh.w3[1][tid] = slow ? a.W3[1][tid] : 0.0f;
    }
    const auto as_operand = [&](const float (&from)[8]) {
        float v[8];
        _Float16 hi[8], lo[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = from[e] * s_w2;
        split(v, hi, lo, minus_one);
        Frag f;
#pragma unroll
        for (int e = 0; e < 8; ++e) { f.hi[e] = hi[e]; f.lo[e] = lo[e]; }
        return f;
    };
    float *out = a.partial ? a.partial + (size_t)blockIdx.x * a.partial_step : nullptr;

    if (forward) {
        if (GRAD) {
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const Frag f = as_operand(w[b]);
                sh.w2t[ub][b][0][lane] = f.hi;
                sh.w2t[ub][b][1][lane] = f.lo;
            }
        }
        Frag w2[KB];
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            float v[8];
            __builtin_memcpy(v, __builtin_assume_aligned(a.W2 + unit * H + 16 * b + 8 * hh, 16), sizeof(v));
            w2[b] = as_operand(v);
        }
        const float b3[2] = {*a.b3[0] + poison, slow ? *a.b3[1] + poison : 0.0f};
        float gw3[16], gw3s[16], gb3[2] = {0.0f, 0.0f}, loss = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k) gw3[k] = gw3s[k] = 0.0f;
        const half8v *image = (const half8v *)a.W1 + (size_t)ub * XB * 2 * 64 + lane;
        // eight values to a sample's row, as pieces
        const auto put = [&](_Float16 *hi_to, _Float16 *lo_to, const float (&v)[8]) {
            _Float16 hi[8], lo[8];
            split(v, hi, lo, minus_one);
            half8v h, l;
#pragma unroll
            for (int e = 0; e < 8; ++e) { h[e] = hi[e]; l[e] = lo[e]; }
            *(half8v *)hi_to = h;
            *(half8v *)lo_to = l;
        };
        // a unit's value after ReLU and dropout: its bit, as a mask
        const auto kept = [](const float z, const unsigned keep, const int e) {
            return __uint_as_float(__float_as_uint(fmaxf(z, 0.0f)) & (unsigned)((int)(keep << (31 - e)) >> 31));
        };
        const floatx16 zero = {0};
        meet();                                             // the first samples are there
        for (int it = 0; it < mine; ++it) {
            const int now = it & 1;
            floatx16 z;
            bool open1[16];
#pragma unroll
            for (int b = 0; b < XB; ++b) {
                const Frag w = {image[(2 * b) * 64], image[(2 * b + 1) * 64]};
                const Frag x = {*(const half8v *)&sh.xs[now][0][nn][16 * b + 8 * hh], *(const half8v *)&sh.xs[now][1][nn][16 * b + 8 * hh]};
                z = product(w, x, b == 0 ? zero : z);
            }
            const float share = with_share ? sh.share[now][nn] : 0.0f;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const unsigned keep = a.drop ? sh.keep[0][nn][4 * ub + hh + 2 * g] : 255u;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int k = u0 + 16 * g + e;
                    float h = fmaf(z[8 * g + e], by_z1, sh.b1[k]);
                    if (EXTRA) h = fmaf(share, sh.wsm[k], h);
                    v[e] = kept(h, keep, e);
                    open1[8 * g + e] = v[e] > 0.0f;
                }
                put(&sh.d1[0][nn][u0 + 16 * g], &sh.d1[1][nn][u0 + 16 * g], v);
            }
            meet();
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const Frag x = {*(const half8v *)&sh.d1[0][nn][16 * b + 8 * hh], *(const half8v *)&sh.d1[1][nn][16 * b + 8 * hh]};
                z = product(w2[b], x, b == 0 ? zero : z);
            }
            float h2[16], zp = 0.0f, zs = 0.0f;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const unsigned keep = a.drop ? sh.keep[1][nn][4 * ub + hh + 2 * g] : 255u;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int k = u0 + 16 * g + e;
                    const float h = kept(fmaf(z[8 * g + e], by_z2, sh.b2[k]), keep, e);
                    h2[8 * g + e] = h;
                    zp = fmaf(sh.w3[0][k], h, zp);
                    if (EXTRA) zs = fmaf(sh.w3[1][k], h, zs);
                }
            }
            zp = both_halves(zp);
            if (EXTRA) zs = both_halves(zs);
            if (hh == 0) { sh.part[0][ub][nn] = zp; if (EXTRA) sh.part[1][ub][nn] = zs; }
            meet();
            const long long sample = tile_of(it) * T + nn;
            const bool real = sh.real[now][nn], speaks = ub == 0 && hh == 0;
            const float bad = sh.bad[now][0][nn] + sh.bad[now][1][nn];
            float dz[2] = {0.0f, 0.0f};
#pragma unroll
            for (int q = 0; q < (EXTRA ? 2 : 1); ++q) {
                if (q == 1 && !slow) break;
                float zq = b3[q] + bad;
#pragma unroll
                for (int k = 0; k < UB; ++k) zq += sh.part[q][k][nn];
                const float y = 1.0f / (1.0f + expf(-zq));
                if (speaks && a.sigma[q] && sample < a.count) a.sigma[q][sample] = real ? y : 0.0f;
                // what nobody has measured (a NaN) has no part in the loss
                const float t = sh.target[now][q][nn], miss = t == t ? y - t : 0.0f;
                dz[q] = t == t ? 2.0f * miss * y * (1.0f - y) : 0.0f;
                if (speaks) { loss = fmaf(miss, miss, loss); gb3[q] += dz[q]; }
            }
            if (!GRAD) continue;
            const float c0 = dz[0] * by_dz, c1 = dz[1] * by_dz;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                float d[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int r = 8 * g + e, k = u0 + 16 * g + e;
                    float v = c0 * sh.w3[0][k];
                    gw3[r] = fmaf(dz[0], h2[r], gw3[r]);
                    if (EXTRA) {
                        v = fmaf(c1, sh.w3[1][k], v);
                        gw3s[r] = fmaf(dz[1], h2[r], gw3s[r]);
                    }
                    d[e] = h2[r] > 0.0f ? v : 0.0f;
                }
                put(&sh.dz2[0][nn][u0 + 16 * g], &sh.dz2[1][nn][u0 + 16 * g], d);
            }
            meet();
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const Frag w = {sh.w2t[ub][b][0][lane], sh.w2t[ub][b][1][lane]};
                const Frag x = {*(const half8v *)&sh.dz2[0][nn][16 * b + 8 * hh], *(const half8v *)&sh.dz2[1][nn][16 * b + 8 * hh]};
                z = product(w, x, b == 0 ? zero : z);
            }
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                float d[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = open1[8 * g + e] ? z[8 * g + e] * by_d1 : 0.0f;
                put(&sh.dz1[0][nn][u0 + 16 * g], &sh.dz1[1][nn][u0 + 16 * g], d);
            }
            meet();
        }
        if (!out) return;
        if (GRAD) {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const float v = group_sum<32>(gw3[k]), vs = EXTRA ? group_sum<32>(gw3s[k]) : 0.0f;
                if (nn == 0) { out[S::W3 + u0 + 16 * (k >> 3) + (k & 7)] = v; out[S::W3S + u0 + 16 * (k >> 3) + (k & 7)] = vs; }
            }
        }
        if (ub == 0) {
            const float v[3] = {group_sum<64>(gb3[0]), group_sum<64>(gb3[1]), group_sum<64>(loss)};
            if (lane == 0)
#pragma unroll
                for (int q = 0; q < 3; ++q) out[S::REST + q] = v[q];
        }
        return;
    }

    // ---- sums, and what is to come.  UB neighbouring lanes take the features of one side of a sample, EACH of them each.
    constexpr int EACH = HALF / UB;
    const int place = tid - 64 * UB, row = place / UB, sub = place % UB, own = row >> 1, side = row & 1;
    float x[EACH], next_target[2] = {0.0f, 0.0f}, next_share = 0.0f;
    int ahead[2] = {-1, -1};                                // the pair that this lane's sample of the tile after the next names
    bool next_real = false;
    const auto look = [&](const int it) {                   // at indices
        ahead[0] = ahead[1] = -1;
        const long long s = tile_of(it) * T + own;
        if (it < mine && s < a.count) { ahead[0] = a.index[0][s]; ahead[1] = a.index[1][s]; }
    };
    const auto fetch = [&](const int it) {                  // features and targets of the samples whose indices have been looked at
        // a sample that names no pair has no part in anything
        next_real = ahead[0] >= 0 && ahead[0] < a.rows[0] && ahead[1] >= 0 && ahead[1] < a.rows[1];
        const long long s = tile_of(it) * T + own;
#pragma unroll
        for (int e = 0; e < EACH; ++e) x[e] = 0.0f;
        if (next_real) {
            const float *from = a.X[side] + (size_t)ahead[side] * a.F + sub * EACH;
            if ((sub + 1) * EACH <= a.F) {
                __builtin_memcpy(x, from, sizeof(x));
            } else {
#pragma unroll
                for (int e = 0; e < EACH; ++e) if (sub * EACH + e < a.F) x[e] = from[e];
            }
        }
        if (sub == 0 && side == 0) {
            const float none = __builtin_nanf("");
            next_target[0] = next_real && a.target[0] ? a.target[0][s] : none;
            next_target[1] = next_real && a.target[1] ? a.target[1][s] : none;
            if (with_share)
                next_share = next_real ? fminf(1.0f - a.X[0][(size_t)ahead[0] * a.F + a.sm_feature[0]], a.X[1][(size_t)ahead[1] * a.F + a.sm_feature[1]]) : 0.0f;
        }
    };
    const auto stage = [&](const int it) {                  // what has been fetched, normalised, as pieces
        const int to = it & 1;
        float sum = 0.0f, mean = 0.0f, by = s_x;
#pragma unroll
        for (int e = 0; e < EACH; ++e) sum += x[e];
        sum = group_sum<UB>(sum);
        if (a.norm) {
            float squares = 0.0f;
            mean = sum / (float)a.F;
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const float d = sub * EACH + e < a.F ? x[e] - mean : 0.0f;
                squares = fmaf(d, d, squares);
            }
            by = s_x / sqrtf(group_sum<UB>(squares) / (float)a.F + a.eps);
        }
        float v[EACH];
        _Float16 hi[EACH], lo[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) v[e] = sub * EACH + e < a.F && next_real ? (x[e] - mean) * by : 0.0f;
        split(v, hi, lo, minus_one);
#pragma unroll
        for (int e = 0; e < EACH; e += 4) {
            *(half4v *)&sh.xs[to][0][own][side * HALF + sub * EACH + e] = half4v{hi[e], hi[e + 1], hi[e + 2], hi[e + 3]};
            *(half4v *)&sh.xs[to][1][own][side * HALF + sub * EACH + e] = half4v{lo[e], lo[e + 1], lo[e + 2], lo[e + 3]};
        }
        if (sub == 0) {
            sh.bad[to][side][own] = next_real ? sum * 0.0f : 0.0f;
            if (side == 0) {
                sh.target[to][0][own] = next_target[0];
                sh.target[to][1][own] = next_target[1];
                sh.share[to][own] = next_share;
                sh.real[to][own] = next_real;
            }
        }
    };
    const auto draw = [&](const int it, const int layer) {  // random bits
#pragma unroll
        for (int q = 0; q < T * (H / 8) / (64 * UB); ++q) {
            const int at = place + q * 64 * UB, s = at / (H / 8), k = at % (H / 8);
            const Words4 bits = drop_bits(a.rule, (unsigned long long)(tile_of(it) * T + s) * (H / 8) + k, layer);
            unsigned keep = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) keep |= drop_keeps(a.rule, bits, e) ? 1u << e : 0u;
            sh.keep[layer][s][k] = (unsigned char)keep;
        }
    };
    look(0);
    fetch(0);
    stage(0);
    look(1);
    if (a.drop) { draw(0, 0); draw(0, 1); }
    floatx16 gw2[GRAD ? UB : 1], gw1[GRAD ? CT : 1];
    float gb1 = 0.0f, gb2 = 0.0f, gsm = 0.0f, one = 1.0f;
    asm volatile("" : "+s"(one));                           // no instruction (see split)
    if (GRAD) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
#pragma unroll
            for (int t = 0; t < UB; ++t) gw2[t][e] = 0.0f;
#pragma unroll
            for (int t = 0; t < CT; ++t) gw1[t][e] = 0.0f;
        }
    }
    const auto columns_of = [&](const _Float16 *hi, const _Float16 *lo, const int pitch, const int first) {
        return Frag{read_columns(hi, pitch, first, lane), read_columns(lo, pitch, first, lane)};
    };
    const auto add_w1 = [&](const int of) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const Frag d = columns_of(&sh.dz1[0][16 * b][0], &sh.dz1[1][16 * b][0], HP, 32 * ub);
#pragma unroll
            for (int t = 0; t < CT; ++t) gw1[t] = product(d, columns_of(&sh.xs[of][0][16 * b][0], &sh.xs[of][1][16 * b][0], XP, 32 * t), gw1[t]);
#pragma unroll
            for (int e = 0; e < 8; ++e) gb1 = __builtin_fmaf((float)d.hi[e], one, __builtin_fmaf((float)d.lo[e], one, gb1));
            if (EXTRA)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float by = sh.share[of][16 * b + 8 * hh + e];
                    gsm = __builtin_fmaf((float)d.hi[e], by, __builtin_fmaf((float)d.lo[e], by, gsm));
                }
        }
    };
    meet();
    for (int it = 0; it < mine; ++it) {
        const bool more = it + 1 < mine;
        if (more) { fetch(it + 1); look(it + 2); }
        if (GRAD && it > 0) add_w1((it + 1) & 1);
        meet();
        if (more) {
            stage(it + 1);
            if (a.drop) draw(it + 1, 0);
        }
        meet();
        if (more && a.drop) draw(it + 1, 1);
        if (!GRAD) continue;
        meet();
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const Frag d = columns_of(&sh.dz2[0][16 * b][0], &sh.dz2[1][16 * b][0], HP, 32 * ub);
#pragma unroll
            for (int t = 0; t < UB; ++t) gw2[t] = product(d, columns_of(&sh.d1[0][16 * b][0], &sh.d1[1][16 * b][0], HP, 32 * t), gw2[t]);
#pragma unroll
            for (int e = 0; e < 8; ++e) gb2 = __builtin_fmaf((float)d.hi[e], one, __builtin_fmaf((float)d.lo[e], one, gb2));
        }
        meet();
    }
    if (!GRAD || !out) return;
    add_w1((mine + 1) & 1);
    const float by2 = 1.0f / (s_dz2 * s_d1), by1 = 1.0f / (s_dz1 * s_x);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int k = 32 * ub + 8 * (e >> 2) + 4 * hh + (e & 3);
#pragma unroll
        for (int t = 0; t < UB; ++t) out[S::W2 + k * H + 32 * t + nn] = gw2[t][e] * by2;
#pragma unroll
        for (int t = 0; t < CT; ++t) out[S::G + k * (32 * CT) + 32 * t + nn] = gw1[t][e] * by1;
    }
    gb1 = both_halves(gb1) / s_dz1;
    gb2 = both_halves(gb2) / s_dz2;
    gsm = EXTRA ? both_halves(gsm) / s_dz1 : 0.0f;
    if (hh == 0) {
        out[S::B1 + 32 * ub + nn] = gb1;
        out[S::B2 + 32 * ub + nn] = gb2;
        out[S::SM + 32 * ub + nn] = gsm;
    }
}

// Sums of what the workgroups left: value v goes where it belongs.
struct FitOut {
    float *W1, *b1, *W2, *b2, *W3, *b3, *W3s, *b3s, *W1sm, *loss, *G;
    int H, F, padded, half, norm, parts;
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
    s *= o.scale;
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
        if (at == REST_LOSS && o.loss) *o.loss = s;
        return;
    }
    at -= 4;
    const int k = at / o.padded, c = at % o.padded, side = c >= o.half, f = c - side * o.half;
    if (o.norm) o.G[at] = s;
    else if (f < o.F) o.W1[(size_t)k * 2 * o.F + side * o.F + f] = s;
}

// dW1 = G diag g + h beta^T, dg_f = sum_k W1[k, f] G[k, f], dbeta = W1^T h.
constexpr int UNFOLD_SLICES = 16;

__global__ __launch_bounds__(64 * UNFOLD_SLICES) void unfold_kernel(const float *W1, const float *G, const float *h, const float *g, const float *beta, int H,
                                                                    int F, int padded, int half, float *dW1, float *dg, float *dbeta)
{
    __shared__ float sums[2][UNFOLD_SLICES][64];
    const int lane = threadIdx.x % 64, slice = threadIdx.x / 64, c = blockIdx.x * 64 + lane, columns = 2 * F, from = c < F ? c : half + c - F;
    float weight = 0.0f, bias = 0.0f;
    if (c < columns)
        for (int k = slice; k < H; k += UNFOLD_SLICES) {
            const float G1 = G[(size_t)k * padded + from], W = W1[(size_t)k * columns + c];
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


FitPlan fit_plan(const mf_ctx *ctx, const mf_predictor *p, long long count)
{
    FitPlan f{};
    f.H = p->H;
    f.columns = 2 * p->F;
    f.wide = p->F >= FIT_WIDE_FROM;
    if (f.wide) {
        mf_plan_wide(ctx, count, &f);
        return f;
    }
    f.half = (p->F + 15) & ~15;
    f.padded = 2 * f.half;
    f.passes = 1;
    f.tiles = f.padded / 32;
    const long long tiles = (count + FIT_ROWS - 1) / FIT_ROWS, units = (ctx->n_cus > 0 ? ctx->n_cus : 256) * (p->H == 64 ? 2 : 1);
    f.grid = (int)(tiles < units ? tiles : units);
    return f;
}

// Where the folded layer 1 and what goes with it lie in the context's scratch (floats).
constexpr int FOLD_BIAS = 128 * 512, FOLD_NORM1 = FOLD_BIAS + 128, FOLD_NORM2 = FOLD_NORM1 + 128, FOLD_RANGES = FOLD_NORM2 + 128, FOLD_SCALE = FOLD_RANGES + 2 * FIT_RANGE_PARTS;
static_assert(FOLD_SCALE < MF_FIT_SCRATCH, "scratch");

template <int H, int CT, bool GRAD, bool EXTRA>
int launch_fit(mf_ctx *ctx, const FitArgs &a, const FitPlan &f)
{
    const int bytes = (int)sizeof(FitShared<H, CT, GRAD>);
    static_assert(sizeof(FitShared<H, CT, GRAD>) <= 160 * 1024, "LDS");
    const unsigned flag = 1u << ((H == 128 ? 16 : 0) + (GRAD ? 8 : 0) + (EXTRA ? 4 : 0) + CT - 1);
    if (!(ctx->fit_configured & flag)) {
        MF_HIP(hipFuncSetAttribute((const void *)fit_kernel<H, CT, GRAD, EXTRA>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
        ctx->fit_configured |= flag;
    }
    hipLaunchKernelGGL((fit_kernel<H, CT, GRAD, EXTRA>), dim3(f.grid), dim3(H * 4), bytes, ctx->stream, a, ctx->fit_W1 + FOLD_SCALE, ctx->fit_W1 + FOLD_NORM1,
                       ctx->fit_W1 + FOLD_NORM2, ctx->fit_W1 + FOLD_RANGES);
    MF_HIP(hipGetLastError());
    return MF_OK;
}

template <int H, bool GRAD, bool EXTRA>
int launch_fit_tiles(mf_ctx *ctx, const FitArgs &a, const FitPlan &f)
{
    if (f.tiles == 1) return launch_fit<H, 1, GRAD, EXTRA>(ctx, a, f);
    return f.tiles == 2 ? launch_fit<H, 2, GRAD, EXTRA>(ctx, a, f) : launch_fit<H, 3, GRAD, EXTRA>(ctx, a, f);
}

template <int H>
int launch_fit_for(mf_ctx *ctx, const FitArgs &a, const FitPlan &f, bool grad)
{
    if (a.W3[1] || a.W1sm) return grad ? launch_fit_tiles<H, true, true>(ctx, a, f) : launch_fit_tiles<H, false, true>(ctx, a, f);
    return grad ? launch_fit_tiles<H, true, false>(ctx, a, f) : launch_fit_tiles<H, false, false>(ctx, a, f);
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
    a.F = p->F; a.columns = f.columns; a.padded = f.padded; a.half = f.half;
    a.index[0] = s->d_on; a.index[1] = s->d_off;
    a.target[0] = s->d_target; a.target[1] = s->d_target_slow;
    a.sigma[0] = d_sigma; a.sigma[1] = d_sigma_slow;
    a.count = s->count;
    a.W1 = ctx->fit_W1; a.b1 = ctx->fit_W1 + FOLD_BIAS;
    a.W2 = p->d_W2; a.b2 = p->d_b2;
    a.W3[0] = p->d_W3; a.W3[1] = p->d_W3_slow;
    a.b3[0] = p->d_b3; a.b3[1] = p->d_b3_slow;
    a.W1sm = p->d_W1sm;
    a.norm = p->d_ln_w != nullptr; a.eps = p->ln_eps;
    a.sm_feature[0] = p->sm_on_feature; a.sm_feature[1] = p->sm_off_feature;
    a.drop = rule && rule->limit > 0;
    if (a.drop) { a.rule = *rule; a.step = (const unsigned long long *)d_step; }
    a.partial = (float *)d_work;
    a.partial_step = f.step(g != nullptr);
    FoldArgs w{};
    w.W1 = p->d_W1; w.b1 = p->d_b1; w.g = p->d_ln_w; w.beta = p->d_ln_b;
    w.H = f.H; w.F = p->F; w.padded = f.padded; w.half = f.half; w.wide = f.wide;
    w.image = ctx->fit_W1; w.bias = ctx->fit_W1 + FOLD_BIAS; w.scale = ctx->fit_W1 + FOLD_SCALE;
    w.norm1 = ctx->fit_W1 + FOLD_NORM1; w.norm2 = ctx->fit_W1 + FOLD_NORM2; w.ranges = ctx->fit_W1 + FOLD_RANGES;
    for (int k = 0; k < 2; ++k) { w.target[k] = a.target[k]; w.X[k] = a.X[k]; w.index[k] = a.index[k]; w.rows[k] = a.rows[k]; }
    w.count = a.count;
    w.features = f.wide || (a.norm && !a.W1sm) ? 0 : 2 * s->count < (long long)n + m ? 2 : 1;
    hipLaunchKernelGGL(fold_kernel, dim3(f.H / 4 + (f.wide ? 0 : FIT_RANGE_PARTS)), dim3(256), 0, ctx->stream, w);
    MF_HIP(hipGetLastError());
    const int rc = f.wide ? mf_launch_wide(ctx, a, f, g != nullptr) : f.H == 64 ? launch_fit_for<64>(ctx, a, f, g != nullptr) : launch_fit_for<128>(ctx, a, f, g != nullptr);
    if (rc != MF_OK || !a.partial) return rc;
    FitOut o{};
    if (g) {
        o.W1 = g->d_W1; o.b1 = g->d_b1; o.W2 = g->d_W2; o.b2 = g->d_b2; o.W3 = g->d_W3; o.b3 = g->d_b3;
        o.W3s = p->d_W3_slow ? g->d_W3_slow : nullptr; o.b3s = p->d_W3_slow ? g->d_b3_slow : nullptr;
        o.W1sm = p->d_W1sm ? g->d_W1sm : nullptr;
    }
    o.loss = d_loss;
    o.G = a.partial + (size_t)f.grid * a.partial_step;
    o.H = f.H; o.F = p->F; o.padded = f.padded; o.half = f.half; o.norm = a.norm; o.parts = f.grid; o.scale = scale;
    const int values = f.values(g != nullptr), first = g ? 0 : values - 4;
    hipLaunchKernelGGL(fit_sum_kernel, dim3((values - first + FIT_SUM_VALUES - 1) / FIT_SUM_VALUES), dim3(FIT_SUM_VALUES * FIT_SUM_SLICES), 0, ctx->stream,
                       a.partial, a.partial_step, first, values, o);
    if (g && a.norm)
        hipLaunchKernelGGL(unfold_kernel, dim3((f.columns + 63) / 64), dim3(64 * UNFOLD_SLICES), 0, ctx->stream, p->d_W1, o.G, g->d_b1, p->d_ln_w, p->d_ln_b,
                           f.H, p->F, f.padded, f.half, g->d_W1, g->d_ln_w, g->d_ln_b);
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
