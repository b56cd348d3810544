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
// values lose absolute precision of 2^-39 of the bound.  The bounds: a normalised row has |u|_2 <= sqrt(F), so z1_k <= |W1_k|_2
// sqrt(2F) + b1_k, and what is below 0 is not passed on; |dz3| <= (1 + max |t|) / 2; and through W3 and W2 by their largest values and columns' sums.  Features that no norm
// bounds, those of an SM share behind a norm among them, are looked for; where one is above FIT_LARGEST all of it is done once more in float32 products
// (wide_kernel), so that what others keep does not depend on it.  Without gradients a sample is scaled by its own SM share instead.
//
// A workgroup takes FIT_ROWS samples at a time.  Half of its wavefronts ("forward", 32 hidden units each) take them through the layers and back;
// activations pass between them through LDS.  The others ("sums") add up the gradients of weights, in accumulators that stay until there are no
// more samples, and get the next samples ready: features, their norm, random bits.  A SIMD has one wavefront of either kind, so that the matrix
// instructions of one run beside the arithmetic of the other:
//     forward   layer 1 -> d1        layer 2 -> output    loss, dz2        W2^T dz2 -> dz1
//     sums      dW2, second half     G                    next features    dW2, first half      (either half: 16 samples)
// so that the matrix pipe has something to do throughout; random bits for the next samples are drawn in all four stages.
//
// Measured: a million samples of 32 features a workload through 128 units, with every option, 0.50 ms, 268 TFLOP/s where float32's matrix
// instructions reach 152; the matrix pipe is busy a third of that, and either kind of wavefront takes some 2000 cycles for each of the four
// stages, its own chain of LDS reads, products and arithmetic.  2000 samples of 16 features through 64 units 18 us; 200,003 predictions 60,
// the loss alone of as many 67; a million samples without a norm 0.49 ms, 2000 of them 20 us (the launches that look for what is too large, and that find nothing,
// 5 and 1 to 4).  Registers do not suffice for what a pass with gradients keeps: the compiler leaves 82 vector registers of 256 in memory with 32 features and 128 units,
// 182 with 64; without gradients none up to 48 features.
//
// NaN: a ReLU that is one instruction turns it into 0, so what is not finite among the weights, their bounds, or a sample's features is
// added to the output as a NaN; its features are 0 otherwise, so that a sample that has neither features nor a target changes no gradient.
#include "fit_parts.h"

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));

namespace {

constexpr int FIT_ROWS = 32;

// The exponent of the largest power of two that takes a value of at most `bound` to below 2^14 (0 for bounds that are none).
__device__ __forceinline__ int exponent_below(float bound)
{
    if (!(bound > 0.0f) || !(bound < INFINITY)) return 0;
    int e;
    (void)frexpf(bound, &e);                                // bound < 2^e
    e = e < -96 ? -96 : e;
    return 14 - e;
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

// Pieces of FIT_ROWS samples: rows of N chunks of eight halves, where chunk c of row s lies at place c ^ turn(s).  LDS serves 256 bytes a cycle
// from 64 banks; sixteen rows' reads of the same chunk, and the four rows by four chunks of a transposing read, then lie in different ones.
// (Rows that were longer by 16 halves instead cost 51 of 141 million LDS cycles in conflicts.)
// A lane's places differ by an exclusive or with a constant, so one of them is kept and the others are made as they are needed.
template <int N>
struct Rows {
    _Float16 v[FIT_ROWS][N * 8];
    static __device__ __forceinline__ int turn(int s)
    {
        if (N == 16) return (s & 3) << 2 | (s >> 2 & 3);
        if (N == 8) return (s & 2) << 1 | (s >> 2 & 3);
        return s >> 2 & 3;
    }
    // byte of chunk c of row s
    static __device__ __forceinline__ int place(int s, int c) { return s * (N * 16) + ((c ^ turn(s)) << 4); }
    __device__ __forceinline__ half8v &chunk(int place) { return *(half8v *)((char *)v + place); }
    // For sums over samples: lane l gets column 32 t + l % 32 of samples 16 b + 8 (l / 32) .. + 7.  The transposing read gives a group
    // of sixteen lanes four rows of sixteen columns, a column to each lane.  from: columns_from() of this lane.
    static __device__ __forceinline__ int columns_from(int lane)
    {
        const int group = lane >> 4, i = lane & 15;
        return place(8 * (group >> 1) + (i >> 2), 2 * (group & 1) + (i >> 1 & 1)) + 8 * (i & 1);
    }
    __device__ __forceinline__ half8v columns(int from, int b, int t) const
    {
        const auto read = [&](const int place) {
            return __builtin_bit_cast(half4v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v *)((const char *)v + place)));
        };
        const half4v p = read((from ^ t << 6) + b * 16 * N * 16), q = read((from ^ (t << 6 | 16)) + (b * 16 + 4) * N * 16);
        return __builtin_shufflevector(p, q, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// Keeps the optimiser from computing everything that follows from a place before the loop, in registers there are not.
__device__ __forceinline__ int afresh(int place)
{
    asm volatile("" : "+v"(place));                         // no instruction
    return place;
}

// Waits for what this wavefront has put into or read from LDS, and for the other wavefronts to have come here, but not for loads and stores of
// global memory on their way: features are fetched a stage before they are looked at.
__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Everything of a workgroup's that wavefronts share.
template <int H, int CT, bool GRAD>
struct FitShared {
    static constexpr int T = FIT_ROWS, UB = H / 32, KB = H / 16, XN = CT >= 3 ? 16 : 4 * CT;
    // d1 of the samples before is kept for a stage longer where there is room for it
    static constexpr int D1 = GRAD && (H == 64 || CT < 3) ? 2 : 1;
    Rows<H / 8> d1[D1][2], dz2[GRAD ? 2 : 1], dz1[GRAD ? 2 : 1];    // [of which samples][piece]
    Rows<XN> xs[2][2];                                      // [of which samples][piece]
    half8v w2t[GRAD ? UB : 1][GRAD ? KB : 1][2][64];        // W2^T as operands: [units of layer 1][of layer 2][piece][lane]
    float part[2][UB][T];                                   // output units: partial sums over 32 hidden units
    float target[2][2][T], bad[2][2][T];                    // bad: NaN where features are not finite
    float share[4][T];                                      // (of three tiles some wavefront may be at)
    int real[2][T], pair[2][2][T];                          // pair: rows of the two sides that samples name, -1 both where they name none
    unsigned char keep[2][2][T][H / 8];                     // [of which samples][layer]: which of eight units stay
    float b1[H], wsm[H], b2[H], w3[2][H];                   // by unit; b1, wsm and b2 with the scale and the dropout's factor of their layer
    float most[10][2 * UB];
};

// Before the pass over the samples, where there is more to know than a workgroup of that pass finds by itself.  Layer 1 as fit_wide.hip takes it: with the
// norm's weight and bias folded in, its rows padded with zeros, a wavefront for each hidden unit.  And in the last `parts` workgroups the largest
// feature, where no norm bounds it: of a predictor without a norm, or of an SM share's two; of all workloads or those that the samples name,
// whichever are fewer.
struct FoldArgs {
    const float *W1, *b1, *g, *beta;
    int F, padded, half, rows_of_weights;
    float *W, *bias, *ranges;                               // [H][padded], [H]; [parts]
    const float *X[2];
    const int32_t *index[2];
    int rows[2], first[2], width, listed, parts;            // features first .. first + width of either side
    long long count;
};

__global__ __launch_bounds__(256) void fold_kernel(FoldArgs a)
{
    const int lane = threadIdx.x & 63;
    if ((int)blockIdx.x >= a.rows_of_weights / 4) {
        __shared__ float most[4];
        const int part = blockIdx.x - a.rows_of_weights / 4;
        const long long first = (long long)part * 256 + threadIdx.x, step = (long long)a.parts * 256;
        float x = 0.0f;
        for (int k = 0; k < 2; ++k) {
            const float *X = (k ? a.X[1] : a.X[0]) + (k ? a.first[1] : a.first[0]);
            const int32_t *index = k ? a.index[1] : a.index[0];
            const int rows = k ? a.rows[1] : a.rows[0];
            const long long all = (a.listed ? a.count : rows) * a.width;
            const int32_t *other = k ? a.index[0] : a.index[1];
            const int other_rows = k ? a.rows[0] : a.rows[1];
#pragma unroll 8
            for (long long e = first; e < all; e += step) {
                int row = (int)(e / a.width);
                if (a.listed) {                             // (of samples that name a pair)
                    if ((unsigned)other[row] >= (unsigned)other_rows) continue;
                    row = index[row];
                }
                if ((unsigned)row >= (unsigned)rows) continue;
                const float v = fabsf(X[(size_t)row * a.F + (int)(e % a.width)]);
                if (v < INFINITY) x = fmaxf(x, v);
            }
        }
        x = wave_max(x);
        if (lane == 0) most[threadIdx.x >> 6] = x;
        __syncthreads();
        if (threadIdx.x == 0) a.ranges[part] = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
        return;
    }
    const int k = blockIdx.x * 4 + (threadIdx.x >> 6);
    float sum = 0.0f;
    for (int c = lane; c < a.padded; c += 64) {
        const int side = c >= a.half, f = c - side * a.half, at = side * a.F + f;
        float v = 0.0f;
        if (f < a.F) {
            v = a.W1[(size_t)k * 2 * a.F + at];
            if (a.g) { sum = fmaf(v, a.beta[at], sum); v *= a.g[at]; }
        }
        a.W[(size_t)k * a.padded + c] = v;
    }
    sum = group_sum<64>(sum);
    if (lane == 0) a.bias[k] = a.b1[k] + sum;
}

// EXTRA: the predictor has the slowdown unit or the SM share (or both).
template <int H, int CT, bool GRAD, bool EXTRA>
__global__ __launch_bounds__(H * 4, 2) void fit_kernel(const FitArgs a, const float *__restrict__ ranges, const int parts)
{
    using L = FitShared<H, CT, GRAD>;
    using S = FitSums<H>;
    constexpr int T = FIT_ROWS, UB = H / 32, KB = H / 16, XB = 2 * CT, HALF = 16 * CT;
    extern __shared__ __align__(16) char lds[];
    L &sh = *(L *)lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), nn = lane & 31, hh = lane >> 5;
    const float minus_one = hidden_minus_one();
    DropRule rule = a.rule;
    if (a.step) { const unsigned long long s = *a.step; rule.s0 = (unsigned)s; rule.s1 = (unsigned)(s >> 32); }
    const bool slow = EXTRA && a.W3[1], with_share = EXTRA && a.W1sm;
    const float factor = a.drop ? rule.factor : 1.0f;
    const long long tiles = (a.count + T - 1) / T;
    const int mine = (int)((tiles - blockIdx.x + gridDim.x - 1) / gridDim.x);
    const auto tile_of = [&](const int it) { return (long long)blockIdx.x + (long long)it * gridDim.x; };
    const bool forward = wave < UB;
    const int ub = forward ? wave : wave - UB, unit = 32 * ub + tile_unit(nn), u0 = 32 * ub + 8 * hh;

    // ---- what is to come, the business of the wavefronts that sum up: UB neighbouring lanes take the features of one side of a sample, EACH of them each; the first of these
    // wavefronts ("scout") looks up what the samples name and what was measured of them, a side to either half of it.
    constexpr int EACH = HALF / UB;
    const int place = tid - 64 * UB, row = place / UB, sub = place % UB, own = row >> 1, side = row & 1;
    const bool scout = ub == 0;
    const float *const features = side ? a.X[1] : a.X[0];
    const int all_features = (side ? a.rows[1] : a.rows[0]) > 0 ? (side ? a.rows[1] : a.rows[0]) * a.F : a.F;       // (at most 2^20 x 64)
    float4v x[EACH / 4];
    bool next_real = false;
    // (the scout's: loads without a condition, from a place that is there anyway, so that nothing waits for them before they are needed)
    const int32_t *const index = hh ? a.index[1] : a.index[0];
    const float *const targets = hh ? a.target[1] : a.target[0], *const shares = hh ? a.X[1] : a.X[0];
    const int share_feature = hh ? a.sm_feature[1] : a.sm_feature[0];
    int looked = 0, looked_first = 0, named = -1;
    float next_target = __builtin_nanf(""), next_share = 0.0f;
    const auto sample_of = [&](const int it) { const long long s = tile_of(it) * T + nn; return s < a.count ? s : a.count - 1; };
    const auto look = [&](const int it, int &to) { to = index[sample_of(it)]; };
    const auto name = [&](const int it, const int looked) { // what has been looked up: a sample that names no pair has no part in anything
        const bool mine_real = tile_of(it) * T + nn < a.count && (unsigned)looked < (unsigned)(hh ? a.rows[1] : a.rows[0]);
        const auto both = __builtin_amdgcn_permlane32_swap((unsigned)mine_real, (unsigned)mine_real, false, false);
        named = (both[0] & both[1]) ? looked : -1;
        sh.pair[it & 1][hh][nn] = named;
    };
    const auto ask = [&](const int it) {                    // what was measured, and the SM share, of the samples named last
        if (targets) next_target = targets[sample_of(it)];
        if (with_share) next_share = shares[(named < 0 ? 0 : named) * a.F + share_feature];
    };
    const auto answer = [&](const int it) {
        const int to = it & 1;
        sh.target[to][hh][nn] = named < 0 ? __builtin_nanf("") : next_target;
        if (with_share) {
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(next_share), __float_as_uint(next_share), false, false);
            const float share = fminf(1.0f - __uint_as_float(both[0]), __uint_as_float(both[1]));
            if (hh == 0) sh.share[it & 3][nn] = named < 0 || !(share * 0.0f == 0.0f) ? 0.0f : share;
        }
        if (hh == 0) sh.real[to][nn] = named >= 0;
    };
    const auto fetch = [&](const int it, const int part) {  // features of the samples named, in two parts
        const int at = sh.pair[it & 1][side][own];
        if (part == 0) next_real = at >= 0;
        // (what a lane reads beyond its row is the next row's, and is left out when it is put to use; beyond the last row it reads nothing)
        const int at_feature = (at < 0 ? 0 : at) * a.F + sub * EACH;
#pragma unroll
        for (int e = 0; e < EACH / 4; ++e) {
            if (e % 2 != part) continue;
            const int first = at_feature + 4 * e;
            if (first + 4 <= all_features) x[e] = *(const float4v *)(features + first);
            else
#pragma unroll
                for (int k = 0; k < 4; ++k) x[e][k] = features[first + k < all_features ? first + k : all_features - 1];
        }
    };
    if (!forward && scout) {                                // (on their way during all that follows)
        look(0, looked_first);
        look(1, looked);
    }

    // ---- bounds, and the scales that follow.  Weights are read as the operands that the forward wavefronts make of them: layer 1's with the
    // norm's weight, W2's transpose (or, without a way back, W2), a unit's in two lanes.
    float w[KB][8], u1[XB][8], bias1 = 0.0f, poison = 0.0f;
    // largest of: targets, features (or, of those that a norm bounds, the SM share's two), output weights of either unit, weights of layers 2 and 1, columns' sums of W2, z1 (not below 0) without features and for each
    float v[9] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    const float length = sqrtf((float)a.F);
    const auto read_w2 = [&](const int b, float (&to)[8]) {
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            const float4 r = *(const float4 *)(a.W2 + unit * H + 16 * b + 8 * hh + e);
            to[e] = r.x; to[e + 1] = r.y; to[e + 2] = r.z; to[e + 3] = r.w;
        }
    };
    if (forward) {
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            if (GRAD) {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[b][e] = a.W2[(16 * b + 8 * hh + e) * H + unit];
            } else {
                read_w2(b, w[b]);
            }
        }
        float more = 0.0f, sum = 0.0f, squares = 0.0f;
#pragma unroll
        for (int b = 0; b < XB; ++b) {
            const int c = 16 * b + 8 * hh, of = c >= HALF, f = c - of * HALF;
            float g[8], beta[8];
            if (a.F % 8 == 0) {
                const int at = f < a.F ? of * a.F + f : 0;
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    const float4v r = *(const float4v *)(a.W1 + (size_t)unit * 2 * a.F + at + e);
                    const float4v rg = a.norm ? *(const float4v *)(a.g + at + e) : float4v{1.0f, 1.0f, 1.0f, 1.0f};
                    const float4v rb = a.norm ? *(const float4v *)(a.beta + at + e) : float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int k = 0; k < 4; ++k) { u1[b][e + k] = r[k]; g[e + k] = rg[k]; beta[e + k] = rb[k]; }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = f + e < a.F ? of * a.F + f + e : 0;
                    u1[b][e] = a.W1[(size_t)unit * 2 * a.F + at];
                    g[e] = a.norm ? a.g[at] : 1.0f;
                    beta[e] = a.norm ? a.beta[at] : 0.0f;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool there = f + e < a.F;
                more += there ? u1[b][e] * beta[e] : 0.0f;
                u1[b][e] = there ? u1[b][e] * g[e] : 0.0f;
                v[5] = fmaxf(v[5], fabsf(u1[b][e]));
                sum += fabsf(u1[b][e]);
                squares = fmaf(u1[b][e], u1[b][e], squares);
            }
        }
        sum = both_halves(sum);
        bias1 = a.b1[unit] + both_halves(more);
        const float w_share = with_share ? a.W1sm[unit] : 0.0f;
        // (|u|_2 <= sqrt(F) on either side, so no entry is more; squares of weights beyond 1.8e19 are no float32)
        const float rest = fabsf(w_share) + (a.norm ? fminf(sqrtf(both_halves(squares)) * length * 1.42f, sum * length * 1.001f) : 0.0f);
        // what the ReLU passes on: a bias that closes the unit lowers it (and rounds what is added to it)
        v[7] = fmaxf(bias1 + rest + 1e-6f * (fabsf(bias1) + rest), 0.0f);
        v[8] = fabsf(w_share) + (a.norm ? 0.0f : sum);
        float column = 0.0f;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int e = 0; e < 8; ++e) { v[4] = fmaxf(v[4], fabsf(w[b][e])); column += fabsf(w[b][e]); }
        v[6] = both_halves(column);
        poison = (v[6] + bias1 + sum + w_share) * 0.0f;     // NaN if one of them is not finite
    }
    if (tid < H) {
        v[2] = fabsf(a.W3[0][tid]);
        v[3] = slow ? fabsf(a.W3[1][tid]) : 0.0f;
        poison += a.b2[tid] * 0.0f;
    }
    if (tid < parts) v[1] = ranges[tid];
    if (GRAD) {                                             // this workgroup's own targets, and 1, which shares of a throughput stay below
        const auto most_at = [&](const int it, long long &at) {
            const long long s = tile_of(it) * T + tid % T;
            at = s < a.count ? s : a.count - 1;
            const float t = fabsf(a.target[0][at]), ts = slow ? fabsf(a.target[1][at]) : 0.0f;
            return fmaxf(t < INFINITY ? t : 0.0f, ts < INFINITY ? ts : 0.0f);
        };
        long long at;
        v[0] = 1.0f;
#pragma unroll 4
        for (int it = tid / T; it < mine; it += H * 4 / T) v[0] = fmaxf(v[0], most_at(it, at));
        if (v[0] > 1.0f) {                                  // only of samples that name a pair: others may have anything there
            v[0] = 1.0f;
#pragma unroll 1
            for (int it = tid / T; it < mine; it += H * 4 / T) {
                const float most = most_at(it, at);
                if ((unsigned)a.index[0][at] < (unsigned)a.rows[0] && (unsigned)a.index[1][at] < (unsigned)a.rows[1]) v[0] = fmaxf(v[0], most);
            }
        }
    }
#pragma unroll
    for (int q = 0; q < 9; ++q) {
        v[q] = wave_max(v[q]);
        if (lane == 0) sh.most[q][wave] = v[q];
    }
    poison = group_sum<64>(poison);
    if (lane == 0) sh.most[9][wave] = poison;
    int named_first = -1;
    if (!forward && scout) {
        name(0, looked_first);
        named_first = named;
        ask(0);
        name(1, looked);
    }
    meet();
    if (!forward) {
        fetch(0, 0);
        fetch(0, 1);
    }
    poison = 0.0f;
    for (int x = 0; x < 2 * UB; ++x) {
#pragma unroll
        for (int q = 0; q < 9; ++q) v[q] = fmaxf(v[q], sh.most[q][x]);
        poison += sh.most[9][x];
    }
    const int e_x = exponent_below(a.norm ? length * 1.001f : v[1]), e_w2 = exponent_below(v[4]), e_w1 = exponent_below(v[5]);
    const float bound2 = 0.5f * (1.0f + v[0]) * (v[2] + v[3]) * factor * 1.001f;
    const int e_dz2 = exponent_below(bound2), e_dz1 = exponent_below(bound2 * factor * v[6] * 1.001f);
    // Without gradients a lane of the forward wavefronts has a sample of its own, whose SM share, where nothing bounds it, scales what is its own and
    // nobody else's (OWN: then by_z1, by_z2, sh.b1 and sh.wsm lack that scale).
    constexpr bool OWN = !GRAD && EXTRA;
    const float most_d1 = (v[7] + (OWN && a.norm ? 0.0f : v[8] * v[1])) * factor * 1.001f, most_share = a.norm ? v[8] * factor * 1.001f : 0.0f;
    const int e_d1 = OWN ? 0 : exponent_below(most_d1);
    // what accumulators of the three products are multiplied with
    // (exponents are added up first: products of scales may be no float32)
    const float by_z1 = ldexpf(factor, e_d1 - e_x - e_w1), by_z2 = ldexpf(factor, -e_d1 - e_w2), by_d1 = ldexpf(factor, e_dz1 - e_dz2 - e_w2), by_dz = ldexpf(factor, e_dz2);
    const float s_x = ldexpf(1.0f, e_x), s_w1 = ldexpf(1.0f, e_w1), s_w2 = ldexpf(1.0f, e_w2), s_d1 = ldexpf(1.0f, e_d1);
    poison += most_d1 * v[4] * 0.0f;                        // NaN where even a bound on layer 2's terms is none
    if (tid < H) {
        sh.wsm[tid] = with_share ? a.W1sm[tid] * (factor * s_d1) : 0.0f;
        sh.b2[tid] = a.b2[tid] * factor;
        sh.w3[0][tid] = a.W3[0][tid];
        sh.w3[1][tid] = slow ? a.W3[1][tid] : 0.0f;
    }
    if (forward && hh == 0) sh.b1[unit] = bias1 * (factor * s_d1);
    const auto as_operand = [&](const float (&from)[8], const float scale) {
        float v[8];
        _Float16 hi[8], lo[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = from[e] * scale;
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
                const Frag f = as_operand(w[b], s_w2);
                sh.w2t[ub][b][0][lane] = f.hi;
                sh.w2t[ub][b][1][lane] = f.lo;
            }
        }
        Frag w2[KB];
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            if (GRAD) read_w2(b, w[b]);
            w2[b] = as_operand(w[b], s_w2);
        }
        const float b3 = (EXTRA && slow && hh ? *a.b3[1] : *a.b3[0]) + poison;
        float gw3[16], gw3s[16], gb3 = 0.0f, loss = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k) gw3[k] = gw3s[k] = 0.0f;
        const int mine_at = Rows<H / 8>::place(nn, hh), features_at = Rows<L::XN>::place(nn, hh);
        Frag w1[XB];
#pragma unroll
        for (int b = 0; b < XB; ++b) w1[b] = as_operand(u1[b], s_w1);
        // eight values to a sample's row, as pieces
        const auto put = [&](Rows<H / 8> *to, const int g, const float (&v)[8]) {
            _Float16 hi[8], lo[8];
            split(v, hi, lo, minus_one);
            half8v h, l;
#pragma unroll
            for (int e = 0; e < 8; ++e) { h[e] = hi[e]; l[e] = lo[e]; }
            const int place = afresh(mine_at) ^ (ub << 6 | g << 5);
            to[0].chunk(place) = h;
            to[1].chunk(place) = l;
        };
        // columns 16 b + 8 hh .. + 7 of this lane's sample
        const auto operand = [&](auto *rows, const int place, const int b) { return Frag{rows[0].chunk(place ^ b << 5), rows[1].chunk(place ^ b << 5)}; };
        // a unit's value after ReLU and dropout: its bit, as a mask
        const auto kept = [](const float z, const unsigned keep, const int e) {
            return __uint_as_float(__float_as_uint(fmaxf(z, 0.0f)) & (unsigned)__builtin_amdgcn_sbfe((int)keep, e >> 1 | (e & 1) << 2, 1));
        };
        const floatx16 zero = {0};
        meet();                                             // the first samples are there
        for (int it = 0; it < mine; ++it) {
            const int now = it & 1;
            floatx16 z;
            bool open1[16];
            {
                const int features_here = afresh(features_at);
                Frag x[XB];
#pragma unroll
                for (int b = 0; b < XB; ++b) x[b] = operand(sh.xs[now], features_here, b);
#pragma unroll
                for (int b = 0; b < XB; ++b) z = product(w1[b], x[b], b == 0 ? zero : z);
            }
            float share = with_share ? sh.share[it & 3][nn] : 0.0f;
            const float own_most = fmaf(most_share, fabsf(share), most_d1);
            const int own_scale = OWN ? exponent_below(own_most) : 0;
            const float s_own = ldexpf(1.0f, own_scale), by_z1_here = OWN ? by_z1 * s_own : by_z1, by_z2_here = OWN ? ldexpf(by_z2, -own_scale) : by_z2;
            if (OWN) share *= s_own;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const unsigned keep = a.drop ? sh.keep[now][0][nn][4 * ub + hh + 2 * g] : 255u;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int k = u0 + 16 * g + e;
                    float h = fmaf(z[8 * g + e], by_z1_here, OWN ? sh.b1[k] * s_own : sh.b1[k]);
                    if (EXTRA) h = fmaf(share, sh.wsm[k], h);
                    v[e] = kept(h, keep, e);
                    open1[8 * g + e] = v[e] > 0.0f;
                }
                put(sh.d1[L::D1 > 1 ? now : 0], g, v);
            }
            meet();
            int here = afresh(mine_at);
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const Frag x = operand(sh.d1[L::D1 > 1 ? now : 0], here, b);
                z = product(w2[b], x, b == 0 ? zero : z);
            }
            float h2[16], zp = 0.0f, zs = 0.0f;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const unsigned keep = a.drop ? sh.keep[now][1][nn][4 * ub + hh + 2 * g] : 255u;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int k = u0 + 16 * g + e;
                    const float h = kept(fmaf(z[8 * g + e], by_z2_here, sh.b2[k]), keep, e);
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
            const bool real = sh.real[now][nn], speaks = ub == 0 && (hh == 0 || slow);
            // (with two output units either half of the wavefront takes one)
            const int unit3 = EXTRA && slow ? hh : 0;
            float z3 = b3 + sh.bad[now][0][nn] + sh.bad[now][1][nn];
            if (OWN) z3 += own_most * v[4] * 0.0f;
#pragma unroll
            for (int k = 0; k < UB; ++k) z3 += sh.part[unit3][k][nn];
            const float y = 1.0f / (1.0f + expf(-z3));
            float *const sigma = EXTRA && unit3 ? a.sigma[1] : a.sigma[0];
            if (speaks && sigma && sample < a.count) sigma[sample] = real ? y : 0.0f;
            // what nobody has measured (a NaN) has no part in the loss
            const float t = sh.target[now][unit3][nn], miss = t == t ? y - t : 0.0f, dz3 = t == t ? 2.0f * miss * y * (1.0f - y) : 0.0f;
            if (speaks) { loss = fmaf(miss, miss, loss); gb3 += dz3; }
            float dz[2] = {dz3, 0.0f};
            if (EXTRA && slow) {
                const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(dz3), __float_as_uint(dz3), false, false);
                dz[0] = __uint_as_float(s[0]);
                dz[1] = __uint_as_float(s[1]);
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
                put(sh.dz2, g, d);
            }
            meet();
            here = afresh(mine_at);
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const Frag w = {sh.w2t[ub][b][0][lane], sh.w2t[ub][b][1][lane]};
                const Frag x = operand(sh.dz2, here, b);
                z = product(w, x, b == 0 ? zero : z);
            }
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                float d[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = open1[8 * g + e] ? z[8 * g + e] * by_d1 : 0.0f;
                put(sh.dz1, g, d);
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
            // (without the slowdown unit the upper half has no part in them)
            gb3 = group_sum<32>(gb3);
            loss = group_sum<64>(loss);
            if (nn == 0) out[S::REST + (hh == 0 ? REST_B3 : REST_B3S)] = gb3;
            if (lane == 0) out[S::REST + REST_LOSS] = loss;
        }
        return;
    }

    // ---- sums, and what is to come
    const float inverse = 1.0f / (float)a.F;
    const auto stage = [&](const int it) {                  // what has been fetched, normalised, as pieces
        const int to = it & 1;
        float sum = 0.0f, mean = 0.0f, by = s_x, v[EACH];
        _Float16 hi[EACH], lo[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            v[e] = sub * EACH + e < a.F && next_real ? x[e / 4][e % 4] : 0.0f;
            sum += v[e];
        }
        sum = group_sum<UB>(sum);
        // What is not finite is added to the output (`bad`) and has no other part: gradients sum up what is passed back, nothing where nothing was measured,
        // times features.
        const float bad = sum * 0.0f;
        if (GRAD && !(bad == 0.0f)) {
            sum = 0.0f;
#pragma unroll
            for (int e = 0; e < EACH; ++e) v[e] = 0.0f;
        }
        if (a.norm) {
            float squares = 0.0f;
            mean = sum * inverse;
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                v[e] = sub * EACH + e < a.F ? v[e] - mean : 0.0f;
                squares = fmaf(v[e], v[e], squares);
            }
            by = s_x * __builtin_amdgcn_rsqf(fmaf(group_sum<UB>(squares), inverse, a.eps));     // (to a step of float32)
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e) v[e] *= by;
        split(v, hi, lo, minus_one);
#pragma unroll
        for (int e = 0; e < EACH; e += 4) {
            const int c = side * HALF + sub * EACH + e;
            const int place = Rows<L::XN>::place(own, c >> 3) + 2 * (c & 4);
            *(half4v *)((char *)&sh.xs[to][0] + place) = half4v{hi[e], hi[e + 1], hi[e + 2], hi[e + 3]};
            *(half4v *)((char *)&sh.xs[to][1] + place) = half4v{lo[e], lo[e + 1], lo[e + 2], lo[e + 3]};
        }
        if (sub == 0) sh.bad[to][side][own] = bad;
    };
    const unsigned short limit = (unsigned short)(rule.limit - 1);      // (a dropout's limit is at least 1)
    const ushort2v below = {limit, limit};
    const auto draw = [&](const int it, const int which) {  // random bits: of four groups of eight units that are this lane's, two a layer, one
        const int layer = which >> 1, at = place + (which & 1) * 64 * UB, s = at / (H / 8), k = at % (H / 8);
        // (groups of a tile share the upper word of their counter, and so half of the first two rounds is the same for all lanes)
        const unsigned long long first = (unsigned long long)tile_of(it) * (T * (H / 8));
        const Words4 bits = philox((unsigned)first + at, (unsigned)(first >> 32) | layer << 16, rule.s0, rule.s1, rule.k0, rule.k1);
        // two halves at a time: 1 where a half is at least the limit.  Element 2 w + h ends as bit w + 4 h.
        unsigned keep = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            unsigned above = __builtin_bit_cast(unsigned, __builtin_elementwise_sub_sat(__builtin_bit_cast(ushort2v, bits.w[w]), below));
            asm volatile("" : "+v"(above));                 // no instruction (and no comparison of either half in the place of two instructions for both)
            keep |= __builtin_bit_cast(unsigned, __builtin_elementwise_min(__builtin_bit_cast(ushort2v, above), ushort2v{1, 1})) << w;
        }
        sh.keep[it & 1][layer][s][k] = (unsigned char)(keep | keep >> 12);
    };
    static_assert(T * (H / 8) == 2 * 64 * UB, "groups");
    stage(0);
    if (scout) {
        const int later = named;
        named = named_first;
        answer(0);
        named = later;
    }
    fetch(1, 0);
    fetch(1, 1);
    if (scout) look(2, looked);
    if (a.drop) for (int q = 0; q < 4; ++q) draw(0, q);
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
    const int units_from = Rows<H / 8>::columns_from(lane), features_from = Rows<L::XN>::columns_from(lane);
    const auto columns_of = [&](const auto *rows, const int from, const int b, const int t) { return Frag{rows[0].columns(from, b, t), rows[1].columns(from, b, t)}; };
    // products of one operand with several, of which consecutive instructions never need one another's result
    const auto products = [&](const Frag &d, const auto &with, floatx16 *sums) {
        constexpr int N = sizeof(with) / sizeof(Frag);
#pragma unroll
        for (int t = 0; t < N; ++t) sums[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(d.hi, with[t].hi, sums[t], 0, 0, 0);
#pragma unroll
        for (int t = 0; t < N; ++t) sums[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(d.hi, with[t].lo, sums[t], 0, 0, 0);
#pragma unroll
        for (int t = 0; t < N; ++t) sums[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(d.lo, with[t].hi, sums[t], 0, 0, 0);
    };
    // (meanwhile: work that needs none of the operands, while they are on their way)
    const auto add_w1 = [&](const int it, const auto &meanwhile) {
        const int of = it & 1;
        Frag d[2], u[2][CT];
        const int units = afresh(units_from), features = afresh(features_from);
        const auto read = [&](const int b) {
            d[b] = columns_of(sh.dz1, units, b, ub);
#pragma unroll
            for (int t = 0; t < CT; ++t) u[b][t] = columns_of(sh.xs[of], features, b, t);
        };
        read(0);
        __builtin_amdgcn_sched_barrier(0);
        meanwhile();
        __builtin_amdgcn_sched_barrier(0);
        read(1);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            products(d[b], u[b], gw1);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (!EXTRA) { gb1 = __builtin_fmaf((float)d[b].hi[e], one, __builtin_fmaf((float)d[b].lo[e], one, gb1)); continue; }
                const float v = __builtin_fmaf((float)d[b].hi[e], one, (float)d[b].lo[e]);
                gb1 += v;
                gsm = fmaf(v, sh.share[it & 3][16 * b + 8 * hh + e], gsm);
            }
        }
    };
    const auto add_w2 = [&](const int of, const int b, const auto &meanwhile) {      // half of a tile's samples
        const int units = afresh(units_from), of_d1 = L::D1 > 1 ? of : 0;
        const Frag d = columns_of(sh.dz2, units, b, ub);
        Frag u[2][UB / 2];
        const auto read = [&](const int half) {
#pragma unroll
            for (int t = 0; t < UB / 2; ++t) u[half][t] = columns_of(sh.d1[of_d1], units, b, half * (UB / 2) + t);
        };
        read(0);
        __builtin_amdgcn_sched_barrier(0);
        meanwhile();
        __builtin_amdgcn_sched_barrier(0);
        read(1);
        products(d, u[0], gw2);
        products(d, u[1], gw2 + UB / 2);
#pragma unroll
        for (int e = 0; e < 8; ++e) gb2 = __builtin_fmaf((float)d.hi[e], one, __builtin_fmaf((float)d.lo[e], one, gb2));
    };
    meet();
    for (int it = 0; it < mine; ++it) {
        const bool more = it + 1 < mine, drawn = more && a.drop;
        const int now = it & 1, before = now ^ 1;
        if (scout && more) ask(it + 1);
        const auto draw_next = [&](const int which) { return [&, which]() { if (drawn) draw(it + 1, which); }; };
        if (L::D1 > 1 && it > 0) add_w2(before, 1, [] {});
        draw_next(0)();
        meet();
        if (scout && more) answer(it + 1);
        if (scout && it + 2 < mine) name(it + 2, looked);
        if (GRAD && it > 0) add_w1(it - 1, [] {});
        draw_next(1)();
        // (features are read right after the last meeting of all)
        if (!GRAD && more) stage(it + 1);
        meet();
        draw_next(2)();
        if (GRAD && more) stage(it + 1);
        if (it + 2 < mine) fetch(it + 2, 0);
        if (!GRAD) {
            draw_next(3)();
            if (it + 2 < mine) fetch(it + 2, 1);
            if (scout) look(it + 3, looked);
            continue;
        }
        meet();
        if (it + 2 < mine) fetch(it + 2, 1);
        if (scout) look(it + 3, looked);
        add_w2(now, 0, draw_next(3));
        if (L::D1 == 1) add_w2(now, 1, [] {});
        meet();
    }
    if (!GRAD || !out) return;
    if (L::D1 > 1) add_w2((mine + 1) & 1, 1, [] {});
    add_w1(mine - 1, [] {});
    const float by2 = ldexpf(1.0f, -e_dz2 - e_d1), by1 = ldexpf(1.0f, -e_dz1 - e_x);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int k = 32 * ub + 8 * (e >> 2) + 4 * hh + (e & 3);
#pragma unroll
        for (int t = 0; t < UB; ++t) out[S::W2 + k * H + 32 * t + nn] = gw2[t][e] * by2;
#pragma unroll
        for (int t = 0; t < CT; ++t) out[S::G + k * (32 * CT) + 32 * t + nn] = gw1[t][e] * by1;
    }
    gb1 = ldexpf(both_halves(gb1), -e_dz1);
    gb2 = ldexpf(both_halves(gb2), -e_dz2);
    gsm = EXTRA ? ldexpf(both_halves(gsm), -e_dz1) : 0.0f;
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
#pragma unroll 4
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
#pragma unroll 4
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

// Where what fold_kernel makes lies in the context's scratch (floats).
constexpr int FOLD_BIAS = 128 * 512, FOLD_RANGES = FOLD_BIAS + 128;
static_assert(FOLD_RANGES + FIT_RANGE_PARTS <= MF_FIT_SCRATCH, "scratch");

template <int H, int CT, bool GRAD, bool EXTRA>
int launch_fit(mf_ctx *ctx, const FitArgs &a, const FitPlan &f)
{
    const int bytes = (int)sizeof(FitShared<H, CT, GRAD>);
    static_assert(sizeof(FitShared<H, CT, GRAD>) <= 160 * 1024, "LDS");
    constexpr unsigned long long flag = lds_bit_fit(H, CT, GRAD, EXTRA);
    if (!(ctx->kernels_configured & flag)) {
        MF_HIP(hipFuncSetAttribute((const void *)fit_kernel<H, CT, GRAD, EXTRA>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
        ctx->kernels_configured |= flag;
    }
    hipLaunchKernelGGL((fit_kernel<H, CT, GRAD, EXTRA>), dim3(f.grid), dim3(H * 4), bytes, ctx->stream, a, ctx->fit_W1 + FOLD_RANGES, f.parts);
    MF_HIP(hipGetLastError());
    return MF_OK;
}

template <int H, bool GRAD, bool EXTRA>
int launch_fit_tiles(mf_ctx *ctx, const FitArgs &a, const FitPlan &f)
{
    if (f.tiles == 1) return launch_fit<H, 1, GRAD, EXTRA>(ctx, a, f);
    if (f.tiles == 2) return launch_fit<H, 2, GRAD, EXTRA>(ctx, a, f);
    return f.tiles == 3 ? launch_fit<H, 3, GRAD, EXTRA>(ctx, a, f) : launch_fit<H, 4, GRAD, EXTRA>(ctx, a, f);
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
    FitPlan f = fit_plan(ctx, p, s->count);
    FitArgs a{};
    a.X[0] = n > 0 ? d_on : ctx->fit_W1; a.X[1] = m > 0 ? d_off : ctx->fit_W1;      // (a row that can be read where there is none)
    a.rows[0] = n; a.rows[1] = m;
    a.F = p->F; a.padded = f.padded; a.half = f.half;
    a.index[0] = s->d_on; a.index[1] = s->d_off;
    a.target[0] = s->d_target; a.target[1] = s->d_target_slow;
    a.sigma[0] = d_sigma; a.sigma[1] = d_sigma_slow;
    a.count = s->count;
    a.W1 = p->d_W1; a.b1 = p->d_b1;
    a.g = p->d_ln_w; a.beta = p->d_ln_b;
    a.W2 = p->d_W2; a.b2 = p->d_b2;
    a.W3[0] = p->d_W3; a.W3[1] = p->d_W3_slow;
    a.b3[0] = p->d_b3; a.b3[1] = p->d_b3_slow;
    a.W1sm = p->d_W1sm;
    a.norm = p->d_ln_w != nullptr; a.eps = p->ln_eps;
    a.sm_feature[0] = p->sm_on_feature; a.sm_feature[1] = p->sm_off_feature;
    a.drop = rule && rule->limit > 0;
    if (a.drop) { a.rule = *rule; a.step = (const unsigned long long *)d_step; }
    // Predictions that the device holds at once, a workgroup each (2048 threads a compute unit, 4 H a pair), without staging and looking for bounds: one of 32 features and
    // 128 units 3.5 us, with them 9.7; 1024 8.4 and 10.0; 2048 14.5 and 10.1.  With 16 and 64: 3.2 and 6.3; 2048 6.4 and 6.5; 4096 10.3 and 6.6.
    if (!d_work && a.count <= (ctx->n_cus > 0 ? ctx->n_cus : 256) * (512ll / f.H)) return mf_launch_few(ctx, a, f.H);
    a.partial = (float *)d_work;
    a.partial_step = f.step(g != nullptr);
    float *const ranges = ctx->fit_W1 + FOLD_RANGES;
    FitArgs folded = a;                                     // as wide_kernel takes it
    // What no norm bounds: features, and the SM share, but where there are no gradients, since there every sample is scaled by its own.
    const bool look = !f.wide && (!a.norm || (a.W1sm && g));
    if (f.wide || look) {
        FoldArgs w{};
        w.W1 = p->d_W1; w.b1 = p->d_b1; w.g = p->d_ln_w; w.beta = p->d_ln_b;
        w.F = p->F; w.padded = f.padded; w.half = f.half; w.rows_of_weights = f.H;
        w.W = ctx->fit_W1; w.bias = ctx->fit_W1 + FOLD_BIAS; w.ranges = ranges;
        w.width = a.norm ? 1 : p->F;
        for (int k = 0; k < 2; ++k) { w.X[k] = a.X[k]; w.index[k] = a.index[k]; w.rows[k] = a.rows[k]; w.first[k] = a.norm ? a.sm_feature[k] : 0; }
        w.count = a.count;
        w.listed = 2 * s->count < (long long)n + m;
        const long long values = w.width * (w.listed ? 2 * a.count : (long long)n + m), parts = (values + 2047) / 2048;      // eight values a thread
        f.parts = w.parts = look ? (int)(parts < 1 ? 1 : parts < FIT_RANGE_PARTS ? parts : FIT_RANGE_PARTS) : 0;
        hipLaunchKernelGGL(fold_kernel, dim3(w.rows_of_weights / 4 + w.parts), dim3(256), 0, ctx->stream, w);
        MF_HIP(hipGetLastError());
        folded.W1 = w.W;
        folded.b1 = w.bias;
    }
    int rc = MF_OK;
    if (!f.wide) rc = f.H == 64 ? launch_fit_for<64>(ctx, a, f, g != nullptr) : launch_fit_for<128>(ctx, a, f, g != nullptr);
    if (rc == MF_OK && (f.wide || look)) rc = mf_launch_wide(ctx, folded, f, ranges, g != nullptr);
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
