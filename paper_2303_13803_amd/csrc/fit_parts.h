// What the kernels of a fit share (fit.hip, fit_wide.hip).
#pragma once
#include "internal.h"
#include "philox.h"
#include "row_sums.h"
#include <math.h>

typedef float floatx16 __attribute__((ext_vector_type(16)));

// Features a workload from which on fit_wide.hip takes over: as many as fit_kernel has accumulators and LDS for.  With 64, 100,000 samples and 128 units it took
// 382 us and fit_kernel takes 135; with 64 units 226 and 116.
constexpr int FIT_WIDE_FROM = 65;
// Features of a predictor without a norm, and those of an SM share, go to fp16 pieces up to this size: what one of them may be, all samples of a call are scaled by, and the
// bits that are left for a z1 of about 1 are then still those of float32.
constexpr float FIT_LARGEST = 4096.0f;
constexpr int FIT_RANGE_PARTS = 256;                        // workgroups that look for the largest feature, at most

struct FitArgs {
    const float *X[2];
    int rows[2], F, padded, half;                           // the 2F columns of layer 1 are laid out as [0, F) and [half, half + F) of `padded` ones
    const int32_t *index[2];
    const float *target[2];                                 // throughput, slowdown (null: not trained)
    float *sigma[2];                                        // (null: not wanted)
    long long count;
    const float *W1, *b1, *g, *beta;                        // for fit_wide.hip W1 and b1 with the norm folded in (see fold_kernel)
    const float *W2, *b2, *W3[2], *b3[2], *W1sm;            // ([1] and W1sm may be null)
    int norm, sm_feature[2];
    float eps;
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

struct FitPlan {
    int H, columns, padded, half, passes, tiles, grid;      // tiles: fit_kernel's, of 32 columns; passes: over the samples, fit_wide.hip's
    int parts;                                              // workgroups that look for bounds
    bool wide;
    int values(bool grad) const { return (H == 64 ? FitSums<64>::G : FitSums<128>::G) + (grad ? H * padded : 0); }
    long long step(bool grad) const { return (values(grad) + 15) & ~15; }
};

int mf_launch_few(mf_ctx *ctx, const FitArgs &a, int H);    // predictions, without dropout and loss: a.count of them
void mf_plan_wide(const mf_ctx *ctx, long long count, FitPlan *f);
int mf_launch_wide(mf_ctx *ctx, const FitArgs &a, const FitPlan &f, const float *ranges, bool grad);     // ranges: f.parts of them

namespace {

// Row r of a 32-row tile of matrix results lies in lane half (r >> 2) & 1; read as unit tile_unit(r), what a lane holds of
// a tile are the units 8 half .. 8 half + 7 and 16 + 8 half .. 16 + 8 half + 7: eight that share a counter.
__device__ __forceinline__ int tile_unit(int r) { return (r & 0x13) | (r & 4) << 1 | (r & 8) >> 1; }

__device__ __forceinline__ float both_halves(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

}  // namespace
