// Operators of a predictor's layers that stand alone: layer norm with its gradient, and dropout.
//
//   layer norm   mu = sum x / C, v = sum (x - mu)^2 / C, r = 1 / sqrt(v + eps), u = (x - mu) r, y = w u + b
//   gradient     g = w dy:  dx = r (g - mean(g) - u mean(g u)),  dw = sum over rows of dy u,  db = sum over rows of dy
//   dropout      y = x * factor where the element's random bits say so, else 0 (philox.h)
//
// All of it is bound by memory: two passes over rows x C values, three for the gradient, which takes the moments again from the
// row that it has in registers anyway.  A row lives in the registers of LANES lanes, NV vectors of 16 bytes each, and is
// summed up there in float32, the squares around the mean that is already known.  Rows may begin at any element: vectors are loaded and
// stored unaligned, and the one that would reach over a row's end is moved back to end with it; what it
// then holds twice is written twice, the same bits, and counted once.
//
// Measured (read and written bytes over time; a large copy reaches 4.7 TB/s): the norm of 1,000,003 x 128 bfloat16 5.2 TB/s, its gradient of 131,072 x 1024 float16
// 5.0, dropout of 500,009 x 251 bfloat16 6.0.  Of 2000 x 64 float32 values the gradient takes 4 us and its sums 2, dropout 2; the norm of 64 x 16 1.7.
#include "internal.h"
#include "philox.h"
#include "row_sums.h"
#include <math.h>

namespace {

constexpr int LAYER_THREADS = 256, LAYER_MAX_WIDTH = 8192;

template <typename T, int VEC> struct Pack { T v[VEC]; };

template <typename T, int VEC>
__device__ __forceinline__ void load_floats(float (&x)[VEC], const T *p)
{
    Pack<T, VEC> q;
    __builtin_memcpy(&q, p, sizeof(q));
#pragma unroll
    for (int t = 0; t < VEC; ++t) x[t] = (float)q.v[t];
}
// One rounding, to the nearest value of the type.
template <typename T, int VEC>
__device__ __forceinline__ void store_floats(T *p, const float (&x)[VEC])
{
    Pack<T, VEC> q;
#pragma unroll
    for (int t = 0; t < VEC; ++t) q.v[t] = (T)x[t];
    __builtin_memcpy(p, &q, sizeof(q));
}

// Where a lane's vectors lie in a row.
template <int VEC, int LANES, int NV>
struct RowPlace {
    int first[NV];                                          // column of the vector's first value, < 0: none
    int skip[NV];                                           // its values before this one are a neighbour's
    __device__ __forceinline__ RowPlace(int lane, int width)
    {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = (j * LANES + lane) * VEC;
            first[j] = col >= width ? -1 : (col + VEC <= width ? col : width - VEC);
            skip[j] = col >= width ? VEC : col - first[j];
        }
    }
};

template <int LANES>
__device__ __forceinline__ float row_sum(float v, float *waves)
{
    if constexpr (LANES <= 64) {
        return group_sum<LANES>(v);
    } else {
        v = group_sum<64>(v);
        __syncthreads();                                    // the last sum has been read
        if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
        __syncthreads();
        return waves[0] + waves[1] + waves[2] + waves[3];
    }
}

struct NormArgs {
    const void *x, *dy;
    void *out;                                              // y, or dx
    int64_t rows, ldx, lddy, ldo;
    int width;
    const float *w, *b;
    float eps;
    float *partial;                                         // [workgroups][2][width]
};

// x - mu of this lane's part of a row (in place) and 1 / sqrt(v + eps).
template <int VEC, int LANES, int NV>
__device__ __forceinline__ float centre(float (&x)[NV][VEC], const RowPlace<VEC, LANES, NV> &at, int width, float eps, float *waves)
{
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int t = 0; t < VEC; ++t) sum += t >= at.skip[j] ? x[j][t] : 0.0f;
    const float mean = row_sum<LANES>(sum, waves) / (float)width;
    float squares = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int t = 0; t < VEC; ++t) {
            x[j][t] -= mean;
            squares += t >= at.skip[j] ? x[j][t] * x[j][t] : 0.0f;
        }
    return 1.0f / sqrtf(row_sum<LANES>(squares, waves) / (float)width + eps);
}

template <typename T, int VEC, int LANES, int NV>
__global__ __launch_bounds__(LAYER_THREADS) void norm_kernel(NormArgs a)
{
    __shared__ float waves[4];
    constexpr int GROUPS = LAYER_THREADS / LANES;
    const int lane = threadIdx.x % LANES;
    const RowPlace<VEC, LANES, NV> at(lane, a.width);
    float w[NV][VEC], b[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (at.first[j] >= 0) { load_floats(w[j], a.w + at.first[j]); load_floats(b[j], a.b + at.first[j]); }
    for (int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES; row < a.rows; row += (int64_t)gridDim.x * GROUPS) {
        float x[NV][VEC];
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (at.first[j] >= 0) load_floats(x[j], (const T *)a.x + row * a.ldx + at.first[j]);
            else
#pragma unroll
                for (int t = 0; t < VEC; ++t) x[j][t] = 0.0f;
        const float rstd = centre<VEC, LANES, NV>(x, at, a.width, a.eps, waves);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (at.first[j] >= 0) {
#pragma unroll
                for (int t = 0; t < VEC; ++t) x[j][t] = fmaf(x[j][t] * rstd, w[j][t], b[j][t]);
                store_floats((T *)a.out + row * a.ldo + at.first[j], x[j]);
            }
    }
}

// One pass: moments again from the row in registers, so that x and dy are read once.  dw and db are summed over a workgroup's rows in registers, over its groups of lanes in LDS, and over workgroups by
// column_sum_kernel, always in the same order.
template <typename T, int VEC, int LANES, int NV>
__global__ __launch_bounds__(LAYER_THREADS) void norm_grad_kernel(NormArgs a)
{
    __shared__ float waves[4];
    constexpr int GROUPS = LAYER_THREADS / LANES, COLUMNS = LANES * NV * VEC;
    __shared__ float all[GROUPS > 1 ? GROUPS * COLUMNS : 1];
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const RowPlace<VEC, LANES, NV> at(lane, a.width);
    const float inverse = 1.0f / (float)a.width;
    float w[NV][VEC], dw[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (at.first[j] >= 0) load_floats(w[j], a.w + at.first[j]);
#pragma unroll
        for (int t = 0; t < VEC; ++t) dw[j][t] = db[j][t] = 0.0f;
    }
    // (whole workgroups go round together: there are barriers in it where a row takes all of one)
    for (int64_t base = (int64_t)blockIdx.x * GROUPS; base < a.rows; base += (int64_t)gridDim.x * GROUPS) {
        const int64_t row = base + group;
        const bool real = row < a.rows;
        float x[NV][VEC], dy[NV][VEC];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (at.first[j] >= 0 && real) {
                load_floats(x[j], (const T *)a.x + row * a.ldx + at.first[j]);
                load_floats(dy[j], (const T *)a.dy + row * a.lddy + at.first[j]);
            } else {
#pragma unroll
                for (int t = 0; t < VEC; ++t) x[j][t] = dy[j][t] = 0.0f;
            }
        }
        const float rstd = centre<VEC, LANES, NV>(x, at, a.width, a.eps, waves);
        float sum = 0.0f, dot = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int t = 0; t < VEC; ++t) {
                x[j][t] *= rstd;
                const bool own = t >= at.skip[j];
                const float g = own ? dy[j][t] * w[j][t] : 0.0f;
                sum += g;
                dot += own ? g * x[j][t] : 0.0f;
                dw[j][t] += own && real ? dy[j][t] * x[j][t] : 0.0f;
                db[j][t] += own && real ? dy[j][t] : 0.0f;
            }
        sum = row_sum<LANES>(sum, waves) * inverse;
        dot = row_sum<LANES>(dot, waves) * inverse;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (at.first[j] >= 0 && real) {
                float dx[VEC];
#pragma unroll
                for (int t = 0; t < VEC; ++t) dx[t] = rstd * (fmaf(dy[j][t], w[j][t], -sum) - x[j][t] * dot);
                store_floats((T *)a.out + row * a.ldo + at.first[j], dx);
            }
    }
    float *mine = a.partial + (int64_t)blockIdx.x * 2 * a.width;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (GROUPS == 1) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int t = 0; t < VEC; ++t)
                    if (t >= at.skip[j]) mine[which * a.width + at.first[j] + t] = which ? db[j][t] : dw[j][t];
            continue;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int t = 0; t < VEC; ++t)
                if (t >= at.skip[j]) all[group * COLUMNS + at.first[j] + t] = which ? db[j][t] : dw[j][t];
        __syncthreads();
        for (int c = threadIdx.x; c < a.width; c += LAYER_THREADS) {
            float s = 0.0f;
            for (int g = 0; g < GROUPS; ++g) s += all[g * COLUMNS + c];
            mine[which * a.width + c] = s;
        }
    }
}

// out[0][c] and out[1][c] = the sums of partial[.][0][c] and partial[.][1][c].
constexpr int SUM_COLUMNS = 32, SUM_SLICES = 32;

__global__ __launch_bounds__(SUM_COLUMNS * SUM_SLICES) void column_sum_kernel(const float *__restrict__ partial, int parts, int width, float *dw, float *db)
{
    __shared__ float sums[SUM_SLICES][SUM_COLUMNS];
    const int c = blockIdx.x * SUM_COLUMNS + threadIdx.x % SUM_COLUMNS, slice = threadIdx.x / SUM_COLUMNS;
    float s = 0.0f;
    if (c < 2 * width)
#pragma unroll 8
        for (int p = slice; p < parts; p += SUM_SLICES) s += partial[(int64_t)p * 2 * width + c];
    sums[slice][threadIdx.x % SUM_COLUMNS] = s;
    __syncthreads();
    if (slice == 0 && c < 2 * width) {
        for (int k = 1; k < SUM_SLICES; ++k) s += sums[k][threadIdx.x];
        if (c < width) dw[c] = s; else db[c - width] = s;
    }
}

template <bool GRAD, typename T, int VEC, int LANES, int NV>
void launch_norm(const mf_ctx *ctx, const NormArgs &a, int grid)
{
    if (GRAD) hipLaunchKernelGGL((norm_grad_kernel<T, VEC, LANES, NV>), dim3(grid), dim3(LAYER_THREADS), 0, ctx->stream, a);
    else hipLaunchKernelGGL((norm_kernel<T, VEC, LANES, NV>), dim3(grid), dim3(LAYER_THREADS), 0, ctx->stream, a);
}

int least(int64_t a, int64_t b) { return (int)(a < b ? a : b); }

// Workgroups of the gradient: rows enough for each that the sums they leave are a small part of what they read, and four to a compute
// unit, as many as registers let in.
int norm_grad_parts(const mf_ctx *ctx, int64_t rows, int64_t width)
{
    const int64_t each = width >= 256 ? 8 : width <= 8 ? 256 : 2048 / width;
    return least((rows + each - 1) / each, 4ll * (ctx->n_cus > 0 ? ctx->n_cus : 256));
}

// As few lanes a row as hold it in one vector each, so that narrow rows share a wavefront; then more vectors a lane, and beyond
// 64 lanes x 4 vectors (2 of a 16-bit type) a whole workgroup.  Rows narrower than one vector go value by value.
template <bool GRAD, typename T>
void launch_norm_for(const mf_ctx *ctx, const NormArgs &a)
{
    constexpr int V = 16 / sizeof(T), WIDE = sizeof(T) == 4 ? 4 : 2;
    const int vectors = (a.width + V - 1) / V, units = ctx->n_cus > 0 ? ctx->n_cus : 256;
    const int parts = GRAD ? norm_grad_parts(ctx, a.rows, a.width) : 0;
    const auto grid = [&](int lanes) {
        const int64_t needed = (a.rows + LAYER_THREADS / lanes - 1) / (LAYER_THREADS / lanes);
        return GRAD ? parts : least(needed, (int64_t)units * 8);
    };
#define MF_NORM(VEC, LANES, NV) return launch_norm<GRAD, T, VEC, LANES, NV>(ctx, a, grid(LANES))
    if (a.width < V) MF_NORM(1, 8, 1);
    if (vectors <= 4) MF_NORM(V, 4, 1);
    if (vectors <= 8) MF_NORM(V, 8, 1);
    if (vectors <= 16) MF_NORM(V, 16, 1);
    if (vectors <= 32) MF_NORM(V, 32, 1);
    if (vectors <= 64) MF_NORM(V, 64, 1);
    if (vectors <= 128) MF_NORM(V, 64, 2);
    if (WIDE == 4 && vectors <= 256) MF_NORM(V, 64, WIDE);
    if (vectors <= 512) MF_NORM(V, 256, 2);
    if (vectors <= 1024) MF_NORM(V, 256, 4);
    if constexpr (WIDE == 4) MF_NORM(V, 256, 8);
#undef MF_NORM
}

template <bool GRAD>
void launch_norm_type(const mf_ctx *ctx, int type, const NormArgs &a)
{
    if (type == MF_F32) launch_norm_for<GRAD, float>(ctx, a);
    else if (type == MF_F16) launch_norm_for<GRAD, _Float16>(ctx, a);
    else launch_norm_for<GRAD, __bf16>(ctx, a);
}

struct DropArgs {
    const void *x;
    void *y;
    int64_t total, ldx, ldy;
    int width;
    DropRule rule;
    const unsigned long long *step;                         // where it is kept on the device (else null)
    unsigned layer;
};

// A thread takes the eight elements of a counter.  APART: rows lie apart in x or y, so an element's place needs its row;
// eight elements that lie in one row are still loaded together.
template <typename T, bool APART>
__global__ __launch_bounds__(LAYER_THREADS) void dropout_kernel(const DropArgs a)
{
    DropRule rule = a.rule;
    if (a.step) { const unsigned long long s = *a.step; rule.s0 = (unsigned)s; rule.s1 = (unsigned)(s >> 32); }
    const int64_t groups = (a.total + 7) / 8;
    for (int64_t g = (int64_t)blockIdx.x * LAYER_THREADS + threadIdx.x; g < groups; g += (int64_t)gridDim.x * LAYER_THREADS) {
        const int64_t first = g * 8;
        int64_t row = 0, col = first;
        if (APART) {
            row = (int64_t)((double)first / (double)a.width);       // first < 2^48: off by one at most
            col = first - row * a.width;
            if (col < 0) { --row; col += a.width; }
            else if (col >= a.width) { ++row; col -= a.width; }
        }
        const T *x = (const T *)a.x + row * a.ldx + col;
        T *y = (T *)a.y + row * a.ldy + col;
        const bool together = first + 8 <= a.total && (!APART || col + 8 <= a.width);
        float v[8];
        if (together) load_floats(v, x);
        const Words4 bits = drop_bits(rule, (uint64_t)g, a.layer);
        if (together) {
#pragma unroll
            for (int t = 0; t < 8; ++t) v[t] = drop_keeps(rule, bits, t) ? v[t] * rule.factor : 0.0f;
            store_floats(y, v);
        } else {
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                if (first + t >= a.total) break;
                const float u = (float)*x;
                *y = (T)(drop_keeps(rule, bits, t) ? u * rule.factor : 0.0f);
                ++x; ++y;
                if (APART && ++col == a.width) { col = 0; x += a.ldx - a.width; y += a.ldy - a.width; }
            }
        }
    }
}

template <typename T>
void launch_dropout(const mf_ctx *ctx, const DropArgs &a, bool apart)
{
    const int64_t needed = ((a.total + 7) / 8 + LAYER_THREADS - 1) / LAYER_THREADS;
    const int grid = least(needed, 1 << 20);
    if (apart) hipLaunchKernelGGL((dropout_kernel<T, true>), dim3(grid), dim3(LAYER_THREADS), 0, ctx->stream, a);
    else hipLaunchKernelGGL((dropout_kernel<T, false>), dim3(grid), dim3(LAYER_THREADS), 0, ctx->stream, a);
}

int check_rows(const mf_ctx *ctx, int type, int64_t rows, int64_t width)
{
    if (!ctx || type < MF_F32 || type > MF_BF16 || rows < 0 || width < 1) return MF_ERR_ARG;
    if (width > LAYER_MAX_WIDTH || rows > (1ll << 48) / width) return MF_ERR_SHAPE;
    return MF_OK;
}
bool whole_values(const void *p, int type) { return ((uintptr_t)p & (type == MF_F32 ? 3u : 1u)) == 0; }
bool good_rows(const void *p, int type, int64_t rows, int64_t width, int64_t ld)
{
    return p && whole_values(p, type) && ld >= width && (rows < 2 || ld <= (1ll << 50) / rows);
}
// What is written in the place of what is read has to have its pitch.
bool same_place(const void *from, int64_t ld, const void *to, int64_t ldo, int64_t rows) { return from != to || ld == ldo || rows < 2; }

}  // namespace

bool mf_drop_rule(const mf_dropout_rule *given, DropRule *rule)
{
    if (!(given->p >= 0.0f) || !(given->p < 1.0f)) return false;
    const uint32_t limit = drop_limit((double)given->p);
    if (limit >= 65536u || ((uintptr_t)given->d_step & 7u)) return false;
    *rule = DropRule{(uint32_t)given->seed, (uint32_t)(given->seed >> 32), (uint32_t)given->step, (uint32_t)(given->step >> 32),
                     limit, (float)(65536.0 / (double)(65536u - limit))};
    return true;
}

extern "C" {

int mf_layer_norm(mf_ctx *ctx, int type, const void *d_x, int64_t rows, int64_t width, int64_t ldx,
                  const float *d_w, const float *d_b, float eps, void *d_y, int64_t ldy)
{
    const int rc = check_rows(ctx, type, rows, width);
    if (rc != MF_OK) return rc;
    if (!d_w || !d_b || !(eps > 0.0f) || isinf(eps) || !whole_values(d_w, MF_F32) || !whole_values(d_b, MF_F32)) return MF_ERR_ARG;
    if (rows == 0) return MF_OK;
    if (!good_rows(d_x, type, rows, width, ldx) || !good_rows(d_y, type, rows, width, ldy) || !same_place(d_x, ldx, d_y, ldy, rows)) return MF_ERR_ARG;
    MF_HIP(hipSetDevice(ctx->device));
    NormArgs a{};
    a.x = d_x; a.out = d_y;
    a.rows = rows; a.ldx = ldx; a.ldo = ldy; a.width = (int)width;
    a.w = d_w; a.b = d_b; a.eps = eps;
    launch_norm_type<false>(ctx, type, a);
    MF_HIP(hipGetLastError());
    return MF_OK;
}

int64_t mf_layer_norm_grad_work(mf_ctx *ctx, int64_t rows, int64_t width)
{
    const int rc = check_rows(ctx, MF_F32, rows, width);
    return rc != MF_OK ? rc : (int64_t)norm_grad_parts(ctx, rows, width) * 2 * width * (int64_t)sizeof(float);
}

int mf_layer_norm_grad(mf_ctx *ctx, int type, const void *d_x, int64_t rows, int64_t width, int64_t ldx,
                       const void *d_dy, int64_t lddy, const float *d_w, float eps, void *d_dx, int64_t lddx,
                       float *d_dw, float *d_db, void *d_work, int64_t work_bytes)
{
    const int rc = check_rows(ctx, type, rows, width);
    if (rc != MF_OK) return rc;
    if (!d_w || !d_dw || !d_db || !(eps > 0.0f) || isinf(eps)) return MF_ERR_ARG;
    if (!whole_values(d_w, MF_F32) || !whole_values(d_dw, MF_F32) || !whole_values(d_db, MF_F32)) return MF_ERR_ARG;
    if (rows > 0) {
        if (!good_rows(d_x, type, rows, width, ldx) || !good_rows(d_dy, type, rows, width, lddy) || !good_rows(d_dx, type, rows, width, lddx)) return MF_ERR_ARG;
        if (!same_place(d_x, ldx, d_dx, lddx, rows) || !same_place(d_dy, lddy, d_dx, lddx, rows)) return MF_ERR_ARG;
        if (!d_work || ((uintptr_t)d_work & 15u) || work_bytes < mf_layer_norm_grad_work(ctx, rows, width)) return MF_ERR_ARG;
    }
    MF_HIP(hipSetDevice(ctx->device));
    NormArgs a{};
    a.x = d_x; a.dy = d_dy; a.out = d_dx;
    a.rows = rows; a.ldx = ldx; a.lddy = lddy; a.ldo = lddx; a.width = (int)width;
    a.w = d_w; a.eps = eps;
    a.partial = (float *)d_work;
    if (rows > 0) launch_norm_type<true>(ctx, type, a);
    hipLaunchKernelGGL(column_sum_kernel, dim3((unsigned)((2 * width + SUM_COLUMNS - 1) / SUM_COLUMNS)), dim3(SUM_COLUMNS * SUM_SLICES), 0, ctx->stream,
                       a.partial, rows > 0 ? norm_grad_parts(ctx, rows, width) : 0, (int)width, d_dw, d_db);
    MF_HIP(hipGetLastError());
    return MF_OK;
}

int mf_dropout(mf_ctx *ctx, int type, const void *d_x, int64_t rows, int64_t width, int64_t ldx,
               const mf_dropout_rule *rule, int layer, void *d_y, int64_t ldy)
{
    const int rc = check_rows(ctx, type, rows, width);
    if (rc != MF_OK) return rc;
    DropArgs a{};
    if (!rule || !mf_drop_rule(rule, &a.rule) || layer < 0 || layer > 65535) return MF_ERR_ARG;
    if (rows == 0) return MF_OK;
    if (!good_rows(d_x, type, rows, width, ldx) || !good_rows(d_y, type, rows, width, ldy) || !same_place(d_x, ldx, d_y, ldy, rows)) return MF_ERR_ARG;
    MF_HIP(hipSetDevice(ctx->device));
    a.x = d_x; a.y = d_y;
    a.total = rows * width; a.ldx = ldx; a.ldy = ldy; a.width = (int)width;
    a.step = (const unsigned long long *)rule->d_step;
    a.layer = (unsigned)layer;
    const bool apart = rows > 1 && (ldx != width || ldy != width);
    if (type == MF_F32) launch_dropout<float>(ctx, a, apart);
    else if (type == MF_F16) launch_dropout<_Float16>(ctx, a, apart);
    else launch_dropout<__bf16>(ctx, a, apart);
    MF_HIP(hipGetLastError());
    return MF_OK;
}

}  // extern "C"
