// Dropout, layer norm and the residual join (dropout, node sum and layer norm in one pass), forward and backward.
//
// Operands are dense [rows][cols] arrays.  Axis 0 normalises every column over the rows (images: each voxel over the maps),
// axis 1 every row over its columns.  With n elements in a position (a column or a row):
//     m = sum x / n,  s = 1 / sqrt(sum (x - m)^2 / n + eps),  h = (x - m) s,  y = w h + b
//     a = w gy,  gx = s (a - mean(a) - h mean(a h)),  gw = sum over positions of gy h,  gb = sum of gy
// Sums are held in 32 bits.  The sum of squares is taken about a first mean m0 and corrected by what is left of the sum there
// (d = x - m0, m = m0 + mean(d), variance mean(d^2) - mean(d)^2), so neither a mean far from zero nor m0's rounding costs digits.
#include <algorithm>
#include <cmath>

#include "random.h"
#include "znn_internal.h"

namespace znn {

int make_drop(double p, const uint64_t* state, uint32_t site, Drop* drop, bool* drops)
{
    if (!(p >= 0.0 && p <= 1.0)) return fail(ZNN_EINVAL, "the probability to drop must lie in [0, 1]");
    const double keep = 4294967296.0 - std::floor(p * 4294967296.0 + 0.5);
    *drops = keep < 4294967296.0;
    *drop = Drop{state, site, *drops ? (unsigned)keep : 0u, keep > 0.0 ? (float)(4294967296.0 / keep) : 0.f};
    if (*drops && !state) return fail(ZNN_EINVAL, "dropout needs a random state");
    if (*drops && ((uintptr_t)state & 7)) return fail(ZNN_EINVAL, "the random state is not 8-byte aligned");
    return ZNN_OK;
}

namespace {

// ---------------------------------------------------------------- dropout
__global__ void __launch_bounds__(256)
k_dropout(long rows, long cols, long quads, Drop D, const float* __restrict__ x, float* __restrict__ y)
{
    const DropKey K = drop_key(D);
    for (long t = (long)blockIdx.x * 256 + threadIdx.x; t < rows * quads; t += (long)gridDim.x * 256) {
        const long row = t / quads, q = t - row * quads, at = row * cols + 4 * q;
        const int count = (int)min(4L, cols - 4 * q);
        store4(y + at, count, dropped4(K, (unsigned)q, (unsigned)row, load4(x + at, count)));
    }
}

__global__ void __launch_bounds__(256) k_copy(long count, const float* __restrict__ x, float* __restrict__ y)
{
    for (long t = (long)blockIdx.x * 256 + threadIdx.x; t < count; t += (long)gridDim.x * 256) y[t] = x[t];
}

__global__ void k_random_advance(uint64_t* state) { state[1] += 1; }

// ---------------------------------------------------------------- layer norm
enum { PLAIN = 0, JOIN = 1, JOIN_DROP = 2 };        // x alone; x + h; x + dropout(h)

struct NormFwd {
    long rows, cols;
    const float *h, *x, *w, *b;     // h: joins only
    float *r, *y, *stats;           // r: joins only; stats may be NULL
    float eps;
    Drop drop;
};
struct NormBwd {
    long rows, cols;
    const float *gy, *gr, *x, *w, *stats;       // gr may be NULL
    float *gx, *gh;                             // gh may be NULL
    Drop drop;
};

// x + h: the sum of the rounded product, as dropout and a node sum give it one after another
__device__ __forceinline__ float joined(float x, float h)
{
#pragma clang fp contract(off)
    return x + h;
}

// From the mean of (x - m0)^2 and the mean of x - m0.  A variance that rounding left below zero is zero; one that is beyond 32 bits
// stays infinite (where the correction may be infinite too), one that is not a number stays that.
__device__ __forceinline__ float inverse_deviation(float square, float delta, float eps)
{
    const float v = square < INFINITY ? square - delta * delta : square;
    return 1.0f / sqrtf((v < 0.f ? 0.f : v) + eps);
}

// Sums of two values over a workgroup, for all its threads.
template <int WAVES>
__device__ __forceinline__ float2 group_sum(float a, float b, float2* red)
{
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) { a += __shfl_xor(a, s); b += __shfl_xor(b, s); }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    float2 v = red[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) { v.x += red[i].x; v.y += red[i].y; }
    return v;
}

// Rows of any length: a workgroup walks a row three times.
template <int MODE>
__global__ void __launch_bounds__(1024) k_norm_rows_any(NormFwd A)
{
    __shared__ float2 red[16];
    DropKey K = {};
    if (MODE == JOIN_DROP) K = drop_key(A.drop);
    const long quads = (A.cols + 3) / 4;
    const float inv = 1.0f / (float)A.cols;
    for (long row = blockIdx.x; row < A.rows; row += gridDim.x) {
        const long base = row * A.cols;
        const float* src = MODE == PLAIN ? A.x : A.r;
        float sum = 0.f;
        for (long q = threadIdx.x; q < quads; q += 1024) {
            const int count = (int)min(4L, A.cols - 4 * q);
            floatu4 v = load4(A.x + base + 4 * q, count);
            if (MODE != PLAIN) {
                floatu4 h = load4(A.h + base + 4 * q, count);
                if (MODE == JOIN_DROP) h = dropped4(K, (unsigned)q, (unsigned)row, h);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = joined(v[e], h[e]);
                store4(A.r + base + 4 * q, count, v);
            }
            sum += (v[0] + v[1]) + (v[2] + v[3]);       // 0 behind the row
        }
        const float m0 = group_sum<16>(sum, 0.f, red).x * inv;
        float d1 = 0.f, d2 = 0.f;
        for (long q = threadIdx.x; q < quads; q += 1024) {
            const int count = (int)min(4L, A.cols - 4 * q);
            const floatu4 v = load4(src + base + 4 * q, count);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < count) { const float d = v[e] - m0; d1 += d; d2 += d * d; }
        }
        const float2 s = group_sum<16>(d1, d2, red);
        const float delta = s.x * inv, rstd = inverse_deviation(s.y * inv, delta, A.eps);
        for (long q = threadIdx.x; q < quads; q += 1024) {
            const int count = (int)min(4L, A.cols - 4 * q);
            floatu4 v = load4(src + base + 4 * q, count);
            const floatu4 w = load4(A.w + 4 * q, count), b = load4(A.b + 4 * q, count);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = ((v[e] - m0) - delta) * rstd * w[e] + b[e];
            store4(A.y + base + 4 * q, count, v);
        }
        if (A.stats && threadIdx.x == 0) { A.stats[row] = m0 + delta; A.stats[A.rows + row] = rstd; }
    }
}

template <int MODE>
__global__ void __launch_bounds__(1024) k_norm_rows_bwd_any(NormBwd A)
{
    __shared__ float2 red[16];
    DropKey K = {};
    if (MODE == JOIN_DROP) K = drop_key(A.drop);
    const long quads = (A.cols + 3) / 4;
    const float inv = 1.0f / (float)A.cols;
    for (long row = blockIdx.x; row < A.rows; row += gridDim.x) {
        const long base = row * A.cols;
        const float mean = A.stats[row], rstd = A.stats[A.rows + row];
        float s1 = 0.f, s2 = 0.f;
        for (long q = threadIdx.x; q < quads; q += 1024) {
            const int count = (int)min(4L, A.cols - 4 * q);
            const floatu4 x = load4(A.x + base + 4 * q, count), g = load4(A.gy + base + 4 * q, count), w = load4(A.w + 4 * q, count);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < count) { const float a = g[e] * w[e]; s1 += a; s2 += a * ((x[e] - mean) * rstd); }
        }
        const float2 s = group_sum<16>(s1, s2, red);
        const float m1 = s.x * inv, m2 = s.y * inv;
        for (long q = threadIdx.x; q < quads; q += 1024) {
            const int count = (int)min(4L, A.cols - 4 * q);
            const floatu4 x = load4(A.x + base + 4 * q, count), g = load4(A.gy + base + 4 * q, count), w = load4(A.w + 4 * q, count);
            floatu4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = rstd * (g[e] * w[e] - m1 - (x[e] - mean) * rstd * m2);
            if (MODE != PLAIN && A.gr) {
                const floatu4 r = load4(A.gr + base + 4 * q, count);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += r[e];
            }
            store4(A.gx + base + 4 * q, count, v);
            if (MODE == JOIN_DROP) v = dropped4(K, (unsigned)q, (unsigned)row, v);
            if (MODE != PLAIN && A.gh) store4(A.gh + base + 4 * q, count, v);
        }
    }
}

// Columns of any height: 64 columns by four slices of the rows, which a workgroup walks three times.
__device__ __forceinline__ float2 slices_sum(float a, float b, float2 (*red)[64])
{
    const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
    __syncthreads();
    red[ty][tx] = make_float2(a, b);
    __syncthreads();
    const float2 v0 = red[0][tx], v1 = red[1][tx], v2 = red[2][tx], v3 = red[3][tx];
    return make_float2((v0.x + v1.x) + (v2.x + v3.x), (v0.y + v1.y) + (v2.y + v3.y));
}

template <int MODE>
__global__ void __launch_bounds__(256) k_norm_cols_any(NormFwd A)
{
    __shared__ float2 red[4][64];
    DropKey K = {};
    if (MODE == JOIN_DROP) K = drop_key(A.drop);
    const int ty = threadIdx.x >> 6;
    const float inv = 1.0f / (float)A.rows;
    for (long c0 = (long)blockIdx.x * 64; c0 < A.cols; c0 += (long)gridDim.x * 64) {
        const long c = c0 + (threadIdx.x & 63);
        const long mine = c < A.cols ? A.rows : 0;       // rows that this thread's column has
        const float* src = MODE == PLAIN ? A.x : A.r;
        float sum = 0.f;
        for (long m = ty; m < mine; m += 4) {
            const long t = m * A.cols + c;
            float v = A.x[t];
            if (MODE != PLAIN) {
                float h = A.h[t];
                if (MODE == JOIN_DROP) {
                    const Words u = drop_words(K, (unsigned)(c >> 2), (unsigned)m);
                    const int e = (int)(c & 3);
                    h = dropped(K, e == 0 ? u.w[0] : e == 1 ? u.w[1] : e == 2 ? u.w[2] : u.w[3], h);
                }
                v = joined(v, h);
                A.r[t] = v;
            }
            sum += v;
        }
        const float m0 = slices_sum(sum, 0.f, red).x * inv;
        float d1 = 0.f, d2 = 0.f;
        for (long m = ty; m < mine; m += 4) { const float d = src[m * A.cols + c] - m0; d1 += d; d2 += d * d; }
        const float2 s = slices_sum(d1, d2, red);
        const float delta = s.x * inv, rstd = inverse_deviation(s.y * inv, delta, A.eps);
        for (long m = ty; m < mine; m += 4)
            A.y[m * A.cols + c] = ((src[m * A.cols + c] - m0) - delta) * rstd * A.w[m] + A.b[m];
        if (A.stats && mine && ty == 0) { A.stats[c] = m0 + delta; A.stats[A.cols + c] = rstd; }
    }
}

template <int MODE>
__global__ void __launch_bounds__(256) k_norm_cols_bwd_any(NormBwd A)
{
    __shared__ float2 red[4][64];
    DropKey K = {};
    if (MODE == JOIN_DROP) K = drop_key(A.drop);
    const int ty = threadIdx.x >> 6;
    const float inv = 1.0f / (float)A.rows;
    for (long c0 = (long)blockIdx.x * 64; c0 < A.cols; c0 += (long)gridDim.x * 64) {
        const long c = c0 + (threadIdx.x & 63);
        const long mine = c < A.cols ? A.rows : 0;
        const float mean = mine ? A.stats[c] : 0.f, rstd = mine ? A.stats[A.cols + c] : 0.f;
        float s1 = 0.f, s2 = 0.f;
        for (long m = ty; m < mine; m += 4) {
            const float a = A.gy[m * A.cols + c] * A.w[m];
            s1 += a;
            s2 += a * ((A.x[m * A.cols + c] - mean) * rstd);
        }
        const float2 s = slices_sum(s1, s2, red);
        const float m1 = s.x * inv, m2 = s.y * inv;
        for (long m = ty; m < mine; m += 4) {
            const long t = m * A.cols + c;
            float v = rstd * (A.gy[t] * A.w[m] - m1 - (A.x[t] - mean) * rstd * m2);
            if (MODE != PLAIN && A.gr) v += A.gr[t];
            A.gx[t] = v;
            if (MODE == JOIN_DROP) {
                const Words u = drop_words(K, (unsigned)(c >> 2), (unsigned)m);
                const int e = (int)(c & 3);
                v = dropped(K, e == 0 ? u.w[0] : e == 1 ? u.w[1] : e == 2 ? u.w[2] : u.w[3], v);
            }
            if (MODE != PLAIN && A.gh) A.gh[t] = v;
        }
    }
}

// ---------------------------------------------------------------- gradients of weight and bias
// Shares of the positions, [share][2][features], added in their order by k_norm_params.
struct NormParams {
    long rows, cols;
    const float *gy, *x, *stats;
    float* parts;
    int shares; long span;          // positions of a share
};

__global__ void __launch_bounds__(256) k_norm_params_rows(NormParams A)
{
    __shared__ float2 red[4][64];
    const long c = (long)blockIdx.x * 64 + (threadIdx.x & 63), r0 = blockIdx.y * A.span;
    const long end = c < A.cols ? min(A.rows, r0 + A.span) : 0;
    float gw = 0.f, gb = 0.f;
    for (long r = r0 + (threadIdx.x >> 6); r < end; r += 4) {
        const float g = A.gy[r * A.cols + c];
        gw += g * ((A.x[r * A.cols + c] - A.stats[r]) * A.stats[A.rows + r]);
        gb += g;
    }
    const float2 s = slices_sum(gw, gb, red);
    if (c < A.cols && threadIdx.x < 64) {
        float* part = A.parts + (long)blockIdx.y * 2 * A.cols;
        part[c] = s.x;
        part[A.cols + c] = s.y;
    }
}

__global__ void __launch_bounds__(256) k_norm_params_cols(NormParams A)
{
    __shared__ float2 red[4];
    const long c0 = blockIdx.y * A.span, end = min(A.cols, c0 + A.span);
    for (long m = blockIdx.x; m < A.rows; m += gridDim.x) {
        float gw = 0.f, gb = 0.f;
        for (long c = c0 + threadIdx.x; c < end; c += 256) {
            const float g = A.gy[m * A.cols + c];
            gw += g * ((A.x[m * A.cols + c] - A.stats[c]) * A.stats[A.cols + c]);
            gb += g;
        }
        const float2 s = group_sum<4>(gw, gb, red);
        if (threadIdx.x == 0) {
            float* part = A.parts + (long)blockIdx.y * 2 * A.rows;
            part[m] = s.x;
            part[A.rows + m] = s.y;
        }
    }
}

__global__ void __launch_bounds__(256)
k_norm_params(long features, int shares, const float* __restrict__ parts, float* __restrict__ gw, float* __restrict__ gb)
{
    const long t = (long)blockIdx.x * 256 + threadIdx.x;
    if (t >= 2 * features) return;
    float v = 0.f;
    for (int s = 0; s < shares; ++s) v += parts[(long)s * 2 * features + t];
    if (t < features) gw[t] = v; else gb[t - features] = v;
}

struct Shares { int count; long span; };
Shares param_shares(long rows, long cols, int axis)
{
    const long positions = axis ? rows : cols, features = axis ? cols : rows;
    const long least = axis ? 64 : 4096, groups = axis ? (features + 63) / 64 : features;
    const long want = std::max(1L, std::min((positions + least - 1) / least, std::max(1L, 2048 / groups)));
    const long span = (positions + want - 1) / want;
    return Shares{(int)((positions + span - 1) / span), span};
}

size_t norm_workspace(long rows, long cols, int axis)
{
    return sizeof(float) * 2 * param_shares(rows, cols, axis).count * (axis ? cols : rows);
}

unsigned groups_of(long work, long each, long most) { return (unsigned)std::min((work + each - 1) / each, most); }

// ---------------------------------------------------------------- checks and launches
int check_array(int64_t rows, int64_t cols)
{
    if (rows < 1 || cols < 1) return fail(ZNN_EINVAL, "rows and columns must be >= 1");
    // row and column / 4 are words of the generator's counter; a flat index has 63 bits
    if (rows > 4294967295LL || cols > 17179869184LL || (double)rows * cols >= 2305843009213693952.0)
        return fail(ZNN_EUNSUPPORTED, "an array of %lld x %lld elements is too large", (long long)rows, (long long)cols);
    return ZNN_OK;
}

int check_axis(int64_t rows, int64_t cols, int32_t axis)
{
    if (axis != 0 && axis != 1) return fail(ZNN_EINVAL, "axis must be 0 (over the rows) or 1 (over the columns)");
    int rc = check_array(rows, cols);
    if (rc == ZNN_OK && (axis ? cols : rows) > 268435456LL)
        rc = fail(ZNN_EUNSUPPORTED, "a norm over %lld elements is too large", (long long)(axis ? cols : rows));
    return rc;
}

template <int MODE>
int norm_fwd(const NormFwd& A, int axis, hipStream_t s)
{
    if (axis) ZNN_LAUNCH("layer norm forward", s, k_norm_rows_any<MODE>, dim3(groups_of(A.rows, 1, 1L << 20)), dim3(1024), 0, A);
    else ZNN_LAUNCH("layer norm forward", s, k_norm_cols_any<MODE>, dim3(groups_of(A.cols, 64, 1L << 20)), dim3(256), 0, A);
    return check_launch("layer norm forward");
}

template <int MODE>
int norm_bwd(const NormBwd& A, int axis, float* gw, float* gb, void* ws, hipStream_t s)
{
    const Shares S = param_shares(A.rows, A.cols, axis);
    const long features = axis ? A.cols : A.rows;
    const NormParams P = {A.rows, A.cols, A.gy, A.x, A.stats, (float*)ws, S.count, S.span};
    if (axis) {
        ZNN_LAUNCH("layer norm backward", s, k_norm_rows_bwd_any<MODE>, dim3(groups_of(A.rows, 1, 1L << 20)), dim3(1024), 0, A);
        ZNN_LAUNCH("layer norm parameters", s, k_norm_params_rows, dim3((unsigned)((A.cols + 63) / 64), (unsigned)S.count), dim3(256), 0, P);
    } else {
        ZNN_LAUNCH("layer norm backward", s, k_norm_cols_bwd_any<MODE>, dim3(groups_of(A.cols, 64, 1L << 20)), dim3(256), 0, A);
        ZNN_LAUNCH("layer norm parameters", s, k_norm_params_cols, dim3(groups_of(A.rows, 1, 1L << 20), (unsigned)S.count), dim3(256), 0, P);
    }
    ZNN_LAUNCH("layer norm parameters", s, k_norm_params, dim3((unsigned)((2 * features + 255) / 256)), dim3(256), 0, features, S.count,
               (const float*)ws, gw, gb);
    return check_launch("layer norm backward");
}

}  // namespace

}  // namespace znn

using namespace znn;

extern "C" {

int znn_random_advance(uint64_t* state, void* stream)
{
    if (!state) return fail(ZNN_EINVAL, "NULL argument");
    if ((uintptr_t)state & 7) return fail(ZNN_EINVAL, "the random state is not 8-byte aligned");
    ZNN_LAUNCH("random state", (hipStream_t)stream, k_random_advance, dim3(1), dim3(1), 0, state);
    return check_launch("random state");
}

int znn_dropout(int64_t rows, int64_t cols, double p, const uint64_t* state, uint32_t site, const float* x, float* y, void* stream)
{
    int rc = check_array(rows, cols);
    if (rc != ZNN_OK) return rc;
    if (!x || !y) return fail(ZNN_EINVAL, "NULL argument");
    Drop D;
    bool drops;
    rc = make_drop(p, state, site, &D, &drops);
    if (rc != ZNN_OK) return rc;
    const hipStream_t s = (hipStream_t)stream;
    const long quads = (cols + 3) / 4;
    if (drops) ZNN_LAUNCH("dropout", s, k_dropout, dim3(groups_of(rows * quads, 256, 1L << 20)), dim3(256), 0, (long)rows, (long)cols, quads, D, x, y);
    else ZNN_LAUNCH("dropout", s, k_copy, dim3(groups_of(rows * cols, 256, 1L << 20)), dim3(256), 0, (long)(rows * cols), x, y);
    return check_launch("dropout");
}

int znn_layernorm_workspace_bytes(int64_t rows, int64_t cols, int32_t axis, size_t* bytes)
{
    int rc = check_axis(rows, cols, axis);
    if (rc != ZNN_OK) return rc;
    if (!bytes) return fail(ZNN_EINVAL, "NULL argument");
    *bytes = norm_workspace(rows, cols, axis);
    return ZNN_OK;
}

static int check_norm(int64_t rows, int64_t cols, int32_t axis, float eps)
{
    int rc = check_axis(rows, cols, axis);
    if (rc != ZNN_OK) return rc;
    if (!(eps > 0.f && eps <= 3.402823466e38f)) return fail(ZNN_EINVAL, "eps must be positive and finite");
    return ZNN_OK;
}

static int check_norm_workspace(int64_t rows, int64_t cols, int32_t axis, const void* ws, size_t ws_bytes)
{
    const size_t need = norm_workspace(rows, cols, axis);
    if (!need) return ZNN_OK;
    if (!ws) return fail(ZNN_EWORKSPACE, "workspace is NULL but %zu bytes are needed", need);
    if ((uintptr_t)ws & 255) return fail(ZNN_EWORKSPACE, "workspace is not 256-byte aligned");
    if (ws_bytes < need) return fail(ZNN_EWORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
    return ZNN_OK;
}

int znn_layernorm_fwd(int64_t rows, int64_t cols, int32_t axis, float eps, const float* x, const float* w, const float* b,
                      float* y, float* stats, void* stream)
{
    int rc = check_norm(rows, cols, axis, eps);
    if (rc != ZNN_OK) return rc;
    if (!x || !w || !b || !y) return fail(ZNN_EINVAL, "NULL argument");
    const NormFwd A = {(long)rows, (long)cols, nullptr, x, w, b, nullptr, y, stats, eps, Drop{}};
    return norm_fwd<PLAIN>(A, axis, (hipStream_t)stream);
}

int znn_layernorm_bwd(int64_t rows, int64_t cols, int32_t axis, const float* gy, const float* x, const float* w, const float* stats,
                      float* gx, float* gw, float* gb, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_axis(rows, cols, axis);
    if (rc != ZNN_OK) return rc;
    if (!gy || !x || !w || !stats || !gx || !gw || !gb) return fail(ZNN_EINVAL, "NULL argument");
    rc = check_norm_workspace(rows, cols, axis, ws, ws_bytes);
    if (rc != ZNN_OK) return rc;
    const NormBwd A = {(long)rows, (long)cols, gy, nullptr, x, w, stats, gx, nullptr, Drop{}};
    return norm_bwd<PLAIN>(A, axis, gw, gb, ws, (hipStream_t)stream);
}

int znn_residual_norm_fwd(int64_t rows, int64_t cols, int32_t axis, float eps, double p, const uint64_t* state, uint32_t site,
                          const float* h, const float* x, const float* w, const float* b, float* r, float* y, float* stats,
                          void* stream)
{
    int rc = check_norm(rows, cols, axis, eps);
    if (rc != ZNN_OK) return rc;
    if (!h || !x || !w || !b || !r || !y) return fail(ZNN_EINVAL, "NULL argument");
    Drop D;
    bool drops;
    rc = make_drop(p, state, site, &D, &drops);
    if (rc != ZNN_OK) return rc;
    const NormFwd A = {(long)rows, (long)cols, h, x, w, b, r, y, stats, eps, D};
    return drops ? norm_fwd<JOIN_DROP>(A, axis, (hipStream_t)stream) : norm_fwd<JOIN>(A, axis, (hipStream_t)stream);
}

int znn_residual_norm_bwd(int64_t rows, int64_t cols, int32_t axis, double p, const uint64_t* state, uint32_t site, const float* gy,
                          const float* gr, const float* r, const float* w, const float* stats, float* gx, float* gh, float* gw,
                          float* gb, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_axis(rows, cols, axis);
    if (rc != ZNN_OK) return rc;
    if (!gy || !r || !w || !stats || !gx || !gw || !gb) return fail(ZNN_EINVAL, "NULL argument");
    Drop D;
    bool drops;
    rc = make_drop(p, state, site, &D, &drops);
    if (rc != ZNN_OK) return rc;
    if (p > 0.0 && !gh) return fail(ZNN_EINVAL, "gh is NULL, which only a join that drops nothing may leave out");
    rc = check_norm_workspace(rows, cols, axis, ws, ws_bytes);
    if (rc != ZNN_OK) return rc;
    const NormBwd A = {(long)rows, (long)cols, gy, gr, r, w, stats, gx, gh, D};
    return drops ? norm_bwd<JOIN_DROP>(A, axis, gw, gb, ws, (hipStream_t)stream) : norm_bwd<JOIN>(A, axis, gw, gb, ws, (hipStream_t)stream);
}

}  // extern "C"
