// Gated recurrence along lines and its Jacobian: h_t = f_t h_(t-1) + (1 - f_t) x_t with f = logistic(z).
#include "znn_internal.h"

#include <algorithm>

namespace znn {
namespace {

// f = 1 / (1 + exp(-z)) and k = 1 - f = 1 / (1 + exp(z)), each to its own last digits: 1 - f would have lost those of a gate that is nearly open.
struct Gate { float f, k; };
__device__ __forceinline__ Gate gate(float z)
{
    const float e = expf(-fabsf(z)), large = 1.f / (1.f + e), small = e * large;
    return z < 0.f ? Gate{small, large} : Gate{large, small};
}
// A factor of 0 takes nothing, not even an infinity: that is how a sequence ends and how padding is passed over.
__device__ __forceinline__ float times(float a, float v) { return a == 0.f ? 0.f : a * v; }

struct Lines {
    long outer, length, inner;
    int reverse;
};
struct LinesFwd { Lines L; const float *z, *x, *h0; float* h; };
struct LinesBwd { Lines L; const float *gh, *z, *x, *h, *h0; float *gz, *gx, *gh0; };

// One thread a line.
__global__ void __launch_bounds__(256) k_lines_fwd(LinesFwd A)
{
    const long lines = A.L.outer * A.L.inner, step = A.L.reverse ? -A.L.inner : A.L.inner;
    for (long l = blockIdx.x * 256L + threadIdx.x; l < lines; l += gridDim.x * 256L) {
        const long o = l / A.L.inner, i = l - o * A.L.inner;
        long at = (o * A.L.length + (A.L.reverse ? A.L.length - 1 : 0)) * A.L.inner + i;
        float h = A.h0 ? A.h0[l] : 0.f;
        for (long t = 0; t < A.L.length; ++t, at += step) {
            const Gate g = gate(A.z[at]);
            h = times(g.f, h) + times(g.k, A.x[at]);
            A.h[at] = h;
        }
    }
}

// What flows backwards is q_t = f_t G_t, G_t = gh_t + q_(t+1): the factors of a step are its own.
__global__ void __launch_bounds__(256) k_lines_bwd(LinesBwd A)
{
    const long lines = A.L.outer * A.L.inner, step = A.L.reverse ? -A.L.inner : A.L.inner;
    for (long l = blockIdx.x * 256L + threadIdx.x; l < lines; l += gridDim.x * 256L) {
        const long o = l / A.L.inner, i = l - o * A.L.inner;
        long at = (o * A.L.length + (A.L.reverse ? 0 : A.L.length - 1)) * A.L.inner + i;
        float q = 0.f;
        for (long t = A.L.length - 1; t >= 0; --t, at -= step) {
            const Gate g = gate(A.z[at]);
            const float G = A.gh[at] + q, before = t > 0 ? A.h[at - step] : A.h0 ? A.h0[l] : 0.f;
            A.gx[at] = times(g.k, G);
            A.gz[at] = g.f == 0.f || g.k == 0.f ? 0.f : G * (before - A.x[at]) * (g.f * g.k);
            q = times(g.f, G);
        }
        if (A.gh0) A.gh0[l] = q;
    }
}

int check_lines(int64_t outer, int64_t length, int64_t inner)
{
    if (outer < 1 || length < 1 || inner < 1) return fail(ZNN_EINVAL, "extents must be >= 1");
    constexpr int64_t most = 1LL << 34;
    if (outer > most || length > most || inner > most || (double)outer * length * inner > 1099511627776.0)
        return fail(ZNN_EUNSUPPORTED, "lines of %lld x %lld x %lld elements are too large", (long long)outer, (long long)length, (long long)inner);
    return ZNN_OK;
}

size_t lines_workspace(const Lines&) { return 0; }

int check_lines_workspace(const Lines& L, const void* ws, size_t ws_bytes)
{
    const size_t need = lines_workspace(L);
    if (!need) return ZNN_OK;
    if (!ws) return fail(ZNN_EWORKSPACE, "workspace is NULL but %zu bytes are needed", need);
    if ((uintptr_t)ws & 255) return fail(ZNN_EWORKSPACE, "workspace is not 256-byte aligned");
    if (ws_bytes < need) return fail(ZNN_EWORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
    return ZNN_OK;
}

}  // namespace
}  // namespace znn

using namespace znn;

extern "C" {

int znn_recurrence_workspace_bytes(int64_t outer, int64_t length, int64_t inner, size_t* bytes)
{
    int rc = check_lines(outer, length, inner);
    if (rc != ZNN_OK) return rc;
    if (!bytes) return fail(ZNN_EINVAL, "NULL argument");
    *bytes = lines_workspace(Lines{(long)outer, (long)length, (long)inner, 0});
    return ZNN_OK;
}

int znn_recurrence_fwd(int64_t outer, int64_t length, int64_t inner, int32_t reverse, const float* z, const float* x, const float* h0,
                       float* h, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_lines(outer, length, inner);
    if (rc != ZNN_OK) return rc;
    if (!z || !x || !h) return fail(ZNN_EINVAL, "NULL argument");
    const LinesFwd A = {{(long)outer, (long)length, (long)inner, reverse != 0}, z, x, h0, h};
    rc = check_lines_workspace(A.L, ws, ws_bytes);
    if (rc != ZNN_OK) return rc;
    const hipStream_t s = (hipStream_t)stream;
    ZNN_LAUNCH("recurrence forward", s, k_lines_fwd, dim3((unsigned)std::min((outer * inner + 255) / 256, (int64_t)1 << 20)), dim3(256), 0, A);
    return check_launch("recurrence forward");
}

int znn_recurrence_bwd(int64_t outer, int64_t length, int64_t inner, int32_t reverse, const float* gh, const float* z, const float* x,
                       const float* h, const float* h0, float* gz, float* gx, float* gh0, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_lines(outer, length, inner);
    if (rc != ZNN_OK) return rc;
    if (!gh || !z || !x || !h || !gz || !gx) return fail(ZNN_EINVAL, "NULL argument");
    const LinesBwd A = {{(long)outer, (long)length, (long)inner, reverse != 0}, gh, z, x, h, h0, gz, gx, gh0};
    rc = check_lines_workspace(A.L, ws, ws_bytes);
    if (rc != ZNN_OK) return rc;
    const hipStream_t s = (hipStream_t)stream;
    ZNN_LAUNCH("recurrence backward", s, k_lines_bwd, dim3((unsigned)std::min((outer * inner + 255) / 256, (int64_t)1 << 20)), dim3(256), 0, A);
    return check_launch("recurrence backward");
}

}  // extern "C"
