// Gated unit y = fn(W x + b) (V x + c) and its Jacobian.
#include "znn_internal.h"

#include <algorithm>

namespace znn {
namespace {

struct Gated { float a, d; };       // fn(u) and its derivative

constexpr float kLargestFloat = 3.402823466e38f;

// fn by its number; every branch is uniform.  Values at infinity are limits: an infinite u times a factor of 0 would not be.
__device__ __forceinline__ Gated gate_fn(int fn, float u)
{
    if (fn == ZNN_GATE_RECTIFY) return Gated{u > 0.f ? u : 0.f, u > 0.f ? 1.f : 0.f};
    if (fn == ZNN_GATE_TANH) {
        const float t = tanhf(u), e = expf(-2.f * fabsf(u)), r = 1.f / (1.f + e);
        return Gated{t, 4.f * e * r * r};           // 1 - t^2 without its cancellation
    }
    const float finite = u > kLargestFloat ? kLargestFloat : u < -kLargestFloat ? -kLargestFloat : u;
    if (fn == ZNN_GATE_GELU) {
        const float p = 0.5f * erfcf(-0.707106781f * finite);
        return Gated{u > 0.f ? u * p : finite * p, fmaf(finite, 0.398942280f * expf(-0.5f * finite * finite), p)};
    }
    const float e = expf(-fabsf(u)), large = 1.f / (1.f + e), small = e * large;
    const float s = u < 0.f ? small : large, t = u < 0.f ? large : small;
    if (fn == ZNN_GATE_LOGISTIC) return Gated{s, s * t};
    return Gated{u > 0.f ? u * s : finite * s, fmaf(finite, s * t, s)};
}

// Strides of an array [features][positions]: images, or rows of features.
struct Place { long feature, position; };
Place place(int axis, long features, long positions) { return axis ? Place{1, features} : Place{positions, 1}; }

struct Operand { const float* p; long outer, k; };     // element (i, k) at p + i outer + k k
struct Product { Operand A, B; long M, N, K; };

constexpr int kTile = 64, kDepth = 16;
struct Tiles { float a[2][kDepth][kTile + 4], b[kDepth][kTile + 4]; };

__device__ __forceinline__ void stage(float (&t)[kDepth][kTile + 4], const Operand& O, long first, long rows, long k0, long K)
{
    for (int e = threadIdx.x; e < kTile * kDepth; e += 256) {
        const int r = O.k == 1 ? e / kDepth : e % kTile, k = O.k == 1 ? e % kDepth : e / kTile;
        t[k][r] = first + r < rows && k0 + k < K ? O.p[(first + r) * O.outer + (k0 + k) * O.k] : 0.f;
    }
}

template <int HALVES>
__device__ __forceinline__ void tile_product(Tiles& S, float (&acc)[HALVES][4][4], const Product& P, long half, long m0, long n0)
{
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (long k0 = 0; k0 < P.K; k0 += kDepth) {
        __syncthreads();
        for (int h = 0; h < HALVES; ++h) stage(S.a[h], Operand{P.A.p + h * half, P.A.outer, P.A.k}, m0, P.M, k0, P.K);
        stage(S.b, P.B, n0, P.N, k0, P.K);
        __syncthreads();
        for (int k = 0; k < kDepth; ++k)
            for (int h = 0; h < HALVES; ++h)
                for (int i = 0; i < 4; ++i)
                    for (int j = 0; j < 4; ++j) acc[h][i][j] = fmaf(S.a[h][k][ty * 4 + i], S.b[k][tx * 4 + j], acc[h][i][j]);
    }
}

struct GatedFwd { Product P; long half; int fn; const float* bias; float *y, *kept; Place to; };

__global__ void __launch_bounds__(256) k_gated_fwd(GatedFwd G)
{
    __shared__ Tiles S;
    const long m0 = (long)blockIdx.y * kTile, n0 = (long)blockIdx.x * kTile;
    float acc[2][4][4] = {};
    tile_product<2>(S, acc, G.P, G.half, m0, n0);
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const long m = m0 + threadIdx.x / 16 * 4 + i, n = n0 + threadIdx.x % 16 * 4 + j;
            if (m >= G.P.M || n >= G.P.N) continue;
            const float u = acc[0][i][j] + (G.bias ? G.bias[m] : 0.f), v = acc[1][i][j] + (G.bias ? G.bias[G.P.M + m] : 0.f);
            const bool rows = G.to.feature == 1;
            G.y[m * G.to.feature + n * G.to.position] = gate_fn(G.fn, u).a * v;
            if (G.kept) {
                const long at = m * G.to.feature + n * G.to.position * (rows ? 2 : 1);
                G.kept[at] = u;
                G.kept[at + G.P.M * G.to.feature] = v;
            }
        }
}

struct Product1 { Product P; float* c; long cm, cn; };
__global__ void __launch_bounds__(256) k_product(Product1 G)
{
    __shared__ Tiles S;
    const long m0 = (long)blockIdx.y * kTile, n0 = (long)blockIdx.x * kTile;
    float acc[1][4][4] = {};
    tile_product<1>(S, acc, G.P, 0, m0, n0);
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const long m = m0 + threadIdx.x / 16 * 4 + i, n = n0 + threadIdx.x % 16 * 4 + j;
            if (m < G.P.M && n < G.P.N) G.c[m * G.cm + n * G.cn] = acc[0][i][j];
        }
}

// [du; dv] from gy and the kept [u; v], in the layout of the kept.
__global__ void __launch_bounds__(256) k_gated_grads(int fn, long features, long positions, int rows, const float* gy, const float* kept, float* g)
{
    const long count = features * positions, step = rows ? features : count;
    for (long e = blockIdx.x * 256L + threadIdx.x; e < count; e += gridDim.x * 256L) {
        const long at = rows ? e + e / features * features : e;
        const Gated a = gate_fn(fn, kept[at]);
        g[at] = gy[e] * kept[at + step] * a.d;
        g[at + step] = gy[e] * a.a;
    }
}

__global__ void __launch_bounds__(256) k_gated_bias(long positions, Place at, const float* g, float* gb)
{
    __shared__ float part[256];
    float s = 0.f;
    for (long n = threadIdx.x; n < positions; n += 256) s += g[blockIdx.x * at.feature + n * at.position];
    part[threadIdx.x] = s;
    for (int w = 128; w > 0; w /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < w) part[threadIdx.x] += part[threadIdx.x + w];
    }
    if (threadIdx.x == 0) gb[blockIdx.x] = part[0];
}

struct Shape { int f, fo, axis; long positions; };

int check_gated(int32_t fan_in, int32_t fan_out, int64_t positions, int32_t axis)
{
    if (fan_in < 1 || fan_out < 1 || positions < 1) return fail(ZNN_EINVAL, "features and positions must be >= 1");
    if (axis != 0 && axis != 1) return fail(ZNN_EINVAL, "axis must be 0 (images) or 1 (rows of features)");
    if (fan_in > 1 << 20 || fan_out > 1 << 20 || positions > 2147483647LL)
        return fail(ZNN_EUNSUPPORTED, "a gated unit of %d to %d features over %lld positions is too large", fan_in, fan_out, (long long)positions);
    return ZNN_OK;
}

size_t gated_workspace(const Shape& S, bool backward) { return backward ? sizeof(float) * 2 * S.fo * S.positions : 0; }

int check_gated_call(int32_t fn, const Shape& S, bool backward, const void* ws, size_t ws_bytes)
{
    if (fn < ZNN_GATE_RECTIFY || fn > ZNN_GATE_GELU) return fail(ZNN_EINVAL, "unknown gate function %d", fn);
    const size_t need = gated_workspace(S, backward);
    if (!need) return ZNN_OK;
    if (!ws) return fail(ZNN_EWORKSPACE, "workspace is NULL but %zu bytes are needed", need);
    if ((uintptr_t)ws & 255) return fail(ZNN_EWORKSPACE, "workspace is not 256-byte aligned");
    if (ws_bytes < need) return fail(ZNN_EWORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
    return ZNN_OK;
}

dim3 tiles_of(long M, long N) { return dim3((unsigned)((N + kTile - 1) / kTile), (unsigned)((M + kTile - 1) / kTile)); }

}  // namespace
}  // namespace znn

using namespace znn;

extern "C" {

int znn_gated_workspace_bytes(int32_t fan_in, int32_t fan_out, int64_t positions, int32_t axis, int32_t pass, size_t* bytes)
{
    int rc = check_gated(fan_in, fan_out, positions, axis);
    if (rc != ZNN_OK) return rc;
    if (pass != ZNN_PASS_FWD && pass != ZNN_PASS_BWD) return fail(ZNN_EINVAL, "pass must be forward or backward");
    if (!bytes) return fail(ZNN_EINVAL, "NULL argument");
    *bytes = gated_workspace(Shape{fan_in, fan_out, axis, (long)positions}, pass == ZNN_PASS_BWD);
    return ZNN_OK;
}

int znn_gated_fwd(int32_t fn, int32_t fan_in, int32_t fan_out, int64_t positions, int32_t axis, const float* x, const float* w,
                  const float* b, float* y, float* kept, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_gated(fan_in, fan_out, positions, axis);
    if (rc != ZNN_OK) return rc;
    if (!x || !w || !y) return fail(ZNN_EINVAL, "NULL argument");
    const Shape S = {fan_in, fan_out, axis, (long)positions};
    rc = check_gated_call(fn, S, false, ws, ws_bytes);
    if (rc != ZNN_OK) return rc;
    const Place in = place(axis, S.f, S.positions);
    const GatedFwd G = {{{w, S.f, 1}, {x, in.position, in.feature}, S.fo, S.positions, S.f}, (long)S.fo * S.f, fn, b, y, kept,
                        place(axis, S.fo, S.positions)};
    ZNN_LAUNCH("gated unit forward", (hipStream_t)stream, k_gated_fwd, tiles_of(S.fo, S.positions), dim3(256), 0, G);
    return check_launch("gated unit forward");
}

int znn_gated_bwd(int32_t fn, int32_t fan_in, int32_t fan_out, int64_t positions, int32_t axis, const float* gy, const float* x,
                  const float* w, const float* kept, float* gx, float* gw, float* gb, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_gated(fan_in, fan_out, positions, axis);
    if (rc != ZNN_OK) return rc;
    if (!gy || !x || !w || !kept || !gw) return fail(ZNN_EINVAL, "NULL argument");
    const Shape S = {fan_in, fan_out, axis, (long)positions};
    rc = check_gated_call(fn, S, true, ws, ws_bytes);
    if (rc != ZNN_OK) return rc;
    const hipStream_t s = (hipStream_t)stream;
    float* const g = (float*)ws;
    const Place in = place(axis, S.f, S.positions), both = place(axis, 2L * S.fo, S.positions);
    const long work = (long)S.fo * S.positions;
    ZNN_LAUNCH("gated unit gradients", s, k_gated_grads, dim3((unsigned)std::min((work + 255) / 256, 1L << 20)), dim3(256), 0, fn, (long)S.fo,
               S.positions, axis, gy, kept, g);
    if (gx) {
        const Product1 P = {{{w, 1, S.f}, {g, both.position, both.feature}, S.f, S.positions, 2L * S.fo}, gx, in.feature, in.position};
        ZNN_LAUNCH("gated unit backward", s, k_product, tiles_of(S.f, S.positions), dim3(256), 0, P);
    }
    const Product1 P = {{{g, both.feature, both.position}, {x, in.feature, in.position}, 2L * S.fo, S.f, S.positions}, gw, S.f, 1};
    ZNN_LAUNCH("gated unit weights", s, k_product, tiles_of(2L * S.fo, S.f), dim3(256), 0, P);
    if (gb) ZNN_LAUNCH("gated unit bias", s, k_gated_bias, dim3(2 * S.fo), dim3(256), 0, S.positions, both, (const float*)g, gb);
    return check_launch("gated unit backward");
}

}  // extern "C"
