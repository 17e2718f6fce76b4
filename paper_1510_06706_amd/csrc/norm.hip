// Dropout, layer norm and the residual join (dropout, node sum and layer norm in one pass), forward and backward.
//
// Operands are dense [rows][cols] arrays.  Axis 0 normalises every column over the rows (images: each voxel over the maps),
// axis 1 every row over its columns.  With n elements in a position (a column or a row):
//     m = sum x / n,  s = 1 / sqrt(sum (x - m)^2 / n + eps),  h = (x - m) s,  y = w h + b
//     a = w gy,  gx = s (a - mean(a) - h mean(a h)),  gw = sum over positions of gy h,  gb = sum of gy
// Sums are held in 32 bits.  The sum of squares is taken about a first mean m0 and corrected by what is left of the sum there
// (d = x - m0, m = m0 + mean(d), variance mean(d^2) - mean(d)^2), so neither a mean far from zero nor m0's rounding costs y digits.  Backward, h is that
// of the statistics, which hold m in 32 bits: off by up to half an ulp of m times s, 2.4e-4 beside a mean of 4096 and a deviation of 1.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "random.h"
#include "znn_internal.h"

namespace znn {

// dropped: how many of 2^32
static int make_drop_parts(double dropped, const uint64_t* state, uint32_t site, Drop* drop, bool* drops)
{
    const double keep = 4294967296.0 - dropped;
    *drops = dropped > 0.0;
    *drop = Drop{state, site, *drops ? (unsigned)keep : 0u, keep > 0.0 ? (float)(4294967296.0 / keep) : 0.f};
    if (*drops && !state) return fail(ZNN_EINVAL, "dropout needs a random state");
    if (*drops && ((uintptr_t)state & 7)) return fail(ZNN_EINVAL, "the random state is not 8-byte aligned");
    return ZNN_OK;
}
static int make_drop(double p, const uint64_t* state, uint32_t site, Drop* drop, bool* drops)
{
    if (!(p >= 0.0 && p <= 1.0)) return fail(ZNN_EINVAL, "the probability to drop must lie in [0, 1]");
    return make_drop_parts(std::floor(p * 4294967296.0 + 0.5), state, site, drop, drops);
}

namespace {

// Rows lie one behind the other, so that the stores of neighbouring lanes fill lines but at a row's ends.  They leave the cache at once, which
// would write them back when the kernel ends, with nothing else left to do.  us before and after: dropout on 36 x 84987 5.6 -> 5.1, norm on
// 16384 x 512 12.4 -> 11.0, on 1000 x 3505 6.5 -> 5.7, joined 10.8 -> 8.9, join on 8192 x 2048 backward 67 -> 57.
__device__ __forceinline__ void store_row(float* p, int count, floatu4 v)
{
    if (count >= 4) __builtin_nontemporal_store(v, reinterpret_cast<floatu4*>(p));
    else store4(p, count, v);
}

// ---------------------------------------------------------------- dropout
// A thread draws the four words of a block for four neighbouring columns.  Bound by memory: 120 x 90^3 (700 MB) 111 us = 6.3 TB/s; the
// generator's 124 vector instructions a wave are a third of that time.
__global__ void __launch_bounds__(256)
k_dropout(long rows, long cols, long quads, Drop D, const float* __restrict__ x, float* __restrict__ y)
{
    const DropKey K = drop_key(D);
    for (long t = (long)blockIdx.x * 256 + threadIdx.x; t < rows * quads; t += (long)gridDim.x * 256) {
        const long row = t / quads, q = t - row * quads, at = row * cols + 4 * q;
        const int count = (int)min(4L, cols - 4 * q);
        store_row(y + at, count, dropped4(K, (unsigned)q, (unsigned)row, load4(x + at, count)));
    }
}

__global__ void __launch_bounds__(256) k_copy(long count, const float* __restrict__ x, float* __restrict__ y)
{
    for (long t = 4 * ((long)blockIdx.x * 256 + threadIdx.x); t < count; t += 4L * gridDim.x * 256) {
        const int n = (int)min(4L, count - t);
        store_row(y + t, n, load4(x + t, n));
    }
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

// Additions that follow each other in a sum over a position of any length.  The sums of such chains are added up in a chain of their own: one
// chain of 2^18 squares of normal values is 955 half-ulps low, because what is less than half an ulp of the sum is lost.
constexpr int kChain = 256;
constexpr long kLongRow = 1024L * kChain;       // columns of which each of 1024 threads adds up kChain

// ---------------------------------------------------------------- columns held in registers
// TX lanes side by side take four neighbouring columns each, TY of them one below the other the rows ty, ty + TY, ... (kRowsHeld of
// them at most), so that an operand is read once.  Sums over a column: over the lanes of a wave, then over the waves by LDS.
constexpr int kRowsHeld = 4;
constexpr unsigned kBufferWord3 = 0x00020000u;      // raw 32-bit buffer elements
typedef unsigned word4 __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));

// Stores of whole 128-byte lines (STREAM) leave the cache at once, as those of rows do (store_row): 120 x 262144 backward 90 -> 72 us,
// 120 x 32768 forward 8.7 -> 6.9.  Parts of lines would be written each on its own: 120 x 262143 forward 44 -> 90.
template <bool STREAM> __device__ __forceinline__ void store_buffer(__amdgpu_buffer_rsrc_t b, unsigned at, float4v v)
{
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(word4, v), b, (int)at, 0, STREAM ? 2 : 0);
}
__device__ __forceinline__ float4v load_buffer(__amdgpu_buffer_rsrc_t b, unsigned at)
{
    return __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(b, (int)at, 0, 0));
}

// Where a thread's elements lie.  Its row number k is row TY k + ty: a buffer that begins with row TY k, whose end cuts off what the
// last rows are short of TY (loads give 0, stores go nowhere), and 32 bits of the thread's own, so that an operand costs no registers
// for addresses (norm_shape keeps TY rows below 2^32 bytes).  At the right border the columns move left until four of them are there;
// the first `skip` of them are then another thread's too, which computes and stores the same values.
template <int TX, int TY> struct ColumnTile {
    long cols, first;           // first: column at which the buffers begin
    int rows, ty, skip;
    unsigned along, at;         // columns from `first` on; bytes from a buffer's begin
    bool border;                // uniform: some thread skips columns
    long row0;                  // the tile's rows are those from row0 on of the array, and the pointers begin there
    __device__ __forceinline__ ColumnTile(long rows_, long cols_, long tile, long row0_ = 0)
        : cols(cols_), first(tile * TX * 4), rows((int)rows_), row0(row0_)
    {
        const int tx = threadIdx.x % TX * 4, last = (int)min(TX * 4L, cols - first) - 4;        // where the last thread may begin: -3 or more
        ty = threadIdx.x / TX;
        border = last < (TX - 1) * 4;
        const int back = border && tile > 0 ? 4 : 0;        // so that the base lies left of every thread
        skip = max(0, tx - last);
        along = (unsigned)(tx - skip + back);
        first -= back;
        at = 4u * ((unsigned)ty * (unsigned)cols + along);
    }
    __device__ __forceinline__ bool any(int k) const { return TY * k < rows; }                                  // uniform
    __device__ __forceinline__ bool has(int k) const { return TY * (k + 1) <= rows || TY * k + ty < rows; }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const float* p, int k) const
    {
        const unsigned bytes = TY * (k + 1) <= rows ? 0xffffffffu : 4u * ((unsigned)(rows - TY * k) * (unsigned)cols - (unsigned)first);
        return __builtin_amdgcn_make_buffer_rsrc((void*)(p + ((long)TY * k * cols + first)), 0, (int)bytes, kBufferWord3);
    }
    __device__ __forceinline__ float4v load(const float* p, int k) const { return load_buffer(buffer(p, k), at); }
    template <bool STREAM> __device__ __forceinline__ void store(float* p, int k, float4v v) const { store_buffer<STREAM>(buffer(p, k), at, v); }
    // an array with one value per column
    __device__ __forceinline__ float4v load_columns(const float* p) const
    {
        return load_buffer(__builtin_amdgcn_make_buffer_rsrc((void*)(p + first), 0, -1, kBufferWord3), 4u * along);
    }
    __device__ __forceinline__ void store_columns(float* p, float4v v) const
    {
        store_buffer<false>(__builtin_amdgcn_make_buffer_rsrc((void*)(p + first), 0, -1, kBufferWord3), 4u * along, v);
    }
    __device__ __forceinline__ float4v drop(const DropKey& K, int k, float4v v) const
    {
        const long c = first + along;
        const unsigned m = (unsigned)row0 + TY * k + ty;
        const Words u = drop_words(K, (unsigned)(c >> 2), m);
        if (border) {           // columns of two quads
            const Words n = drop_words(K, (unsigned)(c >> 2) + 1, m);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int q = e + (int)(c & 3);
                v[e] = dropped(K, q == 0 ? u.w[0] : q == 1 ? u.w[1] : q == 2 ? u.w[2] : q == 3 ? u.w[3] : q == 4 ? n.w[0] : q == 5 ? n.w[1] : n.w[2], v[e]);
            }
        } else
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = dropped(K, u.w[e], v[e]);
        return v;
    }
};

// Tiles in the order of the workgroups, or (`apart`) an eighth of them to every XCD, so that rows that begin in the middle of a line find
// its other part in the same cache: 36 x 105225 forward 9.8 -> 8.8 us, backward 17 -> 14; 200 x 30690 17 -> 14 and 26 -> 19.
struct Tiles { long count; int apart; };
__device__ __forceinline__ long tile_turns(Tiles T) { return T.apart ? (T.count + 7) / 8 * 8 : T.count; }
__device__ __forceinline__ long tile_of(Tiles T, long turn) { return T.apart ? (turn & 7) * ((T.count + 7) / 8) + (turn >> 3) : turn; }

// Sums of N values over ty, for all threads.  `red` must not be that of the call before: a thread may still read it.
template <int TX, int TY, int N> __device__ __forceinline__ void sum_over_ty(float (&v)[N], float (*red)[TX][N])
{
    constexpr int WAVES = TX * TY / 64;
#pragma unroll
    for (int s = TX; s < 64; s <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], s);
    if constexpr (WAVES > 1) {
        const int tx = threadIdx.x % TX, wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) < TX)
#pragma unroll
            for (int i = 0; i < N; ++i) red[wave][tx][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = red[0][tx][i];
#pragma unroll
        for (int q = 1; q < WAVES; ++q)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += red[q][tx][i];
    }
}

// Forward.  Bound by memory: 120 x 96^3 (856 MB) 170 us = 5.05 TB/s, joined with dropout (1.7 GB) 343 us; 40 x 60^3 (71 MB, from the last
// level cache) 13.6 us.  The sums are those of the squares about the first mean, whose rounding the second corrects (top of the file).
template <int MODE, int TX, int TY, bool STREAM>
__global__ void __launch_bounds__(TX * TY, 4) k_norm_cols(NormFwd A, Tiles tiles)
{
    constexpr int WAVES = TX * TY / 64, K = kRowsHeld;
    __shared__ float red[WAVES][TX][4], red2[WAVES][TX][8];
    DropKey D = {};
    if (MODE == JOIN_DROP) D = drop_key(A.drop);
    const float inv = 1.0f / (float)A.rows;
    for (long turn = blockIdx.x; turn < tile_turns(tiles); turn += gridDim.x) {
        const long tile = tile_of(tiles, turn);
        if (tile >= tiles.count) continue;      // uniform
        const ColumnTile<TX, TY> T(A.rows, A.cols, tile);
        float4v v[K];
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (T.any(k)) v[k] = T.load(A.x, k);
        if (MODE != PLAIN) {
            float4v h[K];
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k)) h[k] = T.load(A.h, k);
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k)) {
                    if (MODE == JOIN_DROP) h[k] = T.drop(D, k, h[k]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[k][e] = joined(v[k][e], h[k][e]);
                    T.template store<STREAM>(A.r, k, v[k]);
                }
        }
        float sum[4], d[8], rstd[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (T.any(k))
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += v[k][e];          // 0 where there is no row
        sum_over_ty<TX, TY, 4>(sum, red);
#pragma unroll
        for (int e = 0; e < 4; ++e) { sum[e] *= inv; d[e] = d[4 + e] = 0.f; }
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (T.any(k))
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = T.has(k) ? v[k][e] - sum[e] : 0.f;
                    v[k][e] = a;
                    d[e] += a;
                    d[4 + e] += a * a;
                }
        sum_over_ty<TX, TY, 8>(d, red2);
#pragma unroll
        for (int e = 0; e < 4; ++e) { d[e] *= inv; rstd[e] = inverse_deviation(d[4 + e] * inv, d[e], A.eps); }
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (T.any(k)) {
                const int m = min(TY * k + T.ty, T.rows - 1);
                const float w = A.w[m], b = A.b[m];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[k][e] = (v[k][e] - d[e]) * rstd[e] * w + b;
                T.template store<STREAM>(A.y, k, v[k]);
            }
        if (A.stats && T.ty == 0) {
            T.store_columns(A.stats, float4v{sum[0] + d[0], sum[1] + d[1], sum[2] + d[2], sum[3] + d[3]});
            T.store_columns(A.stats + A.cols, float4v{rstd[0], rstd[1], rstd[2], rstd[3]});
        }
    }
}

// What the columns from c0 to c1 give to the gradients of weight and bias of one feature, by one workgroup.  Over all columns: for few of
// them, where a launch that adds shares up would take as long again.
template <int T> __device__ __forceinline__ float2 row_params(const float* gy, const float* x, const float* mean, const float* rstd, long c0, long c1, float2* red)
{
    float a = 0.f, b = 0.f;
    for (long s0 = c0; s0 < c1; s0 += kChain * T) {
        const long s1 = min(c1, s0 + kChain * T);
        float pa = 0.f, pb = 0.f;
        for (long c = s0 + 4 * threadIdx.x; c < s1; c += 4 * T) {
            const int count = (int)min(4L, s1 - c);
            const floatu4 g = load4(gy + c, count), v = load4(x + c, count), m = load4(mean + c, count), q = load4(rstd + c, count);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < count) { pa += g[e] * ((v[e] - m[e]) * q[e]); pb += g[e]; }
        }
        a += pa;
        b += pb;
    }
    return group_sum<T / 64>(a, b, red);
}

// PARTS: a workgroup takes every gridDim.x-th tile, adds up what its columns give to the parameters' gradients in registers and leaves its
// share.  Otherwise the first workgroups take a feature each (row_params).  What reaches r beside the norm (gr) is requested with the other
// operands, before the sums.  Bound by memory: 120 x 96^3 (1.28 GB) 265 us = 4.8 TB/s, joined with dropout (2.13 GB) 455 us; 40 x 60^3 19 us.
template <int MODE, int TX, int TY, bool STREAM, bool PARTS>
__global__ void __launch_bounds__(TX * TY, 4) k_norm_cols_bwd(NormBwd A, Tiles tiles, float* __restrict__ parts, float* __restrict__ pw, float* __restrict__ pb)
{
    constexpr int WAVES = TX * TY / 64, K = kRowsHeld;
    __shared__ float red[2][WAVES][TX][8];
    const unsigned others = PARTS ? 0 : (unsigned)A.rows;
    if (blockIdx.x < others) {
        const long m = blockIdx.x;
        const float2 s = row_params<TX * TY>(A.gy + m * A.cols, A.x + m * A.cols, A.stats, A.stats + A.cols, 0, A.cols, (float2*)red);
        if (threadIdx.x == 0) { pw[m] = s.x; pb[m] = s.y; }
        return;
    }
    const unsigned block = blockIdx.x - others, blocks = gridDim.x - others;
    DropKey D = {};
    if (MODE == JOIN_DROP) D = drop_key(A.drop);
    const int tx = threadIdx.x % TX, ty = threadIdx.x / TX, rows = (int)A.rows;
    const float inv = 1.0f / (float)rows;
    float gw[K], gb[K], w[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        gw[k] = gb[k] = 0.f;
        w[k] = ty + TY * k < rows ? A.w[ty + TY * k] : 0.f;
    }
    int side = 0;
    for (long turn = block; turn < tile_turns(tiles); turn += blocks) {
        const long tile = tile_of(tiles, turn);
        if (tile >= tiles.count) continue;      // uniform
        const ColumnTile<TX, TY> T(A.rows, A.cols, tile);
        float4v x[K], g[K], r[K];
        const float4v mean = T.load_columns(A.stats), rstd = T.load_columns(A.stats + A.cols);
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (T.any(k)) {
                x[k] = T.load(A.x, k);
                g[k] = T.load(A.gy, k);
            }
        const bool more = MODE != PLAIN && A.gr;
        if (more)
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k)) r[k] = T.load(A.gr, k);
        float s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (T.any(k))
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float gy = g[k][e], own = e >= T.skip ? gy : 0.f, a = gy * w[k];      // 0 where there is no row
                    const float h = T.has(k) ? (x[k][e] - mean[e]) * rstd[e] : 0.f;
                    x[k][e] = h;
                    if (PARTS) {
                        gw[k] += own * h;
                        gb[k] += own;
                    }
                    g[k][e] = a;
                    s[e] += a;
                    s[4 + e] += a * h;
                }
        sum_over_ty<TX, TY, 8>(s, red[side]);
        side ^= 1;
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] *= inv;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (T.any(k)) {
                float4v v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = rstd[e] * (g[k][e] - s[e] - x[k][e] * s[4 + e]);
                if (more)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] += r[k][e];
                T.template store<STREAM>(A.gx, k, v);
                if (MODE == JOIN_DROP) v = T.drop(D, k, v);
                if (MODE != PLAIN && A.gh) T.template store<STREAM>(A.gh, k, v);
            }
    }
    if constexpr (!PARTS) return;
    float* part = parts + (long)block * 2 * rows;
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (TY * k < rows) {
            float a = gw[k], b = gb[k];
#pragma unroll
            for (int i = 1; i < TX; i <<= 1) { a += __shfl_xor(a, i); b += __shfl_xor(b, i); }
            const int m = ty + TY * k;
            if (tx == 0 && m < rows) { part[m] = a; part[rows + m] = b; }
        }
}

// ---------------------------------------------------------------- rows held in registers
// L lanes take a row, NV times four neighbouring columns each: lanes of a wave (the sums stay in it) or a whole workgroup of L.
// T threads in a workgroup, T / L rows at a time.
template <int L> __device__ __forceinline__ float2 row_sum(float a, float b, float2* red)
{
#pragma unroll
    for (int s = 1; s < (L < 64 ? L : 64); s <<= 1) { a += __shfl_xor(a, s); b += __shfl_xor(b, s); }
    if constexpr (L > 64) {         // `red` must not be that of the call before: a thread may still read it
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = make_float2(a, b);
        __syncthreads();
        float2 v = red[0];
#pragma unroll
        for (int i = 1; i < L / 64; ++i) { v.x += red[i].x; v.y += red[i].y; }
        return v;
    }
    return make_float2(a, b);
}
// columns 4 (lane + L j) .. + 3 of a row; only the last quads of a row may lie behind it
template <int L> __device__ __forceinline__ int quad_count(int j, int lane, int cols)
{
    return 4 * L * (j + 1) <= cols ? 4 : max(0, min(4, cols - 4 * (lane + L * j)));
}
// the row of a wave, which the compiler then knows to be one
template <int L> __device__ __forceinline__ long wave_row(long row)
{
    if constexpr (L >= 64) return (long)__builtin_amdgcn_readfirstlane((int)row) & 0xffffffffL;     // rows have 32 bits
    return row;
}

// Forward.  Bound by memory or the last level cache: 20000 x 8000 (1.28 GB) 227 us = 5.6 TB/s, 16384 x 512 (67 MB) 11 us; a single row of 1024
// by its latency, 2.8 us.
template <int MODE, int L, int NV, int T>
__global__ void __launch_bounds__(T) k_norm_rows(NormFwd A)
{
    constexpr int ROWS = T / L;
    constexpr bool KEEP = L * NV <= 2048;       // weights of longer rows come from the cache for every row: their registers let a second workgroup in
    __shared__ float2 red[2][L > 64 ? L / 64 : 1];
    DropKey D = {};
    if (MODE == JOIN_DROP) D = drop_key(A.drop);
    const int lane = threadIdx.x % L, cols = (int)A.cols;
    const float inv = 1.0f / (float)cols;
    floatu4 w[NV], b[NV];
    auto weights = [&]() {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int count = quad_count<L>(j, lane, cols);
            w[j] = load4(A.w + 4 * (lane + L * j), count);
            b[j] = load4(A.b + 4 * (lane + L * j), count);
        }
    };
    if (KEEP) weights();
    for (long row0 = (long)blockIdx.x * ROWS; row0 < A.rows; row0 += (long)gridDim.x * ROWS) {
        const long row = wave_row<L>(row0 + threadIdx.x / L), base = min(row, A.rows - 1) * cols;
        const bool live = row < A.rows;
        floatu4 v[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) v[j] = load4(A.x + base + 4 * (lane + L * j), quad_count<L>(j, lane, cols));
        if (MODE != PLAIN) {
            floatu4 h[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) h[j] = load4(A.h + base + 4 * (lane + L * j), quad_count<L>(j, lane, cols));
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (MODE == JOIN_DROP) h[j] = dropped4(D, (unsigned)(lane + L * j), (unsigned)row, h[j]);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[j][e] = joined(v[j][e], h[j][e]);
                if (live) store_row(A.r + base + 4 * (lane + L * j), quad_count<L>(j, lane, cols), v[j]);
            }
        }
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) sum += (v[j][0] + v[j][1]) + (v[j][2] + v[j][3]);
        const float m0 = row_sum<L>(sum, 0.f, red[0]).x * inv;
        float d1 = 0.f, d2 = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float d = e < quad_count<L>(j, lane, cols) ? v[j][e] - m0 : 0.f;
                v[j][e] = d;
                d1 += d;
                d2 += d * d;
            }
        if (!KEEP) weights();
        const float2 s = row_sum<L>(d1, d2, red[1]);
        const float delta = s.x * inv, rstd = inverse_deviation(s.y * inv, delta, A.eps);
        if (live) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[j][e] = (v[j][e] - delta) * rstd * w[j][e] + b[j][e];
                store_row(A.y + base + 4 * (lane + L * j), quad_count<L>(j, lane, cols), v[j]);
            }
            if (A.stats && lane == 0) { A.stats[row] = m0 + delta; A.stats[A.rows + row] = rstd; }
        }
    }
}

// Gradients of weight and bias of 32 features by one workgroup, over all rows: for few rows, where shares of the workgroups would be as
// large as the operands.  red: T / 32 x 32 float2.
template <int T> __device__ __forceinline__ void column_params(const NormBwd& A, long c0, float* gw, float* gb, float2 (*red)[32])
{
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const long c = c0 + tx;
    float a = 0.f, b = 0.f;
    if (c < A.cols)
#pragma unroll 4
        for (long r = ty; r < A.rows; r += T / 32) {
            const float g = A.gy[r * A.cols + c];
            a += g * ((A.x[r * A.cols + c] - A.stats[r]) * A.stats[A.rows + r]);
            b += g;
        }
    red[ty][tx] = make_float2(a, b);
    __syncthreads();
    if (ty > 0 || c >= A.cols) return;
#pragma unroll 8
    for (int q = 1; q < T / 32; ++q) { a += red[q][tx].x; b += red[q][tx].y; }
    gw[c] = a;
    gb[c] = b;
}

// PARTS: the workgroup adds up what its rows give to the parameters' gradients, in registers or, of long rows, in LDS, and leaves its share.
// Otherwise the first workgroups take 32 features each (column_params).  Bound by memory: 20000 x 8000 (1.92 GB) 348 us = 5.5 TB/s, 5003 x 1001
// (60 MB) 16 us, of them 3 to 4 for the shares' sums, 64 x 1000 2.8 us in one launch.
template <int MODE, int L, int NV, int T, bool PARTS>
__global__ void __launch_bounds__(T) k_norm_rows_bwd(NormBwd A, float* __restrict__ parts, float* __restrict__ pw, float* __restrict__ pb)
{
    constexpr int ROWS = T / L;
    __shared__ float2 red[2][L > 64 ? L / 64 : 1];
    constexpr bool IN_LDS = PARTS && L * NV > 2048;
    __shared__ __align__(16) float sums[IN_LDS ? L * NV * 8 : !PARTS ? T * 2 : ROWS > 1 ? T * NV * 4 : 1];
    const unsigned others = PARTS ? 0 : (unsigned)((A.cols + 31) / 32);
    if (blockIdx.x < others) {
        column_params<T>(A, (long)blockIdx.x * 32, pw, pb, (float2 (*)[32])sums);
        return;
    }
    const unsigned block = blockIdx.x - others, blocks = gridDim.x - others;
    floatu4* held = reinterpret_cast<floatu4*>(sums) + threadIdx.x;     // IN_LDS: the thread's own, gw and gb by turns, T apart
    DropKey D = {};
    if (MODE == JOIN_DROP) D = drop_key(A.drop);
    const int lane = threadIdx.x % L, group = threadIdx.x / L, cols = (int)A.cols;
    const float inv = 1.0f / (float)cols;
    floatu4 w[NV], gw[NV], gb[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        w[j] = load4(A.w + 4 * (lane + L * j), quad_count<L>(j, lane, cols));
        gw[j] = gb[j] = floatu4{0.f, 0.f, 0.f, 0.f};
        if (IN_LDS) held[2 * j * T] = held[(2 * j + 1) * T] = gw[j];
    }
    int turn = 0;
    for (long row0 = (long)block * ROWS; row0 < A.rows; row0 += (long)blocks * ROWS, turn ^= 1) {
        const long at = wave_row<L>(row0 + group), row = min(at, A.rows - 1), base = row * cols;
        const bool live = at < A.rows;
        const float mean = A.stats[row], rstd = A.stats[A.rows + row];
        floatu4 x[NV], g[NV], r[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int count = quad_count<L>(j, lane, cols);
            x[j] = load4(A.x + base + 4 * (lane + L * j), count);
            g[j] = load4(A.gy + base + 4 * (lane + L * j), live ? count : 0);       // gy = 0 behind the row and behind the rows
        }
        const bool more = MODE != PLAIN && A.gr;
        if (more)
#pragma unroll
            for (int j = 0; j < NV; ++j) r[j] = load4(A.gr + base + 4 * (lane + L * j), quad_count<L>(j, lane, cols));
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (IN_LDS) { gw[j] = held[2 * j * T]; gb[j] = held[(2 * j + 1) * T]; }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool in = live && e < quad_count<L>(j, lane, cols);
                const float h = in ? (x[j][e] - mean) * rstd : 0.f, a = g[j][e] * w[j][e];
                x[j][e] = h;
                if (PARTS) {
                    gw[j][e] += g[j][e] * h;
                    gb[j][e] += g[j][e];
                }
                g[j][e] = a;
                s1 += a;
                s2 += a * h;
            }
            if (IN_LDS) { held[2 * j * T] = gw[j]; held[(2 * j + 1) * T] = gb[j]; }
        }
        const float2 s = row_sum<L>(s1, s2, red[turn]);
        const float m1 = s.x * inv, m2 = s.y * inv;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int count = live ? quad_count<L>(j, lane, cols) : 0;
            const long t = base + 4 * (lane + L * j);
            floatu4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = rstd * (g[j][e] - m1 - x[j][e] * m2);
            if (more)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += r[j][e];
            store_row(A.gx + t, count, v);
            if (MODE == JOIN_DROP) v = dropped4(D, (unsigned)(lane + L * j), (unsigned)row, v);
            if (MODE != PLAIN && A.gh) store_row(A.gh + t, count, v);
        }
    }
    if constexpr (!PARTS) return;
    float* part = parts + (long)block * 2 * cols;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const floatu4 (&v)[NV] = which ? gb : gw;
        if constexpr (ROWS > 1) {       // the sums of the workgroup's rows below each other, which all threads add up
            constexpr int W = L * NV * 4;
            if (which) __syncthreads();
#pragma unroll
            for (int j = 0; j < NV; ++j) *reinterpret_cast<floatu4*>(sums + group * W + 4 * (lane + L * j)) = v[j];
            __syncthreads();
            for (int c = threadIdx.x; c < cols; c += T) {
                float a = sums[c];
#pragma unroll
                for (int q = 1; q < ROWS; ++q) a += sums[q * W + c];
                part[which * cols + c] = a;
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                store4(part + which * cols + 4 * (lane + L * j), quad_count<L>(j, lane, cols), IN_LDS ? held[(2 * j + which) * T] : v[j]);
        }
    }
}

// ---------------------------------------------------------------- positions of any size
// Calls f(quad, columns) for the quads of a row that are the thread's, several of them without a branch in between; LONG: and aside() between
// kChain values and the next.
template <bool LONG, class F, class G> __device__ __forceinline__ void row_quads(long cols, F f, G aside)
{
    const long whole = cols / 4;
    if constexpr (!LONG) {
#pragma unroll 4
        for (long q = threadIdx.x; q < whole; q += 1024) f(q, 4);
    } else
        for (long q0 = 0; q0 < whole; q0 += kLongRow / 4) {
            if (q0 > 0) aside();
            const long end = min(whole, q0 + kLongRow / 4);
#pragma unroll 4
            for (long q = q0 + threadIdx.x; q < end; q += 1024) f(q, 4);
        }
    if ((cols & 3) && threadIdx.x == whole % 1024) f(whole, (int)(cols & 3));
}
template <class F> __device__ __forceinline__ void row_quads(long cols, F f) { row_quads<false>(cols, f, [] {}); }

// Rows of any length: a workgroup walks a row three times, backward twice.  2000 x 20000 71 us at a floor of 60.  Those of more than kLongRow columns
// by instances of their own, as setting aside costs the others: joined with dropout 2000 x 20000 149 us without, 159 with it.
template <int MODE, bool LONG>
__global__ void __launch_bounds__(1024) k_norm_rows_any(NormFwd A)
{
    __shared__ float2 red[16];
    DropKey K = {};
    if (MODE == JOIN_DROP) K = drop_key(A.drop);
    const float inv = 1.0f / (float)A.cols;
    for (long row = blockIdx.x; row < A.rows; row += gridDim.x) {
        const long base = row * A.cols;
        const float* src = (MODE == PLAIN ? A.x : A.r) + base;
        float sum = 0.f, d1 = 0.f, d2 = 0.f, far1 = 0.f, far2 = 0.f;        // far: the chains set aside
        row_quads<LONG>(A.cols, [&](long q, int count) {
            floatu4 v = load4(A.x + base + 4 * q, count);
            if (MODE != PLAIN) {
                floatu4 h = load4(A.h + base + 4 * q, count);
                if (MODE == JOIN_DROP) h = dropped4(K, (unsigned)q, (unsigned)row, h);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = joined(v[e], h[e]);
                store4(A.r + base + 4 * q, count, v);
            }
            sum += (v[0] + v[1]) + (v[2] + v[3]);       // 0 behind the row
        }, [&] { far1 += sum; sum = 0.f; });
        if (LONG) sum += far1;
        const float m0 = group_sum<16>(sum, 0.f, red).x * inv;
        far1 = 0.f;
        row_quads<LONG>(A.cols, [&](long q, int count) {
            const floatu4 v = load4(src + 4 * q, count);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < count) { const float d = v[e] - m0; d1 += d; d2 += d * d; }
        }, [&] { far1 += d1; far2 += d2; d1 = d2 = 0.f; });
        if (LONG) { d1 += far1; d2 += far2; }
        const float2 s = group_sum<16>(d1, d2, red);
        const float delta = s.x * inv, rstd = inverse_deviation(s.y * inv, delta, A.eps);
        row_quads(A.cols, [&](long q, int count) {
            floatu4 v = load4(src + 4 * q, count);
            const floatu4 w = load4(A.w + 4 * q, count), b = load4(A.b + 4 * q, count);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = ((v[e] - m0) - delta) * rstd * w[e] + b[e];
            store_row(A.y + base + 4 * q, count, v);
        });
        if (A.stats && threadIdx.x == 0) { A.stats[row] = m0 + delta; A.stats[A.rows + row] = rstd; }
    }
}

template <int MODE, bool LONG>
__global__ void __launch_bounds__(1024) k_norm_rows_bwd_any(NormBwd A)
{
    __shared__ float2 red[16];
    DropKey K = {};
    if (MODE == JOIN_DROP) K = drop_key(A.drop);
    const float inv = 1.0f / (float)A.cols;
    for (long row = blockIdx.x; row < A.rows; row += gridDim.x) {
        const long base = row * A.cols;
        const float mean = A.stats[row], rstd = A.stats[A.rows + row];
        float s1 = 0.f, s2 = 0.f, far1 = 0.f, far2 = 0.f;
        row_quads<LONG>(A.cols, [&](long q, int count) {
            const floatu4 x = load4(A.x + base + 4 * q, count), g = load4(A.gy + base + 4 * q, count), w = load4(A.w + 4 * q, count);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < count) { const float a = g[e] * w[e]; s1 += a; s2 += a * ((x[e] - mean) * rstd); }
        }, [&] { far1 += s1; far2 += s2; s1 = s2 = 0.f; });
        if (LONG) { s1 += far1; s2 += far2; }
        const float2 s = group_sum<16>(s1, s2, red);
        const float m1 = s.x * inv, m2 = s.y * inv;
        row_quads(A.cols, [&](long q, int count) {
            const floatu4 x = load4(A.x + base + 4 * q, count), g = load4(A.gy + base + 4 * q, count), w = load4(A.w + 4 * q, count);
            floatu4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = rstd * (g[e] * w[e] - m1 - (x[e] - mean) * rstd * m2);
            if (MODE != PLAIN && A.gr) {
                const floatu4 r = load4(A.gr + base + 4 * q, count);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += r[e];
            }
            store_row(A.gx + base + 4 * q, count, v);
            if (MODE == JOIN_DROP) v = dropped4(K, (unsigned)q, (unsigned)row, v);
            if (MODE != PLAIN && A.gh) store_row(A.gh + base + 4 * q, count, v);
        });
    }
}

// Columns of any height: tiles of 32 columns by 128 threads below each other, which walk blocks of 512 rows three times, backward twice.
// Bound by the caches: 768 x 32768 58 us at a floor of 38, backward 120 at 57 (one column a thread 164 and 171; 2048 x 4096 332 -> 25).
constexpr int kTallX = 8, kTallY = 128, kTallRows = kTallY * kRowsHeld;
typedef ColumnTile<kTallX, kTallY> TallTile;

// LONG, for more than kLongColumn rows: chains of a thread's sums are set aside in LDS, [value][thread].  Instances of their own, as it costs the others
// registers: 1024 x 110592 joined 457 us without, 473 with it.
constexpr long kLongColumn = (long)kTallY * kChain;
typedef float TallAside[8][1024];
template <int N> __device__ __forceinline__ void set_aside(long r0, long block, TallAside& far, float (&v)[N])
{
    if ((r0 + block) % kLongColumn != 0) return;        // uniform
#pragma unroll
    for (int i = 0; i < N; ++i) {
        far[i][threadIdx.x] = r0 + block == kLongColumn ? v[i] : far[i][threadIdx.x] + v[i];
        v[i] = 0.f;
    }
}
template <int N> __device__ __forceinline__ void add_aside(const TallAside& far, float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += far[i][threadIdx.x];
}

template <int MODE, bool LONG>
__global__ void __launch_bounds__(1024) k_norm_cols_tall(NormFwd A, Tiles tiles)
{
    constexpr int K = kRowsHeld;
    __shared__ float red[16][kTallX][4], red2[16][kTallX][8];
    __shared__ float far[LONG ? 8 : 1][LONG ? 1024 : 1];
    DropKey D = {};
    if (MODE == JOIN_DROP) D = drop_key(A.drop);
    const float inv = 1.0f / (float)A.rows;
    for (long turn = blockIdx.x; turn < tile_turns(tiles); turn += gridDim.x) {
        const long tile = tile_of(tiles, turn);
        if (tile >= tiles.count) continue;      // uniform
        const float* src = MODE == PLAIN ? A.x : A.r;
        float sum[4], d[8], rstd[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = d[e] = d[4 + e] = 0.f;
#pragma unroll 1
        for (long r0 = 0; r0 < A.rows; r0 += kTallRows) {
            const TallTile T(min((long)kTallRows, A.rows - r0), A.cols, tile, r0);
            const long off = r0 * A.cols;
            float4v v[K], h[K];
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k)) {
                    v[k] = T.load(A.x + off, k);
                    if (MODE != PLAIN) h[k] = T.load(A.h + off, k);
                }
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k)) {
                    if (MODE != PLAIN) {
                        if (MODE == JOIN_DROP) h[k] = T.drop(D, k, h[k]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[k][e] = joined(v[k][e], h[k][e]);
                        T.template store<false>(A.r + off, k, v[k]);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] += v[k][e];      // 0 where there is no row
                }
            if constexpr (LONG) set_aside<4>(r0, kTallRows, far, sum);
        }
        if constexpr (LONG) add_aside<4>(far, sum);
        sum_over_ty<kTallX, kTallY, 4>(sum, red);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] *= inv;
#pragma unroll 1
        for (long r0 = 0; r0 < A.rows; r0 += kTallRows) {
            const TallTile T(min((long)kTallRows, A.rows - r0), A.cols, tile, r0);
            float4v v[K];
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k)) v[k] = T.load(src + r0 * A.cols, k);
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k))
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = T.has(k) ? v[k][e] - sum[e] : 0.f;
                        d[e] += a;
                        d[4 + e] += a * a;
                    }
            if constexpr (LONG) set_aside<8>(r0, kTallRows, far, d);
        }
        if constexpr (LONG) add_aside<8>(far, d);
        sum_over_ty<kTallX, kTallY, 8>(d, red2);
#pragma unroll
        for (int e = 0; e < 4; ++e) { d[e] *= inv; rstd[e] = inverse_deviation(d[4 + e] * inv, d[e], A.eps); }
#pragma unroll 1
        for (long r0 = 0; r0 < A.rows; r0 += kTallRows) {
            const TallTile T(min((long)kTallRows, A.rows - r0), A.cols, tile, r0);
            float4v v[K];
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k)) v[k] = T.load(src + r0 * A.cols, k);
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k)) {
                    const long m = min(r0 + kTallY * k + T.ty, A.rows - 1);
                    const float w = A.w[m], b = A.b[m];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[k][e] = ((v[k][e] - sum[e]) - d[e]) * rstd[e] * w + b;
                    T.template store<false>(A.y + r0 * A.cols, k, v[k]);
                }
            if (A.stats && r0 == 0 && T.ty == 0) {
                T.store_columns(A.stats, float4v{sum[0] + d[0], sum[1] + d[1], sum[2] + d[2], sum[3] + d[3]});
                T.store_columns(A.stats + A.cols, float4v{rstd[0], rstd[1], rstd[2], rstd[3]});
            }
        }
    }
}

template <int MODE, bool LONG>
__global__ void __launch_bounds__(1024) k_norm_cols_bwd_tall(NormBwd A, Tiles tiles)
{
    constexpr int K = MODE == PLAIN ? kRowsHeld : 2;        // four of three operands leave no registers: 1024 x 110592 1141 us, two 821
    constexpr long BLOCK = kTallY * K;
    __shared__ float red[2][16][kTallX][8];
    __shared__ float far[LONG ? 8 : 1][LONG ? 1024 : 1];
    DropKey D = {};
    if (MODE == JOIN_DROP) D = drop_key(A.drop);
    const float inv = 1.0f / (float)A.rows;
    int side = 0;
    for (long turn = blockIdx.x; turn < tile_turns(tiles); turn += gridDim.x) {
        const long tile = tile_of(tiles, turn);
        if (tile >= tiles.count) continue;      // uniform
        float s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = 0.f;
        float4v mean, rstd;
#pragma unroll 1
        for (long r0 = 0; r0 < A.rows; r0 += BLOCK) {
            const TallTile T(min(BLOCK, A.rows - r0), A.cols, tile, r0);
            if (r0 == 0) { mean = T.load_columns(A.stats); rstd = T.load_columns(A.stats + A.cols); }
            float4v x[K], g[K];
            float w[K];
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k)) {
                    x[k] = T.load(A.x + r0 * A.cols, k);
                    g[k] = T.load(A.gy + r0 * A.cols, k);
                    w[k] = A.w[min(r0 + kTallY * k + T.ty, A.rows - 1)];
                }
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k))
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = g[k][e] * w[k];         // 0 where there is no row
                        s[e] += a;
                        s[4 + e] += T.has(k) ? a * ((x[k][e] - mean[e]) * rstd[e]) : 0.f;
                    }
            if constexpr (LONG) set_aside<8>(r0, BLOCK, far, s);
        }
        if constexpr (LONG) add_aside<8>(far, s);
        sum_over_ty<kTallX, kTallY, 8>(s, red[side]);
        side ^= 1;
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] *= inv;
#pragma unroll 1
        for (long r0 = 0; r0 < A.rows; r0 += BLOCK) {
            const TallTile T(min(BLOCK, A.rows - r0), A.cols, tile, r0);
            const long off = r0 * A.cols;
            const bool more = MODE != PLAIN && A.gr;
            float4v x[K], g[K], r[K];
            float w[K];
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k)) {
                    x[k] = T.load(A.x + off, k);
                    g[k] = T.load(A.gy + off, k);
                    if (more) r[k] = T.load(A.gr + off, k);
                    w[k] = A.w[min(r0 + kTallY * k + T.ty, A.rows - 1)];
                }
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (T.any(k)) {
                    float4v v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[e] = rstd[e] * (g[k][e] * w[k] - s[e] - (x[k][e] - mean[e]) * rstd[e] * s[4 + e]);
                        if (more) v[e] += r[k][e];
                    }
                    T.template store<false>(A.gx + off, k, v);
                    if (MODE == JOIN_DROP) v = T.drop(D, k, v);
                    if (MODE != PLAIN && A.gh) T.template store<false>(A.gh + off, k, v);
                }
        }
    }
}

// Columns of any height where there are no four of them, or 128 rows pass 2^32 bytes: TX columns by TY slices of the rows.
template <int MODE, int TX, int TY>
__global__ void __launch_bounds__(TX * TY) k_norm_cols_any(NormFwd A)
{
    constexpr int WAVES = TX * TY / 64;
    __shared__ float red[WAVES][TX][1], red2[WAVES][TX][2];
    DropKey K = {};
    if (MODE == JOIN_DROP) K = drop_key(A.drop);
    const int tx = threadIdx.x % TX, ty = threadIdx.x / TX;
    const float inv = 1.0f / (float)A.rows;
    for (long c0 = (long)blockIdx.x * TX; c0 < A.cols; c0 += (long)gridDim.x * TX) {
        const long c = c0 + tx;
        const long mine = c < A.cols ? A.rows : 0;       // rows that this thread's column has
        const float* src = MODE == PLAIN ? A.x : A.r;
        float sum[1] = {0.f}, d[2] = {0.f, 0.f};
        for (long m = ty; m < mine;) {
            float part = 0.f;
            for (int i = 0; i < kChain && m < mine; ++i, m += TY) {
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
                part += v;
            }
            sum[0] += part;
        }
        sum_over_ty<TX, TY, 1>(sum, red);
        const float m0 = sum[0] * inv;
        for (long m = ty; m < mine;) {
            float p1 = 0.f, p2 = 0.f;
            for (int i = 0; i < kChain && m < mine; ++i, m += TY) { const float v = src[m * A.cols + c] - m0; p1 += v; p2 += v * v; }
            d[0] += p1;
            d[1] += p2;
        }
        sum_over_ty<TX, TY, 2>(d, red2);
        const float delta = d[0] * inv, rstd = inverse_deviation(d[1] * inv, delta, A.eps);
        for (long m = ty; m < mine; m += TY)
            A.y[m * A.cols + c] = ((src[m * A.cols + c] - m0) - delta) * rstd * A.w[m] + A.b[m];
        if (A.stats && mine && ty == 0) { A.stats[c] = m0 + delta; A.stats[A.cols + c] = rstd; }
    }
}

template <int MODE, int TX, int TY>
__global__ void __launch_bounds__(TX * TY) k_norm_cols_bwd_any(NormBwd A)
{
    constexpr int WAVES = TX * TY / 64;
    __shared__ float red[2][WAVES][TX][2];
    DropKey K = {};
    if (MODE == JOIN_DROP) K = drop_key(A.drop);
    const int tx = threadIdx.x % TX, ty = threadIdx.x / TX;
    const float inv = 1.0f / (float)A.rows;
    int side = 0;
    for (long c0 = (long)blockIdx.x * TX; c0 < A.cols; c0 += (long)gridDim.x * TX) {
        const long c = c0 + tx;
        const long mine = c < A.cols ? A.rows : 0;
        const float mean = mine ? A.stats[c] : 0.f, rstd = mine ? A.stats[A.cols + c] : 0.f;
        float s[2] = {0.f, 0.f};
        for (long m = ty; m < mine;) {
            float p1 = 0.f, p2 = 0.f;
            for (int i = 0; i < kChain && m < mine; ++i, m += TY) {
                const float a = A.gy[m * A.cols + c] * A.w[m];
                p1 += a;
                p2 += a * ((A.x[m * A.cols + c] - mean) * rstd);
            }
            s[0] += p1;
            s[1] += p2;
        }
        sum_over_ty<TX, TY, 2>(s, red[side]);
        side ^= 1;
        const float m1 = s[0] * inv, m2 = s[1] * inv;
        for (long m = ty; m < mine; m += TY) {
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
    long span;                      // positions of a share
};

// sums over the four waves of a workgroup, lane by lane
__device__ __forceinline__ float2 slices_sum(float a, float b, float2 (*red)[64])
{
    const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
    __syncthreads();
    red[ty][tx] = make_float2(a, b);
    __syncthreads();
    const float2 v0 = red[0][tx], v1 = red[1][tx], v2 = red[2][tx], v3 = red[3][tx];
    return make_float2((v0.x + v1.x) + (v2.x + v3.x), (v0.y + v1.y) + (v2.y + v3.y));
}

__global__ void __launch_bounds__(256) k_norm_params_rows(NormParams A)
{
    __shared__ float2 red[4][64];
    const long c = (long)blockIdx.x * 64 + (threadIdx.x & 63), r0 = blockIdx.y * A.span;
    const long end = c < A.cols ? min(A.rows, r0 + A.span) : 0;
    float gw = 0.f, gb = 0.f;
    for (long s0 = r0 + (threadIdx.x >> 6); s0 < end; s0 += 4 * kChain) {
        const long s1 = min(end, s0 + 4 * kChain);
        float pw = 0.f, pb = 0.f;
        for (long r = s0; r < s1; r += 4) {
            const float g = A.gy[r * A.cols + c];
            pw += g * ((A.x[r * A.cols + c] - A.stats[r]) * A.stats[A.rows + r]);
            pb += g;
        }
        gw += pw;
        gb += pb;
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
        const float2 s = row_params<256>(A.gy + m * A.cols, A.x + m * A.cols, A.stats, A.stats + A.cols, c0, end, red);
        if (threadIdx.x == 0) {
            float* part = A.parts + (long)blockIdx.y * 2 * A.rows;
            part[m] = s.x;
            part[A.rows + m] = s.y;
        }
    }
}

// 16 of the 2 x features values by 64 slices of the shares, each in ascending order of its shares, eight at a time, then the slices by a fixed
// tree.  Bound by the latency of what other caches just wrote: 2 to 4 us.  Workgroups walk from 2^23 features on: one for every 16 values would be 2^32
// threads at 2^25, more than a launch may have.
__global__ void __launch_bounds__(1024)
k_norm_params(long features, int shares, const float* __restrict__ parts, float* __restrict__ gw, float* __restrict__ gb)
{
    __shared__ float red[16][16];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (long t0 = (long)blockIdx.x * 16; t0 < 2 * features; t0 += (long)gridDim.x * 16) {
        const long t = t0 + tx;
        float v = 0.f;
        if (t < 2 * features)
            for (int s0 = ty; s0 < shares; s0 += 8 * 64) {      // eight requests at once
                float a[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) a[i] = parts[(long)min(s0 + 64 * i, shares - 1) * 2 * features + t];
#pragma unroll
                for (int i = 0; i < 8; ++i) a[i] = s0 + 64 * i < shares ? a[i] : 0.f;
                v += ((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7]));
            }
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
        if ((threadIdx.x & 63) < 16) red[threadIdx.x >> 6][tx] = v;
        __syncthreads();
        if (ty == 0 && t < 2 * features) {
#pragma unroll
            for (int q = 1; q < 16; ++q) v += red[q][tx];
            if (t < features) gw[t] = v; else gb[t - features] = v;
        }
        __syncthreads();
    }
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

// How an array is taken, by its extents alone: kernels that hold a position in registers (`held`) where one fits.
struct Shape {
    bool held;
    int tx, ty; Tiles tiles;                // axis 0
    int lanes, quads, threads;              // axis 1
    long most;                              // workgroups that walk over the positions, at most
    bool few;                               // backward: the parameters' gradients by workgroups of their own, in the same launch
    bool tall;                              // axis 0, not held: tiles that are walked several times
};
// Workgroups that leave shares: `most`, twice, four times as many and so on, until a thread adds up 1024 positions at most in one chain, `each` to a
// turn.  With 1024 10000000 x 64 backward takes 1435 us, with 256 1540.
long share_groups(long most, long positions, long each)
{
    while (most < 65536 && positions > most * each * 1024) most *= 2;
    return most;
}

Shape rows_shape(long rows, long cols, bool backward)
{
    Shape S = {};
    // Few rows: as many as would make the shares of the parameters' gradients as large as the operands.  us, by shares and not: 64 x 1000
    // 6.7 and 2.8, 512 x 1024 7.3 and 4.8, 300 x 12000 25 and 13.5, 1000 x 3505 16.7 and 15.3, 1000 x 1000 8.5 and 11.8.
    S.few = backward && (rows <= 512 || (rows <= 1024 && cols > 2048));
    struct Way { int lanes, quads, threads; long most; };
    // Forward: waves for themselves as long as four quads a lane do.  Backward: a quad or two a lane where the sums of the parameters take
    // registers as well (8192 x 2048 join backward: 256 lanes 64 us, 512 lanes 57).  The last number is the most workgroups that walk.  Forward four
    // times as many give the same, a fourth 12.0 us for 11.2 (16384 x 512) and 580 for 345 (20000 x 10000); backward each leaves a share: twice as many
    // 50000 x 16 8.0 us for 7.3, 5003 x 1001 18.6 for 16.2, 8192 x 2048 40.1 for 36.4, half 20000 x 8000 474 for 355 and 60000 x 60 13.1 for 11.8.
    static constexpr Way forward_ways[] = {{4, 1, 256, 4096}, {16, 1, 256, 4096}, {32, 1, 256, 4096}, {64, 1, 256, 4096}, {64, 2, 256, 4096}, {64, 4, 256, 4096},
                                           {256, 2, 256, 4096}, {256, 4, 256, 4096}, {1024, 2, 1024, 4096}, {1024, 3, 1024, 512}, {1024, 4, 1024, 512}};
    static constexpr Way backward_ways[] = {{4, 1, 256, 512}, {16, 1, 256, 1024}, {32, 1, 512, 512}, {64, 1, 512, 512}, {64, 2, 512, 512}, {64, 4, 512, 256},
                                            {512, 1, 512, 512}, {512, 2, 512, 512}, {1024, 2, 1024, 256}, {1024, 3, 1024, 256}, {1024, 4, 1024, 256}};
    static constexpr Way few_ways[] = {{256, 1, 256, 1024}, {512, 1, 512, 1024}, {512, 2, 512, 1024}, {1024, 2, 1024, 1024}, {1024, 3, 1024, 1024},
                                       {1024, 4, 1024, 1024}};
    auto take = [&](auto& ways) {
        for (const Way& w : ways)
            if (!S.held && cols <= 4L * w.lanes * w.quads) { S.held = true; S.lanes = w.lanes; S.quads = w.quads; S.threads = w.threads; S.most = w.most; }
    };
    if (!backward) take(forward_ways);
    else if (S.few) take(few_ways);
    else take(backward_ways);
    // 512 of them: 1030 x 2000 backward 14.8 us for 12.4, 1200 x 4000 20.6 for 19.1, 1700 x 1700 15.6 for 15.2, but 3000 x 1500 17.6 for 20.4
    if (backward && S.lanes == 512 && rows < 4096) S.most = 256;
    if (backward && S.held) S.most = share_groups(S.most, rows, S.threads / S.lanes);
    return S;
}
Shape cols_shape(long rows, long cols, bool backward)
{
    Shape S = {};
    // Tiles of eight lanes (a line of every row) leave the least to wait for at the end of a launch; sums of the parameters' gradients
    // want fewer, wider ones.  us, TX = 8 and 16: 200 x 30690 forward 13.8 and 17.8, backward 19.4 and 27.0; 120 x 262143 forward 43.9 and 45.7,
    // backward 101 and 87; 40 x 216000 13.6 and 14.3, 31 and 24.  Eight and four rows a thread: 120 x 96^3 forward with dropout 384 and 351.
    S.ty = rows <= 16 ? 4 : rows <= 32 ? 8 : rows <= 64 ? 16 : rows <= 128 ? 32 : rows <= 256 ? 64 : 128;
    S.tx = rows <= 16 ? 64 : rows <= 32 ? 32 : rows <= 128 && backward ? 16 : 8;
    // backward what a chip holds at once of 256, 512 and 1024 threads, for four and eight rows half of it
    S.most = !backward ? 1L << 20 : S.ty == 16 ? 1024 : S.ty == 128 ? 256 : 512;
    // rows on 128-byte lines: 120 x 96^3 backward 265 us in order, 277 apart; forward 193 in order, 176 apart, joined 392 and 349
    S.tiles.apart = cols % 32 != 0 || (!backward && S.tx == 8);
    // us, by shares and not: 40 x 1728 6.3 and 3.5, 120 x 8000 8.0 and 4.7, 40 x 32768 7.7 and 18.9, 400 x 8000 12.4 and 14.1
    S.few = backward && cols <= 12288 && rows <= 256;
    const bool tiled = cols >= 4 && S.ty * cols < (1L << 30) - 16;
    S.held = tiled && rows <= S.ty * kRowsHeld;
    S.tall = tiled && !S.held;
    S.tiles.count = (cols + 4 * S.tx - 1) / (4 * S.tx);
    if (backward && S.held) S.most = share_groups(S.most, cols, S.tx);      // of a tile four columns a lane, one after another
    return S;
}
Shape norm_shape(long rows, long cols, int axis, bool backward) { return axis ? rows_shape(rows, cols, backward) : cols_shape(rows, cols, backward); }

// Workgroups that walk over the positions.  Backward each leaves a share of the parameters' gradients.
long position_groups(const Shape& S, long rows)
{
    if (S.lanes) return std::min((rows + S.threads / S.lanes - 1) / (S.threads / S.lanes), S.most);
    return std::min((S.tiles.count + 7) / 8 * 8, S.most);
}

// Shares of the parameters' gradients, 0 where none are left
int norm_share_count(long rows, long cols, int axis)
{
    const Shape S = norm_shape(rows, cols, axis, true);
    return !S.held ? param_shares(rows, cols, axis).count : S.few ? 0 : (int)position_groups(S, rows);
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
    if (rc == ZNN_OK && (axis ? cols : rows) > kNormFeatures)
        rc = fail(ZNN_EUNSUPPORTED, "a norm over %lld elements is too large", (long long)(axis ? cols : rows));
    return rc;
}

// Calls f with the constants of a shape.
template <int... N> struct Numbers {};
template <bool BACKWARD, class F> void with_cols(const Shape& S, F f)
{
    switch (S.ty) {
        case 4: return f(Numbers<64, 4>{});
        case 8: return f(Numbers<32, 8>{});
        case 16: return f(Numbers<BACKWARD ? 16 : 8, 16>{});
        case 32: return f(Numbers<BACKWARD ? 16 : 8, 32>{});
        case 64: return f(Numbers<8, 64>{});
        default: return f(Numbers<8, 128>{});
    }
}
template <bool BACKWARD, bool FEW, class F> void with_rows(const Shape& S, F f)
{
    if constexpr (!FEW) {
        switch (S.lanes * 8 + S.quads) {
            case 4 * 8 + 1: return f(Numbers<4, 1, 256>{});
            case 16 * 8 + 1: return f(Numbers<16, 1, 256>{});
            case 32 * 8 + 1: return f(Numbers<32, 1, BACKWARD ? 512 : 256>{});
            case 64 * 8 + 1: return f(Numbers<64, 1, BACKWARD ? 512 : 256>{});
            case 64 * 8 + 2: return f(Numbers<64, 2, BACKWARD ? 512 : 256>{});
            case 64 * 8 + 4: return f(Numbers<64, 4, BACKWARD ? 512 : 256>{});
        }
        if constexpr (!BACKWARD) {
            if (S.lanes == 256 && S.quads == 2) return f(Numbers<256, 2, 256>{});
            if (S.lanes == 256) return f(Numbers<256, 4, 256>{});
        }
    } else if (S.lanes == 256) return f(Numbers<256, 1, 256>{});
    if constexpr (BACKWARD) {
        if (S.lanes == 512 && S.quads == 1) return f(Numbers<512, 1, 512>{});
        if (S.lanes == 512) return f(Numbers<512, 2, 512>{});
    }
    if (S.quads == 2) return f(Numbers<1024, 2, 1024>{});
    if (S.quads == 3) return f(Numbers<1024, 3, 1024>{});
    return f(Numbers<1024, 4, 1024>{});
}

bool on_lines(std::initializer_list<const float*> arrays)
{
    for (const float* p : arrays) if ((uintptr_t)p & 127) return false;
    return true;
}
template <int MODE, int TX, int TY> void cols_fwd(const NormFwd& A, const Shape& S, Numbers<TX, TY>, hipStream_t s)
{
    const dim3 grid((unsigned)position_groups(S, A.rows));
    if (A.cols % 32 == 0 && on_lines({A.r, A.y}))
        ZNN_LAUNCH("layer norm forward", s, (k_norm_cols<MODE, TX, TY, true>), grid, dim3(TX * TY), 0, A, S.tiles);
    else ZNN_LAUNCH("layer norm forward", s, (k_norm_cols<MODE, TX, TY, false>), grid, dim3(TX * TY), 0, A, S.tiles);
}
template <int MODE, int TX, int TY, bool PARTS>
void cols_bwd(const NormBwd& A, const Shape& S, Numbers<TX, TY>, float* parts, float* gw, float* gb, hipStream_t s)
{
    const dim3 grid((unsigned)(position_groups(S, A.rows) + (PARTS ? 0 : A.rows)));
    if (A.cols % 32 == 0 && on_lines({A.gx, A.gh}))
        ZNN_LAUNCH("layer norm backward", s, (k_norm_cols_bwd<MODE, TX, TY, true, PARTS>), grid, dim3(TX * TY), 0, A, S.tiles, parts, gw, gb);
    else ZNN_LAUNCH("layer norm backward", s, (k_norm_cols_bwd<MODE, TX, TY, false, PARTS>), grid, dim3(TX * TY), 0, A, S.tiles, parts, gw, gb);
}
template <int MODE, int TX, int TY> void few_cols_bwd(const NormBwd& A, const Shape& S, Numbers<TX, TY> n, float* gw, float* gb, hipStream_t s)
{
    cols_bwd<MODE, TX, TY, false>(A, S, n, nullptr, gw, gb, s);
}
template <int MODE, int TX, int TY>
void sum_cols_bwd(const NormBwd& A, const Shape& S, Numbers<TX, TY> n, float* parts, float* gw, float* gb, hipStream_t s)
{
    cols_bwd<MODE, TX, TY, true>(A, S, n, parts, gw, gb, s);
}
template <int MODE, int L, int NV, int T> void rows_fwd(const NormFwd& A, const Shape& S, Numbers<L, NV, T>, hipStream_t s)
{
    ZNN_LAUNCH("layer norm forward", s, (k_norm_rows<MODE, L, NV, T>), dim3((unsigned)position_groups(S, A.rows)), dim3(T), 0, A);
}
template <int MODE, bool PARTS, int L, int NV, int T>
void rows_bwd(const NormBwd& A, const Shape& S, Numbers<L, NV, T>, float* parts, float* gw, float* gb, hipStream_t s)
{
    const long others = PARTS ? 0 : (A.cols + 31) / 32;
    ZNN_LAUNCH("layer norm backward", s, (k_norm_rows_bwd<MODE, L, NV, T, PARTS>), dim3((unsigned)(position_groups(S, A.rows) + others)), dim3(T), 0, A,
               parts, gw, gb);
}

template <int MODE>
int norm_fwd(const NormFwd& A, int axis, hipStream_t s)
{
    const Shape S = norm_shape(A.rows, A.cols, axis, false);
    if (S.held && axis) with_rows<false, false>(S, [&](auto n) { rows_fwd<MODE>(A, S, n, s); });
    else if (S.held) with_cols<false>(S, [&](auto n) { cols_fwd<MODE>(A, S, n, s); });
    else if (axis) {
        const dim3 grid(groups_of(A.rows, 1, 1L << 20));
        if (A.cols > kLongRow) ZNN_LAUNCH("layer norm forward", s, (k_norm_rows_any<MODE, true>), grid, dim3(1024), 0, A);
        else ZNN_LAUNCH("layer norm forward", s, (k_norm_rows_any<MODE, false>), grid, dim3(1024), 0, A);
    } else if (S.tall) {
        const dim3 grid((unsigned)position_groups(S, A.rows));
        if (A.rows > kLongColumn) ZNN_LAUNCH("layer norm forward", s, (k_norm_cols_tall<MODE, true>), grid, dim3(1024), 0, A, S.tiles);
        else ZNN_LAUNCH("layer norm forward", s, (k_norm_cols_tall<MODE, false>), grid, dim3(1024), 0, A, S.tiles);
    } else if (A.cols < 4) ZNN_LAUNCH("layer norm forward", s, (k_norm_cols_any<MODE, 4, 256>), dim3(1), dim3(1024), 0, A);
    else ZNN_LAUNCH("layer norm forward", s, (k_norm_cols_any<MODE, 64, 4>), dim3(groups_of(A.cols, 64, 1L << 20)), dim3(256), 0, A);
    return check_launch("layer norm forward");
}

template <int MODE>
int norm_bwd(const NormBwd& A, int axis, float* gw, float* gb, void* ws, hipStream_t s)
{
    const Shape H = norm_shape(A.rows, A.cols, axis, true);
    const long features = axis ? A.cols : A.rows;
    float* const parts = (float*)ws;
    if (H.held && H.few) {
        if (axis) with_rows<true, true>(H, [&](auto n) { rows_bwd<MODE, false>(A, H, n, parts, gw, gb, s); });
        else with_cols<true>(H, [&](auto n) { few_cols_bwd<MODE>(A, H, n, gw, gb, s); });
        return check_launch("layer norm backward");
    }
    if (H.held && axis) with_rows<true, false>(H, [&](auto n) { rows_bwd<MODE, true>(A, H, n, parts, gw, gb, s); });
    else if (H.held) with_cols<true>(H, [&](auto n) { sum_cols_bwd<MODE>(A, H, n, parts, gw, gb, s); });
    else {
        const Shares S = param_shares(A.rows, A.cols, axis);
        const NormParams P = {A.rows, A.cols, A.gy, A.x, A.stats, parts, S.span};
        if (axis) {
            const dim3 grid(groups_of(A.rows, 1, 1L << 20));
            if (A.cols > kLongRow) ZNN_LAUNCH("layer norm backward", s, (k_norm_rows_bwd_any<MODE, true>), grid, dim3(1024), 0, A);
            else ZNN_LAUNCH("layer norm backward", s, (k_norm_rows_bwd_any<MODE, false>), grid, dim3(1024), 0, A);
            ZNN_LAUNCH("layer norm parameters", s, k_norm_params_rows, dim3((unsigned)((A.cols + 63) / 64), (unsigned)S.count), dim3(256), 0, P);
        } else {
            const dim3 grid((unsigned)position_groups(H, A.rows));
            if (H.tall && A.rows > kLongColumn) ZNN_LAUNCH("layer norm backward", s, (k_norm_cols_bwd_tall<MODE, true>), grid, dim3(1024), 0, A, H.tiles);
            else if (H.tall) ZNN_LAUNCH("layer norm backward", s, (k_norm_cols_bwd_tall<MODE, false>), grid, dim3(1024), 0, A, H.tiles);
            else if (A.cols < 4) ZNN_LAUNCH("layer norm backward", s, (k_norm_cols_bwd_any<MODE, 4, 256>), dim3(1), dim3(1024), 0, A);
            else ZNN_LAUNCH("layer norm backward", s, (k_norm_cols_bwd_any<MODE, 64, 4>), dim3(groups_of(A.cols, 64, 1L << 20)), dim3(256), 0, A);
            ZNN_LAUNCH("layer norm parameters", s, k_norm_params_cols, dim3(groups_of(A.rows, 1, 1L << 20), (unsigned)S.count), dim3(256), 0, P);
        }
    }
    ZNN_LAUNCH("layer norm parameters", s, k_norm_params, dim3(groups_of(2 * features, 16, 1L << 20)), dim3(1024), 0, features,
               norm_share_count(A.rows, A.cols, axis), (const float*)parts, gw, gb);
    return check_launch("layer norm backward");
}

int launch_dropout(long rows, long cols, const Drop& D, bool drops, const float* x, float* y, hipStream_t s)
{
    const long quads = (cols + 3) / 4;
    if (drops) ZNN_LAUNCH("dropout", s, k_dropout, dim3(groups_of(rows * quads, 256, 1L << 20)), dim3(256), 0, rows, cols, quads, D, x, y);
    else ZNN_LAUNCH("dropout", s, k_copy, dim3(groups_of(rows * cols, 1024, 1L << 20)), dim3(256), 0, rows * cols, x, y);
    return check_launch("dropout");
}

}  // namespace

size_t norm_workspace(long rows, long cols, int axis)
{
    return sizeof(float) * 2 * norm_share_count(rows, cols, axis) * (axis ? cols : rows);
}

int dropout_parts(long rows, long cols, unsigned dropped, const uint64_t* state, uint32_t site, const float* x, float* y, hipStream_t s)
{
    Drop D;
    bool drops;
    const int rc = make_drop_parts(dropped, state, site, &D, &drops);
    return rc != ZNN_OK ? rc : launch_dropout(rows, cols, D, drops, x, y, s);
}

int join_parts(long rows, long cols, float eps, unsigned dropped, const uint64_t* state, uint32_t site, const float* h, const float* x,
               const float* w, const float* b, float* r, float* y, float* stats, hipStream_t s)
{
    Drop D;
    bool drops;
    const int rc = make_drop_parts(dropped, state, site, &D, &drops);
    if (rc != ZNN_OK) return rc;
    const NormFwd A = {rows, cols, h, x, w, b, r, y, stats, eps, D};
    return drops ? norm_fwd<JOIN_DROP>(A, 0, s) : norm_fwd<JOIN>(A, 0, s);
}

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
    return launch_dropout((long)rows, (long)cols, D, drops, x, y, (hipStream_t)stream);
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
