// Gated unit y = fn(W x + b) (V x + c) and its Jacobian.
#include "gate.h"
#include "split_parts.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace znn {
namespace {

// fn(u) and its derivative.  That is 1.13 at most, so du = gy (v d) takes it first: gy v may leave the range where du does not, and is no number times a d of 0 then.
struct Gated { float a, d; };

constexpr float kLargestFloat = 3.402823466e38f;

// Values at infinity are limits: an infinite u times a factor of 0 would not be.
template <int FN>
__device__ __forceinline__ Gated gate_fn(float u)
{
    if (FN == ZNN_GATE_RECTIFY) return Gated{u > 0.f ? u : 0.f, u > 0.f ? 1.f : 0.f};
    if (FN == ZNN_GATE_TANH) {
        // f - k of the logistic function at 2 u; below 0.35, where that would lose digits, the series of tanh, whose next term is below 2^-26 there
        const Gate g = gate(2.f * u);
        const float s = u * u;
        float p = fmaf(s, 21844.f / 6081075.f, -1382.f / 155925.f);
        p = fmaf(s, p, 62.f / 2835.f);
        p = fmaf(s, p, -17.f / 315.f);
        p = fmaf(s, p, 2.f / 15.f);
        p = fmaf(s, p, -1.f / 3.f);
        return Gated{fabsf(u) < 0.35f ? fmaf(u * s, p, u) : g.f - g.k, 4.f * g.f * g.k};       // 1 - tanh^2 without its cancellation
    }
    const float finite = __builtin_amdgcn_fmed3f(u, -kLargestFloat, kLargestFloat);
    if (FN == ZNN_GATE_GELU) {
        const float p = 0.5f * erfcf(-0.707106781f * u);       // NaN comes from here: `finite` has a number in its place
        return Gated{u > 0.f ? u * p : finite * p, fmaf(finite, 0.398942280f * expf(-0.5f * finite * finite), p)};
    }
    const Gate g = gate(u);
    if (FN == ZNN_GATE_LOGISTIC) return Gated{g.f, g.f * g.k};
    return Gated{fmaxf(u, -kLargestFloat) * g.f, fmaf(finite, g.f * g.k, g.f)};      // NaN comes from g
}

// f with the function's number as a constant
template <class F>
__device__ __forceinline__ void with_fn(int fn, F f)
{
    switch (fn) {
        case ZNN_GATE_RECTIFY: return f(std::integral_constant<int, ZNN_GATE_RECTIFY>{});
        case ZNN_GATE_LOGISTIC: return f(std::integral_constant<int, ZNN_GATE_LOGISTIC>{});
        case ZNN_GATE_TANH: return f(std::integral_constant<int, ZNN_GATE_TANH>{});
        case ZNN_GATE_SILU: return f(std::integral_constant<int, ZNN_GATE_SILU>{});
        default: return f(std::integral_constant<int, ZNN_GATE_GELU>{});
    }
}

// ---------------------------------------------------------------- products of matrices
// C[i][j] = sum over k of A[i][k] B[j][k] on the fp32 matrix cores, rows j of C contiguous.  A workgroup of WI x WJ waves makes a tile of
// 32 WI AI x 32 WJ AJ results, a wave AI x AJ of 32 x 32.  Both operands go through shared memory as [row][kDepth] in quads along k, whatever way they lie
// in memory; while one step is multiplied the next one's loads are in flight.  Quads of a row change places by the row's number: eight lanes, a
// clock's worth, that read a quad of eight rows or write one of rows four apart touch different banks.
// Bound by the matrix cores: 93 TFLOP/s with three workgroups on a unit.
// v_mfma_f32_32x32x2_f32 takes k = lane / 32; which k that stands for is free as long as both operands agree: lanes below 32 take the first
// quad of eight k, the others the second one, so that a quad feeds four instructions.

typedef float floatx16 __attribute__((ext_vector_type(16)));
using split::bf16x8;
using split::floatx4;
using split::uintx4;
typedef float floatu2 __attribute__((ext_vector_type(2), aligned(4)));
typedef float floatu4 __attribute__((ext_vector_type(4), aligned(4)));      // rows begin at any element

constexpr int kDepth = 32;

// Element (row, k) of an operand at p + row * ld + k (ALONG_K) or at p + k * ld + row.
struct Operand { const float* p; long ld; };

__device__ __forceinline__ int quad_place(int row, int quad) { return row * kDepth + ((quad ^ (row & 7) ^ (row >> 3 & 3)) << 2); }

// A tile's row in the operand.  Halves: 32 rows of the first half lie beside the same rows of the second one, `half` rows on.
template <bool HALVES>
__device__ __forceinline__ long source_row(long first, int row, long rows, long half)
{
    const long r = first + (HALVES ? (row >> 6) * 32 + (row & 31) : row);
    return (r < rows ? r : rows - 1) + (HALVES && (row & 32) ? half : 0);
}

// R rows from `first` on (of `rows`), kDepth k from k0 on (k < K; 0 behind), on their way into shared memory.
template <int R, int THREADS, bool ALONG_K, bool HALVES>
struct Stage {
    static constexpr int kPieces = (R * kDepth / 4 + THREADS - 1) / THREADS;        // quads of a thread
    static constexpr int kBlocks = (R * kDepth / 16 + THREADS - 1) / THREADS;       // or blocks of 4 x 4
    floatx4 v[ALONG_K ? kPieces : 4 * kBlocks];

    __device__ __forceinline__ void load(const Operand& O, long first, long rows, long half, long k0, long K)
    {
        if (ALONG_K) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int e = threadIdx.x + i * THREADS, row = e / (kDepth / 4), quad = e % (kDepth / 4);
                if (R * kDepth / 4 % THREADS && row >= R) break;
                const long k = k0 + quad * 4;
                const float* p = O.p + source_row<HALVES>(first, row, rows, half) * O.ld + k;
                if (k0 + kDepth <= K) v[i] = *(const floatu4*)p;
                else
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[i][c] = k + c < K ? p[c] : 0.f;
            }
        } else {
            const bool whole = k0 + kDepth <= K && first + R <= rows;
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
                const int e = threadIdx.x + i * THREADS, row = e % (R / 4) * 4, quad = e / (R / 4);
                if (R * kDepth / 16 % THREADS && quad >= kDepth / 4) break;
                const long r = first + row, k = k0 + quad * 4;
                const float* p = O.p + k * O.ld + r;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if (whole) v[4 * i + c] = *(const floatu4*)(p + c * O.ld);
                    else
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[4 * i + c][j] = k + c < K && r + j < rows ? p[c * O.ld + j] : 0.f;
                }
            }
        }
    }
    __device__ __forceinline__ void store(float* lds) const
    {
        if (ALONG_K) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int e = threadIdx.x + i * THREADS, row = e / (kDepth / 4), quad = e % (kDepth / 4);
                if (R * kDepth / 4 % THREADS && row >= R) break;
                *(floatx4*)(lds + quad_place(row, quad)) = v[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
                const int e = threadIdx.x + i * THREADS, row = e % (R / 4) * 4, quad = e / (R / 4);
                if (R * kDepth / 16 % THREADS && quad >= kDepth / 4) break;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *(floatx4*)(lds + quad_place(row + j, quad)) = floatx4{v[4 * i][j], v[4 * i + 1][j], v[4 * i + 2][j], v[4 * i + 3][j]};
            }
        }
    }
};

enum Halves { NO_HALVES, HALVES_I, HALVES_J };
template <int WI_, int WJ_, int AI_, int AJ_> struct Waves {
    static constexpr int WI = WI_, WJ = WJ_, AI = AI_, AJ = AJ_, kThreads = 64 * WI * WJ, TI = 32 * WI * AI, TJ = 32 * WJ * AJ;
};

struct Matrices { Operand A, B; long rows_i, rows_j, half, k0, K; };     // rows that there are (of a half); the sum goes over k0 <= k < K

template <class W, bool A_ALONG, bool B_ALONG, Halves H>
__device__ __forceinline__ void tile_product(floatx16 (&acc)[W::AI][W::AJ], const Matrices& M, long i0, long j0)
{
    __shared__ float lds[2][(W::TI + W::TJ) * kDepth];
    Stage<W::TI, W::kThreads, A_ALONG, H == HALVES_I> a;
    Stage<W::TJ, W::kThreads, B_ALONG, H == HALVES_J> b;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 31, side = lane >> 5;
    const int wi = wave / W::WJ * (32 * W::AI) + row, wj = W::TI + wave % W::WJ * (32 * W::AJ) + row;
#pragma unroll
    for (int x = 0; x < W::AI; ++x)
#pragma unroll
        for (int y = 0; y < W::AJ; ++y)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[x][y][r] = 0.f;
    a.load(M.A, i0, M.rows_i, M.half, M.k0, M.K);
    b.load(M.B, j0, M.rows_j, M.half, M.k0, M.K);
    a.store(lds[0]);
    b.store(lds[0] + W::TI * kDepth);
    __syncthreads();
    int buffer = 0;
    for (long k = M.k0; k < M.K; k += kDepth) {
        const bool more = k + kDepth < M.K;
        if (more) {
            a.load(M.A, i0, M.rows_i, M.half, k + kDepth, M.K);
            b.load(M.B, j0, M.rows_j, M.half, k + kDepth, M.K);
        }
        const float* const from = lds[buffer];
#pragma unroll
        for (int q = 0; q < kDepth / 8; ++q) {
            floatx4 u[W::AI], v[W::AJ];
#pragma unroll
            for (int x = 0; x < W::AI; ++x) u[x] = *(const floatx4*)(from + quad_place(wi + 32 * x, 2 * q + side));
#pragma unroll
            for (int y = 0; y < W::AJ; ++y) v[y] = *(const floatx4*)(from + W::TI * kDepth + quad_place(wj - W::TI + 32 * y, 2 * q + side));
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int x = 0; x < W::AI; ++x)
#pragma unroll
                    for (int y = 0; y < W::AJ; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x2f32(u[x][s], v[y][s], acc[x][y], 0, 0, 0);
        }
        if (more) {
            buffer ^= 1;
            a.store(lds[buffer]);
            b.store(lds[buffer] + W::TI * kDepth);
        }
        __syncthreads();
    }
}

// Register r of a 32 x 32 result belongs to this row and to column lane % 32.
__device__ __forceinline__ int result_row(int r) { return r / 4 * 8 + (threadIdx.x >> 5 & 1) * 4 + r % 4; }

// Tiles in the order of their numbers: those of one XCD (number mod 8 as workgroups are dealt) are neighbours, eight rows of tiles at a time.
struct Tiles { unsigned ni, nj, count; };
struct TilePlace { unsigned i, j; };
__device__ __forceinline__ TilePlace tile_place(const Tiles& T, unsigned number)
{
    const unsigned each = T.count / 8, rest = T.count % 8, xcd = number % 8, nth = number / 8;
    const unsigned t = xcd * each + (xcd < rest ? xcd : rest) + nth;
    const unsigned band = t / (8 * T.nj), first = band * 8, high = T.ni - first < 8 ? T.ni - first : 8, in = t - first * T.nj;
    return TilePlace{first + in % high, in / high};
}

// ---------------------------------------------------------------- the same on the bf16 matrix cores
// Operands as three bf16 parts each (split_parts.h), six products of a step of 32 k: the work of the fp32 instruction in 96 clocks of 256.
// A workgroup of WI x 2 waves makes a tile of 64 WI x 128 results, a wave 64 x 64 of them as 4 x 4 tiles of 16 x 16.  Values are taken apart on their way into
// shared memory, [part][row][32 k], of which there are two: while one step is multiplied, the next one is taken apart between its instructions, a
// pair of values at a time, and the loads of the one behind it are issued as soon as registers are free for them.
// Results lie with their rows (the instruction's first operand) along j, so that a lane has four neighbours of a row of C.
// Bound by the matrix cores, 56 to 60 % busy at 1.9 GHz: 8192 x 1024 from 8192 terms in 630 to 670 us as the card's clock has it, 205 to 218 TFLOP/s of fp32 work; vector
// instructions take half of the time beside.

constexpr int kSplitColumns = 128, kSplitWaves = 4;     // rows of waves

// Octet of eight k of a row: eight lanes, a clock's worth, read one octet of eight rows, and take different banks.
__device__ __forceinline__ int octet_place(int row, int octet) { return row * 64 + ((octet ^ (row >> 1 & 3)) << 4); }

// The octets of an operand that a thread moves: one row each (ALONG_K), or one or two neighbouring rows of one octet.
template <int R, int THREADS, bool ALONG_K, bool HALVES>
struct SplitStage {
    static constexpr int kUnits = R * 4 / THREADS, kPart = R * 64;      // bytes of a part
    static_assert(kUnits == 1 || kUnits == 2, "one or two octets of a thread");
    float v[kUnits][8];
    unsigned w[4];
    const float* p[kUnits];         // ALONG_K: the thread's next octets
    const float* base;              // else: row `first` of the next step's first k of this wave's octet
    unsigned at;                    // and this thread's (first) row behind it: rows behind the last one are not moved, several threads move the last ones

    __device__ __forceinline__ static int octet() { return ALONG_K ? threadIdx.x % 4 : __builtin_amdgcn_readfirstlane(threadIdx.x / (THREADS / 4)); }
    __device__ __forceinline__ static int row(int unit)
    {
        return ALONG_K ? threadIdx.x / 4 + THREADS / 4 * unit : threadIdx.x % (THREADS / 4) * kUnits + unit;
    }
    __device__ __forceinline__ void begin(const Operand& O, long first, long rows, long half, long k0)
    {
        if (ALONG_K)
#pragma unroll
            for (int u = 0; u < kUnits; ++u) p[u] = O.p + source_row<HALVES>(first, row(u), rows, half) * O.ld + k0 + octet() * 8;
        else {
            base = O.p + (k0 + octet() * 8) * O.ld + first;
            const long left = rows - first, r = row(0), most = left < kUnits ? 0 : left - kUnits;
            at = (unsigned)(r < most ? r : most);
        }
    }
    // steps that are there as a whole
    __device__ __forceinline__ void load(int unit, const Operand& O)
    {
        if (ALONG_K) {
            *(floatx4*)v[unit] = *(const floatu4*)p[unit];
            *(floatx4*)(v[unit] + 4) = *(const floatu4*)(p[unit] + 4);
            p[unit] += kDepth;
        } else if (unit == kUnits - 1) {
            const float* q = base;
#pragma unroll
            for (int c = 0; c < 8; ++c, q += O.ld) {
                if (kUnits == 2) {
                    const floatu2 two = *(const floatu2*)(q + at);
                    v[0][c] = two[0];
                    v[kUnits - 1][c] = two[1];
                } else v[0][c] = q[at];
            }
            base += kDepth * O.ld;
        }
    }
    __device__ __forceinline__ static bool whole(long first, long rows) { return ALONG_K || first + kUnits <= rows; }
    // any step: `left` k are there of the operand from its first one on
    __device__ __forceinline__ void load_some(const Operand& O, long first, long rows, long left)
    {
        const int most = (int)(left < kDepth ? left : kDepth) - octet() * 8;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const float* const q = ALONG_K ? p[u] : base + at + u;
            const bool there = ALONG_K || first + at + u < rows;
#pragma unroll
            for (int c = 0; c < 8; ++c) v[u][c] = there && c < most ? q[ALONG_K ? c : c * O.ld] : 0.f;
            if (ALONG_K) p[u] += kDepth;
        }
        if (!ALONG_K) base += kDepth * O.ld;
    }
    // twelve pieces of work a unit
    __device__ __forceinline__ void take(char* lds, int piece, float scale)
    {
        const int unit = piece / 12, part = piece % 12 / 4, pair = piece % 4;
        float &x = v[unit][2 * pair], &y = v[unit][2 * pair + 1];
        if (part == 0) { x *= scale; y *= scale; }
        w[pair] = split::take_part(x, y);
        if (pair == 3) *(uintx4*)(lds + part * kPart + octet_place(ALONG_K ? row(unit) : at + unit, octet())) = uintx4{w[0], w[1], w[2], w[3]};
    }
};

// Six products of a step, from zero, smallest first, of one operand (u) with those of four (v) from FROM to TO; meanwhile acc += sign before, which are the
// products before, and request(slot), slot = 0, 1 .., between any two instructions.  ROWS_V: the results' rows are v's.
template <bool ROWS_V, int FROM, int TO, class Request>
__device__ __forceinline__ void products(floatx4 (&t)[4], const bf16x8 (&v)[4][3], const uintx4 (&u)[3], const floatx4 (&before)[4], float sign,
                                         floatx4 (&acc)[4], Request request)
{
    constexpr int of_v[6] = {0, 2, 1, 0, 1, 0}, of_u[6] = {2, 0, 1, 1, 0, 0};
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = 0; g < 6; ++g)
#pragma unroll
        for (int y = FROM; y < TO; ++y) {
            const bf16x8 one = __builtin_bit_cast(bf16x8, u[of_u[g]]);
            const floatx4 c = g ? t[y] : floatx4{0.f, 0.f, 0.f, 0.f};
            t[y] = ROWS_V ? split::mfma(v[y][of_v[g]], one, c) : split::mfma(one, v[y][of_v[g]], c);
            request(g * (TO - FROM) + y - FROM);
            if (g >= 1 && g <= 4) acc[y][g - 1] = fmaf(before[y][g - 1], sign, acc[y][g - 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
}

// acc[x][y], of the wave's 64 x 64: rows i = 16 x + lane % 16 and columns j = 16 y + lane / 16 * 4 + 0 .. 3, or (TURNED) rows
// i = 16 x + lane / 16 * 4 + 0 .. 3 and columns j = 16 y + lane % 16
template <int WI, bool A_ALONG, bool B_ALONG, Halves H, bool TURNED>
__device__ __forceinline__ void split_product(floatx4 (&acc)[4][4], const Matrices& M, long i0, long j0)
{
    typedef SplitStage<64 * WI, 128 * WI, A_ALONG, H == HALVES_I> StageA;
    typedef SplitStage<kSplitColumns, 128 * WI, B_ALONG, H == HALVES_J> StageB;
    constexpr int kBytes = 3 * (StageA::kPart + StageB::kPart), kPieces = 12 * (StageA::kUnits + StageB::kUnits);
    __shared__ __attribute__((aligned(16))) char lds[2 * kBytes];
    StageA a;
    StageB b;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, octet = lane >> 4;
    const int from_a = octet_place(wave / 2 * 64 + row, octet), from_b = 3 * StageA::kPart + octet_place(wave % 2 * 64 + row, octet);
    floatx4 t[2][4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        t[1][x] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < 4; ++y) acc[x][y] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const long steps = (M.K - M.k0 + kDepth - 1) / kDepth;
    // steps from there on are loaded by parts
    const long plain = a.whole(i0, M.rows_i) && b.whole(j0, M.rows_j) ? (M.K - M.k0) / kDepth : 0;
    auto load = [&](long step) {
        if (step < plain) {
#pragma unroll
            for (int u = 0; u < StageA::kUnits; ++u) a.load(u, M.A);
#pragma unroll
            for (int u = 0; u < StageB::kUnits; ++u) b.load(u, M.B);
        } else if (step < steps) {
            a.load_some(M.A, i0, M.rows_i, M.K - M.k0 - step * kDepth);
            b.load_some(M.B, j0, M.rows_j, M.K - M.k0 - step * kDepth);
        }
    };
    auto take = [&](char* to, int piece, float sign) {
        if (piece < 12 * StageA::kUnits) a.take(to, piece, sign * split::kScale);
        else b.take(to + 3 * StageA::kPart, piece - 12 * StageA::kUnits, split::kScale);
    };
    a.begin(M.A, i0, M.rows_i, M.half, M.k0);
    b.begin(M.B, j0, M.rows_j, M.half, M.k0);
    load(0);
#pragma unroll
    for (int n = 0; n < kPieces; ++n) take(lds, n, 1.f);
    load(1);
    __syncthreads();
    float sign = 1.f;
    // One step: its products, and between them the next one taken apart (TAKES) and the loads of the one behind that (LOADS).
    auto step = [&](auto takes, auto loads, const char* here, char* next) {
        bf16x8 v[4][3];
        uintx4 u[2][3];
#pragma unroll
        for (int part = 0; part < 3; ++part) u[0][part] = *(const uintx4*)(here + part * StageA::kPart + from_a);
        auto fetch = [&](int y, int part) {
            v[y][part] = __builtin_bit_cast(bf16x8, *(const uintx4*)(here + part * StageB::kPart + from_b + 1024 * y));
        };
#pragma unroll
        for (int n = 0; n < 6; ++n) fetch(n / 3, n % 3);
        // what is done between the instructions of a step, n = 0 .. 95 of them
        auto between = [&](int n) {
            constexpr int kFirst = 12, kEach = (96 - kFirst) / kPieces;
            const int x = n / 24, slot = n % 24;
            if (n < 6) fetch(2 + n / 3, n % 3);
            if (x < 3 && slot >= 6 && slot < 9) u[~x & 1][slot - 6] = *(const uintx4*)(here + (slot - 6) * StageA::kPart + from_a + 1024 * (x + 1));
            const int piece = (n - kFirst) / kEach;
            if (takes.value && n >= kFirst && (n - kFirst) % kEach == 0 && piece < kPieces) {
                take(next, piece, -sign);
                if (loads.value && piece % 12 == 11) {
                    if (piece < 12 * StageA::kUnits) a.load(piece / 12, M.A);
                    else b.load(piece / 12 - StageA::kUnits, M.B);
                }
            }
        };
        // two columns first: all waves read their operands behind the barrier, and two need fewer of them
        products<!TURNED, 0, 2>(t[0], v, u[0], t[1], -sign, acc[3], [&](int slot) { between(slot); });
        products<!TURNED, 2, 4>(t[0], v, u[0], t[1], -sign, acc[3], [&](int slot) { between(12 + slot); });
#pragma unroll
        for (int x = 1; x < 4; ++x)
            products<!TURNED, 0, 4>(t[x & 1], v, u[x & 1], t[~x & 1], sign, acc[x - 1], [&](int slot) { between(24 * x + slot); });
        sign = -sign;
    };
    typedef std::integral_constant<bool, true> Yes;
    typedef std::integral_constant<bool, false> No;
    long n = 0;
    auto here = [&] { return lds + (n & 1) * kBytes; };
    auto next = [&] { return lds + (~n & 1) * kBytes; };
    for (; n + 2 < plain; ++n) {
        step(Yes{}, Yes{}, here(), next());
        __syncthreads();
    }
    for (; n + 1 < steps; ++n) {
        step(Yes{}, No{}, here(), next());
        load(n + 2);
        __syncthreads();
    }
    step(No{}, No{}, here(), next());
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        split::add_signed<0>(acc[3][y], t[1][y], -sign);
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[x][y] *= split::kUnscale;
    }
}

// A result that is not finite is taken again from memory: parts of infinite operands are no numbers, and sums are 2^32 too large until they are done.
__device__ __noinline__ float again(const float* a, long step_a, const float* b, long step_b, long count)
{
    float s = 0.f;
    for (long k = 0; k < count; ++k, a += step_a, b += step_b) s = fmaf(*a, *b, s);
    return s;
}
template <bool A_ALONG, bool B_ALONG>
__device__ __forceinline__ float again(const Matrices& M, long row_a, long row_b)
{
    const long step_a = A_ALONG ? 1 : M.A.ld, step_b = B_ALONG ? 1 : M.B.ld;
    return again(M.A.p + row_a * (A_ALONG ? M.A.ld : 1) + M.k0 * step_a, step_a, M.B.p + row_b * (B_ALONG ? M.B.ld : 1) + M.k0 * step_b, step_b, M.K - M.k0);
}
__device__ __forceinline__ void store4(float* p, const floatx4& v, int most)
{
    if (most == 4) *(floatu4*)p = v;
    else
#pragma unroll
        for (int r = 0; r < 3; ++r)
            if (r < most) p[r] = v[r];
}
__device__ __forceinline__ floatx4 load4(const float* p, int most)
{
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    if (most == 4) v = *(const floatu4*)p;
    else
#pragma unroll
        for (int r = 0; r < 3; ++r)
            if (r < most) v[r] = p[r];
    return v;
}
__device__ __forceinline__ bool finite(float v) { return fabsf(v) <= split::kLargest; }

template <int C> __device__ __forceinline__ void store_some(float* p, const float (&v)[C], int most)
{
    typedef float vector __attribute__((ext_vector_type(C), aligned(4)));
    if (most == C) {
        vector q;
#pragma unroll
        for (int c = 0; c < C; ++c) q[c] = v[c];
        *(vector*)p = q;
    } else
#pragma unroll
        for (int c = 0; c < C - 1; ++c)
            if (c < most) p[c] = v[c];
}

struct Element { long feature, position; };

// What the split products leave of a gated unit: C neighbours of N groups, finished together.  place(g): feature and position of a group's first one;
// dots(feature, position, u, v) takes both sums again; at(g): where the group lies in y and in kept (and how far apart its halves), and how many are there.
struct Spot { long y, kept; int most; };
template <int N, int C, int AXIS, class Place, class Again, class At>
__device__ __forceinline__ void finish(int fn, const float* bias, int fo, long half, float* y, float* kept, float (&u)[N][C], float (&v)[N][C], Place place, Again dots, At at)
{
    // 0 times any number is 0 but for infinities and NaN
    float test = 0.f;
#pragma unroll
    for (int g = 0; g < N; ++g) {
        const int most = at(g).most;
#pragma unroll
        for (int c = 0; c < C; ++c) test = fmaf(v[g][c], 0.f, fmaf(u[g][c], 0.f, test));
        if (bias && most > 0) {
            const float* const b = bias + place(g).feature;
            if (AXIS) {
                const floatx4 bu = load4(b, most), bv = load4(b + fo, most);
#pragma unroll
                for (int c = 0; c < C; ++c) { u[g][c] += bu[c & 3]; v[g][c] += bv[c & 3]; }
            } else {
                const float bu = *b, bv = b[fo];
#pragma unroll
                for (int c = 0; c < C; ++c) { u[g][c] += bu; v[g][c] += bv; }
            }
        }
    }
    float out[N][C];
    with_fn(fn, [&](auto number) {
#pragma unroll
        for (int g = 0; g < N; ++g)
#pragma unroll
            for (int c = 0; c < C; ++c) out[g][c] = gate_fn<number.value>(u[g][c]).a * v[g][c];
    });
    unsigned bad_u = 0, bad_v = 0;
#pragma unroll
    for (int g = 0; g < N; ++g) {
        const Spot s = at(g);
        if (s.most <= 0) continue;
        store_some(y + s.y, out[g], s.most);
        if (kept) {
            store_some(kept + s.kept, u[g], s.most);
            store_some(kept + s.kept + half, v[g], s.most);
        }
        if (test != 0.f)
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c < s.most) {
                    bad_u |= (unsigned)!finite(u[g][c]) << (C * g + c);
                    bad_v |= (unsigned)!finite(v[g][c]) << (C * g + c);
                }
    }
#pragma unroll 1
    for (unsigned e = 0; e < N * C && (bad_u | bad_v) >> e; ++e) {
        if (!((bad_u | bad_v) >> e & 1)) continue;
        const Element p = place(e / C);
        const Spot s = at(e / C);
        const long c = e % C, feature = p.feature + (AXIS ? c : 0);
        float a, b;
        dots(feature, p.position + (AXIS ? 0 : c), a, b);
        if (bias) {
            a += bias[feature];
            b += bias[fo + feature];
        }
        with_fn(fn, [&](auto number) { y[s.y + c] = gate_fn<number.value>(a).a * b; });
        if (kept && (bad_u >> e & 1)) kept[s.kept + c] = a;
        if (kept && (bad_v >> e & 1)) kept[s.kept + half + c] = b;
    }
}

struct GatedFwd { Matrices M; Tiles T; int fn, fo; const float* bias; float *y, *kept; long ld; };      // rows of y are ld elements apart

// AXIS 0: i = features (halves), j = positions.  AXIS 1: i = positions, j = features (halves); rows of `kept` hold both halves.
template <class W, int AXIS>
__global__ void __launch_bounds__(W::kThreads) k_gated_fwd(GatedFwd G)
{
    const TilePlace P = tile_place(G.T, blockIdx.x);
    const long i0 = (long)P.i * (AXIS ? W::TI : W::TI / 2), j0 = (long)P.j * (AXIS ? W::TJ / 2 : W::TJ);
    floatx16 acc[W::AI][W::AJ];
    tile_product<W, true, AXIS == 1, AXIS ? HALVES_J : HALVES_I>(acc, G.M, i0, j0);
    const int wave = threadIdx.x >> 6, wi = wave / W::WJ, wj = wave % W::WJ, column = threadIdx.x & 31;
    static_assert(AXIS ? W::AJ == 2 : W::AI == 2, "a wave holds both halves");
#pragma unroll
    for (int n = 0; n < (AXIS ? W::AI : W::AJ); ++n) {
        floatx16 &us = AXIS ? acc[n][0] : acc[0][n], &vs = AXIS ? acc[n][1] : acc[1][n];
        const long first = i0 + (AXIS ? wi * (32 * W::AI) + 32 * n : wi * 32), j = j0 + (AXIS ? wj * 32 : wj * (32 * W::AJ) + 32 * n) + column;
        if (j >= G.M.rows_j) continue;
        if (G.bias)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const long i = first + result_row(r), m = AXIS ? j : i < G.M.rows_i ? i : G.M.rows_i - 1;
                us[r] += G.bias[m];
                vs[r] += G.bias[G.fo + m];
            }
        floatx16 y;
        with_fn(G.fn, [&](auto fn) {
#pragma unroll
            for (int r = 0; r < 16; ++r) y[r] = gate_fn<fn.value>(us[r]).a * vs[r];
        });
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const long i = first + result_row(r);
            if (i >= G.M.rows_i) continue;
            G.y[i * G.ld + j] = y[r];
            if (G.kept) {
                float* const at = G.kept + i * (AXIS ? 2 * G.ld : G.ld) + j;
                at[0] = us[r];
                at[AXIS ? G.ld : G.fo * G.ld] = vs[r];
            }
        }
    }
}

template <int WI, int AXIS>
__global__ void __launch_bounds__(128 * WI, WI / 2) k_gated_fwd_split(GatedFwd G)
{
    const TilePlace P = tile_place(G.T, blockIdx.x);
    const long i0 = (long)P.i * (AXIS ? 64 * WI : 32 * WI), j0 = (long)P.j * (AXIS ? kSplitColumns / 2 : kSplitColumns);
    floatx4 acc[4][4];
    split_product<WI, true, AXIS == 1, AXIS ? HALVES_J : HALVES_I, false>(acc, G.M, i0, j0);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // halves are 32 of a wave's 64 rows or columns apart
#pragma unroll
    for (int x = 0; x < (AXIS ? 4 : 2); ++x) {
        constexpr int N = AXIS ? 2 : 4;
        const long i = i0 + wave / 2 * (AXIS ? 64 : 32) + 16 * x + (lane & 15), j = j0 + wave % 2 * (AXIS ? 32 : 64) + (lane >> 4) * 4;
        if (i >= G.M.rows_i) continue;
        float u[N][4], v[N][4];
#pragma unroll
        for (int y = 0; y < N; ++y)
#pragma unroll
            for (int r = 0; r < 4; ++r) { u[y][r] = acc[x][y][r]; v[y][r] = AXIS ? acc[x][(y + 2) & 3][r] : acc[(x + 2) & 3][y][r]; }
        finish<N, 4, AXIS>(G.fn, G.bias, G.fo, AXIS ? G.ld : G.fo * G.ld, G.y, G.kept, u, v,
            [&](int y) { return AXIS ? Element{j + 16 * y, i} : Element{i, j + 16 * y}; },
            [&](long m, long n, float& a, float& b) {
                a = AXIS ? again<true, true>(G.M, n, m) : again<true, false>(G.M, m, n);
                b = AXIS ? again<true, true>(G.M, n, m + G.fo) : again<true, false>(G.M, m + G.fo, n);
            },
            [&](int y) {
                const long left = G.M.rows_j - j - 16 * y;
                return Spot{i * G.ld + j + 16 * y, i * (AXIS ? 2 * G.ld : G.ld) + j + 16 * y, left < 4 ? (int)(left < 0 ? 0 : left) : 4};
            });
    }
}

// ---------------------------------------------------------------- few positions
// Every weight is read for a few products only, so that their bytes are all there is: a wave takes one feature, lanes quads of its two rows of weights, and N
// positions at once.  One row of 1024 -> 4096 5.3 us (33.6 MB from the last level cache).  All weights are read once for eight positions, and images are read a feature
// at a time; us of kernels, so and by the shares that forward_of has for more positions: rows of 1024 -> 4096, 4 of them 6.8 and 17.7, 8 12.4 and 17.7, 9 22.1 and 17.8, 32 40.6
// and 18.6; maps, 4 positions 8.1 and 18.8, 8 20.2 and 19.3, 32 69.3 and 21.6; rows of 256 -> 512, 8 of them 4.5 and 13.8, 32 5.6 and 14.3; maps the same.  The limit of 32
// is right for few weights and not for many, from 9 positions on.

__device__ __forceinline__ float sum_lanes(float v)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
    return v;
}

struct GatedFew { const float *x, *w, *bias; float *y, *kept; int fn, f, fo; long positions, feature, position; };   // strides of x

template <int N, int AXIS>
__global__ void __launch_bounds__(256) k_gated_few(GatedFew G)
{
    const int lane = threadIdx.x & 63, m = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (m >= G.fo) return;
    const long n0 = blockIdx.y * N;
    const float *const wu = G.w + (long)m * G.f, *const wv = wu + (long)G.fo * G.f;
    float u[N], v[N];
#pragma unroll
    for (int p = 0; p < N; ++p) u[p] = v[p] = 0.f;
#pragma unroll 4
    for (int k = lane * 4; k < G.f; k += 256) {
        const int most = G.f - k < 4 ? G.f - k : 4;
        const floatx4 a = load4(wu + k, most), b = load4(wv + k, most);
        floatx4 x[N];
        if (AXIS)
#pragma unroll
            for (int p = 0; p < N; ++p) x[p] = load4(G.x + (n0 + p < G.positions ? n0 + p : G.positions - 1) * G.position + k, most);
        else
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float* const at = G.x + (k + (c < most ? c : 0)) * G.feature + n0;
#pragma unroll
                for (int q = 0; q < (N + 3) / 4; ++q) {
                    const long left = G.positions - n0 - 4 * q;
                    const floatx4 some = N < 4 ? floatx4{at[0], left > 1 ? at[N - 1] : 0.f, 0.f, 0.f} : load4(at + 4 * q, left < 0 ? 0 : left < 4 ? (int)left : 4);
#pragma unroll
                    for (int p = 4 * q; p < 4 * q + 4 && p < N; ++p) x[p][c] = some[p & 3];
                }
            }
#pragma unroll
        for (int p = 0; p < N; ++p)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                // weights behind the last one are zeros, x there a number of its own
                u[p] = c < most ? fmaf(a[c], x[p][c], u[p]) : u[p];
                v[p] = c < most ? fmaf(b[c], x[p][c], v[p]) : v[p];
            }
    }
    float mine_u = 0.f, mine_v = 0.f;       // of position `lane`
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const float su = sum_lanes(u[p]), sv = sum_lanes(v[p]);
        if (lane == p) { mine_u = su; mine_v = sv; }
    }
    const long n = n0 + lane;
    if (lane >= N || n >= G.positions) return;
    if (G.bias) { mine_u += G.bias[m]; mine_v += G.bias[G.fo + m]; }
    with_fn(G.fn, [&](auto fn) { G.y[AXIS ? n * G.fo + m : m * G.positions + n] = gate_fn<fn.value>(mine_u).a * mine_v; });
    if (G.kept) {
        G.kept[AXIS ? n * 2 * G.fo + m : m * G.positions + n] = mine_u;
        G.kept[AXIS ? n * 2 * G.fo + G.fo + m : (G.fo + (long)m) * G.positions + n] = mine_v;
    }
}

// ---------------------------------------------------------------- few features in, many positions
// Up to 128 features of a position are taken apart once and stay in registers, 16 P positions a wave; weights, taken apart beforehand, pass through
// shared memory, 16 features (both halves) at a time, and every wave multiplies all of them.  Nothing of x is read or taken apart twice, and a step's results are
// finished while the other workgroup of the unit multiplies.  Over images the biases of a group are read where they are added, four pairs one after another.  120 -> 240 maps
// of 96^3 700 to 740 us (141 TFLOP/s, 1.8 TB/s; 1380 by tiles); 40 -> 80 of 64^3, kept, 61 us (4.8 TB/s).

// Weights in the order they are read: [16 features][half][step of 32 k][part][lane] of 16 bytes.  Every second step has its sign changed.
constexpr int kNarrowSteps = 4;
constexpr long narrow_bytes(int steps) { return 2L * steps * 3 * 1024; }      // of 16 features

__global__ void __launch_bounds__(256) k_pack_gated(const float* w, int f, int fo, int steps, char* packed)
{
    const long t = blockIdx.x * 256L + threadIdx.x, groups = (fo + 15) / 16;
    const int lane = (int)(t & 63);
    const long piece = t >> 6, step = piece % steps, half = piece / steps % 2, group = piece / steps / 2;
    if (group >= groups) return;
    const long m = group * 16 + (lane & 15);
    const float* const from = w + (half * fo + (m < fo ? m : fo - 1)) * f;
    float v[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const int k = (int)step * kDepth + (lane >> 4) * 8 + c;
        const float one = from[k < f ? k : f - 1] * (step & 1 ? -split::kScale : split::kScale);
        v[c] = k < f ? one : 0.f;
    }
#pragma unroll
    for (int part = 0; part < 3; ++part) *(uintx4*)(packed + (piece * 3 + part) * 1024 + lane * 16) = split::take_part8(v);
}

struct GatedNarrow { const float *x, *w, *bias; const char* packed; float *y, *kept; int fn, f, fo, groups; long positions; };   // groups of 16 features a workgroup

template <int STEPS, int P, int AXIS>
__global__ void __launch_bounds__(256, 2) k_gated_narrow(GatedNarrow G)
{
    constexpr int kBytes = (int)narrow_bytes(STEPS);
    __shared__ __attribute__((aligned(16))) char lds[2][kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), one = lane & 15, octet = lane >> 4;
    const long n0 = ((long)blockIdx.x * 4 + wave) * (16 * P);
    const int first = blockIdx.y * G.groups, all = (G.fo + 15) / 16, groups = all - first < G.groups ? all - first : G.groups;
    const char* from = G.packed + (long)first * kBytes + threadIdx.x * 16;
    auto fetch = [&](char* to) {
#pragma unroll
        for (int i = 0; i < kBytes / 4096; ++i)
            __builtin_amdgcn_global_load_lds((split::global_ptr)(from + i * 4096), (split::lds_ptr)(to + i * 4096 + wave * 1024), 16, 0, 0);
        if (kBytes % 4096 && wave * 1024 < kBytes % 4096)
            __builtin_amdgcn_global_load_lds((split::global_ptr)(from + kBytes / 4096 * 4096), (split::lds_ptr)(to + kBytes / 4096 * 4096 + wave * 1024), 16, 0, 0);
        from += kBytes;
    };
    fetch(lds[0]);
    // images: a lane's P positions lie side by side, so that 16 lanes read and write whole lines; rows of features: 16 positions apart
    bf16x8 x[P][STEPS][3];
    const long mine = n0 + (AXIS ? one : P * one);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int k = s * kDepth + octet * 8;
        float all[P][8];
        if (!AXIS) {
            typedef float vector __attribute__((ext_vector_type(P), aligned(4)));
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const float* const at = G.x + (k + c < G.f ? k + c : 0) * G.positions;
                if (n0 + 16 * P <= G.positions) {
                    const vector some = *(const vector*)(at + mine);
#pragma unroll
                    for (int p = 0; p < P; ++p) all[p][c] = some[p];
                } else
#pragma unroll
                    for (int p = 0; p < P; ++p) all[p][c] = at[mine + p < G.positions ? mine + p : G.positions - 1];
            }
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const long n = mine + 16 * p < G.positions ? mine + 16 * p : G.positions - 1;
            float v[8];
            if (AXIS) {
                const float* const at = G.x + n * G.f + k;
                if ((s + 1) * kDepth <= G.f) {
                    *(floatx4*)v = *(const floatu4*)at;
                    *(floatx4*)(v + 4) = *(const floatu4*)(at + 4);
                } else
#pragma unroll
                    for (int c = 0; c < 8; ++c) v[c] = k + c < G.f ? at[c] : 0.f;
            } else
#pragma unroll
                for (int c = 0; c < 8; ++c) v[c] = k + c < G.f ? all[p][c] : 0.f;
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] *= split::kScale;
#pragma unroll
            for (int part = 0; part < 3; ++part) x[p][s][part] = __builtin_bit_cast(bf16x8, split::take_part8(v));
        }
    }
    __syncthreads();
    for (int g = 0; g < groups; ++g) {
        const char* const here = lds[g & 1] + lane * 16;
        constexpr int of_w[6] = {0, 2, 1, 0, 1, 0}, of_x[6] = {2, 0, 1, 1, 0, 0};
        if (g + 1 < groups) fetch(lds[~g & 1]);
        floatx4 acc[2][P], t[2][2][P];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            bf16x8 w[2][3];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int part = 0; part < 3; ++part) w[h][part] = __builtin_bit_cast(bf16x8, *(const uintx4*)(here + ((h * STEPS + s) * 3 + part) * 1024));
#pragma unroll
            for (int q = 0; q < 6; ++q)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const floatx4 c = q ? t[s & 1][h][p] : floatx4{0.f, 0.f, 0.f, 0.f};
                        t[s & 1][h][p] = split::mfma(w[h][of_w[q]], x[p][s][of_x[q]], c);
                    }
            // a step's products are added once they are done, beside the next one's
            if (s)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int p = 0; p < P; ++p) acc[h][p] = s == 1 ? t[0][h][p] : s & 1 ? acc[h][p] + t[0][h][p] : acc[h][p] - t[1][h][p];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (STEPS == 1) acc[h][p] = t[0][h][p];
                else if (STEPS & 1) acc[h][p] += t[0][h][p];
                else acc[h][p] -= t[1][h][p];
                acc[h][p] *= split::kUnscale;
            }
        __syncthreads();
        // a lane has four features of its P positions
        const long m = (first + g) * 16 + octet * 4, ld = AXIS ? G.fo : G.positions;
        constexpr int N = AXIS ? P : 4, C = AXIS ? 4 : P;
        float u[N][C], v[N][C];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int r = 0; r < 4; ++r) { u[AXIS ? p : r][AXIS ? r : p] = acc[0][p][r]; v[AXIS ? p : r][AXIS ? r : p] = acc[1][p][r]; }
        finish<N, C, AXIS>(G.fn, G.bias, G.fo, AXIS ? ld : G.fo * ld, G.y, G.kept, u, v,
            [&](int i) { return AXIS ? Element{m, mine + 16 * i} : Element{m + i, mine}; },
            [&](long feature, long at, float& a, float& b) {
                const float *const xs = AXIS ? G.x + at * G.f : G.x + at, *const ws = G.w + feature * G.f;
                a = again(ws, 1, xs, AXIS ? 1 : G.positions, G.f);
                b = again(ws + (long)G.fo * G.f, 1, xs, AXIS ? 1 : G.positions, G.f);
            },
            [&](int i) {
                const long row = AXIS ? mine + 16 * i : m + i, column = AXIS ? m : mine, left = row < (AXIS ? G.positions : G.fo) ? ld - column : 0;
                return Spot{row * ld + column, AXIS ? 2 * row * ld + column : row * ld + column, left < C ? (int)(left < 0 ? 0 : left) : C};
            });
    }
}

// A product, or with several shares of the sum over k (`span` of it each) partial ones, one behind the other.
struct Product { Matrices M; Tiles T; float* c; long span; };
template <class W, bool A_ALONG, bool B_ALONG>
__global__ void __launch_bounds__(W::kThreads) k_product(Product G)
{
    const TilePlace P = tile_place(G.T, blockIdx.x);
    const long i0 = (long)P.i * W::TI, j0 = (long)P.j * W::TJ;
    Matrices M = G.M;
    M.k0 = blockIdx.y * G.span;
    if (M.k0 + G.span < M.K) M.K = M.k0 + G.span;
    floatx16 acc[W::AI][W::AJ];
    tile_product<W, A_ALONG, B_ALONG, NO_HALVES>(acc, M, i0, j0);
    float* const c = G.c + blockIdx.y * (M.rows_i * M.rows_j);
    const int wave = threadIdx.x >> 6, column = threadIdx.x & 31;
#pragma unroll
    for (int x = 0; x < W::AI; ++x)
#pragma unroll
        for (int y = 0; y < W::AJ; ++y)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const long i = i0 + wave / W::WJ * (32 * W::AI) + 32 * x + result_row(r), j = j0 + wave % W::WJ * (32 * W::AJ) + 32 * y + column;
                if (i < M.rows_i && j < M.rows_j) c[i * M.rows_j + j] = acc[x][y][r];
            }
}

// TURNED: c [j][i]
template <int WI, bool A_ALONG, bool B_ALONG, bool TURNED>
__global__ void __launch_bounds__(128 * WI, WI / 2) k_product_split(Product G)
{
    const TilePlace P = tile_place(G.T, blockIdx.x);
    const long i0 = (long)P.i * (64 * WI), j0 = (long)P.j * kSplitColumns;
    Matrices M = G.M;
    M.k0 = blockIdx.y * G.span;
    if (M.k0 + G.span < M.K) M.K = M.k0 + G.span;
    floatx4 acc[4][4];
    split_product<WI, A_ALONG, B_ALONG, NO_HALVES, TURNED>(acc, M, i0, j0);
    float* const c = G.c + blockIdx.y * (M.rows_i * M.rows_j);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, one = lane & 15, four = (lane >> 4) * 4;
    const long ld = TURNED ? M.rows_i : M.rows_j;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const long i = i0 + wave / 2 * 64 + 16 * x + (TURNED ? four : one), j = j0 + wave % 2 * 64 + 16 * y + (TURNED ? one : four);
            if (i >= M.rows_i || j >= M.rows_j) continue;
            const long left = TURNED ? M.rows_i - i : M.rows_j - j;
            const int most = left < 4 ? (int)left : 4;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < most && !finite(acc[x][y][r])) acc[x][y][r] = again<A_ALONG, B_ALONG>(M, TURNED ? i + r : i, TURNED ? j : j + r);
            store4(TURNED ? c + j * ld + i : c + i * ld + j, acc[x][y], most);
        }
}

// Sums of shares that several launches have left, in one.  A few shares, or those of many elements, are added in their order, four neighbours a
// thread; of many shares every sixteenth by one wave, and then these in their order.  That takes sixteen threads an element, where a launch has fewer than 2^32.
struct SharedSum { const float* parts; float* out; long count; int shares; unsigned first; };     // first workgroup
struct SharedSums { SharedSum of[3]; int n; };
constexpr int kFewShares = 16;
__host__ __device__ constexpr bool in_order(const SharedSum& S) { return S.shares <= kFewShares || S.count >= 1L << 24; }
// workgroups
unsigned blocks_of(const SharedSum& S) { return (unsigned)((S.count + (in_order(S) ? 4095 : 63)) / (in_order(S) ? 4096 : 64)); }

__global__ void __launch_bounds__(1024) k_sum_shares(SharedSums A)
{
    __shared__ float part[16][64];
    int which = 0;
    while (which + 1 < A.n && blockIdx.x >= A.of[which + 1].first) ++which;       // uniform
    const SharedSum S = A.of[which];
    const long block = blockIdx.x - S.first;
    if (in_order(S)) {
        const long e = block * 4096 + threadIdx.x * 4;
        if (e >= S.count) return;
        const int most = S.count - e < 4 ? (int)(S.count - e) : 4;
        floatx4 s = load4(S.parts + e, most);
        for (int n = 1; n < S.shares; ++n) s += load4(S.parts + n * S.count + e, most);
        store4(S.out + e, s, most);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long e = block * 64 + lane;
    float s = 0.f;
    if (e < S.count) {
        int n = wave;
        for (; n + 48 < S.shares; n += 64) {
            float v[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = S.parts[(n + 16 * c) * S.count + e];
            s += (v[0] + v[1]) + (v[2] + v[3]);
        }
        for (; n < S.shares; n += 16) s += S.parts[n * S.count + e];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && e < S.count) {
#pragma unroll
        for (int w = 1; w < 16; ++w) s += part[w][lane];
        S.out[e] = s;
    }
}

// ---------------------------------------------------------------- gradients of both halves
// [du; dv] from gy and the kept [u; v], in the layout of the kept, and their sums over `span` positions for the biases.

struct Grads { int fn; long fo, positions, span; const float *gy, *kept; float *g, *sums; };      // sums [share][2 f'], or NULL

__device__ __forceinline__ void gradients(int fn, const floatx4& u, const floatx4& v, const floatx4& gy, floatx4& du, floatx4& dv)
{
    with_fn(fn, [&](auto number) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const Gated a = gate_fn<number.value>(u[c]);
            du[c] = gy[c] * (v[c] * a.d);
            dv[c] = gy[c] * a.a;
        }
    });
}

// images: a workgroup a share of one map, four neighbours a thread
__global__ void __launch_bounds__(256) k_gated_grads_maps(Grads G)
{
    __shared__ float part[2][4];
    const long m = blockIdx.x, first = blockIdx.y * G.span, end = first + G.span < G.positions ? first + G.span : G.positions;
    const long at = m * G.positions, other = G.fo * G.positions;
    float su = 0.f, sv = 0.f;
    for (long n = first + threadIdx.x * 4L; n < end; n += 1024) {
        const int most = end - n < 4 ? (int)(end - n) : 4;
        const floatx4 u = load4(G.kept + at + n, most), v = load4(G.kept + at + other + n, most), gy = load4(G.gy + at + n, most);
        floatx4 du, dv;
        gradients(G.fn, u, v, gy, du, dv);
        float tu = 0.f, tv = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c < most) { tu += du[c]; tv += dv[c]; }
        su += tu;
        sv += tv;
        store4(G.g + at + n, du, most);
        store4(G.g + at + other + n, dv, most);
    }
    if (!G.sums) return;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) { su += __shfl_xor(su, d); sv += __shfl_xor(sv, d); }
    if ((threadIdx.x & 63) == 0) { part[0][threadIdx.x >> 6] = su; part[1][threadIdx.x >> 6] = sv; }
    __syncthreads();
    if (threadIdx.x < 2) {
        const float* p = part[threadIdx.x];
        G.sums[blockIdx.y * 2 * G.fo + threadIdx.x * G.fo + m] = p[0] + p[1] + p[2] + p[3];
    }
}

// rows of features: a workgroup a share of 256 columns, four a thread, four rows at a time
__global__ void __launch_bounds__(256) k_gated_grads_rows(Grads G)
{
    __shared__ floatx4 part[2][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long m = blockIdx.x * 256L + lane * 4, first = blockIdx.y * G.span, end = first + G.span < G.positions ? first + G.span : G.positions;
    const int most = G.fo - m < 4 ? G.fo > m ? (int)(G.fo - m) : 0 : 4;
    floatx4 su = {0.f, 0.f, 0.f, 0.f}, sv = su;
    if (most)
        for (long n = first + wave; n < end; n += 4) {
            const long at = n * 2 * G.fo + m;
            const floatx4 u = load4(G.kept + at, most), v = load4(G.kept + at + G.fo, most), gy = load4(G.gy + n * G.fo + m, most);
            floatx4 du, dv;
            gradients(G.fn, u, v, gy, du, dv);
            store4(G.g + at, du, most);
            store4(G.g + at + G.fo, dv, most);
            su += du;
            sv += dv;
        }
    if (!G.sums) return;
    part[0][wave][lane] = su;
    part[1][wave][lane] = sv;
    __syncthreads();
    if (wave < 2 && most) {
        const floatx4* p = part[wave][0] + lane;
        store4(G.sums + blockIdx.y * 2 * G.fo + wave * G.fo + m, (p[0] + p[64]) + (p[128] + p[192]), most);
    }
}

// ---------------------------------------------------------------- backward with few features in
// Over many positions the bytes count, and du and dv, which would be written and read twice, are made where they are used, once for each of the two products.

struct GatedBack { const float *gy, *x, *w, *kept; int fn, f, fo; long positions; };

// gy, u and v of four features from m on (of fo) and C positions
template <int C> struct Raw { float gy[4][C], u[4][C], v[4][C]; };

// Sums taken again where they came out as no numbers: of gx, and of gw.
template <int AXIS> __device__ __forceinline__ void gradient_of(const GatedBack& G, long m, long n, float& du, float& dv)
{
    const long at = AXIS ? n * G.fo + m : m * G.positions + n, kept = AXIS ? n * 2 * G.fo + m : at, half = AXIS ? G.fo : G.fo * G.positions;
    const float gy = G.gy[at], v = G.kept[kept + half], u = G.kept[kept];
    with_fn(G.fn, [&](auto fn) {
        const Gated a = gate_fn<fn.value>(u);
        du = gy * (v * a.d);
        dv = gy * a.a;
    });
}
template <int AXIS> __device__ __noinline__ float gx_again(const GatedBack& G, long i, long n)
{
    float s = 0.f, du, dv;
    for (long m = 0; m < G.fo; ++m) {
        gradient_of<AXIS>(G, m, n, du, dv);
        s = fmaf(G.w[(G.fo + m) * G.f + i], dv, fmaf(G.w[m * G.f + i], du, s));
    }
    return s;
}
template <int AXIS> __device__ __noinline__ float gw_again(const GatedBack& G, long m, int half, long j, long first, long end)
{
    float s = 0.f, du, dv;
    for (long n = first; n < end; ++n) {
        gradient_of<AXIS>(G, m, n, du, dv);
        s = fmaf(half ? dv : du, G.x[AXIS ? n * G.f + j : j * G.positions + n], s);
    }
    return s;
}

// Forward from shares of [u; v], where tiles alone are too few for the chip: their sum, the biases and the gate.
struct GatedJoin { const float* parts; int shares, fn, rows; long fo, positions; const float* bias; float *y, *kept; };
__global__ void __launch_bounds__(256) k_gated_join(GatedJoin G)
{
    // quads of neighbours: of features (rows), or of positions
    const long line = G.rows ? G.fo : G.positions, quads = (line + 3) / 4, lines = G.rows ? G.positions : G.fo, both = 2 * G.fo * G.positions;
    for (long q = blockIdx.x * 256L + threadIdx.x; q < lines * quads; q += gridDim.x * 256L) {
        const long l = q / quads, c = (q - l * quads) * 4, at = G.rows ? 2 * l * line + c : l * line + c, other = at + (G.rows ? G.fo : G.fo * G.positions);
        const int most = line - c < 4 ? (int)(line - c) : 4;
        floatx4 u = load4(G.parts + at, most), v = load4(G.parts + other, most), out;
        for (int n = 1; n < G.shares; ++n) {
            u += load4(G.parts + n * both + at, most);
            v += load4(G.parts + n * both + other, most);
        }
        if (G.bias) {
            if (G.rows) {
                u += load4(G.bias + c, most);
                v += load4(G.bias + G.fo + c, most);
            } else {
                u += G.bias[l];
                v += G.bias[G.fo + l];
            }
        }
        with_fn(G.fn, [&](auto number) {
#pragma unroll
            for (int r = 0; r < 4; ++r) out[r] = gate_fn<number.value>(u[r]).a * v[r];
        });
        store4(G.y + l * line + c, out, most);
        if (G.kept) {
            store4(G.kept + at, u, most);
            store4(G.kept + other, v, most);
        }
    }
}

// Weights as the gradient of x reads them: [16 features][16 inputs][part][lane]; eight k are four features of W and the same of V.  Thread t of those of
// one lane each.
__device__ __forceinline__ void pack_back(const float* w, int f, int fo, int tiles, long t, char* packed)
{
    const long groups = (fo + 15) / 16;
    const int lane = (int)(t & 63);
    const long piece = t >> 6, tile = piece % tiles, group = piece / tiles;
    if (group >= groups) return;
    const long i = tile * 16 + (lane & 15), m = group * 16 + (lane >> 4) * 4;
    float v[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const long row = m + (c & 3);
        const float one = w[((c >> 2) * (long)fo + (row < fo ? row : fo - 1)) * f + (i < f ? i : f - 1)] * (group & 1 ? -split::kScale : split::kScale);
        v[c] = row < fo && i < f ? one : 0.f;
    }
#pragma unroll
    for (int part = 0; part < 3; ++part) *(uintx4*)(packed + (piece * 3 + part) * 1024 + lane * 16) = split::take_part8(v);
}

// gx: a wave takes 32 positions and all TILES x 16 inputs, workgroups of four waves walk over the positions.  The next 16 features' gy, u and v are requested before
// 16 are multiplied.  Their weights are copied into shared memory as well, but waited for at once: gx_again takes G by reference, so that G lies in private memory, its pointers
// are read from there and loads through them are flat ones, which wait for everything before them.  40 -> 80 maps of 61 x 58 x 63 68 us, 3.7 TB/s.
template <int TILES, int AXIS>
__global__ void __launch_bounds__(256, 2) k_gated_gx(GatedBack G, const char* packed, float* gx)
{
    constexpr int P = 2, kBytes = TILES * 3 * 1024;
    __shared__ __attribute__((aligned(16))) char lds[2][kBytes];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, one = lane & 15, octet = lane >> 4;
    const int groups = (G.fo + 15) / 16;
    const long tiles = (G.positions + 64 * P - 1) / (64 * P), half = AXIS ? G.fo : G.fo * G.positions;
    auto fetch = [&](int group, char* to) {
        const char* const from = packed + (long)group * kBytes;
#pragma unroll
        for (int i = 0; i < (kBytes + 4095) / 4096; ++i)
            if (i * 4096 + wave * 1024 < kBytes)
                __builtin_amdgcn_global_load_lds((split::global_ptr)(from + i * 4096 + threadIdx.x * 16), (split::lds_ptr)(to + i * 4096 + wave * 1024), 16, 0, 0);
    };
    Raw<P> raw;
    auto load = [&](long tile, int group) {
        const long n0 = (tile * 4 + wave) * (16 * P);
        const int m = group * 16 + octet * 4;
        if (AXIS) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const long want = n0 + one + 16 * p, n = want < G.positions ? want : G.positions - 1;
                const float *const gy = G.gy + n * G.fo, *const u = G.kept + n * 2 * G.fo, *const v = u + G.fo;
                if (group * 16 + 16 <= G.fo) {
                    const floatx4 a = *(const floatu4*)(gy + m), b = *(const floatu4*)(u + m), c = *(const floatu4*)(v + m);
#pragma unroll
                    for (int r = 0; r < 4; ++r) { raw.gy[r][p] = a[r]; raw.u[r][p] = b[r]; raw.v[r][p] = c[r]; }
                } else
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int row = m + r < G.fo ? m + r : G.fo - 1;
                        raw.gy[r][p] = gy[row]; raw.u[r][p] = u[row]; raw.v[r][p] = v[row];
                    }
            }
        } else
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const long at = (m + r < G.fo ? m + r : G.fo - 1) * G.positions, n = n0 + P * one;
                if (n0 + 16 * P <= G.positions) {
                    const floatu2 a = *(const floatu2*)(G.gy + at + n), b = *(const floatu2*)(G.kept + at + n), c = *(const floatu2*)(G.kept + half + at + n);
#pragma unroll
                    for (int p = 0; p < P; ++p) { raw.gy[r][p] = a[p]; raw.u[r][p] = b[p]; raw.v[r][p] = c[p]; }
                } else
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const long place = at + (n + p < G.positions ? n + p : G.positions - 1);
                        raw.gy[r][p] = G.gy[place]; raw.u[r][p] = G.kept[place]; raw.v[r][p] = G.kept[half + place];
                    }
            }
    };
    const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
    fetch(0, lds[0]);
    load(blockIdx.x, 0);
    __syncthreads();
    int buffer = 0;
    for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        floatx4 acc[TILES][P];
#pragma unroll
        for (int y = 0; y < TILES; ++y)
#pragma unroll
            for (int p = 0; p < P; ++p) acc[y][p] = zero;
        for (int group = 0; group < groups; ++group) {
            const char* const here = lds[buffer] + lane * 16;
            buffer ^= 1;
            const bool last = group + 1 == groups;
            if (!last || tile + gridDim.x < tiles) fetch(last ? 0 : group + 1, lds[buffer]);
            float g[P][8];
            with_fn(G.fn, [&](auto fn) {
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const Gated a = gate_fn<fn.value>(raw.u[r][p]);
                        const bool there = group * 16 + octet * 4 + r < G.fo;
                        g[p][r] = there ? raw.gy[r][p] * (raw.v[r][p] * a.d) * split::kScale : 0.f;
                        g[p][r + 4] = there ? raw.gy[r][p] * a.a * split::kScale : 0.f;
                    }
            });
            if (!last || tile + gridDim.x < tiles) load(last ? tile + gridDim.x : tile, last ? 0 : group + 1);
            bf16x8 x[P][3];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int part = 0; part < 3; ++part) x[p][part] = __builtin_bit_cast(bf16x8, split::take_part8(g[p]));
            const float sign = group & 1 ? -1.f : 1.f;
            constexpr int of_w[6] = {0, 2, 1, 0, 1, 0}, of_x[6] = {2, 0, 1, 1, 0, 0};
            floatx4 t[2][P];
#pragma unroll
            for (int y = 0; y < TILES; ++y) {
                bf16x8 w[3];
#pragma unroll
                for (int part = 0; part < 3; ++part) w[part] = __builtin_bit_cast(bf16x8, *(const uintx4*)(here + (y * 3 + part) * 1024));
#pragma unroll
                for (int q = 0; q < 6; ++q)
#pragma unroll
                    for (int p = 0; p < P; ++p) t[y & 1][p] = split::mfma(w[of_w[q]], x[p][of_x[q]], q ? t[y & 1][p] : zero);
                if (y)
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[y - 1][p][r] = fmaf(t[~y & 1][p][r], sign, acc[y - 1][p][r]);
            }
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[TILES - 1][p][r] = fmaf(t[(TILES - 1) & 1][p][r], sign, acc[TILES - 1][p][r]);
            __syncthreads();
        }
        // a lane has four inputs of its P positions
        const long mine = (tile * 4 + wave) * (16 * P) + (AXIS ? one : P * one);
        float test = 0.f;
#pragma unroll
        for (int y = 0; y < TILES; ++y) {
            const long i = y * 16 + octet * 4;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                acc[y][p] *= split::kUnscale;
#pragma unroll
                for (int r = 0; r < 4; ++r) test = fmaf(acc[y][p][r], 0.f, test);
            }
            if (AXIS) {
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const long n = mine + 16 * p;
                    if (n < G.positions && i < G.f) store4(gx + n * G.f + i, acc[y][p], G.f - i < 4 ? (int)(G.f - i) : 4);
                }
            } else
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float out[2] = {acc[y][0][r], acc[y][1][r]};
                    const long left = G.positions - mine;
                    if (i + r < G.f && left > 0) store_some(gx + (i + r) * G.positions + mine, out, left < P ? (int)left : P);
                }
        }
        if (test != 0.f) {
            unsigned long bad = 0;
#pragma unroll
            for (int y = 0; y < TILES; ++y)
#pragma unroll
                for (int e = 0; e < 4 * P; ++e) bad |= (unsigned long)!finite(acc[y][e >> 2][e & 3]) << (y * 4 * P + e);
#pragma unroll 1
            for (int e = 0; e < 4 * P * TILES; ++e) {
                const long i = e / (4 * P) * 16 + octet * 4 + (e & 3), n = mine + (e >> 2) % P * (AXIS ? 16 : 1);
                if ((bad >> e & 1) && i < G.f && n < G.positions) gx[AXIS ? n * G.f + i : i * G.positions + n] = gx_again<AXIS>(G, i, n);
            }
        }
    }
}

constexpr int kBackWaves = 4;       // of a workgroup: with three on a SIMD

// gw and gb: a wave takes 16 features (both halves) and all TILES x 16 inputs, workgroups a share of the positions, 32 at a time; x is taken apart by all
// waves for all of them.  Workgroups behind the shares pack the weights for k_gated_gx, which comes next.  40 -> 80 maps of 61 x 58 x 63 95 us, 2.6 TB/s, bound by the
// latency of its loads: gw_again takes G by reference, so that G lies in private memory as in k_gated_gx, and the pointers of gy and of the kept are read behind the loads of x and
// waited for with these.  Three waves a SIMD are what the registers leave.
template <int TILES, int AXIS>
__global__ void __launch_bounds__(64 * kBackWaves, 3) k_gated_gw(GatedBack G, long span, int shares, int waves, float* parts, float* sums, char* packed)
{
    if ((int)blockIdx.x >= shares) {
        pack_back(G.w, G.f, G.fo, TILES, ((long)(blockIdx.x - shares) * gridDim.y + blockIdx.y) * waves * 64 + threadIdx.x, packed);
        return;
    }
    constexpr int kBytes = TILES * 3 * 1024;
    __shared__ __attribute__((aligned(16))) char lds[2][kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), one = lane & 15, octet = lane >> 4, threads = waves * 64;
    const long m = ((long)blockIdx.y * waves + wave) * 16 + one, half = AXIS ? G.fo : G.fo * G.positions;
    const long row = m < G.fo ? m : G.fo - 1, first = blockIdx.x * span, end = first + span < G.positions ? first + span : G.positions;
    const bool works = ((long)blockIdx.y * waves + wave) * 16 < G.fo;      // else it moves x alone; uniform
    // octets of x that this thread moves, at most two
    auto unit_row = [&](int u) { return AXIS ? u % (TILES * 16) : u / 4; };
    auto unit_octet = [&](int u) { return AXIS ? u / (TILES * 16) : u % 4; };
    float xs[2][8], gy[8], u[8], v[8];
    auto load = [&](long n0) {
        const bool whole = n0 + kDepth <= end;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int unit = threadIdx.x + c * threads;
            if (unit >= TILES * 64) break;
            const int j = unit_row(unit);
            const long n = n0 + unit_octet(unit) * 8;
            const float* const at = AXIS ? G.x + n * G.f + (j < G.f ? j : G.f - 1) : G.x + (j < G.f ? j : G.f - 1) * G.positions + n;
            if (!AXIS && whole) {
                *(floatx4*)xs[c] = *(const floatu4*)at;
                *(floatx4*)(xs[c] + 4) = *(const floatu4*)(at + 4);
            } else
#pragma unroll
                for (int e = 0; e < 8; ++e) xs[c][e] = n + e < end ? at[AXIS ? e * (long)G.f : e] : 0.f;
        }
        if (!works) return;
        const long n = n0 + octet * 8;
        if (!AXIS && whole) {
            const long at = row * G.positions + n;
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                *(floatx4*)(gy + e) = *(const floatu4*)(G.gy + at + e);
                *(floatx4*)(u + e) = *(const floatu4*)(G.kept + at + e);
                *(floatx4*)(v + e) = *(const floatu4*)(G.kept + half + at + e);
            }
        } else if (whole) {
            const float *const ys = G.gy + n * G.fo + row, *const us = G.kept + n * 2 * G.fo + row;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                gy[e] = ys[e * (long)G.fo];
                u[e] = us[e * 2L * G.fo];
                v[e] = us[e * 2L * G.fo + half];
            }
        } else
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // positions behind the last one: zeros, whose gradients are zeros
                const bool there = n + e < end;
                const long k = there ? n + e : end - 1, at = AXIS ? k * 2 * G.fo + row : row * G.positions + k;
                gy[e] = there ? G.gy[AXIS ? k * G.fo + row : row * G.positions + k] : 0.f;
                u[e] = there ? G.kept[at] : 0.f;
                v[e] = there ? G.kept[half + at] : 0.f;
            }
    };
    auto store = [&](char* to) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int unit = threadIdx.x + c * threads;
            if (unit >= TILES * 64) break;
            const int j = unit_row(unit);
#pragma unroll
            for (int e = 0; e < 8; ++e) xs[c][e] *= split::kScale;
#pragma unroll
            for (int part = 0; part < 3; ++part)
                *(uintx4*)(to + ((j >> 4) * 3 + part) * 1024 + (unit_octet(unit) * 16 + (j & 15)) * 16) = split::take_part8(xs[c]);
        }
    };
    const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
    floatx4 acc[TILES][2];
#pragma unroll
    for (int y = 0; y < TILES; ++y) acc[y][0] = acc[y][1] = zero;
    float su = 0.f, sv = 0.f, sign = 1.f;
    load(first);
    store(lds[0]);
    __syncthreads();
    int buffer = 0;
    for (long n0 = first; n0 < end; n0 += kDepth, sign = -sign) {
        const char* const here = lds[buffer] + lane * 16;
        buffer ^= 1;
        float g[2][8];
        if (works)
            with_fn(G.fn, [&](auto fn) {
                float tu = 0.f, tv = 0.f;       // a step by itself: chains of 8, and of one number a step (span / 32 at most 2048)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const Gated a = gate_fn<fn.value>(u[e]);
                    const float du = gy[e] * (v[e] * a.d), dv = gy[e] * a.a;
                    tu += du;
                    tv += dv;
                    g[0][e] = du * (sign * split::kScale);
                    g[1][e] = dv * (sign * split::kScale);
                }
                su += tu;
                sv += tv;
            });
        const bool more = n0 + kDepth < end;
        if (more) load(n0 + kDepth);
        if (works) {
            bf16x8 a[2][3];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int part = 0; part < 3; ++part) a[h][part] = __builtin_bit_cast(bf16x8, split::take_part8(g[h]));
            constexpr int of_a[6] = {0, 2, 1, 0, 1, 0}, of_x[6] = {2, 0, 1, 1, 0, 0};
            floatx4 t[2][2];
#pragma unroll
            for (int y = 0; y < TILES; ++y) {
                bf16x8 x[3];
#pragma unroll
                for (int part = 0; part < 3; ++part) x[part] = __builtin_bit_cast(bf16x8, *(const uintx4*)(here + (y * 3 + part) * 1024));
#pragma unroll
                for (int q = 0; q < 6; ++q)
#pragma unroll
                    for (int h = 0; h < 2; ++h) t[y & 1][h] = split::mfma(x[of_x[q]], a[h][of_a[q]], q ? t[y & 1][h] : zero);
                if (y)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[y - 1][h][r] = fmaf(t[~y & 1][h][r], sign, acc[y - 1][h][r]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[TILES - 1][h][r] = fmaf(t[(TILES - 1) & 1][h][r], sign, acc[TILES - 1][h][r]);
        }
        if (more) store(lds[buffer]);
        __syncthreads();
    }
    if (!works) return;
    su += __shfl_xor(su, 16);
    sv += __shfl_xor(sv, 16);
    su += __shfl_xor(su, 32);
    sv += __shfl_xor(sv, 32);
    if (sums && octet == 0 && m < G.fo) {
        sums[blockIdx.x * 2L * G.fo + m] = su;
        sums[blockIdx.x * 2L * G.fo + G.fo + m] = sv;
    }
    if (m >= G.fo) return;
    // a lane has four inputs of its feature
    float* const out = parts + blockIdx.x * 2L * G.fo * G.f + m * G.f;
#pragma unroll
    for (int y = 0; y < TILES; ++y)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long j = y * 16 + octet * 4;
            if (j >= G.f) continue;
            const int most = G.f - j < 4 ? (int)(G.f - j) : 4;
            floatx4 s = acc[y][h] * split::kUnscale;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < most && !finite(s[r])) s[r] = gw_again<AXIS>(G, m, h, j + r, first, end);
            store4(out + h * (long)G.fo * G.f + j, s, most);
        }
}

struct Shape { int f, fo, axis; long positions; };

int check_gated(int32_t fan_in, int32_t fan_out, int64_t positions, int32_t axis)
{
    if (fan_in < 1 || fan_out < 1 || positions < 1) return fail(ZNN_EINVAL, "features and positions must be >= 1");
    if (axis != 0 && axis != 1) return fail(ZNN_EINVAL, "axis must be 0 (images) or 1 (rows of features)");
    if (fan_in > 1 << 20 || fan_out > 1 << 20 || positions > 2147483647LL)
        return fail(ZNN_EUNSUPPORTED, "a gated unit of %d to %d features over %lld positions is too large", fan_in, fan_out, (long long)positions);
    // numbers of tiles have 31 bits
    if ((double)std::max(fan_in, fan_out) * positions > 274877906944.0)
        return fail(ZNN_EUNSUPPORTED, "arrays of %d features at %lld positions are too large", (int)std::max(fan_in, fan_out), (long long)positions);
    return ZNN_OK;
}

// ---------------------------------------------------------------- tiles, shares, launches
typedef Waves<1, 4, 2, 1> Wide;         // 64 x 128
typedef Waves<4, 1, 1, 2> Tall;         // 128 x 64

// Tiles of a product and into how many shares its sum goes, by what it is expected to take: a unit takes 2.6 us for a step of 32 k of a tile of 256 x 128 on the
// bf16 matrix cores (205 TFLOP/s in all), and 1.3 us for one of 64 x 128 on the fp32 ones (100 TFLOP/s), which take three tiles side by side; sums of
// shares move their bytes at 4 TB/s and a launch takes 3 us.  Where a product may go in shares, sums of more than 2^16 terms (2048 additions one after another on the bf16
// matrix cores) do whatever it costs, as far as there are shares.
enum Kind { FP32, SPLIT, SPLIT_TURNED };
struct Layout { Kind kind; Tiles T; int shares; long span; double us; };
constexpr long kFewPositions = 32, kUnits = 256, kMostShares = 512, kLeastSpan = kDepth, kMostSpan = 1L << 16;
Tiles tiles_of(long i, long j, long ti, long tj)
{
    const long ni = (i + ti - 1) / ti, nj = (j + tj - 1) / tj;
    return Tiles{(unsigned)ni, (unsigned)nj, (unsigned)(ni * nj)};
}
Layout layout_of(Kind kind, const Tiles& T, long I, long J, long K, bool shares)
{
    const long beside = kind == FP32 ? 3 * kUnits : kUnits;
    Layout best = {};
    best.us = HUGE_VAL;
    for (long wanted = 1; wanted <= (shares ? kMostShares : 1); wanted = wanted < 4 ? wanted + 1 : wanted < kMostShares ? std::min(kMostShares, wanted + wanted / 4) : kMostShares + 1) {
        if (wanted > 1 && K / wanted < kLeastSpan) break;
        Layout L = {kind, T, 1, (K + kDepth - 1) / kDepth * kDepth, 0.0};
        if (wanted > 1) {
            L.span = (K + wanted * kDepth - 1) / (wanted * kDepth) * kDepth;
            L.shares = (int)((K + L.span - 1) / L.span);
        }
        const long tiles = T.count * (long)L.shares, rounds = (tiles + beside - 1) / beside, last = tiles - (rounds - 1) * beside;
        const double steps = (double)(L.span / kDepth), step = kind == FP32 ? 1.3 : 2.6;
        // tiles of the last round that stand alone on their unit take less than three side by side do
        const double tall = kind == FP32 ? 3.0 * (rounds - 1) + (last > 2 * kUnits ? 3.0 : last > kUnits ? 2.0 : 1.2) : rounds;
        L.us = tall * (steps * step + (kind == FP32 ? 2.0 : 5.0));
        if (L.shares > 1) L.us += 3.0 + 1e-6 * I * J * 2 * L.shares;
        if (L.span > kMostSpan && shares && wanted < kMostShares) L.us *= 1e6 * L.span / kMostSpan;
        if (L.us < best.us) best = L;
    }
    return best;
}
Layout product_layout(long I, long J, long K)
{
    Layout best = layout_of(FP32, tiles_of(I, J, Wide::TI, Wide::TJ), I, J, K, true);
    for (Kind kind : {SPLIT, SPLIT_TURNED}) {
        const Tiles T = kind == SPLIT ? tiles_of(I, J, 64 * kSplitWaves, kSplitColumns) : tiles_of(J, I, 64 * kSplitWaves, kSplitColumns);
        const Layout L = layout_of(kind, T, I, J, K, true);
        if (L.us < best.us) best = L;
    }
    return best;
}
size_t product_bytes(const Layout& L, long I, long J) { return L.shares > 1 ? align256(sizeof(float) * L.shares * I * J) : 0; }

void add_shares(SharedSums& A, const float* parts, float* out, long count, int shares)
{
    if (shares <= 1) return;
    const unsigned first = A.n ? A.of[A.n - 1].first + blocks_of(A.of[A.n - 1]) : 0;
    A.of[A.n++] = SharedSum{parts, out, count, shares, first};
}
void sum_shares(const SharedSums& A, hipStream_t s)
{
    if (!A.n) return;
    const SharedSum& last = A.of[A.n - 1];
    ZNN_LAUNCH("gated unit shares", s, k_sum_shares, dim3(last.first + blocks_of(last)), dim3(1024), 0, A);
}
// Few features in: taken apart in registers where enough positions keep the chip busy.
constexpr int narrow_steps(int f) { return f <= kNarrowSteps * kDepth ? (f + kDepth - 1) / kDepth : 0; }
bool takes_narrow(const Shape& S)
{
    // us, in registers and by tiles: maps 40 -> 80 at 12 000 positions 17.1 and 13.1 (weights are taken apart by a launch of their own), at 36 000 20.5 and 23.5, at
    // 100 000 33.1 and 57.8; 100 -> 200 at 12 000 22.4 and 26.1; rows of 128 -> 256 at 100 000 156 and 142
    return narrow_steps(S.f) && S.positions >= 8192 && S.positions * S.f >= 1L << 20 && (!S.axis || S.f < 128);
}
// How the forward pass goes, and its workspace: a few positions, few features, tiles that hold both halves, or shares of all [u; v] joined by a launch behind
// them.
struct Forward { bool few, narrow, split, joined; Layout shares; size_t bytes; };
Forward forward_of(const Shape& S)
{
    Forward F = {};
    F.narrow = takes_narrow(S);
    F.few = !F.narrow && S.positions <= kFewPositions;
    if (F.narrow) F.bytes = align256((size_t)narrow_bytes(narrow_steps(S.f)) * ((S.fo + 15) / 16));
    if (F.narrow || F.few) return F;
    const long I = S.axis ? S.positions : 2L * S.fo, J = S.axis ? 2L * S.fo : S.positions;
    const Layout split = layout_of(SPLIT, tiles_of(I, J, 64 * kSplitWaves, kSplitColumns), I, J, S.f, false);
    const Layout fp32 = layout_of(FP32, S.axis ? tiles_of(I, J, Tall::TI, Tall::TJ) : tiles_of(I, J, Wide::TI, Wide::TJ), I, J, S.f, false);
    F.split = split.us < fp32.us;
    const double best = F.split ? split.us : fp32.us;
    // the launch behind: 3 us, and all shares once more.  64 rows of 1024 -> 4096 49 us by tiles and 24 so, 200 rows 53 and 38
    if (best > 15.0) {
        F.shares = product_layout(I, J, S.f);
        F.joined = F.shares.us + 3.0 + 1e-6 * I * J < best;
        if (F.joined) F.bytes = align256(sizeof(float) * F.shares.shares * I * J);
    }
    return F;
}

// Shares of c [I][J] = sum over k of A B in `parts`, or all of it in c
template <bool A_ALONG, bool B_ALONG>
void product_shares(const Layout& L, const Operand& A, const Operand& B, long I, long J, long K, float* c, hipStream_t s)
{
    Product P = {{A, B, I, J, 0, 0, K}, L.T, c, L.span};
    const dim3 grid(L.T.count, (unsigned)L.shares), wide(128 * kSplitWaves);
    if (L.kind == SPLIT) ZNN_LAUNCH("gated unit product", s, (k_product_split<kSplitWaves, A_ALONG, B_ALONG, false>), grid, wide, 0, P);
    else if (L.kind == SPLIT_TURNED) {
        P.M = Matrices{B, A, J, I, 0, 0, K};
        ZNN_LAUNCH("gated unit product", s, (k_product_split<kSplitWaves, B_ALONG, A_ALONG, true>), grid, wide, 0, P);
    } else ZNN_LAUNCH("gated unit product", s, (k_product<Wide, A_ALONG, B_ALONG>), grid, dim3(Wide::kThreads), 0, P);
}
// c [I][J] = sum over k of A B, once `sums` are taken; `parts` holds product_bytes
template <bool A_ALONG, bool B_ALONG>
int product(const Layout& L, const Operand& A, const Operand& B, long I, long J, long K, float* c, float* parts, SharedSums& sums, hipStream_t s)
{
    product_shares<A_ALONG, B_ALONG>(L, A, B, I, J, K, L.shares > 1 ? parts : c, s);
    add_shares(sums, parts, c, I * J, L.shares);
    return check_launch("gated unit product");
}

// Shares of the biases' sums.  A thread adds up 1024 numbers one after another, each of one position (rows, up to 2^28 of them) or four (images), and no more: roundings of
// terms that are alike do not cancel.
struct BiasShares { int count; long span; };
BiasShares bias_shares(const Shape& S)
{
    const long across = S.axis ? (S.fo + 255) / 256 : S.fo, least = S.axis ? 32 : 1024, most = S.axis ? 4 * 1024 : 1024 * 1024;
    const long wanted = std::min(8 * kUnits / across + 1, (S.positions + least - 1) / least);
    const long count = std::min(std::max(wanted, (S.positions + most - 1) / most), 65535L);
    const long span = ((S.positions + count - 1) / count + 31) / 32 * 32;
    return BiasShares{(int)((S.positions + span - 1) / span), span};
}

// Backward with du and dv made where they are used.  us, so and by products of all of du and dv: maps 10 -> 20 at 4000 positions 29.7 and 23.6, at 12 000
// 26.7 and 23.8, at 300 000 75.7 and 120; 40 -> 80 at 4000 42.1 and 25.7, at 12 000 43.1 and 46.2, at 300 000 232 and 299; 64 -> 128 at 36 000 75.6 and 73.9, at
// 100 000 122 and 146; rows of 40 -> 80 at 4000 42.4 and 29.2, at 12 000 40.9 and 50.2, at 300 000 226 and 332; of 64 -> 128 at 12 000 53.0 and 54.6.  128 inputs take
// registers that more waves would need: 859 and 804 at 300 000.
bool takes_narrow_back(const Shape& S)
{
    return S.f <= 64 && S.positions >= 8192 && (S.axis || S.f <= 48 || S.positions >= 65536);
}
// Backward: shares of the positions, workgroups of up to kBackWaves waves of 16 features each
struct NarrowBack { int tiles, waves, shares; unsigned groups; long span; };
NarrowBack narrow_back(const Shape& S)
{
    NarrowBack N = {};
    if (!takes_narrow_back(S)) return N;
    const int tiles = (S.f + 15) / 16, features = (S.fo + 15) / 16;
    N.tiles = tiles;
    N.groups = (unsigned)((features + kBackWaves - 1) / kBackWaves);
    N.waves = std::max((int)((features + N.groups - 1) / N.groups), (N.tiles + 1) / 2);
    // what a chip holds at once: 40 -> 80 maps of 61 x 58 x 63 95 us, 108 with two thirds of that; and sums of 2^16 positions at most, where many features leave few shares
    const long wanted = std::max(1L, kUnits * (12 / N.waves) / (long)N.groups), steps = (S.positions + kDepth - 1) / kDepth;
    const long each = std::min(std::max(8L, (steps + wanted - 1) / wanted), kMostSpan / kDepth);
    N.span = each * kDepth;
    N.shares = (int)((S.positions + N.span - 1) / N.span);
    return N;
}
// How the backward pass goes, and where things lie in its workspace.
struct Backward {
    NarrowBack narrow;              // tiles 0: du and dv are stored
    Layout gx, gw;
    BiasShares bias;
    size_t sums, parts, more, bytes;
};
Backward backward_of(const Shape& S)
{
    const long both = 2L * S.fo, n = S.positions;
    Backward B = {};
    B.narrow = narrow_back(S);
    if (B.narrow.tiles) {
        B.sums = align256(sizeof(float) * both * S.f * B.narrow.shares);                        // behind the shares of gw
        B.parts = B.sums + align256(sizeof(float) * both * B.narrow.shares);                    // packed weights
        B.bytes = B.parts + align256((size_t)B.narrow.tiles * 3 * 1024 * ((S.fo + 15) / 16));
        return B;
    }
    const long I = S.axis ? n : S.f, J = S.axis ? S.f : n;
    B.gx = product_layout(I, J, both);
    B.gw = product_layout(both, S.f, n);
    B.bias = bias_shares(S);
    B.sums = align256(sizeof(float) * both * n);
    B.parts = B.sums + align256(sizeof(float) * both * B.bias.count);
    B.more = B.parts + product_bytes(B.gx, I, J);
    B.bytes = B.more + product_bytes(B.gw, both, S.f);
    return B;
}

template <class W, int AXIS>
void launch_fwd(GatedFwd G, hipStream_t s)
{
    G.T = AXIS ? tiles_of(G.M.rows_i, G.M.rows_j, W::TI, W::TJ / 2) : tiles_of(G.M.rows_i, G.M.rows_j, W::TI / 2, W::TJ);
    ZNN_LAUNCH("gated unit forward", s, (k_gated_fwd<W, AXIS>), dim3(G.T.count), dim3(W::kThreads), 0, G);
}

template <int AXIS>
void launch_fwd_split(GatedFwd G, hipStream_t s)
{
    G.T = AXIS ? tiles_of(G.M.rows_i, G.M.rows_j, 64 * kSplitWaves, kSplitColumns / 2) : tiles_of(G.M.rows_i, G.M.rows_j, 32 * kSplitWaves, kSplitColumns);
    ZNN_LAUNCH("gated unit forward", s, (k_gated_fwd_split<kSplitWaves, AXIS>), dim3(G.T.count), dim3(128 * kSplitWaves), 0, G);
}

template <int N>
void launch_few(const GatedFew& G, int axis, hipStream_t s)
{
    const dim3 grid((unsigned)((G.fo + 3) / 4), (unsigned)((G.positions + N - 1) / N));
    if (axis) ZNN_LAUNCH("gated unit forward", s, (k_gated_few<N, 1>), grid, dim3(256), 0, G);
    else ZNN_LAUNCH("gated unit forward", s, (k_gated_few<N, 0>), grid, dim3(256), 0, G);
}

template <int STEPS, int P>
void launch_narrow(const GatedNarrow& G, int axis, hipStream_t s)
{
    const long blocks = (G.positions + 64 * P - 1) / (64 * P), all = (G.fo + 15) / 16;
    GatedNarrow A = G;
    // features over several workgroups where positions alone are too few for two of them on every unit
    const long parts = std::min(all, std::max(1L, 2 * kUnits / blocks));
    A.groups = (int)((all + parts - 1) / parts);
    const dim3 grid((unsigned)blocks, (unsigned)((all + A.groups - 1) / A.groups));
    if (axis) ZNN_LAUNCH("gated unit forward", s, (k_gated_narrow<STEPS, P, 1>), grid, dim3(256), 0, A);
    else ZNN_LAUNCH("gated unit forward", s, (k_gated_narrow<STEPS, P, 0>), grid, dim3(256), 0, A);
}

int gated_fwd(const Shape& S, const Forward& F, int fn, const float* x, const float* w, const float* b, float* y, float* kept, char* ws, hipStream_t s)
{
    if (F.narrow) {
        const int steps = narrow_steps(S.f);
        const long threads = (S.fo + 15) / 16 * 2L * steps * 64;
        ZNN_LAUNCH("gated unit weights", s, k_pack_gated, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, w, S.f, S.fo, steps, ws);
        const GatedNarrow G = {x, w, b, ws, y, kept, fn, S.f, S.fo, 0, S.positions};
        if (steps == 1) launch_narrow<1, 4>(G, S.axis, s);
        else if (steps == 2) launch_narrow<2, 4>(G, S.axis, s);
        else if (steps == 3) launch_narrow<3, 2>(G, S.axis, s);
        else launch_narrow<4, 2>(G, S.axis, s);
        return check_launch("gated unit forward");
    }
    if (F.few) {
        const GatedFew G = {x, w, b, y, kept, fn, S.f, S.fo, S.positions, S.axis ? 1 : S.positions, S.axis ? S.f : 1};
        if (S.positions == 1) launch_few<1>(G, S.axis, s);
        else if (S.positions == 2) launch_few<2>(G, S.axis, s);
        else if (S.positions <= 4) launch_few<4>(G, S.axis, s);
        else launch_few<8>(G, S.axis, s);
        return check_launch("gated unit forward");
    }
    const Operand weights = {w, S.f};
    const long half = S.fo;
    if (F.joined) {
        float* const parts = (float*)ws;
        const long n = S.positions;
        if (S.axis) product_shares<true, true>(F.shares, {x, S.f}, weights, n, 2 * half, S.f, parts, s);
        else product_shares<true, false>(F.shares, weights, {x, n}, 2 * half, n, S.f, parts, s);
        const GatedJoin G = {parts, F.shares.shares, fn, S.axis, half, n, b, y, kept};
        const long quads = S.axis ? n * ((half + 3) / 4) : half * ((n + 3) / 4);
        ZNN_LAUNCH("gated unit join", s, k_gated_join, dim3((unsigned)std::min((quads + 255) / 256, 1L << 20)), dim3(256), 0, G);
        return check_launch("gated unit forward");
    }
    if (S.axis) {
        const GatedFwd G = {{{x, S.f}, weights, S.positions, S.fo, half, 0, S.f}, Tiles{}, fn, S.fo, b, y, kept, S.fo};
        if (F.split) launch_fwd_split<1>(G, s);
        else launch_fwd<Tall, 1>(G, s);
    } else {
        const GatedFwd G = {{weights, {x, S.positions}, S.fo, S.positions, half, 0, S.f}, Tiles{}, fn, S.fo, b, y, kept, S.positions};
        if (F.split) launch_fwd_split<0>(G, s);
        else launch_fwd<Wide, 0>(G, s);
    }
    return check_launch("gated unit forward");
}

template <int TILES, int AXIS>
void launch_narrow_back(const GatedBack& G, const NarrowBack& N, float* gx, char* packed, float* parts, float* sums, hipStream_t s)
{
    const long threads = (G.fo + 15) / 16 * (long)TILES * 64, each = (long)N.groups * N.waves * 64;
    const unsigned packers = gx ? (unsigned)((threads + each - 1) / each) : 0;
    ZNN_LAUNCH("gated unit weights", s, (k_gated_gw<TILES, AXIS>), dim3((unsigned)N.shares + packers, N.groups), dim3(64 * N.waves), 0, G, N.span, N.shares,
               N.waves, parts, sums, packed);
    // three workgroups stay on a unit: 40 -> 80 maps of 61 x 58 x 63 68 us, 80 with two of them, 75 with one tile a workgroup
    if (gx)
        ZNN_LAUNCH("gated unit backward", s, (k_gated_gx<TILES, AXIS>), dim3((unsigned)std::min((G.positions + 127) / 128, 3 * kUnits)), dim3(256), 0, G,
                   (const char*)packed, gx);
}

template <int AXIS>
int gated_bwd_narrow(const GatedBack& G, const Backward& B, float* gx, float* gw, float* gb, char* ws, hipStream_t s)
{
    const NarrowBack& N = B.narrow;
    char* const packed = ws + B.parts;
    float *const parts = N.shares > 1 ? (float*)ws : gw, *const sums = gb ? N.shares > 1 ? (float*)(ws + B.sums) : gb : nullptr;
    switch (N.tiles) {
        case 1: launch_narrow_back<1, AXIS>(G, N, gx, packed, parts, sums, s); break;
        case 2: launch_narrow_back<2, AXIS>(G, N, gx, packed, parts, sums, s); break;
        case 3: launch_narrow_back<3, AXIS>(G, N, gx, packed, parts, sums, s); break;
        default: launch_narrow_back<4, AXIS>(G, N, gx, packed, parts, sums, s);
    }
    SharedSums A = {};
    add_shares(A, parts, gw, 2L * G.fo * G.f, N.shares);
    if (gb) add_shares(A, sums, gb, 2L * G.fo, N.shares);
    sum_shares(A, s);
    return check_launch("gated unit backward");
}

int gated_bwd(const Shape& S, const Backward& B, int fn, const float* gy, const float* x, const float* w, const float* kept, float* gx, float* gw,
              float* gb, char* ws, hipStream_t s)
{
    if (B.narrow.tiles) {
        const GatedBack G = {gy, x, w, kept, fn, S.f, S.fo, S.positions};
        return S.axis ? gated_bwd_narrow<1>(G, B, gx, gw, gb, ws, s) : gated_bwd_narrow<0>(G, B, gx, gw, gb, ws, s);
    }
    const BiasShares& bias = B.bias;
    float *const g = (float*)ws, *const sums = (float*)(ws + B.sums), *const parts = (float*)(ws + B.parts), *const more = (float*)(ws + B.more);
    const long both = 2L * S.fo, n = S.positions;
    const Grads G = {fn, S.fo, n, bias.span, gy, kept, g, gb ? (bias.count > 1 ? sums : gb) : nullptr};
    if (S.axis) ZNN_LAUNCH("gated unit gradients", s, k_gated_grads_rows, dim3((unsigned)((S.fo + 255) / 256), (unsigned)bias.count), dim3(256), 0, G);
    else ZNN_LAUNCH("gated unit gradients", s, k_gated_grads_maps, dim3((unsigned)S.fo, (unsigned)bias.count), dim3(256), 0, G);
    int rc = check_launch("gated unit gradients");
    if (rc != ZNN_OK) return rc;
    SharedSums A = {};
    if (gb) add_shares(A, sums, gb, both, bias.count);
    if (S.axis) {
        if (gx) rc = product<true, false>(B.gx, {g, both}, {w, S.f}, n, S.f, both, gx, parts, A, s);
        if (rc == ZNN_OK) rc = product<false, false>(B.gw, {g, both}, {x, S.f}, both, S.f, n, gw, more, A, s);
    } else {
        if (gx) rc = product<false, false>(B.gx, {w, S.f}, {g, n}, S.f, n, both, gx, parts, A, s);
        if (rc == ZNN_OK) rc = product<true, true>(B.gw, {g, n}, {x, n}, both, S.f, n, gw, more, A, s);
    }
    if (rc != ZNN_OK) return rc;
    sum_shares(A, s);
    return check_launch("gated unit shares");
}

int check_gated_call(int32_t fn, size_t need, const void* ws, size_t ws_bytes)
{
    if (fn < ZNN_GATE_RECTIFY || fn > ZNN_GATE_GELU) return fail(ZNN_EINVAL, "unknown gate function %d", fn);
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

int znn_gated_workspace_bytes(int32_t fan_in, int32_t fan_out, int64_t positions, int32_t axis, int32_t pass, size_t* bytes)
{
    int rc = check_gated(fan_in, fan_out, positions, axis);
    if (rc != ZNN_OK) return rc;
    if (pass != ZNN_PASS_FWD && pass != ZNN_PASS_BWD) return fail(ZNN_EINVAL, "pass must be forward or backward");
    if (!bytes) return fail(ZNN_EINVAL, "NULL argument");
    const Shape S = {fan_in, fan_out, axis, (long)positions};
    *bytes = pass == ZNN_PASS_BWD ? backward_of(S).bytes : forward_of(S).bytes;
    return ZNN_OK;
}

int znn_gated_fwd(int32_t fn, int32_t fan_in, int32_t fan_out, int64_t positions, int32_t axis, const float* x, const float* w,
                  const float* b, float* y, float* kept, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_gated(fan_in, fan_out, positions, axis);
    if (rc != ZNN_OK) return rc;
    if (!x || !w || !y) return fail(ZNN_EINVAL, "NULL argument");
    const Shape S = {fan_in, fan_out, axis, (long)positions};
    const Forward F = forward_of(S);
    rc = check_gated_call(fn, F.bytes, ws, ws_bytes);
    const int64_t f = fan_in, both = 2LL * fan_out;
    if (rc == ZNN_OK) rc = check_apart({{y, fan_out * positions}, {kept, both * positions}}, {{x, f * positions}, {w, both * f}, {b, both}});
    if (rc != ZNN_OK) return rc;
    return gated_fwd(S, F, fn, x, w, b, y, kept, (char*)ws, (hipStream_t)stream);
}

int znn_gated_bwd(int32_t fn, int32_t fan_in, int32_t fan_out, int64_t positions, int32_t axis, const float* gy, const float* x,
                  const float* w, const float* kept, float* gx, float* gw, float* gb, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_gated(fan_in, fan_out, positions, axis);
    if (rc != ZNN_OK) return rc;
    if (!gy || !x || !w || !kept || !gw) return fail(ZNN_EINVAL, "NULL argument");
    const Shape S = {fan_in, fan_out, axis, (long)positions};
    const Backward B = backward_of(S);
    rc = check_gated_call(fn, B.bytes, ws, ws_bytes);
    const int64_t f = fan_in, both = 2LL * fan_out;
    if (rc == ZNN_OK)
        rc = check_apart({{gx, f * positions}, {gw, both * f}, {gb, both}},
                         {{gy, fan_out * positions}, {x, f * positions}, {w, both * f}, {kept, both * positions}});
    if (rc != ZNN_OK) return rc;
    return gated_bwd(S, B, fn, gy, x, w, kept, gx, gw, gb, (char*)ws, (hipStream_t)stream);
}

}  // extern "C"
