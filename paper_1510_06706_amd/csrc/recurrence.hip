// Gated recurrence along lines and its Jacobian: h_t = f_t h_(t-1) + (1 - f_t) x_t with f = logistic(z).
#include "gate.h"

#include <algorithm>

namespace znn {
namespace {

// A factor of 0 takes nothing, not even an infinity: that is how a sequence ends and how padding is passed over.
__device__ __forceinline__ float times(float a, float v) { return a == 0.f ? 0.f : a * v; }

struct Lines { long outer, length, inner; };
// `mirror`: steps are taken from the last place of a line to the first.  Forward that is the caller's `reverse`; backward, where
// gradients flow the other way, its opposite.
struct LinesFwd { Lines L; int mirror; const float *z, *x, *h0; float* h; };
struct LinesBwd { Lines L; int mirror; const float *gh, *z, *x, *h, *h0; float *gz, *gx, *gh0; };

// What a run of steps makes of the state before it: state -> a state + b.  a is a product of gates: 0 exactly where one of them is (a state
// of whatever kind is forgotten then), the smallest subnormal where it has only become too small (an infinite state stays one).
struct Run { float a, b; };
__device__ __forceinline__ float gates(float p, float q) { return fmaxf(p * q, fminf(fminf(p, q), 1.401298e-45f)); }
__device__ __forceinline__ Run then(const Run& first, const Run& next)
{
    return Run{gates(first.a, next.a), times(next.a, first.b) + next.b};
}
__device__ __forceinline__ float after(const Run& r, float state) { return times(r.a, state) + r.b; }

// ---------------------------------------------------------------- pieces of a line that wait for each other
// A line too long for one workgroup is cut into pieces, and a workgroup takes a piece where its ticket says: the pieces before it have been taken by
// workgroups that run already.  Each piece leaves what it makes of a state as soon as it has seen its own steps; the last piece of a group of pieces
// leaves what the group does, and the last piece of a group of groups leaves the state after it.  The state before a piece follows from the last such state, the
// groups since then and the pieces since the last of those, joined in one order: results do not depend on who came first, and pieces wait for a
// state to be handed on once in a group of groups only.  A record is one word of 64 bits, so that nothing has to be ordered with it; `kPending` is no
// factor (a factor is in 0 .. 1).  Everything is read once and written once; two launches that read the operands twice would move 20 instead of 12
// bytes an element forward, 32 instead of 24 backward.
constexpr unsigned kPending = 0xffffffffu;
constexpr int kPatience = 1 << 22;      // looks at a record: far more than any wait takes; then the state is NaN instead of a launch that never ends

struct Chain { unsigned* ticket; unsigned long *runs, *groups, *states; };   // ticket NULL: no piece waits for another

__global__ void __launch_bounds__(256) k_lines_begin(Chain C, long records)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) *C.ticket = 0;
    for (long i = blockIdx.x * 256L + threadIdx.x; i < records; i += gridDim.x * 256L) C.runs[i] = ~0ul;
}

__device__ __forceinline__ unsigned take_ticket(const Chain& C)
{
    __shared__ unsigned taken;
    if (!C.ticket) return blockIdx.x;
    if (threadIdx.x == 0) taken = __hip_atomic_fetch_add(C.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(taken);
}
__device__ __forceinline__ void leave(unsigned long* at, const Run& r)
{
    const unsigned long w = (unsigned long)__builtin_bit_cast(unsigned, r.b) << 32 | __builtin_bit_cast(unsigned, r.a);
    __hip_atomic_store(at, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long look(const unsigned long* at)
{
    return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Run await(const unsigned long* at, unsigned long w)
{
    for (int n = 0; (unsigned)w == kPending; ++n) {
        if (n == kPatience) return Run{0.f, __builtin_nanf("")};
        __builtin_amdgcn_s_sleep(1);
        w = look(at);
    }
    return Run{__builtin_bit_cast(float, (unsigned)w), __builtin_bit_cast(float, (unsigned)(w >> 32))};
}

// ---------------------------------------------------------------- across: a lane a line
// Lanes are neighbouring lines, so that a step of 64 lines is one or a few runs of memory.  A wave holds P steps of its lines in registers.  Of the
// waves of a workgroup `beside` lie side by side and `waves` follow each other; what they make of a state goes through shared memory.
// Bound by memory: 65536 x 512 forward 94 us with the launch before it, 4.3 TB/s (a copy: 5.07), 90 where nothing waits; 3 x 5003 x 1001 backward 110 us, 3.3 TB/s,
// its rows on no line.  Steps of a wave, us of the two: 16 and 8 98 and 115, 24 and 12 93 and 111, 32 and 16 94 and 112.

constexpr int kMostWaves = 8;

struct Across { unsigned groups, pieces; int waves, beside; Chain chain; };     // groups of 64 * beside lines, pieces of a line

constexpr int kAcrossGroup = 16;        // pieces of a group, groups of a group of groups

// What `count` records from `at` on, `row` apart, make of a state.
__device__ __forceinline__ Run join_records(const unsigned long* at, long row, int count)
{
    unsigned long w[kAcrossGroup];
#pragma unroll
    for (int i = 0; i < kAcrossGroup; ++i) w[i] = i < count ? look(at + i * row) : 0ul;
    Run seen = {1.f, 0.f};
#pragma unroll
    for (int i = 0; i < kAcrossGroup; ++i)
        if (i < count) seen = then(seen, await(at + i * row, w[i]));
    return seen;
}

// The state before this wave's steps.  All waves of the workgroup call it with what their steps make of a state.
__device__ __forceinline__ float state_before(const Run& mine, const Across& T, unsigned piece, long line, int after_waves, float first)
{
    __shared__ Run runs[kMostWaves][64], pieces[kMostWaves][64];
    __shared__ float states[kMostWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, side = wave - after_waves * T.beside;
    float state = first;
    if (T.waves > 1 || T.pieces > 1) {
        runs[wave][lane] = mine;
        __syncthreads();
    }
    if (T.pieces > 1) {
        // lines behind the last one have records of their own
        const long row = (long)T.groups * 64 * T.beside;
        const unsigned group = piece / kAcrossGroup, at = piece % kAcrossGroup, far = group / kAcrossGroup, group_at = group % kAcrossGroup;
        const bool last = piece + 1 == T.pieces;
        Run all = mine;
        if (after_waves == 0) {
            for (int w = 1; w < T.waves; ++w) all = then(all, runs[w * T.beside + side][lane]);
            if (at + 1 < kAcrossGroup && !last) leave(T.chain.runs + piece * row + line, all);
            const Run seen = join_records(T.chain.runs + (piece - at) * row + line, row, (int)at);
            if (at + 1 == kAcrossGroup && group_at + 1 < kAcrossGroup && !last) leave(T.chain.groups + group * row + line, then(seen, all));
            pieces[side][lane] = seen;
        } else if (after_waves == 1) {
            const Run seen = join_records(T.chain.groups + (group - group_at) * row + line, row, (int)group_at);
            if (far) {
                const unsigned long* const before = T.chain.states + (far - 1) * row + line;
                state = await(before, look(before)).b;
            }
            states[side][lane] = after(seen, state);
        }
        __syncthreads();
        state = after(pieces[side][lane], states[side][lane]);
        if (after_waves == 0 && at + 1 == kAcrossGroup && group_at + 1 == kAcrossGroup && !last)
            leave(T.chain.states + far * row + line, Run{0.f, after(all, state)});
    }
    for (int w = 0; w < after_waves; ++w) state = after(runs[w * T.beside + side][lane], state);
    return state;
}

template <int P>
__global__ void __launch_bounds__(64 * kMostWaves) k_lines_across(LinesFwd A, Across T)
{
    const unsigned ticket = take_ticket(T.chain), piece = ticket / T.groups, group = ticket - piece * T.groups;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, later = wave / T.beside, side = wave - later * T.beside;
    const long lines = A.L.outer * A.L.inner, line = (group * (long)T.beside + side) * 64 + lane, l = line < lines ? line : lines - 1;
    const long o = l / A.L.inner, step = A.mirror ? -A.L.inner : A.L.inner;
    const long t0 = ((long)piece * T.waves + later) * P, left = A.L.length - t0;
    const int n = left > P ? P : left > 0 ? (int)left : 0;       // uniform in a wave
    const long at = (o * A.L.length + (A.mirror ? A.L.length - 1 - t0 : t0)) * A.L.inner + (l - o * A.L.inner);
    float f[P], b[P];
    const float *pz = A.z + at, *px = A.x + at;
#pragma unroll
    for (int i = 0; i < P; ++i, pz += step, px += step)
        if (i < n) { f[i] = *pz; b[i] = *px; }
    Run mine = {1.f, 0.f};
#pragma unroll
    for (int i = 0; i < P; ++i)
        if (i < n) {
            const Gate g = gate(f[i]);
            f[i] = g.f;
            b[i] = times(g.k, b[i]);
            mine = then(mine, Run{f[i], b[i]});
        }
    float h = state_before(mine, T, piece, line, later, A.h0 ? A.h0[l] : 0.f);
    if (line >= lines) return;
    float* ph = A.h + at;
#pragma unroll
    for (int i = 0; i < P; ++i, ph += step)
        if (i < n) *ph = h = times(f[i], h) + b[i];
}

// What flows backwards is q_t = f_t G_t with G_t = gh_t + q_(t+1): the factors of a step are its own.  Of G and the difference the larger one is multiplied by f (1 - f)
// first: their product may leave the range where gz does not.
__device__ __forceinline__ float grads(const Gate& g, float G, float before, float x, float& gz)
{
    const float d = before - x;
    const bool swap = fabsf(G) > fabsf(d);
    gz = g.f == 0.f || g.k == 0.f ? 0.f : (swap ? G : d) * (g.f * g.k) * (swap ? d : G);
    return times(g.k, G);
}

template <int P>
__global__ void __launch_bounds__(64 * kMostWaves) k_lines_across_bwd(LinesBwd A, Across T)
{
    const unsigned ticket = take_ticket(T.chain), piece = ticket / T.groups, group = ticket - piece * T.groups;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, later = wave / T.beside, side = wave - later * T.beside;
    const long lines = A.L.outer * A.L.inner, line = (group * (long)T.beside + side) * 64 + lane, l = line < lines ? line : lines - 1;
    const long o = l / A.L.inner, step = A.mirror ? -A.L.inner : A.L.inner;
    const long t0 = ((long)piece * T.waves + later) * P, left = A.L.length - t0;
    const int n = left > P ? P : left > 0 ? (int)left : 0;
    const long at = (o * A.L.length + (A.mirror ? A.L.length - 1 - t0 : t0)) * A.L.inner + (l - o * A.L.inner);
    float z[P], gh[P], x[P], before[P];
    const float h0 = A.h0 ? A.h0[l] : 0.f;
    const float *pz = A.z + at, *pg = A.gh + at, *px = A.x + at, *ph = A.h + at + step;
#pragma unroll
    for (int i = 0; i < P; ++i, pz += step, pg += step)
        if (i < n) { z[i] = *pz; gh[i] = *pg; }
#pragma unroll
    for (int i = 0; i < P; ++i, px += step, ph += step)
        if (i < n) { x[i] = *px; before[i] = i < n - 1 || n < left ? *ph : h0; }
    Run mine = {1.f, 0.f};
#pragma unroll
    for (int i = 0; i < P; ++i)
        if (i < n) {
            const float f = gate(z[i]).f;
            mine = then(mine, Run{f, times(f, gh[i])});
        }
    float q = state_before(mine, T, piece, line, later, 0.f);
    if (line >= lines) return;
    float *qx = A.gx + at, *qz = A.gz + at;
#pragma unroll
    for (int i = 0; i < P; ++i, qx += step, qz += step)
        if (i < n) {
            const Gate g = gate(z[i]);
            const float G = gh[i] + q;
            *qx = grads(g, G, before[i], x[i], *qz);
            q = times(g.f, G);
        }
    if (A.gh0 && n > 0 && t0 + n == A.L.length) A.gh0[l] = q;
}

// ---------------------------------------------------------------- along: lanes follow a line
// Lines along the fastest extent lie one behind the other, so that the array is one line of outer * length steps in which a line begins every
// `length` steps: a step whose gate takes nothing of the state before it.  A lane holds quads of four neighbouring steps, a wave Q rows of 64
// quads, one after the other; the W waves of a workgroup follow each other.  Bound by memory, and by vector instructions next: 144 000 lines of 60 forward
// 22.8 us (4.55 TB/s), backward 45 (4.6).

constexpr int kFarOff = 1 << 30;
typedef float floatu4 __attribute__((ext_vector_type(4), aligned(4)));      // lines begin at any element

// steps in all and of a workgroup; min(length, kFarOff)
struct Along { long steps; int tile; FastDiv line; Chain chain; };

// The beginnings of lines in a tile.
struct Tile {
    long first;                 // the tile's first step
    int count;                  // its steps
    long line;                  // the line of the first one
    int left;                   // steps of that line from there on, at most kFarOff
    bool begins;                // with its first one
};
__device__ __forceinline__ Tile tile_of(const Lines& L, const Along& T, unsigned number)
{
    const long first = (long)number * T.tile, line = first / L.length, pos = first - line * L.length, left = L.length - pos;
    return Tile{first, (int)(T.steps - first < T.tile ? T.steps - first : T.tile), line, left < kFarOff ? (int)left : kFarOff, pos == 0};
}
// From step `off` of the tile on: its line, whether that begins there, and in how many steps the next one does.
struct Run4 { long line; int until; bool begins; };
__device__ __forceinline__ Run4 place_in_line(const Tile& S, const FastDiv& length, int off)
{
    if (off < S.left) return Run4{S.line, S.left - off, S.begins && off == 0};
    const unsigned u = (unsigned)(off - S.left), n = fdiv_any(u, length), pos = u - n * length.d;
    return Run4{S.line + 1 + n, (int)(length.d - pos), pos == 0};
}
// Does a line begin at the j-th step from there?  Called for j = 1, 2, 3 (4) in order.
__device__ __forceinline__ bool next_begins(Run4& R, const FastDiv& length, int j)
{
    if (j != R.until) return false;
    R.until += (int)length.d;
    ++R.line;
    return true;
}

// Four steps from step e on; `most` of them are there.  Memory runs against the steps where mirrored: step 0 is element `last` then.
__device__ __forceinline__ void load_steps(float (&v)[4], const float* p, long e, int most, bool mirror, long last)
{
    if (most >= 4) {
        const floatu4 q = *(const floatu4*)(mirror ? p + (last - 3 - e) : p + e);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = mirror ? q[3 - j] : q[j];
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = j < most ? (mirror ? p[last - e - j] : p[e + j]) : 0.f;
    }
}
__device__ __forceinline__ void store_steps(const float (&v)[4], float* p, long e, int most, bool mirror, long last)
{
    if (most >= 4) {
        floatu4 q;
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = mirror ? v[3 - j] : v[j];
        *(floatu4*)(mirror ? p + (last - 3 - e) : p + e) = q;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < most) (mirror ? p[last - e - j] : p[e + j]) = v[j];
    }
}

// The value of another lane, by the data path between lanes: `none` where there is no such lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ float other_lane(float none, float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ Run other_lane(const Run& r) { return Run{other_lane<CTRL, ROWS>(1.f, r.a), other_lane<CTRL, ROWS>(0.f, r.b)}; }
__device__ __forceinline__ float last_lane(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// What this lane and those before it make of a state: rows of 16 lanes, then the last lane of the row and of the two rows before.
__device__ __forceinline__ Run scan_lanes(Run r)
{
    r = then(other_lane<0x111>(r), r);          // one to eight lanes up in a row
    r = then(other_lane<0x112>(r), r);
    r = then(other_lane<0x114>(r), r);
    r = then(other_lane<0x118>(r), r);
    r = then(other_lane<0x142, 0xa>(r), r);     // lane 15 of the row before to rows 1 and 3
    r = then(other_lane<0x143, 0xc>(r), r);     // lane 31 to rows 2 and 3
    return r;
}
// The same without this lane (`before`) and for all lanes (the result).
__device__ __forceinline__ Run scan_lanes(const Run& mine, Run& before)
{
    const Run r = scan_lanes(mine);
    before = other_lane<0x138>(r);              // one lane up in the wave
    return Run{last_lane(r.a), last_lane(r.b)};
}

constexpr int kAlongGroup = 64;         // pieces of a group, groups of a group of groups: a lane a record

// What `count` records from `at` on make of a state.
__device__ __forceinline__ Run join_records(const unsigned long* at, int count)
{
    const int lane = threadIdx.x & 63;
    const Run r = scan_lanes(lane < count ? await(at + lane, look(at + lane)) : Run{1.f, 0.f});
    return Run{last_lane(r.a), last_lane(r.b)};
}

// The state before this wave's steps.
template <int W>
__device__ __forceinline__ float state_before(const Run& mine, const Along& T, unsigned number)
{
    __shared__ Run runs[W], pieces;
    __shared__ float state_of_groups;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) runs[wave] = mine;
    __syncthreads();
    float state = 0.f;
    if (T.chain.ticket) {
        const unsigned group = number / kAlongGroup, at = number % kAlongGroup, far = group / kAlongGroup, group_at = group % kAlongGroup;
        Run all = mine;
        if (wave == 0) {
            for (int w = 1; w < W; ++w) all = then(all, runs[w]);
            if (lane == 0 && at + 1 < kAlongGroup) leave(T.chain.runs + number, all);
            const Run seen = join_records(T.chain.runs + (number - at), (int)at);
            if (lane == 0 && at + 1 == kAlongGroup && group_at + 1 < kAlongGroup) leave(T.chain.groups + group, then(seen, all));
            if (lane == 0) pieces = seen;
        } else if (wave == 1) {
            const Run seen = join_records(T.chain.groups + (group - group_at), (int)group_at);
            if (seen.a != 0.f && far) {
                const unsigned long* const before = T.chain.states + (far - 1);
                state = await(before, look(before)).b;
            }
            if (lane == 0) state_of_groups = after(seen, state);
        }
        __syncthreads();
        state = after(pieces, state_of_groups);
        if (threadIdx.x == 0 && at + 1 == kAlongGroup && group_at + 1 == kAlongGroup) leave(T.chain.states + far, Run{0.f, after(all, state)});
    }
    for (int w = 0; w < wave; ++w) state = after(runs[w], state);
    return state;
}

template <int Q, int W>
__global__ void __launch_bounds__(64 * W) k_lines_along(LinesFwd A, Along T)
{
    const unsigned number = take_ticket(T.chain);
    const Tile S = tile_of(A.L, T, number);
    const int off0 = (threadIdx.x >> 6) * (256 * Q) + (threadIdx.x & 63) * 4;
    float f[Q][4], b[Q][4];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int off = off0 + q * 256;
        load_steps(f[q], A.z, S.first + off, S.count - off, A.mirror, T.steps - 1);
        load_steps(b[q], A.x, S.first + off, S.count - off, A.mirror, T.steps - 1);
    }
    Run mine = {1.f, 0.f}, before[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int off = off0 + q * 256;
        Run4 R = place_in_line(S, T.line, off);
        Run r = {1.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool begins = j ? next_begins(R, T.line, j) : R.begins, there = off + j < S.count;
            const Gate g = gate(f[q][j]);
            f[q][j] = there ? g.f : 1.f;
            b[q][j] = there ? times(g.k, b[q][j]) : 0.f;
            if (begins && there) {
                if (A.h0) b[q][j] += times(g.f, A.h0[A.mirror ? A.L.outer - 1 - R.line : R.line]);
                f[q][j] = 0.f;
            }
            r = then(r, Run{f[q][j], b[q][j]});
        }
        const Run all = scan_lanes(r, before[q]);
        before[q] = then(mine, before[q]);
        mine = then(mine, all);
    }
    const float first = state_before<W>(mine, T, number);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int off = off0 + q * 256;
        float h = after(before[q], first);
#pragma unroll
        for (int j = 0; j < 4; ++j) b[q][j] = h = times(f[q][j], h) + b[q][j];
        store_steps(b[q], A.h, S.first + off, S.count - off, A.mirror, T.steps - 1);
    }
}

template <int Q, int W>
__global__ void __launch_bounds__(64 * W) k_lines_along_bwd(LinesBwd A, Along T)
{
    const unsigned number = take_ticket(T.chain);
    const Tile S = tile_of(A.L, T, number);
    const int off0 = (threadIdx.x >> 6) * (256 * Q) + (threadIdx.x & 63) * 4;
    const long last = T.steps - 1;
    float z[Q][4], gh[Q][4], x[Q][4], h[Q][4];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int off = off0 + q * 256;
        load_steps(z[q], A.z, S.first + off, S.count - off, A.mirror, last);
        load_steps(gh[q], A.gh, S.first + off, S.count - off, A.mirror, last);
        load_steps(x[q], A.x, S.first + off, S.count - off, A.mirror, last);
        // the step before is the next one here
        const long e = S.first + off + 1;
        load_steps(h[q], A.h, e, off >= S.count ? 0 : T.steps - e < 4 ? (int)(T.steps - e) : 4, A.mirror, last);
    }
    Run mine = {1.f, 0.f}, before[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int off = off0 + q * 256;
        Run4 R = place_in_line(S, T.line, off);
        Run r = {1.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool begins = j ? next_begins(R, T.line, j) : R.begins, there = off + j < S.count;
            const float f = gate(z[q][j]).f;
            if (there) r = then(r, Run{begins ? 0.f : f, times(f, gh[q][j])});
        }
        const Run all = scan_lanes(r, before[q]);
        before[q] = then(mine, before[q]);
        mine = then(mine, all);
    }
    const float first = state_before<W>(mine, T, number);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int off = off0 + q * 256, most = S.count - off;
        Run4 R = place_in_line(S, T.line, off);
        float state = after(before[q], first);
        if (R.begins) state = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long line = A.mirror ? A.L.outer - 1 - R.line : R.line;
            const bool ends = next_begins(R, T.line, j + 1);
            const Gate g = gate(z[q][j]);
            const float G = gh[q][j] + state;
            if (ends && j < most) h[q][j] = A.h0 ? A.h0[line] : 0.f;
            float gz;
            x[q][j] = grads(g, G, h[q][j], x[q][j], gz);
            z[q][j] = gz;
            state = times(g.f, G);
            if (ends) {
                if (A.gh0 && j < most) A.gh0[line] = state;
                state = 0.f;
            }
        }
        store_steps(x[q], A.gx, S.first + off, most, A.mirror, last);
        store_steps(z[q], A.gz, S.first + off, most, A.mirror, last);
    }
}

// ---------------------------------------------------------------- many lines: a lane a line from its first step to its last
// Where lines alone fill the chip nothing has to be joined: a lane walks its line, the operands of U steps requested together.  Bound by memory: 120 x 96^3 along z
// forward 245 us, backward 497 (5.2 and 5.1 TB/s); by pieces 254 and 723.

template <int U>
__global__ void __launch_bounds__(256) k_lines_walk(LinesFwd A)
{
    const long lines = A.L.outer * A.L.inner, step = A.mirror ? -A.L.inner : A.L.inner;
    for (long l = blockIdx.x * 256L + threadIdx.x; l < lines; l += gridDim.x * 256L) {
        const long o = l / A.L.inner;
        const long at = (o * A.L.length + (A.mirror ? A.L.length - 1 : 0)) * A.L.inner + (l - o * A.L.inner);
        float h = A.h0 ? A.h0[l] : 0.f;
        const float *pz = A.z + at, *px = A.x + at;
        float* ph = A.h + at;
        for (long left = A.L.length; left > 0; left -= U) {
            float z[U], x[U];
#pragma unroll
            for (int i = 0; i < U; ++i, pz += step, px += step)
                if (i < left) { z[i] = *pz; x[i] = *px; }
#pragma unroll
            for (int i = 0; i < U; ++i, ph += step)
                if (i < left) {
                    const Gate g = gate(z[i]);
                    *ph = h = times(g.f, h) + times(g.k, x[i]);
                }
        }
    }
}

template <int U>
__global__ void __launch_bounds__(256) k_lines_walk_bwd(LinesBwd A)
{
    const long lines = A.L.outer * A.L.inner, step = A.mirror ? -A.L.inner : A.L.inner;
    for (long l = blockIdx.x * 256L + threadIdx.x; l < lines; l += gridDim.x * 256L) {
        const long o = l / A.L.inner;
        const long at = (o * A.L.length + (A.mirror ? A.L.length - 1 : 0)) * A.L.inner + (l - o * A.L.inner);
        const float h0 = A.h0 ? A.h0[l] : 0.f;
        float q = 0.f;
        const float *pz = A.z + at, *px = A.x + at, *pg = A.gh + at, *ph = A.h + at + step;
        float *qx = A.gx + at, *qz = A.gz + at;
        for (long left = A.L.length; left > 0; left -= U) {
            float z[U], x[U], gh[U], before[U];
#pragma unroll
            for (int i = 0; i < U; ++i, pz += step, px += step, pg += step, ph += step)
                if (i < left) {
                    z[i] = *pz; x[i] = *px; gh[i] = *pg;
                    before[i] = i + 1 < left ? *ph : h0;
                }
#pragma unroll
            for (int i = 0; i < U; ++i, qx += step, qz += step)
                if (i < left) {
                    const Gate g = gate(z[i]);
                    const float G = gh[i] + q;
                    *qx = grads(g, G, before[i], x[i], *qz);
                    q = times(g.f, G);
                }
        }
        if (A.gh0) A.gh0[l] = q;
    }
}

// ---------------------------------------------------------------- the choice
enum Way { WALK, ACROSS, ALONG };
constexpr int kSteps = 32, kStepsBwd = 16;      // of a wave across
struct Split {
    Way way;
    int waves, beside;      // of a workgroup: one after another, side by side
    long groups, pieces;    // across: groups of lines, pieces of a line; along: tiles
    int quads, tile;        // along: rows of a wave, steps of a tile
    bool chained;
};

Split lines_split(const Lines& L, bool backward)
{
    Split S = {};
    const long lines = L.outer * L.inner;
    if (L.inner == 1) {
        const long steps = L.outer * L.length;
        S.way = ALONG;
        S.beside = 1;
        // Whole lines in a tile where they fill it, so that no tile waits for another, in the smaller one where that does: 144 000 lines of 60
        // forward 24.6 us in tiles of 512, 27.7 of 2048; backward 44.9 and 48.6.  A launch has fewer than 2^32 threads, and these take three or four steps each, six to
        // eight in the larger tiles.
        S.chained = true;
        for (int small = steps < 1L << 33; small >= 0 && S.chained && steps <= 1L << 34; --small) {
            S.quads = small ? 1 : 2;
            S.waves = small ? 2 : 4;
            const long most = 256 * S.quads * S.waves, whole = most / L.length * L.length;
            if (4 * whole >= 3 * most) {
                S.chained = false;
                S.tile = (int)whole;
            }
        }
        // Else large tiles, as tickets are handed out one every 13 to 17 ns; those of 8192 and 4096 steps leave room for two workgroups and more on a unit, which
        // pays where there are many: 4 lines of 10^6 forward 21.8 us with 16 384, 25.6 with 8192, backward 35.5 and 45; 64 lines 277 and 239, 478 and 434.
        if (S.chained) {
            S.quads = 4;
            S.waves = 16;
            if (steps > 1L << 23) {
                S.waves = 8;
                if (backward) S.quads = 2;
            }
            S.tile = 256 * S.quads * S.waves;
        }
        S.pieces = (steps + S.tile - 1) / S.tile;
        S.groups = 1;
        S.chained = S.chained && S.pieces > 1;
        return S;
    }
    const int steps = backward ? kStepsBwd : kSteps;
    if (lines >= 1L << 17 || L.length <= steps / 2) return S;
    S.way = ACROSS;
    S.beside = lines > 1024 ? 2 : 1;
    S.waves = (int)std::min((L.length + steps - 1) / steps, (long)(kMostWaves / S.beside));
    if (L.length > S.waves * steps) S.waves = kMostWaves / S.beside;
    S.pieces = (L.length + S.waves * steps - 1) / (S.waves * steps);
    S.groups = (lines + 64 * S.beside - 1) / (64 * S.beside);
    S.chained = S.pieces > 1;
    return S;
}

// Records of pieces, groups of them and groups of these
struct Records { size_t runs, groups, states; size_t all() const { return runs + groups + states; } };
Records records_of(const Split& S)
{
    const size_t row = S.way == ACROSS ? (size_t)S.groups * 64 * S.beside : 1, group = S.way == ACROSS ? kAcrossGroup : kAlongGroup;
    return Records{S.pieces * row, S.pieces / group * row, S.pieces / (group * group) * row};
}
size_t split_bytes(const Split& S) { return S.chained ? 256 + sizeof(unsigned long) * records_of(S).all() : 0; }

int begin_lines(const Split& S, void* ws, Chain* C, hipStream_t s)
{
    *C = Chain{};
    if (!S.chained) return ZNN_OK;
    unsigned long* const runs = (unsigned long*)((char*)ws + 256);
    const Records R = records_of(S);
    *C = Chain{(unsigned*)ws, runs, runs + R.runs, runs + R.runs + R.groups};
    const long records = (long)R.all();
    ZNN_LAUNCH("recurrence pieces", s, k_lines_begin, dim3((unsigned)std::min((records + 255) / 256, 2048L)), dim3(256), 0, *C, records);
    return check_launch("recurrence pieces");
}

unsigned walk_groups(const Lines& L) { return (unsigned)std::min((L.outer * L.inner + 255) / 256, 1L << 20); }
Along along(const Lines& L, const Split& S, const Chain& C)
{
    return Along{L.outer * L.length, S.tile, make_fastdiv((unsigned)std::min(L.length, (long)kFarOff)), C};
}

// launch(grid, block) for all workgroups of a split.  A launch has fewer than 2^32 threads; pieces of lines may need more, as lines across fill up to whole waves
// (2^31 steps of two lines are 2^32 threads): the next launch goes on where the tickets of the last one end.
template <class Launch>
void for_all_pieces(const Split& S, Launch launch)
{
    const dim3 block(64 * S.waves * S.beside);
    const long all = S.groups * S.pieces, most = S.chained ? (1L << 31) / block.x : all;
    for (long first = 0; first < all; first += most) launch(dim3((unsigned)std::min(all - first, most)), block);
}

int lines_fwd(const LinesFwd& A, void* ws, hipStream_t s)
{
    const Split S = lines_split(A.L, false);
    Chain C;
    const int rc = begin_lines(S, ws, &C, s);
    if (rc != ZNN_OK) return rc;
    if (S.way == ALONG) {
        const Along T = along(A.L, S, C);
        for_all_pieces(S, [&](dim3 grid, dim3 block) {
            if (S.waves == 2) ZNN_LAUNCH("recurrence forward", s, (k_lines_along<1, 2>), grid, block, 0, A, T);
            else if (S.waves == 4) ZNN_LAUNCH("recurrence forward", s, (k_lines_along<2, 4>), grid, block, 0, A, T);
            else if (S.waves == 8) ZNN_LAUNCH("recurrence forward", s, (k_lines_along<4, 8>), grid, block, 0, A, T);
            else ZNN_LAUNCH("recurrence forward", s, (k_lines_along<4, 16>), grid, block, 0, A, T);
        });
    } else if (S.way == ACROSS) {
        const Across T = {(unsigned)S.groups, (unsigned)S.pieces, S.waves, S.beside, C};
        for_all_pieces(S, [&](dim3 grid, dim3 block) { ZNN_LAUNCH("recurrence forward", s, k_lines_across<kSteps>, grid, block, 0, A, T); });
    } else ZNN_LAUNCH("recurrence forward", s, k_lines_walk<8>, dim3(walk_groups(A.L)), dim3(256), 0, A);
    return check_launch("recurrence forward");
}

int lines_bwd(const LinesBwd& A, void* ws, hipStream_t s)
{
    const Split S = lines_split(A.L, true);
    Chain C;
    const int rc = begin_lines(S, ws, &C, s);
    if (rc != ZNN_OK) return rc;
    if (S.way == ALONG) {
        const Along T = along(A.L, S, C);
        for_all_pieces(S, [&](dim3 grid, dim3 block) {
            if (S.waves == 2) ZNN_LAUNCH("recurrence backward", s, (k_lines_along_bwd<1, 2>), grid, block, 0, A, T);
            else if (S.waves == 4) ZNN_LAUNCH("recurrence backward", s, (k_lines_along_bwd<2, 4>), grid, block, 0, A, T);
            else if (S.waves == 8) ZNN_LAUNCH("recurrence backward", s, (k_lines_along_bwd<2, 8>), grid, block, 0, A, T);
            else ZNN_LAUNCH("recurrence backward", s, (k_lines_along_bwd<4, 16>), grid, block, 0, A, T);
        });
    } else if (S.way == ACROSS) {
        const Across T = {(unsigned)S.groups, (unsigned)S.pieces, S.waves, S.beside, C};
        for_all_pieces(S, [&](dim3 grid, dim3 block) { ZNN_LAUNCH("recurrence backward", s, k_lines_across_bwd<kStepsBwd>, grid, block, 0, A, T); });
    } else ZNN_LAUNCH("recurrence backward", s, k_lines_walk_bwd<4>, dim3(walk_groups(A.L)), dim3(256), 0, A);
    return check_launch("recurrence backward");
}

int check_lines(int64_t outer, int64_t length, int64_t inner)
{
    if (outer < 1 || length < 1 || inner < 1) return fail(ZNN_EINVAL, "extents must be >= 1");
    constexpr int64_t most = 1LL << 34;
    if (outer > most || length > most || inner > most || (double)outer * length * inner > 274877906944.0)
        return fail(ZNN_EUNSUPPORTED, "lines of %lld x %lld x %lld elements are too large", (long long)outer, (long long)length, (long long)inner);
    return ZNN_OK;
}

size_t lines_workspace(const Lines& L) { return std::max(split_bytes(lines_split(L, false)), split_bytes(lines_split(L, true))); }

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
    *bytes = lines_workspace(Lines{(long)outer, (long)length, (long)inner});
    return ZNN_OK;
}

int znn_recurrence_fwd(int64_t outer, int64_t length, int64_t inner, int32_t reverse, const float* z, const float* x, const float* h0,
                       float* h, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_lines(outer, length, inner);
    if (rc != ZNN_OK) return rc;
    if (!z || !x || !h) return fail(ZNN_EINVAL, "NULL argument");
    const LinesFwd A = {{(long)outer, (long)length, (long)inner}, reverse != 0, z, x, h0, h};
    rc = check_lines_workspace(A.L, ws, ws_bytes);
    const int64_t lines = outer * inner, all = lines * length;
    if (rc == ZNN_OK) rc = check_apart({{h, all}}, {{z, all}, {x, all}, {h0, lines}});
    if (rc != ZNN_OK) return rc;
    return lines_fwd(A, ws, (hipStream_t)stream);
}

int znn_recurrence_bwd(int64_t outer, int64_t length, int64_t inner, int32_t reverse, const float* gh, const float* z, const float* x,
                       const float* h, const float* h0, float* gz, float* gx, float* gh0, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_lines(outer, length, inner);
    if (rc != ZNN_OK) return rc;
    if (!gh || !z || !x || !h || !gz || !gx) return fail(ZNN_EINVAL, "NULL argument");
    const LinesBwd A = {{(long)outer, (long)length, (long)inner}, reverse == 0, gh, z, x, h, h0, gz, gx, gh0};
    rc = check_lines_workspace(A.L, ws, ws_bytes);
    const int64_t lines = outer * inner, all = lines * length;
    if (rc == ZNN_OK) rc = check_apart({{gz, all}, {gx, all}, {gh0, lines}}, {{gh, all}, {z, all}, {x, all}, {h, all}, {h0, lines}});
    if (rc != ZNN_OK) return rc;
    return lines_bwd(A, ws, (hipStream_t)stream);
}

}  // extern "C"
