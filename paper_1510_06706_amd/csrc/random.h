// Random numbers for dropout: a function of where an element lies, so that no mask is ever stored and the backward pass
// draws the forward pass's numbers again.
//
// The generator is Philox4x32 with ten rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", SC 2011): a bijection of a counter of four 32-bit words under a key of two.  The key is the seed, the counter
// (column / 4, row, site, round); column c takes word c mod 4.
#pragma once

#include "znn_internal.h"

namespace znn {

typedef float floatu4 __attribute__((ext_vector_type(4), aligned(4)));     // rows start at any element

// What a call drops: an element stays where its word is less than `keep`.
struct Drop { const uint64_t* state; unsigned site, keep; float scale; };

struct DropKey { unsigned k0, k1, site, round, keep; float scale; };
__device__ __forceinline__ DropKey drop_key(const Drop& D)
{
    const uint64_t seed = D.state[0], round = D.state[1];
    return DropKey{(unsigned)seed, (unsigned)(seed >> 32), D.site, (unsigned)round, D.keep, D.scale};
}

struct Words { unsigned w[4]; };
__device__ __forceinline__ Words drop_words(const DropKey& K, unsigned quad, unsigned row)
{
    unsigned c0 = quad, c1 = row, c2 = K.site, c3 = K.round, k0 = K.k0, k1 = K.k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
        c0 = (unsigned)(p1 >> 32) ^ c1 ^ k0;
        c1 = (unsigned)p1;
        c2 = (unsigned)(p0 >> 32) ^ c3 ^ k1;
        c3 = (unsigned)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words{{c0, c1, c2, c3}};
}

// A dropped element is zero whatever it held.
__device__ __forceinline__ float dropped(const DropKey& K, unsigned word, float v) { return word < K.keep ? v * K.scale : 0.f; }

// Elements 4 quad + e of a row, e < count.
__device__ __forceinline__ floatu4 dropped4(const DropKey& K, unsigned quad, unsigned row, floatu4 v)
{
    const Words u = drop_words(K, quad, row);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = dropped(K, u.w[e], v[e]);
    return v;
}

// count <= 4 elements from p on, 0 behind them
__device__ __forceinline__ floatu4 load4(const float* p, int count)
{
    if (count >= 4) return *reinterpret_cast<const floatu4*>(p);
    floatu4 v = {0.f, 0.f, 0.f, 0.f};
    if (count > 0) v[0] = p[0];
    if (count > 1) v[1] = p[1];
    if (count > 2) v[2] = p[2];
    return v;
}
__device__ __forceinline__ void store4(float* p, int count, floatu4 v)
{
    if (count >= 4) { *reinterpret_cast<floatu4*>(p) = v; return; }
    if (count > 0) p[0] = v[0];
    if (count > 1) p[1] = v[1];
    if (count > 2) p[2] = v[2];
}

}  // namespace znn
