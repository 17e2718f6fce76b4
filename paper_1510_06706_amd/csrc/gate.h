// The logistic function of a gate, for the gated recurrence and the gated unit.
#pragma once

#include "znn_internal.h"

namespace znn {

// f = 1 / (1 + exp(-z)) and k = 1 - f = 1 / (1 + exp(z)), each to its own last digits: 1 - f would have lost those of a gate that is nearly open.
// exp(-|z|) is 2^t times a correction for what t, rounded, leaves of |z| / ln 2; the quotient takes one step of Newton's method.  Both are within a
// few half-steps, in 15 instructions; expf and a division take 35, and the arithmetic of gates stands beside the memory's time.  Below 2^-126 both are 0.
struct Gate { float f, k; };
__device__ __forceinline__ Gate gate(float z)
{
    const float m = fabsf(z) > 1e30f ? 1e30f : fabsf(z), t = m * -1.44269502f;        // NaN stays
    const float rest = fmaf(m, -1.44269502f, -t) + m * -1.92596299e-8f;     // of -|z| / ln 2 = -|z| (1.44269502 + 1.92596299e-8)
    float e = __builtin_amdgcn_exp2f(t);
    e = fmaf(e, rest * 0.693147182f, e);
    const float d = 1.f + e, guess = __builtin_amdgcn_rcpf(d), large = fmaf(fmaf(-d, guess, 1.f), guess, guess), small = e * large;
    return z < 0.f ? Gate{small, large} : Gate{large, small};
}

}  // namespace znn
