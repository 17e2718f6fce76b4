// What the gated recurrence and the gated unit share: the logistic function of a gate, and the check that results have memory of their own.
#pragma once

#include "znn_internal.h"

#include <initializer_list>

namespace znn {

// f = 1 / (1 + exp(-z)) and k = 1 - f = 1 / (1 + exp(z)), each to its own last digits: 1 - f would have lost those of a gate that is nearly open.
// exp(-|z|) = 2^n 2^r with a whole n and |r| <= 1/2, r by two fused steps (1 / ln 2 = 1.44269502 + 1.92596299e-8) so that it keeps its digits; 2^n goes on
// last, so that the smaller of both is rounded to subnormals from 2^-126 on and is 0 below 2^-150 only, from |z| = 104 on: until then it is a factor,
// and what is not finite passes it.  n stays at that of 200, where r goes on; a z that is NaN makes r NaN.  The quotient takes one step of Newton's method.
// Both are within a few half-steps, in 16 instructions; expf and a division take 35, and the arithmetic of gates stands beside the memory's time.
struct Gate { float f, k; };
__device__ __forceinline__ Gate gate(float z)
{
    const float m = fabsf(z), n = __builtin_rintf(__builtin_amdgcn_fmed3f(m, 0.f, 200.f) * -1.44269502f);
    const float r = fmaf(m, -1.92596299e-8f, fmaf(m, -1.44269502f, -n)), e = __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(r), (int)n);
    const float d = 1.f + e, guess = __builtin_amdgcn_rcpf(d), large = fmaf(fmaf(-d, guess, 1.f), guess, guess), small = e * large;
    return z < 0.f ? Gate{small, large} : Gate{large, small};
}

// Results are written while operands are read, by other workgroups among them: one that shares memory with an operand or another result would change it
// on the way.  Arrays that are not there are NULL.
struct Span { const void* first; int64_t floats; };
inline int check_apart(std::initializer_list<Span> results, std::initializer_list<Span> operands)
{
    auto share = [](const Span& a, const Span& b) {
        const uintptr_t p = (uintptr_t)a.first, q = (uintptr_t)b.first;
        return p && q && p < q + 4 * (uintptr_t)b.floats && q < p + 4 * (uintptr_t)a.floats;
    };
    for (const Span* r = results.begin(); r != results.end(); ++r) {
        for (const Span* other = r + 1; other != results.end(); ++other)
            if (share(*r, *other)) return fail(ZNN_EINVAL, "two results share memory");
        for (const Span& o : operands)
            if (share(*r, o)) return fail(ZNN_EINVAL, "a result shares memory with an operand");
    }
    return ZNN_OK;
}

}  // namespace znn
