// One-pass sums of a softmax and its entropy, in base 2 and fp32.
#pragma once

#include <float.h>

#include "internal.h"

namespace a48f8 {

constexpr float LN2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {  // NaN if either is
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// With t = (x - r) c over the numbers x added: s = sum 2^t, d = sum 2^t t, against the reference r.  Differences come before
// the factor, so that numbers at the end of the range (masks of the lowest value) keep their order.  A NaN or +inf among
// the x makes s no number; -inf adds nothing.
struct Sums {
    float r, s, d;
    __device__ __forceinline__ void start(float largest) {
        r = fminf(fmaxf(largest, -FLT_MAX), FLT_MAX);
        s = d = 0.f;
    }
    __device__ __forceinline__ void add(float x, float c) { add(x, c, s); }
    // The same with the term of s to a sum that is added to s later.
    __device__ __forceinline__ void add(float x, float c, float& to) {
        const float t = max_nan((x - r) * c, -150.f);  // 2^t is 0 from there on, and 0 times -inf would be no number
        const float e = exp2_approx(t);
        to += e;
        d = fmaf(e, t, d);
    }
    __device__ __forceinline__ void move(float to, float c) {  // to another reference
        const float by = max_nan((r - to) * c, -150.f), f = exp2_approx(by);
        d = f * fmaf(s, by, d);
        s *= f;
        r = to;
    }
    __device__ __forceinline__ void join(Sums o, float c) {
        const float to = fmaxf(r, o.r);
        move(to, c);
        o.move(to, c);
        s += o.s;
        d += o.d;
    }
    __device__ __forceinline__ bool valid() const { return s > 0.f && s < INFINITY; }
    // ln of x's share, log_s = log2 s; halves, since numbers at both ends of the range are further apart than the largest one, which
    // a high temperature makes a number again.
    __device__ __forceinline__ float log_share(float x, float inv_t, float log_s) const { return fmaf(0.5f * x - 0.5f * r, 2.f * inv_t, -LN2 * log_s); }
};

}  // namespace a48f8
