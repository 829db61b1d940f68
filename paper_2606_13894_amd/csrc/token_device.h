// Device helpers of the operators at a language model's two ends.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "act8_device.h"

namespace gefen {

__device__ __forceinline__ int64_t token_at(const void* tokens, bool wide, int64_t i)
{
    return wide ? static_cast<const int64_t*>(tokens)[i]
                : static_cast<int64_t>(static_cast<const int32_t*>(tokens)[i]);
}

// The number, which the compiler is to take as one that differs from lane to lane. A row's length is
// the same in all of them, and so are comparisons with it; but where such a comparison stands in
// a loop that lanes leave at different times, this compiler (ROCm 7.2) kept its outcome as a mask of
// the lanes that were still there, and used that mask after the loop for the lanes that had left:
// they took the path of rows shorter than a vector.
__device__ __forceinline__ int64_t by_lane(int64_t n)
{
    asm("" : "+v"(n));
    return n;
}
__device__ __forceinline__ int by_lane(int n)
{
    asm("" : "+v"(n));
    return n;
}

// ---------------------------------------------------------------- sums of exponentials
// Over a set of scores z with m the largest: s = sum 2^d and t = sum d 2^d, d = z log2 e - B, where
// the base B is m log2 e as rounded to float32. One multiply-add forms d from the exact product; that
// B is rounded does not matter, since whatever is made of s and t takes the same B.
// From |m| = 2^20 on d = (z - m) log2 e instead, whose base is m log2 e itself: below, B is off by 1/16 at
// most; with m it would grow until 2^d overflows, or is 0, for every score (from 2^31 on). Where no score
// is above -inf, B is 0: no difference of infinities is formed and each term is 0. In t, d is held at
// -1e4, far below where 2^d is 0, so that -inf adds 0. A NaN or +inf among the scores makes s NaN
// (inf - inf), and nothing that follows takes that away.
constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kScoreFar = 1048576.0f;               // 2^20
constexpr float kScoreLow = -8.507059173023462e37f;   // -2^126: above it z log2 e does not overflow

struct ScoreBase {
    float m, b;
    bool far;
};
__device__ __forceinline__ ScoreBase score_base(float m)
{
    ScoreBase r;
    r.m = m == -INFINITY ? 0.0f : m;
    r.b = r.m * kLog2E;
    r.far = fabsf(r.m) >= kScoreFar;
    return r;
}
__device__ __forceinline__ float score_far(float z, const ScoreBase& r)
{
    return r.far ? (z - r.m) * kLog2E : fmaf(z, kLog2E, -r.b);
}

// One score, whatever it and the base are.
__device__ __forceinline__ void score_add(float z, const ScoreBase& r, float& s, float& t)
{
    const float d = score_far(z, r);
    const float e = __builtin_amdgcn_exp2f(d);
    s += e;
    t = fmaf(e, fmaxf(d, -1e4f), t);
}
// One above kScoreLow, whose base is not far.
__device__ __forceinline__ void score_add_plain(float z, float b, float& s, float& t)
{
    const float d = fmaf(z, kLog2E, -b);
    const float e = __builtin_amdgcn_exp2f(d);
    s += e;
    t = fmaf(e, d, t);
}

struct ScoreSum {
    float m, s, t;
};

// The same sums from another, larger m.
__device__ __forceinline__ void score_rebase(float old, const ScoreBase& to, float& s, float& t)
{
    const ScoreBase from = score_base(old);
    float gap = from.b - to.b;              // of the bases themselves, whichever kind they are
    if (__any(from.far || to.far)) {
        if (from.far) gap = to.far ? (from.m - to.m) * kLog2E : fmaf(from.m, kLog2E, -to.b);
        else if (to.far) gap = -fmaf(to.m, kLog2E, -from.b);
    }
    const float d = old == -INFINITY ? -1e4f : fmaxf(gap, -1e4f);   // (nothing was summed yet)
    const float e = __builtin_amdgcn_exp2f(d);
    t = e * fmaf(s, d, t);
    s *= e;
}

__device__ __forceinline__ ScoreSum score_join(ScoreSum a, ScoreSum b)
{
    ScoreSum r;
    r.m = fmaxf(a.m, b.m);
    const ScoreBase base = score_base(r.m);
    score_rebase(a.m, base, a.s, a.t);
    score_rebase(b.m, base, b.s, b.t);
    r.s = a.s + b.s;
    r.t = a.t + b.t;
    return r;
}

// log p of a score from the row's sums and log2 s; lse = m + ln 2 (log2 s + (B - m log2 e)). Of a finite
// score far below m the product with log2 e overflows (m = 0: from -2.36e38 down, the type's lowest value
// among them), where log p itself does not.
__device__ __forceinline__ float score_logprob(float z, const ScoreBase& base, float log2s)
{
    const float d = score_far(z, base);
    if (d == -INFINITY && z > -INFINITY) return fmaf(-kLn2, log2s, z - base.m);
    return kLn2 * (d - log2s);
}

// A row's results. `taken`: its token's score; `rest`: what rounding left of lse.
struct ScoreRow {
    float lse, rest, entropy, logprob;
};
__device__ __forceinline__ ScoreRow score_row(const ScoreSum& a, int64_t token, int64_t vocab,
                                              float taken)
{
    ScoreRow r;
    r.rest = 0.0f;
    if (a.s != a.s) {                       // NaN
        r.lse = r.entropy = r.logprob = a.s;
    } else if (a.m == -INFINITY) {          // nothing left in the row
        r.lse = r.logprob = -INFINITY;
        r.entropy = 0.0f;
    } else {
        const ScoreBase base = score_base(a.m);
        const float l = log2f(a.s);
        const float over = base.far ? l : l - fmaf(a.m, kLog2E, -base.b);   // of m
        r.lse = fmaf(kLn2, over, a.m);
        const float x = kLn2 * over;
        r.rest = fabsf(a.m) >= fabsf(x) ? (a.m - r.lse) + x : (x - r.lse) + a.m;
        r.entropy = fmaxf(kLn2 * (l - a.t / a.s), 0.0f);
        r.logprob = score_logprob(taken, base, l);
    }
    if (token < 0) r.logprob = 0.0f;
    if (token >= vocab) r.logprob = __uint_as_float(0x7fc00000u);
    return r;
}

// ---------------------------------------------------------------- gradients of scores
//   dz_j = g ([j = token] - p_j) - h p_j (log p_j + H),  p_j = exp(z_j - lse)
// with g the gradient of the token's log probability and h that of the entropy H. A row with
// nothing left (lse -inf) has none. lse may be the sum of two numbers: that it is rounded to one moves p_j by
// |lse| 2^-24 of it, and of a row that a finite number far from 0 masks throughout leaves p_j = 1.
struct ScoreGrad {
    float lse, rest, entropy, g, h;
};
__device__ __forceinline__ ScoreGrad score_grad_row(int64_t token, int64_t vocab, int64_t row,
                                                    const float* lse, const float* rest,
                                                    const float* entropy, const float* dlogprob,
                                                    const float* dentropy)
{
    ScoreGrad r;
    r.lse = lse[row];
    r.rest = rest ? rest[row] : 0.0f;
    r.entropy = entropy[row];
    r.g = dlogprob[row];
    r.h = dentropy ? dentropy[row] : 0.0f;
    if (token < 0 || token >= vocab) r.g = 0.0f;
    if (r.lse == -INFINITY) {
        r.lse = INFINITY;      // p = 0 throughout
        r.rest = r.g = r.h = 0.0f;
    }
    return r;
}
__device__ __forceinline__ float score_gradient(float z, const ScoreGrad& r, bool taken)
{
    const float d = (z - r.lse) - r.rest;
    const float p = __builtin_amdgcn_exp2f(d * kLog2E);
    const float dz = -p * fmaf(r.h, fmaxf(d, -1e4f) + r.entropy, r.g);
    return taken ? dz + r.g : dz;
}

}  // namespace gefen
