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

// ---------------------------------------------------------------- sums of exponentials
// Over a set of scores z: m the largest, s the sum of exp(z - base), t that of (z - base) times it,
// with base = m; 0 where no score is above -inf, so that no difference of infinities is formed:
// each term is then 0. A NaN or an infinity among the scores makes s NaN (inf - inf), and keeps it
// so. In t the difference is held at -1e4, far below where exp is 0, so that -inf adds 0.
constexpr float kLog2E = 1.4426950408889634f;

__device__ __forceinline__ float score_base(float m) { return m == -INFINITY ? 0.0f : m; }

__device__ __forceinline__ void score_add(float z, float base, float& s, float& t)
{
    const float d = z - base;
    const float e = __builtin_amdgcn_exp2f(d * kLog2E);
    s += e;
    t = fmaf(e, fmaxf(d, -1e4f), t);
}

struct ScoreSum {
    float m, s, t;
};

// The same sums with a larger base.
__device__ __forceinline__ void score_rebase(float m, float base, float& s, float& t)
{
    const float d = fmaxf(m - base, -1e4f);   // also where nothing was summed yet
    const float e = __builtin_amdgcn_exp2f(d * kLog2E);
    t = e * fmaf(s, d, t);
    s *= e;
}

__device__ __forceinline__ ScoreSum score_join(ScoreSum a, ScoreSum b)
{
    ScoreSum r;
    r.m = fmaxf(a.m, b.m);
    const float base = score_base(r.m);
    score_rebase(a.m, base, a.s, a.t);
    score_rebase(b.m, base, b.s, b.t);
    r.s = a.s + b.s;
    r.t = a.t + b.t;
    return r;
}

// A row's results. `taken`: its token's score.
struct ScoreRow {
    float lse, entropy, logprob;
};
__device__ __forceinline__ ScoreRow score_row(const ScoreSum& a, int64_t token, int64_t vocab,
                                              float taken)
{
    ScoreRow r;
    if (a.s != a.s) {                       // NaN
        r.lse = r.entropy = r.logprob = a.s;
    } else if (a.m == -INFINITY) {          // nothing left in the row
        r.lse = r.logprob = -INFINITY;
        r.entropy = 0.0f;
    } else {
        const float l = logf(a.s);
        r.lse = a.m + l;
        r.entropy = fmaxf(l - a.t / a.s, 0.0f);
        r.logprob = (taken - a.m) - l;
    }
    if (token < 0) r.logprob = 0.0f;
    if (token >= vocab) r.logprob = __uint_as_float(0x7fc00000u);
    return r;
}

// ---------------------------------------------------------------- gradients of scores
//   dz_j = g ([j = token] - p_j) - h p_j (log p_j + H),  p_j = exp(z_j - lse)
// with g the gradient of the token's log probability and h that of the entropy H. A row with
// nothing left (lse -inf) has none.
struct ScoreGrad {
    float lse, entropy, g, h;
    int64_t token;
};
__device__ __forceinline__ ScoreGrad score_grad_row(const void* tokens, bool wide, int64_t row,
                                                    const float* lse, const float* entropy,
                                                    const float* dlogprob, const float* dentropy)
{
    ScoreGrad r;
    r.token = token_at(tokens, wide, row);
    r.lse = lse[row];
    r.entropy = entropy[row];
    r.g = r.token >= 0 ? dlogprob[row] : 0.0f;
    r.h = dentropy ? dentropy[row] : 0.0f;
    if (r.lse == -INFINITY) {
        r.lse = INFINITY;      // p = 0 throughout
        r.g = r.h = 0.0f;
    }
    return r;
}
__device__ __forceinline__ float score_gradient(float z, const ScoreGrad& r, bool taken)
{
    const float d = z - r.lse;
    const float p = __builtin_amdgcn_exp2f(d * kLog2E);
    const float dz = -p * fmaf(r.h, fmaxf(d, -1e4f) + r.entropy, r.g);
    return taken ? dz + r.g : dz;
}

}  // namespace gefen
