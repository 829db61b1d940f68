// The gated feed-forward block's forward products for a few tokens (serving): bound by the
// weights, which are read once, straight into the matrix cores' registers.
//
// A workgroup takes R rows of a weight matrix (of both, for gate and up) and its waves share the
// sum over k. R = 16: a matrix-core op takes 16 rows x 32 k of weights and up to 16 tokens.
// R = 8, for up to 8 tokens: 8 rows x 64 k, the second 32 k as eight more rows against eight more
// columns of the same tokens, whose other halves are not used: a row's cache line is loaded whole
// by one instruction, and twice as many workgroups share the matrix. Rows need no alignment and k
// no multiple: a lane's 16 bytes are loaded at any address, the row's last whole
// vector shifted at its end. The waves' float32 sums are added through LDS, in order.
//
// One token, 2048 to 8192 columns and back, on weights that change from call to call (2.4 GB of
// them): gate/up 14.3 us (67 MB, 4.7 TB/s), down 8.3 (34 MB, 4.0), 22.5 a call; on the same ones
// again, which the last-level cache holds, 12.6 and 7.8, 20.0 a call. Weight loads that bypass the
// caches were 2 % faster on cold weights and 20 % slower where a small model's weights stay in the
// caches, so they are plain. A is rounded to bfloat16 as in ffn_gemm.hip.
#include "act8_device.h"
#include "ffn_internal.h"
#include "token_device.h"

namespace gefen {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Elements k .. k + 7 of a row of `n`; zero from n on.
__device__ __forceinline__ bf16x8 row_piece(const uint16_t* __restrict__ row, int k, int n)
{
    return __builtin_bit_cast(bf16x8, load_vector<2>(row, k, n));
}

// The wave's share of the sums of R rows of the weights from n0 on.
template <int NM, int R, int W>
__device__ __forceinline__ void sum_rows(const FfnTokens& g, int64_t n0, int wave, int lane,
                                         f32x4 (&acc)[NM])
{
    constexpr int D = R == 8 ? 64 : 32;      // k of a step
    const int q = lane >> 4, l16 = lane & 15;
    const int K = static_cast<int>(g.K);
    const int64_t row = min(n0 + l16 % R, g.N - 1);     // what is summed past N is not stored
    const int token = l16 % R, k0 = (R == 8 ? 4 * (l16 & 8) : 0) + 8 * q;
    const uint16_t* wp[NM];
#pragma unroll
    for (int m = 0; m < NM; ++m) wp[m] = g.w[m] + row * g.K;
    const int xn = token < g.tokens ? K : 0;            // 0: no such token
    const uint16_t* xp = g.x + (xn ? token : 0) * g.ldx;
    const int steps = (K + D - 1) / D;
    const int from = static_cast<int>(int64_t(steps) * wave / W);
    const int to = static_cast<int>(int64_t(steps) * (wave + 1) / W);
#pragma unroll
    for (int m = 0; m < NM; ++m) acc[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int U = W == 16 && NM == 2 ? 4 : 8;       // steps whose loads go out together
    for (int s = from; s < to; s += U) {
        bf16x8 wv[U][NM], xv[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int k = D * (s + i) + k0;
            const bool on = s + i < to;                 // past the wave's steps: zeros
#pragma unroll
            for (int m = 0; m < NM; ++m) wv[i][m] = row_piece(wp[m], k, on ? K : 0);
            xv[i] = row_piece(xp, k, on ? xn : 0);
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int m = 0; m < NM; ++m)
                acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[i][m], xv[i], acc[m], 0, 0, 0);
    }
}

// Lane l of the waves' sums holds elements n = 4 (l / 16) + 0..3 of token l % 16; with R = 8 the other
// half of the sum of element n of token t is element 8 + n of token 8 + t, 40 lanes on.
template <int R>
__device__ __forceinline__ bool holds_sums(const FfnTokens& g, int lane)
{
    return (lane & 15) % R < g.tokens && !(R == 8 && (lane >= 32 || (lane & 8)));
}
template <int R, int W, int NM>
__device__ __forceinline__ f32x4 all_waves(const f32x4 (&sums)[W][NM][64], int m, int lane)
{
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int w = 0; w < W; ++w) {
        v += sums[w][m][lane];
        if (R == 8) v += sums[w][m][(lane + 40) & 63];
    }
    return v;
}

template <bool DUAL, int R, int W>
__global__ __launch_bounds__(64 * W) void k_ffn_tokens(const FfnTokens g)
{
    constexpr int NM = DUAL ? 2 : 1;
    __shared__ f32x4 sums[W][NM][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane >> 4, token = (lane & 15) % R;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * R;
    f32x4 acc[NM];
    sum_rows<NM, R, W>(g, n0, wave, lane, acc);
#pragma unroll
    for (int m = 0; m < NM; ++m) sums[wave][m][lane] = acc[m];
    __syncthreads();
    if (threadIdx.x >= 64 || !holds_sums<R>(g, lane)) return;
    f32x4 v[NM];
#pragma unroll
    for (int m = 0; m < NM; ++m) v[m] = all_waves<R, W, NM>(sums, m, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float r = v[0][i];
        if constexpr (DUAL) {
            float z = r;
            if (g.act == kActGelu) z = 1.5957691216057308f * r * fmaf(0.044715f, r * r, 1.0f);
            r = r * __builtin_amdgcn_rcpf(1.0f + __expf(-z)) * v[NM - 1][i];
        }
        const int64_t n = n0 + 4 * q + i;
        if (n < g.N) g.o[token * g.ldo + n] = bf16_bits(r);
    }
}

// The output head's scores of a few tokens: each token's statistics over the workgroup's R rows of the
// weight (ffn_internal.h), [token][3][workgroup]. One token, 128256 x 2048: 83 us (525 MB, 6.3 TB/s),
// and 7.8 for the join of 16032 workgroups' statistics, which one workgroup reads at the rate of its CU
// alone. More rows to a workgroup leave less to join and cost more: three times R one after the other
// 90 us, two or four groups of waves with R each 98 and 110.
//
// Short rows: G groups of R, of W = 1 wave each, which has no one to wait for, and one slot for them all.
// Four waves to R rows are bound by the dispatch of so many workgroups there (16032 take 47 us): one token,
// 128256 x 256 23 us in all, and 47 so; 200000 x 768 58 (5.4 TB/s) and 74.
template <int R, int W, int G>
__global__ __launch_bounds__(64 * W * G) void k_head_tokens(const FfnTokens g)
{
    static_assert(W == 1 || G == 1, "groups are of one wave");
    __shared__ f32x4 sums[G][W][1][64];
    __shared__ ScoreSum stats[G][R];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = G > 1 ? wave : 0, in = G > 1 ? 0 : wave;
    const int q = lane >> 4, token = (lane & 15) % R;
    const int64_t n0 = (static_cast<int64_t>(blockIdx.x) * G + group) * R;
    f32x4 acc[1];
    sum_rows<1, R, W>(g, n0, in, lane, acc);
    sums[group][in][0][lane] = acc[0];
    __syncthreads();
    if (in == 0) {
        const bool on = holds_sums<R>(g, lane);
        const f32x4 v = all_waves<R, W, 1>(sums[group], 0, lane);
        float z[4], m = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            z[i] = on && n0 + 4 * q + i < g.N ? v[i] : -INFINITY;
            m = fmaxf(m, z[i]);
        }
        // a token's four lanes (two, with R = 8) join; the others hold -inf
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const ScoreBase base = score_base(m);
        float s = 0.0f, t = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) score_add(z[i], base, s, t);
        s += __shfl_xor(s, 16);
        t += __shfl_xor(t, 16);
        s += __shfl_xor(s, 32);
        t += __shfl_xor(t, 32);
        if (on && q == 0) stats[group][token] = ScoreSum{m, s, t};
        const int64_t at = token_at(g.head.tokens, g.head.wide, on ? token : 0) - n0 - 4 * q;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (on && at == i && n0 + 4 * q + i < g.N) g.head.taken[token] = v[i];
    }
    if (G > 1) __syncthreads();
    if (threadIdx.x >= g.tokens) return;
    ScoreSum c = stats[0][threadIdx.x];
#pragma unroll
    for (int i = 1; i < G; ++i) c = score_join(c, stats[i][threadIdx.x]);
    float* __restrict__ o = g.head.stats + (int64_t(threadIdx.x) * 3 * gridDim.x + blockIdx.x);
    o[0] = c.m;
    o[gridDim.x] = c.s;
    o[2 * int64_t(gridDim.x)] = c.t;
}

template <bool DUAL, int R>
hipError_t launch_waves(const FfnTokens& g, hipStream_t stream)
{
    const int waves = ffn_token_waves(g.N, g.K, R);
    const dim3 grid(static_cast<unsigned>(ffn_ceil(g.N, R)));
    if (waves == 4)
        hipLaunchKernelGGL((k_ffn_tokens<DUAL, R, 4>), grid, dim3(256), 0, stream, g);
    else if (waves == 8)
        hipLaunchKernelGGL((k_ffn_tokens<DUAL, R, 8>), grid, dim3(512), 0, stream, g);
    else
        hipLaunchKernelGGL((k_ffn_tokens<DUAL, R, 16>), grid, dim3(1024), 0, stream, g);
    return hipGetLastError();
}

template <int R>
hipError_t launch_head(const FfnTokens& g, int groups, hipStream_t stream)
{
    const int waves = ffn_token_waves(g.N, g.K, R);
    const dim3 grid(static_cast<unsigned>(ffn_ceil(g.N, R * groups)));
    if (groups == 4)
        hipLaunchKernelGGL((k_head_tokens<R, 1, 4>), grid, dim3(256), 0, stream, g);
    else if (groups != 1)
        return hipErrorInvalidValue;
    else if (waves == 4)
        hipLaunchKernelGGL((k_head_tokens<R, 4, 1>), grid, dim3(256), 0, stream, g);
    else if (waves == 8)
        hipLaunchKernelGGL((k_head_tokens<R, 8, 1>), grid, dim3(512), 0, stream, g);
    else
        hipLaunchKernelGGL((k_head_tokens<R, 16, 1>), grid, dim3(1024), 0, stream, g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_ffn_tokens(const FfnTokens& g, hipStream_t stream)
{
    if (g.tokens < 1 || g.tokens > kFfnFewTokens) return hipErrorInvalidValue;
    if (ffn_token_rows(g.tokens) == 8)
        return g.w[1] ? launch_waves<true, 8>(g, stream) : launch_waves<false, 8>(g, stream);
    return g.w[1] ? launch_waves<true, 16>(g, stream) : launch_waves<false, 16>(g, stream);
}

hipError_t launch_head_tokens(const FfnTokens& g, int groups, hipStream_t stream)
{
    if (g.tokens < 1 || g.tokens > kFfnFewTokens) return hipErrorInvalidValue;
    return ffn_token_rows(g.tokens) == 8 ? launch_head<8>(g, groups, stream)
                                         : launch_head<16>(g, groups, stream);
}

}  // namespace gefen
