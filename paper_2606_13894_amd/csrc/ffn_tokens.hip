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

namespace gefen {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Elements k .. k + 7 of a row of `n`; zero from n on.
__device__ __forceinline__ bf16x8 row_piece(const uint16_t* __restrict__ row, int k, int n)
{
    return __builtin_bit_cast(bf16x8, load_vector<2>(row, k, n));
}

template <bool DUAL, int R, int W>
__global__ __launch_bounds__(64 * W) void k_ffn_tokens(const FfnTokens g)
{
    constexpr int NM = DUAL ? 2 : 1;
    constexpr int D = R == 8 ? 64 : 32;      // k of a step
    __shared__ f32x4 sums[W][NM][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane >> 4, l16 = lane & 15;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * R;
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
    f32x4 acc[NM];
#pragma unroll
    for (int m = 0; m < NM; ++m) acc[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int U = W == 16 && DUAL ? 4 : 8;          // steps whose loads go out together
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
#pragma unroll
    for (int m = 0; m < NM; ++m) sums[wave][m][lane] = acc[m];
    __syncthreads();
    // Lane l holds elements n = 4 (l / 16) + 0..3 of token l % 16; with R = 8 the other half of
    // the sum of element n of token t is element 8 + n of token 8 + t, 40 lanes on.
    if (threadIdx.x >= 64 || token >= g.tokens || (R == 8 && (q >= 2 || l16 >= 8))) return;
    f32x4 v[NM];
#pragma unroll
    for (int m = 0; m < NM; ++m) {
        v[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int w = 0; w < W; ++w) {
            v[m] += sums[w][m][lane];
            if (R == 8) v[m] += sums[w][m][lane + 40];
        }
    }
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

}  // namespace

hipError_t launch_ffn_tokens(const FfnTokens& g, hipStream_t stream)
{
    if (g.tokens < 1 || g.tokens > kFfnFewTokens) return hipErrorInvalidValue;
    if (ffn_token_rows(g.tokens) == 8)
        return g.w[1] ? launch_waves<true, 8>(g, stream) : launch_waves<false, 8>(g, stream);
    return g.w[1] ? launch_waves<true, 16>(g, stream) : launch_waves<false, 16>(g, stream);
}

}  // namespace gefen
