// Dropout whose mask is a function of the element's index: nothing is stored, and the backward
// pass is the same call on the gradient.
//
// Element i is kept where 16-bit piece i mod 8 (a word's low half first) of the Philox-4x32-10 block
// (J. Salmon, M. Moraes, R. Dror, D. Shaw, Parallel random numbers: as easy as 1, 2, 3, SC 2011) with
// key `seed` and counter (i / 8, offset), each two words of 32 bits, is at least `least`. A block
// serves eight elements, what a lane loads at once.
//
// Bound by memory where there is enough of it: 8192 x 2048 bfloat16 with a residual 17.4 us (101 MB, 5.8
// TB/s), without 12.8 (67 MB, 5.2 TB/s: a block's 20 products of 32 x 32 bits stand beside 32 bytes).
// 64 x 512 takes 2.8 us, of 6.5 that the host needs for the call. Eight elements to a block: 16 bits
// count p in steps of 2^-16, where 32 would take twice the products.
#include "token_internal.h"

#include "token_device.h"

namespace gefen {
namespace {

__device__ __forceinline__ u32x4a philox(uint64_t block, uint64_t offset, uint64_t seed)
{
    uint32_t c0 = static_cast<uint32_t>(block), c1 = static_cast<uint32_t>(block >> 32);
    uint32_t c2 = static_cast<uint32_t>(offset), c3 = static_cast<uint32_t>(offset >> 32);
    uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u;
        const uint64_t b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
        c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
        c1 = static_cast<uint32_t>(b);
        c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
        c3 = static_cast<uint32_t>(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4a{c0, c1, c2, c3};
}

template <bool BF16, bool RESIDUAL>
__global__ __launch_bounds__(256) void k_dropout(const DropoutArgs a)
{
    uint64_t seed = a.seed, offset = a.offset;
    if (a.state) {
        seed = static_cast<uint64_t>(a.state[0]);
        offset += static_cast<uint64_t>(a.state[1]);
    }
    const int64_t blocks = (a.n + 7) / 8, n = by_lane(a.n);
    const int64_t step = int64_t(gridDim.x) * 256;
    for (int64_t b = int64_t(blockIdx.x) * 256 + threadIdx.x; b < blocks; b += step) {
        const int64_t e = 8 * b;
        float x[8], r[8];
        load_row8<BF16>(a.x, e, n, x);
        if constexpr (RESIDUAL) load_row8<BF16>(a.residual, e, n, r);
        const u32x4a w = philox(static_cast<uint64_t>(b), offset, seed);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t piece = (w[j >> 1] >> (16 * (j & 1))) & 0xffffu;
            const float v = piece >= a.least ? x[j] * a.scale : 0.0f;
            x[j] = RESIDUAL ? v + r[j] : v;
        }
        store_row8<BF16>(a.y, e, n, x);
    }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, bool bf16, hipStream_t stream)
{
    const int64_t groups = ((a.n + 7) / 8 + 255) / 256;
    if (groups == 0) return hipSuccess;
    const dim3 grid(static_cast<unsigned>(groups < (1 << 20) ? groups : (1 << 20)));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a); };
    if (bf16 && a.residual) go(k_dropout<true, true>);
    else if (bf16) go(k_dropout<true, false>);
    else if (a.residual) go(k_dropout<false, true>);
    else go(k_dropout<false, false>);
    return hipGetLastError();
}

}  // namespace gefen
