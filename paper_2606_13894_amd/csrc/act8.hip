// 8-bit activation checkpoints, and the RMS norm that writes and reads them.
//
// All of these are bound by memory: every element is read once and written once, in vectors of
// eight (16 bytes of bfloat16) per lane. A checkpoint's group of 64 is eight neighbouring lanes'
// vectors, so its scale is three lane exchanges away and nothing is read twice.
#include "act8_device.h"
#include "ffn_internal.h"

#include <algorithm>

namespace gefen {
namespace {

// ---------------------------------------------------------------- encode and decode
// A workgroup takes 256 vectors: 2^lx lanes along a row (a whole number of groups) by
// 256 >> lx rows, from the workgroup `first` along a row on (RowGrid). Rows that are whole groups
// long are one long row to these kernels.
// 8192 x 8192 bfloat16: encode 39.8 us, decode 38.2 (5.1 and 5.3 TB/s, a large copy's rate); 8192 x
// 2048 decode 11.8 (4.3 TB/s); one row of 2048 1.9 and 1.7, a launch's time.
template <bool BF16>
__global__ __launch_bounds__(256) void k_act8_encode(const void* __restrict__ x, int64_t rows,
                                                     int64_t cols, int64_t groups, int lx,
                                                     int64_t first, int8_t* __restrict__ codes,
                                                     uint8_t* __restrict__ exps)
{
    const int64_t e = (((first + blockIdx.x) << lx) + (threadIdx.x & ((1 << lx) - 1))) * 8;
    const int64_t step = static_cast<int64_t>(gridDim.y) << (8 - lx);
    for (int64_t r = (static_cast<int64_t>(blockIdx.y) << (8 - lx)) + (threadIdx.x >> lx);
         r < rows; r += step) {
        float v[8];
        const int64_t at = r * cols;
        load_row8<BF16>(static_cast<const char*>(x) + at * (BF16 ? 2 : 4), e, cols, v);
        act8_write_group(v, e, cols, codes + at, exps + r * groups);
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void k_act8_decode(const int8_t* __restrict__ codes,
                                                     const uint8_t* __restrict__ exps,
                                                     const float* __restrict__ gain, int64_t rows,
                                                     int64_t cols, int64_t groups, int lx,
                                                     int64_t first, void* __restrict__ out,
                                                     int64_t ldo)
{
    const int64_t e = (((first + blockIdx.x) << lx) + (threadIdx.x & ((1 << lx) - 1))) * 8;
    const int64_t step = static_cast<int64_t>(gridDim.y) << (8 - lx);
    float g[8];
    if (gain) load_row8<false>(gain, e, cols, g);
    for (int64_t r = (static_cast<int64_t>(blockIdx.y) << (8 - lx)) + (threadIdx.x >> lx);
         r < rows; r += step) {
        float v[8];
        act8_read8(codes + r * cols, exps + r * groups, e, cols, v);
        if (gain) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= g[j];
        }
        store_row8<BF16>(static_cast<char*>(out) + r * ldo * (BF16 ? 2 : 4), e, ldo, v);
    }
}

// launch(grid, first workgroup along a row), until all of them have had their launch.
template <typename Launch>
hipError_t launch_along(const RowGrid& g, const Launch& launch)
{
    for (int64_t first = 0; first < g.gx; first += g.most) {
        launch(dim3(static_cast<unsigned>(std::min(g.most, g.gx - first)),
                    static_cast<unsigned>(g.gy)), first);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

// ---------------------------------------------------------------- RMS norm
// A row is held in the registers of TPR lanes (a wave, or a whole workgroup), NV vectors each:
// one pass over memory. Workgroups take several rows, so that the weight is read once.
constexpr int kNormThreads(int tpr) { return tpr < 256 ? 256 : tpr; }

// The sum over the row's lanes, in every lane. All threads of the workgroup call it.
template <int TPR, typename F>
__device__ __forceinline__ F row_sum(F s, F* red)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    if constexpr (TPR > 64) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();   // the last row's sum has been read
        if ((threadIdx.x & 63) == 0) red[wave] = s;
        __syncthreads();
        s = red[0];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) s += red[w];
    }
    return s;
}

// x^(-1/2): the float32 one with a Newton step in 64 bits. A mean square past float32's range
// either way goes through the 64-bit functions.
__device__ __forceinline__ double inverse_root(double x)
{
    const float f = static_cast<float>(x);
    if (!(f > 1e-36f && f < 1e36f)) return 1.0 / sqrt(x);
    const double r = static_cast<double>(__builtin_amdgcn_rsqf(f));
    return r * fma(-0.5 * x * r, r, 1.5);
}

// The sum of squares and rstd are in 64 bits, and so are the products that the codes are rounded
// from: a checkpoint's code is the formula's, whatever the order of the sum (the pass is bound by
// memory: no time is lost). A row's vectors are all fetched before the first is used; 4096
// workgroups at most, so that a row's wait is covered by other workgroups'. 8192 x 2048 bfloat16
// with a residual and a checkpoint: 26.2 us (5.8 TB/s); 1000 x 1601 float32 6.6. Rows of 4096
// run at 5.4 TB/s, of 8192 to 16384 at 4.2 (past 8192 with 20 bytes a lane through scratch, 44 in
// float32).
template <bool BF16, int TPR, int NV>
__global__ __launch_bounds__(kNormThreads(TPR)) void k_rms_norm(const NormArgs a, int64_t groups)
{
    constexpr int kRows = kNormThreads(TPR) / TPR;
    constexpr int kSize = BF16 ? 2 : 4;
    __shared__ double red[TPR / 64];
    const int lane = threadIdx.x & (TPR - 1);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
    const int cols = static_cast<int>(a.cols);
    const double inv_n = 1.0 / static_cast<double>(cols);
    constexpr bool kHold = TPR * NV < 2048;   // the widest rows read the weight again each time
    float w[NV][8];
    if constexpr (kHold) {
#pragma unroll
        for (int i = 0; i < NV; ++i) load_row8<false>(a.weight, (i * TPR + lane) * 8, cols, w[i]);
    }
    // rows advance together in a workgroup: every thread takes part in the row's sum
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kRows; base < a.rows; base += step) {
        const int64_t row = base + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
        const bool on = row < a.rows;
        const int n = on ? cols : 0;
        const int64_t at = on ? row * cols : 0;
        float v[NV][8];
        double s = 0.0;
        {
            u32x4a x[NV][BF16 ? 1 : 2], r[NV][BF16 ? 1 : 2];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int e = (i * TPR + lane) * 8;
                fetch8<BF16>(static_cast<const char*>(a.x) + at * kSize, e, n, x[i]);
                if (a.r) fetch8<BF16>(static_cast<const char*>(a.r) + at * kSize, e, n, r[i]);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int e = (i * TPR + lane) * 8;
                settle8<BF16>(x[i], e, n, v[i]);
                if (a.r) {
                    float q[8];
                    settle8<BF16>(r[i], e, n, q);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[i][j] += q[j];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                s = fma(static_cast<double>(v[i][j]), static_cast<double>(v[i][j]), s);
        s = row_sum<TPR>(s, red);
        const double rstd = inverse_root(fma(s, inv_n, a.eps));
        const float rf = static_cast<float>(rstd);
        if (!on) continue;
        if (lane == 0) a.rstd[row] = rf;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * TPR + lane) * 8;
            if (a.h) store_row8<BF16>(static_cast<char*>(a.h) + at * kSize, e, n, v[i]);
            if constexpr (!kHold) load_row8<false>(a.weight, e, cols, w[i]);
            float f[8], y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f[j] = static_cast<float>(static_cast<double>(v[i][j]) * rstd);
                y[j] = f[j] * w[i][j];
            }
            store_row8<BF16>(static_cast<char*>(a.y) + at * kSize, e, n, y);
            if (a.codes)
                act8_write_products(v[i], rstd, f, e, n, a.codes + at, a.exps + row * groups);
        }
    }
}

// A row's vectors as they were loaded.
template <bool BF16, bool CODES, int NV>
struct GradRow {
    u32x4a dy[NV][BF16 ? 1 : 2], dh[NV][BF16 ? 1 : 2], h[NV][BF16 ? 1 : 2];   // h: codes in one half
    uint32_t ex[NV];
    float rstd;
};

// The compiler no longer knows what a row's vectors hold.
template <bool BF16, bool CODES, int NV>
__device__ __forceinline__ void hide(GradRow<BF16, CODES, NV>& r)
{
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int b = 0; b < (BF16 ? 1 : 2); ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t p = r.dy[i][b][j], q = r.h[i][b][j];
                asm volatile("" : "+v"(p), "+v"(q));
                r.dy[i][b][j] = p;
                r.h[i][b][j] = q;
            }
}

// dn = dy w;  dx = rstd (dn - n mean(dn n)) + dh;  dw = the sum over rows of dy n. A workgroup
// keeps its rows' share of dw in registers and writes it once; k_norm_dw adds the shares in
// order, so that dw does not depend on timing. The next row's vectors are on their way while a
// row is worked on, so few workgroups are enough (768: three to a CU) and the shares stay small.
// Bound by memory: 8192 x 2048 bfloat16 from codes 23.5 us (5.0 TB/s) and 4.0 for k_norm_dw;
// 1023 x 768 float32 5.6 and 3.5, launches. Rows of 4096 and 8192 run at 4.4 TB/s, of 16384 at
// 3.1 (2.8 in float32; 2.0 before their values were formed twice): a 1024-thread workgroup has 128
// registers to a lane, which hold one row as it was loaded and dw, and 12 to 172 bytes of a lane
// go through scratch all the same.
template <bool BF16, bool CODES, int TPR, int NV>
__global__ __launch_bounds__(kNormThreads(TPR)) void k_rms_norm_grad(const NormGradArgs a,
                                                                     int64_t groups)
{
    constexpr int kRows = kNormThreads(TPR) / TPR;
    constexpr int kSize = BF16 ? 2 : 4;
    __shared__ float red[TPR / 64];
    __shared__ float share[kRows > 1 ? kRows - 1 : 1][kRows > 1 ? TPR * NV * 8 : 1];
    const int lane = threadIdx.x & (TPR - 1);
    const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
    const int cols = static_cast<int>(a.cols);
    const float inv_n = 1.0f / static_cast<float>(cols);
    constexpr bool kHold = TPR * NV < 2048;   // the widest rows: one to a workgroup
    float w[NV][8], dw[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if constexpr (kHold) load_row8<false>(a.weight, (i * TPR + lane) * 8, cols, w[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = 0.0f;
    }
    typedef GradRow<BF16, CODES, NV> Row;
    auto fetch = [&](int64_t base, Row& r) {
        const int64_t row = base + sub;
        const bool on = row < a.rows;
        const int n = on ? cols : 0;
        const int64_t at = on ? row * cols : 0;
        r.rstd = on ? a.rstd[row] : 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * TPR + lane) * 8;
            fetch8<BF16>(static_cast<const char*>(a.dy) + at * kSize, e, n, r.dy[i]);
            if constexpr (CODES) {
                r.ex[i] = e < n ? a.exps[(on ? row : 0) * groups + (e >> 6)] : 0u;
                const u32x2a c = fetch_codes8(a.codes + at, e, n);
                r.h[i][0] = u32x4a{c.x, c.y, 0u, 0u};
            } else {
                fetch8<BF16>(static_cast<const char*>(a.h) + at * kSize, e, n, r.h[i]);
            }
            if (kHold && a.dh)   // else when dx is formed
                fetch8<BF16>(static_cast<const char*>(a.dh) + at * kSize, e, n, r.dh[i]);
        }
    };
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kRows;
    Row next;
    if (kHold && first < a.rows) fetch(first, next);
    for (int64_t base = first; base < a.rows; base += step) {
        // the widest rows' registers do not hold two rows: the row is fetched here, and what is
        // formed of it is formed again after its sum
        if constexpr (!kHold) fetch(base, next);
        Row r = next;
        if (kHold && base + step < a.rows) fetch(base + step, next);
        const int64_t row = base + sub;
        const bool on = row < a.rows;
        float d[NV][8], v[NV][8];
        float s = 0.0f;
        auto values = [&](int i) {   // d = dy and v = n of the row's vector i
            const int e = (i * TPR + lane) * 8, n = on ? cols : 0;
            settle8<BF16>(r.dy[i], e, n, d[i]);
            if constexpr (CODES) {
                const float scale = act8_scale(r.ex[i]);
                const u32x2a c = settle_codes8(u32x2a{r.h[i][0].x, r.h[i][0].y}, e, n);
#pragma unroll
                for (int j = 0; j < 8; ++j)   // a NaN group's scale is not to reach past the row
                    v[i][j] = e + j < n ? act8_value(c[j >> 2], j & 3) * scale : 0.0f;
            } else {
                settle8<BF16>(r.h[i], e, n, v[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] *= r.rstd;
            }
            if constexpr (!kHold) load_row8<false>(a.weight, e, cols, w[i]);
        };
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            values(i);
            if constexpr (!kHold) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dw[i][j] = fmaf(d[i][j], v[i][j], dw[i][j]);
                d[i][j] *= w[i][j];
                s = fmaf(d[i][j], v[i][j], s);
            }
        }
        s = row_sum<TPR>(s, red);
        if constexpr (!kHold) hide(r);   // so that the values are formed again, not kept
        if (!on) continue;
        const float c = s * inv_n;
        const int64_t at = row * cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * TPR + lane) * 8;
            if constexpr (!kHold) {
                __builtin_amdgcn_sched_barrier(0);
                values(i);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[i][j] *= w[i][j];
            }
            float g[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
            if (!kHold && a.dh)   // dx may be dh: of a shifted vector only the lane's own count
                fetch8<BF16>(static_cast<const char*>(a.dh) + at * kSize, e, cols, r.dh[i]);
            if (a.dh) settle8<BF16>(r.dh[i], e, cols, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = fmaf(r.rstd, fmaf(-v[i][j], c, d[i][j]), g[j]);
            store_row8<BF16>(static_cast<char*>(a.dx) + at * kSize, e, cols, g);
        }
    }
    if constexpr (kRows > 1) {
        __syncthreads();
        if (sub > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) share[sub - 1][(j * NV + i) * TPR + lane] = dw[i][j];
        }
        __syncthreads();
        if (sub > 0) return;
#pragma unroll
        for (int q = 0; q < kRows - 1; ++q)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) dw[i][j] += share[q][(j * NV + i) * TPR + lane];
    }
    float* __restrict__ out = a.partial + static_cast<int64_t>(blockIdx.x) * a.cols;
#pragma unroll
    for (int i = 0; i < NV; ++i) store_row8<false>(out, (i * TPR + lane) * 8, cols, dw[i]);
}

// dw[c] = the sum over p of partial[p][c]: a workgroup takes 16 columns, 64 threads each, so that
// a thread's few loads are all in flight at once; the threads' sums are added in order. 768 shares
// of 2048 columns (6.3 MB, from the L2 and the last-level cache): 4.0 us.
__global__ __launch_bounds__(1024) void k_norm_dw(const float* __restrict__ partial, int64_t parts,
                                                  int64_t cols, float* __restrict__ dw)
{
    __shared__ float t[64][17];
    const int col = threadIdx.x & 15, slot = threadIdx.x >> 4;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 16 + col;
    float s = 0.0f;
    if (c < cols) {
#pragma unroll 8
        for (int64_t p = slot; p < parts; p += 64) s += partial[p * cols + c];
    }
    t[slot][col] = s;
    __syncthreads();
    if (threadIdx.x >= 256) return;
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) s += t[slot * 4 + k][col];
    // sixteen slots are left, lanes 16 apart in four waves
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    __shared__ float u[4][16];
    if ((threadIdx.x & 63) < 16) u[threadIdx.x >> 6][col] = s;
    __syncthreads();
    if (threadIdx.x < 16 && c < cols) dw[c] = (u[0][col] + u[1][col]) + (u[2][col] + u[3][col]);
}

__global__ __launch_bounds__(256) void k_fill_zero(float* __restrict__ p, int64_t n)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i < n) p[i] = 0.0f;
}

int64_t norm_rows_per_group(int64_t cols) { return cols <= 1024 ? 4 : 1; }

}  // namespace

hipError_t launch_act8_encode(const void* x, bool bf16, int64_t rows, int64_t cols, int8_t* codes,
                              uint8_t* exps, hipStream_t stream)
{
    if (rows <= 0 || cols <= 0) return hipSuccess;
    if (cols % kAct8Group == 0) {
        cols *= rows;
        rows = 1;
    }
    const int64_t groups = act8_groups(cols);
    const RowGrid g = row_grid(rows, groups * 8);
    return launch_along(g, [&](dim3 grid, int64_t first) {
        if (bf16)
            hipLaunchKernelGGL(k_act8_encode<true>, grid, dim3(256), 0, stream, x, rows, cols,
                               groups, g.lx, first, codes, exps);
        else
            hipLaunchKernelGGL(k_act8_encode<false>, grid, dim3(256), 0, stream, x, rows, cols,
                               groups, g.lx, first, codes, exps);
    });
}

hipError_t launch_act8_decode(const int8_t* codes, const uint8_t* exps, const float* gain,
                              int64_t rows, int64_t cols, void* out, bool bf16, int64_t ldo,
                              hipStream_t stream)
{
    if (rows <= 0 || cols <= 0) return hipSuccess;
    if (ldo < cols || ldo >= cols + kAct8Group) return hipErrorInvalidValue;
    if (cols % kAct8Group == 0 && ldo == cols && !gain) {
        cols *= rows;
        ldo = cols;
        rows = 1;
    }
    const int64_t groups = act8_groups(cols);
    const RowGrid g = row_grid(rows, groups * 8);
    return launch_along(g, [&](dim3 grid, int64_t first) {
        if (bf16)
            hipLaunchKernelGGL(k_act8_decode<true>, grid, dim3(256), 0, stream, codes, exps, gain,
                               rows, cols, groups, g.lx, first, out, ldo);
        else
            hipLaunchKernelGGL(k_act8_decode<false>, grid, dim3(256), 0, stream, codes, exps, gain,
                               rows, cols, groups, g.lx, first, out, ldo);
    });
}

// The kernel for a row width: a wave per row while the row fits its registers, else a workgroup.
#define GEFEN_NORM_WIDTHS(LAUNCH, T8, N8)                                                  \
    do {                                                                                   \
        if (cols <= 512) LAUNCH(64, 1);                                                    \
        else if (cols <= 1024) LAUNCH(64, 2);                                              \
        else if (cols <= 2048) LAUNCH(256, 1);                                             \
        else if (cols <= 4096) LAUNCH(256, 2);                                             \
        else if (cols <= 8192) LAUNCH(T8, N8);                                             \
        else LAUNCH(1024, 2);                                                              \
    } while (0)

hipError_t launch_rms_norm(const NormArgs& a, bool bf16, hipStream_t stream)
{
    const int64_t cols = a.cols;
    if (cols < 1 || cols > kNormMaxCols) return hipErrorInvalidValue;
    if (a.rows <= 0) return hipSuccess;
    const int64_t per = norm_rows_per_group(cols);
    const int64_t blocks = std::min<int64_t>((a.rows + per - 1) / per, 4096);
    const int64_t groups = act8_groups(cols);
    const dim3 grid(static_cast<unsigned>(blocks));
#define LAUNCH(TPR, NV)                                                                    \
    do {                                                                                   \
        if (bf16)                                                                          \
            hipLaunchKernelGGL((k_rms_norm<true, TPR, NV>), grid, dim3(kNormThreads(TPR)), \
                               0, stream, a, groups);                                      \
        else                                                                               \
            hipLaunchKernelGGL((k_rms_norm<false, TPR, NV>), grid,                         \
                               dim3(kNormThreads(TPR)), 0, stream, a, groups);             \
    } while (0)
    GEFEN_NORM_WIDTHS(LAUNCH, 1024, 1);
#undef LAUNCH
    return hipGetLastError();
}

int64_t norm_grad_parts(int64_t rows, int64_t cols)
{
    const int64_t per = norm_rows_per_group(cols);
    return std::min<int64_t>((rows + per - 1) / per, 768);
}

hipError_t launch_rms_norm_grad(const NormGradArgs& a, bool bf16, hipStream_t stream)
{
    const int64_t cols = a.cols;
    if (cols < 1 || cols > kNormMaxCols) return hipErrorInvalidValue;
    const dim3 dw_grid(static_cast<unsigned>((cols + 15) / 16));
    if (a.rows <= 0) {
        hipLaunchKernelGGL(k_fill_zero, dim3(static_cast<unsigned>((cols + 255) / 256)), dim3(256),
                           0, stream, a.dw, cols);
        return hipGetLastError();
    }
    const int64_t parts = norm_grad_parts(a.rows, cols);
    const int64_t groups = act8_groups(cols);
    const dim3 grid(static_cast<unsigned>(parts));
#define LAUNCH_AS(BF, CODES, TPR, NV)                                                       \
    hipLaunchKernelGGL((k_rms_norm_grad<BF, CODES, TPR, NV>), grid, dim3(kNormThreads(TPR)), 0, \
                       stream, a, groups)
#define LAUNCH(TPR, NV)                                                                    \
    do {                                                                                   \
        if (bf16 && a.codes) LAUNCH_AS(true, true, TPR, NV);                               \
        else if (bf16) LAUNCH_AS(true, false, TPR, NV);                                    \
        else if (a.codes) LAUNCH_AS(false, true, TPR, NV);                                 \
        else LAUNCH_AS(false, false, TPR, NV);                                             \
    } while (0)
    GEFEN_NORM_WIDTHS(LAUNCH, 512, 2);
#undef LAUNCH
#undef LAUNCH_AS
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(k_norm_dw, dw_grid, dim3(1024), 0, stream, a.partial, parts, cols, a.dw);
    return hipGetLastError();
}

}  // namespace gefen
