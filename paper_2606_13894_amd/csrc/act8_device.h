// Device helpers of the feed-forward operators: eight-element vectors of a row at any alignment,
// and the 8-bit checkpoint code (ffn_internal.h defines it).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "ffn_internal.h"

namespace gefen {

typedef float f32x2a __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2a __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4a __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2a __attribute__((ext_vector_type(2)));

// 16, 8 bytes from or to any address (a global access of that width at any alignment).
__device__ __forceinline__ u32x4a load16(const void* p)
{
    u32x4a v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
__device__ __forceinline__ u32x2a load8b(const void* p)
{
    u32x2a v;
    __builtin_memcpy(&v, p, 8);
    return v;
}
__device__ __forceinline__ void store16(void* p, const u32x4a& v) { __builtin_memcpy(p, &v, 16); }
__device__ __forceinline__ void store8b(void* p, const u32x2a& v) { __builtin_memcpy(p, &v, 8); }

__device__ __forceinline__ float bf16_float(uint32_t b) { return __uint_as_float(b << 16); }

// Two float32 to bfloat16, rounded to nearest even (NaN stays NaN), low half first.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    const f32x2a x = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2a));
}
__device__ __forceinline__ uint16_t bf16_bits(float x)
{
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}

// At a row's end the last whole vector of the row is loaded instead and shifted down, so that
// every vector is one load (element by element, each waiting for the one before, the 15 last
// codes of a row took 10 us). w >> bits, zeros from above; bits from 128 on give 0.
__device__ __forceinline__ u32x4a shift_down(const u32x4a& w, uint32_t bits)
{
    uint64_t lo = w[0] | (static_cast<uint64_t>(w[1]) << 32);
    uint64_t hi = w[2] | (static_cast<uint64_t>(w[3]) << 32);
    if (bits >= 64) {
        lo = bits >= 128 ? 0 : hi >> (bits - 64);
        hi = 0;
    } else if (bits > 0) {
        lo = (lo >> bits) | (hi << (64 - bits));
        hi >>= bits;
    }
    return u32x4a{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32),
                  static_cast<uint32_t>(hi), static_cast<uint32_t>(hi >> 32)};
}

// The 16 bytes of elements of SIZE bytes from element e of a row of n on; zero from n on. (e is a
// multiple of their number.) In two steps, so that several vectors' loads can go out before the
// first is shifted: what lies at e or, past the row's last whole vector, that one; and its shift.
template <int SIZE, typename I>
__device__ __forceinline__ u32x4a fetch_vector(const void* row, I e, I n)
{
    constexpr int kCount = 16 / SIZE;
    const char* p = static_cast<const char*>(row);
    if (n >= kCount) return load16(p + (e < n - kCount ? e : n - kCount) * SIZE);
    u32x4a w = {0u, 0u, 0u, 0u};   // a row shorter than a vector
    if (e == 0) {
#pragma unroll
        for (int j = 0; j < kCount - 1; ++j)
            if (j < n) {
                if constexpr (SIZE == 4) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
                else if constexpr (SIZE == 2)
                    w[j >> 1] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(p)[j])
                                 << (16 * (j & 1));
                else w[j >> 2] |= static_cast<uint32_t>(static_cast<uint8_t>(p[j])) << (8 * (j & 3));
            }
    }
    return w;
}
template <int SIZE, typename I>
__device__ __forceinline__ u32x4a settle_vector(const u32x4a& w, I e, I n)
{
    constexpr int kCount = 16 / SIZE;
    if (n < kCount || e + kCount <= n) return w;
    const I past = e + kCount - n;
    return shift_down(w, past < kCount ? static_cast<uint32_t>(past) * 8 * SIZE : 128u);
}
template <int SIZE, typename I>
__device__ __forceinline__ u32x4a load_vector(const void* row, I e, I n)
{
    return settle_vector<SIZE>(fetch_vector<SIZE>(row, e, n), e, n);
}

// Eight elements, bfloat16 or float32, in the same two steps.
template <bool BF16, typename I>
__device__ __forceinline__ void fetch8(const void* row, I e, I n, u32x4a (&v)[BF16 ? 1 : 2])
{
#pragma unroll
    for (int b = 0; b < (BF16 ? 1 : 2); ++b)
        v[b] = fetch_vector<BF16 ? 2 : 4>(row, static_cast<I>(e + 4 * b), n);
}
template <bool BF16, typename I>
__device__ __forceinline__ void settle8(const u32x4a (&w)[BF16 ? 1 : 2], I e, I n, float (&v)[8])
{
    if constexpr (BF16) {
        const u32x4a t = settle_vector<2>(w[0], e, n);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = bf16_float(t[j]);
            v[2 * j + 1] = __uint_as_float(t[j] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const u32x4a t = settle_vector<4>(w[b], static_cast<I>(e + 4 * b), n);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * b + j] = __uint_as_float(t[j]);
        }
    }
}

// Elements e .. e + 7 of a row of n at `row`, as float32; zero from n on.
template <bool BF16, typename I>
__device__ __forceinline__ void load_row8(const void* row, I e, I n, float (&v)[8])
{
    u32x4a w[BF16 ? 1 : 2];
    fetch8<BF16>(row, e, n, w);
    settle8<BF16>(w, e, n, v);
}

template <bool BF16, typename I>
__device__ __forceinline__ void store_row8(void* row, I e, I n, const float (&v)[8])
{
    if (e + 8 <= n) {
        if constexpr (BF16) {
            u32x4a w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = bf16_pair(v[2 * j], v[2 * j + 1]);
            store16(static_cast<uint16_t*>(row) + e, w);
        } else {
            u32x4a a, b;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a[j] = __float_as_uint(v[j]);
                b[j] = __float_as_uint(v[4 + j]);
            }
            store16(static_cast<float*>(row) + e, a);
            store16(static_cast<float*>(row) + e + 4, b);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (e + j < n) {
                if constexpr (BF16)
                    static_cast<uint16_t*>(row)[e + j] = bf16_bits(v[j]);
                else
                    static_cast<float*>(row)[e + j] = v[j];
            }
    }
}

// ---------------------------------------------------------------- the 8-bit code
// Absolute values are compared by their bits, which order as the values do and put infinity and
// NaN last, so that a group's largest bits tell whether it holds one.
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// E of a group from its largest bits: the exponent less 6 puts |x| / scale into [64, 128); from
// 127.5 / 64 in the leading digits on (the carry of 0x10000) one more, so that no code is 128.
// At most kAct8Top: one more would have 64 stand for 2^128.
__device__ __forceinline__ int act8_exponent(uint32_t top)
{
    const int e = static_cast<int>((top + 0x10000u) >> 23) - 6;
    return top >= 0x7f800000u ? 255 : min(max(e, 1), kAct8Top);
}

// 1 / scale: a power of two, so that products with it are exact (0 for the NaN group).
__device__ __forceinline__ float act8_inverse(int e)
{
    return e == 255 ? 0.0f : __uint_as_float(static_cast<uint32_t>(254 - e) << 23);
}

__device__ __forceinline__ float act8_scale(uint32_t e)
{
    return __uint_as_float(e == 255u ? 0x7fc00000u : e << 23);
}

// rint(x * inv) in the low byte, within +-127 (only kAct8Top needs it): adding 1.5 * 2^23 rounds
// to a whole number, ties to even, and leaves its two's complement in the low bits.
__device__ __forceinline__ uint32_t act8_code(float x, float inv)
{
    return __float_as_uint(__builtin_amdgcn_fmed3f(x * inv, -127.0f, 127.0f) + 12582912.0f);
}

__device__ __forceinline__ uint32_t act8_pack(float a, float b, float c, float d, float inv)
{
    const uint32_t lo = __builtin_amdgcn_perm(act8_code(b, inv), act8_code(a, inv), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(act8_code(d, inv), act8_code(c, inv), 0x04000c0cu);
    return lo | hi;
}

// Code j (0..3) of four packed ones, as float32.
__device__ __forceinline__ float act8_value(uint32_t w, int j)
{
    return static_cast<float>(static_cast<int8_t>(w >> (8 * j)));
}

// Largest over the eight lanes of an aligned run of eight.
__device__ __forceinline__ uint32_t max_over_8(uint32_t m)
{
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 1)));
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 2)));
    return max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 4)));
}

// One group's eight lanes write its codes (w: eight packed ones each) and its exponent.
template <typename I>
__device__ __forceinline__ void act8_store_group(const u32x2a& w, int ex, I e, I n,
                                                 int8_t* __restrict__ codes,
                                                 uint8_t* __restrict__ exps)
{
    if (e + 8 <= n) {
        store8b(codes + e, w);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (e + j < n) codes[e + j] = static_cast<int8_t>((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
    }
    if ((e & 63) == 0 && e < n) exps[e >> 6] = static_cast<uint8_t>(ex);
}

// One group's eight lanes, each with eight elements e .. e + 7 of a row of n (zero from n on),
// write the group's codes and its exponent. Every lane of the eight takes part.
template <typename I>
__device__ __forceinline__ void act8_write_group(const float (&v)[8], I e, I n,
                                                 int8_t* __restrict__ codes,
                                                 uint8_t* __restrict__ exps)
{
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, abs_bits(v[j]));
    const int ex = act8_exponent(max_over_8(top));
    const float inv = act8_inverse(ex);
    u32x2a w = {0u, 0u};   // the codes of a NaN group are zero
    if (ex != 255) {
        w.x = act8_pack(v[0], v[1], v[2], v[3], inv);
        w.y = act8_pack(v[4], v[5], v[6], v[7], inv);
    }
    act8_store_group(w, ex, e, n, codes, exps);
}

// The same of products v[j] * by with `by` in 64 bits: float32 would move about one code in a
// million across a rounding boundary. f: the products rounded to float32; below kAct8Top.
template <typename I>
__device__ __forceinline__ void act8_write_products(const float (&v)[8], double by,
                                                    const float (&f)[8], I e, I n,
                                                    int8_t* __restrict__ codes,
                                                    uint8_t* __restrict__ exps)
{
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, abs_bits(f[j]));
    const int ex = act8_exponent(max_over_8(top));
    const double to = by * static_cast<double>(act8_inverse(ex));
    u32x2a w = {0u, 0u};
    if (ex != 255) {
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)   // 1.5 * 2^52, as in act8_code
            c[j] = static_cast<uint32_t>(__double2loint(
                fma(static_cast<double>(v[j]), to, 6755399441055744.0)));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t lo = __builtin_amdgcn_perm(c[4 * j + 1], c[4 * j], 0x0c0c0400u);
            const uint32_t hi = __builtin_amdgcn_perm(c[4 * j + 3], c[4 * j + 2], 0x04000c0cu);
            w[j] = lo | hi;
        }
    }
    act8_store_group(w, ex, e, n, codes, exps);
}

// Codes e .. e + 7 of a row of n; zero from n on; in the same two steps.
template <typename I>
__device__ __forceinline__ u32x2a fetch_codes8(const int8_t* __restrict__ codes, I e, I n)
{
    if (n >= 8) return load8b(codes + (e < n - 8 ? e : n - 8));
    u32x2a w = {0u, 0u};
    if (e == 0) {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < n) w[j >> 2] |= static_cast<uint32_t>(static_cast<uint8_t>(codes[j])) << (8 * (j & 3));
    }
    return w;
}
template <typename I>
__device__ __forceinline__ u32x2a settle_codes8(const u32x2a& w, I e, I n)
{
    if (n < 8 || e + 8 <= n) return w;
    const I past = e + 8 - n;
    const uint64_t v = w.x | (static_cast<uint64_t>(w.y) << 32);
    const uint64_t r = past < 8 ? v >> (8 * static_cast<uint32_t>(past)) : 0;
    return u32x2a{static_cast<uint32_t>(r), static_cast<uint32_t>(r >> 32)};
}

// Elements e .. e + 7 of a checkpointed row of n; zero from n on.
template <typename I>
__device__ __forceinline__ void act8_read8(const int8_t* __restrict__ codes,
                                           const uint8_t* __restrict__ exps, I e, I n,
                                           float (&v)[8])
{
    const float s = e < n ? act8_scale(exps[e >> 6]) : 0.0f;
    const u32x2a w = settle_codes8(fetch_codes8(codes, e, n), e, n);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = act8_value(w[j >> 2], j & 3) * s;
    if (e + 8 > n) {   // a NaN group's padding is zero too
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (e + j >= n) v[j] = 0.0f;
    }
}

}  // namespace gefen
