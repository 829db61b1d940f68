// Matrix products of the gated feed-forward block on the CDNA4 matrix cores.
//
//   C[m][n] = sum_k A(m, k) B(n, k), bfloat16 operands, float32 accumulators,
//
// where an operand is stored with k contiguous (rows m or n) or with m (n) contiguous (rows k):
// the forward products read rows of k throughout, the input gradients read the weights by rows
// of k, the weight gradients read both operands so. Nothing is transposed in memory: tiles of
// rows of k go through the transposing LDS read (ds_read_b64_tr_b16), which gives a lane four
// consecutive k of its column.
//
// A workgroup computes a 256 x 256 tile with eight waves (4 x 2 of 64 x 128), or a 128 x 128
// tile with four (4 x 1 of 32 x 128) where that fills the chip better. Tiles of 64 k are loaded
// straight into LDS (no registers) through buffer resources, whose range check gives zeros past
// the operand's rows; two LDS stages, the next one in flight while the current one feeds the
// matrix cores, one barrier per stage. LDS rows are not padded: 16-byte pieces (32-byte ones
// for rows of k) are permuted within a row by its low bits, on the loading side through the
// lane's global address, so that fragment reads hit distinct banks.
//
// The products are computed as C^T (the n fragment is the instruction's first operand), so
// that after one exchange between the wave's halves a lane holds 16 consecutive n of one row
// m: the epilogues work on such runs and store them as whole 16-byte pieces, without LDS.
//
// Epilogues:
//   gate/up   the wave's 128 columns are 64 of the gate and the same 64 of the up product:
//             A = act(G) U, and the 8-bit checkpoints of G and U (a group of 64 is one wave's).
//   backward  with dA = dy Wd in the accumulators and the checkpoints of G and U:
//             dG = dA U act'(G), dU = dA act(G), and act(G) U again for the down projection's
//             gradient, so that neither A nor dA is kept.
//   plain     bfloat16, times a factor per column where given; or float32 partial sums of a
//             product split over k, which k_ffn_join adds in order.
#include "act8_device.h"
#include "ffn_internal.h"

#include <type_traits>

namespace gefen {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int BK = 64;
constexpr int NI = 4;                     // 32-column blocks of a wave (128 columns)
constexpr uint32_t kOut = 0x80000000u;    // a vector offset past every resource's range

template <bool BIG>
struct Shape {
    static constexpr int kWaves = BIG ? 8 : 4;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int T = BIG ? 256 : 128;       // tile rows and columns
    static constexpr int MI = BIG ? 2 : 1;          // 32-row blocks of a wave
    static constexpr int kStage = 2 * T * BK;       // elements of one LDS stage (A, then B)
};

// The permutation of a row of k's 32-byte pieces: distinct for four consecutive rows within 128
// bytes, and within 256 bytes for two neighbouring pieces of each.
__device__ __forceinline__ int piece_key(int row) { return (row & 3) | ((row & 1) << 2); }

// One operand's share of the stage loads: four 1 KiB pieces a wave.
template <bool BIG, bool KMAJOR>
struct Loader {
    using S = Shape<BIG>;
    uint32_t off[4];     // byte offsets of the lane's 16 bytes
    int klim;            // rows of n or m: stages from this k on have nothing for this lane

    // DUAL: LDS rows are 64 of the first matrix, 64 of the second, and so on.
    template <bool DUAL>
    __device__ __forceinline__ void init(int wave, int lane, int64_t ld, int64_t klen)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int q = wave * 4 + j;
            if constexpr (KMAJOR) {
                int row = q * 8 + (lane >> 3);
                if constexpr (DUAL) row = (row >> 7) * 64 + (row & 63);
                const int chunk = (lane & 7) ^ (lane >> 3);
                off[j] = static_cast<uint32_t>((row * ld + chunk * 8) * 2);
                klim = static_cast<int>(klen) - chunk * 8;
            } else {
                constexpr int kPer = S::T / 8;            // 16-byte pieces of a row
                const int row = q * (64 / kPer) + lane / kPer;
                const int pc = lane % kPer;
                const int chunk = (((pc >> 1) ^ piece_key(row)) << 1) | (pc & 1);
                off[j] = static_cast<uint32_t>((row * ld + chunk * 8) * 2);
            }
        }
    }
};

struct Work {
    int32_t tm, tn, batch, split;
};

// Work items are dealt to the eight XCDs in contiguous runs; a run walks bands of eight tile
// rows column by column, so that the tiles that run together share panels in the XCD's L2.
__device__ __forceinline__ bool decode_work(const FfnGemm& g, Work& w)
{
    const uint32_t tiles = static_cast<uint32_t>(g.tiles_m * g.tiles_n);
    const uint32_t total = tiles * g.batch * g.splits;
    const uint32_t per = (total + 7) / 8;
    const uint32_t id = (blockIdx.x % 8) * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || id >= total) return false;
    const uint32_t t = id % tiles, rest = id / tiles;
    w.batch = rest % g.batch;
    w.split = rest / g.batch;
    const uint32_t band = t / (8 * g.tiles_n), in = t % (8 * g.tiles_n);
    const uint32_t rows = min(8u, static_cast<uint32_t>(g.tiles_m) - band * 8);
    w.tm = band * 8 + in % rows;
    w.tn = in / rows;
    return true;
}

// A 32 x 32 accumulator block to runs: lane l of half h holds v[0..15] = columns 16 h + 0..15
// of row l % 32. (Element 4 q + i of a lane is column 8 q + 4 h + i.) The two lanes of a row
// exchange elements: both are to be active.
__device__ __forceinline__ void to_run(const f32x16& acc, float (&v)[16])
{
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const auto s = __builtin_amdgcn_permlane32_swap(
                __float_as_uint(acc[4 * q + i]), __float_as_uint(acc[4 * (q + 2) + i]), false,
                false);
            v[8 * q + i] = __uint_as_float(s[0]);
            v[8 * q + 4 + i] = __uint_as_float(s[1]);
        }
}

// Sixteen consecutive elements of a row of n, from column c on, rounded to bfloat16.
__device__ __forceinline__ void store_run(uint16_t* __restrict__ row, int64_t c, int64_t n,
                                          const float (&v)[16])
{
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const float* p = v + 8 * half;
        const float w[8] = {p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7]};
        store_row8<true>(row, c + 8 * half, n, w);
    }
}

// The activation a = act(g) and its derivative; both from one logistic p = 1 / (1 + e^-z):
// silu: a = g p, a' = p + a (1 - p);  gelu in its tanh form, (1 + tanh z) / 2 = the logistic
// of 2 z: a = g p, a' = p + a (1 - p) z', with z = 2 sqrt(2 / pi) (g + 0.044715 g^3).
__device__ __forceinline__ float logistic(float z) { return 1.0f / (1.0f + __expf(-z)); }

template <bool SLOPE>
__device__ __forceinline__ float activation(float g, int act, float& slope)
{
    float z = g, dz = 1.0f;
    if (act == kActGelu) {
        const float q = g * g;
        z = 1.5957691216057308f * g * fmaf(0.044715f, q, 1.0f);
        if (SLOPE) dz = 1.5957691216057308f * fmaf(0.134145f, q, 1.0f);
    }
    const float p = logistic(z);
    const float a = g * p;
    if (SLOPE) slope = fmaf(a * (1.0f - p), dz, p);
    return a;
}

// Sixteen codes of a run and, once a group, its exponent. v2: the wave's other run of the same
// rows (a lane and its partner in the other half hold a group of 64 between them).
__device__ __forceinline__ void write_codes(const float (&v0)[16], const float (&v1)[16],
                                            int64_t c0, int64_t n, int half,
                                            int8_t* __restrict__ codes, uint8_t* __restrict__ exps,
                                            bool on)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, max(abs_bits(v0[i]), abs_bits(v1[i])));
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32)));
    const int ex = act8_exponent(top);
    const float inv = act8_inverse(ex);
    if (!on) return;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const float* v = b ? v1 : v0;
        const int64_t c = c0 + 32 * b + 16 * half;
        u32x4a w = {0u, 0u, 0u, 0u};
        if (ex != 255) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                w[q] = act8_pack(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3], inv);
        }
        if (c + 16 <= n) {
            store16(codes + c, w);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (c + i < n) codes[c + i] = static_cast<int8_t>(w[i >> 2] >> (8 * (i & 3)));
        }
    }
    if (half == 0 && c0 < n) exps[c0 >> 6] = static_cast<uint8_t>(ex);
}

__device__ __forceinline__ u32x4a read_codes(const int8_t* __restrict__ row, int64_t c, int64_t n)
{
    if (c + 16 <= n) return load16(row + c);
    u32x4a w = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (c + i < n) w[i >> 2] |= static_cast<uint32_t>(static_cast<uint8_t>(row[c + i])) << (8 * (i & 3));
    return w;
}

template <int KIND, bool AK, bool BKM, bool BIG>
__global__ __launch_bounds__(Shape<BIG>::kThreads, 2) void k_ffn_gemm(const FfnGemm g)
{
    using S = Shape<BIG>;
    constexpr int T = S::T, MI = S::MI;
    constexpr bool DUAL = KIND == kFfnGateUp;
    // two arrays, so that the compiler sees that reads of one do not wait for loads to the other
    __shared__ __attribute__((aligned(16))) uint16_t lds0[S::kStage];
    __shared__ __attribute__((aligned(16))) uint16_t lds1[S::kStage];
    Work w;
    if (!decode_work(g, w)) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = BIG ? wave >> 1 : wave, wn = BIG ? wave & 1 : 0;
    const int64_t row0 = int64_t(w.tm) * T;
    const int64_t col0 = int64_t(w.tn) * (DUAL ? T / 2 : T);   // DUAL: columns of each matrix

    Loader<BIG, AK> la;
    Loader<BIG, BKM> lb;
    la.template init<false>(wave, lane, g.lda, g.kpad);
    lb.template init<DUAL>(wave, lane, g.ldb, g.kpad);

    const int per_seg = g.stages;                     // stages of one segment of the sum
    const int all = per_seg * g.segments;
    const int first = static_cast<int>(int64_t(all) * w.split / g.splits);
    const int nk = static_cast<int>(int64_t(all) * (w.split + 1) / g.splits) - first;

    auto resource = [](const uint16_t* p, int64_t bytes) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), 0,
                                                 static_cast<int>(bytes), 0x00020000);
    };
    auto load = [&](uint16_t* lds, int it) {
        const int st = first + it;
        const int seg = st >= per_seg ? 1 : 0;
        const int k0 = (st - seg * per_seg) * BK;
        const int ia = g.segments > 1 ? seg : w.batch;
        auto piece = [&](__amdgpu_buffer_rsrc_t r, uint16_t* dst, uint32_t off, int soff) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)dst, 16, off, soff, 0, 0);
        };
        {
            uint16_t* dst = lds + wave * 4 * 512;
            if constexpr (AK) {
                const auto r = resource(g.a[ia] + row0 * g.lda,
                                        2 * min(int64_t(T), g.M - row0) * g.lda);
                const bool in = k0 < la.klim;
#pragma unroll
                for (int j = 0; j < 4; ++j) piece(r, dst + j * 512, in ? la.off[j] : kOut, 2 * k0);
            } else {
                const auto r = resource(g.a[ia] + k0 * g.lda + row0,
                                        2 * (min(int64_t(BK), g.K - k0) * g.lda - row0));
#pragma unroll
                for (int j = 0; j < 4; ++j) piece(r, dst + j * 512, la.off[j], 0);
            }
        }
        {
            uint16_t* dst = lds + T * BK + wave * 4 * 512;
            if constexpr (DUAL) {
                const int64_t bytes = 2 * min(int64_t(T / 2), g.N - col0) * g.ldb;
                const auto r0 = resource(g.b[0] + col0 * g.ldb, bytes);
                const auto r1 = resource(g.b[1] + col0 * g.ldb, bytes);
                const bool in = k0 < lb.klim;
                // a wave's 32 LDS rows lie in one 64-row half
                const bool second = (wave * 32) & 64;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    piece(second ? r1 : r0, dst + j * 512, in ? lb.off[j] : kOut, 2 * k0);
            } else if constexpr (BKM) {
                const auto r = resource(g.b[seg] + col0 * g.ldb,
                                        2 * min(int64_t(T), g.N - col0) * g.ldb);
                const bool in = k0 < lb.klim;
#pragma unroll
                for (int j = 0; j < 4; ++j) piece(r, dst + j * 512, in ? lb.off[j] : kOut, 2 * k0);
            } else {
                const auto r = resource(g.b[seg] + k0 * g.ldb + col0,
                                        2 * (min(int64_t(BK), g.K - k0) * g.ldb - col0));
#pragma unroll
                for (int j = 0; j < 4; ++j) piece(r, dst + j * 512, lb.off[j], 0);
            }
        }
    };

    // Fragments of one 16-deep step: lane l holds row l % 32, k = 8 (l / 32) .. + 7.
    const int half = lane >> 5, l32 = lane & 31;
    auto frag_k = [&](const uint16_t* t, int row, int ks) -> bf16x8 {
        const int chunk = (2 * ks + half) ^ (l32 & 7);
        return *reinterpret_cast<const bf16x8*>(t + (row + l32) * BK + chunk * 8);
    };
    const int trow = 8 * half + ((lane >> 2) & 3);    // row of k this lane reads a piece of
    const int tkey = piece_key((lane >> 2) & 3);
    auto frag_t = [&](const uint16_t* t, int col, int ks) -> bf16x8 {
        const int piece = ((col >> 4) + ((lane >> 4) & 1)) ^ tkey;
        const uint16_t* p = t + (16 * ks + trow) * T + piece * 16 + (lane & 3) * 4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * T));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(bf16x8, v);
    };
    typedef bf16x8 FragA[MI];
    typedef bf16x8 FragB[NI];
    auto frags = [&](FragA& fa, FragB& fb, const uint16_t* lds, int ks) {
        const uint16_t* sb = lds + T * BK;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            const int r = (wm * MI + mi) * 32;
            fa[mi] = AK ? frag_k(lds, r, ks) : frag_t(lds, r, ks);
        }
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) {
            const int c = wn * 128 + ni * 32;
            fb[ni] = BKM ? frag_k(sb, c, ks) : frag_t(sb, c, ks);
        }
    };
    f32x16 acc[MI][NI];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[mi][ni][v] = 0.0f;
    auto mfmas = [&](const FragA& fa, const FragB& fb, int from, int to) {
#pragma unroll
        for (int q = from; q < to; ++q)
            acc[q / NI][q % NI] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                fb[q % NI], fa[q / NI], acc[q / NI][q % NI], 0, 0, 0);
    };
    constexpr int kMM = MI * NI;
    FragA fa[2];
    FragB fb[2];
    // Instruction order inside a step, by scheduling groups: one matrix-core op, then its share
    // of the step's fragment reads, so that no more than two steps' fragments are ever live.
    constexpr int kMfma = 0x008, kDsRead = 0x100;
    constexpr int kReads = MI * (AK ? 1 : 2) + NI * (BKM ? 1 : 2);
    auto interleave = [&](auto ops) {
        constexpr int n = decltype(ops)::value;
#pragma unroll
        for (int q = 0; q < n; ++q) {
            __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
            const int share = (q + 1) * kReads / n - q * kReads / n;
            if (share == 1) __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
            if (share == 2) __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 0);
            if (share == 3) __builtin_amdgcn_sched_group_barrier(kDsRead, 3, 0);
            if (share == 4) __builtin_amdgcn_sched_group_barrier(kDsRead, 4, 0);
            if (share == 5) __builtin_amdgcn_sched_group_barrier(kDsRead, 5, 0);
        }
    };
    typedef std::integral_constant<int, kMM> WholeStep;
    typedef std::integral_constant<int, kMM / 2> HalfStep;
    // One stage: the next stage's loads go out first; each step's matrix-core ops run while the
    // next step's fragments are read; in the middle of the last step the barrier, then the next
    // stage's first fragments under the other half (after the last stage, of what is there).
    auto body = [&](const uint16_t* cur, uint16_t* nxt, int it) {
        if (it + 1 < nk) load(nxt, it + 1);
        __builtin_amdgcn_sched_barrier(0);   // not to be moved behind the matrix-core ops
#pragma unroll
        for (int ks = 0; ks < 3; ++ks) {
            frags(fa[(ks + 1) & 1], fb[(ks + 1) & 1], cur, ks + 1);
            mfmas(fa[ks & 1], fb[ks & 1], 0, kMM);
            interleave(WholeStep{});
        }
        mfmas(fa[1], fb[1], 0, kMM / 2);
        __builtin_amdgcn_sched_group_barrier(kMfma, kMM / 2, 0);
        __syncthreads();
        frags(fa[0], fb[0], nxt, 0);
        mfmas(fa[1], fb[1], kMM / 2, kMM);
        interleave(HalfStep{});
    };
    if (nk > 0) {
        load(lds0, 0);
        __syncthreads();
        frags(fa[0], fb[0], lds0, 0);
        for (int it = 0;; it += 2) {
            body(lds0, lds1, it);
            if (it + 1 >= nk) break;
            body(lds1, lds0, it + 1);
            if (it + 2 >= nk) break;
        }
    }

    // ------------------------------------------------------------------ epilogues
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
        const int64_t row = row0 + (wm * MI + mi) * 32 + l32;
        const bool on = row < g.M;
        if constexpr (KIND == kFfnGateUp) {
            const int64_t c = col0 + wn * 64;
            float gv[2][16], uv[2][16];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                to_run(acc[mi][b], gv[b]);
                to_run(acc[mi][2 + b], uv[b]);
            }
            if (g.gcodes) {
                write_codes(gv[0], gv[1], c, g.N, half, g.gcodes + row * g.N,
                            g.gexps + row * g.groups, on);
                write_codes(uv[0], uv[1], c, g.N, half, g.ucodes + row * g.N,
                            g.uexps + row * g.groups, on);
            }
            if (on) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    float av[16], none;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        av[i] = activation<false>(gv[b][i], g.act, none) * uv[b][i];
                    // columns from N to ldo are read by the next product as zeros
                    store_run(g.o[0] + row * g.ldo, c + 32 * b + 16 * half, g.ldo, av);
                }
            }
        } else if constexpr (KIND == kFfnGateGrad) {
            if (!on) continue;
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                const int64_t c = col0 + wn * 128 + ni * 32 + 16 * half;
                float d[16], dg[16], du[16], av[16];
                to_run(acc[mi][ni], d);   // both halves of the wave take part
                if (c >= g.ldo) continue;
                u32x4a gw = {0u, 0u, 0u, 0u}, uw = gw;
                float gs = 0.0f, us = 0.0f;
                if (c < g.N) {
                    gw = read_codes(g.gcodes + row * g.N, c, g.N);
                    uw = read_codes(g.ucodes + row * g.N, c, g.N);
                    gs = act8_scale(g.gexps[row * g.groups + (c >> 6)]);
                    us = act8_scale(g.uexps[row * g.groups + (c >> 6)]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const bool in = c + i < g.N;
                    const float gv = act8_value(gw[i >> 2], i & 3) * gs;
                    const float uv = act8_value(uw[i >> 2], i & 3) * us;
                    float slope;
                    const float a = activation<true>(gv, g.act, slope);
                    av[i] = in ? a * uv : 0.0f;
                    dg[i] = in ? d[i] * uv * slope : 0.0f;
                    du[i] = in ? d[i] * a : 0.0f;
                }
                store_run(g.o[0] + row * g.ldo, c, g.ldo, dg);
                store_run(g.o[1] + row * g.ldo, c, g.ldo, du);
                store_run(g.o2 + row * g.ldo, c, g.ldo, av);
            }
        } else {
            if (!on) continue;
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                const int64_t c = col0 + wn * 128 + ni * 32 + 16 * half;
                float v[16];
                to_run(acc[mi][ni], v);
                if (g.partial) {
                    float* __restrict__ p =
                        g.partial + ((int64_t(w.split) * g.batch + w.batch) * g.M + row) * g.N;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const float* s = v + 8 * q;
                        const float x[8] = {s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7]};
                        store_row8<false>(p, c + 8 * q, g.N, x);
                    }
                } else {
                    if (g.col_scale) {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (c + i < g.N) v[i] *= g.col_scale[c + i];
                    }
                    store_run(g.o[w.batch] + row * g.ldo, c, g.N, v);
                }
            }
        }
    }
}

// o[b] = the sum over the splits, in order, of the partial products, times the column factors.
__global__ __launch_bounds__(256) void k_ffn_join(const FfnGemm g)
{
    const int64_t e = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
    const int64_t plane = g.M * g.N;
    const int b = blockIdx.y;
    if (e >= plane) return;
    const float* __restrict__ p = g.partial + b * plane;
    float s[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    for (int q = 0; q < g.splits; ++q) {
        float v[8];
        load_row8<false>(p + int64_t(q) * g.batch * plane, e, plane, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += v[j];
    }
    if (g.col_scale) {
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] *= g.col_scale[(e + j) % g.N];
    }
    store_row8<true>(g.o[b], e, plane, s);   // the output is dense
}

// dst (rows of ldd, a multiple of 8) = src (dense rows of `cols`), zero past them.
__global__ __launch_bounds__(256) void k_ffn_pad(const FfnPads p)
{
    const FfnPad& m = p.m[blockIdx.z];
    const int64_t e = (static_cast<int64_t>(blockIdx.x) * 64 + (threadIdx.x & 63)) * 8;
    if (e >= m.ldd) return;
    for (int64_t r = static_cast<int64_t>(blockIdx.y) * 4 + (threadIdx.x >> 6); r < m.rows;
         r += static_cast<int64_t>(gridDim.y) * 4) {
        float v[8];
        load_row8<true>(m.src + r * m.cols, e, m.cols, v);
        store_row8<true>(m.dst + r * m.ldd, e, m.ldd, v);
    }
}

__global__ __launch_bounds__(256) void k_ffn_zero(uint16_t* __restrict__ p, int64_t n)
{
    const int64_t step = 256LL * gridDim.x;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += step) p[i] = 0;
}

template <int KIND, bool AK, bool BKM>
hipError_t launch_kind(const FfnGemm& g, hipStream_t stream)
{
    const int64_t total = int64_t(g.tiles_m) * g.tiles_n * g.batch * g.splits;
    const dim3 grid(static_cast<unsigned>((total + 7) / 8 * 8));
    if (g.big)
        hipLaunchKernelGGL((k_ffn_gemm<KIND, AK, BKM, true>), grid, dim3(Shape<true>::kThreads), 0,
                           stream, g);
    else
        hipLaunchKernelGGL((k_ffn_gemm<KIND, AK, BKM, false>), grid, dim3(Shape<false>::kThreads),
                           0, stream, g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_ffn_gemm(const FfnGemm& g, hipStream_t stream)
{
    hipError_t err;
    if (g.kind == kFfnGateUp)
        err = launch_kind<kFfnGateUp, true, true>(g, stream);
    else if (g.kind == kFfnGateGrad)
        err = launch_kind<kFfnGateGrad, true, false>(g, stream);
    else if (g.a_rows_k)
        err = launch_kind<kFfnPlain, false, false>(g, stream);
    else if (g.b_rows_k)
        err = launch_kind<kFfnPlain, true, false>(g, stream);
    else
        err = launch_kind<kFfnPlain, true, true>(g, stream);
    if (err != hipSuccess || !g.partial) return err;
    const int64_t vectors = (g.M * g.N + 7) / 8;
    hipLaunchKernelGGL(k_ffn_join,
                       dim3(static_cast<unsigned>((vectors + 255) / 256), g.batch),
                       dim3(256), 0, stream, g);
    return hipGetLastError();
}

hipError_t launch_ffn_pads(const FfnPads& p, hipStream_t stream)
{
    int64_t rows = 0, ldd = 0;
    for (int i = 0; i < p.n; ++i) {
        rows = p.m[i].rows > rows ? p.m[i].rows : rows;
        ldd = p.m[i].ldd > ldd ? p.m[i].ldd : ldd;
    }
    if (!p.n || !rows) return hipSuccess;
    const int64_t gy = (rows + 3) / 4;
    hipLaunchKernelGGL(k_ffn_pad,
                       dim3(static_cast<unsigned>((ldd + 511) / 512),
                            static_cast<unsigned>(gy < 65535 ? gy : 65535), p.n),
                       dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_zero_bf16(uint16_t* p, int64_t n, hipStream_t stream)
{
    if (n <= 0) return hipSuccess;
    const int64_t groups = (n + 255) / 256;
    hipLaunchKernelGGL(k_ffn_zero, dim3(static_cast<unsigned>(groups < 4096 ? groups : 4096)),
                       dim3(256), 0, stream, p, n);
    return hipGetLastError();
}

}  // namespace gefen
