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

namespace gefen {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) uint16_t lds_u16;

constexpr int BK = 32;                    // depth of a stage
constexpr int kStages = 4;                // stages in LDS: three in flight
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

// The permutation of a row's eight 16-byte pieces of k: a fragment read takes 16 rows at a time,
// which are to fill 256 bytes of banks. (With row & 7 as the key, rows 8 apart met in a bank:
// half of the read cycles were conflicts.)
__device__ __forceinline__ int chunk_key(int row) { return (row >> 2) & 3; }

// The permutation of a row of k's 32-byte pieces: distinct for four consecutive rows within 128
// bytes, and within 256 bytes for two neighbouring pieces of each.
__device__ __forceinline__ int piece_key(int row) { return (row & 3) | ((row & 1) << 2); }

// One operand's share of the stage loads: four 1 KiB pieces a wave.
template <bool BIG, bool KMAJOR>
struct Loader {
    using S = Shape<BIG>;
    uint32_t off[2];     // byte offsets of the lane's 16 bytes
    int klim;            // rows of n or m: nothing for this lane at stages from k = klim on

    // DUAL: LDS rows are 64 of the first matrix, 64 of the second, and so on.
    template <bool DUAL>
    __device__ __forceinline__ void init(int wave, int lane, int64_t ld, int64_t klen)
    {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int q = wave * 2 + j;
            if constexpr (KMAJOR) {
                int row = q * 16 + (lane >> 2);
                if constexpr (DUAL) row = (row >> 7) * 64 + (row & 63);
                const int chunk = (lane & 3) ^ chunk_key(row);
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

// Fragments of two 16-deep steps from rows of k (of T elements), N 32-wide blocks at the byte
// addresses at[]: four transposing reads each, of four rows of k. One block with its own wait,
// so that the compiler neither uses nor reuses a register that is still to be written. (It
// would wait for every load to LDS in flight before this instruction's builtin, whatever buffer
// that is for.)
template <int T>
__device__ __forceinline__ void read_t(const uint32_t (&p)[4], u32x2a (&o)[16])
{
    asm volatile("ds_read_b64_tr_b16 %[o0], %[p0]\n\t"
                 "ds_read_b64_tr_b16 %[o1], %[p0] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o2], %[p0] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o3], %[p0] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o4], %[p1]\n\t"
                 "ds_read_b64_tr_b16 %[o5], %[p1] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o6], %[p1] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o7], %[p1] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o8], %[p2]\n\t"
                 "ds_read_b64_tr_b16 %[o9], %[p2] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o10], %[p2] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o11], %[p2] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o12], %[p3]\n\t"
                 "ds_read_b64_tr_b16 %[o13], %[p3] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o14], %[p3] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o15], %[p3] offset:%[s3]\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : [o0] "=&v"(o[0]), [o1] "=&v"(o[1]), [o2] "=&v"(o[2]), [o3] "=&v"(o[3]), [o4]
                   "=&v"(o[4]), [o5] "=&v"(o[5]), [o6] "=&v"(o[6]), [o7] "=&v"(o[7]), [o8]
                   "=&v"(o[8]), [o9] "=&v"(o[9]), [o10] "=&v"(o[10]), [o11] "=&v"(o[11]), [o12]
                   "=&v"(o[12]), [o13] "=&v"(o[13]), [o14] "=&v"(o[14]), [o15] "=&v"(o[15])
                 : [p0] "v"(p[0]), [p1] "v"(p[1]), [p2] "v"(p[2]), [p3] "v"(p[3]), [s1] "n"(8 *
                   T), [s2] "n"(32 * T), [s3] "n"(40 * T)
                 : "memory");
}

template <int T>
__device__ __forceinline__ void read_t(const uint32_t (&p)[5], u32x2a (&o)[20])
{
    asm volatile("ds_read_b64_tr_b16 %[o0], %[p0]\n\t"
                 "ds_read_b64_tr_b16 %[o1], %[p0] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o2], %[p0] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o3], %[p0] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o4], %[p1]\n\t"
                 "ds_read_b64_tr_b16 %[o5], %[p1] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o6], %[p1] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o7], %[p1] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o8], %[p2]\n\t"
                 "ds_read_b64_tr_b16 %[o9], %[p2] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o10], %[p2] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o11], %[p2] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o12], %[p3]\n\t"
                 "ds_read_b64_tr_b16 %[o13], %[p3] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o14], %[p3] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o15], %[p3] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o16], %[p4]\n\t"
                 "ds_read_b64_tr_b16 %[o17], %[p4] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o18], %[p4] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o19], %[p4] offset:%[s3]\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : [o0] "=&v"(o[0]), [o1] "=&v"(o[1]), [o2] "=&v"(o[2]), [o3] "=&v"(o[3]), [o4]
                   "=&v"(o[4]), [o5] "=&v"(o[5]), [o6] "=&v"(o[6]), [o7] "=&v"(o[7]), [o8]
                   "=&v"(o[8]), [o9] "=&v"(o[9]), [o10] "=&v"(o[10]), [o11] "=&v"(o[11]), [o12]
                   "=&v"(o[12]), [o13] "=&v"(o[13]), [o14] "=&v"(o[14]), [o15] "=&v"(o[15]), [o16]
                   "=&v"(o[16]), [o17] "=&v"(o[17]), [o18] "=&v"(o[18]), [o19] "=&v"(o[19])
                 : [p0] "v"(p[0]), [p1] "v"(p[1]), [p2] "v"(p[2]), [p3] "v"(p[3]), [p4] "v"(p[4]),
                   [s1] "n"(8 * T), [s2] "n"(32 * T), [s3] "n"(40 * T)
                 : "memory");
}

template <int T>
__device__ __forceinline__ void read_t(const uint32_t (&p)[6], u32x2a (&o)[24])
{
    asm volatile("ds_read_b64_tr_b16 %[o0], %[p0]\n\t"
                 "ds_read_b64_tr_b16 %[o1], %[p0] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o2], %[p0] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o3], %[p0] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o4], %[p1]\n\t"
                 "ds_read_b64_tr_b16 %[o5], %[p1] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o6], %[p1] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o7], %[p1] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o8], %[p2]\n\t"
                 "ds_read_b64_tr_b16 %[o9], %[p2] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o10], %[p2] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o11], %[p2] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o12], %[p3]\n\t"
                 "ds_read_b64_tr_b16 %[o13], %[p3] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o14], %[p3] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o15], %[p3] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o16], %[p4]\n\t"
                 "ds_read_b64_tr_b16 %[o17], %[p4] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o18], %[p4] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o19], %[p4] offset:%[s3]\n\t"
                 "ds_read_b64_tr_b16 %[o20], %[p5]\n\t"
                 "ds_read_b64_tr_b16 %[o21], %[p5] offset:%[s1]\n\t"
                 "ds_read_b64_tr_b16 %[o22], %[p5] offset:%[s2]\n\t"
                 "ds_read_b64_tr_b16 %[o23], %[p5] offset:%[s3]\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : [o0] "=&v"(o[0]), [o1] "=&v"(o[1]), [o2] "=&v"(o[2]), [o3] "=&v"(o[3]), [o4]
                   "=&v"(o[4]), [o5] "=&v"(o[5]), [o6] "=&v"(o[6]), [o7] "=&v"(o[7]), [o8]
                   "=&v"(o[8]), [o9] "=&v"(o[9]), [o10] "=&v"(o[10]), [o11] "=&v"(o[11]), [o12]
                   "=&v"(o[12]), [o13] "=&v"(o[13]), [o14] "=&v"(o[14]), [o15] "=&v"(o[15]), [o16]
                   "=&v"(o[16]), [o17] "=&v"(o[17]), [o18] "=&v"(o[18]), [o19] "=&v"(o[19]), [o20]
                   "=&v"(o[20]), [o21] "=&v"(o[21]), [o22] "=&v"(o[22]), [o23] "=&v"(o[23])
                 : [p0] "v"(p[0]), [p1] "v"(p[1]), [p2] "v"(p[2]), [p3] "v"(p[3]), [p4] "v"(p[4]),
                   [p5] "v"(p[5]), [s1] "n"(8 * T), [s2] "n"(32 * T), [s3] "n"(40 * T)
                 : "memory");
}

__device__ __forceinline__ bf16x8 join(const u32x2a& a, const u32x2a& b)
{
    const u32x4a v = {a[0], a[1], b[0], b[1]};
    return __builtin_bit_cast(bf16x8, v);
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
    __shared__ __attribute__((aligned(16))) uint16_t lds2[S::kStage];
    __shared__ __attribute__((aligned(16))) uint16_t lds3[S::kStage];
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

    auto resource = [](const uint16_t* p, int bytes) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), 0, bytes, 0x00020000);
    };
    auto load_piece = [](__amdgpu_buffer_rsrc_t r, uint16_t* dst, uint32_t off) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)dst, 16, off, 0, 0, 0);
    };
    // Where the next stage's pieces come from, moved on stage by stage in scalar registers; past
    // the last stage, ranges of no bytes.
    const int lda = static_cast<int>(g.lda), ldb = static_cast<int>(g.ldb);
    const int klen = static_cast<int>(g.K), kend = per_seg * BK;
    const int a_rows = static_cast<int>(min(int64_t(T), g.M - row0));
    const int b_rows = static_cast<int>(min(int64_t(DUAL ? T / 2 : T), g.N - col0));
    const int a_col = static_cast<int>(row0), b_col = static_cast<int>(col0);   // rows of k
    const uint16_t* a_base[2];
    const uint16_t* b_base[2];
    a_base[0] = g.a[g.segments > 1 ? 0 : w.batch] + (AK ? row0 * g.lda : row0);
    a_base[1] = g.a[1] + (AK ? row0 * g.lda : row0);
    // DUAL: a wave's 32 LDS rows lie in one 64-row half
    b_base[0] = g.b[DUAL ? (wave * 32) >> 6 & 1 : 0] + (BKM ? col0 * g.ldb : col0);
    b_base[1] = g.b[1] + (BKM ? col0 * g.ldb : col0);
    const int64_t a_step = AK ? BK : int64_t(BK) * g.lda, b_step = BKM ? BK : int64_t(BK) * g.ldb;
    const bool second = first >= per_seg;
    struct Source {
        const uint16_t *a, *b;
        int k0, left;      // left: stages still to be loaded
    } at;
    at.k0 = (first - (second ? per_seg : 0)) * BK;
    at.a = a_base[second] + (AK ? at.k0 : at.k0 * g.lda);
    at.b = b_base[second] + (BKM ? at.k0 : at.k0 * g.ldb);
    at.left = nk;
    auto a_bytes = [&]() {
        return at.left <= 0 ? 0
                            : 2 * (AK ? a_rows * lda - at.k0 : min(BK, klen - at.k0) * lda - a_col);
    };
    auto b_bytes = [&]() {
        return at.left <= 0
                   ? 0
                   : 2 * (BKM ? b_rows * ldb - at.k0 : min(BK, klen - at.k0) * ldb - b_col);
    };
    auto advance = [&]() {
        --at.left;
        at.k0 += BK;
        at.a += a_step;
        at.b += b_step;
        if (at.k0 == kend) {   // on to the second segment, if there is one
            at.k0 = 0;
            at.a = a_base[1];
            at.b = b_base[1];
        }
    };
    // The wave's four pieces of a stage: two of A, two of B.
    auto load = [&](uint16_t* lds) {
        const int an = a_bytes(), bn = b_bytes();
#pragma unroll
        for (int j = 0; j < 2; ++j)
            load_piece(resource(at.a, an), lds + (wave * 2 + j) * 512,
                       AK && at.k0 >= la.klim ? kOut : la.off[j]);
#pragma unroll
        for (int j = 0; j < 2; ++j)
            load_piece(resource(at.b, bn), lds + T * BK + (wave * 2 + j) * 512,
                       BKM && at.k0 >= lb.klim ? kOut : lb.off[j]);
        advance();
    };

    // A stage's fragments, two 16-deep steps: lane l holds row l % 32, k = 8 (l / 32) .. + 7.
    const int half = lane >> 5, l32 = lane & 31;
    bf16x8 fa[2][MI], fb[2][NI];
    auto frag_k = [&](const uint16_t* t, int row, int ks) -> bf16x8 {
        const int chunk = (2 * ks + half) ^ chunk_key(l32);
        return *reinterpret_cast<const bf16x8*>(t + (row + l32) * BK + chunk * 8);
    };
    // Rows of k: byte address of the lane's 8 bytes of the first step's first four rows.
    const int trow = 8 * half + ((lane >> 2) & 3);
    const int tkey = piece_key((lane >> 2) & 3);
    auto addr_t = [&](const uint16_t* t, int col) -> uint32_t {
        const int piece = ((col >> 4) + ((lane >> 4) & 1)) ^ tkey;
        return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(
                   (lds_u16*)(t + trow * T + piece * 16 + (lane & 3) * 4)));
    };
    auto frags = [&](const uint16_t* lds) {
        const uint16_t* sb = lds + T * BK;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            if constexpr (AK) {
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) fa[ks][mi] = frag_k(lds, (wm * MI + mi) * 32, ks);
            }
            if constexpr (BKM) {
#pragma unroll
                for (int ni = 0; ni < NI; ++ni) fb[ks][ni] = frag_k(sb, wn * 128 + ni * 32, ks);
            }
        }
        if constexpr (!BKM) {   // rows of k: B, and A with it
            constexpr int NA = AK ? 0 : MI;
            uint32_t at[NI + NA];
            u32x2a o[4 * (NI + NA)];
#pragma unroll
            for (int i = 0; i < NI + NA; ++i)
                at[i] = i < NI ? addr_t(sb, wn * 128 + i * 32)
                               : addr_t(lds, (wm * MI + i - NI) * 32);
            read_t<T>(at, o);
#pragma unroll
            for (int i = 0; i < NI + NA; ++i)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    const bf16x8 f = join(o[4 * i + 2 * ks], o[4 * i + 2 * ks + 1]);
                    if (i < NI) fb[ks][i] = f;
                    else fa[ks][i - NI] = f;
                }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    static_assert(AK || !BKM, "an A of rows of k goes with such a B");
    f32x16 acc[MI][NI];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[mi][ni][v] = 0.0f;
    auto mfmas = [&]() {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int q = 0; q < MI * NI; ++q)
                acc[q / NI][q % NI] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    fb[ks][q % NI], fa[ks][q / NI], acc[q / NI][q % NI], 0, 0, 0);
    };
    auto barrier = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    // This wave's LDS reads are done, and its loads but for the newest two stages' (four each).
    auto settled = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0070 | 4 * (kStages - 2));
    };
    // A stage is two phases with a barrier after each: fragments out of LDS and the loads of
    // the stage three ahead; then the matrix-core ops. With eight waves, two to a SIMD, the
    // second four run one phase behind the first: each SIMD's matrix core works for one wave
    // while the other reads. The loads go to the buffer of the stage before this one, whose
    // reads ended before the last barrier; a stage's loads have settled in every wave before
    // the barrier that its first readers pass.
    auto body = [&](const uint16_t* cur, uint16_t* to) {
        if constexpr (!BIG) {
            settled();
            barrier();
        }
        frags(cur);
        load(to);
        if constexpr (BIG) {
            settled();
            barrier();
            __builtin_amdgcn_s_setprio(1);
        }
        mfmas();
        if constexpr (BIG) {
            __builtin_amdgcn_s_setprio(0);
            barrier();
        }
    };
    if (nk > 0) {
        load(lds0);
        load(lds1);
        load(lds2);
        if constexpr (BIG) {
            settled();
            barrier();
            if (wave >= 4) barrier();
        }
        for (int it = 0; it < nk; it += 4) {
            body(lds0, lds3);
            body(lds1, lds0);
            body(lds2, lds1);
            body(lds3, lds2);
        }
        if (BIG && wave < 4) barrier();
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
