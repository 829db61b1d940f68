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
// A workgroup computes a 256 x 256 tile with eight waves (4 x 2 of 64 x 128), or a 128 x 128 or
// 64 x 128 tile with four (4 x 1 of 32 x 128, 16 x 128) where that fills the chip better. Stages
// of 64 k are loaded straight into LDS (no registers) through buffer resources, whose range
// check gives zeros past the operand's rows; a stage is used in two parts (B's column halves)
// and the loads of the next parts stay in flight while one feeds the matrix cores. In the
// largest tile the waves are two groups, one part behind the other, so that one group's matrix
// instructions cover the other's LDS reads. LDS rows are not padded: 16-byte pieces (32-byte
// ones for rows of k) are permuted within a row by its low bits, on the loading side through
// the lane's global address, so that fragment reads hit distinct banks (counters: no conflict).
//
// The products are computed as C^T (the n fragment is the instruction's first operand), so
// that after an exchange among the four lanes of a row a lane holds 16 consecutive n of one row
// m: the epilogues work on such runs and store them as whole 16-byte pieces, without LDS.
//
// Bound by the matrix cores and the card's power at large sizes. 8192 tokens, 2048 to 8192
// columns and back (flops of the product alone; the card's plain large product reaches 1.42
// PFLOP/s, the library's six products of these sizes 1.16 to 1.60):
//   gate/up 438 us (1.26 PFLOP/s with the checkpoints), down 187 (1.47), the gradients of the
//   gate 325 (0.85: over a quarter of it is the epilogue, whose reads and writes come in bursts since
//   all workgroups reach it together, and whose values leave no register free: 48 bytes a lane go
//   through scratch), weight gradients 632 (1.30), dx 382 (1.44).
// Smaller ones are bound by latency per stage and by the partial sums of a split product: 1000
// tokens take 53 us for gate/up and 48 + 6 for down, of 72 at the large product's rate.
// Measured and slower: loads between the matrix instructions, a stage's A loaded for two parts
// at once, 32-k stages, 32 x 32 x 16 instructions, smaller tiles for the gate's gradients.
//
// Epilogues:
//   gate/up   the wave's 128 columns are 64 of the gate and the same 64 of the up product:
//             A = act(G) U, and the 8-bit checkpoints of G and U (a group of 64 is one wave's).
//   backward  with dA = dy Wd in the accumulators and the checkpoints of G and U:
//             dG = dA U act'(G), dU = dA act(G), and act(G) U again for the down projection's
//             gradient, so that neither A nor dA is kept.
//   plain     bfloat16, times a factor per column where given; or float32 partial sums of a
//             product split over k, which k_ffn_join adds in order.
// A, dG and dU are rounded to bfloat16, as the next product's matrix instructions read them (float32
// operands run at a sixteenth of the rate): an output then lies 0.0024 of its norm from the formula,
// where its own rounding alone leaves 0.0017.
#include "act8_device.h"
#include "ffn_internal.h"

#include <type_traits>

namespace gefen {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) uint16_t lds_u16;

constexpr int BK = 64;                    // k of a stage: 128 bytes of a row
constexpr int NJ = 4;                     // 16-column blocks of a wave in each half of B
constexpr uint32_t kOut = 0x80000000u;    // a vector offset past every resource's range

// The tiles (kFfnTile*): rows of C, and columns in two halves.
template <int SIZE>
struct Shape {
    static constexpr bool kPhases = SIZE == kFfnTile256;        // two waves to a SIMD, in turn
    static constexpr int kWaves = kPhases ? 8 : 4;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int TM = SIZE == kFfnTile256 ? 256 : SIZE == kFfnTile128 ? 128 : 64;
    static constexpr int H = kPhases ? 128 : 64;                // columns of each half
    static constexpr int MI = TM / 64;                          // 16-row blocks of a wave
    static constexpr int kLoadsA = TM / (8 * kWaves);           // 1 KiB loads of a wave and stage
};

// The permutation of a row's eight 16-byte pieces of k: a fragment read takes 16 rows at a time,
// which are to fill 256 bytes of banks. (With row & 7 as the key, rows 8 apart met in a bank:
// half of the read cycles were conflicts.)
__device__ __forceinline__ int chunk_key(int row) { return (row >> 1) & 7; }

// The permutation of a row of k's 32-byte pieces (WIDE / 16 of them): a transposing read takes
// four consecutive rows, and those eight further on, which are to lie in distinct 32 bytes of
// 256 bytes of banks. (Rows of 64 elements alternate between its halves by themselves.)
template <int WIDE>
__device__ __forceinline__ int piece_key(int row)
{
    static_assert(WIDE >= 64, "four pieces");
    return WIDE == 64 ? ((row >> 1) & 1) | ((row >> 2) & 2) : (row & 3) | ((row >> 1) & 4);
}

// Where a lane's 16 bytes of its wave's N loads of 1 KiB come from, in bytes from the stage's
// first element: of a K-major tile 8 rows of 64 k a load, else 1024 / (2 WIDE) rows of WIDE.
template <bool KMAJOR, int WIDE, int N>
__device__ __forceinline__ void lane_offsets(int wave, int lane, int64_t ld, uint32_t (&off)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int q = wave * N + j;
        int row, chunk;
        if constexpr (KMAJOR) {
            row = q * 8 + (lane >> 3);
            chunk = (lane & 7) ^ chunk_key(row);
        } else {
            constexpr int kPer = WIDE / 8;            // 16-byte pieces of a row
            row = q * (64 / kPer) + lane / kPer;
            const int pc = lane % kPer;
            chunk = (((pc >> 1) ^ piece_key<WIDE>(row)) << 1) | (pc & 1);
        }
        off[j] = static_cast<uint32_t>((row * ld + chunk * 8) * 2);
    }
}

struct Work {
    int32_t tm, tn, batch, split;
};

// Work items are dealt to the eight XCDs in contiguous runs; a run walks bands of eight tile
// rows column by column, so that the tiles that run together share panels in the XCD's L2.
__device__ __forceinline__ bool decode_work(const FfnGemm& g, uint32_t block, Work& w)
{
    const uint32_t tiles = static_cast<uint32_t>(g.tiles_m * g.tiles_n);
    const uint32_t total = tiles * g.batch * g.splits;
    const uint32_t per = (total + 7) / 8;
    const uint32_t id = (block % 8) * per + block / 8;
    if (block / 8 >= per || id >= total) return false;
    const uint32_t t = id % tiles, rest = id / tiles;
    w.batch = rest % g.batch;
    w.split = rest / g.batch;
    const uint32_t band = t / (8 * g.tiles_n), in = t % (8 * g.tiles_n);
    const uint32_t rows = min(8u, static_cast<uint32_t>(g.tiles_m) - band * 8);
    w.tm = band * 8 + in % rows;
    w.tn = in / rows;
    return true;
}

// Four 16 x 16 accumulator blocks side by side to runs: lane l, q = l / 16, holds element i of
// column 16 j + 4 q + i of row l % 16 as acc[j][i], and gets columns 16 q + 0..15 of the same row
// as v. The four lanes of a row exchange elements: all are to be active.
__device__ __forceinline__ void to_run(const f32x4 (&acc)[NJ], float (&v)[16])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto e = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[0][i]),
                                                        __float_as_uint(acc[2][i]), false, false);
        const auto o = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[1][i]),
                                                        __float_as_uint(acc[3][i]), false, false);
        const auto lo = __builtin_amdgcn_permlane16_swap(e[0], o[0], false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(e[1], o[1], false, false);
        v[i] = __uint_as_float(lo[0]);
        v[4 + i] = __uint_as_float(lo[1]);
        v[8 + i] = __uint_as_float(hi[0]);
        v[12 + i] = __uint_as_float(hi[1]);
    }
}

// Sixteen consecutive elements of a row of n, from column c on, rounded to bfloat16. FULL: they
// are all there (in each of these functions).
template <bool FULL>
__device__ __forceinline__ void store_run(uint16_t* __restrict__ row, int64_t c, int64_t n,
                                          const float (&v)[16])
{
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const float* p = v + 8 * half;
        const float w[8] = {p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7]};
        store_row8<true>(row, c + 8 * half, FULL ? c + 8 * half + 8 : n, w);
    }
}

// The activation a = act(g) and its derivative; both from one logistic p = 1 / (1 + e^-z):
// silu: a = g p, a' = p + a (1 - p);  gelu in its tanh form, (1 + tanh z) / 2 = the logistic
// of 2 z: a = g p, a' = p + a (1 - p) z', with z = 2 sqrt(2 / pi) (g + 0.044715 g^3).
// (The reciprocal is the hardware's, within one unit in the last place.)
__device__ __forceinline__ float logistic(float z)
{
    return __builtin_amdgcn_rcpf(1.0f + __expf(-z));
}

template <int ACT, bool SLOPE>
__device__ __forceinline__ float activation(float g, float& slope)
{
    float z = g, dz = 1.0f;
    if (ACT == kActGelu) {
        const float s = fminf(g * g, 1e30f);   // an infinite z' times a zero would be NaN
        z = 1.5957691216057308f * g * fmaf(0.044715f, s, 1.0f);
        if (SLOPE) dz = 1.5957691216057308f * fmaf(0.134145f, s, 1.0f);
    }
    const float p = logistic(z);
    const float a = g * p;
    if (SLOPE) slope = fmaf(a * (1.0f - p), dz, p);
    return a;
}

// The codes of a run and, once a group, its exponent: the four lanes of a row hold a group of 64,
// from column c - 16 q on.
template <bool FULL>
__device__ __forceinline__ void write_codes(const float (&v)[16], int64_t c, int64_t n, int q,
                                            int8_t* __restrict__ codes, uint8_t* __restrict__ exps,
                                            bool on)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, abs_bits(v[i]));
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 16)));
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32)));
    const int ex = act8_exponent(top);
    const float inv = act8_inverse(ex);
    if (!FULL && !on) return;
    u32x4a w = {0u, 0u, 0u, 0u};
    if (ex != 255) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            w[k] = act8_pack(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3], inv);
    }
    if (FULL || c + 16 <= n) {
        store16(codes + c, w);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (c + i < n) codes[c + i] = static_cast<int8_t>(w[i >> 2] >> (8 * (i & 3)));
    }
    if (q == 0 && (FULL || c < n)) exps[c >> 6] = static_cast<uint8_t>(ex);
}

template <bool FULL>
__device__ __forceinline__ u32x4a read_codes(const int8_t* __restrict__ row, int64_t c, int64_t n)
{
    return FULL ? load16(row + c) : load_vector<1>(row, c, n);
}

// Fragments of a stage's two 32-deep steps from rows of k, of 16-wide blocks at the byte
// addresses p[]: four transposing reads each, of four rows of k; first A's blocks (rows of SA
// bytes), then four of B's (rows of SB bytes). One block with its own wait, so that the compiler
// neither uses nor reuses a register that is still to be written. (It would wait for every load
// to LDS in flight before this instruction's builtin, whatever buffer that is for.)
template <int SA, int SB>
__device__ __forceinline__ void read_t(const uint32_t (&p)[4], u32x2a (&o)[16])
{
    asm volatile("ds_read_b64_tr_b16 %[o0], %[p0]\n\t"
                 "ds_read_b64_tr_b16 %[o1], %[p0] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o2], %[p0] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o3], %[p0] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o4], %[p1]\n\t"
                 "ds_read_b64_tr_b16 %[o5], %[p1] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o6], %[p1] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o7], %[p1] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o8], %[p2]\n\t"
                 "ds_read_b64_tr_b16 %[o9], %[p2] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o10], %[p2] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o11], %[p2] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o12], %[p3]\n\t"
                 "ds_read_b64_tr_b16 %[o13], %[p3] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o14], %[p3] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o15], %[p3] offset:%[b3]\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : [o0] "=&v"(o[0]), [o1] "=&v"(o[1]), [o2] "=&v"(o[2]), [o3] "=&v"(o[3]), [o4]
                   "=&v"(o[4]), [o5] "=&v"(o[5]), [o6] "=&v"(o[6]), [o7] "=&v"(o[7]), [o8]
                   "=&v"(o[8]), [o9] "=&v"(o[9]), [o10] "=&v"(o[10]), [o11] "=&v"(o[11]), [o12]
                   "=&v"(o[12]), [o13] "=&v"(o[13]), [o14] "=&v"(o[14]), [o15] "=&v"(o[15])
                 : [p0] "v"(p[0]), [p1] "v"(p[1]), [p2] "v"(p[2]), [p3] "v"(p[3]), [b1] "n"(4 *
                   SB), [b2] "n"(32 * SB), [b3] "n"(36 * SB)
                 : "memory");
}

template <int SA, int SB>
__device__ __forceinline__ void read_t(const uint32_t (&p)[5], u32x2a (&o)[20])
{
    asm volatile("ds_read_b64_tr_b16 %[o0], %[p0]\n\t"
                 "ds_read_b64_tr_b16 %[o1], %[p0] offset:%[a1]\n\t"
                 "ds_read_b64_tr_b16 %[o2], %[p0] offset:%[a2]\n\t"
                 "ds_read_b64_tr_b16 %[o3], %[p0] offset:%[a3]\n\t"
                 "ds_read_b64_tr_b16 %[o4], %[p1]\n\t"
                 "ds_read_b64_tr_b16 %[o5], %[p1] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o6], %[p1] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o7], %[p1] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o8], %[p2]\n\t"
                 "ds_read_b64_tr_b16 %[o9], %[p2] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o10], %[p2] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o11], %[p2] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o12], %[p3]\n\t"
                 "ds_read_b64_tr_b16 %[o13], %[p3] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o14], %[p3] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o15], %[p3] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o16], %[p4]\n\t"
                 "ds_read_b64_tr_b16 %[o17], %[p4] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o18], %[p4] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o19], %[p4] offset:%[b3]\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : [o0] "=&v"(o[0]), [o1] "=&v"(o[1]), [o2] "=&v"(o[2]), [o3] "=&v"(o[3]), [o4]
                   "=&v"(o[4]), [o5] "=&v"(o[5]), [o6] "=&v"(o[6]), [o7] "=&v"(o[7]), [o8]
                   "=&v"(o[8]), [o9] "=&v"(o[9]), [o10] "=&v"(o[10]), [o11] "=&v"(o[11]), [o12]
                   "=&v"(o[12]), [o13] "=&v"(o[13]), [o14] "=&v"(o[14]), [o15] "=&v"(o[15]), [o16]
                   "=&v"(o[16]), [o17] "=&v"(o[17]), [o18] "=&v"(o[18]), [o19] "=&v"(o[19])
                 : [p0] "v"(p[0]), [p1] "v"(p[1]), [p2] "v"(p[2]), [p3] "v"(p[3]), [p4] "v"(p[4]),
                   [a1] "n"(4 * SA), [a2] "n"(32 * SA), [a3] "n"(36 * SA), [b1] "n"(4 * SB), [b2]
                   "n"(32 * SB), [b3] "n"(36 * SB)
                 : "memory");
}

template <int SA, int SB>
__device__ __forceinline__ void read_t(const uint32_t (&p)[6], u32x2a (&o)[24])
{
    asm volatile("ds_read_b64_tr_b16 %[o0], %[p0]\n\t"
                 "ds_read_b64_tr_b16 %[o1], %[p0] offset:%[a1]\n\t"
                 "ds_read_b64_tr_b16 %[o2], %[p0] offset:%[a2]\n\t"
                 "ds_read_b64_tr_b16 %[o3], %[p0] offset:%[a3]\n\t"
                 "ds_read_b64_tr_b16 %[o4], %[p1]\n\t"
                 "ds_read_b64_tr_b16 %[o5], %[p1] offset:%[a1]\n\t"
                 "ds_read_b64_tr_b16 %[o6], %[p1] offset:%[a2]\n\t"
                 "ds_read_b64_tr_b16 %[o7], %[p1] offset:%[a3]\n\t"
                 "ds_read_b64_tr_b16 %[o8], %[p2]\n\t"
                 "ds_read_b64_tr_b16 %[o9], %[p2] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o10], %[p2] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o11], %[p2] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o12], %[p3]\n\t"
                 "ds_read_b64_tr_b16 %[o13], %[p3] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o14], %[p3] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o15], %[p3] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o16], %[p4]\n\t"
                 "ds_read_b64_tr_b16 %[o17], %[p4] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o18], %[p4] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o19], %[p4] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o20], %[p5]\n\t"
                 "ds_read_b64_tr_b16 %[o21], %[p5] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o22], %[p5] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o23], %[p5] offset:%[b3]\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : [o0] "=&v"(o[0]), [o1] "=&v"(o[1]), [o2] "=&v"(o[2]), [o3] "=&v"(o[3]), [o4]
                   "=&v"(o[4]), [o5] "=&v"(o[5]), [o6] "=&v"(o[6]), [o7] "=&v"(o[7]), [o8]
                   "=&v"(o[8]), [o9] "=&v"(o[9]), [o10] "=&v"(o[10]), [o11] "=&v"(o[11]), [o12]
                   "=&v"(o[12]), [o13] "=&v"(o[13]), [o14] "=&v"(o[14]), [o15] "=&v"(o[15]), [o16]
                   "=&v"(o[16]), [o17] "=&v"(o[17]), [o18] "=&v"(o[18]), [o19] "=&v"(o[19]), [o20]
                   "=&v"(o[20]), [o21] "=&v"(o[21]), [o22] "=&v"(o[22]), [o23] "=&v"(o[23])
                 : [p0] "v"(p[0]), [p1] "v"(p[1]), [p2] "v"(p[2]), [p3] "v"(p[3]), [p4] "v"(p[4]),
                   [p5] "v"(p[5]), [a1] "n"(4 * SA), [a2] "n"(32 * SA), [a3] "n"(36 * SA), [b1]
                   "n"(4 * SB), [b2] "n"(32 * SB), [b3] "n"(36 * SB)
                 : "memory");
}

template <int SA, int SB>
__device__ __forceinline__ void read_t(const uint32_t (&p)[8], u32x2a (&o)[32])
{
    asm volatile("ds_read_b64_tr_b16 %[o0], %[p0]\n\t"
                 "ds_read_b64_tr_b16 %[o1], %[p0] offset:%[a1]\n\t"
                 "ds_read_b64_tr_b16 %[o2], %[p0] offset:%[a2]\n\t"
                 "ds_read_b64_tr_b16 %[o3], %[p0] offset:%[a3]\n\t"
                 "ds_read_b64_tr_b16 %[o4], %[p1]\n\t"
                 "ds_read_b64_tr_b16 %[o5], %[p1] offset:%[a1]\n\t"
                 "ds_read_b64_tr_b16 %[o6], %[p1] offset:%[a2]\n\t"
                 "ds_read_b64_tr_b16 %[o7], %[p1] offset:%[a3]\n\t"
                 "ds_read_b64_tr_b16 %[o8], %[p2]\n\t"
                 "ds_read_b64_tr_b16 %[o9], %[p2] offset:%[a1]\n\t"
                 "ds_read_b64_tr_b16 %[o10], %[p2] offset:%[a2]\n\t"
                 "ds_read_b64_tr_b16 %[o11], %[p2] offset:%[a3]\n\t"
                 "ds_read_b64_tr_b16 %[o12], %[p3]\n\t"
                 "ds_read_b64_tr_b16 %[o13], %[p3] offset:%[a1]\n\t"
                 "ds_read_b64_tr_b16 %[o14], %[p3] offset:%[a2]\n\t"
                 "ds_read_b64_tr_b16 %[o15], %[p3] offset:%[a3]\n\t"
                 "ds_read_b64_tr_b16 %[o16], %[p4]\n\t"
                 "ds_read_b64_tr_b16 %[o17], %[p4] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o18], %[p4] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o19], %[p4] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o20], %[p5]\n\t"
                 "ds_read_b64_tr_b16 %[o21], %[p5] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o22], %[p5] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o23], %[p5] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o24], %[p6]\n\t"
                 "ds_read_b64_tr_b16 %[o25], %[p6] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o26], %[p6] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o27], %[p6] offset:%[b3]\n\t"
                 "ds_read_b64_tr_b16 %[o28], %[p7]\n\t"
                 "ds_read_b64_tr_b16 %[o29], %[p7] offset:%[b1]\n\t"
                 "ds_read_b64_tr_b16 %[o30], %[p7] offset:%[b2]\n\t"
                 "ds_read_b64_tr_b16 %[o31], %[p7] offset:%[b3]\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : [o0] "=&v"(o[0]), [o1] "=&v"(o[1]), [o2] "=&v"(o[2]), [o3] "=&v"(o[3]), [o4]
                   "=&v"(o[4]), [o5] "=&v"(o[5]), [o6] "=&v"(o[6]), [o7] "=&v"(o[7]), [o8]
                   "=&v"(o[8]), [o9] "=&v"(o[9]), [o10] "=&v"(o[10]), [o11] "=&v"(o[11]), [o12]
                   "=&v"(o[12]), [o13] "=&v"(o[13]), [o14] "=&v"(o[14]), [o15] "=&v"(o[15]), [o16]
                   "=&v"(o[16]), [o17] "=&v"(o[17]), [o18] "=&v"(o[18]), [o19] "=&v"(o[19]), [o20]
                   "=&v"(o[20]), [o21] "=&v"(o[21]), [o22] "=&v"(o[22]), [o23] "=&v"(o[23]), [o24]
                   "=&v"(o[24]), [o25] "=&v"(o[25]), [o26] "=&v"(o[26]), [o27] "=&v"(o[27]), [o28]
                   "=&v"(o[28]), [o29] "=&v"(o[29]), [o30] "=&v"(o[30]), [o31] "=&v"(o[31])
                 : [p0] "v"(p[0]), [p1] "v"(p[1]), [p2] "v"(p[2]), [p3] "v"(p[3]), [p4] "v"(p[4]),
                   [p5] "v"(p[5]), [p6] "v"(p[6]), [p7] "v"(p[7]), [a1] "n"(4 * SA), [a2] "n"(32 *
                   SA), [a3] "n"(36 * SA), [b1] "n"(4 * SB), [b2] "n"(32 * SB), [b3] "n"(36 * SB)
                 : "memory");
}

__device__ __forceinline__ bf16x8 join(const u32x2a& a, const u32x2a& b)
{
    const u32x4a v = {a[0], a[1], b[0], b[1]};
    return __builtin_bit_cast(bf16x8, v);
}

template <int KIND, bool AK, bool BKM, int SIZE>
__global__ __launch_bounds__(Shape<SIZE>::kThreads, 2) void k_ffn_gemm(const FfnGemms gs)
{
    using S = Shape<SIZE>;
    constexpr int TM = S::TM, H = S::H, MI = S::MI, LA = S::kLoadsA;
    constexpr bool PHASES = S::kPhases;
    constexpr bool DUAL = KIND == kFfnGateUp;
    // two stages of A, and B's halves, as arrays of their own: so the compiler sees that reads of
    // one do not wait for loads to the others
    __shared__ __attribute__((aligned(16))) uint16_t lds_a0[TM * BK], lds_a1[TM * BK];
    __shared__ __attribute__((aligned(16))) uint16_t lds_b00[H * BK], lds_b01[H * BK];
    __shared__ __attribute__((aligned(16))) uint16_t lds_b10[H * BK], lds_b11[H * BK];
    // the weight gradients' two products are one launch
    const bool other = !AK && blockIdx.x >= gs.blocks;
    const FfnGemm& g = gs.g[other];
    Work w;
    if (!decode_work(g, blockIdx.x - (other ? gs.blocks : 0), w)) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = PHASES ? wave >> 1 : wave, wn = PHASES ? wave & 1 : 0;
    const int64_t row0 = int64_t(w.tm) * TM;
    const int64_t col0 = int64_t(w.tn) * (DUAL ? H : 2 * H);   // DUAL: columns of each matrix

    const int stages = g.stages;                      // of one segment of the sum
    const int all = stages * g.segments;
    const int first = static_cast<int>(int64_t(all) * w.split / g.splits);
    const int nk = static_cast<int>(int64_t(all) * (w.split + 1) / g.splits) - first;

    // A stage's tiles: A (TM rows of m), and B's two halves of H columns of n, which are two
    // parts of one matrix, or of the gate's and the up matrix. Their sources move on stage
    // by stage in scalar registers; past the last stage they are ranges of no bytes.
    uint32_t off_a[LA], off_b[2];
    lane_offsets<AK, TM>(wave, lane, g.lda, off_a);
    lane_offsets<BKM, H>(wave, lane, g.ldb, off_b);
    int klim[2];   // K-major: load j has nothing for this lane at stages from k = klim[j & 1] on
#pragma unroll
    for (int j = 0; j < 2; ++j)
        klim[j] = static_cast<int>(g.kpad) - 8 * ((lane & 7) ^ chunk_key(8 * j + (lane >> 3)));
    const int lda = static_cast<int>(g.lda), ldb = static_cast<int>(g.ldb);
    const int klen = static_cast<int>(g.K), kend = stages * BK;
    const int a_rows = static_cast<int>(min(int64_t(TM), g.M - row0));
    int b_rows[2], b_col[2];
    const uint16_t *a_next, *b_next[2];               // where the second segment starts
    struct Source {
        const uint16_t* p;
        int k0, left;                                 // left: stages still to be loaded
    } at_a, at_b[2];
    const bool second = first >= stages;
    const int start = (first - (second ? stages : 0)) * BK;
    {
        const int64_t skip = AK ? row0 * g.lda : row0;
        a_next = g.a[1] + skip;
        at_a.p = (second ? g.a[1] : g.a[g.segments > 1 ? 0 : w.batch]) + skip +
                 (AK ? start : start * g.lda);
        at_a.k0 = start;
        at_a.left = nk;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t col = DUAL ? col0 : col0 + h * H;
        const int64_t skip = BKM ? col * g.ldb : col;
        b_next[h] = g.b[1] + skip;
        at_b[h].p = g.b[DUAL ? h : second] + skip + (BKM ? start : start * g.ldb);
        at_b[h].k0 = start;
        at_b[h].left = nk;
        b_rows[h] = static_cast<int>(max(int64_t(0), min(int64_t(H), g.N - col)));
        b_col[h] = static_cast<int>(col);
    }
    auto resource = [](const uint16_t* p, int bytes) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), 0, bytes, 0x00020000);
    };
    auto load_piece = [](__amdgpu_buffer_rsrc_t r, uint16_t* dst, uint32_t off) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)dst, 16, off, 0, 0, 0);
    };
    auto advance = [&](Source& at, const uint16_t* next, int64_t step) {
        --at.left;
        at.k0 += BK;
        at.p += step;
        if (at.k0 == kend) {
            at.k0 = 0;
            at.p = next;
        }
    };
    struct Tiles {
        uint16_t *a, *b[2];
    };
    const Tiles t0 = {lds_a0, {lds_b00, lds_b01}}, t1 = {lds_a1, {lds_b10, lds_b11}};
    auto load_a = [&](const Tiles& t) {               // LA loads
        const int n = AK ? a_rows * lda - at_a.k0
                         : min(BK, klen - at_a.k0) * lda - static_cast<int>(row0);
#pragma unroll
        for (int j = 0; j < LA; ++j)
            load_piece(resource(at_a.p, at_a.left > 0 ? 2 * n : 0), t.a + (wave * LA + j) * 512,
                       AK && at_a.k0 >= klim[j & 1] ? kOut : off_a[j]);
        advance(at_a, a_next, AK ? BK : int64_t(BK) * g.lda);
    };
    auto load_b = [&](const Tiles& t, int h) {        // two
        Source& at = at_b[h];
        const int n = BKM ? b_rows[h] * ldb - at.k0 : min(BK, klen - at.k0) * ldb - b_col[h];
#pragma unroll
        for (int j = 0; j < 2; ++j)
            load_piece(resource(at.p, at.left > 0 && n > 0 ? 2 * n : 0),
                       t.b[h] + (wave * 2 + j) * 512,
                       BKM && at.k0 >= klim[j] ? kOut : off_b[j]);
        advance(at, b_next[h], BKM ? BK : int64_t(BK) * g.ldb);
    };

    // Fragments of two 32-deep steps: lane l holds row l % 16, k = 8 (l / 16) .. + 7.
    const int q = lane >> 4, l16 = lane & 15;
    bf16x8 fa[2][MI], fb[2][NJ];
    auto frag_k = [&](const uint16_t* t, int row, int ks) -> bf16x8 {
        const int chunk = (4 * ks + q) ^ chunk_key(l16);
        return *reinterpret_cast<const bf16x8*>(t + (row + l16) * BK + chunk * 8);
    };
    // Rows of k: byte address of the lane's 8 bytes of the first four rows.
    const int trow = 8 * q + (l16 >> 2);
    auto addr_t = [&](const uint16_t* t, auto width, int col) -> uint32_t {
        constexpr int wide = decltype(width)::value;
        const int piece = (col >> 4) ^ piece_key<wide>(trow);
        return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(
                   (lds_u16*)(t + trow * wide + piece * 16 + (lane & 3) * 4)));
    };
    typedef std::integral_constant<int, TM> WideA;
    typedef std::integral_constant<int, H> WideB;
    // All of A's with B's first half, or B's second half.
    auto frags = [&](const Tiles& t, auto part) {
        constexpr int h = decltype(part)::value;
        constexpr int NA = AK || h ? 0 : MI;
        const uint16_t* sb = t.b[h];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            if constexpr (AK && h == 0) {
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) fa[ks][mi] = frag_k(t.a, (wm * MI + mi) * 16, ks);
            }
            if constexpr (BKM) {
#pragma unroll
                for (int j = 0; j < NJ; ++j) fb[ks][j] = frag_k(sb, wn * 64 + j * 16, ks);
            }
        }
        if constexpr (!BKM) {   // rows of k: B, and A with it
            uint32_t at[NA + NJ];
            u32x2a o[4 * (NA + NJ)];
#pragma unroll
            for (int i = 0; i < NA + NJ; ++i)
                at[i] = i < NA ? addr_t(t.a, WideA{}, (wm * MI + i) * 16)
                               : addr_t(sb, WideB{}, wn * 64 + (i - NA) * 16);
            read_t<2 * TM, 2 * H>(at, o);
#pragma unroll
            for (int i = 0; i < NA + NJ; ++i)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    const bf16x8 f = join(o[4 * i + 2 * ks], o[4 * i + 2 * ks + 1]);
                    if (i < NA) fa[ks][i] = f;
                    else fb[ks][i - NA] = f;
                }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    static_assert(AK || !BKM, "an A of rows of k goes with such a B");
    f32x4 acc[MI][2][NJ];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[mi][h][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto mfmas = [&](auto part) {
        constexpr int h = decltype(part)::value;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    acc[mi][h][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        fb[ks][j], fa[ks][mi], acc[mi][h][j], 0, 0, 0);
    };
    auto barrier = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    // This wave's LDS reads are done, and all but its newest loads, two parts' worth: A and B's
    // first half, and B's second half.
    auto settled = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0070 | (LA + 4));
    };
    // A stage is two parts, by B's halves; A's fragments stay for the second. A part is two
    // phases: its fragments out of LDS and loads for a later part; then the matrix-core ops.
    // With eight waves, two to a SIMD, a barrier follows each phase and the second four run one
    // phase behind the first: each SIMD's matrix core works for one wave while the other reads.
    // Three parts' loads are in flight: A and B's first half of the stage after next go out in
    // the second part, into this stage's buffer, where all waves have read them before the last
    // barrier; B's second half in the next stage's first part. A part's loads have settled in
    // every wave before the barrier that its first readers pass.
    auto part = [&](auto which, const Tiles& cur, const Tiles& to) {
        constexpr int h = decltype(which)::value;
        if constexpr (!PHASES) {
            settled();
            barrier();
        }
        frags(cur, which);
        if constexpr (h == 0) {
            load_b(to, 1);
        } else {
            load_a(to);
            load_b(to, 0);
        }
        if constexpr (PHASES) {
            settled();
            barrier();
            __builtin_amdgcn_s_setprio(1);
        }
        mfmas(which);
        if constexpr (PHASES) {
            __builtin_amdgcn_s_setprio(0);
            barrier();
        }
    };
    typedef std::integral_constant<int, 0> First;
    typedef std::integral_constant<int, 1> Second;
    if (nk > 0) {
        load_a(t0);
        load_b(t0, 0);
        load_b(t0, 1);
        load_a(t1);
        load_b(t1, 0);
        if constexpr (PHASES) {
            settled();
            barrier();
            if (wave >= 4) barrier();
        }
        for (int it = 0; it < nk; it += 2) {
            part(First{}, t0, t1);
            part(Second{}, t0, t0);
            part(First{}, t1, t0);
            part(Second{}, t1, t1);
        }
        if (PHASES && wave < 4) barrier();
    }

    // ------------------------------------------------------------------ epilogues
    // Tiles that lie wholly inside take a path without bounds.
    auto gate_up = [&](auto whole, auto act) {
        constexpr bool FULL = decltype(whole)::value;
        constexpr int ACT = decltype(act)::value;
        const int64_t c = col0 + wn * 64 + 16 * q;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            const int64_t row = row0 + (wm * MI + mi) * 16 + l16;
            const bool on = FULL || row < g.M;
            float gv[16], uv[16];
            to_run(acc[mi][0], gv);
            to_run(acc[mi][1], uv);
            if (!FULL && c + 16 > g.N) {   // (an infinity in x makes NaN of the zeros there)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (c + i >= g.N) gv[i] = uv[i] = 0.0f;
            }
            if (g.gcodes) {
                write_codes<FULL>(gv, c, g.N, q, g.gcodes + row * g.N, g.gexps + row * g.groups,
                                  on);
                write_codes<FULL>(uv, c, g.N, q, g.ucodes + row * g.N, g.uexps + row * g.groups,
                                  on);
            }
            if (!on) continue;
            float none;
#pragma unroll
            for (int i = 0; i < 16; ++i) gv[i] = activation<ACT, false>(gv[i], none) * uv[i];
            // columns from N to ldo are read by the next product as zeros
            store_run<FULL>(g.o[0] + row * g.ldo, c, g.ldo, gv);
        }
    };
    auto gate_grad = [&](auto whole, auto act) {
        constexpr bool FULL = decltype(whole)::value;
        constexpr int ACT = decltype(act)::value;
        // the next rows' codes are loaded while these are worked on
        u32x4a gw[2][2], uw[2][2];
        uint32_t ge[2][2], ue[2][2];
        auto fetch = [&](int mi) {
            const int64_t row = row0 + (wm * MI + mi) * 16 + l16;
            const int s = mi & 1;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t c = col0 + h * H + wn * 64 + 16 * q;
                gw[s][h] = uw[s][h] = u32x4a{0u, 0u, 0u, 0u};
                ge[s][h] = ue[s][h] = 0;
                if (FULL || (row < g.M && c < g.N)) {
                    gw[s][h] = read_codes<FULL>(g.gcodes + row * g.N, c, g.N);
                    uw[s][h] = read_codes<FULL>(g.ucodes + row * g.N, c, g.N);
                    ge[s][h] = g.gexps[row * g.groups + (c >> 6)];
                    ue[s][h] = g.uexps[row * g.groups + (c >> 6)];
                }
            }
        };
        fetch(0);
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            if (mi + 1 < MI) fetch(mi + 1);
            const int64_t row = row0 + (wm * MI + mi) * 16 + l16;
            const int s = mi & 1;
            if (!FULL && row >= g.M) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t c = col0 + h * H + wn * 64 + 16 * q;
                float v[16], dg[16], av[16];
                to_run(acc[mi][h], v);   // all four lanes of the row take part
                if (!FULL && c >= g.ldo) continue;
                const float gs = act8_scale(ge[s][h]), us = act8_scale(ue[s][h]);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float gv = act8_value(gw[s][h][i >> 2], i & 3) * gs;
                    const float uv = act8_value(uw[s][h][i >> 2], i & 3) * us;
                    float slope;
                    const float a = activation<ACT, true>(gv, slope);
                    av[i] = a * uv;
                    dg[i] = v[i] * uv * slope;
                    v[i] *= a;
                }
                if (!FULL && c + 16 > g.N) {   // columns from N to ldo are read as zeros
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c + i >= g.N) av[i] = dg[i] = v[i] = 0.0f;
                }
                store_run<FULL>(g.o[0] + row * g.ldo, c, g.ldo, dg);
                store_run<FULL>(g.o[1] + row * g.ldo, c, g.ldo, v);
                store_run<FULL>(g.o2 + row * g.ldo, c, g.ldo, av);
            }
        }
    };
    auto plain = [&](auto whole) {
        constexpr bool FULL = decltype(whole)::value;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            const int64_t row = row0 + (wm * MI + mi) * 16 + l16;
            if (!FULL && row >= g.M) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t c = col0 + h * H + wn * 64 + 16 * q;
                float v[16];
                to_run(acc[mi][h], v);
                if (g.partial) {
                    float* __restrict__ p =
                        g.partial + ((int64_t(w.split) * g.batch + w.batch) * g.M + row) * g.N;
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const float* s = v + 8 * b;
                        const float x[8] = {s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7]};
                        store_row8<false>(p, c + 8 * b, FULL ? c + 8 * b + 8 : g.N, x);
                    }
                } else {
                    if (g.col_scale) {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (FULL || c + i < g.N) v[i] *= g.col_scale[c + i];
                    }
                    store_run<FULL>(g.o[w.batch] + row * g.ldo, c, g.N, v);
                }
            }
        }
    };
    typedef std::integral_constant<bool, true> Whole;
    typedef std::integral_constant<bool, false> Edge;
    typedef std::integral_constant<int, kActSilu> Silu;
    typedef std::integral_constant<int, kActGelu> Gelu;
    const bool inside = row0 + TM <= g.M && col0 + (DUAL ? H : 2 * H) <= g.N;
    if constexpr (KIND == kFfnPlain) {
        if (inside) plain(Whole{});
        else plain(Edge{});
    } else if constexpr (KIND == kFfnGateUp) {
        if (inside && g.act == kActSilu) gate_up(Whole{}, Silu{});
        else if (inside) gate_up(Whole{}, Gelu{});
        else if (g.act == kActSilu) gate_up(Edge{}, Silu{});
        else gate_up(Edge{}, Gelu{});
    } else {
        if (inside && g.act == kActSilu) gate_grad(Whole{}, Silu{});
        else if (inside) gate_grad(Whole{}, Gelu{});
        else if (g.act == kActSilu) gate_grad(Edge{}, Silu{});
        else gate_grad(Edge{}, Gelu{});
    }
}

// o[b] = the sum over the splits, in order, of the partial products, times the column factors. The
// partial sums come from the L2 and the last-level cache: 5.6 us for 1000 x 2048.
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

// dst (rows of ldd, a multiple of 8) = src (dense rows of `cols`), zero past them: rows of odd
// widths are copied to 16-byte alignment once, so that the products' loads to LDS are whole. A
// thread takes four vectors of eight, 256 apart in the flat order, all loaded before the first is
// stored. Memory and a launch: 6.7 us a pass for 777 tokens and three weights of 765 x 2047 (21 MB
// read and written).
__global__ __launch_bounds__(256) void k_ffn_pad(const FfnPads p)
{
    const FfnPad& m = p.m[blockIdx.y];
    const int64_t vectors = m.ldd / 8, all = m.rows * vectors;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * 1024; base < all;
         base += static_cast<int64_t>(gridDim.x) * 1024) {
        const int64_t first = base + threadIdx.x;
        int64_t row[4], e[4];
        row[0] = first / vectors;
        e[0] = first - row[0] * vectors;
#pragma unroll
        for (int i = 1; i < 4; ++i) {
            row[i] = row[i - 1];
            e[i] = e[i - 1] + 256;
            while (e[i] >= vectors) {
                e[i] -= vectors;
                ++row[i];
            }
        }
        u32x4a v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = fetch_vector<2>(m.src + row[i] * m.cols, 8 * e[i], row[i] < m.rows ? m.cols : 0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (row[i] < m.rows)
                store16(m.dst + row[i] * m.ldd + 8 * e[i], settle_vector<2>(v[i], 8 * e[i], m.cols));
    }
}

__global__ __launch_bounds__(256) void k_ffn_zero(uint16_t* __restrict__ p, int64_t n)
{
    const int64_t step = 256LL * gridDim.x;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += step) p[i] = 0;
}

template <int KIND, bool AK, bool BKM>
hipError_t launch_kind(const FfnGemm& one, const FfnGemm* two, hipStream_t stream)
{
    auto blocks = [](const FfnGemm& g) {   // whole rounds over the XCDs
        return (int64_t(g.tiles_m) * g.tiles_n * g.batch * g.splits + 7) / 8 * 8;
    };
    FfnGemms g{};
    g.g[0] = one;
    g.blocks = static_cast<uint32_t>(blocks(one));
    if (two) g.g[1] = *two;
    const dim3 grid(g.blocks + static_cast<uint32_t>(two ? blocks(*two) : 0));
    if (one.tile == kFfnTile256)
        hipLaunchKernelGGL((k_ffn_gemm<KIND, AK, BKM, kFfnTile256>), grid,
                           dim3(Shape<kFfnTile256>::kThreads), 0, stream, g);
    else if (one.tile == kFfnTile128)
        hipLaunchKernelGGL((k_ffn_gemm<KIND, AK, BKM, kFfnTile128>), grid,
                           dim3(Shape<kFfnTile128>::kThreads), 0, stream, g);
    else
        hipLaunchKernelGGL((k_ffn_gemm<KIND, AK, BKM, kFfnTile64>), grid,
                           dim3(Shape<kFfnTile64>::kThreads), 0, stream, g);
    return hipGetLastError();
}

}  // namespace

static hipError_t launch_join(const FfnGemm& g, hipStream_t stream)
{
    if (!g.partial) return hipSuccess;
    const int64_t vectors = (g.M * g.N + 7) / 8;
    hipLaunchKernelGGL(k_ffn_join, dim3(static_cast<unsigned>((vectors + 255) / 256), g.batch),
                       dim3(256), 0, stream, g);
    return hipGetLastError();
}

hipError_t launch_ffn_gemm(const FfnGemm& g, hipStream_t stream)
{
    hipError_t err;
    if (g.kind == kFfnGateUp)
        err = launch_kind<kFfnGateUp, true, true>(g, nullptr, stream);
    else if (g.kind == kFfnGateGrad)
        err = launch_kind<kFfnGateGrad, true, false>(g, nullptr, stream);
    else if (g.b_rows_k)
        err = launch_kind<kFfnPlain, true, false>(g, nullptr, stream);
    else
        err = launch_kind<kFfnPlain, true, true>(g, nullptr, stream);
    return err == hipSuccess ? launch_join(g, stream) : err;
}

hipError_t launch_ffn_weight_grads(const FfnGemm& one, const FfnGemm& two, hipStream_t stream)
{
    if (one.tile != two.tile) return hipErrorInvalidValue;
    hipError_t err = launch_kind<kFfnPlain, false, false>(one, &two, stream);
    if (err == hipSuccess) err = launch_join(one, stream);
    return err == hipSuccess ? launch_join(two, stream) : err;
}

hipError_t launch_ffn_pads(const FfnPads& p, hipStream_t stream)
{
    int64_t most = 0;
    for (int i = 0; i < p.n; ++i) {
        const int64_t vectors = p.m[i].rows * (p.m[i].ldd / 8);
        most = vectors > most ? vectors : most;
    }
    if (!most) return hipSuccess;
    const int64_t groups = (most + 1023) / 1024;
    hipLaunchKernelGGL(k_ffn_pad, dim3(static_cast<unsigned>(groups < 65536 ? groups : 65536), p.n),
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
