// Feed-forward operators: what the ABI (ffn_abi.hip) and the kernels (act8.hip, ffn_gemm.hip,
// ffn_tokens.hip) share.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "ffn_plan.h"

namespace gefen {

// ---------------------------------------------------------------- 8-bit activation checkpoints
// A row of `cols` values is cut into groups of kAct8Group, the last one shorter. A group's scale
// is 2^(E - 127), E one byte: the smallest from 1 on for which rint(|x| / scale) <= 127
// throughout, at most kAct8Top; E = 255 marks a group that holds an infinity or NaN, which stands
// for NaN throughout. Codes are rint(x / scale), ties to even, within +-127, one signed byte each.
constexpr int kAct8Group = 64;
constexpr int kAct8Top = 248;

inline int64_t act8_groups(int64_t cols) { return (cols + kAct8Group - 1) / kAct8Group; }

hipError_t launch_act8_encode(const void* x, bool bf16, int64_t rows, int64_t cols, int8_t* codes,
                              uint8_t* exps, hipStream_t stream);
// out (rows of ldo >= cols elements; columns cols .. ldo - 1 are set to zero) = the values, times
// gain[column] where gain is given.
hipError_t launch_act8_decode(const int8_t* codes, const uint8_t* exps, const float* gain,
                              int64_t rows, int64_t cols, void* out, bool bf16, int64_t ldo,
                              hipStream_t stream);

// ---------------------------------------------------------------- RMS norm
constexpr int64_t kNormMaxCols = 16384;

struct NormArgs {
    const void* x;
    const void* r;          // residual, or null
    const float* weight;
    int64_t rows, cols;
    double eps;
    void* y;
    void* h;                // x + r, or null
    float* rstd;
    int8_t* codes;          // of h * rstd, or null
    uint8_t* exps;
};
hipError_t launch_rms_norm(const NormArgs& a, bool bf16, hipStream_t stream);

struct NormGradArgs {
    const void* dy;
    const void* dh;         // gradient of h, or null
    const void* h;          // the normalised rows' input, or null: codes
    const int8_t* codes;
    const uint8_t* exps;
    const float* rstd;
    const float* weight;
    int64_t rows, cols;
    void* dx;
    float* dw;
    float* partial;         // norm_grad_parts(rows, cols) rows of cols
};
int64_t norm_grad_parts(int64_t rows, int64_t cols);
hipError_t launch_rms_norm_grad(const NormGradArgs& a, bool bf16, hipStream_t stream);

// ---------------------------------------------------------------- gated feed-forward block
enum : int32_t { kActSilu = 0, kActGelu = 1 };
enum : int32_t { kFfnGateUp = 0, kFfnPlain = 1, kFfnGateGrad = 2, kHeadStats = 3, kHeadGrad = 4 };

// The output head's products: what their epilogues read and write beside the sums (token_device.h
// gives the formulas).
struct HeadRows {
    const void* tokens;          // of the rows
    bool wide;                   // 64-bit ones
    int64_t first;               // the vocabulary entry of column 0
    int64_t vocab;               // of all
    float* stats;                // [head_slots][3][M]
    float* taken;                // [M]: the tokens' scores
    const float* lse;
    const float* entropy;
    const float* dlogprob;
    const float* dentropy;       // or null
};

// One product (ffn_gemm.hip). Leading dimensions are multiples of 8 and operands 16-byte
// aligned; an operand with rows of m or n is zero in its columns K .. kpad - 1.
struct FfnGemm {
    int32_t kind;
    int32_t act;
    int32_t tile;                // kFfnTile*
    bool b_rows_k;               // B is stored as rows of k (with A in the weight gradients)
    const uint16_t* a[2];        // by segment of the sum, or by batch entry
    const uint16_t* b[2];        // by segment of the sum, or gate and up
    int64_t lda, ldb;
    int64_t M, N, K, kpad;       // kpad: K rounded up to 8
    int32_t segments, batch;     // not both above 1
    int32_t stages;              // of 64 k, per segment
    int32_t tiles_m, tiles_n;
    int32_t splits;              // of all stages; above 1 only with `partial`
    float* partial;              // [splits][batch][M][N] float32, or null
    uint16_t* o[2];              // by batch entry; the gate's and up's gradients
    uint16_t* o2;                // act(G) U again (gate gradients)
    int64_t ldo;
    const float* col_scale;      // or null
    int8_t* gcodes;              // checkpoints of G and U, dense rows of N (or null)
    int8_t* ucodes;
    uint8_t* gexps;
    uint8_t* uexps;
    int64_t groups;              // exponents per row
    bool add;                    // to what `partial` holds
    HeadRows head;
};
struct FfnGemms {
    FfnGemm g[2];
    uint32_t blocks;             // workgroups of the first
};
hipError_t launch_ffn_gemm(const FfnGemm& g, hipStream_t stream);
// The same without the join of its parts, and the join alone.
hipError_t launch_ffn_parts(const FfnGemm& g, hipStream_t stream);
hipError_t launch_ffn_join(const FfnGemm& g, hipStream_t stream);
// One plain product whose operands are both stored as rows of k.
hipError_t launch_ffn_weight_grad(const FfnGemm& g, hipStream_t stream);
// Two plain products whose operands are both stored as rows of k, of one tile size.
hipError_t launch_ffn_weight_grads(const FfnGemm& one, const FfnGemm& two, hipStream_t stream);

// One forward product of a few tokens (ffn_tokens.hip): o[t][n] = sum_k x[t][k] w[n][k] over
// dense rows of K, or act(G) U of two such products where w[1] is given.
struct FfnTokens {
    const uint16_t* x;
    int64_t ldx;
    const uint16_t* w[2];
    int64_t tokens, N, K;
    int32_t act;
    uint16_t* o;
    int64_t ldo;
    HeadRows head;               // launch_head_tokens alone, which writes no o
};
hipError_t launch_ffn_tokens(const FfnTokens& g, hipStream_t stream);
hipError_t launch_head_tokens(const FfnTokens& g, int groups, hipStream_t stream);

struct FfnPad {
    const uint16_t* src;
    uint16_t* dst;
    int64_t rows, cols, ldd;
};
struct FfnPads {
    FfnPad m[5];
    int32_t n;
};
hipError_t launch_ffn_pads(const FfnPads& p, hipStream_t stream);
hipError_t launch_zero_bf16(uint16_t* p, int64_t n, hipStream_t stream);

}  // namespace gefen
