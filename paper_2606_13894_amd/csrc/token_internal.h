// The operators at a language model's two ends: what the ABI (token_abi.hip) and the kernels
// (embedding.hip, dropout.hip, logprobs.hip; the head's products in ffn_gemm.hip) share.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "ffn_internal.h"
#include "token_plan.h"

namespace gefen {

// Tokens are 32- or 64-bit (wide). One below 0 stands for none: no row, no loss.
struct Tokens {
    const void* p;
    bool wide;
};

// ---------------------------------------------------------------- embedding
struct EmbedArgs {
    Tokens tokens;
    const void* table;
    int64_t n, vocab, width;
    float scale;
    void* y;
};
hipError_t launch_embedding(const EmbedArgs& a, bool table_bf16, bool y_bf16, hipStream_t stream);

struct EmbedGradArgs {
    Tokens tokens;
    const void* dy;
    int64_t n, vocab, width;
    float scale;
    void* dtable;
    uint32_t* keys[2];       // n each: the tokens, sorted in turns
    uint32_t* rows[2];       // n each: where they stood
    uint32_t* counts;        // the sort's by blocks (embed_space)
    float* partial;          // 2 embed_chunks(n) rows of `width`
};
hipError_t launch_embedding_grad(const EmbedGradArgs& a, bool dy_bf16, bool table_bf16,
                                 hipStream_t stream);

// ---------------------------------------------------------------- dropout
struct DropoutArgs {
    const void* x;
    const void* residual;    // or null
    void* y;
    int64_t n;
    uint32_t least;          // pieces below it are dropped; 65536 drops everything
    float scale;
    uint64_t seed, offset;
    const int64_t* state;    // device: seed, and what is added to offset; or null
};
hipError_t launch_dropout(const DropoutArgs& a, bool bf16, hipStream_t stream);

// ---------------------------------------------------------------- log probabilities
struct ScoreArgs {
    const void* z;
    int64_t ld;              // elements between rows
    Tokens tokens;
    int64_t rows, vocab;
    int32_t top;
    ScorePlan plan;
    float* logprob;
    float* entropy;
    float* lse;
    float* rest;             // what rounding left of lse; or null
    float* top_logprob;      // rows x top
    int64_t* top_token;
    float* stats;            // rows x parts x 3, where there are parts
    uint64_t* keys;          // rows x parts x top
};
hipError_t launch_scores(const ScoreArgs& a, bool bf16, hipStream_t stream);

struct ScoreGradArgs {
    const void* z;
    int64_t ld;
    Tokens tokens;
    int64_t rows, vocab;
    const float* lse;
    const float* rest;       // or null (0)
    const float* entropy;
    const float* dlogprob;
    const float* dentropy;   // or null
    void* dz;                // may be z
    int64_t ldd;
};
hipError_t launch_score_grad(const ScoreGradArgs& a, bool bf16, hipStream_t stream);

// The head's rows from the statistics of its tiles or workgroups: `slots` of them, each three numbers
// (HeadRows::stats), which lie [slots][3][rows], or by rows: [rows][3][slots].
struct HeadJoinArgs {
    const float* stats;
    bool by_rows;
    const float* taken;
    Tokens tokens;
    int64_t rows, vocab, slots;
    float* logprob;
    float* entropy;
    float* lse;
};
hipError_t launch_head_join(const HeadJoinArgs& a, hipStream_t stream);

}  // namespace gefen
