// Host-side plans of the operators at a language model's two ends: how work is cut, and where
// what lies between the kernels stands in the caller's workspace. Plain C++ (no HIP), so that it can
// be checked on a host.
#pragma once
#include <algorithm>
#include <cstdint>

#include "ffn_plan.h"

namespace gefen {

// ---------------------------------------------------------------- embedding
// Sorting by digits of at most kSortBits: passes, and the bits of each, for keys 0 .. most.
constexpr int kSortBits = 9;
struct SortPlan {
    int passes;
    int bits[4];
};
inline SortPlan sort_plan(int64_t most)
{
    int all = 1;
    while (most >> all) ++all;
    SortPlan s{};
    s.passes = (all + kSortBits - 1) / kSortBits;
    for (int p = 0, left = all; p < s.passes; ++p) {
        s.bits[p] = (left + s.passes - p - 1) / (s.passes - p);
        left -= s.bits[p];
    }
    return s;
}

// Up to kSortRank tokens are sorted by counting, and each token's run is added up by one workgroup: the
// gradient of 1024 tokens takes 13 us so and 22 by digits and chunks (1000 x 64), 24 and 32 (50257 x
// 768); of 2048 21 and 22, and where all of them are one token 81 and 24 (1024: 43).
constexpr int64_t kSortRank = 1024;

// More tokens than kSortFew are sorted by blocks: the gradient of 16384 takes 48 us by one launch a
// digit and 51 by blocks (128256 x 64), of 65536 114 and 63, of 2^22 7.5 ms and 0.54.
constexpr int64_t kSortFew = 20480;
constexpr int kSortBlock = 4096;
inline int64_t sort_blocks(int64_t n) { return ffn_ceil(n, kSortBlock); }

// Sorted positions are summed in chunks, by a wave each: short ones while the waves are few, longer ones
// so that the sums of their ends, two rows of float32 each, stay a small part of what is read.
inline int64_t embed_chunk(int64_t n) { return n <= 65536 ? 16 : n <= (1 << 19) ? 64 : 256; }
inline int64_t embed_chunks(int64_t n) { return ffn_ceil(n, embed_chunk(n)); }

struct EmbedSpace {
    int64_t keys[2], rows[2], counts, partial, bytes = 0;
};
inline EmbedSpace embed_space(int64_t n, int64_t width)
{
    EmbedSpace s;
    auto take = [&](int64_t bytes) {
        const int64_t at = s.bytes;
        s.bytes += (bytes + 255) / 256 * 256;
        return at;
    };
    for (int i = 0; i < 2; ++i) {
        s.keys[i] = take(4 * n);
        s.rows[i] = take(4 * n);
    }
    s.counts = take(n > kSortFew ? 4 * (sort_blocks(n) + 1) * (1 << kSortBits) : 0);
    s.partial = take(n > kSortRank ? 8 * embed_chunks(n) * width : 0);
    return s;
}

// ---------------------------------------------------------------- log probabilities
constexpr int64_t kScoreMaxTop = 32;
constexpr int64_t kScoreMaxParts = 64;
constexpr int kScoreThreads = 256, kScoreFewThreads = 1024;
constexpr int64_t kScorePart = 1 << 15;   // 16-byte vectors: 512 KiB of a row

// A row is taken by `parts` workgroups, each `per` vectors of 16 bytes of it.
struct ScorePlan {
    int64_t parts = 1;
    int64_t per = 0;
    int threads = kScoreThreads;
};
inline ScorePlan score_plan(int64_t rows, int64_t vocab, bool bf16)
{
    const int64_t vectors = ffn_ceil(vocab, bf16 ? 8 : 4);
    ScorePlan p;
    // Few rows are taken by workgroups of 1024 threads each, and cut into parts only where they are
    // longer than vocabularies are. Rows of 128256 in a graph, microseconds so, and in eight parts (four of
    // 128 rows) of 256 threads with the second launch that joins them:
    //   rows                  1           8           32          128
    //   no alternatives   12.2  7.5   12.5  8.8   12.7  9.6   14.2 14.6
    //   5                 15.8 11.8   16.4 13.5   16.6 14.2   18.2 19.3
    //   20                16.4 15.5   17.1 17.3   17.3 18.1   19.1 23.2
    // But a plain call, which the host bounds, takes 12 to 19 us so, and 15 to 23 with the workspace and
    // second launch.
    if (rows <= 512) p.threads = kScoreFewThreads;
    const int64_t most = std::min(kScoreMaxParts, ffn_ceil(vectors, kScorePart));
    p.parts = std::max<int64_t>(1, std::min(most, 1024 / std::max<int64_t>(rows, 1)));
    p.per = ffn_ceil(vectors, p.parts);
    p.parts = ffn_ceil(vectors, p.per);
    return p;
}

struct ScoreSpace {
    int64_t stats = -1, keys = -1, bytes = 0;
};
inline ScoreSpace score_space(const ScorePlan& p, int64_t rows, int64_t top)
{
    ScoreSpace s;
    if (p.parts > 1) {
        s.keys = 0;
        s.stats = 8 * rows * p.parts * top;
        s.bytes = s.stats + 12 * rows * p.parts;
    }
    return s;
}

// ---------------------------------------------------------------- output head
// Statistics of a row and tile: one for each wave's 128 columns.
inline int64_t head_slots(int32_t tile, int64_t vocab)
{
    return ffn_ceil(vocab, ffn_tile_cols(tile)) * (tile == kFfnTile256 ? 2 : 1);
}

// The scores' gradients exist for a range of the vocabulary at a time, of at most this many bytes
// (or 256 columns), and of rows whose tiles stay within 32-bit offsets.
constexpr int64_t kHeadGradBytes = int64_t(1) << 30;

// Up to this many tokens the scores' gradients are two bfloat16 numbers each, the rounded one and what
// rounding left of it, and the products that read them take both: an output then lies 0.0017 of its norm
// from the formula, as its own rounding alone leaves it, and not 0.0024. The backward pass of 256
// tokens, bound by the weight's bytes more than by the products, takes 741 us so (128256 x 2048) and that
// of 257 688; 50257 x 768 158 and 129. At 8192 tokens it would cost two thirds more.
constexpr int64_t kHeadExactTokens = 256;

// Whether the forward pass takes the few-token kernel, which reads the weight as it lies. Measured, it
// against the tiles, in a graph and on weights that change from call to call (each wave reads all tokens,
// so that more of them take longer): 1 token, 128256 x 2048 92 us and 110; 2 tokens, 50257 x 1280 29 and
// 32; 4 tokens, 128256 x 2048 102 and 109, 200064 x 1536 123 and 119; 8 tokens, 16384 x 8192 70 and 79,
// 32000 x 4096 69 and 62. With groups, below: 1 token, 200000 x 768 58 and 65, 50257 x 768 23 and 23.
// Where the tiles need a copy of the weight: 1 token, 128256 x 401 41 and 68, 50257 x 769 47 and 53; 4
// tokens, 128256 x 1601 249 and 250; 8 tokens, 128256 x 1601 320 and 252; 16 tokens, 128256 x 1001 137 and
// 156, 128256 x 401 61 and 69, 1003 x 509 11 and 15. Rows that begin near a multiple of 512 bytes apart are
// slower than others: 8 tokens, 50257 x 513 54 and 41, 50257 x 601 40 and 45.
inline bool head_few(int64_t T, int64_t K, int64_t V, bool copy)
{
    if (!copy && K < 1024) return T <= 2 && V >= 65536;
    if (!copy) return T <= (K < 2048 ? 2 : K < 8192 ? 4 : 8);
    if (T <= 2 || V * K < (1 << 24)) return T <= kFfnFewTokens;
    return T <= (K < 1024 ? kFfnFewTokens : 4) && (2 * K + 16) % 512 >= 32;
}

// Groups of rows, of a wave each, to a workgroup of that kernel, where four waves to a group of rows are
// too little work: 1 token, 200000 x 768 58 us and 74, 128256 x 401 41 and 59, 128256 x 1024 50 and 51, x
// 1280 63 and 59; 1003 x 509, which has too few of them, 10.9 and 10.4.
inline int head_groups(int64_t K, int64_t V) { return K < 1024 && V >= 16384 ? 4 : 1; }

struct HeadSpace {
    int64_t x = -1, w = -1;            // padded copies
    int64_t stats = -1, taken = -1;    // forward
    int64_t slots = 0;
    int64_t dz = -1, partial = -1;     // backward
    int64_t bytes = 0;
    int64_t columns = 0, chunks = 1;   // of the vocabulary, in the backward pass
    int64_t ldz = 0;
    bool exact = false;
    int64_t planes_x = 0;              // float32 sums of dx
    int64_t partial_w = 0;             // where dweight's parts begin behind them
    FfnTile score, dx, dw;
};

// copy: the operands' rows are no multiple of 8, or not aligned.
inline HeadSpace head_space(int64_t T, int64_t K, int64_t V, bool backward, bool copy)
{
    HeadSpace s;
    auto take = [&](int64_t bytes) {
        const int64_t at = s.bytes;
        s.bytes += (bytes + 255) / 256 * 256;
        return at;
    };
    const int64_t K8 = ffn_up8(K);
    if (!backward && head_few(T, K, V, copy)) {   // a slot for each workgroup of the few-token kernel
        s.slots = ffn_ceil(V, ffn_token_rows(T) * head_groups(K, V));
        s.stats = take(12 * T * s.slots);
        s.taken = take(4 * T);
        return s;
    }
    if (copy) {
        s.x = take(2 * T * K8);
        s.w = take(2 * V * K8);
    }
    if (!backward) {
        const FfnResult z = {T, V, 1};
        s.score = ffn_choose(&z, 1, K, 1, false, false, kFfnActivate);
        s.slots = head_slots(s.score.tile, V);
        s.stats = take(12 * T * s.slots);
        s.taken = take(4 * T);
        return s;
    }
    const int64_t most = std::min(
        kFfnMaxWidth, std::max<int64_t>(256, kHeadGradBytes / (2 * T) / 256 * 256));
    s.columns = V;
    if (V > most) {
        s.columns = ffn_ceil(ffn_ceil(V, ffn_ceil(V, most)), 256) * 256;
        s.chunks = ffn_ceil(V, s.columns);
    }
    s.ldz = ffn_up8(s.columns);
    s.exact = T <= kHeadExactTokens;
    const int halves = s.exact ? 2 : 1;
    s.dz = take(2 * halves * T * s.ldz);
    const FfnResult z = {T, s.columns, 1}, dx = {halves * T, K, 1}, dw = {s.columns, K, 1};
    s.score = ffn_choose(&z, 1, K, 1, false, false, kFfnActivate);
    s.dx = ffn_choose(&dx, 1, s.columns, 1, false, true, kFfnStore);
    s.dw = ffn_choose(&dw, 1, T, halves, false, true, kFfnStore);
    // dx of the halves, and of ranges, is summed in float32
    s.planes_x = s.chunks > 1 || s.exact || s.dx.splits > 1 ? halves * s.dx.splits : 0;
    s.partial_w = 4 * T * K * s.planes_x;
    const int64_t partial = s.partial_w + ffn_partial_bytes(s.dw, s.columns, K, 1);
    if (partial) s.partial = take(partial);
    return s;
}

}  // namespace gefen
