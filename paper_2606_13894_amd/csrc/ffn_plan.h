// Host-side plan of the gated feed-forward block's products: which tile, over how many parts of
// the sum, and where the intermediate matrices lie in the caller's workspace. Plain C++ (no
// HIP), so that it can be checked on a host.
#pragma once
#include <algorithm>
#include <cstdint>

namespace gefen {

constexpr int64_t kFfnMaxTokens = int64_t(1) << 24;
constexpr int64_t kFfnMaxWidth = int64_t(1) << 20;   // a tile's rows stay within 32-bit offsets
constexpr int kFfnDepth = 64;                       // k of a stage

// The products' tiles: 64 x 128 (three workgroups to a CU), 128 x 128 (two), 256 x 256 (one).
enum FfnTileSize : int32_t { kFfnTile64 = 0, kFfnTile128 = 1, kFfnTile256 = 2 };
inline int64_t ffn_tile_rows(int32_t size) { return size == kFfnTile256 ? 256 : size == kFfnTile128 ? 128 : 64; }
inline int64_t ffn_tile_cols(int32_t size) { return size == kFfnTile256 ? 256 : 128; }

inline int64_t ffn_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t ffn_up8(int64_t a) { return (a + 7) / 8 * 8; }

struct FfnTile {
    int32_t tile = kFfnTile128;
    int32_t splits = 1;
    int32_t stages = 0;
    double us = 0.0;
};

// What a tile does with its sums, by the time it takes beside the sum itself: a plain store, the
// gate's activation and checkpoints, or the gate's gradients.
enum FfnEpilogue : int { kFfnStore = 0, kFfnActivate = 1, kFfnGradient = 2 };

// Estimated time in microseconds of `groups` workgroups that each sum `stages` stages, and of
// their epilogues, fitted to measurements from 32 to 8192 rows. A stage's time grows with the
// number of workgroups that load at once: from 0.38 us alone to 0.48 with one on every CU and 1.2
// with three for the 64-row tile, 0.5, 0.72 and (with two) 1.2 for the 128-row one, 1.0 to 1.5
// for the largest.
inline double ffn_stage_us(int32_t tile, int64_t groups)
{
    const double cu = double(groups) / 256.0;
    if (tile == kFfnTile256) return 1.0 + 0.5 * cu;
    if (tile == kFfnTile128) return cu <= 1.0 ? 0.5 + 0.22 * cu : 0.72 + 0.48 * (cu - 1.0);
    return cu <= 1.0 ? 0.38 + 0.1 * cu : 0.48 + 0.36 * (cu - 1.0);
}

inline double ffn_sum_us(int32_t tile, int64_t groups, int64_t stages, FfnEpilogue epilogue)
{
    static const double ends[3][3] = {{3.5, 4.0, 7.0}, {5.0, 5.0, 14.0}, {6.0, 9.0, 38.0}};
    const int64_t slots = tile == kFfnTile256 ? 256 : tile == kFfnTile128 ? 512 : 768;
    const int64_t full = groups / slots, rest = groups % slots;
    double us = double(full) * (ffn_stage_us(tile, slots) * double(stages) + ends[tile][epilogue]);
    if (rest) us += ffn_stage_us(tile, rest) * double(stages) + ends[tile][epilogue];
    return us;
}

// One launch's results: C of M x N, `batch` of them.
struct FfnResult {
    int64_t M, N;
    int batch;
};

// The tile and split with the least estimated time for `n` results (one, or two in one launch)
// summed over `segments` of K. `halves`: the tile's columns are two matrices' (gate and up).
// `may_split`: the sum may be cut into parts, whose float32 results are written, and read by a
// second kernel.
inline FfnTile ffn_choose(const FfnResult* r, int n, int64_t K, int segments, bool halves,
                          bool may_split, FfnEpilogue epilogue)
{
    FfnTile best;
    const int64_t stages = ffn_ceil(K, kFfnDepth), all = stages * segments;
    for (int32_t tile : {kFfnTile64, kFfnTile128, kFfnTile256}) {
        const int64_t rows = ffn_tile_rows(tile), cols = ffn_tile_cols(tile) / (halves ? 2 : 1);
        int64_t groups = 0, elems = 0;
        for (int i = 0; i < n; ++i) {
            groups += ffn_ceil(r[i].M, rows) * ffn_ceil(r[i].N, cols) * r[i].batch;
            elems += r[i].M * r[i].N * r[i].batch;
        }
        for (int64_t s : {1, 2, 3, 4, 6, 8, 12, 16}) {
            if (s > 1 && (!may_split || all / s < 4)) break;
            double us = ffn_sum_us(tile, groups * s, ffn_ceil(all, s), epilogue);
            if (s > 1) {
                const double mb = 4e-6 * double(elems) * double(s);
                us += 3.5 * n + mb / 4.0 + mb / 6.0;
            }
            if (best.stages == 0 || us < best.us) {
                best.tile = tile;
                best.splits = static_cast<int32_t>(s);
                best.stages = static_cast<int32_t>(stages);
                best.us = us;
            }
        }
    }
    return best;
}

// ---------------------------------------------------------------- launches
// The few-token products (ffn_tokens.hip): rows of the weights to a workgroup, and its waves, which
// share the sum over k: about sixteen a CU in all, at least 128 k each.
constexpr int64_t kFfnFewTokens = 16;
inline int ffn_token_rows(int64_t tokens) { return tokens <= 8 ? 8 : 16; }
inline int ffn_token_waves(int64_t N, int64_t K, int rows)
{
    const int64_t groups = ffn_ceil(N, rows);
    int waves = 4;
    while (waves < 16 && groups * waves < 4096 && K >= 256 * waves) waves *= 2;
    return waves;
}

// The checkpoint kernels' launches for `rows` rows of `vectors` vectors of eight, a whole number
// of groups: 2^lx lanes along a row by 256 >> lx rows to a workgroup. A dispatch has fewer than
// 2^32 threads along an axis (one row of 2^35 elements would have as many), so that of the gx
// workgroups along a row each launch takes the next `most`. (One launch whose workgroups went on
// along the row took 6 to 15 % longer at 8192 x 8192.) gy workgroups walk down the rows.
struct RowGrid {
    int lx;
    int64_t gx, most, gy;
};
inline RowGrid row_grid(int64_t rows, int64_t vectors)
{
    RowGrid g;
    g.lx = 3;
    while (g.lx < 8 && (int64_t(1) << g.lx) < vectors) ++g.lx;
    g.gx = (vectors + (int64_t(1) << g.lx) - 1) >> g.lx;
    g.most = std::min<int64_t>(g.gx, int64_t(1) << 23);
    g.gy = std::min<int64_t>((rows + (256 >> g.lx) - 1) / (256 >> g.lx), 65535);
    return g;
}

// Byte offsets into the workspace; -1: not needed. T tokens, K the block's width, F its inner
// width; rows of K8 or F8 elements are rounded up to 8 so that 16-byte loads stay aligned.
struct FfnSpace {
    int64_t x = -1, dy = -1, w_gate = -1, w_up = -1, w_down = -1;   // padded copies
    int64_t a = -1, dg = -1, du = -1;                               // T x F8 each
    int64_t partial = -1;
    int64_t bytes = 0;
    FfnTile gate_up, down;                        // forward
    FfnTile grad_inner, dx, dw;                   // backward
};

inline int64_t ffn_partial_bytes(const FfnTile& t, int64_t M, int64_t N, int batch)
{
    return t.splits > 1 ? 4 * M * N * batch * t.splits : 0;
}

// copy_*: the operand's copy is needed (its rows are no multiple of 8, or it is not aligned).
inline FfnSpace ffn_space(int64_t T, int64_t K, int64_t F, bool backward, bool copy_k, bool copy_f)
{
    FfnSpace s;
    auto take = [&](int64_t bytes) {
        const int64_t at = s.bytes;
        s.bytes += (bytes + 255) / 256 * 256;
        return at;
    };
    const int64_t K8 = ffn_up8(K), F8 = ffn_up8(F);
    int64_t partial = 0;
    if (copy_k) {
        if (!backward) s.x = take(2 * T * K8);
        if (backward) s.dy = take(2 * T * K8);
        s.w_gate = take(2 * F * K8);
        s.w_up = take(2 * F * K8);
    }
    if (copy_f) s.w_down = take(2 * K * F8);
    s.a = take(2 * T * F8);
    if (!backward) {
        const FfnResult inner = {T, F, 1}, y = {T, K, 1};
        s.gate_up = ffn_choose(&inner, 1, K, 1, true, false, kFfnActivate);
        s.down = ffn_choose(&y, 1, F, 1, false, true, kFfnStore);
        partial = ffn_partial_bytes(s.down, T, K, 1);
    } else {
        s.x = take(2 * T * K8);   // decoded, or copied
        s.dg = take(2 * T * F8);
        s.du = take(2 * T * F8);
        const FfnResult inner = {T, F, 1}, dx = {T, K, 1}, dw[2] = {{K, F, 1}, {F, K, 2}};
        s.grad_inner = ffn_choose(&inner, 1, K, 1, false, false, kFfnGradient);
        s.dx = ffn_choose(&dx, 1, F, 2, false, true, kFfnStore);
        s.dw = ffn_choose(dw, 2, T, 1, false, true, kFfnStore);
        // the weight gradients' parts lie one after the other
        partial = std::max(ffn_partial_bytes(s.dx, T, K, 1), ffn_partial_bytes(s.dw, K, F, 3));
    }
    if (partial) s.partial = take(partial);
    return s;
}

}  // namespace gefen
