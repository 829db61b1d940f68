// Products as the entry points launch them, from the host's plan.
#pragma once
#include "abi_checks.h"
#include "ffn_internal.h"

namespace gefen {

// A product over the plan's tile.
inline FfnGemm product(int32_t kind, const FfnTile& t, int64_t M, int64_t N, int64_t K, void* ws,
                int64_t partial)
{
    FfnGemm g{};
    g.kind = kind;
    g.tile = t.tile;
    g.M = M;
    g.N = N;
    g.K = K;
    g.kpad = ffn_up8(K);
    g.segments = g.batch = 1;
    g.stages = t.stages;
    g.tiles_m = static_cast<int32_t>(ffn_ceil(M, ffn_tile_rows(t.tile)));
    g.tiles_n = static_cast<int32_t>(
        ffn_ceil(N, ffn_tile_cols(t.tile) / (kind == kFfnGateUp ? 2 : 1)));
    g.splits = t.splits;
    g.partial = t.splits > 1 ? at<float>(ws, partial) : nullptr;
    return g;
}

// Each launch's threads are fewer than 2^32, as a dispatch has them.
inline int check_launch(const FfnGemm& one, const FfnGemm* two = nullptr)
{
    const int64_t threads = one.tile == kFfnTile256 ? 512 : 256;
    int64_t groups = 0;
    for (const FfnGemm* g : {&one, two}) {
        if (!g) continue;
        groups += ffn_ceil(int64_t(g->tiles_m) * g->tiles_n * g->batch * g->splits, 8) * 8;
        if (g->partial && ffn_ceil(g->M * g->N, 8 * 256) * 256 > 0xffffffffLL)   // the parts' sum
            return fail(GEFEN_EINVAL, "too many elements of a split sum");
    }
    if (groups * threads > 0xffffffffLL) return fail(GEFEN_EINVAL, "too many tiles");
    return GEFEN_OK;
}

// The operand itself, or its padded copy in the workspace, noted in `pads`.
inline const uint16_t* operand(const void* p, int64_t rows, int64_t cols, bool copy, void* ws, int64_t off,
                        FfnPads& pads)
{
    if (!copy) return static_cast<const uint16_t*>(p);
    FfnPad& m = pads.m[pads.n++];
    m.src = static_cast<const uint16_t*>(p);
    m.dst = at<uint16_t>(ws, off);
    m.rows = rows;
    m.cols = cols;
    m.ldd = ffn_up8(cols);
    return m.dst;
}

}  // namespace gefen
