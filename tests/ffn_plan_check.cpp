// Checks of ffn_plan.h on a host: tiles cover the product, splits leave every part stages to
// sum, the workspace's regions do not overlap and hold what is put there.
#include "ffn_plan.h"

#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

using namespace gefen;

static void need(bool ok, const char* what, int64_t a, int64_t b, int64_t c)
{
    if (ok) return;
    std::printf("FAILED: %s (%lld, %lld, %lld)\n", what, (long long)a, (long long)b, (long long)c);
    std::exit(1);
}

static void check_tile(const FfnTile& t, int64_t M, int64_t N, int64_t K, int segments,
                       bool may_split)
{
    need(t.tile == kFfnTile64 || t.tile == kFfnTile128 || t.tile == kFfnTile256, "tile", M, N, K);
    need(int64_t(t.stages) * kFfnDepth >= K && (t.stages - 1) * int64_t(kFfnDepth) < K, "stages", M,
         N, K);
    need(t.splits >= 1 && (may_split || t.splits == 1), "splits", M, N, K);
    need(t.splits == 1 || int64_t(t.stages) * segments / t.splits >= 4, "a short part", M, N, K);
}

struct Region {
    int64_t at, bytes;
};

static void check_space(int64_t T, int64_t K, int64_t F, bool backward, bool unaligned)
{
    const bool ck = unaligned || K % 8, cf = unaligned || F % 8;
    const FfnSpace s = ffn_space(T, K, F, backward, ck, cf);
    const int64_t K8 = ffn_up8(K), F8 = ffn_up8(F);
    std::vector<Region> r;
    auto add = [&](int64_t at, int64_t bytes, bool wanted) {
        need(wanted == (at >= 0), "a region that is wanted is there", T, K, F);
        if (at < 0) return;
        need(at % 256 == 0 && at + bytes <= s.bytes, "a region's place", T, K, F);
        r.push_back({at, bytes});
    };
    add(s.x, 2 * T * K8, backward || ck);
    add(s.dy, 2 * T * K8, backward && ck);
    add(s.w_gate, 2 * F * K8, ck);
    add(s.w_up, 2 * F * K8, ck);
    add(s.w_down, 2 * K * F8, cf);
    add(s.a, 2 * T * F8, true);
    add(s.dg, 2 * T * F8, backward);
    add(s.du, 2 * T * F8, backward);
    int64_t partial = 0;
    if (!backward) {
        check_tile(s.gate_up, T, F, K, 1, false);
        check_tile(s.down, T, K, F, 1, true);
        partial = ffn_partial_bytes(s.down, T, K, 1);
    } else {
        check_tile(s.grad_inner, T, F, K, 1, false);
        check_tile(s.dx, T, K, F, 2, true);
        check_tile(s.dw, K, F, T, 1, true);
        // the two weight gradients' parts are live together
        partial = ffn_partial_bytes(s.dx, T, K, 1);
        const int64_t both = ffn_partial_bytes(s.dw, K, F, 1) + ffn_partial_bytes(s.dw, F, K, 2);
        partial = both > partial ? both : partial;
    }
    add(s.partial, partial, partial > 0);
    for (size_t i = 0; i < r.size(); ++i)
        for (size_t j = 0; j < i; ++j)
            need(r[i].at >= r[j].at + r[j].bytes || r[j].at >= r[i].at + r[i].bytes, "overlap", T, K,
                 F);
}

int main()
{
    std::mt19937_64 rng(1);
    auto size = [&](int64_t hi) {
        std::uniform_real_distribution<double> u(0.0, std::log2(double(hi)));
        return std::max<int64_t>(1, int64_t(std::exp2(u(rng))));
    };
    for (int i = 0; i < 20000; ++i)
        check_space(size(1 << 17), size(1 << 15), size(1 << 15), i & 1, i & 2);
    for (int64_t t : {1, 63, 64, 65, 127, 128, 129, 255, 256, 257, 8192})
        for (int64_t k : {1, 7, 8, 64, 768, 2048})
            for (int64_t f : {1, 8, 63, 64, 65, 2047, 8192})
                for (int b = 0; b < 4; ++b) check_space(t, k, f, b & 1, b & 2);
    std::printf("ok\n");
    return 0;
}
