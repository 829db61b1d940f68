// What the plan makes of the output head's sizes given as arguments (tokens width vocabulary ...): one
// line per product, "kind tile splits stages", "few rows waves" (of a group of rows) where the few-token kernel scores
// them, and "ranges n" for the ranges of the backward pass.
#include "token_plan.h"

#include <cstdio>
#include <cstdlib>

using namespace gefen;

static void tile(const char* kind, const FfnTile& t)
{
    const int rows = t.tile == kFfnTile256 ? 256 : t.tile == kFfnTile128 ? 128 : 64;
    std::printf("%s %d %d %d\n", kind, rows, t.splits, t.stages);
}

int main(int argc, char** argv)
{
    for (int i = 1; i + 2 < argc; i += 3) {
        const int64_t T = std::atoll(argv[i]), K = std::atoll(argv[i + 1]), V = std::atoll(argv[i + 2]);
        const bool copy = K % 8;
        const HeadSpace b = head_space(T, K, V, true, copy);
        if (head_few(T, K, V, copy)) {
            const int rows = ffn_token_rows(T);
            std::printf("few %d %d\n", rows,
                        head_groups(K, V) > 1 ? 1 : ffn_token_waves(V, K, rows));
        } else {
            tile("scores", head_space(T, K, V, false, copy).score);
        }
        tile(b.exact ? "gradients2" : "gradients1", b.score);
        tile(b.exact ? "dx2" : "dx1", b.dx);
        tile(b.exact ? "dweight2" : "dweight1", b.dw);
        std::printf("ranges %lld\n", (long long)b.chunks);
    }
    return 0;
}
