// What the plan makes of sizes given as arguments (tokens width inner ...): one line per product,
// "kind tile splits stages", and per few-token product "kind rows waves".
#include "ffn_plan.h"

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
        const int64_t T = std::atoll(argv[i]), K = std::atoll(argv[i + 1]), F = std::atoll(argv[i + 2]);
        const FfnSpace f = ffn_space(T, K, F, false, K % 8, F % 8);
        const FfnSpace b = ffn_space(T, K, F, true, K % 8, F % 8);
        tile("gate_up", f.gate_up);
        tile("down", f.down);
        tile("gate_grad", b.grad_inner);
        tile("dx", b.dx);
        tile("dw", b.dw);
        if (T <= kFfnFewTokens) {
            const int rows = ffn_token_rows(T);
            std::printf("few_gate_up %d %d\n", rows, ffn_token_waves(F, K, rows));
            std::printf("few_down %d %d\n", rows, ffn_token_waves(K, F, rows));
        }
    }
    return 0;
}
