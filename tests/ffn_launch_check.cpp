// Checks of ffn_plan.h's launches on a host: every vector of every row is some lane's, and no
// launch has 2^32 threads or more along an axis, which the device's dispatch does not take.
#include "ffn_plan.h"

#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

using namespace gefen;

static void need(bool ok, const char* what, int64_t rows, int64_t vectors)
{
    if (ok) return;
    std::printf("FAILED: %s (%lld rows of %lld vectors)\n", what, (long long)rows,
                (long long)vectors);
    std::exit(1);
}

static void check_row_grid(int64_t rows, int64_t vectors)
{
    const RowGrid g = row_grid(rows, vectors);
    need(g.lx >= 3 && g.lx <= 8, "lanes along a row", rows, vectors);
    need(g.most >= 1 && g.most <= g.gx && g.gy >= 1 && g.gy <= 65535, "workgroups", rows, vectors);
    need((g.gx << g.lx) >= vectors && ((g.gx - 1) << g.lx) < vectors, "a row", rows, vectors);
    need(g.most * 256 < (int64_t(1) << 32), "threads along a row", rows, vectors);
}

// The kernels' walk, lane by lane, over launches that are small enough to follow.
static void check_walk(int64_t rows, int64_t vectors, const RowGrid& g)
{
    std::vector<int> seen(static_cast<size_t>(rows * vectors), 0);
    for (int64_t first = 0; first < g.gx; first += g.most)
        for (int64_t by = 0; by < g.gy; ++by)
            for (int64_t bx = 0; bx < std::min(g.most, g.gx - first); ++bx)
                for (int t = 0; t < 256; ++t) {
                    const int64_t v = ((first + bx) << g.lx) + (t & ((1 << g.lx) - 1));
                    if (v >= vectors) continue;   // past the row nothing is stored
                    for (int64_t r = (by << (8 - g.lx)) + (t >> g.lx); r < rows;
                         r += g.gy << (8 - g.lx))
                        ++seen[static_cast<size_t>(r * vectors + v)];
                }
    for (int n : seen) need(n == 1, "a vector is one lane's", rows, vectors);
}

int main()
{
    std::mt19937_64 rng(1);
    auto size = [&](double hi) {
        std::uniform_real_distribution<double> u(0.0, hi);
        return std::max<int64_t>(1, int64_t(std::exp2(u(rng))));
    };
    // up to 2^40 elements, whole groups (eight vectors) along a row
    for (int i = 0; i < 20000; ++i) {
        const int64_t groups = size(34.0);
        check_row_grid(size(std::log2(double(int64_t(1) << 34) / double(groups)) + 0.5), groups * 8);
    }
    for (int64_t log2 = 20; log2 <= 34; ++log2)
        for (int64_t d = -1; d <= 1; ++d) check_row_grid(1, ((int64_t(1) << log2) + d) * 8);
    for (int64_t rows : {1, 3, 33, 100})
        for (int64_t groups : {1, 2, 5, 40, 200}) {
            RowGrid g = row_grid(rows, groups * 8);
            check_walk(rows, groups * 8, g);
            g.most = std::min<int64_t>(g.gx, 3);          // in more than one launch
            g.gy = 1;
            check_walk(rows, groups * 8, g);
        }
    std::printf("ok\n");
    return 0;
}
