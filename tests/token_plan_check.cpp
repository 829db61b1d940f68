// Checks of token_plan.h on a host: the sort's digits hold every key, each vector of a row and each
// entry of a vocabulary is some workgroup's, and what lies in a workspace lies apart.
#include "token_plan.h"

#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

using namespace gefen;

static void need(bool ok, const char* what, int64_t a, int64_t b, int64_t c)
{
    if (ok) return;
    std::printf("FAILED: %s (%lld %lld %lld)\n", what, (long long)a, (long long)b, (long long)c);
    std::exit(1);
}

static void check_sort(int64_t most)
{
    const SortPlan s = sort_plan(most);
    need(s.passes >= 1 && s.passes <= 4, "passes", most, s.passes, 0);
    int all = 0;
    for (int p = 0; p < s.passes; ++p) {
        need(s.bits[p] >= 1 && s.bits[p] <= kSortBits, "bits", most, p, s.bits[p]);
        all += s.bits[p];
    }
    need(most >> all == 0, "the largest key", most, all, 0);
    // the last pass has a workgroup for each of its digits
    need((most >> (all - s.bits[s.passes - 1])) < (int64_t(1) << s.bits[s.passes - 1]), "last digit",
         most, all, 0);
}

static void check_embed(int64_t n, int64_t width)
{
    const EmbedSpace s = embed_space(n, width);
    const int64_t c = embed_chunk(n), chunks = embed_chunks(n);
    need(chunks * c >= n && (chunks - 1) * c < n, "chunks", n, c, chunks);
    need(c <= 256 && (c & (c - 1)) == 0, "a chunk", n, c, chunks);
    int64_t at = 0;
    for (int i = 0; i < 2; ++i) {
        need(s.keys[i] >= at && s.keys[i] % 16 == 0, "keys", n, width, i);
        need(s.rows[i] >= s.keys[i] + 4 * n && s.rows[i] % 16 == 0, "rows", n, width, i);
        at = s.rows[i] + 4 * n;
    }
    need(s.counts >= at && s.counts % 16 == 0, "counts", n, width, 0);
    if (n > kSortFew) at = s.counts + 4 * (sort_blocks(n) + 1) * (1 << kSortBits);
    need(s.partial >= at && s.partial % 16 == 0, "partial", n, width, 0);
    need(s.bytes >= s.partial + (n > kSortRank ? 8 * chunks * width : 0), "bytes", n, width, s.bytes);
}

static void check_scores(int64_t rows, int64_t vocab, bool bf16, int64_t top)
{
    const ScorePlan p = score_plan(rows, vocab, bf16);
    const int64_t vectors = ffn_ceil(vocab, bf16 ? 8 : 4);
    need(p.parts >= 1 && p.parts <= kScoreMaxParts, "parts", rows, vocab, p.parts);
    need(p.parts * p.per >= vectors && (p.parts - 1) * p.per < vectors, "a row", rows, vocab, p.per);
    need(p.threads == kScoreThreads || p.threads == kScoreFewThreads, "threads", rows, vocab, 0);
    const ScoreSpace s = score_space(p, rows, top);
    need((p.parts > 1) == (s.bytes > 0 && rows > 0) || rows == 0, "space", rows, vocab, s.bytes);
    if (p.parts > 1) {
        need(s.keys % 8 == 0 && s.stats >= s.keys + 8 * rows * p.parts * top, "keys", rows, vocab, top);
        need(s.bytes >= s.stats + 12 * rows * p.parts, "stats", rows, vocab, top);
    }
}

static void check_head(int64_t T, int64_t K, int64_t V, bool copy)
{
    const int64_t K8 = ffn_up8(K);
    const HeadSpace f = head_space(T, K, V, false, copy);
    std::vector<std::pair<int64_t, int64_t>> used;
    auto take = [&](int64_t at, int64_t bytes) {
        if (at < 0) return;
        need(at % 16 == 0, "alignment", T, K, V);
        for (auto& u : used) need(at >= u.first + u.second || at + bytes <= u.first, "apart", T, K, V);
        used.push_back({at, bytes});
    };
    const bool few = head_few(T, K, V, copy);
    need(!few || T <= kFfnFewTokens, "few tokens", T, K, V);
    if (!few) {
        need(copy == (f.x >= 0) && copy == (f.w >= 0), "copies", T, K, V);
        need(f.slots == head_slots(f.score.tile, V) && f.score.splits == 1, "slots", T, K, V);
    } else {
        const int64_t rows = ffn_token_rows(T) * head_groups(K, V);
        need(f.slots * rows >= V && (f.slots - 1) * rows < V, "slots", T, K, V);
    }
    take(f.x, 2 * T * K8);
    take(f.w, 2 * V * K8);
    take(f.stats, 12 * T * f.slots);
    take(f.taken, 4 * T);
    for (auto& u : used) need(u.first + u.second <= f.bytes, "forward bytes", T, K, V);

    const HeadSpace b = head_space(T, K, V, true, copy);
    used.clear();
    take(b.x, 2 * T * K8);
    take(b.w, 2 * V * K8);
    const int halves = b.exact ? 2 : 1;
    take(b.dz, 2 * halves * T * b.ldz);
    const int64_t dw = ffn_partial_bytes(b.dw, b.columns, K, 1);
    need((b.partial >= 0) == (b.planes_x > 0 || dw > 0), "sums", T, K, V);
    if (b.partial >= 0) take(b.partial, b.partial_w + dw);
    need(b.partial_w == 4 * T * K * b.planes_x && b.partial_w % 4 == 0, "dx sums", T, K, V);
    for (auto& u : used) need(u.first + u.second <= b.bytes, "backward bytes", T, K, V);
    need(b.exact == (T <= kHeadExactTokens) && b.score.splits == 1, "numbers", T, K, V);
    need(b.planes_x % halves == 0, "halves", T, K, V);
    // the ranges: whole multiples of what rows of 16 bytes need, all of the vocabulary, none empty
    need(b.columns <= kFfnMaxWidth && b.ldz >= b.columns && b.ldz % 8 == 0, "columns", T, K, V);
    need(b.chunks * b.columns >= V && (b.chunks - 1) * b.columns < V, "ranges", T, K, V);
    need(b.chunks == 1 || b.columns % 256 == 0, "whole tiles", T, K, V);
    need(b.chunks == 1 || b.planes_x > 0, "sums over ranges", T, K, V);
    need(b.columns <= 256 || 2 * T * b.columns <= kHeadGradBytes + 2 * T * 256, "budget", T, K, V);
}

int main()
{
    for (int64_t m = 1; m < 3000; ++m) check_sort(m);
    for (int e = 9; e <= 24; ++e)
        for (int d = -2; d <= 2; ++d) check_sort((int64_t(1) << e) + d);
    std::mt19937_64 rng(5);
    auto log_int = [&](int64_t lo, int64_t hi) {
        std::uniform_real_distribution<double> u(std::log(double(lo)), std::log(double(hi) + 1));
        return std::min(hi, int64_t(std::exp(u(rng))));
    };
    for (int i = 0; i < 20000; ++i) {
        check_embed(log_int(1, int64_t(1) << 24), log_int(1, 1 << 14));
        check_scores(log_int(1, 1 << 20), log_int(1, int64_t(1) << 24), i & 1, i % 33);
        check_head(log_int(1, 1 << 20), log_int(1, 1 << 14), log_int(1, int64_t(1) << 24), i & 1);
    }
    for (int64_t n : {1, 15, 16, 17, 1024, 1025, 20480, 20481, 65535, 65536, 65537}) check_embed(n, 8);
    for (int64_t V : {1, 255, 256, 257, 1 << 20, (1 << 20) + 1, 1 << 24})
        for (int64_t T : {1, 256, 257, 1 << 24}) check_head(T, 1, V, true);
    std::printf("ok\n");
    return 0;
}
