// Embedding lookup and its gradient.
//
// Forward: y_r = scale E[t_r], one pass over the rows asked for.
//
// Backward: dE[v] = scale sum_{r: t_r = v} dy_r, in float32 in increasing r, rounded once. The tokens
// are sorted (stably, so that the order of a sum depends on the tokens alone), then a wave owns a
// few rows of the table: it finds its first one among the sorted tokens, 64 probes at a time, and
// writes every row once, zeros where no token asked for it. A token that stands often would leave its
// row's wave with a long sum: wherever one token fills a whole aligned chunk of sorted positions, that
// chunk's sum is formed before, by a wave of its own, and the row takes it as one term.
//
// Sort: by digits of up to nine bits from the lowest; one workgroup for each value of the digit
// reads all the tokens, counts those with a smaller digit, which is where its own begin, and those
// of each of its waves, and writes its own in order. No workgroup waits for another.
#include "token_internal.h"

#include "token_device.h"

namespace gefen {
namespace {

// Lanes along a row of a workgroup: a power of two, 256 at most.
inline int row_lanes(int64_t width)
{
    int l = 1;
    while (l < 256 && 8 * l < width) l *= 2;
    return l;
}

template <bool TABLE16, bool Y16>
__global__ __launch_bounds__(256) void k_embedding(const EmbedArgs a, int lanes)
{
    const int per = 256 / lanes;                    // rows of a workgroup at once
    const int lane = threadIdx.x % lanes;
    constexpr int TS = TABLE16 ? 2 : 4, YS = Y16 ? 2 : 4;
    const int64_t width = by_lane(a.width);
    for (int64_t r = int64_t(blockIdx.x) * per + threadIdx.x / lanes; r < a.n;
         r += int64_t(gridDim.x) * per) {
        const int64_t t = token_at(a.tokens.p, a.tokens.wide, r);
        const bool on = t >= 0 && t < a.vocab;
        const char* from = static_cast<const char*>(a.table) + (on ? t : 0) * width * TS;
        char* to = static_cast<char*>(a.y) + r * width * YS;
        const float rest = t < 0 ? 0.0f : __uint_as_float(0x7fc00000u);
        for (int64_t e = 8 * lane; e < width; e += 8 * lanes) {
            float v[8];
            load_row8<TABLE16>(from, e, width, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = on ? v[j] * a.scale : rest;
            store_row8<Y16>(to, e, width, v);
        }
    }
}

// ---------------------------------------------------------------- sort
struct SortPass {
    Tokens tokens;               // the first pass's keys; p null: keys
    const uint32_t* keys;
    const uint32_t* rows;
    uint32_t* keys_out;
    uint32_t* rows_out;
    int64_t n;
    uint32_t vocab;              // the key of a token outside 0 .. vocab - 1
    int shift, bits;
};

__device__ __forceinline__ uint32_t sort_key(const SortPass& a, int64_t i)
{
    if (!a.tokens.p) return a.keys[i];
    const int64_t t = token_at(a.tokens.p, a.tokens.wide, i);
    return t >= 0 && t < a.vocab ? static_cast<uint32_t>(t) : a.vocab;
}

constexpr int kSortWaves = 16, kSortKeys = 8;   // keys of a lane that are loaded together

__global__ __launch_bounds__(64 * kSortWaves) void k_sort_pass(const SortPass a)
{
    __shared__ int64_t below[kSortWaves], mine[kSortWaves];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t digit = blockIdx.x, mask = (1u << a.bits) - 1;
    const int64_t from = a.n * wave / kSortWaves, to = a.n * (wave + 1) / kSortWaves;
    constexpr int kStep = 64 * kSortKeys;
    uint32_t key[kSortKeys];
    auto load = [&](int64_t i) {                    // past the wave's share: no digit
#pragma unroll
        for (int u = 0; u < kSortKeys; ++u) {
            const int64_t at = i + 64 * u + lane;
            key[u] = at < to ? sort_key(a, at) : 0;
        }
    };
    auto digit_of = [&](int64_t i, int u) {
        return i + 64 * u + lane < to ? (key[u] >> a.shift) & mask : mask + 1;
    };
    int64_t less = 0, same = 0;
    for (int64_t i = from; i < to; i += kStep) {
        load(i);
#pragma unroll
        for (int u = 0; u < kSortKeys; ++u) {
            const uint32_t d = digit_of(i, u);
            less += __popcll(__ballot(d < digit));
            same += __popcll(__ballot(d == digit));
        }
    }
    if (lane == 0) {
        below[wave] = less;
        mine[wave] = same;
    }
    __syncthreads();
    if (!same) return;
    int64_t at = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        at += below[w];
        if (w < wave) at += mine[w];
    }
    const bool again = to - from > kStep;           // else the keys are still there
    for (int64_t i = from; i < to; i += kStep) {
        if (again) load(i);
#pragma unroll
        for (int u = 0; u < kSortKeys; ++u) {
            const bool hit = digit_of(i, u) == digit;
            const uint64_t hits = __ballot(hit);
            if (hit) {
                const int64_t from_row = i + 64 * u + lane;
                const int64_t o = at + __popcll(hits & ((uint64_t(1) << lane) - 1));
                a.keys_out[o] = key[u];
                a.rows_out[o] = a.tokens.p ? static_cast<uint32_t>(from_row) : a.rows[from_row];
            }
            at += __popcll(hits);
        }
    }
}

// ---------------------------------------------------------------- sums
struct EmbedSum {
    const uint32_t* keys;        // sorted
    const uint32_t* rows;
    const void* dy;
    int64_t n, vocab, width;
    int64_t chunk;               // a power of two
    float* partial;              // [n / chunk][width]
    float scale;
    void* dtable;
    int lanes;                   // along a row, a power of two, 256 at most
    int64_t per;                 // rows of the table for a workgroup
};

// acc += the rows at sorted positions p .. to - 1, eight elements from e on, in order. U rows are on
// their way at a time.
template <bool DY16, int U>
__device__ __forceinline__ void add_rows(const EmbedSum& a, int64_t width, int64_t p, int64_t to,
                                         int64_t e, float (&acc)[8])
{
    constexpr int S = DY16 ? 2 : 4;
    const char* dy = static_cast<const char*>(a.dy);
    for (; p < to; p += U) {
        uint32_t r[U];
        u32x4a w[U][DY16 ? 1 : 2];
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = a.rows[p + u < to ? p + u : to - 1];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u < to) fetch8<DY16>(dy + int64_t(r[u]) * width * S, e, width, w[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u < to) {
                float v[8];
                settle8<DY16>(w[u], e, width, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += v[j];
            }
    }
}

// acc += rows c .. to - 1 of the chunks' sums.
__device__ __forceinline__ void add_chunks(const EmbedSum& a, int64_t width, int64_t c, int64_t to,
                                           int64_t e, float (&acc)[8])
{
    constexpr int U = 4;
    for (; c < to; c += U) {
        u32x4a w[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c + u < to) fetch8<false>(a.partial + (c + u) * width, e, width, w[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c + u < to) {
                float v[8];
                settle8<false>(w[u], e, width, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += v[j];
            }
    }
}

// The sums of whole chunks of one token. A wave takes 512 columns of a chunk.
template <bool DY16>
__global__ __launch_bounds__(64) void k_embed_chunks(const EmbedSum a, int64_t slabs)
{
    const int64_t width = by_lane(a.width);
    const int64_t all = a.n / a.chunk * slabs;
    for (int64_t i = blockIdx.x; i < all; i += gridDim.x) {
        const int64_t c = i / slabs, e = (i % slabs) * 512 + 8 * threadIdx.x;
        const uint32_t key = a.keys[c * a.chunk];
        if (key >= a.vocab || key != a.keys[(c + 1) * a.chunk - 1] || e >= width) continue;
        float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        add_rows<DY16, DY16 ? 16 : 8>(a, width, c * a.chunk, (c + 1) * a.chunk, e, acc);
        store_row8<false>(a.partial + c * width, e, width, acc);
    }
}

// The first sorted position in [lo, n) whose key is not below `key`; all lanes together.
__device__ __forceinline__ int64_t lower_bound(const uint32_t* keys, int64_t lo, int64_t n,
                                               uint32_t key, int lane)
{
    int64_t hi = n;              // in [lo, hi]
    while (lo < hi) {
        const int64_t step = (hi - lo + 63) / 64;
        const int64_t i = lo + (lane + 1) * step - 1;   // the last of the lane's step
        const bool under = i < hi && keys[i] < key;
        const int64_t whole = __popcll(__ballot(under)); // steps that lie below altogether
        lo += whole * step;
        hi = min(hi, lo + step - 1);
        if (step == 1) break;
    }
    return lo;
}

// A workgroup writes `per` rows of the table: `lanes` lanes a row, so that wide rows are shared by
// its waves and narrow ones lie side by side in one.
template <bool DY16, bool T16>
__global__ __launch_bounds__(256) void k_embed_sum(const EmbedSum a)
{
    const int lane = threadIdx.x & 63;
    const int sub = threadIdx.x / a.lanes, along = threadIdx.x % a.lanes;
    const int together = 256 / a.lanes;
    // the rows of this wave: the (first + k)-th of `together`, k < mine
    const int first_sub = __builtin_amdgcn_readfirstlane(sub);
    const int mine = a.lanes >= 64 ? 1 : 64 / a.lanes;
    constexpr int TS = T16 ? 2 : 4;
    const int64_t width = by_lane(a.width);
    const int64_t groups = (a.vocab + a.per - 1) / a.per;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t v0 = g * a.per, v1 = min(a.vocab, v0 + a.per);
        int64_t at = lower_bound(a.keys, 0, a.n, static_cast<uint32_t>(v0), lane);
        auto window = [&]() { return at + lane < a.n ? a.keys[at + lane] : 0xffffffffu; };
        uint32_t keys = window();                    // 64 of them, one a lane, from `at` on
        auto bound = [&](int64_t v) {                // the first position of a key >= v > v0
            int64_t end = at + __popcll(__ballot(keys < static_cast<uint32_t>(v)));
            if (end == at + 64) {                    // further than the window
                end = at = lower_bound(a.keys, end, a.n, static_cast<uint32_t>(v), lane);
                keys = window();
            }
            return end;
        };
        for (int64_t v = v0; v < v1; v += together) {
            int64_t first = 0, last = 0;             // of the lane's row
            const int64_t w = v + first_sub;
            if (w < v1) {
                int64_t pos = bound(w);
                for (int k = 0; k < mine && w + k < v1; ++k) {
                    const int64_t end = bound(w + k + 1);
                    if (first_sub + k == sub) {
                        first = pos;
                        last = end;
                    }
                    pos = end;
                }
            }
            if (v + sub >= v1) continue;
            char* to = static_cast<char*>(a.dtable) + (v + sub) * width * TS;
            for (int64_t e = 8 * along; e < width; e += 8 * a.lanes) {
                float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
                if (first < last) {
                    const int64_t c0 = (first + a.chunk - 1) / a.chunk, c1 = last / a.chunk;
                    const bool chunks = c0 < c1;
                    add_rows<DY16, 8>(a, width, first, chunks ? c0 * a.chunk : last, e, acc);
                    if (chunks) {
                        add_chunks(a, width, c0, c1, e, acc);
                        add_rows<DY16, 8>(a, width, c1 * a.chunk, last, e, acc);
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[j] *= a.scale;
                }
                store_row8<T16>(to, e, width, acc);
            }
        }
    }
}

inline unsigned capped(int64_t groups, int64_t most) { return static_cast<unsigned>(groups < most ? groups : most); }

}  // namespace

hipError_t launch_embedding(const EmbedArgs& a, bool table_bf16, bool y_bf16, hipStream_t stream)
{
    if (a.n == 0) return hipSuccess;
    const int lanes = row_lanes(a.width);
    const int64_t per = 256 / lanes;
    const dim3 grid(capped((a.n + per - 1) / per, 1 << 20));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, lanes); };
    if (table_bf16 && y_bf16) go(k_embedding<true, true>);
    else if (table_bf16) go(k_embedding<true, false>);
    else if (y_bf16) go(k_embedding<false, true>);
    else go(k_embedding<false, false>);
    return hipGetLastError();
}

hipError_t launch_embedding_grad(const EmbedGradArgs& a, bool dy_bf16, bool table_bf16,
                                 hipStream_t stream)
{
    const SortPlan plan = sort_plan(a.vocab);
    SortPass s{};
    s.n = a.n;
    s.vocab = static_cast<uint32_t>(a.vocab);
    int out = 0;
    if (a.n > 0) {
        for (int p = 0, shift = 0; p < plan.passes; shift += plan.bits[p], ++p) {
            s.tokens = a.tokens;
            if (p > 0) s.tokens.p = nullptr;
            s.keys = a.keys[out];
            s.rows = a.rows[out];
            out ^= 1;
            s.keys_out = a.keys[out];
            s.rows_out = a.rows[out];
            s.shift = shift;
            s.bits = plan.bits[p];
            // the last digit ends with the largest key's
            const int64_t digits = p + 1 < plan.passes ? int64_t(1) << s.bits : (a.vocab >> shift) + 1;
            hipLaunchKernelGGL(k_sort_pass, dim3(static_cast<unsigned>(digits)),
                               dim3(64 * kSortWaves), 0, stream, s);
        }
    }
    EmbedSum m{};
    m.keys = a.keys[out];
    m.rows = a.rows[out];
    m.dy = a.dy;
    m.n = a.n;
    m.vocab = a.vocab;
    m.width = a.width;
    m.chunk = embed_chunk(a.n);
    m.partial = a.partial;
    m.scale = a.scale;
    m.dtable = a.dtable;
    m.lanes = row_lanes(a.width);
    m.per = 8 * (256 / m.lanes);
    if (a.n >= m.chunk) {
        const int64_t slabs = (a.width + 511) / 512;
        const dim3 grid(capped(a.n / m.chunk * slabs, 1 << 24));
        if (dy_bf16) hipLaunchKernelGGL(k_embed_chunks<true>, grid, dim3(64), 0, stream, m, slabs);
        else hipLaunchKernelGGL(k_embed_chunks<false>, grid, dim3(64), 0, stream, m, slabs);
    }
    const int64_t groups = (a.vocab + m.per - 1) / m.per;
    const dim3 grid(capped(groups, 1 << 22));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, m); };
    if (dy_bf16 && table_bf16) go(k_embed_sum<true, true>);
    else if (dy_bf16) go(k_embed_sum<true, false>);
    else if (table_bf16) go(k_embed_sum<false, true>);
    else go(k_embed_sum<false, false>);
    return hipGetLastError();
}

}  // namespace gefen
