// Embedding lookup and its gradient.
//
// Forward: y_r = scale E[t_r], one pass over the rows asked for: 8192 of 2048 bfloat16 columns 11.5 us
// (34 MB read, tokens that stand often from the caches, and 34 written: 5.8 TB/s), one row 1.7.
//
// Backward: dE[v] = scale sum_{r: t_r = v} dy_r, in float32 in increasing r, rounded once. The tokens
// are sorted (stably, so that the order of a sum depends on the tokens alone), and the sorted
// positions cut into chunks of equal length, a wave for each (and 512 columns). A token that lies in
// one chunk altogether gets its row of the table from there; one that goes over an end leaves the sum
// of its part, and a second launch adds such parts in order: a token that stands often, as some
// always do, is shared by as many waves as it fills chunks. Most rows of a table are asked for by no
// token: the whole table is set to zero by workgroups beside those of the sort, which wait for
// memory most of their time, and what of a long table these have no time for by a launch of its own.
// Bound by those zeros: of 8192 tokens, 128256 x 2048 bfloat16, the two launches of the sort take 15 and
// 11 us with 42 MB of zeros each, the other 441 MB 66 (6.6 TB/s), the chunks 13 and the ends of chunks 8.
//
// Sort: by digits of up to nine bits from the lowest, no workgroup waiting for another. Up to
// kSortFew tokens one launch a digit: a workgroup for each of its values reads all the tokens, counts
// those with a smaller one, which is where its own begin, and those of each of its waves, and
// writes its own in order. More take three: counts of each value in blocks of 4096 tokens, their sums
// over the blocks, and the tokens to their places.
//
// Up to kSortRank tokens two launches do it all: each token's place is the number of those before it,
// counted one by one, and a workgroup for each token that is the first of its run adds the run up. 1023
// tokens, 50257 x 768 float32: 13 us with 42 MB of zeros, 18 for the other 112, and 5.
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

// ---------------------------------------------------------------- zeros
// Bytes [from, to) of the table, by `groups` workgroups of T threads. One workgroup of 1024 on each CU
// leaves room for the sort's; with two the sort waits (262 MB and a pass of 8192 tokens 51 us, not
// 47). Past the caches (not temporal), so that the sums behind them find their rows there: 2 us more
// a launch here, 8 fewer there. The address is a multiple of 16 for every table that is.
struct Zeros {
    char* table;
    int64_t from, to;
    uint32_t groups;
};
template <int T>
__device__ __forceinline__ void write_zeros(const Zeros& z, uint32_t group)
{
    const u32x4a none = {0u, 0u, 0u, 0u};
    const int64_t step = int64_t(z.groups) * T * 16;
    int64_t at = z.from + (int64_t(group) * T + threadIdx.x) * 16;
    if (reinterpret_cast<uintptr_t>(z.table) % 16 == 0) {
        for (; at + 16 <= z.to; at += step)
            __builtin_nontemporal_store(none, reinterpret_cast<u32x4a*>(z.table + at));
    } else {
        for (; at + 16 <= z.to; at += step) store16(z.table + at, none);
    }
    for (; at < z.to; at += 2) *reinterpret_cast<uint16_t*>(z.table + at) = 0;
}

// The rest of a long table, 16 bytes a thread: 6.8 TB/s, where those beside the sort reach 5.1. So each
// launch of the sort takes as much as it has time for: a gradient of 128256 x 2048 bfloat16 takes 124.8 us
// with all zeros beside the sort of 8192 tokens, 115.9 with 10 MiB at each launch, 113.7 with 40 and
// 116.1 with 80. (Two vectors a thread 122.4.) Twice that much is left to them before a launch more pays.
constexpr int64_t kZerosBeside = int64_t(40) << 20;
__global__ __launch_bounds__(256) void k_zeros(const Zeros z) { write_zeros<256>(z, blockIdx.x); }

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
    uint32_t digits;             // the digit's values
    uint32_t* counts;            // [digits][blocks], then their sums over the blocks before
    uint32_t* totals;            // [digits]
    int64_t blocks;
    Zeros zeros;                 // the first workgroups write them
};

__device__ __forceinline__ uint32_t sort_key(const SortPass& a, int64_t i)
{
    if (!a.tokens.p) return a.keys[i];
    const int64_t t = token_at(a.tokens.p, a.tokens.wide, i);
    return t >= 0 && t < a.vocab ? static_cast<uint32_t>(t) : a.vocab;
}

constexpr int kSortWaves = 16, kSortKeys = 8;   // keys of a lane that are loaded together

__global__ __launch_bounds__(64 * kSortWaves, 8) void k_sort_pass(const SortPass a)
{
    __shared__ int64_t below[kSortWaves], mine[kSortWaves];
    if (blockIdx.x < a.zeros.groups) {
        write_zeros<64 * kSortWaves>(a.zeros, blockIdx.x);
        return;
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t digit = blockIdx.x - a.zeros.groups, mask = (1u << a.bits) - 1;
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

// The place of each of 64 tokens: the number of smaller ones, and of equal ones that stand before it.
// A lane has a token, and each wave the others to compare it with, 64 in its lanes at a time.
__global__ __launch_bounds__(64 * kSortWaves) void k_sort_rank(const SortPass a)
{
    __shared__ uint32_t counts[kSortWaves][64];
    if (blockIdx.x < a.zeros.groups) {
        write_zeros<64 * kSortWaves>(a.zeros, blockIdx.x);
        return;
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = static_cast<int>(a.n);
    const int i = (blockIdx.x - a.zeros.groups) * 64 + lane;
    const uint32_t key = i < n ? sort_key(a, i) : 0;
    const int to = n * (wave + 1) / kSortWaves;
    uint32_t less = 0;
    for (int j = n * wave / kSortWaves; j < to; j += 64) {
        const uint32_t other = j + lane < to ? sort_key(a, j + lane) : 0xffffffffu;
        const int m = min(64, to - j);
        for (int k = 0; k < m; ++k) {
            const uint32_t o = __builtin_amdgcn_readlane(other, k);
            less += o < key + (j + k < i);
        }
    }
    counts[wave][lane] = less;
    __syncthreads();
    if (wave > 0 || i >= n) return;
    for (int w = 1; w < kSortWaves; ++w) less += counts[w][lane];
    a.keys_out[less] = key;
    a.rows_out[less] = static_cast<uint32_t>(i);
}

constexpr int kSortThreads = 64 * kSortWaves;
constexpr int kSortEach = kSortBlock / kSortThreads;   // keys of a lane
static_assert(kSortEach * kSortThreads == kSortBlock && (1 << kSortBits) <= kSortThreads, "a block");

__global__ __launch_bounds__(kSortThreads) void k_sort_count(const SortPass a)
{
    __shared__ uint32_t counts[1 << kSortBits];
    if (blockIdx.x < a.zeros.groups) {
        write_zeros<kSortThreads>(a.zeros, blockIdx.x);
        return;
    }
    const int64_t block = blockIdx.x - a.zeros.groups;
    const uint32_t tid = threadIdx.x;
    if (tid < a.digits) counts[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSortEach; ++u) {
        const int64_t i = block * kSortBlock + u * kSortThreads + tid;
        if (i < a.n) atomicAdd(&counts[(sort_key(a, i) >> a.shift) & ((1u << a.bits) - 1)], 1u);
    }
    __syncthreads();
    if (tid < a.digits) a.counts[tid * a.blocks + block] = counts[tid];
}

// The inclusive sum over a wave's lanes.
__device__ __forceinline__ uint32_t wave_sum_upto(uint32_t v, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t from = __shfl_up(v, d);
        if (lane >= d) v += from;
    }
    return v;
}

// A digit value's counts to their sums over the blocks before.
__global__ __launch_bounds__(256) void k_sort_scan(const SortPass a)
{
    __shared__ uint32_t of_wave[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t* __restrict__ counts = a.counts + int64_t(blockIdx.x) * a.blocks;
    uint32_t before = 0;
    for (int64_t b = 0; b < a.blocks; b += 256) {
        const int64_t i = b + threadIdx.x;
        const uint32_t v = i < a.blocks ? counts[i] : 0;
        const uint32_t upto = wave_sum_upto(v, lane);
        if (lane == 63) of_wave[wave] = upto;
        __syncthreads();
        uint32_t start = before;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) start += of_wave[w];
            before += of_wave[w];
        }
        if (i < a.blocks) counts[i] = start + upto - v;
        __syncthreads();
    }
    if (threadIdx.x == 0) a.totals[blockIdx.x] = before;
}

__global__ __launch_bounds__(kSortThreads) void k_sort_place(const SortPass a)
{
    __shared__ uint32_t of_waves[kSortWaves][1 << kSortBits];
    __shared__ uint32_t place[1 << kSortBits];       // of the block's first key of each value
    __shared__ uint32_t upto_wave[kSortWaves];
    if (blockIdx.x < a.zeros.groups) {
        write_zeros<kSortThreads>(a.zeros, blockIdx.x);
        return;
    }
    const int64_t block = blockIdx.x - a.zeros.groups;
    const uint32_t tid = threadIdx.x;
    const int lane = tid & 63, wave = tid >> 6;
    const uint32_t total = tid < a.digits ? a.totals[tid] : 0;
    const uint32_t upto = wave_sum_upto(total, lane);
    if (lane == 63) upto_wave[wave] = upto;
    for (uint32_t d = lane; d < a.digits; d += 64) of_waves[wave][d] = 0;
    __syncthreads();
    if (tid < a.digits) {
        uint32_t start = upto - total;
        for (int w = 0; w < wave; ++w) start += upto_wave[w];
        place[tid] = start + a.counts[tid * a.blocks + block];
    }
    // a wave's keys in order, 64 at a time: a key's rank among those of its value in the wave
    volatile uint32_t* mine = of_waves[wave];
    const int64_t first = block * kSortBlock + int64_t(wave) * (64 * kSortEach);
    uint32_t key[kSortEach], digit[kSortEach], rank[kSortEach];
#pragma unroll
    for (int u = 0; u < kSortEach; ++u) {
        const int64_t i = first + 64 * u + lane;
        key[u] = i < a.n ? sort_key(a, i) : 0;
    }
#pragma unroll
    for (int u = 0; u < kSortEach; ++u) {
        const bool in = first + 64 * u + lane < a.n;
        digit[u] = (key[u] >> a.shift) & ((1u << a.bits) - 1);
        uint64_t same = __ballot(in);
        for (int b = 0; b < a.bits; ++b) {
            const bool set = digit[u] >> b & 1;
            const uint64_t sets = __ballot(set);
            same &= set ? sets : ~sets;
        }
        const uint64_t lower = same & ((uint64_t(1) << lane) - 1);
        rank[u] = 0;
        if (in) {
            const uint32_t before = mine[digit[u]];
            rank[u] = before + __popcll(lower);
            if (lower == 0) mine[digit[u]] = before + __popcll(same);
        }
    }
    __syncthreads();
    if (tid < a.digits) {
        uint32_t start = place[tid];
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t n = of_waves[w][tid];
            of_waves[w][tid] = start;
            start += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSortEach; ++u) {
        const int64_t i = first + 64 * u + lane;
        if (i >= a.n) continue;
        const uint32_t o = of_waves[wave][digit[u]] + rank[u];
        a.keys_out[o] = key[u];
        a.rows_out[o] = a.tokens.p ? static_cast<uint32_t>(i) : a.rows[i];
    }
}

// ---------------------------------------------------------------- sums
struct EmbedSum {
    const uint32_t* keys;        // sorted
    const uint32_t* rows;
    const void* dy;
    int64_t n, vocab, width;
    int64_t chunk, chunks;       // sorted positions of a chunk
    float* head;                 // [chunks][width]: of the token that a chunk begins with, where it
                                 // came from the chunk before
    float* tail;                 // of the one that it ends with, where it goes on
    float scale;
    void* dtable;
};

template <bool T16>
__device__ __forceinline__ void store_sum(const EmbedSum& a, uint32_t key, int64_t e,
                                          const float (&acc)[8])
{
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = acc[j] * a.scale;
    store_row8<T16>(static_cast<char*>(a.dtable) + int64_t(key) * a.width * (T16 ? 2 : 4), e,
                    a.width, v);
}

// A wave's chunk: what it does depends on the keys alone, so that its lanes stay together; U rows
// are on their way at a time.
template <bool DY16, bool T16>
__global__ __launch_bounds__(64) void k_embed_chunks(const EmbedSum a, int64_t slabs)
{
    constexpr int U = 16, S = DY16 ? 2 : 4;
    const char* dy = static_cast<const char*>(a.dy);
    const int64_t all = a.chunks * slabs;
    for (int64_t i = blockIdx.x; i < all; i += gridDim.x) {
        const int64_t c = i / slabs, p0 = c * a.chunk, p1 = min(a.n, p0 + a.chunk);
        const int64_t e = (i % slabs) * 512 + 8 * threadIdx.x;
        const int64_t mine = min(e, (a.width - 1) / 8 * 8);   // lanes past the row read its end again
        const bool on = e < a.width;
        // lane l has the key at position p - 1 + l and the row at p + l, U of them used
        auto keys_at = [&](int64_t p) {
            const int64_t at = p - 1 + static_cast<int>(threadIdx.x);
            return at >= 0 && at < a.n ? a.keys[at] : 0xffffffffu;
        };
        uint32_t keys = keys_at(p0);
        const uint32_t before = __builtin_amdgcn_readlane(keys, 0);
        uint32_t now = __builtin_amdgcn_readlane(keys, 1), after = now;
        if (now >= a.vocab) continue;            // from here on no token of the table
        bool head = now == before;               // the token came from the chunk before
        float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        for (int64_t p = p0; p < p1; p += U) {
            if (p > p0) keys = keys_at(p);
            const uint32_t rows = a.rows[min(p + static_cast<int>(threadIdx.x), p1 - 1)];
            const int m = static_cast<int>(min(p1 - p, int64_t(U)));
            u32x4a w[U][DY16 ? 1 : 2];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t row = __builtin_amdgcn_readlane(rows, u);
                fetch8<DY16>(dy + row * a.width * S, mine, a.width, w[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t key = __builtin_amdgcn_readlane(keys, u + 1);
                if (u >= m || key >= a.vocab) continue;
                if (key != now) {
                    if (head && on) store_row8<false>(a.head + c * a.width, e, a.width, acc);
                    if (!head && on) store_sum<T16>(a, now, e, acc);
                    head = false;
                    now = key;
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[j] = 0.0f;
                }
                float v[8];
                settle8<DY16>(w[u], mine, a.width, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += v[j];
            }
            after = __builtin_amdgcn_readlane(keys, m + 1);
        }
        if (!on) continue;
        // a token that fills the chunk from the one before on is a head, whether it goes on or not
        if (head) store_row8<false>(a.head + c * a.width, e, a.width, acc);
        else if (now == after) store_row8<false>(a.tail + c * a.width, e, a.width, acc);
        else store_sum<T16>(a, now, e, acc);
    }
}

// Tokens that go over the ends of chunks: by the workgroup of the chunk in which they begin, whose
// four waves take a quarter of the other chunks each.
template <bool T16>
__global__ __launch_bounds__(256) void k_embed_spans(const EmbedSum a, int64_t slabs)
{
    constexpr int U = 16;
    __shared__ float parts[3][8][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t all = a.chunks * slabs;
    for (int64_t i = blockIdx.x; i < all; i += gridDim.x) {
        const int64_t c = i / slabs, e = (i % slabs) * 512 + 8 * lane;
        const int64_t mine = min(e, (a.width - 1) / 8 * 8);
        const int64_t p0 = c * a.chunk, p1 = p0 + a.chunk;
        if (p1 >= a.n) continue;
        const uint32_t key = a.keys[p1 - 1];
        if (key >= a.vocab || key != a.keys[p1]) continue;
        if (p0 > 0 && a.keys[p0 - 1] == key) continue;      // it began before
        // chunks c + 1 .. end - 1 begin with it: 64 steps of what is left at a time
        int64_t end = c + 1, hi = a.chunks;
        while (end < hi) {
            const int64_t step = (hi - end + 63) / 64, at = end + (lane + 1) * step - 1;
            const int64_t whole = __popcll(__ballot(at < hi && a.keys[at * a.chunk] == key));
            end += whole * step;
            hi = min(hi, end + step - 1);
            if (step == 1) break;
        }
        const int64_t d0 = c + 1 + (end - c - 1) * wave / 4, d1 = c + 1 + (end - c - 1) * (wave + 1) / 4;
        float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (wave == 0) load_row8<false>(a.tail + c * a.width, mine, a.width, acc);
        for (int64_t d = d0; d < d1; d += U) {
            u32x4a w[U][2];
#pragma unroll
            for (int u = 0; u < U; ++u)
                fetch8<false>(a.head + min(d + u, d1 - 1) * a.width, mine, a.width, w[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (d + u >= d1) continue;
                float v[8];
                settle8<false>(w[u], mine, a.width, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += v[j];
            }
        }
        if (wave > 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) parts[wave - 1][j][lane] = acc[j];
        }
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int w = 0; w < 3; ++w)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += parts[w][j][lane];
            if (e < a.width) store_sum<T16>(a, key, e, acc);
        }
        __syncthreads();
    }
}

// Few tokens: a workgroup for each sorted position and 512 columns, which has something to do where a
// token begins. Its waves share runs of more than kAlone.
template <bool DY16, bool T16>
__global__ __launch_bounds__(256) void k_embed_runs(const EmbedSum a, int64_t slabs)
{
    constexpr int U = 16, kAlone = 16, S = DY16 ? 2 : 4;
    __shared__ float parts[3][8][64];
    const char* dy = static_cast<const char*>(a.dy);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = static_cast<int>(a.n);
    const int first = static_cast<int>(blockIdx.x / slabs);
    const int64_t e = (blockIdx.x % slabs) * 512 + 8 * lane;
    const int64_t mine = min(e, (a.width - 1) / 8 * 8);
    // the keys from the one before on, 64 of them, and the end of the run
    const int at = first - 1 + lane;
    const uint32_t keys = at >= 0 && at < n ? a.keys[at] : 0xffffffffu;
    const uint32_t key = __builtin_amdgcn_readlane(keys, 1);
    if (key >= a.vocab || static_cast<uint32_t>(__builtin_amdgcn_readlane(keys, 0)) == key) return;
    const uint64_t others = ~__ballot(keys == key) >> 2;    // from the second of the run on
    int end = first + 63;
    if (others) {
        end = first + __ffsll(static_cast<unsigned long long>(others));
    } else {                                                // longer than that: 64 probes at a time
        int hi = n;
        while (end < hi) {
            const int step = (hi - end + 63) / 64, p = end + (lane + 1) * step - 1;
            end += __popcll(__ballot(p < hi && a.keys[p] == key)) * step;
            hi = min(hi, end + step - 1);
            if (step == 1) break;
        }
    }
    const int m = end - first;
    if (m <= kAlone && wave > 0) return;
    const int p0 = m <= kAlone ? first : first + m * wave / 4;
    const int p1 = m <= kAlone ? end : first + m * (wave + 1) / 4;
    float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = p0; p < p1; p += U) {
        const uint32_t rows = a.rows[min(p + lane, p1 - 1)];
        u32x4a w[U][DY16 ? 1 : 2];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u < p1)
                fetch8<DY16>(dy + int64_t(__builtin_amdgcn_readlane(rows, u)) * a.width * S, mine,
                             a.width, w[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u >= p1) continue;
            float v[8];
            settle8<DY16>(w[u], mine, a.width, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += v[j];
        }
    }
    if (m > kAlone) {
        if (wave > 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) parts[wave - 1][j][lane] = acc[j];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < 3; ++w)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += parts[w][j][lane];
    }
    if (e < a.width) store_sum<T16>(a, key, e, acc);
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
    const int64_t bytes = a.vocab * a.width * (table_bf16 ? 2 : 4);
    // The zeros are shared by the sort's launches, as far as these have time. One workgroup on each CU
    // writes them, so that the sort's have the other half of it.
    const bool rank = a.n <= kSortRank;
    const int passes = rank ? 1 : plan.passes;
    const bool blocks = a.n > kSortFew;
    const int shares = blocks ? 2 * passes : passes;
    const int64_t beside = bytes > 2 * shares * kZerosBeside ? shares * kZerosBeside : bytes;
    int out = 0, share = 0;
    auto zeros = [&]() {
        Zeros z;
        z.table = static_cast<char*>(a.dtable);
        z.from = beside * share / shares / 16 * 16;
        ++share;
        z.to = share < shares ? beside * share / shares / 16 * 16 : beside;
        z.groups = capped((z.to - z.from + 16 * kSortThreads - 1) / (16 * kSortThreads), 256);
        return z;
    };
    for (int p = 0, shift = 0; p < passes; shift += plan.bits[p], ++p) {
        SortPass s{};
        s.n = a.n;
        s.vocab = static_cast<uint32_t>(a.vocab);
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
        s.digits = p + 1 < passes
            ? 1u << s.bits : static_cast<uint32_t>(a.vocab >> shift) + 1;
        s.zeros = zeros();
        if (rank) {
            const unsigned groups = static_cast<unsigned>((a.n + 63) / 64);
            hipLaunchKernelGGL(k_sort_rank, dim3(s.zeros.groups + groups), dim3(64 * kSortWaves), 0,
                               stream, s);
            continue;
        }
        if (!blocks) {
            hipLaunchKernelGGL(k_sort_pass, dim3(s.zeros.groups + s.digits), dim3(kSortThreads), 0,
                               stream, s);
            continue;
        }
        s.counts = a.counts;
        s.blocks = sort_blocks(a.n);
        s.totals = a.counts + s.blocks * (1 << kSortBits);
        const auto grid = [&]() {
            return dim3(s.zeros.groups + static_cast<unsigned>(s.blocks));
        };
        hipLaunchKernelGGL(k_sort_count, grid(), dim3(kSortThreads), 0, stream, s);
        hipLaunchKernelGGL(k_sort_scan, dim3(s.digits), dim3(256), 0, stream, s);
        s.zeros = zeros();
        hipLaunchKernelGGL(k_sort_place, grid(), dim3(kSortThreads), 0, stream, s);
    }
    if (beside < bytes) {
        Zeros z{static_cast<char*>(a.dtable), beside, bytes, 0};
        z.groups = capped((bytes - beside + 16 * 256 - 1) / (16 * 256), 1 << 23);
        hipLaunchKernelGGL(k_zeros, dim3(z.groups), dim3(256), 0, stream, z);
    }
    if (a.n == 0) return hipGetLastError();
    EmbedSum m{};
    m.keys = a.keys[out];
    m.rows = a.rows[out];
    m.dy = a.dy;
    m.n = a.n;
    m.vocab = a.vocab;
    m.width = a.width;
    m.chunk = embed_chunk(a.n);
    m.chunks = embed_chunks(a.n);
    m.head = a.partial;
    m.tail = a.partial + m.chunks * a.width;
    m.scale = a.scale;
    m.dtable = a.dtable;
    const int64_t slabs = (a.width + 511) / 512;
    if (rank) {
        const dim3 each(static_cast<unsigned>(a.n * slabs));
        auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, each, dim3(256), 0, stream, m, slabs); };
        if (dy_bf16 && table_bf16) run(k_embed_runs<true, true>);
        else if (dy_bf16) run(k_embed_runs<true, false>);
        else if (table_bf16) run(k_embed_runs<false, true>);
        else run(k_embed_runs<false, false>);
        return hipGetLastError();
    }
    const dim3 grid(capped(m.chunks * slabs, 1 << 23));
    auto go = [&](auto kernel, int threads) {
        hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, m, slabs);
    };
    if (dy_bf16 && table_bf16) go(k_embed_chunks<true, true>, 64);
    else if (dy_bf16) go(k_embed_chunks<true, false>, 64);
    else if (table_bf16) go(k_embed_chunks<false, true>, 64);
    else go(k_embed_chunks<false, false>, 64);
    if (table_bf16) go(k_embed_spans<true>, 256);
    else go(k_embed_spans<false>, 256);
    return hipGetLastError();
}

}  // namespace gefen
