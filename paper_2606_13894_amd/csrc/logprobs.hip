// Log probabilities of given tokens, their entropy and best alternatives, and the gradients, from rows
// of scores; and the output head's rows from its tiles' statistics.
//
// One pass over a row: each lane keeps the largest score m of what it has read, s = sum 2^d and
// t = sum d 2^d with d = (z - m) log2 e (token_device.h), so that lse = m + ln 2 log2 s, the entropy is
// ln 2 (log2 s - t / s), and a token's log probability ln 2 (d - log2 s). Lanes, waves and, where
// rows are few, workgroups that share a row are joined in a fixed order.
//
// Best alternatives, by value and among equals by the lower index: a lane also keeps where its
// largest score first stood. The lanes are 64 groups (of lanes 64 apart), and the k-th largest of the
// groups' largest scores is reached by k scores at least: only the vectors of lanes that reach it are
// read again, and the few scores that do are ranked by counting. (They go to a list in LDS; where it
// does not hold them, the k best are taken one by one.) A score and its place are one 64-bit key, the
// place inverted, so that no two are equal and no order of arrival counts.
//
// Many rows are bound by memory: 2048 of 128256 bfloat16 with 5 alternatives 106 us (525 MB, 5.0 TB/s);
// 1023 of 50257 float32 38 us (206 MB, 5.5 TB/s). One row is bound by its CU's arithmetic: 128256 with
// 20 alternatives 15.5 us.
//
// Gradients: dz_j = g ([j = token] - p_j) - h p_j (log p_j + H), p_j = exp(z_j - lse), elementwise:
// 1023 of 50257 float32 68 to 71 us (411 MB, 5.8 to 6.0 TB/s).
#include "token_internal.h"

#include "token_device.h"

#include <type_traits>

namespace gefen {
namespace {

constexpr int kList = 1024;              // keys of a row that LDS holds beside the lanes'
constexpr int kJoinThreads = 1024;

// Scores order as these do; -0 is 0.
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u)
{
    return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ uint64_t score_key(float v, int64_t place)
{
    return (static_cast<uint64_t>(ordered(v)) << 32) | static_cast<uint32_t>(~place);
}

// 16 bytes of a row of n as scores. (A row has 2^24 of them at most.)
template <bool BF16>
struct Vec {
    static constexpr int N = BF16 ? 8 : 4;
    static __device__ __forceinline__ u32x4a fetch(const void* row, int v, int n)
    {
        return fetch_vector<BF16 ? 2 : 4>(row, v * N, n);
    }
    static __device__ __forceinline__ void unpack(const u32x4a& w, float (&z)[N])
    {
#pragma unroll
        for (int j = 0; j < N; ++j)
            z[j] = BF16 ? __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16)
                        : __uint_as_float(w[j]);
    }
    // With -inf from n on.
    static __device__ __forceinline__ void settle(const u32x4a& w, int v, int n, float (&z)[N])
    {
        unpack(settle_vector<BF16 ? 2 : 4>(w, v * N, n), z);
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (v * N + j >= n) z[j] = -INFINITY;
    }
};

// The sums of the lanes that are FROM apart: the largest m first, so that each lane moves its sums to
// that base once.
template <int FROM = 1>
__device__ __forceinline__ ScoreSum wave_join(ScoreSum a)
{
    float m = a.m;
#pragma unroll
    for (int d = FROM; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    score_rebase(a.m, score_base(m), a.s, a.t);
    a.m = m;
#pragma unroll
    for (int d = FROM; d < 64; d *= 2) {
        a.s += __shfl_xor(a.s, d);
        a.t += __shfl_xor(a.t, d);
    }
    return a;
}

// Several of a lane's, in order, the same way.
template <int U>
__device__ __forceinline__ void join_all(ScoreSum& a, ScoreSum (&v)[U])
{
    float m = a.m;
#pragma unroll
    for (int u = 0; u < U; ++u) m = fmaxf(m, v[u].m);
    const ScoreBase base = score_base(m);
    score_rebase(a.m, base, a.s, a.t);
    a.m = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        score_rebase(v[u].m, base, v[u].s, v[u].t);
        a.s += v[u].s;
        a.t += v[u].t;
    }
}

template <int L>
struct ListSpace {
    unsigned long long groups[64];     // 0, as the counts, before the row
    uint64_t list[kList];
    uint64_t best[L / 64];
    uint64_t least;
    int lanes[L];
    int found, count;
};

// The number of keys[0 .. n) above `key`.
__device__ __forceinline__ int count_above(const uint64_t* keys, int n, uint64_t key)
{
    int above = 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i) above += keys[i] > key;
    return above;
}

// A bound that k of the distinct keys that a wave's lanes hold reach, and few more, bit by bit from the
// top; 0 where they are fewer than k (keys of 0 are none).
__device__ __forceinline__ uint64_t least_of_top(uint64_t key, int k)
{
    uint64_t least = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t with = least | (uint64_t(1) << bit);
        const int n = __popcll(__ballot(key >= with));
        if (n >= k) {
            least = with;
            if (n <= k + k / 2 + 2) break;
        }
    }
    return least;
}

// The k largest keys of vectors v0 .. v1 - 1 of a row, in order, to out; 0 where there are fewer.
// `key`: of the lane's largest score, its place that vector's number; 0 where it has read none.
template <bool BF16, int L>
__device__ void select_top(const void* row, int n, int v0, int v1, int k, uint64_t key,
                           ListSpace<L>& s, uint64_t* __restrict__ out)
{
    constexpr int N = Vec<BF16>::N, kWaves = L / 64;
    const int tid = threadIdx.x;
    n = by_lane(n);
    if (key) atomicMax(&s.groups[tid & 63], static_cast<unsigned long long>(key));
    __syncthreads();
    if (tid < 64) {
        const uint64_t of_groups = least_of_top(s.groups[tid], k);
        if (tid == 0) s.least = of_groups;
    }
    __syncthreads();
    const uint64_t least = s.least;
    if (key && key >= least) s.lanes[atomicAdd(&s.found, 1)] = tid;
    __syncthreads();
    const int per = (v1 - v0 + L - 1) / L;
    for (int i = tid; i < s.found * per; i += L) {
        const int v = v0 + s.lanes[i / per] + (i % per) * L;
        if (v >= v1) continue;
        float z[N];
        Vec<BF16>::settle(Vec<BF16>::fetch(row, v, n), v, n, z);
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (v * N + j < n && score_key(z[j], v) >= least) {
                const int at = atomicAdd(&s.count, 1);
                if (at < kList) s.list[at] = score_key(z[j], v * N + j);
            }
    }
    __syncthreads();
    const int count = s.count;
    if (count <= kList) {
        for (int i = tid; i < count; i += L) {
            const int at = count_above(s.list, count, s.list[i]);
            if (at < k) out[at] = s.list[i];
        }
        for (int i = count + tid; i < k; i += L) out[i] = 0;
    } else {
        uint64_t before = ~uint64_t(0);
        for (int r = 0; r < k; ++r) {
            uint64_t best = 0;
            for (int v = v0 + tid; v < v1; v += L) {
                float z[N];
                Vec<BF16>::settle(Vec<BF16>::fetch(row, v, n), v, n, z);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const uint64_t q = score_key(z[j], v * N + j);
                    if (v * N + j < n && q < before && q > best) best = q;
                }
            }
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const uint64_t other = __shfl_xor(static_cast<unsigned long long>(best), d);
                best = other > best ? other : best;
            }
            if ((tid & 63) == 0) s.best[tid >> 6] = best;
            __syncthreads();
            for (int w = 0; w < kWaves; ++w) best = s.best[w] > best ? s.best[w] : best;
            if (tid == 0) out[r] = best;
            before = best;
            __syncthreads();
        }
    }
    __syncthreads();
}

// The row's best alternatives from their keys in order.
__device__ __forceinline__ void write_top(const ScoreArgs& a, int64_t row, const ScoreSum& sum,
                                          int i, uint64_t key)
{
    const int64_t o = row * a.top + i;
    const float v = unordered(static_cast<uint32_t>(key >> 32));
    const bool bad = sum.s != sum.s;
    a.top_logprob[o] = bad ? sum.s : v == -INFINITY ? v
                                   : score_logprob(v, score_base(sum.m), log2f(sum.s));
    a.top_token[o] = bad ? -1 : static_cast<int64_t>(~static_cast<uint32_t>(key));
}

__device__ __forceinline__ void write_row(const ScoreArgs& a, int64_t row, const ScoreSum& sum,
                                          int64_t token, float taken)
{
    const ScoreRow r = score_row(sum, token, a.vocab, taken);
    a.logprob[row] = r.logprob;
    a.entropy[row] = r.entropy;
    a.lse[row] = r.lse;
    if (a.rest) a.rest[row] = r.rest;
}

template <bool BF16>
__device__ __forceinline__ float score_at(const void* z, int64_t i)
{
    if constexpr (BF16) return bf16_float(static_cast<const uint16_t*>(z)[i]);
    else return static_cast<const float*>(z)[i];
}

template <bool BF16, bool TOP, int L>
__global__ __launch_bounds__(L) void k_scores(const ScoreArgs a)
{
    using V = Vec<BF16>;
    constexpr int N = V::N, U = 4, S = BF16 ? 2 : 4, kWaves = L / 64;
    __shared__ ScoreSum sums[kWaves];
    __shared__ typename std::conditional<TOP, ListSpace<L>, int>::type list;
    __shared__ uint64_t best[TOP ? kScoreMaxTop : 1];
    const int tid = threadIdx.x;
    const int vocab = static_cast<int>(a.vocab);
    const int vectors = (vocab + N - 1) / N, whole = vocab / N;
    const int64_t items = a.rows * a.plan.parts;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t r = item / a.plan.parts, part = item % a.plan.parts;
        const char* row = static_cast<const char*>(a.z) + r * a.ld * S;
        const int v0 = static_cast<int>(part * a.plan.per);
        const int v1 = min(vectors, v0 + static_cast<int>(a.plan.per));
        const bool one = a.plan.parts == 1;
        int64_t token = -1;
        float taken = 0.0f;
        if (one && tid == 0) {
            token = token_at(a.tokens.p, a.tokens.wide, r);
            if (token >= 0 && token < vocab) taken = score_at<BF16>(row, token);
        }
        if constexpr (TOP) {
            if (tid < 64) list.groups[tid] = 0;
            if (tid == 0) list.found = list.count = 0;
        }
        ScoreSum c = {-INFINITY, 0.0f, 0.0f};
        float top = -INFINITY;
        int place = -1;
        // A lane's vectors are L apart; U of them are worked on while the next U are on their way.
        // (A vector past the end is the last one again, and left out below.)
        u32x4a next[U];
        auto load = [&](int b) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                next[u] = V::fetch(row, min(b + u * L + tid, vectors - 1), vocab);
        };
        auto work = [&](const u32x4a (&w)[U], int b, auto is_full) {
            constexpr bool FULL = decltype(is_full)::value;
            float z[U][N];
            float m = -INFINITY, low = INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = b + u * L + tid;
                if constexpr (FULL) {
                    V::unpack(w[u], z[u]);
                } else if (v < v1) {
                    V::settle(w[u], v, vocab, z[u]);
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j) z[u][j] = -INFINITY;
                }
                float vm = z[u][0], vl = z[u][0];
#pragma unroll
                for (int j = 1; j < N; ++j) {
                    vm = fmaxf(vm, z[u][j]);
                    vl = fminf(vl, z[u][j]);
                }
                m = fmaxf(m, vm);
                low = fminf(low, vl);
                if constexpr (TOP) {
                    if ((FULL || v < v1) && (place < 0 || vm > top)) {
                        top = vm;
                        place = v;
                    }
                }
            }
            const float old = c.m;
            c.m = fmaxf(old, m);
            const ScoreBase base = score_base(c.m);
            score_rebase(old, base, c.s, c.t);
            if (__all(!base.far && low > kScoreLow)) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < N; ++j) score_add_plain(z[u][j], base.b, c.s, c.t);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < N; ++j) score_add(z[u][j], base, c.s, c.t);
            }
        };
        load(v0);
        for (int b = v0; b < v1; b += U * L) {
            u32x4a w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) w[u] = next[u];
            if (b + U * L < v1) load(b + U * L);
            if (b + U * L <= min(v1, whole)) work(w, b, std::integral_constant<bool, true>{});
            else work(w, b, std::integral_constant<bool, false>{});
        }
        c = wave_join(c);
        if ((tid & 63) == 0) sums[tid >> 6] = c;
        __syncthreads();
        c = tid % 64 < kWaves ? sums[tid % 64] : ScoreSum{-INFINITY, 0.0f, 0.0f};
        c = wave_join(c);
        if constexpr (TOP) {
            // (a NaN as the largest of a vector ends in a row whose alternatives are not given)
            const uint64_t key = place >= 0 ? score_key(top, place) : 0;
            select_top<BF16, L>(row, vocab, v0, v1, a.top, key, list, best);
            if (tid < a.top) {
                if (one) write_top(a, r, c, tid, best[tid]);
                else a.keys[item * a.top + tid] = best[tid];
            }
        }
        if (tid == 0) {
            if (one) {
                write_row(a, r, c, token, taken);
            } else {
                a.stats[3 * item] = c.m;
                a.stats[3 * item + 1] = c.s;
                a.stats[3 * item + 2] = c.t;
            }
        }
        __syncthreads();
    }
}

// A row from its parts: their sums in order, and the best of their best. A workgroup a row; each wave
// joins the sums, all of them rank the keys (a row of 2^22 float32 scores with 32 alternatives takes 44
// us in all; where one wave ranked them, 290).
template <bool BF16>
__global__ __launch_bounds__(kJoinThreads) void k_scores_join(const ScoreArgs a)
{
    __shared__ uint64_t keys[kScoreMaxParts * kScoreMaxTop];
    __shared__ uint64_t list[kScoreMaxParts * kScoreMaxTop];
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & 63;
    const int parts = static_cast<int>(a.plan.parts);
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        ScoreSum c = {-INFINITY, 0.0f, 0.0f};
        if (lane < parts) {
            const float* p = a.stats + 3 * (r * parts + lane);
            c = ScoreSum{p[0], p[1], p[2]};
        }
        c = wave_join(c);
        if (tid == 0) {
            const int64_t token = token_at(a.tokens.p, a.tokens.wide, r);
            float taken = 0.0f;
            if (token >= 0 && token < a.vocab) taken = score_at<BF16>(a.z, r * a.ld + token);
            write_row(a, r, c, token, taken);
        }
        if (a.top) {
            const int n = parts * a.top;
            if (tid == 0) count = 0;
            for (int i = tid; i < n; i += kJoinThreads) keys[i] = a.keys[r * n + i];
            __syncthreads();
            // no key below the k-th largest of the parts' largest ones is among the k largest
            uint64_t least = 1;
            if (parts >= a.top) {
                const uint64_t first = lane < parts ? keys[lane * a.top] : 0;
                least = max(least_of_top(first, a.top), least);
            }
            for (int i = tid; i < n; i += kJoinThreads)
                if (keys[i] >= least) list[atomicAdd(&count, 1)] = keys[i];
            __syncthreads();
            const int found = count;
            for (int i = tid; i < found; i += kJoinThreads) {
                const int rank = count_above(list, found, list[i]);
                if (rank < a.top) write_top(a, r, c, rank, list[i]);
            }
            __syncthreads();
        }
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void k_score_grad(const ScoreGradArgs a, int64_t segments)
{
    constexpr int U = 2, S = BF16 ? 2 : 4;
    const int64_t items = a.rows * segments;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t r = item / segments;
        const int64_t e0 = (item % segments) * (256 * 8 * U) + 8 * threadIdx.x;
        const int64_t token = token_at(a.tokens.p, a.tokens.wide, r);
        const ScoreGrad g = score_grad_row(token, a.vocab, r, a.lse, a.rest, a.entropy,
                                           a.dlogprob, a.dentropy);
        const char* z = static_cast<const char*>(a.z) + r * a.ld * S;
        char* dz = static_cast<char*>(a.dz) + r * a.ldd * S;
        u32x4a w[U][BF16 ? 1 : 2];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (e0 + 2048 * u < a.vocab) fetch8<BF16>(z, e0 + 2048 * u, a.vocab, w[u]);
        // (in place: the lane that ends a row may find gradients of the lane before it in its
        // vector, in the elements that it shifts out)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t e = e0 + 2048 * u;
            if (e >= a.vocab) continue;
            float v[8];
            settle8<BF16>(w[u], e, a.vocab, v);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] = score_gradient(v[j], g, token == e + j);
            store_row8<BF16>(dz, e, a.vocab, v);
        }
    }
}

// ---------------------------------------------------------------- output head
// A workgroup joins R rows, 1024 / R lanes to a row by the slots, U of a lane's on their way at once.
// R = 1: statistics that lie by rows. 8192 rows of 1002 slots 36 us (99 MB, 2.8 TB/s), one row of 16032
// slots 7.8.
template <int R, int U>
__global__ __launch_bounds__(1024) void k_head_join(const HeadJoinArgs a)
{
    constexpr int kWays = 1024 / R, kWaves = 16;
    __shared__ ScoreSum sums[kWaves][R];
    const int in = threadIdx.x % R, way = threadIdx.x / R, wave = threadIdx.x >> 6;
    const int64_t r = int64_t(blockIdx.x) * R + in;
    const int64_t row = min(r, a.rows - 1);
    ScoreSum c = {-INFINITY, 0.0f, 0.0f};
    for (int64_t s = 0; s < a.slots; s += U * kWays) {
        ScoreSum v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = min(s + u * kWays + way, a.slots - 1);
            const float* p = a.stats + (R == 1 ? 3 * row * a.slots + at : 3 * at * a.rows + row);
            const int64_t next = R == 1 ? a.slots : a.rows;
            v[u] = ScoreSum{p[0], p[next], p[2 * next]};
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s + u * kWays + way >= a.slots) v[u] = ScoreSum{-INFINITY, 0.0f, 0.0f};
        join_all(c, v);
    }
    c = wave_join<R>(c);
    if ((threadIdx.x & 63) < R) sums[wave][in] = c;
    __syncthreads();
    if (threadIdx.x >= R || r >= a.rows) return;
    ScoreSum v[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v[w] = sums[w][in];
    c = ScoreSum{-INFINITY, 0.0f, 0.0f};
    join_all(c, v);
    const int64_t token = token_at(a.tokens.p, a.tokens.wide, r);
    const float taken = token >= 0 && token < a.vocab ? a.taken[r] : 0.0f;
    const ScoreRow o = score_row(c, token, a.vocab, taken);
    a.logprob[r] = o.logprob;
    a.entropy[r] = o.entropy;
    a.lse[r] = o.lse;
}

}  // namespace

hipError_t launch_scores(const ScoreArgs& a, bool bf16, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    const int64_t items = a.rows * a.plan.parts;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(items, 1 << 20)));
    auto go = [&](auto few, auto many) {
        if (a.plan.threads == kScoreThreads)
            hipLaunchKernelGGL(many, grid, dim3(kScoreThreads), 0, stream, a);
        else
            hipLaunchKernelGGL(few, grid, dim3(kScoreFewThreads), 0, stream, a);
    };
    constexpr int F = kScoreFewThreads, M = kScoreThreads;
    if (bf16 && a.top) go(k_scores<true, true, F>, k_scores<true, true, M>);
    else if (bf16) go(k_scores<true, false, F>, k_scores<true, false, M>);
    else if (a.top) go(k_scores<false, true, F>, k_scores<false, true, M>);
    else go(k_scores<false, false, F>, k_scores<false, false, M>);
    if (a.plan.parts > 1) {
        const dim3 rows(static_cast<unsigned>(std::min<int64_t>(a.rows, 1 << 20)));
        if (bf16) hipLaunchKernelGGL(k_scores_join<true>, rows, dim3(kJoinThreads), 0, stream, a);
        else hipLaunchKernelGGL(k_scores_join<false>, rows, dim3(kJoinThreads), 0, stream, a);
    }
    return hipGetLastError();
}

hipError_t launch_score_grad(const ScoreGradArgs& a, bool bf16, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    const int64_t segments = (a.vocab + 4095) / 4096;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(a.rows * segments, 1 << 22)));
    if (bf16) hipLaunchKernelGGL(k_score_grad<true>, grid, dim3(256), 0, stream, a, segments);
    else hipLaunchKernelGGL(k_score_grad<false>, grid, dim3(256), 0, stream, a, segments);
    return hipGetLastError();
}

hipError_t launch_head_join(const HeadJoinArgs& a, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    if (a.by_rows)
        hipLaunchKernelGGL((k_head_join<1, 16>), dim3(static_cast<unsigned>(a.rows)), dim3(1024), 0,
                           stream, a);
    else
        hipLaunchKernelGGL((k_head_join<16, 4>), dim3(static_cast<unsigned>((a.rows + 15) / 16)),
                           dim3(1024), 0, stream, a);
    return hipGetLastError();
}

}  // namespace gefen
