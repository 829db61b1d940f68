// C ABI of the operators at a language model's two ends: argument checks, workspace layout and
// launches.
#include "abi_checks.h"
#include "ffn_launch.h"
#include "token_internal.h"
#include "token_plan.h"

#include <cmath>

using namespace gefen;

namespace {

constexpr int64_t kMaxVocab = int64_t(1) << 24;

int check_tokens(int64_t n, int32_t token_bytes)
{
    if (n < 0 || n > kFfnMaxTokens)
        return fail(GEFEN_EINVAL, "tokens must be in [0, %lld]", (long long)kFfnMaxTokens);
    if (token_bytes != 4 && token_bytes != 8)
        return fail(GEFEN_EINVAL, "token_bytes must be 4 or 8");
    return GEFEN_OK;
}

int check_table(int64_t n, int64_t vocab, int64_t width)
{
    if (vocab < 1 || vocab > kMaxVocab)
        return fail(GEFEN_EINVAL, "vocab must be in [1, %lld]", (long long)kMaxVocab);
    if (width < 1 || width > kFfnMaxWidth)
        return fail(GEFEN_EINVAL, "width must be in [1, %lld]", (long long)kFfnMaxWidth);
    if (vocab > kMaxElems / width || n > kMaxElems / width)
        return fail(GEFEN_EINVAL, "more than 2^40 elements");
    return GEFEN_OK;
}

int check_scale(double scale)
{
    if (!std::isfinite(static_cast<float>(scale)))
        return fail(GEFEN_EINVAL, "scale must be finite in float32");
    return GEFEN_OK;
}

int check_scores(int64_t rows, int64_t vocab, int64_t ld)
{
    if (rows < 0) return fail(GEFEN_EINVAL, "rows must not be negative");
    if (vocab < 1 || vocab > kMaxVocab)
        return fail(GEFEN_EINVAL, "vocab must be in [1, %lld]", (long long)kMaxVocab);
    if (ld < vocab) return fail(GEFEN_EINVAL, "rows that are %lld apart overlap", (long long)ld);
    if (rows > kMaxElems / ld) return fail(GEFEN_EINVAL, "more than 2^40 elements");
    return GEFEN_OK;
}

int check_top(int32_t top, int64_t vocab)
{
    if (top < 0 || top > kScoreMaxTop || top > vocab)
        return fail(GEFEN_EINVAL, "top must be in [0, %lld]",
                    (long long)std::min(kScoreMaxTop, vocab));
    return GEFEN_OK;
}

int check_head(int64_t tokens, int64_t width, int64_t vocab)
{
    int rc;
    if ((rc = check_tokens(tokens, 8)) || (rc = check_table(tokens, vocab, width))) return rc;
    if (tokens > 0 && vocab > kMaxElems / tokens)
        return fail(GEFEN_EINVAL, "more than 2^40 elements");
    return GEFEN_OK;
}

int scores(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t vocab,
           const void* tokens, int32_t token_bytes, int32_t top, float* logprob, float* entropy,
           float* lse, float* rest, float* top_logprobs, int64_t* top_tokens, void* workspace,
           int64_t workspace_bytes, void* stream)
{
    int rc;
    if ((rc = check_dtype(dtype)) || (rc = check_scores(rows, vocab, ld)) ||
        (rc = check_tokens(0, token_bytes)) || (rc = check_top(top, vocab)))
        return rc;
    if (!rows) return GEFEN_OK;
    if (!logits || !tokens || !logprob || !entropy || !lse || (top && (!top_logprobs || !top_tokens)))
        return fail(GEFEN_EINVAL, "NULL argument");
    ScoreArgs a{};
    a.plan = score_plan(rows, vocab, dtype == GEFEN_BF16);
    const ScoreSpace s = score_space(a.plan, rows, top);
    if ((rc = check_space(workspace, workspace_bytes, s.bytes))) return rc;
    a.z = logits;
    a.ld = ld;
    a.tokens = Tokens{tokens, token_bytes == 8};
    a.rows = rows;
    a.vocab = vocab;
    a.top = top;
    a.logprob = logprob;
    a.entropy = entropy;
    a.lse = lse;
    a.rest = rest;
    a.top_logprob = top_logprobs;
    a.top_token = top_tokens;
    if (s.bytes) {
        a.keys = at<uint64_t>(workspace, s.keys);
        a.stats = at<float>(workspace, s.stats);
    }
    GEFEN_HIP(launch_scores(a, dtype == GEFEN_BF16, as_stream(stream)));
    return GEFEN_OK;
}

int scores_backward(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t vocab,
                    const void* tokens, int32_t token_bytes, const float* lse, const float* rest,
                    const float* entropy, const float* dlogprob, const float* dentropy,
                    void* dlogits, int64_t ldd, void* stream)
{
    int rc;
    if ((rc = check_dtype(dtype)) || (rc = check_scores(rows, vocab, ld)) ||
        (rc = check_scores(rows, vocab, ldd)) || (rc = check_tokens(0, token_bytes)))
        return rc;
    if (!rows) return GEFEN_OK;
    if (!logits || !tokens || !lse || !entropy || !dlogprob || !dlogits)
        return fail(GEFEN_EINVAL, "NULL argument");
    if (logits == dlogits && ld != ldd)
        return fail(GEFEN_EINVAL, "dlogits in the place of logits has its rows as far apart");
    ScoreGradArgs a{};
    a.z = logits;
    a.ld = ld;
    a.tokens = Tokens{tokens, token_bytes == 8};
    a.rows = rows;
    a.vocab = vocab;
    a.lse = lse;
    a.rest = rest;
    a.entropy = entropy;
    a.dlogprob = dlogprob;
    a.dentropy = dentropy;
    a.dz = dlogits;
    a.ldd = ldd;
    GEFEN_HIP(launch_score_grad(a, dtype == GEFEN_BF16, as_stream(stream)));
    return GEFEN_OK;
}

}  // namespace

extern "C" {

int gefen_embedding(const void* tokens, int32_t token_bytes, int64_t n, const void* table,
                    int32_t table_dtype, int64_t vocab, int64_t width, double scale, void* y,
                    int32_t dtype, void* stream)
{
    int rc;
    if ((rc = check_dtype(table_dtype)) || (rc = check_dtype(dtype)) ||
        (rc = check_tokens(n, token_bytes)) || (rc = check_table(n, vocab, width)) ||
        (rc = check_scale(scale)))
        return rc;
    if (!n) return GEFEN_OK;
    if (!tokens || !table || !y) return fail(GEFEN_EINVAL, "NULL argument");
    EmbedArgs a{};
    a.tokens = Tokens{tokens, token_bytes == 8};
    a.table = table;
    a.n = n;
    a.vocab = vocab;
    a.width = width;
    a.scale = static_cast<float>(scale);
    a.y = y;
    GEFEN_HIP(launch_embedding(a, table_dtype == GEFEN_BF16, dtype == GEFEN_BF16,
                               as_stream(stream)));
    return GEFEN_OK;
}

int gefen_embedding_backward_workspace(int64_t n, int64_t vocab, int64_t width, int64_t* bytes)
{
    int rc;
    if (!bytes) return fail(GEFEN_EINVAL, "bytes is NULL");
    if ((rc = check_tokens(n, 8)) || (rc = check_table(n, vocab, width))) return rc;
    *bytes = n ? embed_space(n, width).bytes : 0;
    return GEFEN_OK;
}

int gefen_embedding_backward(const void* dy, int32_t dtype, const void* tokens,
                             int32_t token_bytes, int64_t n, int64_t vocab, int64_t width,
                             double scale, void* dtable, int32_t table_dtype, void* workspace,
                             int64_t workspace_bytes, void* stream)
{
    int rc;
    if ((rc = check_dtype(dtype)) || (rc = check_dtype(table_dtype)) ||
        (rc = check_tokens(n, token_bytes)) || (rc = check_table(n, vocab, width)) ||
        (rc = check_scale(scale)))
        return rc;
    if (!dtable || (n && (!dy || !tokens))) return fail(GEFEN_EINVAL, "NULL argument");
    EmbedGradArgs a{};
    if (n) {
        const EmbedSpace s = embed_space(n, width);
        if ((rc = check_space(workspace, workspace_bytes, s.bytes))) return rc;
        for (int i = 0; i < 2; ++i) {
            a.keys[i] = at<uint32_t>(workspace, s.keys[i]);
            a.rows[i] = at<uint32_t>(workspace, s.rows[i]);
        }
        a.counts = at<uint32_t>(workspace, s.counts);
        a.partial = at<float>(workspace, s.partial);
    }
    a.tokens = Tokens{tokens, token_bytes == 8};
    a.dy = dy;
    a.n = n;
    a.vocab = vocab;
    a.width = width;
    a.scale = static_cast<float>(scale);
    a.dtable = dtable;
    GEFEN_HIP(launch_embedding_grad(a, dtype == GEFEN_BF16, table_dtype == GEFEN_BF16,
                                    as_stream(stream)));
    return GEFEN_OK;
}

int gefen_dropout(const void* x, const void* residual, int32_t dtype, int64_t n, double p,
                  uint64_t seed, uint64_t offset, const int64_t* state, void* y, void* stream)
{
    int rc;
    if ((rc = check_dtype(dtype))) return rc;
    if (n < 0 || n > kMaxElems) return fail(GEFEN_EINVAL, "n must be in [0, 2^40]");
    if (!(p >= 0.0 && p <= 1.0)) return fail(GEFEN_EINVAL, "p must be in [0, 1]");
    if (!n) return GEFEN_OK;
    if (!x || !y) return fail(GEFEN_EINVAL, "NULL argument");
    DropoutArgs a{};
    a.x = x;
    a.residual = residual;
    a.y = y;
    a.n = n;
    a.least = static_cast<uint32_t>(std::nearbyint(65536.0 * p));
    a.scale = a.least < 65536 ? static_cast<float>(65536.0 / (65536.0 - a.least)) : 0.0f;
    a.seed = seed;
    a.offset = offset;
    a.state = state;
    GEFEN_HIP(launch_dropout(a, dtype == GEFEN_BF16, as_stream(stream)));
    return GEFEN_OK;
}

int gefen_token_logprobs_workspace(int32_t dtype, int64_t rows, int64_t vocab, int32_t top,
                                   int64_t* bytes)
{
    int rc;
    if (!bytes) return fail(GEFEN_EINVAL, "bytes is NULL");
    if ((rc = check_dtype(dtype)) || (rc = check_scores(rows, vocab, vocab)) ||
        (rc = check_top(top, vocab)))
        return rc;
    *bytes = score_space(score_plan(rows, vocab, dtype == GEFEN_BF16), rows, top).bytes;
    return GEFEN_OK;
}

int gefen_token_logprobs(const void* logits, int64_t ld, int32_t dtype, int64_t rows,
                         int64_t vocab, const void* tokens, int32_t token_bytes, int32_t top,
                         float* logprob, float* entropy, float* lse, float* top_logprobs,
                         int64_t* top_tokens, void* workspace, int64_t workspace_bytes,
                         void* stream)
{
    return scores(logits, ld, dtype, rows, vocab, tokens, token_bytes, top, logprob, entropy, lse,
                  nullptr, top_logprobs, top_tokens, workspace, workspace_bytes, stream);
}

int gefen_token_logprobs_split(const void* logits, int64_t ld, int32_t dtype, int64_t rows,
                               int64_t vocab, const void* tokens, int32_t token_bytes, int32_t top,
                               float* logprob, float* entropy, float* lse, float* lse_rest,
                               float* top_logprobs, int64_t* top_tokens, void* workspace,
                               int64_t workspace_bytes, void* stream)
{
    if (rows > 0 && !lse_rest) return fail(GEFEN_EINVAL, "NULL argument");
    return scores(logits, ld, dtype, rows, vocab, tokens, token_bytes, top, logprob, entropy, lse,
                  lse_rest, top_logprobs, top_tokens, workspace, workspace_bytes, stream);
}

int gefen_token_logprobs_backward(const void* logits, int64_t ld, int32_t dtype, int64_t rows,
                                  int64_t vocab, const void* tokens, int32_t token_bytes,
                                  const float* lse, const float* entropy, const float* dlogprob,
                                  const float* dentropy, void* dlogits, int64_t ldd, void* stream)
{
    return scores_backward(logits, ld, dtype, rows, vocab, tokens, token_bytes, lse, nullptr,
                           entropy, dlogprob, dentropy, dlogits, ldd, stream);
}

int gefen_token_logprobs_backward_split(const void* logits, int64_t ld, int32_t dtype,
                                        int64_t rows, int64_t vocab, const void* tokens,
                                        int32_t token_bytes, const float* lse,
                                        const float* lse_rest, const float* entropy,
                                        const float* dlogprob, const float* dentropy,
                                        void* dlogits, int64_t ldd, void* stream)
{
    if (rows > 0 && !lse_rest) return fail(GEFEN_EINVAL, "NULL argument");
    return scores_backward(logits, ld, dtype, rows, vocab, tokens, token_bytes, lse, lse_rest,
                           entropy, dlogprob, dentropy, dlogits, ldd, stream);
}

int gefen_head_logprobs_workspace(int64_t tokens, int64_t width, int64_t vocab, int32_t flags,
                                  int64_t* bytes)
{
    int rc;
    if (!bytes) return fail(GEFEN_EINVAL, "bytes is NULL");
    if (flags & ~(GEFEN_FFN_BACKWARD | GEFEN_FFN_UNALIGNED))
        return fail(GEFEN_EINVAL, "unknown flags");
    if ((rc = check_head(tokens, width, vocab))) return rc;
    *bytes = tokens ? head_space(tokens, width, vocab, flags & GEFEN_FFN_BACKWARD,
                                 flags & GEFEN_FFN_UNALIGNED || width % 8).bytes
                    : 0;
    return GEFEN_OK;
}

int gefen_head_logprobs(const uint16_t* x, const uint16_t* weight, const void* tokens,
                        int32_t token_bytes, int64_t n, int64_t width, int64_t vocab,
                        float* logprob, float* entropy, float* lse, void* workspace,
                        int64_t workspace_bytes, void* stream_)
{
    int rc;
    const int64_t T = n, K = width, V = vocab;
    if ((rc = check_head(T, K, V)) || (rc = check_tokens(T, token_bytes))) return rc;
    if (!T) return GEFEN_OK;
    if (!x || !weight || !tokens || !logprob || !entropy || !lse)
        return fail(GEFEN_EINVAL, "NULL argument");
    hipStream_t stream = as_stream(stream_);
    const bool copy = K % 8 || !aligned16(x) || !aligned16(weight);
    const HeadSpace s = head_space(T, K, V, false, copy);
    if ((rc = check_space(workspace, workspace_bytes, s.bytes))) return rc;
    HeadRows rows{};
    rows.tokens = tokens;
    rows.wide = token_bytes == 8;
    rows.vocab = V;
    rows.stats = at<float>(workspace, s.stats);
    rows.taken = at<float>(workspace, s.taken);
    HeadJoinArgs j{};
    j.stats = rows.stats;
    j.by_rows = head_few(T, K, V, copy);
    j.taken = rows.taken;
    j.tokens = Tokens{tokens, token_bytes == 8};
    j.rows = T;
    j.vocab = V;
    j.slots = s.slots;
    j.logprob = logprob;
    j.entropy = entropy;
    j.lse = lse;
    if (head_few(T, K, V, copy)) {
        FfnTokens t{};
        t.x = x;
        t.ldx = K;
        t.w[0] = weight;
        t.tokens = T;
        t.N = V;
        t.K = K;
        t.head = rows;
        GEFEN_HIP(launch_head_tokens(t, head_groups(K, V), stream));
        GEFEN_HIP(launch_head_join(j, stream));
        return GEFEN_OK;
    }
    FfnPads pads{};
    FfnGemm z = product(kHeadStats, s.score, T, V, K, workspace, -1);
    z.a[0] = operand(x, T, K, copy, workspace, s.x, pads);
    z.b[0] = operand(weight, V, K, copy, workspace, s.w, pads);
    z.lda = z.ldb = ffn_up8(K);
    z.head = rows;
    if ((rc = check_launch(z))) return rc;
    GEFEN_HIP(launch_ffn_pads(pads, stream));
    GEFEN_HIP(launch_ffn_parts(z, stream));
    GEFEN_HIP(launch_head_join(j, stream));
    return GEFEN_OK;
}

int gefen_head_logprobs_backward(const uint16_t* x, const uint16_t* weight, const void* tokens,
                                 int32_t token_bytes, int64_t n, int64_t width, int64_t vocab,
                                 const float* lse, const float* entropy, const float* dlogprob,
                                 const float* dentropy, uint16_t* dx, uint16_t* dweight,
                                 void* workspace, int64_t workspace_bytes, void* stream_)
{
    int rc;
    const int64_t T = n, K = width, V = vocab;
    if ((rc = check_head(T, K, V)) || (rc = check_tokens(T, token_bytes))) return rc;
    hipStream_t stream = as_stream(stream_);
    if (!T) {
        if (dweight) GEFEN_HIP(launch_zero_bf16(dweight, V * K, stream));
        return GEFEN_OK;
    }
    if (!x || !weight || !tokens || !lse || !entropy || !dlogprob || (!dx && !dweight))
        return fail(GEFEN_EINVAL, "NULL argument");
    const bool copy = K % 8 || !aligned16(x) || !aligned16(weight);
    const HeadSpace s = head_space(T, K, V, true, copy);
    if ((rc = check_space(workspace, workspace_bytes, s.bytes))) return rc;
    const int64_t K8 = ffn_up8(K);
    FfnPads pads{};
    const uint16_t* xp = operand(x, T, K, copy, workspace, s.x, pads);
    const uint16_t* wp = operand(weight, V, K, copy, workspace, s.w, pads);

    // Over the vocabulary from entry `first` on: the scores again and their gradients, and the two
    // products that read them. dx is summed over the ranges in float32.
    for (int pass = 0; pass < 2; ++pass) {     // all launches are checked before the first one
        if (pass == 1) GEFEN_HIP(launch_ffn_pads(pads, stream));
        for (int64_t first = 0; first < V; first += s.columns) {
            const int64_t C = std::min(s.columns, V - first);
            FfnGemm z = product(kHeadGrad, s.score, T, C, K, workspace, -1);
            z.a[0] = xp;
            z.b[0] = wp + first * K8;
            z.lda = z.ldb = K8;
            z.o[0] = at<uint16_t>(workspace, s.dz);
            z.o[1] = s.exact ? z.o[0] + T * s.ldz : nullptr;
            z.ldo = s.ldz;
            z.head.tokens = tokens;
            z.head.wide = token_bytes == 8;
            z.head.first = first;
            z.head.vocab = V;
            z.head.lse = lse;
            z.head.entropy = entropy;
            z.head.dlogprob = dlogprob;
            z.head.dentropy = dentropy;

            FfnGemm gx = product(kFfnPlain, s.dx, s.exact ? 2 * T : T, K, C, workspace,
                                 s.partial);                                    // dz W
            gx.stages = static_cast<int32_t>(ffn_ceil(C, kFfnDepth));
            gx.b_rows_k = true;
            gx.a[0] = z.o[0];
            gx.lda = s.ldz;
            gx.b[0] = z.b[0];
            gx.ldb = K8;
            gx.o[0] = dx;
            gx.ldo = K;
            if (s.planes_x) gx.partial = at<float>(workspace, s.partial);
            gx.add = first > 0;
            FfnGemm sum = gx;                     // both halves of dz are rows of gx
            sum.M = T;
            sum.splits = static_cast<int32_t>(s.planes_x);

            FfnGemm gw = product(kFfnPlain, s.dw, C, K, T, workspace, s.partial + s.partial_w);
            gw.a[0] = z.o[0];                                                   // dz^T x
            gw.a[1] = z.o[1];
            gw.lda = s.ldz;
            gw.b[0] = gw.b[1] = xp;
            gw.segments = s.exact ? 2 : 1;
            gw.ldb = K8;
            gw.o[0] = dweight ? dweight + first * K : nullptr;
            gw.ldo = K;
            if (pass == 0) {
                if ((rc = check_launch(z)) || (rc = check_launch(gx)) || (rc = check_launch(sum)) || (rc = check_launch(gw)))
                    return rc;
                continue;
            }
            GEFEN_HIP(launch_ffn_parts(z, stream));
            if (dx) GEFEN_HIP(launch_ffn_parts(gx, stream));
            if (dx && first + C == V) GEFEN_HIP(launch_ffn_join(sum, stream));
            if (dweight) GEFEN_HIP(launch_ffn_weight_grad(gw, stream));
        }
    }
    return GEFEN_OK;
}

}  // extern "C"
