// C ABI of the feed-forward operators: argument checks, workspace layout and launches.
#include "gefen.h"
#include "ffn_internal.h"
#include "ffn_plan.h"
#include "gefen_internal.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>

using namespace gefen;

namespace {

int fail(int code, const char* fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_last_error(buf);
    return code;
}

#define GEFEN_HIP(call)                                                                  \
    do {                                                                                 \
        hipError_t e_ = (call);                                                          \
        if (e_ != hipSuccess)                                                            \
            return fail(GEFEN_EHIP, "%s failed: %s", #call, hipGetErrorString(e_));      \
    } while (0)

hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

constexpr int64_t kMaxElems = int64_t(1) << 40;

int check_rows(int64_t rows, int64_t cols, int64_t max_cols)
{
    if (rows < 0) return fail(GEFEN_EINVAL, "rows must not be negative");
    if (cols < 1 || cols > max_cols)
        return fail(GEFEN_EINVAL, "cols must be in [1, %lld]", (long long)max_cols);
    if (rows > kMaxElems / cols) return fail(GEFEN_EINVAL, "more than 2^40 elements");
    return GEFEN_OK;
}

int check_dtype(int32_t dtype)
{
    if (dtype != GEFEN_F32 && dtype != GEFEN_BF16)
        return fail(GEFEN_EDTYPE, "dtype must be GEFEN_F32 or GEFEN_BF16");
    return GEFEN_OK;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename P>
P* at(void* ws, int64_t off)
{
    return reinterpret_cast<P*>(static_cast<char*>(ws) + off);
}

int check_ffn(int64_t T, int64_t K, int64_t F)
{
    if (T < 0 || T > kFfnMaxTokens)
        return fail(GEFEN_EINVAL, "tokens must be in [0, %lld]", (long long)kFfnMaxTokens);
    if (K < 1 || K > kFfnMaxWidth || F < 1 || F > kFfnMaxWidth)
        return fail(GEFEN_EINVAL, "width and inner must be in [1, %lld]", (long long)kFfnMaxWidth);
    if (T > 0 && std::max(K, F) > kMaxElems / T)
        return fail(GEFEN_EINVAL, "more than 2^40 elements");
    return GEFEN_OK;
}

int check_space(const void* ws, int64_t have, int64_t need)
{
    if (need > 0 && (!ws || have < need))
        return fail(GEFEN_EINVAL, "workspace of %lld bytes, %lld needed", (long long)have,
                    (long long)need);
    if (!aligned16(ws)) return fail(GEFEN_EINVAL, "workspace must be 16-byte aligned");
    return GEFEN_OK;
}

// A product over the plan's tile.
FfnGemm product(int32_t kind, const FfnTile& t, int64_t M, int64_t N, int64_t K, void* ws,
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
int check_launch(const FfnGemm& one, const FfnGemm* two = nullptr)
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
const uint16_t* operand(const void* p, int64_t rows, int64_t cols, bool copy, void* ws, int64_t off,
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

}  // namespace

extern "C" {

int gefen_checkpoint_encode(const void* x, int32_t dtype, int64_t rows, int64_t cols,
                            int8_t* codes, uint8_t* exponents, void* stream)
{
    int rc;
    if ((rc = check_dtype(dtype)) || (rc = check_rows(rows, cols, kMaxElems))) return rc;
    if (!rows) return GEFEN_OK;
    if (!x || !codes || !exponents) return fail(GEFEN_EINVAL, "NULL argument");
    GEFEN_HIP(launch_act8_encode(x, dtype == GEFEN_BF16, rows, cols, codes, exponents,
                                 as_stream(stream)));
    return GEFEN_OK;
}

int gefen_checkpoint_decode(const int8_t* codes, const uint8_t* exponents, const float* gain,
                            int64_t rows, int64_t cols, void* out, int32_t dtype, void* stream)
{
    int rc;
    if ((rc = check_dtype(dtype)) || (rc = check_rows(rows, cols, kMaxElems))) return rc;
    if (!rows) return GEFEN_OK;
    if (!codes || !exponents || !out) return fail(GEFEN_EINVAL, "NULL argument");
    GEFEN_HIP(launch_act8_decode(codes, exponents, gain, rows, cols, out, dtype == GEFEN_BF16,
                                 cols, as_stream(stream)));
    return GEFEN_OK;
}

int gefen_rms_norm(const void* x, const void* residual, int32_t dtype, const float* weight,
                   int64_t rows, int64_t cols, double eps, void* y, void* h, float* rstd,
                   int8_t* codes, uint8_t* exponents, void* stream)
{
    int rc;
    if ((rc = check_dtype(dtype)) || (rc = check_rows(rows, cols, kNormMaxCols))) return rc;
    if (!(eps >= 0.0) || !std::isfinite(eps))
        return fail(GEFEN_EINVAL, "eps must be finite and not negative");
    if (!codes != !exponents) return fail(GEFEN_EINVAL, "codes and exponents go together");
    if (!rows) return GEFEN_OK;
    if (!x || !weight || !y || !rstd) return fail(GEFEN_EINVAL, "NULL argument");
    NormArgs a{};
    a.x = x;
    a.r = residual;
    a.weight = weight;
    a.rows = rows;
    a.cols = cols;
    a.eps = eps;
    a.y = y;
    a.h = h;
    a.rstd = rstd;
    a.codes = codes;
    a.exps = exponents;
    GEFEN_HIP(launch_rms_norm(a, dtype == GEFEN_BF16, as_stream(stream)));
    return GEFEN_OK;
}

int gefen_rms_norm_backward_workspace(int64_t rows, int64_t cols, int64_t* bytes)
{
    int rc;
    if (!bytes) return fail(GEFEN_EINVAL, "bytes is NULL");
    if ((rc = check_rows(rows, cols, kNormMaxCols))) return rc;
    *bytes = 4 * norm_grad_parts(rows, cols) * cols;
    return GEFEN_OK;
}

int gefen_rms_norm_backward(const void* dy, const void* dh, int32_t dtype, const void* h,
                            const int8_t* codes, const uint8_t* exponents, const float* rstd,
                            const float* weight, int64_t rows, int64_t cols, void* dx,
                            float* dweight, void* workspace, int64_t workspace_bytes,
                            void* stream)
{
    int rc;
    if ((rc = check_dtype(dtype)) || (rc = check_rows(rows, cols, kNormMaxCols))) return rc;
    if (!dweight) return fail(GEFEN_EINVAL, "NULL argument");
    if (rows) {
        if (!dy || !rstd || !weight || !dx) return fail(GEFEN_EINVAL, "NULL argument");
        if (!h == !codes || !codes != !exponents)
            return fail(GEFEN_EINVAL, "either h or codes with exponents");
        if ((rc = check_space(workspace, workspace_bytes, 4 * norm_grad_parts(rows, cols) * cols)))
            return rc;
    }
    NormGradArgs a{};
    a.dy = dy;
    a.dh = dh;
    a.h = h;
    a.codes = codes;
    a.exps = exponents;
    a.rstd = rstd;
    a.weight = weight;
    a.rows = rows;
    a.cols = cols;
    a.dx = dx;
    a.dw = dweight;
    a.partial = static_cast<float*>(workspace);
    GEFEN_HIP(launch_rms_norm_grad(a, dtype == GEFEN_BF16, as_stream(stream)));
    return GEFEN_OK;
}

int gefen_gated_ffn_workspace(int64_t tokens, int64_t width, int64_t inner, int32_t flags,
                              int64_t* bytes)
{
    int rc;
    if (!bytes) return fail(GEFEN_EINVAL, "bytes is NULL");
    if (flags & ~(GEFEN_FFN_BACKWARD | GEFEN_FFN_UNALIGNED))
        return fail(GEFEN_EINVAL, "unknown flags");
    if ((rc = check_ffn(tokens, width, inner))) return rc;
    const bool copy = flags & GEFEN_FFN_UNALIGNED;
    *bytes = tokens ? ffn_space(tokens, width, inner, flags & GEFEN_FFN_BACKWARD,
                                copy || width % 8, copy || inner % 8).bytes
                    : 0;
    return GEFEN_OK;
}

int gefen_gated_ffn(const uint16_t* x, const uint16_t* w_gate, const uint16_t* w_up,
                    const uint16_t* w_down, int64_t tokens, int64_t width, int64_t inner,
                    int32_t activation, uint16_t* y, int8_t* gate_codes, uint8_t* gate_exponents,
                    int8_t* up_codes, uint8_t* up_exponents, void* workspace,
                    int64_t workspace_bytes, void* stream_)
{
    int rc;
    const int64_t T = tokens, K = width, F = inner;
    if ((rc = check_ffn(T, K, F))) return rc;
    if (activation != GEFEN_SILU && activation != GEFEN_GELU)
        return fail(GEFEN_EINVAL, "activation must be GEFEN_SILU or GEFEN_GELU");
    const int given = !!gate_codes + !!gate_exponents + !!up_codes + !!up_exponents;
    if (given != 0 && given != 4)
        return fail(GEFEN_EINVAL, "the checkpoints' four arrays go together");
    if (!T) return GEFEN_OK;
    if (!x || !w_gate || !w_up || !w_down || !y) return fail(GEFEN_EINVAL, "NULL argument");
    hipStream_t stream = as_stream(stream_);
    if (T <= kFfnFewTokens && !gate_codes) {
        if ((rc = check_space(workspace, workspace_bytes, 2 * T * F))) return rc;
        FfnTokens t{};
        t.x = x;
        t.ldx = K;
        t.w[0] = w_gate;
        t.w[1] = w_up;
        t.tokens = T;
        t.N = F;
        t.K = K;
        t.act = activation;
        t.o = static_cast<uint16_t*>(workspace);
        t.ldo = F;
        GEFEN_HIP(launch_ffn_tokens(t, stream));
        t.x = t.o;
        t.ldx = F;
        t.w[0] = w_down;
        t.w[1] = nullptr;
        t.N = K;
        t.K = F;
        t.o = y;
        t.ldo = K;
        GEFEN_HIP(launch_ffn_tokens(t, stream));
        return GEFEN_OK;
    }
    const bool copy_k = K % 8 || !aligned16(x) || !aligned16(w_gate) || !aligned16(w_up);
    const bool copy_f = F % 8 || !aligned16(w_down);
    const FfnSpace s = ffn_space(T, K, F, false, copy_k, copy_f);
    if ((rc = check_space(workspace, workspace_bytes, s.bytes))) return rc;
    FfnPads pads{};
    const uint16_t* xp = operand(x, T, K, copy_k, workspace, s.x, pads);
    const uint16_t* gp = operand(w_gate, F, K, copy_k, workspace, s.w_gate, pads);
    const uint16_t* up = operand(w_up, F, K, copy_k, workspace, s.w_up, pads);
    const uint16_t* dp = operand(w_down, K, F, copy_f, workspace, s.w_down, pads);

    FfnGemm inner_product = product(kFfnGateUp, s.gate_up, T, F, K, workspace, s.partial);
    inner_product.act = activation;
    inner_product.a[0] = xp;
    inner_product.b[0] = gp;
    inner_product.b[1] = up;
    inner_product.lda = inner_product.ldb = ffn_up8(K);
    inner_product.o[0] = at<uint16_t>(workspace, s.a);
    inner_product.ldo = ffn_up8(F);
    inner_product.gcodes = gate_codes;
    inner_product.ucodes = up_codes;
    inner_product.gexps = gate_exponents;
    inner_product.uexps = up_exponents;
    inner_product.groups = act8_groups(F);

    FfnGemm down = product(kFfnPlain, s.down, T, K, F, workspace, s.partial);
    down.a[0] = at<uint16_t>(workspace, s.a);
    down.b[0] = dp;
    down.lda = down.ldb = ffn_up8(F);
    down.o[0] = y;
    down.ldo = K;

    if ((rc = check_launch(inner_product)) || (rc = check_launch(down))) return rc;
    GEFEN_HIP(launch_ffn_pads(pads, stream));
    GEFEN_HIP(launch_ffn_gemm(inner_product, stream));
    GEFEN_HIP(launch_ffn_gemm(down, stream));
    return GEFEN_OK;
}

int gefen_gated_ffn_backward(const uint16_t* dy, const uint16_t* x, const int8_t* x_codes,
                             const uint8_t* x_exponents, const float* gain,
                             const int8_t* gate_codes, const uint8_t* gate_exponents,
                             const int8_t* up_codes, const uint8_t* up_exponents,
                             const uint16_t* w_gate, const uint16_t* w_up, const uint16_t* w_down,
                             int64_t tokens, int64_t width, int64_t inner, int32_t activation,
                             uint16_t* dx, uint16_t* dw_gate, uint16_t* dw_up, uint16_t* dw_down,
                             void* workspace, int64_t workspace_bytes, void* stream_)
{
    int rc;
    const int64_t T = tokens, K = width, F = inner;
    if ((rc = check_ffn(T, K, F))) return rc;
    if (activation != GEFEN_SILU && activation != GEFEN_GELU)
        return fail(GEFEN_EINVAL, "activation must be GEFEN_SILU or GEFEN_GELU");
    if (!dw_gate || !dw_up || !dw_down) return fail(GEFEN_EINVAL, "NULL argument");
    hipStream_t stream = as_stream(stream_);
    if (!T) {
        GEFEN_HIP(launch_zero_bf16(dw_gate, F * K, stream));
        GEFEN_HIP(launch_zero_bf16(dw_up, F * K, stream));
        GEFEN_HIP(launch_zero_bf16(dw_down, K * F, stream));
        return GEFEN_OK;
    }
    if (!dy || !w_gate || !w_up || !w_down || !dx || !gate_codes || !gate_exponents || !up_codes ||
        !up_exponents)
        return fail(GEFEN_EINVAL, "NULL argument");
    if (!x == !x_codes || !x_codes != !x_exponents)
        return fail(GEFEN_EINVAL, "either x or x_codes with x_exponents");
    if (gain && x) return fail(GEFEN_EINVAL, "gain goes with x_codes");
    const bool copy_k = K % 8 || !aligned16(dy) || !aligned16(w_gate) || !aligned16(w_up) ||
                        (x && !aligned16(x));
    const bool copy_f = F % 8 || !aligned16(w_down);
    const FfnSpace s = ffn_space(T, K, F, true, copy_k, copy_f);
    if ((rc = check_space(workspace, workspace_bytes, s.bytes))) return rc;
    const int64_t K8 = ffn_up8(K), F8 = ffn_up8(F);
    FfnPads pads{};
    const uint16_t* dyp = operand(dy, T, K, copy_k, workspace, s.dy, pads);
    const uint16_t* gp = operand(w_gate, F, K, copy_k, workspace, s.w_gate, pads);
    const uint16_t* up = operand(w_up, F, K, copy_k, workspace, s.w_up, pads);
    const uint16_t* dp = operand(w_down, K, F, copy_f, workspace, s.w_down, pads);
    const uint16_t* xp = x ? operand(x, T, K, copy_k, workspace, s.x, pads)
                           : at<uint16_t>(workspace, s.x);
    uint16_t* a = at<uint16_t>(workspace, s.a);
    uint16_t* dg = at<uint16_t>(workspace, s.dg);
    uint16_t* du = at<uint16_t>(workspace, s.du);

    FfnGemm grad_inner = product(kFfnGateGrad, s.grad_inner, T, F, K, workspace, s.partial);
    grad_inner.act = activation;
    grad_inner.a[0] = dyp;
    grad_inner.lda = K8;
    grad_inner.b[0] = dp;
    grad_inner.b_rows_k = true;
    grad_inner.ldb = F8;
    grad_inner.o[0] = dg;
    grad_inner.o[1] = du;
    grad_inner.o2 = a;
    grad_inner.ldo = F8;
    grad_inner.gcodes = const_cast<int8_t*>(gate_codes);
    grad_inner.ucodes = const_cast<int8_t*>(up_codes);
    grad_inner.gexps = const_cast<uint8_t*>(gate_exponents);
    grad_inner.uexps = const_cast<uint8_t*>(up_exponents);
    grad_inner.groups = act8_groups(F);

    FfnGemm dwd = product(kFfnPlain, s.dw, K, F, T, workspace, s.partial);      // dy^T A
    dwd.a[0] = dyp;
    dwd.lda = K8;
    dwd.b[0] = a;
    dwd.ldb = F8;
    dwd.o[0] = dw_down;
    dwd.ldo = F;
    FfnGemm dwi = product(kFfnPlain, s.dw, F, K, T, workspace,                  // dG^T x, dU^T x
                          s.partial + ffn_partial_bytes(s.dw, K, F, 1));
    dwi.batch = 2;
    dwi.a[0] = dg;
    dwi.a[1] = du;
    dwi.lda = F8;
    dwi.b[0] = xp;
    dwi.ldb = K8;
    dwi.col_scale = gain;
    dwi.o[0] = dw_gate;
    dwi.o[1] = dw_up;
    dwi.ldo = K;

    FfnGemm dxp = product(kFfnPlain, s.dx, T, K, F, workspace, s.partial);      // dG Wg + dU Wu
    dxp.segments = 2;
    dxp.b_rows_k = true;
    dxp.a[0] = dg;
    dxp.a[1] = du;
    dxp.lda = F8;
    dxp.b[0] = gp;
    dxp.b[1] = up;
    dxp.ldb = K8;
    dxp.o[0] = dx;
    dxp.ldo = K;

    if ((rc = check_launch(grad_inner)) || (rc = check_launch(dwd, &dwi)) ||
        (rc = check_launch(dxp)))
        return rc;
    GEFEN_HIP(launch_ffn_pads(pads, stream));
    // The input's values are exact in bfloat16; its gain goes into the weight gradients' columns.
    if (!x)
        GEFEN_HIP(launch_act8_decode(x_codes, x_exponents, nullptr, T, K, at<void>(workspace, s.x),
                                     true, K8, stream));
    GEFEN_HIP(launch_ffn_gemm(grad_inner, stream));
    GEFEN_HIP(launch_ffn_weight_grads(dwd, dwi, stream));
    GEFEN_HIP(launch_ffn_gemm(dxp, stream));
    return GEFEN_OK;
}

}  // extern "C"
